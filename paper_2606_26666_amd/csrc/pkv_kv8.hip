// HIP kernels of the 8-bit paged KV cache on CDNA4 (gfx950): the quantising write, the read-back,
// and single-token attention over the records (layout: pkv_kv8.h).
#include <atomic>

#include <hip/hip_runtime.h>

#include "pkv_kv8.h"

namespace pkv {
namespace {

constexpr int D = kHeadDim;
constexpr int P = kPageSize;

typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));
typedef unsigned short v2h __attribute__((ext_vector_type(2)));

// Cache-policy operand of a buffer access: non-temporal. A call reads a record once unless rows share pages, which
// it cannot tell beforehand: 64 rows of 4160 tokens 98 us against 110 with the default policy, 32 of 16512
// 182 against 201; with all but the last 64 or 128 tokens shared 78 against 76 and 145 against 135.
constexpr int kNt = 2;
constexpr int kOutOfRange = (int)0x80000000u;  // an offset past any buffer: reads as zero, without memory
constexpr int kSc1 = 16;  // cache-policy operand of a buffer access: coherent across the XCDs' L2 caches
constexpr float kLowest = -3.0e38f;  // a finite start for running maxima: no infinity is subtracted from another

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ unsigned as_u32(float x) { return __builtin_bit_cast(unsigned, x); }
__device__ __forceinline__ float as_f32(unsigned x) { return __builtin_bit_cast(float, x); }

template <int CTRL>
__device__ __forceinline__ int dpp(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true); }
// The value of lane 15 - c of the same 16 lanes.
__device__ __forceinline__ float mirror16(float x) { return as_f32((unsigned)dpp<0x140>((int)as_u32(x))); }

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

// Lanes l, l ^ 16, l ^ 32 and l ^ 48 combined; every one of them receives the result. The copy that a
// swap takes is opaque to the compiler, which has folded a value swapped with itself.
template <typename F>
__device__ __forceinline__ float across_rows(float x, F f) {
  unsigned a = as_u32(x), b = a;
  asm volatile("" : "+v"(b));
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  unsigned c = as_u32(f(as_f32((unsigned)r[0]), as_f32((unsigned)r[1]))), d = c;
  asm volatile("" : "+v"(d));
  const auto t = __builtin_amdgcn_permlane32_swap(c, d, false, false);
  return f(as_f32((unsigned)t[0]), as_f32((unsigned)t[1]));
}

template <typename F>
__device__ __forceinline__ b8v load8(unsigned lo, unsigned hi) {
  const v2u a = F::load4(lo), b = F::load4(hi);
  return __builtin_bit_cast(b8v, v4u{a.x, a.y, b.x, b.y});
}

// The 16 lanes of a row, all 64 lanes, or the 32 of each half combined, in a fixed order.
template <typename F>
__device__ __forceinline__ float across_row(float x, F f) {
  x = f(x, as_f32((unsigned)dpp<0xB1>((int)as_u32(x))));
  x = f(x, as_f32((unsigned)dpp<0x4E>((int)as_u32(x))));
  x = f(x, as_f32((unsigned)dpp<0x141>((int)as_u32(x))));
  return f(x, as_f32((unsigned)dpp<0x140>((int)as_u32(x))));
}
template <typename F>
__device__ __forceinline__ float across_wave(float x, F f) { return across_rows(across_row(x, f), f); }
template <typename F>
__device__ __forceinline__ float half_wave(float x, F f) {
  x = across_row(x, f);
  unsigned a = as_u32(x), b = a;
  asm volatile("" : "+v"(b));
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return f(as_f32((unsigned)r[0]), as_f32((unsigned)r[1]));
}

// ---------------------------------------------------------------------------------
// Formats. `load4` makes bf16 operands of codes (exact: int8 has 8 and e4m3 4 significant bits).
// `code4` rounds quotients t = x * top / m, x and m of 11 bits each. A t that is not on a rounding
// border is 2^-19 of its size or more away from the nearest one, and a border has at most 9 bits. So
// x * (top / m) in fp32, off by less than 2^-23, is first rounded to 21 bits (round21), which puts a
// t on a border back on it and no other there: the code is that of real arithmetic, ties included,
// with one division a vector instead of one a value.
__device__ __forceinline__ float round21(float y) { return as_f32((as_u32(y) + 4u) & ~7u); }

struct Int8 {
  static constexpr float top = 127.0f;
  // 1.5 * 2^23 + y rounds y to an integer (ties to even), which is then the low bits of the sum.
  static __device__ __forceinline__ unsigned code4(float a, float b, float c, float d) {
    const unsigned x = __builtin_amdgcn_perm(as_u32(b + 12582912.0f), as_u32(a + 12582912.0f), 0x0C0C0400u);
    const unsigned y = __builtin_amdgcn_perm(as_u32(d + 12582912.0f), as_u32(c + 12582912.0f), 0x04000C0Cu);
    return x | y;
  }
  static __device__ __forceinline__ float value(unsigned w, int at) { return (float)(signed char)(w >> (8 * at)); }
  // Four codes as bf16: fp32 integers of at most 8 bits, whose upper 16 bits are the bf16s.
  static __device__ __forceinline__ v2u load4(unsigned w) {
    asm volatile("" : "+v"(w));  // one register: the compiler would carry the masked codes in one each
    const float a = (float)(signed char)(w & 255u), b = (float)(signed char)((w >> 8) & 255u);
    const float c = (float)(signed char)((w >> 16) & 255u), d = (float)(signed char)(w >> 24);
    return v2u{__builtin_amdgcn_perm(as_u32(b), as_u32(a), 0x07060302u), __builtin_amdgcn_perm(as_u32(d), as_u32(c), 0x07060302u)};
  }
  // Q.K in integers: K enters the matrix cores as it lies in memory, and a query vector as four
  // balanced base-256 digits of x = q * 2^24, x = 2^24 d3 + 2^16 d2 + 2^8 d1 + d0 with d3 in [-64, 64], the
  // others in [-128, 127] (a digit's borders moved up by the digits below it). Below 64 any fp16 is such an
  // integer of at most 30 bits. With larger values in a head, x = q * 2^k, k the largest with all below 2^30,
  // and what that leaves of smaller values is two digits more, for which `low` says that there are any. So
  // the sums of digits times codes are exact, whatever lies beside a large value; two or three of them
  // are joined in fp32 (d3 and d1 in column h, d2 and d0 in column 15 - h). A channel of 100 in every head: one row
  // of 77 tokens 8.6 us against 8.0, of 32 K 24.7 against 24.0, larger calls the same.
  // A head's columns have to hold the same score to the last bit, since they hold parts of the same weight: they
  // are added before the scales come in, so that no product can be fused into the sum of one column and
  // not into the other's.
  struct Query {
    v4u b[2][2];    // [d3 and d2, d1 and d0][half]
    v4u b_low[2];
    float unit;     // 2^-k * scale
    float up;       // 2^8 in the columns of d3 and d1, 1 in the others
    float up_low;   // of the digits beyond: up * 2^(k - 24)
    bool low;
    // Bytes of four digits: of x[i] + bias, the byte that `at` picks of a pair.
    static __device__ __forceinline__ unsigned four(const unsigned* x, unsigned bias, unsigned at) {
      return __builtin_amdgcn_perm(x[1] + bias, x[0] + bias, at) | __builtin_amdgcn_perm(x[3] + bias, x[2] + bias, at) << 16;
    }
    __device__ __forceinline__ void set(const v4u (&raw)[4], bool, int col, float scale) {
      v4u r[4];
      v2h most = {0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        r[j] = raw[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(v2h, raw[j][e] & 0x7FFF7FFFu));
      }
      // Bytes of a pair with nothing above: d3 that of 2^24 of x + 2^23 + 2^15 + 2^7, and so on.
      const unsigned bias1 = col < 8 ? 0x808080u : 0x8080u, bias0 = col < 8 ? 0x80u : 0u;
      const unsigned at1 = col < 8 ? 0x0C0C0703u : 0x0C0C0602u, at0 = col < 8 ? 0x0C0C0501u : 0x0C0C0400u;
      unsigned top = max((unsigned)most.x, (unsigned)most.y);
      up = col < 8 ? 256.0f : 1.0f;
      float raise = 0x1p24f;
      unit = 0x1p-24f * scale;
      low = false;
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(top >= 0x5400u) != 0, 0)) {  // a value of 64 or more
        top = as_u32(across_rows(as_f32(top), [](float y, float z) { return as_f32(max(as_u32(y), as_u32(z))); }));
        const bool finite = top < 0x7C00u;
        const int k = finite ? min(24, 44 - (int)(top >> 10)) : 24;  // |q| < 2^(exponent bits - 14)
        raise = as_f32((unsigned)(127 + k) << 23);
        unit = finite ? as_f32((unsigned)(127 - k) << 23) * scale : __builtin_nanf("");
        up_low = up * as_f32((unsigned)(103 + k) << 23);
        const float rest = as_f32((unsigned)(151 - k) << 23);
        unsigned any = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          r[j] = finite ? r[j] : v4u{0, 0, 0, 0};
          const h8v y = __builtin_bit_cast(h8v, r[j]);
          unsigned x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float f = (float)y[e] * raise;
            x[e] = (unsigned)(int)((f - __builtin_truncf(f)) * rest);
            any |= x[e];
          }
          b_low[j >> 1][2 * (j & 1)] = four(x, bias0, at0);
          b_low[j >> 1][2 * (j & 1) + 1] = four(x + 4, bias0, at0);
        }
        low = __builtin_amdgcn_ballot_w64(any != 0) != 0;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // (columns without a head hold the first one's)
        const h8v y = __builtin_bit_cast(h8v, r[j]);
        unsigned x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (unsigned)(int)((float)y[e] * raise);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          b[0][j >> 1][2 * (j & 1) + i] = four(x + 4 * i, bias1, at1);
          b[1][j >> 1][2 * (j & 1) + i] = four(x + 4 * i, bias0, at0);
        }
      }
    }
    __device__ __forceinline__ v4f scores(const v4u (&k)[2], v4f ks) const {
      v4i c = {0, 0, 0, 0}, c0 = {0, 0, 0, 0};
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        c = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, k[half]), __builtin_bit_cast(v4i, b[0][half]), c, 0, 0, 0);
        c0 = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, k[half]), __builtin_bit_cast(v4i, b[1][half]), c0, 0, 0, 0);
      }
      v4f x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf((float)c[i], 65536.0f * up, (float)c0[i] * up);
      if (__builtin_expect(low, 0)) {
        v4i d = {0, 0, 0, 0};
#pragma unroll
        for (int half = 0; half < 2; ++half)
          d = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, k[half]), __builtin_bit_cast(v4i, b_low[half]), d, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf((float)d[i], up_low, x[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (x[i] + mirror16(x[i])) * (ks[i] * unit);
      return x;
    }
  };
};
struct E4m3 {
  static constexpr float top = 448.0f;
  static __device__ __forceinline__ unsigned code4(float a, float b, float c, float d) {
    const int x = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, x, true);
  }
  static __device__ __forceinline__ float value(unsigned w, int at) {
    return at == 0 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 0)
                   : at == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 1)
                             : at == 2 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 2) : __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
  }
  static __device__ __forceinline__ v2u load4(unsigned w) {
    return v2u{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))};
  }
  // Q.K in bf16: K exactly, a query value as its bf16 high half in column h and low half in column
  // 15 - h (exact: fp16 has 11 bits); the two columns' sums are added.
  struct Query {
    b8v b[4];
    float unit;
    __device__ __forceinline__ void set(const v4u (&raw)[4], bool there, int col, float scale) {
      unit = scale;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const h8v y = __builtin_bit_cast(h8v, raw[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float f = there ? (float)y[e] : 0.0f;
          const __bf16 hi = (__bf16)f;
          b[j][e] = col < 8 ? hi : (__bf16)(f - (float)hi);
        }
      }
    }
    __device__ __forceinline__ v4f scores(const v4u (&k)[2], v4f ks) const {
      v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(load8<E4m3>(k[j >> 1][2 * (j & 1)], k[j >> 1][2 * (j & 1) + 1]), b[j], x, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (x[i] + mirror16(x[i])) * (ks[i] * unit);
      return x;
    }
  };
};

// ---------------------------------------------------------------------------------
// Append and gather.
//
// Both are bound by their bytes (776 a token and KV head): 532 K token-heads written in 88 us, 4.7
// TB/s (the vector ALU is busy for 60% of it), 459 K read back in 70 us, 5.1 TB/s, which is what a
// large copy moves. A wave takes a window of four packed
// tokens and a range of KV heads, sixteen lanes a token, eight values a lane: 256-byte rows of fp16
// on one side, 128-byte rows of K codes on the other. V codes lie in groups of four tokens: where
// the wave's four are such a group, a transpose between the four lane groups (two swaps) makes whole
// dwords, eight bytes a lane; else single bytes. A window's tokens may start inside a group, so a wave
// takes the groups that begin in its window: a group begins at its row's first token or at a
// position that is a multiple of four. Calls of few tokens per row (kScatter: one token per row, or
// fewer than four on average) take the window's tokens side by side instead, in bytes.

// The last i with offsets[i] <= t (0 if there is none), with the wave's 64 lanes at once. In range
// for any offsets.
__device__ __forceinline__ int row_of(const Kv8MoveArgs& a, int t, int lane) {
  int lo = 0, n = a.B;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int i = lane * step;
    const bool below = i < n && a.offsets[lo + i] <= t;
    const int c = max(__popcll(__builtin_amdgcn_ballot_w64(below)) - 1, 0);
    lo += c * step;
    n = min(step, n - c * step);
  }
  return uniform(lo);
}

// A token's place. `there`: it is to be moved; `zero`: it is to be read back as zeros (both false:
// it is left alone). `begin`, `end`: the row's packed tokens.
struct Place {
  int row, pos, begin, end;
  bool there, zero;
};
// `last`: offsets[B], behind which tokens are left alone.
__device__ __forceinline__ Place place(const Kv8MoveArgs& a, int t, int row, int begin, int end, int last, int len) {
  Place p{row, 0, begin, end, false, false};
  if (a.offsets && (t < begin || t >= last)) return p;
  p.zero = true;
  if (!a.offsets && len == 0) return p;
  // (begin <= t here) the row's tokens end after t and are no more than its length
  if (len < 0 || len > a.max_pages_per_row * P || begin < 0 || end <= t || end - begin > len) {
    atomicOr(a.err, (unsigned)PKV_DEVERR_SEQ_LEN);
    return p;
  }
  p.there = true;
  p.zero = false;
  p.pos = len - (end - t);
  return p;
}
__device__ __forceinline__ Place place(const Kv8MoveArgs& a, int t, int row) {
  if (!a.offsets) return place(a, t, row, t, t + 1, a.B, a.seq_lens[row]);
  return place(a, t, row, a.offsets[row], a.offsets[row + 1], a.offsets[a.B], a.seq_lens[row]);
}

// The page of a position as an offset of records; a bad id takes the token out.
__device__ __forceinline__ size_t page_at(const Kv8MoveArgs& a, int row, int pos, bool& there, bool& zero) {
  const int id = a.block_table[(size_t)row * a.max_pages_per_row + pos / P];
  if (id >= 0 && id < a.num_pages) return (size_t)id * a.Hkv * kKv8Record;
  atomicOr(a.err, (unsigned)PKV_DEVERR_PAGE_ID);
  there = false;
  zero = true;
  return 0;
}

// Sixteen-bit units between the four 16-lane groups: lane group j gives its units 0 .. 3 (two dwords)
// and receives unit j of groups 0 .. 3, as bytes: word i of the result holds byte i of the units.
__device__ __forceinline__ v2u groups_to_words(v2u w) {
  const auto r = __builtin_amdgcn_permlane32_swap(w.x, w.y, false, false);
  const unsigned x = (unsigned)r[0], y = (unsigned)r[1];
  const unsigned p = __builtin_amdgcn_perm(y, x, 0x05040100u), q = __builtin_amdgcn_perm(y, x, 0x07060302u);
  const auto t = __builtin_amdgcn_permlane16_swap(p, q, false, false);
  const unsigned even = (unsigned)t[0], odd = (unsigned)t[1];  // groups 0 and 2, groups 1 and 3
  return v2u{__builtin_amdgcn_perm(odd, even, 0x06020400u), __builtin_amdgcn_perm(odd, even, 0x07030501u)};
}
// The way back.
__device__ __forceinline__ v2u words_to_groups(v2u w) {
  const unsigned even = __builtin_amdgcn_perm(w.y, w.x, 0x06020400u), odd = __builtin_amdgcn_perm(w.y, w.x, 0x07030501u);
  const auto t = __builtin_amdgcn_permlane16_swap(even, odd, false, false);
  const unsigned p = (unsigned)t[0], q = (unsigned)t[1];
  const unsigned x = __builtin_amdgcn_perm(q, p, 0x05040100u), y = __builtin_amdgcn_perm(q, p, 0x07060302u);
  const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
  return v2u{(unsigned)r[0], (unsigned)r[1]};
}

__device__ __forceinline__ unsigned row_max16(unsigned m) {
  m = max(m, (unsigned)dpp<0xB1>((int)m));
  m = max(m, (unsigned)dpp<0x4E>((int)m));
  m = max(m, (unsigned)dpp<0x141>((int)m));
  return max(m, (unsigned)dpp<0x140>((int)m));
}

// Eight values a lane, sixteen lanes a vector, to codes and the vector's scale.
template <typename F>
__device__ __forceinline__ v2u quantise(v4u raw, float& scale) {
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) m = max(m, max(raw[j] & 0x7FFFu, (raw[j] >> 16) & 0x7FFFu));
  m = row_max16(m);
  const bool finite = m < 0x7C00u;
  const float top = (float)__builtin_bit_cast(_Float16, (uint16_t)m);
  const float inv = finite && m > 0 ? F::top / top : 0.0f;
  scale = finite ? top / F::top : as_f32(0x7FC00000u);
  const h8v x = __builtin_bit_cast(h8v, raw);
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = inv > 0.0f ? round21((float)x[j] * inv) : 0.0f;  // (also a vector of -0: codes 0)
  return v2u{F::code4(y[0], y[1], y[2], y[3]), F::code4(y[4], y[5], y[6], y[7])};
}

// One KV head of a window: `there` and `zero` per 16 lanes (see Place), token t, slot s of the record's
// page at rec; `group`: all four lane groups are one group of the record.
struct Window {
  int t, s, grp, c;
  bool there, zero, group;
  size_t rec;
};

struct Append {
  typedef v4u Values[2];
  static __device__ __forceinline__ void fetch(const Kv8MoveArgs& a, const Window& w, int h, Values& x) {
    x[0] = x[1] = v4u{0, 0, 0, 0};
    if (!w.there) return;
    x[0] = *reinterpret_cast<const v4u*>(a.k + (size_t)w.t * a.k_stride + h * D + w.c * 8);
    x[1] = *reinterpret_cast<const v4u*>(a.v + (size_t)w.t * a.v_stride + h * D + w.c * 8);
  }
  template <typename F>
  static __device__ __forceinline__ void finish(const Kv8MoveArgs& a, const Window& w, int h, const Values& x) {
    uint8_t* rec = a.cache + w.rec + (size_t)h * kKv8Record;
    float scale[2];
    const v2u kc = quantise<F>(x[0], scale[0]);
    v2u vc = quantise<F>(x[1], scale[1]);
    uint8_t* v = rec + kKv8CodeBytes + (w.s / 4) * (4 * D);
    if (w.group) {
      vc = groups_to_words(vc);
      *reinterpret_cast<v2u*>(v + (w.c * 8 + 2 * w.grp) * 4) = vc;
    }
    if (!w.there) return;
    *reinterpret_cast<v2u*>(rec + w.s * D + w.c * 8) = kc;
    if (!w.group) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[(w.c * 8 + j) * 4 + w.s % 4] = (uint8_t)(vc[j >> 2] >> (8 * (j & 3)));
    }
    if (w.c < 2) reinterpret_cast<float*>(rec + kKv8ScaleAt)[w.c * P + w.s] = w.c ? scale[1] : scale[0];
  }
};

struct Gather {
  struct Values {
    v2u k, v;
    float ks, vs;
  };
  static __device__ __forceinline__ void fetch(const Kv8MoveArgs& a, const Window& w, int h, Values& x) {
    x = Values{};
    const uint8_t* rec = a.cache + w.rec + (size_t)h * kKv8Record;
    const uint8_t* v = rec + kKv8CodeBytes + (w.s / 4) * (4 * D);
    if (w.there) {
      x.k = *reinterpret_cast<const v2u*>(rec + w.s * D + w.c * 8);
      x.ks = reinterpret_cast<const float*>(rec + kKv8ScaleAt)[w.s];
      x.vs = reinterpret_cast<const float*>(rec + kKv8ScaleAt)[P + w.s];
    }
    if (w.group) {
      x.v = *reinterpret_cast<const v2u*>(v + (w.c * 8 + 2 * w.grp) * 4);
    } else if (w.there) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x.v[j >> 2] |= (unsigned)v[(w.c * 8 + j) * 4 + w.s % 4] << (8 * (j & 3));
    }
  }
  template <typename F>
  static __device__ __forceinline__ void finish(const Kv8MoveArgs& a, const Window& w, int h, const Values& x) {
    const v2u v = w.group ? words_to_groups(x.v) : x.v;
    if (!w.there && !w.zero) return;
    h8v p, q;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = (_Float16)(F::value(x.k[j >> 2], j & 3) * x.ks);
      q[j] = (_Float16)(F::value(v[j >> 2], j & 3) * x.vs);
    }
    // streamed past the caches: 6% faster than kept in them, where the records' lines then stay
    __builtin_nontemporal_store(p, reinterpret_cast<h8v*>(a.k + (size_t)w.t * a.k_stride + h * D + w.c * 8));
    __builtin_nontemporal_store(q, reinterpret_cast<h8v*>(a.v + (size_t)w.t * a.v_stride + h * D + w.c * 8));
  }
};

constexpr int kMoveWaves = 4;  // of a workgroup

template <typename Op, typename F, bool kScatter>
__global__ __launch_bounds__(kMoveWaves * 64) void move_kernel(Kv8MoveArgs a, int chunks, int chunk) {
  const int lane = threadIdx.x & 63, grp = lane >> 4, c = lane & 15;
  const long long units = ((long long)a.tokens + 3) / 4 * chunks;
  for (long long unit = (long long)blockIdx.x * kMoveWaves + uniform(threadIdx.x >> 6); unit < units;
       unit += (long long)gridDim.x * kMoveWaves) {
    const int w0 = (int)(unit / chunks) * 4, h0 = (int)(unit % chunks) * chunk, h1 = min(h0 + chunk, a.Hkv);
    auto heads = [&](int t, bool there, bool zero, size_t rec, int s, bool group) __attribute__((always_inline)) {
      const Window w{t, s, grp, c, there, zero, group, rec};
      typename Op::Values x[2];  // a head's loads are under way while the one before it is finished
      Op::fetch(a, w, h0, x[0]);
      for (int h = h0; h < h1; h += 2) {
        if (h + 1 < h1) Op::fetch(a, w, h + 1, x[1]);
        Op::template finish<F>(a, w, h, x[0]);
        if (h + 2 < h1) Op::fetch(a, w, h + 2, x[0]);
        if (h + 1 < h1) Op::template finish<F>(a, w, h + 1, x[1]);
      }
    };
    const int left = a.tokens - w0;
    if (kScatter) {
      const int t = w0 + min(grp, left - 1);
      int row = min(t, a.B - 1);
      if (a.offsets) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = row_of(a, w0 + min(j, left - 1), lane);
          if (grp == j) row = r;
        }
      }
      Place p = place(a, t, row);
      size_t rec = 0;
      if (p.there) rec = page_at(a, p.row, p.pos, p.there, p.zero);
      heads(t, p.there && grp < left, p.zero && grp < left, rec, p.pos % P, false);
      continue;
    }
    const int w1 = left < 4 ? a.tokens : w0 + 4;
    // Few rows: their offsets and lengths a lane each, one round of loads for all tokens.
    const bool few = a.B < 64;
    const int off = few && lane <= a.B ? a.offsets[lane] : 0, len = few && lane < a.B ? a.seq_lens[lane] : 0;
    for (int t = w0; t < w1;) {
      Place p;
      if (few) {
        const int row = max(__popcll(__builtin_amdgcn_ballot_w64(lane < a.B && off <= t)) - 1, 0);
        p = place(a, t, row, __builtin_amdgcn_readlane(off, row), __builtin_amdgcn_readlane(off, row + 1),
                  __builtin_amdgcn_readlane(off, a.B), __builtin_amdgcn_readlane(len, row));
      } else {
        p = place(a, t, row_of(a, t, lane));
      }
      if (!p.there) {  // left alone, or zeros, a token at a time
        if (p.zero) heads(t, false, grp == 0, 0, 0, false);
        ++t;
        continue;
      }
      const int first = p.pos & 3;
      const int n = min(min(p.end, a.tokens) - t, 4 - first);
      if (t == p.begin || first == 0) {
        bool there = grp >= first && grp < first + n, zero = false, page = true;
        const size_t rec = page_at(a, p.row, p.pos, page, zero);
        heads(t + grp - first, there && page, there && !page, rec, (p.pos & ~3) % P + grp, n == 4 && page);
      }
      t += n;
    }
  }
}

// ---------------------------------------------------------------------------------
// Attention.
//
// Work. A row of n tokens has ceil(n / 32) page pairs for each KV head; a segment is the pairs of
// one (row, KV head) plus kSegment units for its start and end. Segments lie one after another in
// order of (row, head), and the units of them all are dealt evenly to the waves of the launch, so
// no wave has more to read than another whatever the lengths are. A wave runs through its pairs
// as one stream, two of them in flight, with one online-softmax state at a time. A segment that
// lies within one wave goes straight to the output; a state that ends or begins at another wave
// meets the others of its segment in LDS, and what crosses workgroups goes to the workspace, where
// the last workgroup to arrive merges.
//
// A pair on the matrix cores. S^T = K Q^T: A = 16 tokens of a page, B = the queries, head h in
// columns h and 15 - h (see the formats). The result has lane (grp, col) = (lane / 16, lane % 16)
// holding tokens 4 grp .. 4 grp + 3 of its column's head: the layout that the second product's B
// operand has, so the weights go from one product to the next without leaving their lanes.
// P V: A = V^T, 16 dims by the pair's 32 tokens, B = the weights (times the tokens' V scales)
// in bf16 parts, the first in column h, the second in column 15 - h, the last in a product of its
// own. The record's V layout gives each lane its four tokens of eight dims as whole dwords, and K is
// token-major: codes go from HBM into registers and from there into the matrix cores, without LDS.
//
// What bounds it: reading the records. 32 rows of up to 32 K tokens (928 MB) take 153 us, 6.1 TB/s of
// the 6.9 that a large read reaches; without any arithmetic the same loads take 149. What is left over in
// smaller calls is 13 us at 69 MB and 13-21 at 212-309 MB: the start of the waves with their first ids and
// pages, the spread of the waves' ends, the join, and states that go through memory to the last workgroup. (A
// call that has neither long rows nor a merge takes 8 in all.) The vector ALU is busy for 43% of the time, the
// matrix cores for 11%. Short rows are bound by the chain of a pair (about 1.6 us: one row of 512 tokens, two
// pairs a wave, 11.0, of 1024 14.2), not by bytes. Wave priorities by progress and workgroups numbered by XCD
// were within 4% either way; four waves of a workgroup instead of eight were slower (64 rows of 128-4096 tokens
// 55 us against 52), and so were two pairs at a time under one maximum (rows of 16-1024 tokens at G = 8 73 us
// against 67: every odd pair costs two).
constexpr int kLogW = 3, W = 1 << kLogW;  // waves of a workgroup
constexpr int kSegment = 1;  // units of a segment beyond its pairs
// Up to so many pairs of the longest row (half of them unless the waves have several segments each)
// a wave takes whole segments: what it has more or less than others costs less than states that
// meet (int8, 8 KV heads: 256 rows of 10-60 tokens 20.7 -> 14.8 us, of 60-130 27.1 -> 24.4, of 100-250
// 31.4 -> 30.0; 32 KV heads, 64 rows of 100-300 32.1 -> 29.8). Towards the limit it goes either way (256 rows
// of 100-400 in int8 37.5 -> 39.2, in e4m3 37.8 -> 36.6; 32 KV heads, 128 rows of 100-500 in int8 69.0 -> 73.6,
// in e4m3 69.8 -> 70.1), beyond it does not pay (512 rows of 100-600 in int8 80 -> 91, in e4m3 78 -> 88).
constexpr int kWhole = 16;
constexpr int kIdPairs = 32;  // page pairs whose ids a wave holds (one id a lane)
// Pairs of the longest row times the segments per workgroup, up to which workgroups have segments of
// their own: four pairs a wave. With one segment a workgroup that is where the chain is as long as that
// of a merge over workgroups (int8, one row of 1024 tokens 14.2 us either way, of 512 11.0 against 14.4); with
// two it pays throughout (8 KV heads, 64 rows of 100-300 tokens 14.5 against 18.2, of 100-500 16.1 against 21.0;
// 32 KV heads, 16 rows of 100-500 15.8 against 21.0). With four it would also beyond, at eight pairs a wave (128
// rows of 100-500 24.8 against 28.8; 32 KV heads, 32 rows of 100-400 21.7 against 25.5). With two pairs or one
// a segment a wave for each is faster (64 rows of 20-60 9.0 against 9.6), or as fast (128 of 20-60 11.2 against 10.8).
constexpr int kOwn = 32;
static_assert(kOwn <= kIdPairs && W == 8, "the ids fetched ahead are a segment's first");

struct Pair {
  v4u k[2][2], v[2][2];  // [page][half]
  // Scales of the lane row's tokens 4 grp + i, one a lane: K of page p in lane 4 p + i, V in 8 + 4 p + i.
  // One dword a lane in one load where four of a float4 would be a third of the load instructions and 15
  // registers more (one row of 77 tokens 8.0 -> 7.8 us, of 32 K 23.7 -> 23.4, long rows the same).
  float scale;
};
// The value of lane N of the own 16.
template <int N>
__device__ __forceinline__ float of_lane(float x) { return as_f32((unsigned)dpp<0x150 + N>((int)as_u32(x))); }
// Scales of page p: AT = 0: K, 8: V.
template <int AT>
__device__ __forceinline__ v4f scales_of(float s, int p) {
  return p == 0 ? v4f{of_lane<AT>(s), of_lane<AT + 1>(s), of_lane<AT + 2>(s), of_lane<AT + 3>(s)}
                : v4f{of_lane<AT + 4>(s), of_lane<AT + 5>(s), of_lane<AT + 6>(s), of_lane<AT + 7>(s)};
}

// The partial states of a segment in a workgroup: those entries of Lds::seg whose bits are set.
struct Group {
  int seg;
  unsigned states;
  int first, last;  // workgroups with states of the segment
};

struct Lds {
  int pre[kMaxPlanBatch + 64];  // units before each row, for one KV head
  int len[kMaxPlanBatch];
  int wave_sum[W], wave_max[W];
  int seg[2 * W];    // segment of each wave's partial states (-1: none): one it continues, one it begins
  int base[2 * W], pairs[2 * W];  // the segment's first unit and its pairs
  Group group[2 * W];
  int groups, last[2];
  float head_l[2][kKv8MaxG];
  __align__(16) float part[2 * W * (kKv8MaxG * D + 2 * kKv8MaxG)];
};

__device__ __forceinline__ int pairs_of(int len) { return (int)(((unsigned)len + 2 * P - 1) / (2 * P)); }

// Four values of an output from their sums, the sum of weights and whether the row is zeroed.
__device__ __forceinline__ void store_out(uint16_t* out, v4f A, float L, bool zero) {
  const float inv = zero || L == 0.0f ? 0.0f : 1.0f / L;
  uint16_t o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = zero ? 0 : __builtin_bit_cast(uint16_t, (_Float16)(A[e] * inv));
  *reinterpret_cast<v2u*>(out) = __builtin_bit_cast(v2u, o);
}

// A page's K as loaded (columns below 8: token col, dims of the lower half, and token 8 + col, upper
// half; the others: the other halves of the same tokens) into token col's lower and upper half.
__device__ __forceinline__ void sort_rows(v4u (&k)[2], int col) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const unsigned own = col < 8 ? k[0][e] : k[1][e], other = col < 8 ? k[1][e] : k[0][e];
    k[0][e] = own;
    k[1][e] = (unsigned)dpp<0x128>((int)other);  // row_ror by 8: the lane eight apart
  }
}

// The part of a segment that a wave has: pairs p0 .. p1 - 1 of `pairs`.
struct Segment {
  int row, head, p0, p1, pairs, len, base;  // base: its first unit
};

template <typename F>
__global__ __launch_bounds__(W * 64, 2) void kv8_decode_kernel(Kv8DecodeArgs a) {
  __shared__ Lds s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int grp = lane >> 4, col = lane & 15;
  const int G = a.G;
  const int slot = G * D + ((2 * G + 3) / 4) * 4;  // floats of a state: acc [G][D], then (m, l) of each head

  auto fetch_ids = [&](int row, int p) {  // of page pairs p .. p + kIdPairs - 1, one id a lane
    return 2 * p + lane < a.max_pages_per_row ? a.block_table[(size_t)row * a.max_pages_per_row + 2 * p + lane] : 0;
  };
  // Few segments, none of them long: one for each workgroup, or 2 or 4, each with 8, 4 or 2 waves. The
  // ids are fetched while the lengths are.
  const int segments = a.B * a.Hkv, wgs = (int)gridDim.x;
  const bool few = segments <= 4 * wgs;
  const int log_per = segments <= wgs ? 0 : segments <= 2 * wgs ? 1 : 2, log_waves = kLogW - log_per;
  const int own_seg = ((int)blockIdx.x << log_per) + (wave >> log_waves);
  const int own_row = few ? min(own_seg / a.Hkv, a.B - 1) : -1;
  const int own_ids = few ? fetch_ids(own_row, 0) : 0;

  // Lengths -> units before each row (for one KV head), and the longest row's pairs. A length out of
  // range counts as none.
  auto length = [&](int i) {
    const int n = a.seq_lens[i];
    if (n >= 0 && n <= a.max_pages_per_row * P) return n;
    if (blockIdx.x == 0) atomicOr(a.err, (unsigned)PKV_DEVERR_SEQ_LEN);
    return 0;
  };
  auto scan = [&](int x) {  // over the lanes, inclusive
    x += dpp<0x111>(x);  // row_shr by 1, 2, 4, 8, then the rows' last lanes
    x += dpp<0x112>(x);
    x += dpp<0x114>(x);
    x += dpp<0x118>(x);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
    return x + __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  };
  if (lane < 2) s.seg[2 * wave + lane] = -1;
  int longest;
  if (a.B <= 64) {  // every wave for itself, all the same: no barrier
    const int n = lane < a.B ? length(lane) : 0, c = lane < a.B ? pairs_of(n) + kSegment : 0;
    const int sum = scan(c);
    s.len[lane] = n;
    s.pre[lane + 1] = sum;
    if (lane == 0) s.pre[0] = 0;
    longest = (int)across_wave((float)pairs_of(n), [](float x, float y) { return fmaxf(x, y); });
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  } else {
    const int per = (a.B + W * 64 - 1) / (W * 64);
    int sum = 0, most = 0;
    for (int j = 0; j < per; ++j) {
      const int i = tid * per + j;
      if (i >= a.B) break;
      const int n = length(i);
      s.len[i] = n;
      sum += pairs_of(n) + kSegment;
      most = max(most, pairs_of(n));
    }
    const int run = scan(sum);
    const float m = across_wave((float)most, [](float x, float y) { return fmaxf(x, y); });
    if (lane == 63) {
      s.wave_sum[wave] = run;
      s.wave_max[wave] = (int)m;
    }
    __syncthreads();
    int at = run - sum;
    longest = 0;
    for (int w = 0; w < W; ++w) {
      at += w < wave ? s.wave_sum[w] : 0;
      longest = max(longest, s.wave_max[w]);
    }
    for (int j = 0; j < per; ++j) {
      const int i = tid * per + j;
      if (i >= a.B) break;
      s.pre[i] = at;
      at += pairs_of(s.len[i]) + kSegment;
      if (i == a.B - 1) s.pre[a.B] = at;
    }
    __syncthreads();
  }

  // Segments of a workgroup's own (whole ones of a wave if several would have a pair or two each).
  const bool own = few && uniform(longest) << log_per <= kOwn && (log_per == 0 || uniform(longest) > 2);
  const int total = uniform(s.pre[a.B]) * a.Hkv;
  const int nw = own ? segments << log_waves : min(wgs * W, total);  // waves with work
  const int q_units = total / nw, r_units = total - q_units * nw;
  auto begin_of = [&](int w) { return w * q_units + min(w, r_units); };
  auto wave_of = [&](int u) {
    const int big = r_units * (q_units + 1);
    return (u < big ? 0 : r_units) + (u < big ? u : u - big) / (u < big ? q_units + 1 : q_units);
  };
  // A wave has whole segments, those that begin in its units.
  const bool whole = !own && uniform(longest) <= kWhole && uniform(longest) <= max(kWhole / 2, 2 * q_units);
  if ((int)blockIdx.x * W >= nw) return;

  const int gw = uniform((int)blockIdx.x * W + wave);
  if (gw < nw) {
    // ---- the wave's segments, one after another
    int u, u_end, row, head, off;  // units u .. u_end - 1, from pair `off` of (row, head) on
    if (own) {
      row = own_row;
      head = own_seg - row * a.Hkv;
      const int pairs = pairs_of(uniform(s.len[row])), i = wave & ((1 << log_waves) - 1);
      u = off = pairs * i >> log_waves;
      u_end = pairs > 0 ? pairs * (i + 1) >> log_waves : (i == 0 ? kSegment : 0);
    } else {
      u = begin_of(gw);
      u_end = begin_of(gw + 1);
      const int x = u / a.Hkv;
      int lo = 0, n = a.B;  // the last row with pre <= x
      while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const bool below = i < n && s.pre[lo + i] <= x;
        const int c = __popcll(__builtin_amdgcn_ballot_w64(below)) - 1;
        lo += c * step;
        n = min(step, n - c * step);
      }
      row = uniform(lo);
      const int c = uniform(s.pre[row + 1] - s.pre[row]);
      const int rel = u - uniform(s.pre[row]) * a.Hkv;
      head = rel / c;
      off = rel - head * c;
      if (whole && off > 0) {
        u += c - off;
        off = 0;
        if (++head == a.Hkv) {
          head = 0;
          ++row;
        }
      }
    }
    auto out_of = [&](const Segment& g) { return a.out + ((size_t)g.row * a.Hq + (size_t)g.head * G) * D; };
    // The next segment with pairs in the wave's range; empty rows on the way are written as zeros.
    auto next_segment = [&](Segment& g) __attribute__((always_inline)) {
      while (u < u_end) {
        const int len = uniform(s.len[row]), pairs = pairs_of(len);
        const int n = whole ? pairs + kSegment : min(pairs + kSegment - off, u_end - u);
        g = Segment{row, head, off, min(off + n, pairs), pairs, len, u - off};
        const bool first = off == 0;
        u += n;
        off = 0;
        if (++head == a.Hkv) {
          head = 0;
          ++row;
        }
        if (pairs == 0 && first)
          for (int j = lane; j < G * D / 8; j += 64) reinterpret_cast<v4u*>(out_of(g))[j] = v4u{0, 0, 0, 0};
        if (g.p0 < g.p1) return true;
      }
      return false;
    };

    // ---- the load cursor: pairs go into two buffers, those at an even distance from the start of
    // the wave's part of a segment into the first. A pair that there is not loads through an empty
    // descriptor, which reads nothing: with the same loads on every path the compiler waits for a
    // buffer's own loads only, not for all that may be under way.
    Segment ls, cs;
    int lp = 0;                            // next pair of ls to load
    int ids = 0, ids_p = 0;                // ids of ls's pairs ids_p ..
    int ids_next = own_ids, tag_row = own_row, tag_p = 0;  // fetched ahead: those of tag_row's pairs tag_p ..
    bool bad = false, bad_before = false;  // a bad page in ls; in cs when ls is ahead of it
    bool ahead = false;                    // ls is the segment after cs
    ls.p1 = 0;
    v4u qraw[4];
    const int myhead = col < 8 ? col : 15 - col;
    auto enter_ids = [&](int p) __attribute__((always_inline)) {
      if (tag_row != ls.row || p < tag_p || p >= tag_p + kIdPairs) {
        tag_row = ls.row;
        tag_p = p;
        ids_next = fetch_ids(tag_row, tag_p);
      }
      ids = ids_next;
      asm volatile("" : "+v"(ids));  // waited for here, not where each pair reads it
      ids_p = tag_p;
      // what comes next: this segment's next pairs, or the next segment's first (of the next row, if
      // that is not an empty one)
      if (ids_p + kIdPairs < ls.p1) {
        tag_p = ids_p + kIdPairs;
        ids_next = fetch_ids(tag_row, tag_p);
      } else if (u < u_end) {
        tag_row = row;
        tag_p = 0;
        ids_next = fetch_ids(tag_row, tag_p);
      }
    };
    auto enter_segment = [&]() __attribute__((always_inline)) {
      if (!next_segment(ls)) {
        ls.p1 = lp = 0;
        return;
      }
      ahead = true;
      lp = ls.p0;
      bad_before = bad;
      bad = false;
      const uint16_t* q = a.q + (size_t)ls.row * a.q_stride + ((size_t)ls.head * G + (myhead < G ? myhead : 0)) * D + grp * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j) qraw[j] = *reinterpret_cast<const v4u*>(q + (j >> 1) * 64 + (j & 1) * 8);
      enter_ids(lp);
    };
    // K: a load covers eight tokens' whole rows of 128 bytes, the two halves of a row in lanes eight
    // apart (sort_rows puts them in order): by halves of sixteen rows, 1-2% of the time is lost.
    const int k_at = (col & 7) * D + (col >> 3) * 64 + grp * 16, v_at = kKv8CodeBytes + grp * (4 * D) + col * 16;
    const int s_at = kKv8ScaleAt + (col >> 3) * (P * 4) + grp * 16 + (col & 3) * 4;
    auto load = [&](Pair& b) __attribute__((always_inline)) {
      const bool there = lp < ls.p1;
      const int left = there ? ls.len - lp * 2 * P : 0;  // tokens from the pair on
      if (there && lp - ids_p == kIdPairs) enter_ids(lp);
      const uint8_t* recs[2];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        int id = there ? __builtin_amdgcn_readlane(ids, (2 * (lp - ids_p) + pg) & 63) : 0;
        const bool page = left > pg * P;
        const bool good = id >= 0 && id < a.num_pages;
        if (page && !good) bad = true;
        id = page && good ? id : 0;
        recs[pg] = a.cache + ((size_t)id * a.Hkv + (there ? ls.head : 0)) * kKv8Record;
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t*>(recs[pg]), (short)0, page && good ? kKv8Record : 0, 0x00020000);
        b.k[pg][0] = __builtin_amdgcn_raw_buffer_load_b128(r, k_at, 0, kNt);
        b.k[pg][1] = __builtin_amdgcn_raw_buffer_load_b128(r, (k_at ^ 64) + 8 * D, 0, kNt);
        b.v[pg][0] = __builtin_amdgcn_raw_buffer_load_b128(r, v_at, 0, kNt);
        b.v[pg][1] = __builtin_amdgcn_raw_buffer_load_b128(r, v_at + 256, 0, kNt);
      }
      // (of a page that there is not: record 0's, for no token)
      b.scale = __builtin_nontemporal_load(reinterpret_cast<const float*>((col & 4 ? recs[1] : recs[0]) + s_at));
      lp += there;
    };

    // ---- the segment being computed
    typename F::Query q;
    v4f acc[8];  // tile t, row 4 grp + i: dim 16 grp + 4 i + t (t < 4) or 64 + 16 grp + 4 i + t - 4
    float m, l;
    int cp = 0;
    auto begin_segment = [&]() __attribute__((always_inline)) {
      cs = ls;
      ahead = false;
      cp = cs.p0;
      q.set(qraw, myhead < G, col, a.scale_log2);
      m = kLowest;
      l = 0.0f;
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    };
    auto end_segment = [&]() __attribute__((always_inline)) {
      const bool wrong = ahead ? bad_before : bad;
#pragma unroll
      for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] += mirror16(acc[t][i]);  // the second parts' sums join
      const float sum = across_rows(l, [](float x, float y) { return x + y; });
      const bool begins = cs.p0 == 0, ends = cs.p1 == cs.pairs;
      if (wrong && lane == 0) atomicOr(a.err, (unsigned)PKV_DEVERR_PAGE_ID);
      if (begins && ends) {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        uint16_t* out = out_of(cs);
        if (col < G) {
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              h8v o;
#pragma unroll
              for (int e = 0; e < 8; ++e) o[e] = (_Float16)(wrong ? 0.0f : acc[4 * half + (e & 3)][2 * j + (e >> 2)] * inv);
              *reinterpret_cast<h8v*>(out + col * D + half * 64 + grp * 16 + j * 8) = o;
            }
        }
      } else {
        const int at = 2 * wave + (begins ? 1 : 0);
        float* part = s.part + at * slot;
        if (col < G) {
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<v4f*>(part + col * D + half * 64 + grp * 16 + i * 4) =
                  v4f{acc[4 * half][i], acc[4 * half + 1][i], acc[4 * half + 2][i], acc[4 * half + 3][i]};
          if (grp == 0) {
            part[G * D + 2 * col] = m;
            part[G * D + 2 * col + 1] = wrong ? -1.0f : sum;
          }
        }
        if (lane == 0) {
          s.seg[at] = cs.row * a.Hkv + cs.head;
          s.base[at] = cs.base;
          s.pairs[at] = cs.pairs;
        }
      }
    };
    auto attend = [&](Pair& b, int pair) __attribute__((always_inline)) {
      v4f x[2], vs[2];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        sort_rows(b.k[pg], col);
        x[pg] = q.scores(b.k[pg], scales_of<0>(b.scale, pg));
        vs[pg] = scales_of<8>(b.scale, pg);
      }
      const int left = cs.len - pair * 2 * P;
      if (left < 2 * P) {  // tokens past the row's end: no weight, whatever the record holds there
        asm volatile("");  // kept a branch: as selects in every pair it is a fifth of the arithmetic
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          const int n = min(max(left - pg * P - 4 * grp, 0), 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[pg][i] = i < n ? x[pg][i] : -__builtin_inff();
            vs[pg][i] = i < n ? vs[pg][i] : 0.0f;
          }
          const unsigned keep = n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
#pragma unroll
          for (int h = 0; h < 2; ++h) b.v[pg][h] &= v4u{keep, keep, keep, keep};
        }
      }
      float top = m;
#pragma unroll
      for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, x[pg][i]);
      top = across_rows(top, [](float y, float z) { return fmaxf(y, z); });
      if (__builtin_amdgcn_ballot_w64(top > m) != 0) {
        const float c = ex2(m - top);
        l *= c;
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[t] *= v4f{c, c, c, c};
        m = top;
      }
      // A weight times its token's V scale in three bf16 parts of eight bits each, from the top down: all 24 bits
      // of it, so values that cancel in the sum cost no more than in fp32. bf16 has fp32's range, so no
      // scale is too small or large for it. The last part, for which the columns have no place, is a product
      // of its own (eight more matrix instructions a pair: 64 rows of 128-4096 tokens 52.7 us against 52.5
      // without it; with up to four heads in columns left over it is no faster, at 19 registers more).
      v4u w, w0;
#pragma unroll
      for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          float own[2], low[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float e = ex2(x[pg][i + j] - m);
            l += e;
            const float f = e * vs[pg][i + j];
            const float rest = f - as_f32(as_u32(f) & 0xFFFF0000u), last = rest - as_f32(as_u32(rest) & 0xFFFF0000u);
            own[j] = col < 8 ? f : rest;
            low[j] = col < 8 ? last : 0.0f;
          }
          w[2 * pg + i / 2] = __builtin_amdgcn_perm(as_u32(own[1]), as_u32(own[0]), 0x07060302u);  // upper halves
          w0[2 * pg + i / 2] = __builtin_amdgcn_perm(as_u32(low[1]), as_u32(low[0]), 0x07060302u);
        }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const b8v v = load8<F>(b.v[0][t >> 2][t & 3], b.v[1][t >> 2][t & 3]);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(b8v, w), acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(b8v, w0), acc[t], 0, 0, 0);
        if (t & 1) __builtin_amdgcn_sched_barrier(0);  // the conversions of a few tiles at a time: else they spill
      }
    };

    // ---- the stream: two pairs are computed, each one's buffer then loads the pair after the other's
    // (three buffers: one row of 32 K 26 us against 23.5, rows of 16-1024 tokens 72 against 68)
    Pair b0, b1;
    for (bool live = false;;) {
      if (live) attend(b0, cp);
      if (lp >= ls.p1) enter_segment();
      load(b0);
      if (live && cp + 1 < cs.p1) attend(b1, cp + 1);
      load(b1);
      if (live) {
        cp += 2;
        if (cp < cs.p1) continue;
        end_segment();
      }
      if (!ahead) break;
      begin_segment();
      live = true;
    }
  }
  if (whole) return;
  __syncthreads();

  // ---- states of segments that several waves share: runs of equal entries of s.seg
  const int SB = slot * (int)sizeof(float);
  if (wave == 0) {
    const int mine = lane < 2 * W ? s.seg[lane] : -1;
    const unsigned valid = (unsigned)__builtin_amdgcn_ballot_w64(mine >= 0);
    const unsigned below = lane < 2 * W ? valid & ((1u << lane) - 1) : 0;
    const int prev = __shfl(mine, below ? 31 - __builtin_clz(below) : 0);
    const unsigned starts = (unsigned)__builtin_amdgcn_ballot_w64(mine >= 0 && (!below || prev != mine));
    if (lane < 2 * W && (starts >> lane & 1)) {
      Group& g = s.group[__popcll(starts & ((1u << lane) - 1))];
      const unsigned next = starts & ~((2u << lane) - 1);
      const int base = s.base[lane], end = base + s.pairs[lane];
      g.seg = mine;
      g.states = valid & (next ? (1u << __builtin_ctz(next)) - 1 : 0xFFFFFFFFu) & ~((1u << lane) - 1);
      g.first = g.last = (int)blockIdx.x;
      // the workgroups that hold states of the segment: those of its first to its last pair
      if (!own && (base < begin_of(blockIdx.x * W) || end > begin_of(blockIdx.x * W + W))) {
        g.first = wave_of(base) / W;
        g.last = wave_of(end - 1) / W;
      }
    }
    if (lane == 0) {
      s.groups = __popcll(starts);
      s.last[0] = s.last[1] = -1;
    }
  }
  __syncthreads();
  // Whole waves take a segment, 32 lanes a head, four values a lane; as many side by side as there
  // are waves for. Lane j of a head's 32 makes the weight of state j.
  const int cols = G * (D / 4);  // float4 columns of a state
  const int team_waves = (cols + 63) / 64;
  const __amdgpu_buffer_rsrc_t pr =
      __builtin_amdgcn_make_buffer_rsrc(a.partials, (short)0, 2 * kKv8MaxWorkgroups * SB, 0x00020000);
  const int groups = uniform(s.groups), teams = W / team_waves, my_team = wave / team_waves;
  for (int gi = my_team; gi < groups && my_team < teams; gi += teams) {
    const int e4 = (wave - my_team * team_waves) * 64 + lane, h = e4 / (D / 4), hl = lane & 31;
    const int seg = uniform(s.group[gi].seg), first = uniform(s.group[gi].first), last = uniform(s.group[gi].last);
    const unsigned states = (unsigned)uniform((int)s.group[gi].states);
    const bool in = e4 < cols;
    const bool has = in && hl < 2 * W && (states >> hl & 1);
    const v2f ml = has ? *reinterpret_cast<const v2f*>(s.part + hl * slot + G * D + 2 * h) : v2f{kLowest, 0.0f};
    const float M = half_wave(ml.x, [](float y, float z) { return fmaxf(y, z); });
    const bool zero = half_wave(ml.y, [](float y, float z) { return fminf(y, z); }) < 0.0f;
    const float c = ex2(ml.x - M);
    const float L = half_wave(c * ml.y, [](float y, float z) { return y + z; });
    v4f A = {0.0f, 0.0f, 0.0f, 0.0f};
    for (unsigned todo = states; todo != 0;) {
      v4f x[4];
      float w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // past the last one: its weight is that of a state that is not
        const int j = todo ? __builtin_ctz(todo) : 31;
        todo &= todo - 1;
        x[i] = *reinterpret_cast<const v4f*>(s.part + min(j, 2 * W - 1) * slot + (in ? 4 * e4 : 0));
        w[i] = __shfl(c, (lane & 32) + j);
        if (j == 31) x[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) A[e] = __builtin_fmaf(w[i], x[i][e], A[e]);
    }
    if (!in) continue;
    if (first == last) {
      store_out(a.out + (size_t)seg * G * D + 4 * e4, A, L, zero);
    } else {
      const int so = (2 * blockIdx.x + (first == (int)blockIdx.x ? 1 : 0)) * SB;
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, A), pr, so + e4 * 16, 0, kSc1);
      if (hl == 0)
        __builtin_amdgcn_raw_buffer_store_b64(v2u{as_u32(M), as_u32(zero ? -1.0f : L)}, pr, so + (G * D + 2 * h) * 4, 0, kSc1);
    }
  }
  if (own) return;

  // ---- completion count of the (at most two) segments that cross into other workgroups
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (tid < groups) {
    const Group g = s.group[tid];
    if (g.first != g.last) {
      const int prev = __hip_atomic_fetch_add(&a.counters[g.seg], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (prev == g.last - g.first) {
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        s.last[g.first == (int)blockIdx.x ? 1 : 0] = tid;
        a.counters[g.seg] = 0;
      }
    }
  }
  __syncthreads();

  // ---- merge of the segments whose last state this workgroup brought, by half of it each if there
  // are two. The states of a column of four values are summed in `ng` runs (every ng-th state one
  // run, whether a whole workgroup has the segment or half of one: the order of sums is the same),
  // the runs then in order. The waves make the weights of a head each.
  const int found0 = uniform(s.last[0]), found1 = uniform(s.last[1]);
  if (found0 < 0 && found1 < 0) return;
  const bool two = found0 >= 0 && found1 >= 0;
  const int team = two ? wave / (W / 2) : 0, threads = two ? W * 32 : W * 64;
  const int gi = team == 1 || found0 < 0 ? found1 : found0;
  const int seg = uniform(s.group[gi].seg), first = uniform(s.group[gi].first), n = uniform(s.group[gi].last) - first + 1;
  auto slot_at = [&](int j) { return j < n ? (2 * (first + j) + (j == 0 ? 1 : 0)) * SB : kOutOfRange; };
  const int ttid = tid - team * (W * 32);
  const int ng = W * 64 / cols, per = threads / cols, mine = ttid / cols, e4 = ttid - mine * cols, h = e4 / (D / 4);
  auto load = [&](int j) __attribute__((always_inline)) {
    return __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(pr, slot_at(mine < per ? j : n) + e4 * 16, 0, kSc1));
  };
  // The first sixteen states of the run, or the first eight of two runs, behind the loads of the first
  // maxima and sums.
  v4f x[16];
  auto preload = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j0 = (two ? i & 7 : i) * ng;
      if (j0 < n) x[i] = load(two && i >= 8 ? mine + per + j0 : mine + j0);
      else x[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
  };
  const int head0 = wave - team * (W / 2);
  if (head0 >= G) preload();
  float* wt = s.part + team * (kKv8MaxWorkgroups * kKv8MaxG);                     // [n][G] weights
  float* sums = s.part + 2 * kKv8MaxWorkgroups * kKv8MaxG + team * (W * 64 * 4);  // [ng][G * D]
  for (int hh = head0; hh < G; hh += threads / 64) {
    constexpr int kRounds = kKv8MaxWorkgroups / 64;
    v2u ml[kRounds];
    float M = kLowest, L = 0.0f, low = 0.0f;
#pragma unroll
    for (int i = 0; i < kRounds; ++i)
      if (64 * i < n) ml[i] = __builtin_amdgcn_raw_buffer_load_b64(pr, slot_at(64 * i + lane) + (G * D + 2 * hh) * 4, 0, kSc1);
    if (hh == head0) preload();
#pragma unroll
    for (int i = 0; i < kRounds; ++i)
      if (64 * i + lane < n) {
        M = fmaxf(M, as_f32(ml[i].x));
        low = fminf(low, as_f32(ml[i].y));
      }
    M = across_wave(M, [](float y, float z) { return fmaxf(y, z); });
    low = across_wave(low, [](float y, float z) { return fminf(y, z); });
#pragma unroll
    for (int i = 0; i < kRounds; ++i)
      if (64 * i + lane < n) {
        const float c = ex2(as_f32(ml[i].x) - M);
        wt[(64 * i + lane) * G + hh] = c;
        L = __builtin_fmaf(c, as_f32(ml[i].y), L);
      }
    L = across_wave(L, [](float y, float z) { return y + z; });
    if (lane == 0) s.head_l[team][hh] = low < 0.0f ? -1.0f : L;
  }
  __syncthreads();
  for (int run = mine; run < ng && mine < per; run += per) {
    v4f A = {0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](int j, v4f y) __attribute__((always_inline)) {
      const float c = j < n ? wt[j * G + h] : 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) A[e] = __builtin_fmaf(c, y[e], A[e]);
    };
    int j = run;
    if (run == mine || run == mine + per) {
#pragma unroll
      for (int i = 0; i < 8; ++i) add(j + i * ng, run == mine ? x[i] : x[i + 8]);
      j += 8 * ng;
      if (!two) {
#pragma unroll
        for (int i = 0; i < 8; ++i) add(j + i * ng, x[i + 8]);
        j += 8 * ng;
      }
    }
    for (; j < n; j += 4 * ng) {
      v4f y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = load(j + i * ng);
#pragma unroll
      for (int i = 0; i < 4; ++i) add(j + i * ng, y[i]);
    }
    *reinterpret_cast<v4f*>(sums + (run * cols + e4) * 4) = A;
  }
  __syncthreads();
  if (mine == 0) {
    v4f A = *reinterpret_cast<const v4f*>(sums + e4 * 4);
    for (int j = 1; j < ng; ++j) A += *reinterpret_cast<const v4f*>(sums + (j * cols + e4) * 4);
    const float L = s.head_l[team][h];
    store_out(a.out + (size_t)seg * G * D + 4 * e4, A, L, L < 0.0f);
  }
}

// Compute units of the current device.
int device_units() {
  static std::atomic<int> units[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return 256;
  int n = units[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) n = 256;
    units[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

}  // namespace

hipError_t launch_kv8_decode(const Kv8DecodeArgs& a, int format, hipStream_t s) {
  // One workgroup per compute unit, fewer where the block table cannot hold as many units of work (but
  // one for each segment, if there are no more).
  const long long most = (long long)a.B * a.Hkv * ((a.max_pages_per_row + 1) / 2 + kSegment);
  long long grid = (most + W - 1) / W;
  if (grid < (long long)a.B * a.Hkv) grid = (long long)a.B * a.Hkv;
  const int cap = device_units() < kKv8MaxWorkgroups ? device_units() : kKv8MaxWorkgroups;
  if (grid > cap) grid = cap;
  if (format == PKV_KV8_INT8) hipLaunchKernelGGL(kv8_decode_kernel<Int8>, dim3((unsigned)grid), dim3(W * 64), 0, s, a);
  else hipLaunchKernelGGL(kv8_decode_kernel<E4m3>, dim3((unsigned)grid), dim3(W * 64), 0, s, a);
  return hipGetLastError();
}

namespace {

// Heads per wave: one, as long as the waves then are no more than twice what the device holds, so
// that small calls spread; beyond, several, which share the lookups (16 rows of up to 8192 tokens read
// back: one head a wave 114 us, up to 65536 waves 91, 16384 or 4096 82, and 71 with two heads under
// way; chunks of eight rows 14.4 us at 16384, 14.0 at 4096).
constexpr long long kMoveUnits = 4096;

template <typename Op, typename F>
hipError_t launch_move(const Kv8MoveArgs& a, hipStream_t s) {
  const long long windows = ((long long)a.tokens + 3) / 4;
  long long chunk = (windows * a.Hkv + kMoveUnits - 1) / kMoveUnits;
  if (chunk > a.Hkv) chunk = a.Hkv;
  const long long chunks = (a.Hkv + chunk - 1) / chunk;
  long long blocks = (windows * chunks + kMoveWaves - 1) / kMoveWaves;
  if (blocks > 1 << 22) blocks = 1 << 22;  // a launch's size in threads has 32 bits
  const bool scatter = !a.offsets || a.tokens < 4ll * a.B;
  if (scatter) hipLaunchKernelGGL((move_kernel<Op, F, true>), dim3((unsigned)blocks), dim3(kMoveWaves * 64), 0, s, a, (int)chunks, (int)chunk);
  else hipLaunchKernelGGL((move_kernel<Op, F, false>), dim3((unsigned)blocks), dim3(kMoveWaves * 64), 0, s, a, (int)chunks, (int)chunk);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv8_append(const Kv8MoveArgs& a, int format, hipStream_t s) {
  return format == PKV_KV8_INT8 ? launch_move<Append, Int8>(a, s) : launch_move<Append, E4m3>(a, s);
}

hipError_t launch_kv8_gather(const Kv8MoveArgs& a, int format, hipStream_t s) {
  return format == PKV_KV8_INT8 ? launch_move<Gather, Int8>(a, s) : launch_move<Gather, E4m3>(a, s);
}

}  // namespace pkv
