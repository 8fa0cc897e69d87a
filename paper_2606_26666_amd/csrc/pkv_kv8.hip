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
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));

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

// ---------------------------------------------------------------------------------
// Formats. `load8` makes the bf16 operand of eight codes (exact: int8 has 8 and e4m3 4 significant
// bits); `code` rounds x * top / m, where the product is exact in fp32 (11 + 7 bits) and the
// division correctly rounded: a quotient of such numbers that is not on a rounding border is at
// least 2^-19 of its size away from it, so the code is that of real arithmetic.
struct Int8 {
  static constexpr float top = 127.0f;
  static __device__ __forceinline__ unsigned code(float y) { return (unsigned)(int)__builtin_rintf(y) & 255u; }
  static __device__ __forceinline__ float value(unsigned c) { return (float)(signed char)c; }
  // Two fp32 halves each with an integer of at most 8 bits: their upper 16 bits are the bf16s.
  static __device__ __forceinline__ v2u load4(unsigned w) {
    const float a = (float)(signed char)(w & 255u), b = (float)(signed char)((w >> 8) & 255u);
    const float c = (float)(signed char)((w >> 16) & 255u), d = (float)(signed char)(w >> 24);
    return v2u{__builtin_amdgcn_perm(as_u32(b), as_u32(a), 0x07060302u), __builtin_amdgcn_perm(as_u32(d), as_u32(c), 0x07060302u)};
  }
};
struct E4m3 {
  static constexpr float top = 448.0f;
  static __device__ __forceinline__ unsigned code(float y) {
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 255u;
  }
  static __device__ __forceinline__ float value(unsigned c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }
  static __device__ __forceinline__ v2u load4(unsigned w) {
    return v2u{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))};
  }
};

template <typename F>
__device__ __forceinline__ b8v load8(unsigned lo, unsigned hi) {
  const v2u a = F::load4(lo), b = F::load4(hi);
  return __builtin_bit_cast(b8v, v4u{a.x, a.y, b.x, b.y});
}

// ---------------------------------------------------------------------------------
// Append and gather.

// Where packed token t goes: its row (the last i with offsets[i] <= t) and position. False when the
// token is not to be touched; `zero`: it is to be read back as zeros. Safe for any offsets.
struct Place {
  int row, pos;
  bool there, zero;
};
__device__ __forceinline__ Place place(const Kv8MoveArgs& a, int t) {
  Place p{t, 0, true, false};
  int end = t + 1;
  if (a.offsets) {
    int lo = 0, hi = a.B;  // offsets[lo] <= t < offsets[hi], as far as they ascend
    if (t >= a.offsets[a.B] || t < a.offsets[0]) return Place{0, 0, false, false};
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.offsets[mid] <= t) lo = mid; else hi = mid;
    }
    p.row = lo;
    end = a.offsets[lo + 1];
  }
  const int len = a.seq_lens[p.row];
  const int begin = a.offsets ? a.offsets[p.row] : t;
  if (!a.offsets && len == 0) return Place{0, 0, false, true};
  if (len < 0 || len > a.max_pages_per_row * P || begin < 0 || end < begin || end - begin > len) {
    atomicOr(a.err, (unsigned)PKV_DEVERR_SEQ_LEN);
    return Place{0, 0, false, true};
  }
  p.pos = len - (end - t);
  return p;
}

__device__ __forceinline__ uint8_t* record(const Kv8MoveArgs& a, Place& p, int h) {
  const int id = a.block_table[(size_t)p.row * a.max_pages_per_row + p.pos / P];
  if (id < 0 || id >= a.num_pages) {
    atomicOr(a.err, (unsigned)PKV_DEVERR_PAGE_ID);
    p.there = false;
    p.zero = true;
    return a.cache;
  }
  return a.cache + ((size_t)id * a.Hkv + h) * kKv8Record;
}

// Sixteen lanes per (token, KV head), eight values a lane.
template <typename F>
__global__ __launch_bounds__(256) void append_kernel(Kv8MoveArgs a) {
  const int c = threadIdx.x & 15;
  const long long n = (long long)a.tokens * a.Hkv;
  for (long long i = (blockIdx.x * 256ll + threadIdx.x) >> 4; i < n; i += gridDim.x * 16ll) {
    const int t = (int)(i / a.Hkv), h = (int)(i % a.Hkv);
    Place p = place(a, t);
    if (!p.there) continue;
    uint8_t* rec = record(a, p, h);
    if (!p.there) continue;
    const int s = p.pos % P;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const uint16_t* src = kv ? a.v + (size_t)t * a.v_stride : a.k + (size_t)t * a.k_stride;
      const v4u raw = *reinterpret_cast<const v4u*>(src + (size_t)h * D + c * 8);
      unsigned m = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m = max(m, raw[j] & 0x7FFFu);
        m = max(m, (raw[j] >> 16) & 0x7FFFu);
      }
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, x));
      const bool finite = m < 0x7C00u;
      const float top = (float)__builtin_bit_cast(_Float16, (uint16_t)m);
      const h8v x = __builtin_bit_cast(h8v, raw);
      uint8_t code[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) code[j] = finite && m > 0 ? (uint8_t)F::code((float)x[j] * F::top / top) : 0;
      if (kv == 0) {
        *reinterpret_cast<v2u*>(rec + s * D + c * 8) = __builtin_bit_cast(v2u, code);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) rec[kKv8CodeBytes + (s / 4) * (4 * D) + (c * 8 + j) * 4 + s % 4] = code[j];
      }
      if (c == 0) reinterpret_cast<float*>(rec + kKv8ScaleAt)[kv * P + s] = finite ? top / F::top : as_f32(0x7FC00000u);
    }
  }
}

template <typename F>
__global__ __launch_bounds__(256) void gather_kernel(Kv8MoveArgs a) {
  const int c = threadIdx.x & 15;
  const long long n = (long long)a.tokens * a.Hkv;
  for (long long i = (blockIdx.x * 256ll + threadIdx.x) >> 4; i < n; i += gridDim.x * 16ll) {
    const int t = (int)(i / a.Hkv), h = (int)(i % a.Hkv);
    Place p = place(a, t);
    const uint8_t* rec = a.cache;
    if (p.there) rec = record(a, p, h);
    if (!p.there && !p.zero) continue;
    const int s = p.pos % P;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      h8v x = {};
      if (p.there) {
        const float scale = reinterpret_cast<const float*>(rec + kKv8ScaleAt)[kv * P + s];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint8_t code = kv == 0 ? rec[s * D + c * 8 + j]
                                       : rec[kKv8CodeBytes + (s / 4) * (4 * D) + (c * 8 + j) * 4 + s % 4];
          x[j] = (_Float16)(F::value(code) * scale);
        }
      }
      uint16_t* dst = kv ? a.v + (size_t)t * a.v_stride : a.k + (size_t)t * a.k_stride;
      *reinterpret_cast<h8v*>(dst + (size_t)h * D + c * 8) = x;
    }
  }
}

// ---------------------------------------------------------------------------------
// Attention.
//
// Work. A row of n tokens has ceil(n / 32) page pairs for each KV head; a segment is the pairs of
// one (row, KV head) plus kSegment units for its start and end. Segments lie one after another in
// order of (row, head), and the units of them all are dealt evenly to the waves of the launch, so
// no wave has more to read than another whatever the lengths are. A wave runs through its units
// with one online-softmax state at a time. A segment that lies within one wave goes straight to
// the output; a state that ends or begins at another wave meets the others of its segment in LDS,
// and what crosses workgroups goes to the workspace, where the last workgroup to arrive merges.
//
// A pair on the matrix cores. K S^T: A = 16 tokens of a page by 32 dims, B = the queries as bf16
// high and low halves (exact: fp16 has 11 bits), head h in column h and its low half in column
// 15 - h; the two columns are added by a mirror of the 16 lanes. The result has lane (grp, col) =
// (lane / 16, lane % 16) holding tokens 4 grp .. 4 grp + 3 of head col: the layout that the second
// product's B operand has, so the weights go from one product to the next without leaving their
// lanes. P V: A = V^T, 16 dims by the pair's 32 tokens, B = the weights (times the tokens' V scales)
// as bf16 high halves in column h and low halves in column 15 - h. The record's V layout gives each
// lane its four tokens of eight dims as whole dwords, and K is token-major: codes go from HBM into
// registers and from there, converted, into the matrix cores, without LDS.
constexpr int W = 8;        // waves of a workgroup
constexpr int kSegment = 1;  // units of a segment beyond its pairs

struct Pair {
  v4u k[2][2], v[2][2];  // [page][half]
  v4f ks[2], vs[2];
};

// State of one segment in a wave: head col < G (col >= 8: the low halves' sums).
struct State {
  v4f acc[8];  // tile t, dims 16 grp + .. (see write_state)
  float m, l;
};

struct Lds {
  int pre[kMaxPlanBatch + 1];
  int wave_sum[W];
  int seg[2 * W];    // segment of each wave's partial states (-1: none): one it continues, one it begins
  int group_at[2 * W], group_n[2 * W];
  int groups, last[2];
  __align__(16) float part[2 * W * (kKv8MaxG * D + 2 * kKv8MaxG)];
};

__device__ __forceinline__ int pairs_of(int len) { return (int)(((unsigned)len + 2 * P - 1) / (2 * P)); }

template <typename F>
__global__ __launch_bounds__(W * 64, 2) void kv8_decode_kernel(Kv8DecodeArgs a) {
  __shared__ Lds s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int grp = lane >> 4, col = lane & 15;
  const int G = a.G;
  const int slot = G * D + ((2 * G + 3) / 4) * 4;  // floats of a state: acc [G][D], then (m, l) of each head

  // Lengths -> units before each row (for one KV head). A length out of range counts as none.
  const int per = (a.B + W * 64 - 1) / (W * 64);
  auto length = [&](int i) {
    const int n = a.seq_lens[i];
    return n < 0 || n > a.max_pages_per_row * P ? 0 : n;
  };
  {
    int sum = 0;
    for (int j = 0; j < per; ++j) {
      const int i = tid * per + j;
      if (i >= a.B) break;
      const int n = a.seq_lens[i];
      if (blockIdx.x == 0 && (n < 0 || n > a.max_pages_per_row * P)) atomicOr(a.err, (unsigned)PKV_DEVERR_SEQ_LEN);
      sum += pairs_of(length(i)) + kSegment;
    }
    int run = sum;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int y = __shfl(run, lane - x);
      if (lane >= x) run += y;
    }
    if (lane == 63) s.wave_sum[wave] = run;
    if (lane < 2) s.seg[2 * wave + lane] = -1;
    __syncthreads();
    int at = run - sum;
    for (int w = 0; w < wave; ++w) at += s.wave_sum[w];
    for (int j = 0; j < per; ++j) {
      const int i = tid * per + j;
      if (i >= a.B) break;
      s.pre[i] = at;
      at += pairs_of(length(i)) + kSegment;
      if (i == a.B - 1) s.pre[a.B] = at;
    }
  }
  __syncthreads();

  const int total = uniform(s.pre[a.B]) * a.Hkv;
  const int nw = min((int)gridDim.x * W, total);  // waves with work
  const int q_units = total / nw, r_units = total - q_units * nw;
  auto begin_of = [&](int w) { return w * q_units + min(w, r_units); };
  auto wave_of = [&](int u) {
    const int big = r_units * (q_units + 1);
    return u < big ? u / (q_units + 1) : r_units + (u - big) / q_units;
  };
  if ((int)blockIdx.x * W >= nw) return;

  // A finished state: out of this wave's registers into `out`.
  State st;
  bool bad = false;
  auto total_l = [&] { return across_rows(st.l, [](float x, float y) { return x + y; }); };
  auto halves = [&] {  // the low halves' sums join those of the high halves
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.acc[t][i] += mirror16(st.acc[t][i]);
  };
  // Tile t, row 4 grp + i of the products is dim 16 grp + 4 i + t (t < 4) or 64 + 16 grp + 4 i + t - 4.

  const int gw = uniform((int)blockIdx.x * W + wave);
  if (gw < nw) {
    int u = begin_of(gw);
    const int u_end = begin_of(gw + 1);
    // the row of unit u
    int row;
    {
      const int x = u / a.Hkv;
      int lo = 0, hi = a.B;  // pre[lo] <= x < pre[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.pre[mid] <= x) lo = mid; else hi = mid;
      }
      row = uniform(lo);
    }
    int c_units = uniform(s.pre[row + 1] - s.pre[row]);
    int rel = u - uniform(s.pre[row]) * a.Hkv;
    int head = rel / c_units;
    int off = rel - head * c_units;
    while (u < u_end) {
      const int pairs = c_units - kSegment;
      const int n_units = min(c_units - off, u_end - u);
      const int p0 = off, p1 = min(off + n_units, pairs);
      const int len = uniform(length(row));
      uint16_t* out = a.out + ((size_t)row * a.Hq + (size_t)head * G) * D;
      if (pairs == 0) {
        if (off == 0)
          for (int j = lane; j < G * D / 8; j += 64) reinterpret_cast<v4u*>(out)[j] = v4u{0, 0, 0, 0};
      } else if (p0 < p1) {
        // ---- the segment's queries
        const int myhead = col < 8 ? col : 15 - col;
        v4u qraw[4];
        {
          const uint16_t* q = a.q + (size_t)row * a.q_stride + ((size_t)head * G + (myhead < G ? myhead : 0)) * D + grp * 16;
#pragma unroll
          for (int j = 0; j < 4; ++j) qraw[j] = *reinterpret_cast<const v4u*>(q + (j >> 1) * 64 + (j & 1) * 8);
        }
        // ---- page ids, 64 at a time, the next 64 ahead
        const int pages = (len + P - 1) / P;
        const int* table = a.block_table + (size_t)row * a.max_pages_per_row;
        auto fetch_ids = [&](int pair) { return 2 * pair + lane < pages ? table[2 * pair + lane] : 0; };
        int ids = fetch_ids(p0), ids_next = fetch_ids(p0 + 32);
        auto load = [&](Pair& b, int pair) __attribute__((always_inline)) {
          const int j = pair - p0;
          if (j > 0 && (j & 31) == 0) {
            ids = ids_next;
            ids_next = fetch_ids(pair + 32);
          }
#pragma unroll
          for (int pg = 0; pg < 2; ++pg) {
            int id = __builtin_amdgcn_readlane(ids, 2 * (j & 31) + (2 * pair + pg < pages ? pg : 0));
            if (id < 0 || id >= a.num_pages) {
              bad = true;
              id = 0;
            }
            const uint8_t* rec = a.cache + ((size_t)id * a.Hkv + head) * kKv8Record;
            const v4u* kp = reinterpret_cast<const v4u*>(rec + col * D + grp * 16);
            const v4u* vp = reinterpret_cast<const v4u*>(rec + kKv8CodeBytes + grp * (4 * D) + col * 16);
            const v4f* sp = reinterpret_cast<const v4f*>(rec + kKv8ScaleAt + grp * 16);
            b.k[pg][0] = __builtin_nontemporal_load(kp);
            b.k[pg][1] = __builtin_nontemporal_load(kp + 4);
            b.v[pg][0] = __builtin_nontemporal_load(vp);
            b.v[pg][1] = __builtin_nontemporal_load(vp + 16);
            b.ks[pg] = __builtin_nontemporal_load(sp);
            b.vs[pg] = __builtin_nontemporal_load(sp + 4);
          }
        };
        bad = false;
        Pair b0, b1;
        load(b0, p0);
        if (p0 + 1 < p1) load(b1, p0 + 1);
        b8v q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const h8v x = __builtin_bit_cast(h8v, qraw[j]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float f = myhead < G ? (float)x[e] : 0.0f;
            const __bf16 hi = (__bf16)f;
            q[j][e] = col < 8 ? hi : (__bf16)(f - (float)hi);
          }
        }
        st.m = kLowest;
        st.l = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) st.acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

        auto attend = [&](Pair& b, int pair) __attribute__((always_inline)) {
          v4f x[2];
#pragma unroll
          for (int pg = 0; pg < 2; ++pg) {
            x[pg] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const v4u& kk = b.k[pg][j >> 1];
              x[pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(load8<F>(kk[2 * (j & 1)], kk[2 * (j & 1) + 1]), q[j], x[pg], 0, 0, 0);
            }
          }
#pragma unroll
          for (int pg = 0; pg < 2; ++pg)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[pg][i] = (x[pg][i] + mirror16(x[pg][i])) * (b.ks[pg][i] * a.scale_log2);
          const int left = len - pair * 2 * P;
          if (left < 2 * P) {  // tokens past the row's end: no weight, whatever the record holds there
#pragma unroll
            for (int pg = 0; pg < 2; ++pg) {
              const int n = min(max(left - pg * P - 4 * grp, 0), 4);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                x[pg][i] = i < n ? x[pg][i] : -__builtin_inff();
                b.vs[pg][i] = i < n ? b.vs[pg][i] : 0.0f;
              }
              const unsigned keep = n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
#pragma unroll
              for (int h = 0; h < 2; ++h) b.v[pg][h] &= v4u{keep, keep, keep, keep};
            }
          }
          float m = st.m;
#pragma unroll
          for (int pg = 0; pg < 2; ++pg)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = fmaxf(m, x[pg][i]);
          m = across_rows(m, [](float y, float z) { return fmaxf(y, z); });
          if (__builtin_amdgcn_ballot_w64(m > st.m) != 0) {
            const float c = ex2(st.m - m);
            st.l *= c;
#pragma unroll
            for (int t = 0; t < 8; ++t) st.acc[t] *= v4f{c, c, c, c};
            st.m = m;
          }
          b8v w;
#pragma unroll
          for (int pg = 0; pg < 2; ++pg)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float e = ex2(x[pg][i] - st.m);
              st.l += e;
              const float f = e * b.vs[pg][i];
              const __bf16 hi = (__bf16)f;
              w[4 * pg + i] = col < 8 ? hi : (__bf16)(f - (float)hi);
            }
#pragma unroll
          for (int t = 0; t < 8; ++t)
            st.acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(load8<F>(b.v[0][t >> 2][t & 3], b.v[1][t >> 2][t & 3]), w, st.acc[t], 0, 0, 0);
        };
        for (int pair = p0; pair < p1; pair += 2) {
          attend(b0, pair);
          if (pair + 2 < p1) load(b0, pair + 2);
          if (pair + 1 < p1) {
            attend(b1, pair + 1);
            if (pair + 3 < p1) load(b1, pair + 3);
          }
        }

        // ---- the end of the wave's part of the segment
        halves();
        const float l = total_l();
        const bool begins = p0 == 0, ends = p1 == pairs;
        if (bad && lane == 0) atomicOr(a.err, (unsigned)PKV_DEVERR_PAGE_ID);
        if (begins && ends) {
          const float inv = bad || l == 0.0f ? 0.0f : 1.0f / l;
          if (col < G) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                h8v o;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const float y = st.acc[4 * half + (e & 3)][2 * j + (e >> 2)] * inv;
                  o[e] = (_Float16)(bad ? 0.0f : y);
                }
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
                    v4f{st.acc[4 * half][i], st.acc[4 * half + 1][i], st.acc[4 * half + 2][i], st.acc[4 * half + 3][i]};
            if (grp == 0) {
              part[G * D + 2 * col] = st.m;
              part[G * D + 2 * col + 1] = bad ? -1.0f : l;
            }
          }
          if (lane == 0) s.seg[at] = row * a.Hkv + head;
        }
      }
      // ---- on to the next segment
      u += n_units;
      off = 0;
      if (++head == a.Hkv) {
        head = 0;
        ++row;
        if (u < u_end) c_units = uniform(s.pre[row + 1] - s.pre[row]);
      }
    }
  }
  __syncthreads();

  // ---- states of segments that several waves share: runs of equal entries of s.seg
  if (wave == 0) {
    const int mine = lane < 2 * W ? s.seg[lane] : -1;
    const unsigned long long valid = __builtin_amdgcn_ballot_w64(mine >= 0);
    const unsigned long long below = valid & ((1ull << lane) - 1);
    const int prev = __shfl(mine, below ? 63 - __builtin_clzll(below) : 0);
    const unsigned long long starts = __builtin_amdgcn_ballot_w64(mine >= 0 && (!below || prev != mine));
    const int g = __popcll(starts & ((1ull << lane) - 1));
    if (starts >> lane & 1) {
      s.group_at[g] = lane;
      const unsigned long long next = lane < 63 ? starts >> (lane + 1) << (lane + 1) : 0;
      s.group_n[g] = (next ? __builtin_ctzll(next) : 2 * W) - lane;
    }
    if (lane == 0) {
      s.groups = __popcll(starts);
      s.last[0] = s.last[1] = 0;
    }
  }
  __syncthreads();
  const int cols = G * (D / 4);  // float4 columns of a state
  const int SB = slot * (int)sizeof(float);
  const __amdgpu_buffer_rsrc_t pr =
      __builtin_amdgcn_make_buffer_rsrc(a.partials, (short)0, 2 * kKv8MaxWorkgroups * SB, 0x00020000);
  // The workgroups that hold states of a segment: those of its first and its last pair.
  auto span = [&](int seg, int& first, int& last) {
    const int r = seg / a.Hkv, h = seg - r * a.Hkv;
    const int c = s.pre[r + 1] - s.pre[r];
    const int base = s.pre[r] * a.Hkv + h * c;
    first = wave_of(base) / W;
    last = wave_of(base + c - kSegment - 1) / W;
  };
  const int groups = uniform(s.groups);
  for (int it = tid; it < groups * cols; it += W * 64) {
    const int g = it / cols, e4 = it - g * cols, h = e4 / (D / 4);
    const int at = s.group_at[g], n = s.group_n[g];
    const int seg = s.seg[at];
    int first, last;
    span(seg, first, last);
    float M = kLowest, L = 0.0f;
    bool zero = false;
    for (int j = at; j < at + n; ++j) {
      if (s.seg[j] != seg) continue;
      const float* part = s.part + j * slot;
      M = fmaxf(M, part[G * D + 2 * h]);
      zero |= part[G * D + 2 * h + 1] < 0.0f;
    }
    v4f A = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int j = at; j < at + n; ++j) {
      if (s.seg[j] != seg) continue;
      const float* part = s.part + j * slot;
      const float c = ex2(part[G * D + 2 * h] - M);
      const v4f x = *reinterpret_cast<const v4f*>(part + 4 * e4);
      L = __builtin_fmaf(c, part[G * D + 2 * h + 1], L);
#pragma unroll
      for (int e = 0; e < 4; ++e) A[e] = __builtin_fmaf(c, x[e], A[e]);
    }
    if (first == last) {
      const float inv = zero || L == 0.0f ? 0.0f : 1.0f / L;
      uint16_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = zero ? 0 : __builtin_bit_cast(uint16_t, (_Float16)(A[e] * inv));
      *reinterpret_cast<v2u*>(a.out + (size_t)seg * G * D + 4 * e4) = __builtin_bit_cast(v2u, o);
    } else {
      const int so = (2 * blockIdx.x + (first == (int)blockIdx.x ? 1 : 0)) * SB;
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, A), pr, so + e4 * 16, 0, kSc1);
      if (e4 % (D / 4) == 0)
        __builtin_amdgcn_raw_buffer_store_b64(v2u{as_u32(M), as_u32(zero ? -1.0f : L)}, pr, so + (G * D + 2 * h) * 4, 0, kSc1);
    }
  }

  // ---- completion count of the (at most two) segments that cross into other workgroups
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (tid < groups) {
    const int seg = s.seg[s.group_at[tid]];
    int first, last;
    span(seg, first, last);
    if (first != last) {
      const int prev = __hip_atomic_fetch_add(&a.counters[seg], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (prev == last - first) {
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        s.last[first == (int)blockIdx.x ? 1 : 0] = seg + 1;
        a.counters[seg] = 0;
      }
    }
  }
  __syncthreads();

  for (int which = 0; which < 2; ++which) {
    const int seg = uniform(s.last[which]) - 1;
    if (seg < 0) continue;
    int first, last;
    span(seg, first, last);
    const int n = last - first + 1;
    auto slot_at = [&](int j) { return (2 * (first + j) + (j == 0 ? 1 : 0)) * SB; };
    float* wm = s.part;                          // [n][G] maxima, then weights
    float* wl = wm + kKv8MaxWorkgroups * kKv8MaxG;  // [n][G] sums
    for (int i = tid; i < n * G; i += W * 64) {
      const int j = i / G, h = i - j * G;
      const v2u ml = __builtin_amdgcn_raw_buffer_load_b64(pr, slot_at(j) + (G * D + 2 * h) * 4, 0, kSc1);
      wm[i] = as_f32(ml.x);
      wl[i] = as_f32(ml.y);
    }
    __syncthreads();
    float M = kLowest, L = 0.0f;
    bool zero = false;
    const int h = (tid % cols) / (D / 4), e4 = tid % cols, g = tid / cols, ng = W * 64 / cols;
    for (int j = 0; j < n; ++j) {
      M = fmaxf(M, wm[j * G + h]);
      zero |= wl[j * G + h] < 0.0f;
    }
    for (int j = 0; j < n; ++j) L = __builtin_fmaf(ex2(wm[j * G + h] - M), wl[j * G + h], L);
    v4f A = {0.0f, 0.0f, 0.0f, 0.0f};
    if (g < ng)
      for (int j = g; j < n; j += ng) {
        const v4f x = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(pr, slot_at(j) + e4 * 16, 0, kSc1));
        const float c = ex2(wm[j * G + h] - M);
#pragma unroll
        for (int e = 0; e < 4; ++e) A[e] = __builtin_fmaf(c, x[e], A[e]);
      }
    float* sums = wl + kKv8MaxWorkgroups * kKv8MaxG;  // [ng][G * D]
    if (g < ng) *reinterpret_cast<v4f*>(sums + (g * cols + e4) * 4) = A;
    __syncthreads();
    if (g == 0) {
      for (int j = 1; j < ng; ++j) A += *reinterpret_cast<const v4f*>(sums + (j * cols + e4) * 4);
      const float inv = zero || L == 0.0f ? 0.0f : 1.0f / L;
      uint16_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = zero ? 0 : __builtin_bit_cast(uint16_t, (_Float16)(A[e] * inv));
      *reinterpret_cast<v2u*>(a.out + (size_t)seg * G * D + 4 * e4) = __builtin_bit_cast(v2u, o);
    }
    __syncthreads();
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
  // One workgroup per compute unit, fewer when the block table cannot hold as many units of work.
  const long long most = (long long)a.B * a.Hkv * ((a.max_pages_per_row + 1) / 2 + kSegment);
  long long grid = (most + W - 1) / W;
  const int cap = device_units() < kKv8MaxWorkgroups ? device_units() : kKv8MaxWorkgroups;
  if (grid > cap) grid = cap;
  if (format == PKV_KV8_INT8) hipLaunchKernelGGL(kv8_decode_kernel<Int8>, dim3((unsigned)grid), dim3(W * 64), 0, s, a);
  else hipLaunchKernelGGL(kv8_decode_kernel<E4m3>, dim3((unsigned)grid), dim3(W * 64), 0, s, a);
  return hipGetLastError();
}

namespace {
unsigned move_grid(const Kv8MoveArgs& a) {
  const long long blocks = ((long long)a.tokens * a.Hkv + 15) / 16;
  return (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
}
}  // namespace

hipError_t launch_kv8_append(const Kv8MoveArgs& a, int format, hipStream_t s) {
  if (format == PKV_KV8_INT8) hipLaunchKernelGGL(append_kernel<Int8>, dim3(move_grid(a)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(append_kernel<E4m3>, dim3(move_grid(a)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv8_gather(const Kv8MoveArgs& a, int format, hipStream_t s) {
  if (format == PKV_KV8_INT8) hipLaunchKernelGGL(gather_kernel<Int8>, dim3(move_grid(a)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(gather_kernel<E4m3>, dim3(move_grid(a)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace pkv
