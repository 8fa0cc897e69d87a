// Internal interface of the 8-bit paged KV cache: between its C ABI (pkv_kv8_capi.cpp) and its
// kernels (pkv_kv8.hip).
#pragma once

#include "pkv_internal.h"

namespace pkv {

// One record per (page, KV head): K codes [16][128], V codes [4][128][4] (token 4a + b of dim c at
// [a][c][b]), K scales fp32 [16], V scales fp32 [16]. 33 lines of 128 bytes.
constexpr int kKv8CodeBytes = kPageSize * kHeadDim;
constexpr int kKv8ScaleAt = 2 * kKv8CodeBytes;
constexpr int kKv8Record = kKv8ScaleAt + 2 * kPageSize * 4;
constexpr int kKv8MaxG = 8;             // query heads per KV head
constexpr int kKv8MaxWorkgroups = 512;  // of an attention launch: two state slots each in the workspace

struct Kv8DecodeArgs {
  const uint16_t* q;
  const uint8_t* cache;
  const int32_t* block_table;
  const int32_t* seq_lens;
  uint16_t* out;
  unsigned* err;
  int32_t* counters;
  float* partials;
  int64_t q_stride;  // halves between rows of q
  int32_t num_pages, max_pages_per_row;
  int32_t B, Hq, Hkv, G;
  float scale_log2;  // sm_scale * log2(e)
};

// Append (x is read) and gather (x is written).
struct Kv8MoveArgs {
  uint16_t* k;
  uint16_t* v;
  uint8_t* cache;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const int32_t* offsets;  // null: one token per row
  unsigned* err;
  int64_t k_stride, v_stride;  // halves between tokens
  int32_t tokens, num_pages, max_pages_per_row, B, Hkv;
};

hipError_t launch_kv8_decode(const Kv8DecodeArgs& a, int format, hipStream_t s);
hipError_t launch_kv8_append(const Kv8MoveArgs& a, int format, hipStream_t s);
hipError_t launch_kv8_gather(const Kv8MoveArgs& a, int format, hipStream_t s);

}  // namespace pkv
