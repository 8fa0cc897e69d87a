// C ABI of the 8-bit paged KV cache: argument validation. Every check runs on the host before
// anything is enqueued.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdint>
#include <cstring>

#include "pkv_kv8.h"

using namespace pkv;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int from_hip(hipError_t e) { return e == hipSuccess ? PKV_OK : PKV_ERR_HIP; }

// Pool, block table, lengths and workspace: what every call has.
int check_cache(const void* cache, int32_t num_pages, const int32_t* bt, int32_t maxp, const int32_t* seq_lens,
                int32_t B, int32_t Hkv, int32_t d, int32_t format, const void* ws) {
  if (!cache || !bt || !seq_lens || !ws) return PKV_ERR_INVALID_ARG;
  if (B < 1 || Hkv < 1 || num_pages < 1 || maxp < 1) return PKV_ERR_INVALID_ARG;
  if (!aligned(cache, 16) || !aligned(ws, 16) || !aligned(bt, 4) || !aligned(seq_lens, 4)) return PKV_ERR_INVALID_ARG;
  if (d != kHeadDim || (format != PKV_KV8_INT8 && format != PKV_KV8_E4M3)) return PKV_ERR_UNSUPPORTED;
  if ((int64_t)maxp * kPageSize > INT32_MAX) return PKV_ERR_INVALID_ARG;
  return PKV_OK;
}

// State slots of an attention call, whatever its lengths.
size_t slots_bytes(int G) { return (size_t)2 * kKv8MaxWorkgroups * slot_floats(G) * sizeof(float); }

// A strided [tokens, heads, d] fp16 operand: rows of `heads * d` halves, 16-byte aligned.
int check_rows(const void* p, int64_t stride, int64_t heads, int32_t d) {
  if (!p || !aligned(p, 16) || stride < heads * d || stride % 8 != 0) return PKV_ERR_INVALID_ARG;
  return PKV_OK;
}

int move_args(uint16_t* k, uint16_t* v, int64_t k_stride, int64_t v_stride, const int32_t* offsets, int32_t tokens,
              void* cache, int32_t num_pages, const int32_t* bt, int32_t maxp, const int32_t* seq_lens, int32_t B,
              int32_t Hkv, int32_t d, int32_t format, void* ws, size_t ws_bytes, Kv8MoveArgs* a) {
  int st = check_cache(cache, num_pages, bt, maxp, seq_lens, B, Hkv, d, format, ws);
  if (st != PKV_OK) return st;
  if (tokens < 0 || (!offsets && tokens != B) || !aligned(offsets, 4)) return PKV_ERR_INVALID_ARG;
  if (tokens > 0 && ((st = check_rows(k, k_stride, Hkv, d)) != PKV_OK || (st = check_rows(v, v_stride, Hkv, d)) != PKV_OK))
    return st;
  if (ws_bytes < kWsHeaderBytes) return PKV_ERR_WORKSPACE;
  *a = Kv8MoveArgs{k, v, static_cast<uint8_t*>(cache), bt, seq_lens, offsets, static_cast<unsigned*>(ws), k_stride, v_stride,
                   tokens, num_pages, maxp, B, Hkv};
  return PKV_OK;
}

}  // namespace

extern "C" {

size_t pkv_kv8_record_bytes(int32_t d) { return d == kHeadDim ? (size_t)kKv8Record : 0; }

size_t pkv_kv8_workspace_size(int32_t B, int32_t Hq, int32_t Hkv, int32_t d) {
  if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || Hq / Hkv > kKv8MaxG || d != kHeadDim) return 0;
  if ((int64_t)B * Hkv > INT32_MAX) return 0;
  return partials_offset(B, Hkv) + slots_bytes(Hq / Hkv);
}

int pkv_kv8_append(const uint16_t* k, const uint16_t* v, int64_t k_stride, int64_t v_stride, const int32_t* offsets,
                   int32_t tokens, void* cache, int32_t num_pages, const int32_t* block_table,
                   int32_t max_pages_per_row, const int32_t* seq_lens, int32_t B, int32_t Hkv, int32_t d,
                   int32_t format, void* ws, size_t ws_bytes, hipStream_t stream) {
  Kv8MoveArgs a;
  const int st = move_args(const_cast<uint16_t*>(k), const_cast<uint16_t*>(v), k_stride, v_stride, offsets, tokens, cache,
                           num_pages, block_table, max_pages_per_row, seq_lens, B, Hkv, d, format, ws, ws_bytes, &a);
  if (st != PKV_OK || tokens == 0) return st;
  return from_hip(launch_kv8_append(a, format, stream));
}

int pkv_kv8_gather(const void* cache, int32_t num_pages, const int32_t* block_table, int32_t max_pages_per_row,
                   const int32_t* seq_lens, const int32_t* offsets, int32_t tokens, int32_t B, int32_t Hkv, int32_t d,
                   int32_t format, uint16_t* k, uint16_t* v, int64_t k_stride, int64_t v_stride, void* ws,
                   size_t ws_bytes, hipStream_t stream) {
  Kv8MoveArgs a;
  const int st = move_args(k, v, k_stride, v_stride, offsets, tokens, const_cast<void*>(cache), num_pages, block_table,
                           max_pages_per_row, seq_lens, B, Hkv, d, format, ws, ws_bytes, &a);
  if (st != PKV_OK || tokens == 0) return st;
  return from_hip(launch_kv8_gather(a, format, stream));
}

int pkv_kv8_decode(const uint16_t* q, int64_t q_stride, const void* cache, int32_t num_pages,
                   const int32_t* block_table, int32_t max_pages_per_row, const int32_t* seq_lens, int32_t B,
                   int32_t Hq, int32_t Hkv, int32_t d, int32_t format, float sm_scale, uint16_t* out, void* ws,
                   size_t ws_bytes, hipStream_t stream) {
  int st = check_cache(cache, num_pages, block_table, max_pages_per_row, seq_lens, B, Hkv, d, format, ws);
  if (st != PKV_OK) return st;
  if (Hq < 1 || Hq % Hkv != 0) return PKV_ERR_INVALID_ARG;
  if (Hq / Hkv > kKv8MaxG || B > kMaxPlanBatch) return PKV_ERR_UNSUPPORTED;
  if ((st = check_rows(q, q_stride, Hq, d)) != PKV_OK) return st;
  if (!out || !aligned(out, 16) || !std::isfinite(sm_scale)) return PKV_ERR_INVALID_ARG;
  if (ws_bytes < pkv_kv8_workspace_size(B, Hq, Hkv, d)) return PKV_ERR_WORKSPACE;
  // units of work (page pairs) are numbered in 32 bits
  if ((int64_t)Hkv * B > INT32_MAX || (int64_t)Hkv * B * ((int64_t)max_pages_per_row / 2 + 2) > INT32_MAX) return PKV_ERR_UNSUPPORTED;
  char* w = static_cast<char*>(ws);
  Kv8DecodeArgs a;
  std::memset(&a, 0, sizeof(a));
  a.G = Hq / Hkv;
  a.q = q;
  a.cache = static_cast<const uint8_t*>(cache);
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.out = out;
  a.err = reinterpret_cast<unsigned*>(w);
  a.counters = reinterpret_cast<int32_t*>(w + kWsHeaderBytes);
  // The slots are the workspace's end, so that no batch's slots lie on the counters of one with more rows.
  a.partials = reinterpret_cast<float*>(w + (ws_bytes - slots_bytes(a.G)) / 256 * 256);
  a.q_stride = q_stride;
  a.num_pages = num_pages;
  a.max_pages_per_row = max_pages_per_row;
  a.B = B;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.scale_log2 = (float)((double)sm_scale * 1.4426950408889634);  // log2(e)
  return from_hip(launch_kv8_decode(a, format, stream));
}

}  // extern "C"
