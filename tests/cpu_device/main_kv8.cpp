// One call of the 8-bit cache through the C ABI on the CPU. argv[1]: a file with the request header
// (below), then arrays; argv[2]: where the answer goes.
#include "hip/hip_runtime.h"
#undef asm
#undef volatile
#include <sys/mman.h>

#include "pkv_kv8.h"

namespace {

struct Request {
  int32_t what, order, compute_units, calls;  // what: 0 append, 1 gather, 2 decode
  int32_t B, hq, hkv, num_pages, max_pages, format, tokens, has_offsets;
  int32_t k_stride, v_stride, q_stride, workspace_rows;  // of a batch that the workspace is for (0: this one)
  int32_t last_workgroup;
  float sm_scale;
};

// Memory between unmapped pages, so that an access past it ends the program.
char* guarded(size_t bytes) {
  const size_t page = 4096, n = (bytes + page - 1) / page * page;
  char* m = (char*)mmap(nullptr, n + 2 * page, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
  if (m == MAP_FAILED || mprotect(m + page, n, PROT_READ | PROT_WRITE) != 0) std::abort();
  return m + page + (n - (bytes + 15) / 16 * 16);
}
template <typename T>
T* read(FILE* f, size_t count) {
  T* p = (T*)guarded(count * sizeof(T));
  if (std::fread(p, sizeof(T), count, f) != count) std::abort();
  return p;
}

}  // namespace

int main(int argc, char** argv) {
  if (argc != 3) return 2;
  FILE* f = std::fopen(argv[1], "rb");
  Request r;
  if (!f || std::fread(&r, sizeof(r), 1, f) != 1) return 2;
  emu::order = (unsigned)r.order;
  emu::compute_units = r.compute_units;
  emu::last_workgroup = r.last_workgroup;
  const size_t pool = (size_t)r.num_pages * r.hkv * pkv_kv8_record_bytes(128), qn = (size_t)r.B * r.hq * 128;
  uint8_t* cache = read<uint8_t>(f, pool);
  int32_t *table = read<int32_t>(f, (size_t)r.B * r.max_pages), *lens = read<int32_t>(f, r.B);
  const size_t rows = (size_t)r.tokens;
  uint16_t *k = nullptr, *v = nullptr, *q = nullptr;
  // the last row ends after its heads, not after its stride
  if (r.what == 2) q = read<uint16_t>(f, (size_t)(r.B - 1) * r.q_stride + r.hq * 128);
  else if (rows > 0) {
    k = read<uint16_t>(f, (rows - 1) * r.k_stride + r.hkv * 128);
    v = read<uint16_t>(f, (rows - 1) * r.v_stride + r.hkv * 128);
  }
  int32_t* offsets = r.has_offsets ? read<int32_t>(f, r.B + 1) : nullptr;
  const int ws_rows = r.workspace_rows > 0 ? r.workspace_rows : r.B;
  const size_t ws_bytes = pkv_kv8_workspace_size(ws_rows, r.hq, r.hkv, 128);
  char* ws = guarded(ws_bytes);
  std::memset(ws, 0xFF, ws_bytes);
  uint16_t* out = (uint16_t*)guarded(2 * qn);
  FILE* g = std::fopen(argv[2], "wb");
  if (!g || pkv_workspace_init(ws, ws_bytes, ws_rows, r.hkv, nullptr) != PKV_OK) return 2;
  for (int c = 0; c < r.calls; ++c) {
    std::memset(out, 0xFF, 2 * qn);
    int st;
    if (r.what == 0)
      st = pkv_kv8_append(k, v, r.k_stride, r.v_stride, offsets, r.tokens, cache, r.num_pages, table, r.max_pages, lens, r.B,
                          r.hkv, 128, r.format, ws, ws_bytes, nullptr);
    else if (r.what == 1)
      st = pkv_kv8_gather(cache, r.num_pages, table, r.max_pages, lens, offsets, r.tokens, r.B, r.hkv, 128, r.format, k, v,
                          r.k_stride, r.v_stride, ws, ws_bytes, nullptr);
    else
      st = pkv_kv8_decode(q, r.q_stride, cache, r.num_pages, table, r.max_pages, lens, r.B, r.hq, r.hkv, 128, r.format,
                          r.sm_scale, out, ws, ws_bytes, nullptr);
    uint32_t bits = 0;
    int32_t left = 0;  // completion counters that are not zero
    for (int i = 0; i < ws_rows * r.hkv; ++i) left += reinterpret_cast<int32_t*>(ws + pkv::kWsHeaderBytes)[i] != 0;
    pkv_check_device_status(ws, nullptr, &bits);
    int32_t head[3] = {st, (int32_t)bits, left};
    std::fwrite(head, 4, 3, g);
    if (r.what == 0) std::fwrite(cache, 1, pool, g);
    else if (r.what == 2) std::fwrite(out, 2, qn, g);
    else if (rows > 0) {
      std::fwrite(k, 2, (rows - 1) * r.k_stride + r.hkv * 128, g);
      std::fwrite(v, 2, (rows - 1) * r.v_stride + r.hkv * 128, g);
    }
  }
  return std::fclose(g) == 0 ? 0 : 2;
}
