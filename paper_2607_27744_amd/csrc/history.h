// Internal interface of the history attention and the cache's page operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rocs {

// One call of history attention (packed: kv_off) or paged attention (table).
struct HistArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  const int32_t* q_off;     // [R + 1]
  const int32_t* kv_off;    // [R + 1], packed
  const int32_t* table;     // [S, width], paged
  const int32_t* lens;      // [S]
  const int32_t* slots;     // [R] or NULL
  const int32_t* prefix;    // [R] or NULL
  const int32_t* q_docs;    // [N] or NULL
  const int32_t* kv_docs;
  const float* slopes;      // [H] or NULL
  int64_t N, q_stride, kv_stride, page_stride;   // strides in elements
  int64_t width, pages;     // table columns, pages in the cache
  int R, S, H, Hk, G, D, page_size;              // G = H / Hk
  uint32_t page_magic;      // 2^32 / (page_size / 16) + 1 (MFMA kernels); for a 4-bit
  int page_shift;           // pool see set_page_divisor
  float scale, cap;
  int causal;
  int64_t max_len;          // bound on a history's length
  // History split over workgroups: `splits` chunks of `chunk` keys; partial
  // results per (split, row, head): {max (log2 units), sum} and the sums.
  int splits, chunk;
  int heads;                // K/V heads a workgroup of the 32-row kernel: 1, 2 or 4
  int deal;                 // 128-row kernel: XCDs that a head's tiles are dealt to, or 1
  float* part_ml;           // [splits][N * H][2]
  float* part_o;            // [splits][N * H][D]
};

// How a call is cut up: a rule on sizes only, so that the workspace size
// follows from them.
struct HistPlan {
  int rows;                 // query rows a workgroup: 128, 32 (MFMA) or 16 (general)
  int splits, chunk, heads;
  size_t ml_bytes, o_bytes; // of the workspace, 256-byte aligned
};
HistPlan history_plan(int64_t R, int64_t N, int H, int Hk, int D, int64_t max_len, bool bf16);
hipError_t launch_history_tile(const HistArgs& a, hipStream_t s);
hipError_t launch_history_split(const HistArgs& a, hipStream_t s);
hipError_t launch_history(const HistArgs& a, int rows, bool bf16, bool fast, hipStream_t s);

hipError_t launch_reserve(const int32_t* slots, const int32_t* row_off, int64_t n, int64_t M,
                          int32_t* table, int64_t width, int32_t* lens, int64_t S, int32_t* refs,
                          int64_t P, int page, int32_t* rows, int32_t* status, int32_t* ws,
                          hipStream_t s);
hipError_t launch_cache_write(const void* x, int64_t x_stride, const int32_t* rows, int64_t M,
                              void* pool, int64_t pool_rows, int64_t row_bytes, hipStream_t s);
hipError_t launch_fork(const int32_t* parents, const int32_t* children, int64_t n, int32_t* table,
                       int64_t width, int32_t* lens, int64_t S, int32_t* refs, int64_t P,
                       int page, void* pool, int64_t layers, int64_t row_bytes, int32_t* status,
                       int32_t* ws, hipStream_t s);
hipError_t launch_free(const int32_t* slots, int64_t n, int32_t* table, int64_t width,
                       int32_t* lens, int64_t S, int32_t* refs, int64_t P, int page,
                       hipStream_t s);
hipError_t launch_compact(int32_t* table, int64_t width, int64_t S, int32_t* refs, int64_t P,
                          void* pool, int64_t layers, int64_t page_bytes, int32_t* status,
                          int32_t* ws, hipStream_t s);
hipError_t launch_cache_copy(const int32_t* src, const int32_t* dst, int64_t n,
                             const void* src_pool, int64_t src_pages, void* dst_pool,
                             int64_t dst_pages, int64_t layers, int64_t page_bytes,
                             hipStream_t s);

}  // namespace rocs
