// Internal interface of the adapter linear, the rotated append and the
// attention over a cache in 4 bits.
#pragma once

#include "history.h"

namespace rocs {

// ---------------------------------------------------------------------------
// A row of the 4-bit form: [K values | V values | K scales | V scales], padded
// to 16 bytes. Offsets in bytes; `v` 0: K, 1: V.
// ---------------------------------------------------------------------------
constexpr int kFp4Block = 32;             // values of a scale

struct Fp4Row {
  int Hk, D;
  __host__ __device__ int values(int v, int h) const { return (v * Hk + h) * (D / 2); }
  __host__ __device__ int scales(int v, int h) const { return Hk * D + (v * Hk + h) * (D / kFp4Block); }
  __host__ __device__ int64_t bytes() const {
    return ((int64_t)Hk * D + (int64_t)Hk * (D / 16) + 15) / 16 * 16;
  }
};

// The rows of new events, or of queries alone (k NULL).
struct AppendArgs {
  const void* q;            // [M, H, D] or NULL
  const void* k;            // [M, Hk, D] or NULL
  const void* v;
  void* q_out;              // [M, H, D]
  void* pool;
  const int32_t* rows;      // [M], with k
  const float* freqs;       // [half]
  const int32_t* positions; // [M], or
  const int32_t* off;       // [R + 1]
  const int32_t* slots;     // [R] or NULL
  const int32_t* lens;      // [S]
  int64_t M, q_stride, kv_stride, pool_rows;
  int R, S, H, Hk, D, half, interleaved;
  int bf16, fp4;
};
hipError_t launch_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_read_fp4(const int32_t* rows, int64_t M, const void* pool, int64_t pool_rows,
                           int Hk, int D, bool bf16, void* out, hipStream_t s);

struct AdapterArgs {
  const void* x;
  const void* w;            // [D, K]
  const void* a;            // [A, rank, K]
  const void* b;            // [A, D, rank]
  const float* scales;      // [A] or NULL
  const float* bias;        // [D] or NULL
  const int32_t* off;       // [R + 1]
  const int32_t* ids;       // [R]
  void* out;
  void* t;                  // workspace: s A x of every row, [N, adapter_cols(rank)]
  int64_t N, x_stride;
  int R, K, D, rank, A;
  int bf16, relu;
};
// Columns of a row of t: whole steps of the matrix instruction.
inline int adapter_cols(int rank) { return (rank + 15) / 16 * 16; }
hipError_t launch_adapter(const AdapterArgs& a, bool fast, hipStream_t s);

// What the fast path's product reads beside x and W.
struct LowRank {
  const __bf16* t;          // [N, cols]: s A x, rounded; nothing from rank on
  const __bf16* b;          // [A, D, rank]
  int32_t* aid;             // [N] each row's adapter, or -1
  const int32_t* off;       // [R + 1]
  int64_t x_stride;
  int cols, rank, adapters, R;
};
// Whether the tiled kernel's grid, which grows with the rank, holds the call.
bool adapter_shrink_fits(const AdapterArgs& a);
hipError_t launch_adapter_shrink(const AdapterArgs& a, const LowRank& lr, hipStream_t s);
hipError_t launch_adapter_gemm(const AdapterArgs& a, const LowRank& lr, hipStream_t s);
// Bytes of t in the workspace; the rows' adapters [N] lie behind them on the fast path.
inline size_t adapter_t_bytes(int64_t N, int rank) { return ((size_t)N * adapter_cols(rank) * 4 + 255) & ~size_t(255); }

// Attention over a 4-bit pool: HistArgs with k = the pool, kv_stride = bytes of
// a row and page_stride = bytes of a page.
HistPlan fp4_plan(int64_t R, int64_t N, int H, int Hk, int D, int64_t max_len, bool bf16);
hipError_t launch_history_fp4(const HistArgs& a, int rows, bool bf16, bool fast, hipStream_t s);
hipError_t launch_history_fp4_few(const HistArgs& a, hipStream_t s);
hipError_t launch_history_fp4_tile(const HistArgs& a, hipStream_t s);

}  // namespace rocs
