// A shared projection with the low-rank adapter of each row's request beside it:
//
//   out[n] = act( W x[n] + bias + B_a t[n] ),  t[n] = s_a A_a x[n],  a = ids[request of n]
//
// t comes first, in a launch of its own (every output column needs all of it).
#include "adapter.h"
#include "launch.h"

namespace rocs {
namespace {

__device__ __forceinline__ int64_t rows_of(const AdapterArgs& a) {
  return min(a.N, max((int64_t)a.off[a.R], (int64_t)0));
}

// Adapter of row n, -1: none.
__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int64_t n) {
  const int id = a.ids[owner_of(a.off, a.R, n)];
  return (uint32_t)id < (uint32_t)a.A ? id : -1;
}

// ---------------------------------------------------------------------------
// General path: any dtype, sizes and alignment; t in fp32.
// ---------------------------------------------------------------------------

// A wave a row: four of the row's rank at a time. Bound by the loads of A, from L2.
template <typename T>
__global__ __launch_bounds__(256) void shrink_general(const AdapterArgs a, int cols) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n_rows = rows_of(a);
  for (int64_t n = (int64_t)blockIdx.x * 4 + wave; n < n_rows; n += (int64_t)gridDim.x * 4) {
    const int id = adapter_of(a, n);
    if (id < 0) continue;
    const T* x = static_cast<const T*>(a.x) + n * a.x_stride;
    const T* w = static_cast<const T*>(a.a) + (int64_t)id * a.rank * a.K;
    const float s = a.scales != nullptr ? a.scales[id] : 1.f;
    float* t = static_cast<float*>(a.t) + n * cols;
    for (int j0 = 0; j0 < a.rank; j0 += 4) {
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      for (int k = lane; k < a.K; k += 64) {
        const float xv = load_f32(x + k);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum[i] += xv * load_f32(w + (int64_t)min(j0 + i, a.rank - 1) * a.K + k);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum[i] += __shfl_xor(sum[i], o);
        if (lane == 0 && j0 + i < a.rank) t[j0 + i] = s * sum[i];
      }
    }
  }
}

// A 16 x 16 tile (features x rows) a workgroup and step; its four waves split K and
// the rank, and add up through LDS in a fixed order. Products as in the general
// linear: the fp32 matrix instruction, operands from global memory, four
// consecutive k a lane. Bound by the latency of those loads: with t, 3,000 fp32 rows,
// 600 -> 600, rank 16, take 81 us (28 TFLOP/s), 203 of 101 -> 77, rank 5, 10.3.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void adapter_general(const AdapterArgs a, int cols, int tiles_m,
                                                       int64_t tiles) {
  __shared__ f32x4 red[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l = lane & 15, g = lane >> 4;
  const int64_t n_rows = rows_of(a);
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int d0 = (int)(tile % tiles_m) * 16;
    const int64_t n0 = tile / tiles_m * 16;
    if (n0 >= n_rows) return;              // the later tiles lie behind the rows as well
    const int d = d0 + l;
    const int64_t n = n0 + l;
    const bool dok = d < a.D, nok = n < n_rows;
    const T* x = static_cast<const T*>(a.x) + n * a.x_stride;
    const T* w = static_cast<const T*>(a.w) + (int64_t)d * a.K;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 16 * wave + 4 * g; k < (a.K + 15) / 16 * 16; k += 64) {
      const int left = a.K - k;
      const f32x4 av = load4_f32<T, VEC>(w + k, dok ? left : 0);
      const f32x4 bv = load4_f32<T, VEC>(x + k, nok ? left : 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(av[i], bv[i], acc, 0, 0, 0);
    }
    // Element i: feature d0 + 4 g + i of row n.
    const int id = nok ? adapter_of(a, n) : -1;
    if (id >= 0) {
      const T* b = static_cast<const T*>(a.b) + ((int64_t)id * a.D + d0 + 4 * g) * a.rank;
      const float* t = static_cast<const float*>(a.t) + n * cols;
      for (int j = wave; j < a.rank; j += 4) {
        const float tv = t[j];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (d0 + 4 * g + i < a.D) acc[i] += tv * load_f32(b + (int64_t)i * a.rank + j);
      }
    }
    red[wave][lane] = acc;
    __syncthreads();
    if (wave == 0 && nok) {
      f32x4 s = ((red[0][lane] + red[1][lane]) + red[2][lane]) + red[3][lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int df = d0 + 4 * g + i;
        if (df >= a.D) break;
        if (a.bias != nullptr) s[i] += a.bias[df];
        if (a.relu) s[i] = fmaxf(s[i], 0.f);
        static_cast<T*>(a.out)[n * a.D + df] = from_f32<T>(s[i]);
      }
    }
    __syncthreads();                       // red is free for the next tile
  }
}

// ---------------------------------------------------------------------------
// Fast path, first launch: t = s A x in bf16 (a rounding whose error is half a
// bf16 step of the adapter's part of the result, and lets its product with B run at
// the bf16 rate), and the rows' adapters.
//
// Requests of few rows: a workgroup takes 32 rows of one request (tiles as in common.h:
// tile_base) and all of the rank, 32 RK columns at a time; its eight waves split K,
// operands straight from global memory, and add up through LDS in a fixed order.
// Requests of many rows take the tiled linear (linear.hip: SHRINK). Bound by latency, one
// trip over K / 8: 128 rows of 48 adapters, K 1,024, rank 16: 5.1 us; 8 rows, K 256: 3.4.
// ---------------------------------------------------------------------------
template <int RK>
__global__ __launch_bounds__(512) void shrink_rows(const AdapterArgs a, const LowRank lr) {
  constexpr int U = 8 / RK;                    // steps of a wave in flight
  __shared__ f32x4 red[8][4][kWave];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const int r = request_of_slot(a.off, a.R, blockIdx.x, 1, 32);
  const int64_t end = min((int64_t)a.off[r + 1], a.N);
  const int64_t n0 = a.off[r] + ((int64_t)blockIdx.x - tile_base(a.off, r, 1, 32)) * 32;
  const int rows = (int)max(min(end - n0, (int64_t)32), (int64_t)0);
  if (rows == 0) return;
  const int given = a.ids[r], id = (uint32_t)given < (uint32_t)a.A ? given : -1;
  if (tid < rows) lr.aid[n0 + tid] = id;
  if (id < 0) return;
  const float scale = a.scales != nullptr ? a.scales[id] : 1.f;
  bf16_t* const t = const_cast<bf16_t*>(lr.t);
  const bf16_t* x = static_cast<const bf16_t*>(a.x) + (n0 + min(l32, rows - 1)) * a.x_stride + 8 * hh;
  for (int j0 = 0; j0 < a.rank; j0 += 32 * RK) {
    const bf16_t* w[RK];
#pragma unroll
    for (int k = 0; k < RK; ++k)
      w[k] = static_cast<const bf16_t*>(a.a) + ((int64_t)id * a.rank + min(j0 + 32 * k + l32, a.rank - 1)) * a.K + 8 * hh;
    f32x16 acc[RK];
#pragma unroll
    for (int k = 0; k < RK; ++k) acc[k] = f32x16{};
    // Step s of a wave: 16 k; four steps are a 128-byte line of each row.
    auto k_of = [&](int s) { return 512 * (s / 4) + 64 * wave + 16 * (s % 4); };
    for (int s = 0; k_of(s) < a.K; s += U) {
      u32x4 av[U][RK], xv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k_of(s + u);
        const bool ok = k + 8 * hh < a.K;
#pragma unroll
        for (int i = 0; i < RK; ++i) av[u][i] = load16(w[i] + k, ok);
        xv[u] = load16(x + k, ok);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k_of(s + u) >= a.K) break;
#pragma unroll
        for (int i = 0; i < RK; ++i) acc[i] = mfma32(as_bf16x8(av[u][i]), as_bf16x8(xv[u]), acc[i]);
      }
    }
    // Quad q of a block: columns 8 q + 4 hh .. + 3 of row l32.
#pragma unroll
    for (int i = 0; i < RK; ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        red[wave][q][lane] = f32x4{acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]};
      __syncthreads();
      if (tid < 256) {
        const int q = tid >> 6;
        f32x4 s = red[0][q][lane];
#pragma unroll
        for (int w8 = 1; w8 < 8; ++w8) s += red[w8][q][lane];
        const int j = j0 + 32 * i + 8 * q + 4 * hh;
        if (l32 < rows && j < a.rank)
          *reinterpret_cast<u32x2*>(t + (n0 + l32) * lr.cols + j) =
              u32x2{pack_bf16x2(s[0] * scale, s[1] * scale), pack_bf16x2(s[2] * scale, s[3] * scale)};
      }
      __syncthreads();
    }
  }
}

template <int RK>
hipError_t launch_shrink(const AdapterArgs& a, const LowRank& lr, hipStream_t s) {
  const int64_t slots = a.R + (a.N + 31) / 32;
  if (!grid_fits(slots, 512)) return hipErrorInvalidConfiguration;
  return launch_kernel(shrink_rows<RK>, dim3((uint32_t)slots), dim3(512), s, a, lr);
}

// ---------------------------------------------------------------------------
// Fast path, few rows: 32 features x 32 rows a workgroup, whose eight waves split K;
// then a wave adds the adapters of four of the rows, one after the other with t zero for
// all rows but its own of them, and a row keeps what is its own by a select. Operands come
// straight from global memory, partial sums are added up through LDS in a fixed order.
// Bound by latency: the first loads depend on nothing (rows up to num_rows are read; those
// behind the last request are dropped), and B's are issued before the first products.
// 128 rows of 48 adapters, 1,024 -> 1,536, rank 16: 7.9 us; 8 rows, 256 -> 512: 4.4 (of
// which 3 are an empty kernel's).
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(512) void adapter_few(const AdapterArgs a, const LowRank lr, int tiles_m) {
  constexpr int U = 8;                         // steps of a wave in flight
  __shared__ f32x4 red[8][4][kWave];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const int d0 = (int)(blockIdx.x % (uint32_t)tiles_m) * 32;
  const int64_t n0 = (int64_t)(blockIdx.x / (uint32_t)tiles_m) * 32;
  const int64_t n = min(n0 + l32, a.N - 1);
  const int d = min(d0 + l32, a.D - 1);
  int mine = adapter_at(lr, n);
  const int64_t n_rows = rows_of(a);
  const bf16_t* x = static_cast<const bf16_t*>(a.x) + n * a.x_stride + 8 * hh;
  const bf16_t* w = static_cast<const bf16_t*>(a.w) + (int64_t)d * a.K + 8 * hh;
  auto k_of = [&](int s) { return 512 * (s / 4) + 64 * wave + 16 * (s % 4); };
  u32x4 wv[U], xv[U];
  auto load_k = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k_of(s + u);
      const bool ok = k + 8 * hh < a.K;
      wv[u] = load16(w + k, ok);
      xv[u] = load16(x + k, ok);
    }
  };
  load_k(0);
  if (n0 >= n_rows) return;
  if (n0 + l32 >= n_rows) mine = -1;
  // Pair p of this wave: step p / 4 of the adapter of its row p % 4.
  constexpr int V = 4;                         // pairs in flight
  const int pairs = lr.cols / 16 * 4;
  int ids[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) ids[i] = __builtin_amdgcn_readlane(mine, 4 * wave + i);
  const bool in_wave = (l32 >> 2) == wave;
  const bf16_t* t = lr.t + n * lr.cols + 8 * hh;
  const bf16_t* b = lr.b + (int64_t)d * lr.rank + 8 * hh;
  u32x4 bv[V], tv[V];
  auto load_b = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int at = p0 / 4 * 16;
      const bool ok = ids[i] >= 0 && at + 8 * hh < lr.rank;
      bv[i] = load16(b + (int64_t)ids[i] * a.D * lr.rank + at, ok);
      tv[i] = load16(t + at, ok && in_wave && mine == ids[i]);
    }
  };
  static_assert(V == 4, "a pair of each row");
  load_b(0);
  f32x16 acc = {};
  for (int s = 0; k_of(s) < a.K; s += U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k_of(s + u) >= a.K) break;
      acc = mfma32(as_bf16x8(wv[u]), as_bf16x8(xv[u]), acc);
    }
    if (k_of(s + U) < a.K) load_k(s + U);
  }
  for (int p0 = 0; p0 < pairs; p0 += V) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bool again = ids[i] < 0;                 // none, or a row before it has the same
#pragma unroll
      for (int e = 0; e < i; ++e) again = again || ids[e] == ids[i];
      if (again) continue;
      const f32x16 y = mfma32(as_bf16x8(bv[i]), as_bf16x8(tv[i]), acc);
      const bool own = in_wave && mine == ids[i];
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] = own ? y[e] : acc[e];
    }
    if (p0 + V < pairs) load_b(p0 + V);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    red[wave][q][lane] = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
  __syncthreads();
  if (wave >= 4) return;
  // Quad `wave`: features 8 wave + 4 hh .. + 3 of row l32.
  f32x4 s = red[0][wave][lane];
#pragma unroll
  for (int i = 1; i < 8; ++i) s += red[i][wave][lane];
  const int df = d0 + 8 * wave + 4 * hh;
  if (n0 + l32 >= n_rows || df >= a.D) return;
  if (a.bias != nullptr)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += a.bias[df + i];
  const uint32_t lo = act_floor(a.relu);
  *reinterpret_cast<u32x2*>(static_cast<bf16_t*>(a.out) + n * a.D + df) =
      u32x2{act_bf16x2(pack_bf16x2(s[0], s[1]), lo), act_bf16x2(pack_bf16x2(s[2], s[3]), lo)};
}

hipError_t launch_few(const AdapterArgs& a, const LowRank& lr, hipStream_t s) {
  const int tiles_m = (a.D + 31) / 32;
  const int64_t blocks = (a.N + 31) / 32 * tiles_m;
  if (!grid_fits(blocks, 512)) return hipErrorInvalidConfiguration;
  return launch_kernel(adapter_few, dim3((uint32_t)blocks), dim3(512), s, a, lr, tiles_m);
}

template <typename T>
hipError_t launch_general(const AdapterArgs& a, hipStream_t s) {
  const int cols = adapter_cols(a.rank);
  if (a.A > 0) {
    const int64_t blocks = (a.N + 3) / 4 < (1 << 20) ? (a.N + 3) / 4 : 1 << 20;
    const hipError_t e = launch_kernel(shrink_general<T>, dim3((uint32_t)blocks), dim3(256), s, a, cols);
    if (e != hipSuccess) return e;
  }
  const int tiles_m = (a.D + 15) / 16;
  const int64_t tiles = (a.N + 15) / 16 * tiles_m;
  const uint32_t grid = (uint32_t)(tiles < (1 << 20) ? tiles : 1 << 20);
  auto ok = [](const void* p, int64_t stride) {
    return stride % 4 == 0 && reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0;
  };
  const bool vec = a.K % 4 == 0 && ok(a.x, a.x_stride) && ok(a.w, 0);
  return launch_kernel(vec ? adapter_general<T, true> : adapter_general<T, false>, dim3(grid),
                       dim3(256), s, a, cols, tiles_m, tiles);
}

}  // namespace

hipError_t launch_adapter(const AdapterArgs& a, bool fast, hipStream_t s) {
  if (!fast) return a.bf16 ? launch_general<bf16_t>(a, s) : launch_general<float>(a, s);
  bf16_t* t = static_cast<bf16_t*>(a.t);
  int32_t* aid = reinterpret_cast<int32_t*>(static_cast<char*>(a.t) + adapter_t_bytes(a.N, a.rank));
  const LowRank lr{t, static_cast<const bf16_t*>(a.b), aid, a.off, a.x_stride, adapter_cols(a.rank), a.rank,
                   a.A, a.R};
  // The tiled linear for t pays where its tiles fill and there are enough of them (the
  // whole call in us, shrink_rows / tiled; K x D, rank): 9,001 rows of 24 requests,
  // 1,024 x 1,536, 32: 45 / 41; 32,768 of 16, 2,048 x 2,048, 64: 316 / 285; 8,000 of 400,
  // 1,024 x 1,024, 64: 59 / 51; 1,024 of 64, 64: 24 / 22; but 4,096 of 256, 16: 29 / 30; 2,048 of
  // 128, 32: 30 / 32; 8,000 of 1,000, 16: 49 / 51. A grid of shrink_rows holds whatever the limits allow.
  const bool tiled = a.N / a.R >= 16 && a.N >= (a.rank > 32 ? 1024 : 8000) && adapter_shrink_fits(a);
  const hipError_t e = tiled          ? launch_adapter_shrink(a, lr, s)
                       : a.rank > 32 ? launch_shrink<2>(a, lr, s)
                                     : launch_shrink<1>(a, lr, s);
  if (e != hipSuccess) return e;
  // Few tiles of the linear leave CUs idle, and its K is one chain; single events of many
  // adapters also make its blocks of 32 rows take them one after the other. In us, linear /
  // adapter_few: 128 rows, 1,024 x 1,024, rank 16, one adapter 16.7 / 15.4, a row each of 30
  // 20.7 / 13.2 (32 tiles); 192 rows, 1,024 x 2,048 (96 tiles), 17.5 / 20.7, a row each of 8
  // 16.6 / 18.6, of 64 23.6 / 19.3; 256 rows, 2,048 x 2,048, rank 64, of 64 (128 tiles) 71 / 53; 512 rows,
  // rank 16, of 64 (256 tiles) 34 / 51. (Both rules go by averages: 127 single rows of 64 adapters and a
  // chunk of 4,000, 1,024 x 1,536, rank 16, take 58 as one call, 12 + 31 as two.)
  const int64_t tiles = (int64_t)((a.N + 63) / 64) * ((a.D + 63) / 64);
  const bool few = tiles <= 64 || (tiles <= 128 && a.N < 4 * (int64_t)a.R && a.A >= 16);
  return few ? launch_few(a, lr, s) : launch_adapter_gemm(a, lr, s);
}

}  // namespace rocs
