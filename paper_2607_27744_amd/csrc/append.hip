// New rows into a cache's pages with the position rotation on the way, and
// rows of a 4-bit cache read back.
//
// A workgroup takes RB rows: first the rows' positions (the request found by a
// search that the whole wave makes) and the cosines and sines of their angles
// into LDS, once for all heads; then its threads walk the rows' pieces of 8
// dims, query heads, K heads, V heads. The angle p f is formed and reduced to one
// turn in 64 bits (a position of 2^20 leaves an fp32 product 0.06 rad off). A piece's partner dims (the next
// one, or rot_dim / 2 away) are read again by the piece that holds them: the
// second read is from cache. In 4 bits four pieces are a block; their maximum
// goes over four lanes.
// A turned value is one fp32 value whatever the path: cosine and sine formed in 64
// bits and rounded once, products and their sum rounded each (no multiply-add), so
// that a row gets the same codes in 4 bits in every layout of the call.
// What bounds it: HBM where rows are many: 32,771 rows, 8 query and 8 + 8 heads x 128,
// into 4 bits: 73 to 83 us by the card, 3.7 to 4.2 TB/s of the rows' bytes in and out (a large
// copy: 5.2); 12,007 rows, 16 + 4 + 4 heads x 64, in bf16 16.1 us, in fp32 34 (4.3 TB/s). A thread
// keeps its piece of a head over the workgroup's rows: where that took 83 us, walking them two
// or four at a time took 87, four pieces in flight a thread 96, sixteen rows 101. For
// single events the launch and the chain lens -> position -> angle: 128 rows 4.8 us.
#include "fp4.h"
#include "launch.h"

namespace rocs {
namespace {

constexpr int kMaxHalf = 128;             // rotated pairs of a head
constexpr int kMaxRb = 8;                 // rows of a workgroup

// Eight elements of a row, zeros past n.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int n, float (&x)[8]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 2) {
      const u32x4 b = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(b[i]);
        x[2 * i + 1] = bf16_hi(b[i]);
      }
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = a[i];
        x[4 + i] = b[i];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? load_f32(p + i) : 0.f;
  }
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, int n, const float (&x)[8]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                           pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    } else {
      *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_f32<T>(x[i]);
  }
}

// The request that owns row m < off[R]: the last r with off[r] <= m. Every lane
// of the wave takes part; m is wave-uniform.
__device__ __forceinline__ int owner_wave(const int32_t* off, int R, int64_t m) {
  const int lane = (int)(threadIdx.x & 63);
  int lo = 0, n = R;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int r = lo + min(lane * step, n - 1);
    const bool ok = lane * step < n && (int64_t)off[r] <= m;
    const uint64_t mask = __ballot(ok) | 1;
    const int k = 63 - __builtin_clzll(mask);
    lo += k * step;
    n = min(step, n - k * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Eight dims from d0 of a head, turned. cs: {cos, sin} of the row's pairs.
template <typename T, bool VEC>
__device__ __forceinline__ void turned(const T* head, int d0, int D, int half, int interleaved,
                                       const float2* cs, float (&x)[8]) {
#pragma clang fp contract(off)
  const int n = min(D - d0, 8);
  load8<T, VEC>(head + d0, n, x);
  const int rot = 2 * half;
  if (d0 >= rot) return;
  if (interleaved) {                      // rot is even: a pair is whole or none
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if (d0 + i >= rot) break;
      const float2 t = cs[(d0 + i) / 2];
      const float a = x[i], b = x[i + 1];
      x[i] = a * t.x - b * t.y;
      x[i + 1] = a * t.y + b * t.x;
    }
    return;
  }
  // Vector pieces lie on one side of the border (half is a multiple of 8 there).
  if constexpr (VEC) {
    const bool low = d0 < half;
    float y[8];
    load8<T, true>(head + (low ? d0 + half : d0 - half), 8, y);
    const float2* c = cs + (low ? d0 : d0 - half);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 t = c[i];
      x[i] = low ? x[i] * t.x - y[i] * t.y : y[i] * t.y + x[i] * t.x;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = d0 + i;
      if (d >= rot || d >= D) break;
      const bool low = d < half;
      const float y = load_f32(head + (low ? d + half : d - half));
      const float2 t = cs[low ? d : d - half];
      x[i] = low ? x[i] * t.x - y * t.y : y * t.y + x[i] * t.x;
    }
  }
}

template <typename T, bool VEC, bool FP4>
__global__ __launch_bounds__(256) void append_rows(const AppendArgs a, int rb) {
  __shared__ float2 cs[kMaxRb][kMaxHalf];
  __shared__ int64_t place[kMaxRb];       // pool row, or -1: K and V are passed over
  __shared__ int known[kMaxRb];           // the row is a request's
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t m0 = (int64_t)blockIdx.x * rb;
  for (int i = wave; i < rb; i += 4) {
    const int64_t m = m0 + i;
    bool ok = m < a.M;
    int64_t pos = 0;
    if (ok && a.positions != nullptr) {
      pos = a.positions[m];
      if (a.off != nullptr) ok = m < a.off[a.R];
    } else if (ok && a.off != nullptr) {
      ok = m < a.off[a.R];
      if (ok) {
        const int r = owner_wave(a.off, a.R, m);
        if (a.lens != nullptr) {
          const int s = (int)min((uint32_t)(a.slots != nullptr ? a.slots[r] : r), (uint32_t)(a.S - 1));
          pos = (int64_t)a.lens[s] - a.off[r + 1] + m;
        }
      }
    }
    for (int p = lane; ok && p < a.half; p += 64) {
      // One turn is 2 pi: t / pi = 2 (u - round u) with u = p f / (2 pi).
      const double u = (double)pos * (double)a.freqs[p] * 0.15915494309189533577;
      double sn, c;
      sincospi(2.0 * (u - rint(u)), &sn, &c);
      cs[i][p] = make_float2((float)c, (float)sn);
    }
    if (lane == 0) {
      known[i] = ok;
      int64_t at = -1;
      if (ok && a.k != nullptr) {
        at = a.rows[m];
        if (at >= a.pool_rows) at = -1;
      }
      place[i] = at;
    }
  }
  __syncthreads();
  const int D = a.D, H = a.H, Hk = a.Hk;
  const int pieces = (D + 7) / 8;
  const int heads = (a.q != nullptr ? H : 0) + (a.k != nullptr ? 2 * Hk : 0);
  const int qh = a.q != nullptr ? H : 0;
  const Fp4Row fr{Hk, D};
  // A thread keeps its piece and steps over the (row, head) pairs, so that nothing is
  // divided in the loop; threads past the last whole head of 256 have none.
  const int step = 256 / pieces, piece = tid % pieces;
  const int d0 = 8 * piece, n = min(D - d0, 8);
  int head = tid / pieces, i = 0;
  if (head >= step) return;
  for (;; head += step) {
    for (; head >= heads; head -= heads) ++i;
    if (i >= rb) break;
    const int64_t m = m0 + i;
    if (!known[i]) continue;
    float x[8];
    if (head < qh) {
      turned<T, VEC>(static_cast<const T*>(a.q) + m * a.q_stride + (int64_t)head * D, d0, D, a.half,
                     a.interleaved, cs[i], x);
      store8<T, VEC>(static_cast<T*>(a.q_out) + (m * H + head) * D + d0, n, x);
      continue;
    }
    const int64_t at = place[i];
    if (at < 0) continue;
    const int kv = head - qh >= Hk, h = (head - qh) - kv * Hk;
    if (kv == 0)
      turned<T, VEC>(static_cast<const T*>(a.k) + m * a.kv_stride + (int64_t)h * D, d0, D, a.half,
                     a.interleaved, cs[i], x);
    else
      load8<T, VEC>(static_cast<const T*>(a.v) + m * a.kv_stride + (int64_t)h * D + d0, n, x);
    if constexpr (FP4) {
      // Four lanes hold a block (pieces are a multiple of four). A NaN is not the largest
      // of anything: it is looked for by itself.
      float most = 0.f;
      bool odd = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        most = fmaxf(most, fabsf(x[e]));
        odd = odd || !(fabsf(x[e]) < INFINITY);
      }
      if (odd) most = INFINITY;
      most = fmaxf(most, __shfl_xor(most, 1));
      most = fmaxf(most, __shfl_xor(most, 2));
      const uint32_t e = fp4_exponent(most);
      char* row = static_cast<char*>(a.pool) + at * fr.bytes();
      *reinterpret_cast<uint32_t*>(row + fr.values(kv, h) + d0 / 2) =
          e == 255u ? 0u : fp4_from_f32x8(x, fp4_scale(e));
      if (piece % 4 == 0) row[fr.scales(kv, h) + d0 / kFp4Block] = (char)e;
    } else {
      store8<T, VEC>(static_cast<T*>(a.pool) + (at * 2 + kv) * (int64_t)Hk * D + (int64_t)h * D + d0,
                     n, x);
    }
  }
}

// Eight values of a row a thread. Bound by HBM, the values' write most: 32,771 rows of 8 + 8
// heads x 128: 44 us, 3.9 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void read_rows_fp4(const int32_t* __restrict__ rows, int64_t M,
                                                     const char* __restrict__ pool,
                                                     int64_t pool_rows, int Hk, int D,
                                                     T* __restrict__ out) {
  const int per = 2 * Hk * D / 8;
  const Fp4Row fr{Hk, D};
  const int64_t total = M * per, step = (int64_t)gridDim.x * 256;
  for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += step) {
    const int64_t m = idx / per;
    const int p = (int)(idx - m * per);                  // values and scales are in out's order
    const int64_t at = rows[m];
    float x[8] = {};
    if (at >= 0 && at < pool_rows) {
      const char* row = pool + at * fr.bytes();
      const uint32_t w = *reinterpret_cast<const uint32_t*>(row + 4 * p);
      const float s = fp4_scale((uint8_t)row[fr.scales(0, 0) + p / 4]);
      const u32x4 b = fp4_to_bf16x8(w, s);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(b[i]);
        x[2 * i + 1] = bf16_hi(b[i]);
      }
    }
    store8<T, true>(out + idx * 8, 8, x);
  }
}

template <typename T>
hipError_t launch_rows(const AppendArgs& a, hipStream_t s) {
  const int heads = (a.q != nullptr ? a.H : 0) + (a.k != nullptr ? 2 * a.Hk : 0);
  if (heads == 0) return hipSuccess;
  // Rows a workgroup: up to a thousand pieces and more, while the rows make two
  // workgroups a CU. In us, by this rule / eight rows wherever there are enough: 32,771 rows of 384
  // pieces (four rows) into 4 bits 73 / 75, into a bf16 pool 85.5 / 92.5; 8,003 of 768 (two
  // rows) 42 / 49; 12,007 of 192 takes eight by both.
  int64_t rb = 1;
  while (rb < kMaxRb && rb * heads * ((a.D + 7) / 8) < 1024 && a.M / (2 * rb) >= 512) rb *= 2;
  const int64_t blocks = (a.M + rb - 1) / rb;
  if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
  auto ok = [&](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0;
  };
  const bool vec = a.D % 8 == 0 && (a.interleaved || a.half % 8 == 0) && ok(a.q, a.q_stride) &&
                   ok(a.q_out, 0) && ok(a.k, a.kv_stride) && ok(a.v, a.kv_stride) && ok(a.pool, 0);
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, dim3((uint32_t)blocks), dim3(256), s, a, (int)rb);
  };
  if (a.fp4) return vec ? go(append_rows<T, true, true>) : go(append_rows<T, false, true>);
  return vec ? go(append_rows<T, true, false>) : go(append_rows<T, false, false>);
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  return a.bf16 ? launch_rows<bf16_t>(a, s) : launch_rows<float>(a, s);
}

hipError_t launch_read_fp4(const int32_t* rows, int64_t M, const void* pool, int64_t pool_rows,
                           int Hk, int D, bool bf16, void* out, hipStream_t s) {
  const int64_t total = M * (2 * (int64_t)Hk * D / 8);
  int64_t blocks = (total + 255) / 256;
  if (blocks > (1 << 20)) blocks = 1 << 20;
  const char* p = static_cast<const char*>(pool);
  if (bf16)
    return launch_kernel(read_rows_fp4<bf16_t>, dim3((uint32_t)blocks), dim3(256), s, rows, M, p,
                         pool_rows, Hk, D, static_cast<bf16_t*>(out));
  return launch_kernel(read_rows_fp4<float>, dim3((uint32_t)blocks), dim3(256), s, rows, M, p,
                       pool_rows, Hk, D, static_cast<float*>(out));
}

}  // namespace rocs
