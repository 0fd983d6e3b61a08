// Attention of a request's own rows over its history, packed or paged: the rule
// that cuts a call up, the general kernel and the join of a split history.
#include "history_device.h"
#include "launch.h"
#include "layer.h"
#include "status.h"

namespace rocs {
namespace {

// ---------------------------------------------------------------------------
// General kernel: any dtype, head_dim <= 256, strides and page sizes.
//
// A workgroup takes 16 rows (token, head) of one request and K/V head; its four
// waves share the keys in blocks of 16 and merge their partial softmaxes
// through LDS. Scores and outputs run on the fp32 matrix instructions
// (16x16x4; bf16 converts exactly): S^T = K Q^T leaves lane (l16, g) keys
// 4 g .. + 3 of row l16, the B operand of O^T = V^T P^T as it stands. A score
// is summed in four chains, one for each of four neighbouring dims.
// Rows of four aligned elements and head_dim up to 128 (PIPE): lane l16 takes
// the NB dims from NB l16 of V^T, so that V comes in 16-byte loads as K does; a
// block's V and the next one's K are in flight over its scores and weights, and
// the next block's page numbers before them. Loads are clamped into the
// history and the head, never skipped; what stands in past an end meets a
// weight or a query of 0, or a column that is not stored.
// What bounds it: HBM where rows are few (fp32, 64 rows over 2,048 keys each, 8
// heads x 128: 277 us, 3.9 TB/s; 952 us with 4-byte V loads, one block at a time),
// else the fp32 matrix rate, an eighth of bf16's.
// ---------------------------------------------------------------------------
constexpr int kGenTile = 16;

template <typename T, bool VEC>
__device__ __forceinline__ f32x4 row4(const T* row, int d, int D) {
  if constexpr (VEC) {                     // D and d are multiples of four
    const f32x4 v = load4_f32<T, true>(row + min(d, D - 4), 4);
    return d < D ? v : f32x4{0.f, 0.f, 0.f, 0.f};
  } else {
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = load_f32(row + min(d + i, D - 1));
      v[i] = d + i < D ? x : 0.f;
    }
    return v;
  }
}

// DP: head_dim rounded up to 32, 64, 128 or 256. VEC: rows of q, k and v are
// aligned to four elements and head_dim is a multiple of four. FP4: a cache in 4
// bits, of which lane (l16, g) takes a quarter of key l16's dims, DP / 4 from DP / 4 g,
// and the NB dims from NB l16 of V's keys, as PIPE does.
template <typename T, int DP, bool VEC, bool FP4 = false>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(DP == 256 && sizeof(T) == 4 ? 1 : 2))) void history_general(
    const HistArgs a) {
  constexpr int NB = DP / 16;              // 16-dim blocks
  constexpr bool PIPE = VEC && DP <= 128 && !FP4;
  constexpr int LP = DP + 4;               // LDS row (floats), padded against bank conflicts
  __shared__ __attribute__((aligned(16))) float po[4][kGenTile][LP];
  __shared__ float pm[4][kGenTile], pl[4][kGenTile];
  __shared__ int odd[kGenTile];            // rows to form again
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int hk = blockIdx.y, split = blockIdx.z;
  const HistTile t = hist_tile(a, blockIdx.x, kGenTile);
  if (t.rows <= 0) return;
  const int D = a.D;
  if (tid < kGenTile) odd[tid] = 0;
  const int row = t.row0 + min(l16, t.rows - 1);         // clamped; extra rows never stored
  const int token = row / a.G, h = hk * a.G + row % a.G;
  const int pos = position_of(t, token), lim = limit_of(a, t, token);
  const float slope = a.slopes != nullptr ? a.slopes[h] : 0.f;
  const int doc = a.q_docs != nullptr ? a.q_docs[t.q0 + token] : 0;
  const int lo = split * a.chunk;
  const int most = limit_of(a, t, (t.row0 + t.rows - 1) / a.G);    // the tile's last row sees most
  const int hi = split_end(a, split, most);
  const bool alone = tile_alone(a, most), direct = a.splits == 1 || alone;
  if (alone && split > 0) return;
  const T* q = static_cast<const T*>(a.q) + (t.q0 + token) * a.q_stride + (int64_t)h * D;
  const T* k = static_cast<const T*>(a.k) + (int64_t)hk * D;
  const T* v = static_cast<const T*>(a.v) + (int64_t)hk * D;
  f32x4 qf[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) qf[b] = row4<T, VEC>(q, FP4 ? 4 * NB * g + 4 * b : 16 * b + 4 * g, D);
  float m = -INFINITY, lsum = 0.f;
  f32x4 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  // Scores of the block at kb in s4 -> weights in p, and the running max.
  auto softmax = [&](int kb, const f32x4& dot, f32x4& p) __attribute__((always_inline)) {
    f32x4 s4;
    bool seen[4];
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = kb + 4 * g + i;
      seen[i] = j < lim && j < hi;
      if (a.q_docs != nullptr) seen[i] = seen[i] && a.kv_docs[t.kv0 + min(j, hi - 1)] == doc;
      float s = dot[i] * a.scale;
      if (a.cap > 0.f) s = a.cap * tanhf(s / a.cap);
      if (a.slopes != nullptr) s -= slope * fabsf((float)(pos - j));
      s4[i] = seen[i] ? s : -INFINITY;
      mx = fmaxf(mx, s4[i]);
    }
    const float mn = fmaxf(m, max_across_rows(mx));
    const float ms = mn == -INFINITY ? 0.f : mn;         // no finite score yet: weights 0
    const float alpha = expf(m - ms);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = seen[i] ? expf(s4[i] - ms) : 0.f;
    lsum = lsum * alpha + ((p[0] + p[1]) + (p[2] + p[3]));
    m = mn;
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b] *= alpha;
  };
  if constexpr (FP4) {
    // Words of eight values; past the head the last ones stand in, where q is 0 and
    // the result is not stored.
    const Fp4Row fr{a.Hk, D};
    const char* base = static_cast<const char*>(a.k);
    // The next block's words load while this one is computed, where registers allow it: fp32 q, 128
    // single rows over 3,100 keys of 8 heads of 128, 587 us and 759 without; of 256 it spills in bf16
    // (1,711 and 1,246).
    constexpr bool AHEAD = DP <= 128;
    constexpr int WORDS = (DP / 4 + 7) / 8, VW = (NB + 7) / 8;
    uint32_t kn[WORDS], vn[4][VW], ken[WORDS], ven[4][VW];
    PoolKey at[5];                         // key l16, and V's 4 g .. + 3
    auto look_up = [&](int kb) __attribute__((always_inline)) {
      at[4] = pool_key(a, t.pages, min(kb + l16, hi - 1));
#pragma unroll
      for (int i = 0; i < 4; ++i) at[i] = pool_key(a, t.pages, min(kb + 4 * g + i, hi - 1));
    };
    auto load = [&]() __attribute__((always_inline)) {
      const char* kr = base + (int64_t)pool_row(a, at[4]) * a.kv_stride;
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        const int d = min(DP / 4 * g + 8 * w, D - 8);
        kn[w] = *reinterpret_cast<const uint32_t*>(kr + fr.values(0, hk) + d / 2);
        ken[w] = (uint8_t)kr[fr.scales(0, hk) + d / kFp4Block];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char* vr = base + (int64_t)pool_row(a, at[i]) * a.kv_stride;
#pragma unroll
        for (int c = 0; c < VW; ++c) {
          const int d = min(NB * l16 + 8 * c, D - 1);
          vn[i][c] = *reinterpret_cast<const uint32_t*>(vr + fr.values(1, hk) + d / 8 * 4);
          ven[i][c] = (uint8_t)vr[fr.scales(1, hk) + d / kFp4Block];
        }
      }
    };
    const int first = lo + 16 * wave;
    if (AHEAD && first < hi) {
      look_up(first);
      load();
      look_up(first + 64);
    }
    for (int kb = first; kb < hi; kb += 64) {
      uint32_t kw[WORDS], vw[4][VW];
      float ks[WORDS], vs[4][VW];
      if constexpr (!AHEAD) {
        look_up(kb);
        load();
      }
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        kw[w] = kn[w];
        ks[w] = fp4_scale(ken[w]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < VW; ++c) {
          vw[i][c] = vn[i][c] >> (4 * (min(NB * l16 + 8 * c, D - 1) % 8));
          vs[i][c] = fp4_scale(ven[i][c]);
        }
      if constexpr (AHEAD) {
        load();                            // the next block; past the end the last key
        look_up(kb + 128);
      }
      f32x4 part[4] = {};
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
#pragma unroll
        for (int i = 0; i < (DP / 4 < 8 ? DP / 4 : 8); ++i)
          part[i % 4] = __builtin_amdgcn_mfma_f32_16x16x4f32(fp4_value(kw[w], i, ks[w]), qf[2 * w + i / 4][i % 4],
                                                             part[i % 4], 0, 0, 0);
      }
      f32x4 p;
      softmax(kb, (part[0] + part[1]) + (part[2] + part[3]), p);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fp4_value(vw[i][b / 8], b % 8, vs[i][b / 8]), p[i], o[b], 0, 0, 0);
    }
  } else if constexpr (PIPE) {
    constexpr int NV = NB < 4 ? NB : 4;    // dims of one V load
    auto key_at = [&](int j) __attribute__((always_inline)) { return key_row(a, t, min(j, hi - 1)); };
    int64_t kr = 0, vr[4] = {};
    f32x4 kf[NB];
    auto load_k = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < NB; ++b) kf[b] = load4_f32<T, true>(k + kr + min(16 * b + 4 * g, D - 4), 4);
    };
    const int first = lo + 16 * wave;
    if (first < hi) {
      kr = key_at(first + l16);
#pragma unroll
      for (int i = 0; i < 4; ++i) vr[i] = key_at(first + 4 * g + i);
      load_k();
    }
    for (int kb = first; kb < hi; kb += 64) {
      float vv[4][NB];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < NB / NV; ++c) {
          const T* src = v + vr[i] + min(NB * l16 + NV * c, D - NV);
          if constexpr (NV == 4) {
            const f32x4 x = load4_f32<T, true>(src, 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) vv[i][4 * c + e] = x[e];
          } else {
#pragma unroll
            for (int e = 0; e < NV; ++e) vv[i][NV * c + e] = load_f32(src + e);
          }
        }
      kr = key_at(kb + 64 + l16);
#pragma unroll
      for (int i = 0; i < 4; ++i) vr[i] = key_at(kb + 64 + 4 * g + i);
      f32x4 part[4] = {};
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          part[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[b][i], qf[b][i], part[i], 0, 0, 0);
      load_k();
      f32x4 p;
      softmax(kb, (part[0] + part[1]) + (part[2] + part[3]), p);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[i][b], p[i], o[b], 0, 0, 0);
    }
  } else {
    for (int kb = lo + 16 * wave; kb < hi; kb += 64) {
      const T* kr = k + key_row(a, t, min(kb + l16, hi - 1));
      const T* vr[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) vr[i] = v + key_row(a, t, min(kb + 4 * g + i, hi - 1));
      f32x4 part[4] = {};
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const f32x4 kf = row4<T, VEC>(kr, 16 * b + 4 * g, D);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          part[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i], qf[b][i], part[i], 0, 0, 0);
      }
      f32x4 p;
      softmax(kb, (part[0] + part[1]) + (part[2] + part[3]), p);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float vf = load_f32(vr[i] + min(16 * b + l16, D - 1));
          o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(kb + 4 * g + i < hi ? vf : 0.f, p[i], o[b], 0, 0, 0);
        }
    }
  }
  lsum = sum_across_rows(lsum);
  if (g == 0) {
    pm[wave][l16] = m;
    pl[wave][l16] = lsum;
  }
  // Element i of o[b] is dim 16 b + 4 g + i of row l16, or (PIPE, FP4) NB (4 g + i) + b.
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      po[wave][l16][PIPE || FP4 ? NB * (4 * g + i) + b : 16 * b + 4 * g + i] = o[b][i];
  __syncthreads();
  // Merge the four partial softmaxes, four dims a step.
  const int64_t part0 = (int64_t)split * a.N * a.H;
  for (int idx = tid; idx < t.rows * (DP / 4); idx += 256) {
    const int i = idx / (DP / 4), d0 = 4 * (idx % (DP / 4));
    if (d0 >= D) continue;
    const float mx = fmaxf(fmaxf(pm[0][i], pm[1][i]), fmaxf(pm[2][i], pm[3][i]));
    const float ms = mx == -INFINITY ? 0.f : mx;
    float l = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = expf(pm[w][i] - ms);
      l += pl[w][i] * f;
      y += *reinterpret_cast<const f32x4*>(&po[w][i][d0]) * f;
    }
    if (!(finite(y[0]) && finite(y[1]) && finite(y[2]) && finite(y[3])) && may_differ(l, D, DP)) odd[i] = 1;
    const int rw = t.row0 + i;
    const int64_t at = (t.q0 + rw / a.G) * a.H + hk * a.G + rw % a.G;
    if (a.splits > 1 && d0 == 0) {
      a.part_ml[2 * (part0 + at)] = mx * kLog2e;
      a.part_ml[2 * (part0 + at) + 1] = alone ? kDone : l;
    }
    if (!direct) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (d0 + e < D && l != 0.f) a.part_o[(part0 + at) * D + d0 + e] = y[e];
    } else {
      T* out = static_cast<T*>(a.out) + at * D;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (d0 + e < D) out[d0 + e] = from_f32<T>(l == 0.f ? 0.f : y[e] / l);
    }
  }
  __syncthreads();
  for (int i = wave; i < t.rows; i += 4)
    if (__builtin_amdgcn_readfirstlane(odd[i]) != 0)
      redo_row<T, FP4>(a, t, t.row0 + i, hk, lo, hi, split, direct);
}

// ---------------------------------------------------------------------------
// Join of a split history: out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.
// W waves a row (four for few rows, else one): each forms all weights (a lane a
// part), then they share the parts, eight in flight. A part without a seen key
// has l = 0 and no O; its loads are not skipped (a branch would put one latency
// after the other) but dropped. Rows that are done already (kDone) are left.
// Bound by latency for few rows (8 rows in 9 parts: 2.9 us; 1,024 in 11:
// 5.4), else by the read of the parts.
// ---------------------------------------------------------------------------
constexpr int kMaxSplits = 256;

template <typename T, int NC, int W>       // NC: head_dim / 64, rounded up
__global__ __launch_bounds__(256) void history_join(const float* __restrict__ ml,
                                                    const float* __restrict__ po,
                                                    const int32_t* __restrict__ q_end,
                                                    T* __restrict__ out, int64_t rows, int H, int D,
                                                    int splits) {
  constexpr int NS = kMaxSplits / 64;
  __shared__ float weight[4][kMaxSplits], ysum[4][64 * NC];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = W == 4 ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  // Rows behind the last request have no parts and stay as they are. (Uniform
  // over the row's waves.)
  if (row >= rows || row >= (int64_t)*q_end * H || ml[2 * row + 1] == kDone) return;
  const int first = W == 4 ? wave : 0;
  float ms[NS], ls[NS], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const int s = 64 * i + lane;
    const float* p = ml + 2 * ((int64_t)min(s, splits - 1) * rows + row);
    ms[i] = p[0];
    ls[i] = s < splits ? p[1] : 0.f;
    if (ls[i] != 0.f) m = fmaxf(m, ms[i]);
  }
  m = wave_max(m);
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const float f = ls[i] != 0.f ? exp2f(ms[i] - m) : 0.f;
    if (ls[i] != 0.f) l += f * ls[i];
    weight[wave][64 * i + lane] = ls[i] != 0.f ? f : -1.f;     // -1: no O
  }
  l = wave_sum(l);
  float y[NC] = {};
  for (int i = first; i < splits; i += 8 * W) {
    float x[8][NC], f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int s = min(i + W * j, splits - 1);
      f[j] = i + W * j < splits ? weight[wave][s] : -1.f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
        x[j][c] = po[((int64_t)s * rows + row) * D + min(lane + 64 * c, D - 1)];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (!(f[j] < 0.f)) y[c] += x[j][c] * f[j];
  }
  if constexpr (W == 4) {
#pragma unroll
    for (int c = 0; c < NC; ++c) ysum[wave][lane + 64 * c] = y[c];
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += 256) {
      const float t = (ysum[0][d] + ysum[1][d]) + (ysum[2][d] + ysum[3][d]);
      out[row * D + d] = from_f32<T>(l == 0.f ? 0.f : t / l);
    }
  } else {
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (lane + 64 * c < D) out[row * D + lane + 64 * c] = from_f32<T>(l == 0.f ? 0.f : y[c] / l);
  }
}

template <typename T, int DP>
hipError_t launch_general(const HistArgs& a, hipStream_t s) {
  const int64_t slots = a.R + (a.N * a.G + kGenTile - 1) / kGenTile;
  if (!grid_fits(slots, 256)) return hipErrorInvalidConfiguration;
  const uintptr_t all = reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) |
                        reinterpret_cast<uintptr_t>(a.v);
  const bool vec = a.D % 4 == 0 && a.q_stride % 4 == 0 && a.kv_stride % 4 == 0 &&
                   a.page_stride % 4 == 0 && all % (4 * sizeof(T)) == 0;
  return launch_kernel(vec ? history_general<T, DP, true> : history_general<T, DP, false>,
                       dim3((uint32_t)slots, (uint32_t)a.Hk, (uint32_t)a.splits), dim3(256), s, a);
}

// A 4-bit cache: head_dim is a multiple of 32, so q's rows are aligned to four
// elements if its pointer and stride are.
template <typename T, int DP>
hipError_t launch_general_fp4(const HistArgs& args, hipStream_t s) {
  HistArgs a = args;
  set_page_divisor(a);
  const int64_t slots = a.R + (a.N * a.G + kGenTile - 1) / kGenTile;
  if (!grid_fits(slots, 256)) return hipErrorInvalidConfiguration;
  const bool vec = a.q_stride % 4 == 0 && reinterpret_cast<uintptr_t>(a.q) % (4 * sizeof(T)) == 0;
  return launch_kernel(vec ? history_general<T, DP, true, true> : history_general<T, DP, false, true>,
                       dim3((uint32_t)slots, (uint32_t)a.Hk, (uint32_t)a.splits), dim3(256), s, a);
}
template <typename T>
hipError_t launch_general_fp4(const HistArgs& a, hipStream_t s) {
  if (a.D <= 32) return launch_general_fp4<T, 32>(a, s);
  if (a.D <= 64) return launch_general_fp4<T, 64>(a, s);
  if (a.D <= 128) return launch_general_fp4<T, 128>(a, s);
  return launch_general_fp4<T, 256>(a, s);
}

template <typename T>
hipError_t launch_general(const HistArgs& a, hipStream_t s) {
  if (a.D <= 32) return launch_general<T, 32>(a, s);
  if (a.D <= 64) return launch_general<T, 64>(a, s);
  if (a.D <= 128) return launch_general<T, 128>(a, s);
  return launch_general<T, 256>(a, s);
}

template <typename T, int NC>
hipError_t launch_join(const HistArgs& a, hipStream_t s) {
  const int64_t rows = a.N * a.H;
  const bool few = rows <= 2048;
  const int64_t blocks = few ? rows : (rows + 3) / 4;
  if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
  return launch_kernel(few ? history_join<T, NC, 4> : history_join<T, NC, 1>, dim3((uint32_t)blocks),
                       dim3(256), s, a.part_ml, a.part_o, a.q_off + a.R, static_cast<T*>(a.out), rows,
                       a.H, a.D, a.splits);
}
template <typename T>
hipError_t launch_join(const HistArgs& a, hipStream_t s) {
  return a.D <= 64    ? launch_join<T, 1>(a, s)
         : a.D <= 128 ? launch_join<T, 2>(a, s)
                      : launch_join<T, 4>(a, s);
}

}  // namespace

// The plan with histories in `splits` chunks of whole stages, and what that needs.
static HistPlan cut_in(HistPlan p, int64_t splits, int64_t N, int H, int D, int64_t max_len) {
  if (splits > kMaxSplits) splits = kMaxSplits;
  if (splits < 1) splits = 1;
  p.chunk = (int)(((max_len + splits - 1) / splits + 63) / 64 * 64);
  p.splits = p.chunk > 0 ? (int)((max_len + p.chunk - 1) / p.chunk) : 1;
  if (p.splits < 1) p.splits = 1;
  if (p.splits > 1) {
    p.ml_bytes = align256((size_t)p.splits * N * H * 2 * sizeof(float));
    p.o_bytes = align256((size_t)p.splits * N * H * D * sizeof(float));
  }
  return p;
}

HistPlan history_plan(int64_t R, int64_t N, int H, int Hk, int D, int64_t max_len, bool bf16) {
  HistPlan p{};
  const int64_t each = (N * (H / Hk) + R - 1) / R;       // rows a request and K/V head
  p.rows = !(bf16 && D % 8 == 0 && D <= 128) ? kGenTile : each <= 32 ? 32 : 128;
  p.heads = 1;
  const int64_t tiles = R * ((each + p.rows - 1) / p.rows) * Hk;
  const auto parts = [max_len](int64_t most, int64_t least_keys) {
    const int64_t n = (max_len + least_keys - 1) / least_keys;
    return n < most ? n : most;
  };
  // A history is cut where the tiles alone leave the chip idle: two workgroups a
  // CU, chunks of at least 256 keys. (More parts than that do not pay at 128 rows:
  // chunks over six cached histories of 2,400 to 12,800 rows take 418 us in 504
  // whole tiles, 508 in four parts.)
  int64_t splits = parts(512 / tiles, 256);
  if (p.rows == 32) {
    // Few rows: a read of K and V. With two rounds of the chip in chunks of 512
    // keys, chunks are many, so that ragged histories end together, and a workgroup
    // takes as many heads, up to four, as still make two rounds (128 histories of
    // 3,100 rows on average, 8 heads x 128: 287 us; a head a workgroup: 323; 40 of
    // them: 96 by two heads, 102 as below). With less, the waves of a head share
    // its keys, which is fewer steps one after the other (one history of 16,384
    // rows: 20 us, by four heads 24).
    const int64_t chunks = (max_len + 511) / 512;
    int hw = Hk % 4 == 0 ? 4 : Hk % 2 == 0 ? 2 : 1;
    while (hw > 1 && R * (Hk / hw) * chunks < 1024) hw /= 2;
    const int64_t wide = R * (Hk / hw);
    if (wide * chunks >= 1024) {
      p.heads = hw;
      splits = parts(4096 / wide, 512);
    } else {
      const int64_t more = parts(2048 / tiles, 1024);
      if (more > splits) splits = more;
    }
  }
  return cut_in(p, splits, N, H, D, max_len);
}

hipError_t launch_history(const HistArgs& a, int rows, bool bf16, bool fast, hipStream_t s) {
  hipError_t e = fast && rows == 128  ? launch_history_tile(a, s)
                 : fast && rows == 32 ? launch_history_split(a, s)
                 : bf16              ? launch_general<bf16_t>(a, s)
                                     : launch_general<float>(a, s);
  if (e != hipSuccess || a.splits == 1) return e;
  return bf16 ? launch_join<bf16_t>(a, s) : launch_join<float>(a, s);
}

// bf16: history_fp4_few up to 32 rows of a request and K/V head, two tiles of its 16 read the
// keys twice through L2 (32 rows a wave cost more: registers for two of the three waves of a SIMD;
// 64 requests, 3,125 keys, 8 heads on 2 x 128: 32 rows 60 us, by 16 55), then the 128-row tiles. In us,
// few / tiles, 8 heads on 2 x 128, by the rows of a request and head: 64 requests over 3,125 keys
// 16: 41 / 56, 24: 47 / 54, 32: 55 / 48, 40: 63 / 54, 64: 90 / 57; 128 requests 32: 92 / 113, 40: 107 / 109,
// 48: 121 / 113; 8 on 8 x 64, 64 requests, 32: 105 / 133, 48: 133 / 122; one history of 8,000 rows 14 / 14
// throughout. Where one or two K/V heads leave the tiles' grid small already, they win from about 28
// rows on: one row of 32 heads on 1 x 128, 64 requests 36 / 30, 128 requests 53 / 44 (of 16 heads 24 / 27, 37 /
// 46); of 64 on 2 x 128, 64 requests 53 / 44, 128 requests 87 / 81; heads of 64 26 / 25, 35 / 32. The border is
// one for all, between those and 8 K/V heads, which gain at 32. The cut of few rows is that of
// history_plan, with chunks of 512 keys in either case: 128 single rows over 3,125 keys, 8 heads x 128: by four heads a workgroup 129 us, two 136,
// one 207; chunks of 256 to 1,536 keys 128 to 164.
HistPlan fp4_plan(int64_t R, int64_t N, int H, int Hk, int D, int64_t max_len, bool bf16) {
  const int64_t each = (N * (H / Hk) + R - 1) / R;       // rows a request and K/V head
  if (bf16 && D <= 128 && each > 32) return history_plan(R, N, H, Hk, D, max_len, true);
  if (!(bf16 && D <= 128)) {
    HistPlan general = history_plan(R, N, H, Hk, D, max_len, false);
    general.rows = 0;
    return general;
  }
  HistPlan p{};
  p.rows = 16;
  const auto parts = [max_len](int64_t most, int64_t least_keys) {
    const int64_t n = (max_len + least_keys - 1) / least_keys;
    return n < most ? n : most;
  };
  const int64_t chunks = (max_len + 511) / 512;
  int hw = Hk % 4 == 0 ? 4 : Hk % 2 == 0 ? 2 : 1;
  while (hw > 1 && R * (Hk / hw) * chunks < 1024) hw /= 2;
  const int64_t wide = R * (Hk / hw);
  p.heads = wide * chunks >= 1024 ? hw : 1;
  int64_t splits = wide * chunks >= 1024 ? parts(4096 / wide, 512) : parts(2048 / (R * Hk), 512);
  return cut_in(p, splits, N, H, D, max_len);
}

hipError_t launch_history_fp4(const HistArgs& a, int rows, bool bf16, bool fast, hipStream_t s) {
  const hipError_t e = fast && rows == 128 ? launch_history_fp4_tile(a, s)
                       : fast && rows > 0  ? launch_history_fp4_few(a, s)
                       : bf16              ? launch_general_fp4<bf16_t>(a, s)
                                           : launch_general_fp4<float>(a, s);
  if (e != hipSuccess || a.splits == 1) return e;
  return bf16 ? launch_join<bf16_t>(a, s) : launch_join<float>(a, s);
}

}  // namespace rocs
