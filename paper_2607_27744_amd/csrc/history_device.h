// Device-side parts shared by the history attention kernels.
#pragma once

#include "common.h"
#include "history.h"

namespace rocs {

constexpr float kLog2e = 1.4426950408889634f;

// The request, its keys and the tile of its query rows that a workgroup has.
// The rows of one K/V head are request r's (token, head of the group) pairs,
// token-major: row i is token i / G, head hk G + i % G, so a group's heads share the
// K/V they read, and a single token fills G rows.
struct HistTile {
  int r, n;                 // request; its query tokens
  int row0, rows;           // first row of the tile among the request's n G; rows in it
  int64_t q0;               // first query token of the request
  int64_t kv0;              // first K/V row (packed)
  const int32_t* pages;     // the slot's page table row (paged)
  int L, prefix;
};

// Slot `slot` of the tiles of TR rows (see tile_base); rows == 0: idle.
__device__ __forceinline__ HistTile hist_tile(const HistArgs& a, int64_t slot, int TR) {
  HistTile t;
  t.r = request_of_slot(a.q_off, a.R, slot, a.G, TR);
  t.q0 = a.q_off[t.r];
  t.n = a.q_off[t.r + 1] - (int)t.q0;
  t.row0 = (int)(slot - tile_base(a.q_off, t.r, a.G, TR)) * TR;
  t.rows = max(min(t.n * a.G - t.row0, TR), 0);
  t.kv0 = 0;
  t.pages = nullptr;
  if (a.table != nullptr) {
    const int s = a.slots != nullptr ? (int)min((uint32_t)a.slots[t.r], (uint32_t)(a.S - 1)) : t.r;
    t.pages = a.table + (int64_t)s * a.width;
    t.L = (int)max(min((int64_t)a.lens[s], a.width * a.page_size), (int64_t)0);
  } else {
    t.kv0 = a.kv_off[t.r];
    t.L = a.kv_off[t.r + 1] - (int)t.kv0;
  }
  t.prefix = a.prefix != nullptr ? a.prefix[t.r] : 0;
  return t;
}

// Position of the request's token, and the number of leading keys its mask
// leaves (before documents).
__device__ __forceinline__ int position_of(const HistTile& t, int token) { return t.L - t.n + token; }
__device__ __forceinline__ int limit_of(const HistArgs& a, const HistTile& t, int token) {
  if (!a.causal) return t.L;
  return max(min(max(position_of(t, token) + 1, t.prefix), t.L), 0);
}

// End of split `split` of keys [0, most); the last one takes what is left.
__device__ __forceinline__ int split_end(const HistArgs& a, int split, int most) {
  if (split + 1 >= a.splits) return most;
  return (int)min((int64_t)(split + 1) * a.chunk, (int64_t)most);
}

// A tile of a split call whose rows see no key past the first part: that part's
// workgroup writes the result itself and marks it (a sum of -1) for the join;
// the others leave. So histories shorter than a part cost no partial results.
__device__ __forceinline__ bool tile_alone(const HistArgs& a, int most) {
  return a.splits > 1 && most <= a.chunk;
}
constexpr float kDone = -1.f;

// Element offset of K/V row j (of all heads).
__device__ __forceinline__ int64_t key_row(const HistArgs& a, const HistTile& t, int j) {
  if (t.pages == nullptr) return (t.kv0 + j) * a.kv_stride;
  const int c = (int)((uint32_t)j / (uint32_t)a.page_size);
  const int64_t p = min((uint32_t)t.pages[c], (uint32_t)(a.pages - 1));
  return p * a.page_stride + (int64_t)(j - c * a.page_size) * a.kv_stride;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// ---------------------------------------------------------------------------
// One row by itself, by one wave, over keys [lo, hi): the kernels give a row a
// weight of 0 for each key that it does not see, and 0 times an infinity or
// NaN in that key's V is NaN. They test their results, and a row that is not
// finite is formed again here, where only the keys that it sees are touched.
// Slow (a wave's dot products from global memory: 1,024 rows over themselves, 8
// heads x 128, 4.3 ms instead of 21 us), for inputs that hold such values.
// Results as the partial form: max in log2 units, sum, and dims lane, lane + 64, ..
// of the weighted sum.
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void lone_row(const HistArgs& a, const HistTile& t, int row, int hk,
                                         int lo, int hi, float& m, float& l, float (&acc)[4]) {
  const int lane = (int)(threadIdx.x & 63);
  const int token = row / a.G, h = hk * a.G + row % a.G;
  const T* q = static_cast<const T*>(a.q) + (t.q0 + token) * a.q_stride + (int64_t)h * a.D;
  const T* k = static_cast<const T*>(a.k) + (int64_t)hk * a.D;
  const T* v = static_cast<const T*>(a.v) + (int64_t)hk * a.D;
  const int pos = position_of(t, token);
  hi = min(hi, limit_of(a, t, token));
  const float slope = a.slopes != nullptr ? a.slopes[h] : 0.f;
  const int doc = a.q_docs != nullptr ? a.q_docs[t.q0 + token] : 0;
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c) acc[c] = 0.f;
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + lane;
    const bool seen = j < hi && (a.q_docs == nullptr || a.kv_docs[t.kv0 + j] == doc);
    const int64_t at = key_row(a, t, min(j, hi - 1));
    float s = -INFINITY;
    if (seen) {
      s = 0.f;
      for (int d = 0; d < a.D; ++d) s += load_f32(q + d) * load_f32(k + at + d);
      s *= a.scale;
      if (a.cap > 0.f) s = a.cap * tanhf(s / a.cap);
      if (a.slopes != nullptr) s -= slope * fabsf((float)(pos - j));
    }
    const float mn = fmaxf(m, wave_max(s));
    const float ms = mn == -INFINITY ? 0.f : mn;
    const float f = expf(m - ms);
    const float p = seen ? expf(s - ms) : 0.f;
    l = l * f + wave_sum(p);
    m = mn;
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] *= f;
    uint64_t todo = __ballot(seen);
    while (todo != 0) {
      const int i = __builtin_ctzll(todo);
      todo &= todo - 1;
      const float pj = __shfl(p, i);
      const int64_t row_at = __shfl(at, i);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (lane + 64 * c < a.D) acc[c] += pj * load_f32(v + row_at + lane + 64 * c);
    }
  }
  m *= kLog2e;
}

// The lone row's result where the kernel's own would have gone.
template <typename T>
__device__ __forceinline__ void redo_row(const HistArgs& a, const HistTile& t, int row, int hk,
                                         int lo, int hi, int split, bool direct) {
  float m, l, acc[4];
  lone_row<T>(a, t, row, hk, lo, hi, m, l, acc);
  const int lane = (int)(threadIdx.x & 63);
  const int64_t at = (t.q0 + row / a.G) * a.H + hk * a.G + row % a.G;
  if (!direct) {
    const int64_t to = (int64_t)split * a.N * a.H + at;
    if (lane == 0) {
      a.part_ml[2 * to] = m;
      a.part_ml[2 * to + 1] = l;
    }
    for (int c = 0; c < 4; ++c)
      if (lane + 64 * c < a.D) a.part_o[to * a.D + lane + 64 * c] = acc[c];
  } else {
    T* o = static_cast<T*>(a.out) + at * a.D;
    for (int c = 0; c < 4; ++c)
      if (lane + 64 * c < a.D) o[lane + 64 * c] = from_f32<T>(l == 0.f ? 0.f : acc[c] / l);
  }
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// Whether forming a row with the sum `l` again can change it. Only keys that
// the row sees have a part in the sum: where it is NaN, so is the result. (But
// below the kernel's own width, head_dim D of DP, zeros of q meet what stands in
// past K's end, and an infinity there makes NaN of a score that is none.)
__device__ __forceinline__ bool may_differ(float l, int D, int DP) { return D != DP || l == l; }

}  // namespace rocs
