// Shared by the bf16 MFMA kernels of the history attention (history_tile.hip,
// history_split.hip): K/V addressing by groups of 16 rows, the score rules in
// exp2 units, masks, and the document stages of a tile.
//
// Register layout (as in attention.hip): scores are computed transposed,
// S^T = K Q^T on 32x32x16, so lane (l32, hh) holds for query row l32 the keys
// 32 kb + 8 (e / 4) + 4 hh + e % 4 of a 64-key stage in element e of block kb.
#pragma once

#include <type_traits>

#include "history_device.h"

namespace rocs {

constexpr int kStageKeys = 64;
// SCORE: a cap up to kCapTurn, a bias by distance, a cap above kCapTurn.
constexpr int kCap = 1, kBias = 2, kWideCap = 4;
constexpr float kCapTurn = 128.0f;
constexpr float kLazyMove = 64.0f;          // log2 of the largest unnormalised weight
constexpr float kStageBound = 0x1p64f;      // per-lane stage sum taken without a row max

// ---------------------------------------------------------------------------
// K/V rows. A group is 16 keys from a multiple of 16: it lies in one page (a
// page is a multiple of 16 rows), so its address is uniform over a wave and its
// table entry a scalar load. Lanes add the row in the group and their chunk.
// ---------------------------------------------------------------------------
struct KeyFeed {
  const int32_t* pages;    // page table row, or null: packed
  int64_t page_bytes, row_bytes, kv0_bytes;
  uint32_t page16, magic, max_page;   // page size in groups; 2^32 / page16 + 1
  int page_size;

  __device__ __forceinline__ KeyFeed(const HistArgs& a, const HistTile& t)
      : pages(t.pages), page_bytes(a.page_stride * 2), row_bytes(a.kv_stride * 2),
        kv0_bytes(t.kv0 * a.kv_stride * 2), page16((uint32_t)a.page_size / 16), magic(a.page_magic),
        max_page((uint32_t)(a.pages - 1)), page_size(a.page_size) {}

  // Byte offset of the group that starts at key g0 (uniform).
  __device__ __forceinline__ int64_t group(int g0) const {
    if (pages == nullptr) return kv0_bytes + (int64_t)g0 * row_bytes;
    const uint32_t g = (uint32_t)g0 / 16;
    uint32_t c = page16 == 1 ? g : (uint32_t)(((uint64_t)g * magic) >> 32);
    if (c * page16 > g) --c;                 // the product is at most one too large
    const uint32_t p = min((uint32_t)pages[c], max_page);
    return (int64_t)p * page_bytes + (int64_t)(g0 - (int)(c * page_size)) * row_bytes;
  }
};

// ---------------------------------------------------------------------------
// Scores. The cap in exp2 units: cap tanh(x / cap) = cap (1 - 2 / (1 + e^(2x/cap))),
// two transcendentals; both tails come out exactly (rcp of infinity and of 1).
// Around 0 the difference cancels: its error is up to 2^-22 cap, absolute, at
// any score (2.5e-5 at a cap of 128, what an fp32 sum of 128 products is off by;
// at 1e5 it would be 0.02, at 1e8 all scores one value). Caps above kCapTurn
// therefore take another form, whose error is relative to the score as that of the
// score itself is. It costs more instructions (16 requests of 2,048 rows, 8 heads x
// 128, causal: 207 us, 195 with a cap of 30, 167 without one; 370 where all stages
// hold scores past a quarter of the cap), so the caps in use keep this form.
// The bias in a stage that lies wholly before a row needs no distance: -slope
// (p - j) is linear in j.
// ---------------------------------------------------------------------------
struct RowRule {
  float scale2;            // scale log2(e)
  float cap_in, cap2;      // 2 scale log2(e) / cap (wide: scale / cap), cap log2(e)
  float slope2;            // slope log2(e)
  int pos, lim, doc;
};

// The score rules of query head `head`. Both limits to finite values: a factor
// of infinity would make a score of 0 NaN.
template <int SCORE>
__device__ __forceinline__ void score_rules(RowRule& r, const HistArgs& a, int head) {
  constexpr float kMax = 3.402823466e38f;
  r.scale2 = a.scale * kLog2e;
  r.cap_in = r.cap2 = r.slope2 = 0.f;
  if constexpr ((SCORE & kCap) != 0) r.cap_in = fminf(2.0f * r.scale2 / a.cap, kMax);
  if constexpr ((SCORE & kWideCap) != 0) r.cap_in = fminf(a.scale / a.cap, kMax);
  if constexpr ((SCORE & (kCap | kWideCap)) != 0) r.cap2 = fminf(a.cap * kLog2e, kMax);
  if constexpr ((SCORE & kBias) != 0) r.slope2 = a.slopes[head] * kLog2e;
}

// A capped score in exp2 units without the cancellation. Up to u = x / cap of 1/4 the
// series tanh(u) / u = 1 - u^2/3 + 2u^4/15 - 17u^6/315 + 62u^8/2835 (its next
// term is below 2^-26 there): scale log2(e) times it, from w = u^2.
constexpr float kSeriesEnd = 1.0f / 16.0f;  // of w
__device__ __forceinline__ float cap_series(float w, const RowRule& r) {
  float t = fmaf(w, 62.0f / 2835.0f * r.scale2, -17.0f / 315.0f * r.scale2);
  t = fmaf(w, t, 2.0f / 15.0f * r.scale2);
  t = fmaf(w, t, -1.0f / 3.0f * r.scale2);
  return fmaf(w, t, r.scale2);
}
// Beyond it the form with the exponential, whose value is no longer small
// against its error (2^-19 relative at most).
__device__ __forceinline__ float wide_cap(float s, const RowRule& r) {
  const float u = s * r.cap_in, w = u * u;
  const float e = __builtin_amdgcn_exp2f(u * (2.0f * kLog2e));
  const float far = r.cap2 * fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + e), 1.0f);
  return w <= kSeriesEnd ? s * cap_series(w, r) : far;
}

// One score in exp2 units for a stage that needs no mask and lies before the
// row: key offset c in the stage, shift = plain_shift, less the running max.
template <int SCORE>
__device__ __forceinline__ float plain_shift(const RowRule& r, int base, int hh) {
  float x = (SCORE & kCap) != 0 ? r.cap2 : 0.f;
  if constexpr ((SCORE & kBias) != 0) x -= r.slope2 * (float)(r.pos - base - 4 * hh);
  return x;
}
// A wide cap takes the series whatever the score; reach follows the largest w,
// and a stage that it takes past kSeriesEnd forms its scores again.
template <int SCORE>
__device__ __forceinline__ float plain_score(float s, int c, const RowRule& r, float shift, float& reach) {
  if constexpr ((SCORE & kBias) != 0) shift = fmaf(r.slope2, (float)c, shift);
  if constexpr ((SCORE & kCap) != 0)
    return fmaf(-2.0f * r.cap2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s * r.cap_in)), shift);
  if constexpr ((SCORE & kWideCap) != 0) {
    const float u = s * r.cap_in, w = u * u;
    reach = fmaxf(reach, w);
    return fmaf(s, cap_series(w, r), shift);
  }
  return fmaf(s, r.scale2, shift);
}

// Scores of one 16-key step (elements 8 half .. + 7 of the block at key offset
// 32 kb) in exp2 units, less `ref`, in place; keys from `base` (of the stage).
template <int SCORE, typename V>
__device__ __forceinline__ void score_step(V& s, int kb, int half, const RowRule& r, int base, int hh,
                                           float ref) {
  const float rel = (float)(r.pos - base - 4 * hh);
  const float none = (SCORE & kCap) != 0 ? r.cap2 - ref : -ref;
#pragma unroll
  for (int e = 8 * half; e < 8 * half + 8; ++e) {
    const int c = 32 * kb + 8 * (e / 4) + e % 4;
    float shift = none;
    if constexpr ((SCORE & kBias) != 0) shift = fmaf(-r.slope2, fabsf(rel - (float)c), none);
    if constexpr ((SCORE & kCap) != 0)
      s[e] = fmaf(-2.0f * r.cap2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[e] * r.cap_in)), shift);
    else if constexpr ((SCORE & kWideCap) != 0)
      s[e] = wide_cap(s[e], r) + shift;
    else
      s[e] = fmaf(s[e], r.scale2, shift);
  }
}

// -inf for the keys of the step that the row does not see. docs: the stage's
// document ids in LDS (DOCS).
template <bool DOCS, typename V>
__device__ __forceinline__ void mask_step(V& s, int kb, int half, const RowRule& r, int base, int hh,
                                          const ROCS_LDS int32_t* docs) {
  const int rel = r.lim - base - 4 * hh;
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int q = 2 * half; q < 2 * half + 2; ++q) {
    i32x4 id = {};
    if constexpr (DOCS) id = *reinterpret_cast<const ROCS_LDS i32x4*>(docs + 32 * kb + 8 * q + 4 * hh);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool hide = 32 * kb + 8 * q + i >= rel || (DOCS && id[i] != r.doc);
      if (hide) s[4 * q + i] = -INFINITY;
    }
    // A few lane masks at a time: all at once they would not fit the scalar registers.
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The order of a run of PRODUCTS matrix instructions, each with READS LDS reads
// for it AHEAD products earlier. (Left alone, the compiler puts a product's
// reads right before it and waits for their latency each time.)
template <int AHEAD, int READS, int PRODUCTS>
__device__ __forceinline__ void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * READS, 0);        // LDS reads
#pragma unroll
  for (int i = 0; i < PRODUCTS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);                    // a matrix instruction
    if (i + AHEAD < PRODUCTS) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// 4 bytes per lane from global memory into LDS, lane i at dst + 4 i.
__device__ __forceinline__ void lds_dma4(const void* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(src), "s"(dst) : "m0");
}

// ---------------------------------------------------------------------------
// Documents. The stages of [lo, hi) that can hold a key of one of the tile's
// documents: the id ranges of the stage and of the tile's rows meet. Each entry of the list
// is the stage's number, with kMixed unless all its keys and all the rows are
// of one document. Four lanes read a stage's ids. Histories of more stages
// than the list holds are walked whole.
// ---------------------------------------------------------------------------
constexpr int kDocStages = 2048;            // 131,072 keys
constexpr int kMixed = 0x8000;

struct DocList {
  uint16_t entry[kDocStages];
  uint8_t kind[kDocStages];                 // 0: passed over, 1: one document, 2: mixed
  int lo[4], hi[4];                         // the waves' id ranges
  int count;
};

// Fills `list` (all threads of a workgroup of four waves; row_doc: the lane's
// row's document, of a row that exists). Returns the number of entries, -1: no
// list. Ends with a barrier.
__device__ __forceinline__ int doc_stages(DocList& list, const int32_t* kv_docs, int row_doc, int lo,
                                          int hi) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = (hi - lo + kStageKeys - 1) / kStageKeys;
  if (n > kDocStages) return -1;
  int qlo = row_doc, qhi = row_doc;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    qlo = min(qlo, __shfl_xor(qlo, o));
    qhi = max(qhi, __shfl_xor(qhi, o));
  }
  if (lane == 0) {
    list.lo[wave] = qlo;
    list.hi[wave] = qhi;
  }
  __syncthreads();
  qlo = min(min(list.lo[0], list.lo[1]), min(list.lo[2], list.lo[3]));
  qhi = max(max(list.hi[0], list.hi[1]), max(list.hi[2], list.hi[3]));
  typedef int32_t ids4 __attribute__((ext_vector_type(4), aligned(4)));
  const int part = tid & 3;
  for (int s0 = 0; s0 < n; s0 += 64) {                   // uniform: the shuffles need every lane
    const int s = s0 + tid / 4;
    const int key = lo + min(s, n - 1) * kStageKeys + 16 * part;
    int a = 0x7fffffff, b = -0x7fffffff - 1;
    if (key + 16 <= hi) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const ids4 v = *reinterpret_cast<const ids4*>(kv_docs + key + 4 * i);
        a = min(min(a, min(v[0], v[1])), min(v[2], v[3]));
        b = max(max(b, max(v[0], v[1])), max(v[2], v[3]));
      }
    } else {
      for (int i = 0; i < 16; ++i) {
        const int v = kv_docs[min(key + i, hi - 1)];
        a = min(a, v);
        b = max(b, v);
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      a = min(a, __shfl_xor(a, o));
      b = max(b, __shfl_xor(b, o));
    }
    if (part == 0 && s < n) list.kind[s] = b < qlo || a > qhi ? 0 : a == b && qlo == qhi ? 1 : 2;
  }
  __syncthreads();
  if (wave == 0) {
    int at = 0;
    for (int s0 = 0; s0 < n; s0 += 64) {
      const int k = s0 + lane < n ? list.kind[s0 + lane] : 0;
      const uint64_t m = __ballot(k != 0);
      if (k != 0)
        list.entry[at + __builtin_popcountll(m & ((1ull << lane) - 1))] =
            (uint16_t)((s0 + lane) | (k == 2 ? kMixed : 0));
      at += __builtin_popcountll(m);
    }
    if (lane == 0) list.count = at;
  }
  __syncthreads();
  return list.count;
}

// SCORE of a call.
inline int score_of(const HistArgs& a) {
  const int cap = a.cap > kCapTurn ? kWideCap : a.cap > 0.f ? kCap : 0;
  return cap | (a.slopes != nullptr ? kBias : 0);
}

// Whether the accumulators hold an infinity or NaN (0 times either is NaN).
template <typename V, int N>
__device__ __forceinline__ bool any_odd(const V (&o)[N], float l) {
  float t = l * 0.f;
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) t = fmaf(o[d][e], 0.f, t);
  return !(t == 0.f);
}

}  // namespace rocs
