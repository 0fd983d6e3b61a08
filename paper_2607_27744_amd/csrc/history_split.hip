// History attention, the bf16 kernel for few rows: 32 rows (token, head of the
// group) of one request a wave.
//
// A single new event has as many rows as a K/V head has query heads, so one
// tile holds them all and the call is a read of K and V. A workgroup's four
// waves take up to four K/V heads of the same keys, which lie next to each
// other in memory (with a head a workgroup, each 256 bytes of a row are read
// from another XCD at another time: 128 ragged histories of 3,125 rows on
// average, 8 heads x 128, at 5.0 TB/s instead of 5.65); what is left of the four
// shares the keys in turn (HW heads x 4 / HW key ways). Each wave stages 32 keys of K
// and of V in LDS of its own by DMA (the next K under the softmax, the next V
// under the next scores), so the waves run freely and two workgroups share a
// CU (64 KiB of LDS at head_dim 128): up to 128 KiB a CU in flight. Long
// histories are cut over workgroups as well (HistArgs::splits). Scores, masks
// and the running max are those of history_tile; the partial softmaxes of one
// head's waves meet in LDS at the end.
// What bounds it: HBM with many or long histories, otherwise the latency of a
// wave's chain of stages: 128 cached histories of 3,125 rows with a distance
// bias 281 us (5.8 TB/s, where a large copy reaches 4.9); one of 2,051 rows, 8
// heads on 2: 9 us and 3 for the join.
#include "history_mfma.h"
#include "launch.h"

namespace rocs {
namespace {

constexpr int kRows = 32;
constexpr int kKeys = 32;                 // keys of a wave's stage
constexpr int kWaves = 4;

template <int D, int SCORE, bool DOCS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void history_split(
    const HistArgs a, int64_t slots) {
  constexpr int KS = D / 16, DB = D / 32, PS = kKeys / 16;
  constexpr int ROWB = 2 * D, CR = D / 8;
  constexpr int STAGE = kKeys * ROWB;
  constexpr int KPI = 1024 / ROWB;        // rows of a DMA load
  constexpr int NI = kKeys / KPI;         // loads of a stage and operand
  constexpr int kAhead = 4;               // fragments in flight (see reads_ahead)
  static_assert(kRows * D * 4 <= 2 * STAGE, "a wave's partial output takes its staging");
  __shared__ __attribute__((aligned(1024))) char lds[kWaves * 2 * STAGE];
  __shared__ __attribute__((aligned(16))) int32_t doc_ids[DOCS ? kWaves * 2 * 64 : 4];
  __shared__ float pm[kWaves][kRows], pl[kWaves][kRows];
  __shared__ int odd[kWaves][kRows];       // by head and row: to form again
  ROCS_LDS char* const lds3 = (ROCS_LDS char*)lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  // Neighbours in the work order, which run at the same time on different XCDs, are the
  // head groups and parts of one history: they read neighbouring memory. Each
  // eight are rotated against the eight before, so that no XCD gets only the
  // last parts, which most histories do not reach.
  const uint32_t b8 = blockIdx.x & ~7u;
  const uint32_t work = b8 + 8 > gridDim.x ? blockIdx.x : b8 + ((blockIdx.x + (blockIdx.x >> 3)) & 7u);
  const int HW = a.heads, KW = kWaves / HW;
  const uint32_t groups_n = (uint32_t)(a.Hk / HW);
  const int hk0 = (int)(work % groups_n) * HW, hk = hk0 + wave % HW;
  const uint32_t rest = work / groups_n;
  const int split = (int)(rest % (uint32_t)a.splits);
  const HistTile t = hist_tile(a, slots - 1 - rest / (uint32_t)a.splits, kRows);
  if (t.rows <= 0) return;
  if (tid < kWaves * kRows) odd[0][tid] = 0;

  const int row = t.row0 + min(l32, t.rows - 1);              // clamped; extra rows never stored
  const int token = row / a.G, head = hk * a.G + row % a.G;
  RowRule rule;
  score_rules<SCORE>(rule, a, head);
  rule.pos = position_of(t, token);
  rule.lim = limit_of(a, t, token);
  rule.doc = DOCS ? a.q_docs[t.q0 + token] : 0;
  const int first = t.row0 / a.G, last = (t.row0 + t.rows - 1) / a.G;
  const int lim_lo = limit_of(a, t, first);
  const int plain = DOCS ? 0 : (SCORE & kBias) != 0 ? min(lim_lo, position_of(t, first) + 1) : lim_lo;
  const int most = limit_of(a, t, last);
  const int lo = split * a.chunk, hi = split_end(a, split, most);
  const bool alone = tile_alone(a, most), direct = a.splits == 1 || alone;
  if (alone && split > 0) return;

  const KeyFeed feed(a, t);
  const char* kbase = reinterpret_cast<const char*>(static_cast<const bf16_t*>(a.k) + (int64_t)hk * a.D);
  const char* vbase = reinterpret_cast<const char*>(static_cast<const bf16_t*>(a.v) + (int64_t)hk * a.D);
  const uint32_t kdst = lds_addr(lds) + (uint32_t)(wave * 2 * STAGE);
  const uint32_t ids0 = DOCS ? lds_addr(doc_ids) + (uint32_t)(wave * 2 * 64 * 4) : 0;
  // Load i of a stage fills rows KPI i + lane / CR (of group KPI i / 16), chunk
  // position lane % CR, with chunk (lane % CR) ^ kv_swizzle.
  const int top = a.D / 8 - 1;            // the head's last chunk stands in past its end
  auto issue = [&](const char* src, int base, const int64_t (&off)[2], uint32_t dst) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const char* s = uniform_ptr(src + off[g]);
      const int end = hi - 1 - min(base + 16 * g, (hi - 1) & ~15);   // last row that there is
#pragma unroll
      for (int i = 0; i < NI / 2; ++i) {
        const int r = KPI * i + lane / CR;
        lds_dma16_sv(s, (uint32_t)(min(r, end) * feed.row_bytes) + 16u * (uint32_t)min((lane % CR) ^ kv_swizzle<D>(r), top),
                     dst + 1024u * (NI / 2 * g + i));
      }
    }
  };
  auto groups = [&](int base, int64_t (&off)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < 2; ++g) off[g] = feed.group(min(base + 16 * g, (hi - 1) & ~15));
  };
  auto issue_k = [&](int base, const int64_t (&off)[2], int slot) __attribute__((always_inline)) {
    if constexpr (DOCS) lds_dma4(a.kv_docs + t.kv0 + min(base + lane, hi - 1), ids0 + 256u * slot);
    issue(kbase, base, off, kdst);
  };
  int base = lo + kKeys * (wave / HW);
  int64_t off[2];
  if (base < hi) {
    groups(base, off);
    issue_k(base, off, 0);
    issue(vbase, base, off, kdst + STAGE);
  }
  // The query rows, with the first stage in flight; resident before the loop,
  // in which only DMA loads are in flight, which its waits count.
  bf16x8 qf[KS];
  {
    const bf16_t* q = static_cast<const bf16_t*>(a.q) + (t.q0 + token) * a.q_stride + (int64_t)head * a.D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = as_bf16x8(load16(q + 16 * ks + 8 * hh, 16 * ks + 8 * hh < a.D));
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" :: "v"(as_u32x4(qf[ks])));

  const uint32_t kb0 = (uint32_t)(wave * 2 * STAGE);
  const uint32_t ka0 = kb0 + (uint32_t)(l32 * ROWB + 16 * (hh ^ kv_swizzle<D>(l32)));
  uint32_t va0[2];
#pragma unroll
  for (int rr = 0; rr < 2; ++rr) {
    const int g = lane >> 4, jl = lane & 15;
    const int key = 4 * (g >> 1) + 8 * rr + (jl >> 2);
    const int chunk0 = 2 * (g & 1) + ((jl & 3) >> 1);
    va0[rr] = kb0 + (uint32_t)(STAGE + key * ROWB + 16 * (chunk0 ^ kv_swizzle<D>(key)) + 8 * (jl & 1));
  }
  float m = -INFINITY, l_part = 0.f;
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};

  for (int slot = 0; base < hi; base += KW * kKeys, slot ^= 1) {
    const int next = base + KW * kKeys;
    const bool more = next < hi;
    if (more) groups(next, off);
    wait_vmcnt<NI>();                                     // K of this stage (V may be in flight)
    asm volatile("" ::: "memory");
    f32x16 s = {};
    {
      auto frag = [&](int ks) __attribute__((always_inline)) {
        return *reinterpret_cast<const ROCS_LDS bf16x8*>(lds3 + (ka0 ^ (32u * ks)));
      };
      bf16x8 f[kAhead];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < kAhead; ++ks) f[ks] = frag(ks);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = mfma32(f[ks % kAhead], qf[ks], s);
        if (ks + kAhead < KS) f[ks % kAhead] = frag(ks + kAhead);
      }
      reads_ahead<kAhead, 1, KS>();
    }
    wait_lgkmcnt0();                                      // K's fragments are in registers
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    if (more) issue_k(next, off, slot ^ 1);
    if constexpr (SCORE != 0) {
      score_step<SCORE>(s, 0, 0, rule, base, hh, 0.f);
      score_step<SCORE>(s, 0, 1, rule, base, hh, 0.f);
    }
    if (base + kKeys > plain) {
      const ROCS_LDS int32_t* ids = (const ROCS_LDS int32_t*)doc_ids + (DOCS ? (2 * wave + slot) * 64 : 0);
      mask_step<DOCS>(s, 0, 0, rule, base, hh, ids);
      mask_step<DOCS>(s, 0, 1, rule, base, hh, ids);
    }
    uint32_t pk[PS][4];
    auto weights = [&](float ms) __attribute__((always_inline)) {
      const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
      float part[PS];
#pragma unroll
      for (int ps = 0; ps < PS; ++ps) {
        part[ps] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {                     // each pair a scalar of its own
          float e0 = s[8 * ps + 2 * w], e1 = s[8 * ps + 2 * w + 1];
          if constexpr (SCORE == 0) {
            e0 = fmaf(e0, rule.scale2, -ms);
            e1 = fmaf(e1, rule.scale2, -ms);
          } else {
            e0 -= ms;
            e1 -= ms;
          }
          pk[ps][w] = pack_bf16x2(__builtin_amdgcn_exp2f(e0), __builtin_amdgcn_exp2f(e1));
          part[ps] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[ps][w]), ones, part[ps], false);
        }
      }
      static_assert(PS == 2, "two sums");
      return part[0] + part[1];
    };
    float sum = weights(m);
    if (__builtin_expect(__ballot(!(sum <= kStageBound)) != 0, 0)) {
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
      mx = max_across_halves(mx) * (SCORE == 0 ? rule.scale2 : 1.0f);
      const bool need = mx > m + kLazyMove;
      const float alpha = need ? exp2f(m - mx) : 1.0f;
      if (need) m = mx;
      l_part *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
      sum = weights(m == -INFINITY ? 0.f : m);            // no key seen yet: weights 0
    }
    l_part += sum;
    if (more) wait_vmcnt<NI + (DOCS ? 1 : 0)>(); else wait_vmcnt<0>();   // V of this stage
    asm volatile("" ::: "memory");
    {
      auto frag = [&](int i) __attribute__((always_inline)) {
        const uint32_t o = (i / DB) * 16 * ROWB, db = i % DB;
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (ROCS_LDS i16x4*)(lds3 + ((va0[0] ^ (64u * db)) + o))));
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (ROCS_LDS i16x4*)(lds3 + ((va0[1] ^ (64u * db)) + o))));
        return as_bf16x8(u32x4{x[0], x[1], y[0], y[1]});
      };
      bf16x8 f[kAhead];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) f[i] = frag(i);
#pragma unroll
      for (int i = 0; i < PS * DB; ++i) {
        const uint32_t (&w)[4] = pk[i / DB];
        oacc[i % DB] = mfma32(f[i % kAhead], as_bf16x8(u32x4{w[0], w[1], w[2], w[3]}), oacc[i % DB]);
        if (i + kAhead < PS * DB) f[i % kAhead] = frag(i + kAhead);
      }
      reads_ahead<kAhead, 2, PS * DB>();
    }
    wait_lgkmcnt0();                                      // V's fragments are in registers
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    if (more) issue(vbase, next, off, kdst + STAGE);
  }

  // This wave's partial softmax into its staging area, 16-byte pieces of a row
  // swizzled by the row: element 4 q + i of oacc[db] is O[l32][32 db + 8 q + 4 hh + i].
  const float l_sum = sum_across_halves(l_part);
  if (hh == 0) {
    pm[wave][l32] = m;
    pl[wave][l32] = l_sum;
  }
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<ROCS_LDS f32x4*>(lds3 + kb0 + l32 * D * 4 + 16 * ((8 * db + 2 * q + hh) ^ (l32 & 15))) =
          f32x4{oacc[db][4 * q], oacc[db][4 * q + 1], oacc[db][4 * q + 2], oacc[db][4 * q + 3]};
  __syncthreads();
  // 16-byte pieces of (head, row); the head's waves are hs, hs + HW, ..
  const int CF = a.D / 4;
  for (int c = tid; c < HW * t.rows * CF; c += 256) {
    const int piece = c % CF, i = c / CF % t.rows, hs = c / CF / t.rows;
    float mx = pm[hs][i];
    for (int w = hs + HW; w < kWaves; w += HW) mx = fmaxf(mx, pm[w][i]);
    const float ms = mx == -INFINITY ? 0.f : mx;
    float l = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int w = hs; w < kWaves; w += HW) {
      const float f = exp2f(pm[w][i] - ms);
      l += pl[w][i] * f;
      y += *reinterpret_cast<const ROCS_LDS f32x4*>(lds3 + w * 2 * STAGE + i * D * 4 + 16 * (piece ^ (i & 15))) * f;
    }
    if (!(finite(y[0]) && finite(y[1]) && finite(y[2]) && finite(y[3])) && may_differ(l, a.D, D)) odd[hs][i] = 1;
    const int rw = t.row0 + i;
    const int64_t at = (t.q0 + rw / a.G) * a.H + (hk0 + hs) * a.G + rw % a.G;
    const int64_t to = (int64_t)split * a.N * a.H + at;
    if (a.splits > 1 && piece == 0) {
      a.part_ml[2 * to] = mx;
      a.part_ml[2 * to + 1] = alone ? kDone : l;
    }
    if (!direct) {
      if (l != 0.f) *reinterpret_cast<f32x4*>(a.part_o + to * a.D + 4 * piece) = y;
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      *reinterpret_cast<u32x2*>(static_cast<bf16_t*>(a.out) + at * a.D + 4 * piece) =
          u32x2{pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv)};
    }
  }
  __syncthreads();
  for (int i = wave; i < HW * t.rows; i += kWaves)        // see lone_row
    if (__builtin_amdgcn_readfirstlane(odd[i / t.rows][i % t.rows]) != 0)
      redo_row<bf16_t>(a, t, t.row0 + i % t.rows, hk0 + i / t.rows, lo, hi, split, direct);
}

template <int D, int SCORE>
hipError_t launch_score(const HistArgs& a, int64_t slots, int64_t blocks, hipStream_t s) {
  return launch_kernel(a.q_docs != nullptr ? history_split<D, SCORE, true> : history_split<D, SCORE, false>,
                       dim3((uint32_t)blocks), dim3(256), s, a, slots);
}

template <int D>
hipError_t launch_dim(const HistArgs& a, int64_t slots, int64_t blocks, hipStream_t s) {
  switch (score_of(a)) {
    case kCap: return launch_score<D, kCap>(a, slots, blocks, s);
    case kWideCap: return launch_score<D, kWideCap>(a, slots, blocks, s);
    case kBias: return launch_score<D, kBias>(a, slots, blocks, s);
    case kCap | kBias: return launch_score<D, kCap | kBias>(a, slots, blocks, s);
    case kWideCap | kBias: return launch_score<D, kWideCap | kBias>(a, slots, blocks, s);
    default: return launch_score<D, 0>(a, slots, blocks, s);
  }
}

}  // namespace

hipError_t launch_history_split(const HistArgs& a, hipStream_t s) {
  const int64_t slots = a.R + (a.N * a.G + kRows - 1) / kRows;
  const int64_t blocks = slots * (a.Hk / a.heads) * a.splits;
  if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
  return a.D > 64 ? launch_dim<128>(a, slots, blocks, s) : launch_dim<64>(a, slots, blocks, s);
}

}  // namespace rocs
