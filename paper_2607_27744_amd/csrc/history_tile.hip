// History attention, the tiled bf16 kernel: 128 rows (token, head) of one
// request and K/V head a workgroup.
//
// Structure and reasons are those of the candidate attention's tiled kernel
// (dca_attn_bf16): four waves of 32 rows share K/V stages of 64 keys that come
// into two-slot LDS rings by DMA, K two stages and V one stage ahead; the
// scores of the next stage run on the matrix cores while the VALU forms the
// weights of this one; weights are taken against a running max that moves only
// when a stage could pass 2^64. What differs:
//
// Masks. A row sees a leading run of keys (causal, prefix, the history's end)
// and, with documents, part of it. A wave ends with the stage that its last
// row sees, and stages that all its rows see whole run without a test: two
// copies of the stage, the masked one with the general form of the bias.
// The rows of a tile need not have seen a key yet when a stage starts
// (documents), so a row's max may stay -inf; its weights are then 0.
// Work order. Under the causal mask a request's last tiles are the longest:
// they come first, so that the launch does not end with them. An XCD takes one
// head (or few) and a run of requests (see launch_history_tile).
// Head dims. D is 64 or 128; a head_dim below it (a multiple of 8) has zeros in
// the query fragments' places past its end, its last 16 bytes once more in the
// K/V stage's, and those columns of the result are not stored.
// Grouped heads. Rows are (token, head of the group), so the heads of a group
// share the K/V stage.
//
// What bounds it, in long calls: the matrix cores and the VALU together, at a
// clock that the power holds down (one history of 16,384 rows, 8 heads x 128,
// causal: 480 us, 1,145 TFLOP/s; a large bf16 product reaches 1,258). A cap
// makes it the VALU (three transcendentals a score, 690 TFLOP/s). Where ragged
// histories are a few stages long, latency: from a tile's start to its first
// stage, and between stages of which half are masked (256 of 640 rows, 4 heads x
// 64, with a bias: 146 us, 442 TFLOP/s, 2.3 TB/s).
#include "history_mfma.h"
#include "launch.h"

namespace rocs {
namespace {

constexpr int kRows = 128;
constexpr int kRing = 2;

template <int D, int SCORE, bool DOCS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2))) void
history_tile(const HistArgs a, int64_t slots) {
  constexpr int KB = 2, KS = D / 16, DB = D / 32, PS = 4;
  constexpr int ROWB = 2 * D, CR = D / 8;
  constexpr int STAGE = kStageKeys * ROWB;
  constexpr int KPI = 1024 / ROWB;          // rows of a DMA load
  constexpr int NI = 16 / KPI;              // loads a wave, operand and stage (its 16 rows)
  __shared__ __attribute__((aligned(1024))) char lds[2 * kRing * STAGE];
  __shared__ __attribute__((aligned(16))) int32_t doc_ids[DOCS ? 2 * kStageKeys : 4];
  __shared__ typename std::conditional<DOCS, DocList, int>::type doc_list;
  ROCS_LDS char* const lds3 = (ROCS_LDS char*)lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const uint32_t per_head = (uint32_t)slots * (uint32_t)a.splits;
  uint32_t hk, rest;
  if (a.deal > 1) {
    const uint32_t m = (uint32_t)a.deal, xcd = blockIdx.x % kNumXcd;
    hk = xcd / m;
    rest = blockIdx.x / kNumXcd * m + xcd % m;
    if (rest >= per_head) return;
  } else {
    const uint32_t work = xcd_remap(blockIdx.x, gridDim.x);
    hk = work / per_head;
    rest = work - hk * per_head;
  }
  const int split = (int)(rest % (uint32_t)a.splits);
  const HistTile t = hist_tile(a, slots - 1 - rest / (uint32_t)a.splits, kRows);
  if (t.rows <= 0) return;

  const int wrow0 = wave * 32;
  const bool active = wrow0 < t.rows;
  const int row = t.row0 + min(wrow0 + l32, t.rows - 1);      // clamped; extra rows never stored
  const int token = row / a.G, head = hk * a.G + row % a.G;
  RowRule rule;
  score_rules<SCORE>(rule, a, head);
  rule.pos = position_of(t, token);
  rule.lim = limit_of(a, t, token);
  rule.doc = DOCS ? a.q_docs[t.q0 + token] : 0;
  // The wave's first and last rows bound what it sees.
  const int first = (t.row0 + min(wrow0, t.rows - 1)) / a.G;
  const int last = (t.row0 + min(wrow0 + 31, t.rows - 1)) / a.G;
  const int lim_lo = limit_of(a, t, first);
  const int lim_hi = active ? limit_of(a, t, last) : 0;
  const int plain = (SCORE & kBias) != 0 ? min(lim_lo, position_of(t, first) + 1) : lim_lo;
  const int most = limit_of(a, t, (t.row0 + t.rows - 1) / a.G);
  const int lo = split * a.chunk, hi = split_end(a, split, most);
  const bool alone = tile_alone(a, most), direct = a.splits == 1 || alone;
  if (alone && split > 0) return;

  bf16x8 qf[KS];
  {
    const bf16_t* q = static_cast<const bf16_t*>(a.q) + (t.q0 + token) * a.q_stride + (int64_t)head * a.D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = as_bf16x8(load16(q + 16 * ks + 8 * hh, 16 * ks + 8 * hh < a.D));
  }

  const KeyFeed feed(a, t);
  const char* kbase = reinterpret_cast<const char*>(static_cast<const bf16_t*>(a.k) + (int64_t)hk * a.D);
  const char* vbase = reinterpret_cast<const char*>(static_cast<const bf16_t*>(a.v) + (int64_t)hk * a.D);
  // DMA lane map: load i of this wave's 16 rows of a stage fills rows KPI i +
  // lane / CR, chunk position lane % CR, with chunk (lane % CR) ^ kv_swizzle.
  int srow[NI];
  uint32_t schunk[NI], soff[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    srow[i] = KPI * i + lane / CR;
    schunk[i] = 16u * (uint32_t)min((lane % CR) ^ kv_swizzle<D>(srow[i]), a.D / 8 - 1);
    soff[i] = (uint32_t)(srow[i] * feed.row_bytes) + schunk[i];
  }
  const uint32_t lds_base = lds_addr(lds);
  // This wave's group of the stage at key `base`: past the end the group of
  // the last key stands in.
  auto group_of = [&](int base) __attribute__((always_inline)) {
    return feed.group(min(base + 16 * wave, (hi - 1) & ~15));
  };
  auto issue = [&](const char* src, int base, int64_t off, uint32_t dst) __attribute__((always_inline)) {
    const char* s = uniform_ptr(src + off);
    dst += 16 * wave * ROWB;
    if (base + 16 * wave + 16 <= hi) {
#pragma unroll
      for (int i = 0; i < NI; ++i) lds_dma16_sv(s, soff[i], dst + 1024u * i);
    } else {
      const int end = hi - 1 - min(base + 16 * wave, (hi - 1) & ~15);    // last row of the group
#pragma unroll
      for (int i = 0; i < NI; ++i)
        lds_dma16_sv(s, (uint32_t)(min(srow[i], end) * feed.row_bytes) + schunk[i], dst + 1024u * i);
    }
  };
  auto issue_k = [&](int slot, int base, int64_t off) { issue(kbase, base, off, lds_base + slot * STAGE); };
  auto issue_v = [&](int slot, int base, int64_t off) {
    issue(vbase, base, off, lds_base + (kRing + slot) * STAGE);
    if constexpr (DOCS) {
      if (wave == 0)
        lds_dma4(a.kv_docs + t.kv0 + min(base + lane, hi - 1), lds_addr(doc_ids) + 4u * kStageKeys * slot);
    }
  };

  const uint32_t ka0 = (uint32_t)(l32 * ROWB + 16 * (hh ^ kv_swizzle<D>(l32)));
  uint32_t va0[2];
#pragma unroll
  for (int rr = 0; rr < 2; ++rr) {
    const int g = lane >> 4, jl = lane & 15;
    const int key = 4 * (g >> 1) + 8 * rr + (jl >> 2);
    const int chunk0 = 2 * (g & 1) + ((jl & 3) >> 1);
    va0[rr] = (uint32_t)(kRing * STAGE + key * ROWB + 16 * (chunk0 ^ kv_swizzle<D>(key)) + 8 * (jl & 1));
  }

  int n = hi > lo ? (hi - lo + kStageKeys - 1) / kStageKeys : 0;
  bool listed = false;
  if constexpr (DOCS) {
    if (n > 0) {
      const int found = doc_stages(doc_list, a.kv_docs + t.kv0, rule.doc, lo, hi);
      listed = found >= 0;
      if (listed) n = found;
    }
  }
  // First key of the i-th stage; mixed: keys of it may be of another document
  // than rows of the tile.
  auto stage_at = [&](int i, bool& mixed) __attribute__((always_inline)) -> int {
    if constexpr (DOCS) {
      const int e = listed ? __builtin_amdgcn_readfirstlane((int)doc_list.entry[i]) : i;
      mixed = !listed || (e & kMixed) != 0;
      return lo + (listed ? e & (kMixed - 1) : i) * kStageKeys;
    }
    mixed = false;
    return lo + i * kStageKeys;
  };

  float m_run = -INFINITY, l_part = 0.f;
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};

  // Products run with their K or V fragments read kAhead ahead of them (left alone, the
  // compiler waits for the latency of each).
  constexpr int kAhead = D == 64 ? 2 : 3, NM = KS * KB;
  auto k_frag = [&](int slot, int i) __attribute__((always_inline)) {
    return *reinterpret_cast<const ROCS_LDS bf16x8*>(
        lds3 + ((ka0 ^ (32u * (i / KB))) + slot * STAGE + (i % KB) * 32 * ROWB));
  };
  // Scores of the stage in K's slot.
  auto qk = [&](int slot, f32x16 (&s)[KB]) __attribute__((always_inline)) {
    bf16x8 kf[kAhead];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) s[kb] = f32x16{};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) kf[i] = k_frag(slot, i);
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      s[i % KB] = mfma32(kf[i % kAhead], qf[i / KB], s[i % KB]);
      if (i + kAhead < NM) kf[i % kAhead] = k_frag(slot, i + kAhead);
    }
    reads_ahead<kAhead, 1, NM>();
  };
  // Weights of step ps as packed bf16 B fragments, from scores in exp2 units less
  // the max. bf16 weights let their product with V run at eight times the
  // rate of the fp32 instruction; the row's sum adds the rounded weights, so that
  // a common part of the rounding cancels. Results are off by 2.1e-3 relative,
  // 1.7e-3 of it their own rounding to bf16 (the errors' squares add). Each pair
  // is a scalar of its own (see dca_attn_bf16).
  const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
  auto weights = [&](const f32x16 (&s)[KB], int ps, uint32_t (&pk)[4], float& sum) __attribute__((always_inline)) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int el = 8 * (ps % 2) + 2 * w;
      pk[w] = pack_bf16x2(__builtin_amdgcn_exp2f(s[ps / 2][el]), __builtin_amdgcn_exp2f(s[ps / 2][el + 1]));
      sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[w]), ones, sum, false);
    }
  };
  auto row_max = [&](const f32x16& s) __attribute__((always_inline)) {
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    return mx;
  };
  // The stage's weights could pass 2^64 (or are not finite): the running max of the
  // rows that need it moves to mx, and what has been summed is rescaled.
  auto move_max = [&](float mx) __attribute__((always_inline)) {
    const bool need = mx > m_run + kLazyMove;
    const float alpha = need ? exp2f(m_run - mx) : 1.0f;       // 0 for a row's first keys
    if (need) m_run = mx;
    l_part *= alpha;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
    return m_run == -INFINITY ? 0.f : m_run;                   // no key seen yet: weights 0
  };
  // V times the weights of `count` 16-key steps from ps0.
  auto pv = [&](int slot, int ps0, auto count, const uint32_t (&pk)[decltype(count)::value][4])
      __attribute__((always_inline)) {
    constexpr int NF = decltype(count)::value * DB;
    auto frag = [&](int i) __attribute__((always_inline)) {
      const int db = i % DB;
      const uint32_t off = slot * STAGE + (ps0 + i / DB) * 16 * ROWB;
      const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (ROCS_LDS i16x4*)(lds3 + ((va0[0] ^ (64u * db)) + off))));
      const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (ROCS_LDS i16x4*)(lds3 + ((va0[1] ^ (64u * db)) + off))));
      return as_bf16x8(u32x4{x[0], x[1], y[0], y[1]});
    };
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 vf[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) vf[i] = frag(i);
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const uint32_t (&w)[4] = pk[i / DB];
      oacc[i % DB] = mfma32(vf[i % kAhead], as_bf16x8(u32x4{w[0], w[1], w[2], w[3]}), oacc[i % DB]);
      if (i + kAhead < NF) vf[i % kAhead] = frag(i + kAhead);
    }
    reads_ahead<kAhead, 2, NF>();
  };
  // A stage that every row of the wave sees whole: its weights and PV product,
  // with the scores of the next stage on the matrix cores meanwhile. A matrix
  // instruction holds up its wave until the last one is through, so they are
  // dealt out: step i issues one product and forms two weights, of which each
  // transcendental waits a step for the one before it (D = 128; 16 requests of
  // 2,048 rows behind a prefix, 8 heads on 2, capped: 323 us in the compiler's
  // order, 281 so; one of 16,384 rows, 8 heads, no cap: 530 and 480).
  auto stage = [&](int slot, int base, f32x16 (&s)[KB], f32x16 (&sn)[KB]) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) sn[kb] = f32x16{};
    uint32_t pk[PS][4];
    float sum = 0.f, reach = 0.f;
    constexpr int NP = 4 * PS, LAG = (SCORE & kCap) != 0 ? 2 : 0;  // pairs; steps from score to weight
    bf16x8 kf[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) kf[i] = k_frag(slot ^ 1, i);
    const float lin = plain_shift<SCORE>(rule, base, hh) - m_run;
    float x[NP][2];
#pragma unroll
    for (int i = 0; i < NP + LAG + 1; ++i) {
      if (i < NP && i % (NP / NM) == 0) {
        const int j = i / (NP / NM);
        sn[j % KB] = mfma32(kf[j % kAhead], qf[j / KB], sn[j % KB]);
        if (j + kAhead < NM) kf[j % kAhead] = k_frag(slot ^ 1, j + kAhead);
      }
      const int d = i - LAG - 1;
      if (d >= 0 && d < NP) {
        pk[d / 4][d % 4] = pack_bf16x2(x[d][0], x[d][1]);
        sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[d / 4][d % 4]), ones, sum, false);
      }
      float in[3][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        auto raw = [&](int at) __attribute__((always_inline)) { return s[at / 8][2 * (at % 8) + h]; };
        auto key = [&](int at) { return 32 * (at / 8) + 8 * ((2 * (at % 8)) / 4) + (2 * (at % 8)) % 4 + h; };
        if constexpr ((SCORE & kCap) != 0) {
          if (i < NP) in[0][h] = raw(i) * rule.cap_in;
          if (i >= 1 && i - 1 < NP) in[1][h] = 1.0f + x[i - 1][h];
          if (i >= 2 && i - 2 < NP) {
            float shift = lin;
            if constexpr ((SCORE & kBias) != 0) shift = fmaf(rule.slope2, (float)key(i - 2), shift);
            in[2][h] = fmaf(-2.0f * rule.cap2, x[i - 2][h], shift);
          }
        } else {
          if (i < NP) in[0][h] = plain_score<SCORE>(raw(i), key(i), rule, lin, reach);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (i < NP) x[i][h] = __builtin_amdgcn_exp2f(in[0][h]);
        if (LAG == 2 && i >= 1 && i - 1 < NP) x[i - 1][h] = __builtin_amdgcn_rcpf(in[1][h]);
        if (LAG == 2 && i >= 2 && i - 2 < NP) x[i - 2][h] = __builtin_amdgcn_exp2f(in[2][h]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    bool again = !(sum <= kStageBound);
    if constexpr ((SCORE & kWideCap) != 0) again = again || !(reach <= kSeriesEnd);
    if (__builtin_expect(__ballot(again) != 0, 0)) {
      RowRule anew = rule;
      // (Laundered: or what the first pass formed is kept for this one, in scratch.)
      if constexpr ((SCORE & kWideCap) != 0) asm volatile("" : "+v"(anew.cap_in));
#pragma unroll
      for (int ps = 0; ps < PS; ++ps) score_step<SCORE>(s[ps / 2], ps / 2, ps % 2, anew, base, hh, 0.f);
      const float ms = move_max(max_across_halves(fmaxf(row_max(s[0]), row_max(s[1]))));
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] -= ms;
      sum = 0.f;
#pragma unroll
      for (int ps = 0; ps < PS; ++ps) weights(s, ps, pk[ps], sum);
    }
    l_part += sum;
    __builtin_amdgcn_s_setprio(1);
    pv(slot, 0, std::integral_constant<int, PS>{}, pk);
    __builtin_amdgcn_s_setprio(0);
  };
  // Half a stage (32 keys) of any other kind: the mask, where rows without a max
  // so far take theirs before the weights, and no work for keys that no row sees.
  auto half = [&](int slot, int base, int kb, f32x16 (&s)[KB]) __attribute__((always_inline)) {
    const int key = base + 32 * kb;
    if (key >= lim_hi) return;
    const ROCS_LDS int32_t* ids = (const ROCS_LDS int32_t*)doc_ids + (DOCS ? kStageKeys * slot : 0);
    float ref = m_run == -INFINITY ? 0.f : m_run;              // what the scores are less
#pragma unroll
    for (int h = 0; h < 2; ++h) score_step<SCORE>(s[kb], kb, h, rule, base, hh, ref);
    if (DOCS || key + 32 > lim_lo) {
#pragma unroll
      for (int h = 0; h < 2; ++h) mask_step<DOCS>(s[kb], kb, h, rule, base, hh, ids);
    }
    if (__ballot(m_run == -INFINITY) != 0) {
      const float mx = max_across_halves(row_max(s[kb]));
      if (m_run == -INFINITY) m_run = mx;                      // nothing summed yet
      const float to = m_run == -INFINITY ? 0.f : m_run;
      s[kb] -= to - ref;
      ref = to;
    }
    uint32_t pk[2][4];
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) weights(s, 2 * kb + h, pk[h], sum);
    if (__builtin_expect(__ballot(!(sum <= kStageBound)) != 0, 0)) {
      s[kb] -= move_max(max_across_halves(row_max(s[kb])) + ref) - ref;
      sum = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) weights(s, 2 * kb + h, pk[h], sum);
    }
    if (DOCS && __ballot(sum != 0.f) == 0) return;
    l_part += sum;
    pv(slot, 2 * kb, std::integral_constant<int, 2>{}, pk);
  };

  if (n > 0) {
    // The wave's own stages, and how many of them (each with a stage after it)
    // need no mask.
    int nw = 0, free = 0;
    if constexpr (DOCS) {
      if (listed) {
        for (int i = 0; i < n; i += 64)
          nw += __builtin_popcountll(__ballot(
              i + lane < n && lo + (doc_list.entry[i + lane] & (kMixed - 1)) * kStageKeys < lim_hi));
      } else {
        nw = max(min(n, (lim_hi - lo + kStageKeys - 1) / kStageKeys), 0);
      }
    } else {
      nw = max(min(n, (lim_hi - lo + kStageKeys - 1) / kStageKeys), 0);
      free = max(min((plain - lo) / kStageKeys, nw - 1), 0);
    }
    nw = __builtin_amdgcn_readfirstlane(nw);
    // The stages at kt, kt + 1 and kt + 2 (first keys), and the group offsets
    // of the two that are still to be loaded; a stage's table entry is read a
    // step before its first load.
    bool x0, x1, x2;
    int b0 = stage_at(0, x0), b1 = stage_at(min(1, n - 1), x1), b2 = stage_at(min(2, n - 1), x2);
    const int64_t o0 = group_of(b0);
    int64_t o1 = group_of(b1), o2 = group_of(b2);
    issue_k(0, b0, o0);
    issue_v(0, b0, o0);
    if (n > 1) issue_k(1, b1, o1);
    wait_vmcnt<0>();                                      // the query fragments included
    ring_barrier();
    f32x16 s_a[KB], s_b[KB];
    if (nw > 0) qk(0, s_a);
    ring_barrier();                                       // K slot 0 has been read
    // A step reads K of stage kt + 1 and V of stage kt; their other slots were
    // released by the last barrier and take K of kt + 2 and V of kt + 1.
    auto load = [&](int kt, int slot) __attribute__((always_inline)) {
      if (kt + 2 < n) issue_k(slot, b2, o2);
      if (kt + 1 < n) issue_v(slot ^ 1, b1, o1);
    };
    auto pass = [&](int kt) __attribute__((always_inline)) {
      b0 = b1;
      b1 = b2;
      x0 = x1;
      x1 = x2;
      o1 = o2;
      if (kt + 3 < n) {
        b2 = stage_at(kt + 3, x2);
        o2 = group_of(b2);
      }
      wait_vmcnt<0>();
      ring_barrier();
    };
    int kt = 0;
    auto step = [&](int slot, f32x16 (&cur)[KB], f32x16 (&nxt)[KB]) __attribute__((always_inline)) {
      load(kt, slot);
      stage(slot, b0, cur, nxt);
      pass(kt);
      ++kt;
    };
    // A stage with a mask, then the next scores: in step with them it would need
    // more registers than there are.
    auto masked = [&]() __attribute__((always_inline)) {
      const int slot = kt & 1;
      load(kt, slot);
      half(slot, b0, 0, s_a);
      half(slot, b0, 1, s_a);
      if (kt + 1 < nw) qk(slot ^ 1, s_a);
      pass(kt);
      ++kt;
    };
    if constexpr (DOCS) {
      // Packed documents: a document's first stages, its whole ones, the last.
      // (With a bias at head_dim 128 both forms do not fit the registers.)
      if constexpr (D == 64 || (SCORE & kBias) == 0) {
        auto whole = [&]() __attribute__((always_inline)) {
          return kt + 2 < nw && !x0 && !x1 && b1 + kStageKeys <= plain;
        };
        while (kt < nw && !whole()) masked();
        while (whole()) {
          const int slot = kt & 1;
          step(slot, s_a, s_b);
          step(slot ^ 1, s_b, s_a);
        }
      }
    } else {
      // The first stage finds the rows' max before its weights, as masked ones do.
      if (nw > 0) masked();
      while (kt + 1 < free) {                             // the score buffers swap roles
        step(1, s_a, s_b);
        step(0, s_b, s_a);
      }
    }
    while (kt < nw) masked();
    for (; kt < n; ++kt) {                                // the other waves' stages
      load(kt, kt & 1);
      pass(kt);
    }
  }

  // Epilogue. The addresses come from a laundered lane index, so that they are
  // not held through the main loop.
  if (!active) return;
  int lane_e = lane;
  asm volatile("" : "+v"(lane_e));
  const int l32e = lane_e & 31, hhe = lane_e >> 5;
  const float l = sum_across_halves(l_part);
  const uint64_t odd = __ballot(any_odd(oacc, l) && may_differ(l, a.D, D));
  const int mine = min(t.rows - wrow0, 32);
  uint32_t again = ((uint32_t)odd | (uint32_t)(odd >> 32)) & (mine == 32 ? ~0u : (1u << mine) - 1u);
  auto out_row = [&](int i) -> int64_t {                  // row i of the wave
    const int rw = t.row0 + wrow0 + i;
    return (t.q0 + rw / a.G) * a.H + hk * a.G + rw % a.G;
  };
  if (a.splits > 1 && l32e < mine) {
    const int64_t to = (int64_t)split * a.N * a.H + out_row(l32e);
    if (hhe == 0) {
      a.part_ml[2 * to] = m_run;
      a.part_ml[2 * to + 1] = alone ? kDone : l;
    }
    if (!direct && l != 0.f) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (32 * db + 8 * q < a.D)
            *reinterpret_cast<f32x4*>(a.part_o + to * a.D + 32 * db + 8 * q + 4 * hhe) =
                f32x4{oacc[db][4 * q], oacc[db][4 * q + 1], oacc[db][4 * q + 2], oacc[db][4 * q + 3]};
    }
  }
  if (direct) {
    // Through this wave's share of the idle ring: row-contiguous stores.
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const uint32_t obase = (uint32_t)(wave * 32 * ROWB);
    auto swz = [](int r) { return CR == 16 ? (r & 15) : ((r >> 1) & 7); };
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f32x16& o = oacc[db];
        const uint32_t e0 = pack_bf16x2(o[8 * j] * inv, o[8 * j + 1] * inv);
        const uint32_t e1 = pack_bf16x2(o[8 * j + 2] * inv, o[8 * j + 3] * inv);
        const uint32_t o0 = pack_bf16x2(o[8 * j + 4] * inv, o[8 * j + 5] * inv);
        const uint32_t o1 = pack_bf16x2(o[8 * j + 6] * inv, o[8 * j + 7] * inv);
        const auto x = __builtin_amdgcn_permlane32_swap(e0, o0, false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(e1, o1, false, false);
        *reinterpret_cast<ROCS_LDS u32x4*>(lds3 + obase + l32e * ROWB +
                                           16 * ((4 * db + 2 * j + hhe) ^ swz(l32e))) =
            u32x4{x[0], y[0], x[1], y[1]};
      }
    constexpr int RPS = 1024 / ROWB, NST = 32 / RPS;
#pragma unroll
    for (int i = 0; i < NST; ++i) {
      const int r = RPS * i + lane_e / CR;
      const u32x4 v = *reinterpret_cast<const ROCS_LDS u32x4*>(
          lds3 + obase + r * ROWB + 16 * ((lane_e % CR) ^ swz(r)));
      if (r < mine && lane_e % CR < a.D / 8)
        *reinterpret_cast<u32x4*>(static_cast<bf16_t*>(a.out) + out_row(r) * a.D + 8 * (lane_e % CR)) = v;
    }
  }
  while (again != 0) {                                    // see lone_row
    const int i = __builtin_ctz(again);
    again &= again - 1;
    redo_row<bf16_t>(a, t, t.row0 + wrow0 + i, hk, lo, hi, split, direct);
  }
}

template <int D, int SCORE>
hipError_t launch_score(const HistArgs& a, int64_t slots, int64_t blocks, hipStream_t s) {
  return launch_kernel(a.q_docs != nullptr ? history_tile<D, SCORE, true> : history_tile<D, SCORE, false>,
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

hipError_t launch_history_tile(const HistArgs& args, hipStream_t s) {
  HistArgs a = args;
  const int64_t slots = a.R + (a.N * a.G + kRows - 1) / kRows, per_head = slots * a.splits;
  // Where m XCDs share a head, each takes a run of its requests, whose K and V then
  // pass through one L2. Few requests that do not come out even leave XCDs idle;
  // those are dealt out tile by tile (one of 16,384 rows, 8 heads on 4: 499 us
  // instead of 753; 3 of 4,096: 124 and 143; on 2 K/V heads 5: 189 and 211, but 11:
  // 388 and 368; 16 of 2,048 on one: 172 and 155).
  const int m = kNumXcd % a.Hk == 0 ? (int)kNumXcd / a.Hk : 1;
  a.deal = a.R % m != 0 && a.R < (2 * m > 8 ? 2 * m : 8) ? m : 1;
  const int64_t blocks = a.deal > 1 ? (per_head + m - 1) / m * kNumXcd : per_head * a.Hk;
  if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
  return a.D > 64 ? launch_dim<128>(a, slots, blocks, s) : launch_dim<64>(a, slots, blocks, s);
}

}  // namespace rocs
