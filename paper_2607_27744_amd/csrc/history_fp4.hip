// Attention over a cache held in 4 bits: the tiled kernel's launch, and the bf16 kernel for few rows: 16
// rows (token, head of the group) of one request a wave.
//
// A call over single events is a read of the cache, of which 4 bits leave a
// quarter of the bytes: what a byte costs in instructions decides. K goes to the
// matrix cores as it is stored: lane (l16, g) holds key l16's dims from D / 4 g on
// (16 bytes at head_dim 128: one block of a scale), which the conversion instruction
// turns into the A operands of D / 32 products; the order of a product's inner dims is
// free as long as q's fragments follow it. Loads have neighbouring lanes on
// neighbouring bytes (loaded in the operands' order, each lane's 16 bytes are a cache
// access of their own: 33 million of them in 128 histories of 3,125 rows, 8 heads, which
// kept the address units busy for half of 151 us), so K's change lanes through LDS.
// V's products run over keys, and a lane has them for one dim: V is converted a
// block a lane (its scale with it) and turned around through LDS, 32 keys at a time, by
// the transposing read. (Turned as codes, a quarter of the LDS bytes, a scale would
// have to go into the weights, of another block and key in each.)
// 16 x 16 x 32 products: the heads of a group rarely fill more rows, and a score
// costs an exponential. Waves and parts share a call as in history_split.
// 128 single rows over 3,125 keys on average, 8 heads x 128: 125 us, 3.4 TB/s (a cache in
// bf16: 287 us at 5.7 TB/s); 48 over 18,750, 16 heads on 2, capped: 91; 1 over 4,099: 8.2.
// With 8 rows of a group two lanes hold the same row and form the same exponentials,
// and K and V are converted for half a tile; the cap costs nothing to speak of (the grouped call with
// none 90 us, 20: 88, 50: 96, 200: 95).
// What bounds it: the loads of a stage and the work on it overlap only over the three
// waves of a SIMD; without the work the loads take 88 us and 20 more for the scales, the
// work alone 78. Two stages of registers (150 us), V's loads before K's products (136),
// equal shares of stages for each workgroup (149) and K's and V's scales in one load (130 with
// the join, 131 without) did not help.
#include "history_tile.h"
#include "launch.h"

namespace rocs {
namespace {

constexpr int kWaves = 4, kFewRows = 16;

// 16-byte chunk of a staged V row at which chunk c of `key` stands: c ^ this. The
// eight rows of a half wave's transposing read and the quarter wave of a write fall on
// distinct banks.
template <int D>
__device__ __forceinline__ int v_swizzle(int key) {
  if constexpr (D == 128) return (key & 3) | ((((key >> 2) & 3) ^ ((key & 1) << 1)) << 2);
  else return ((key >> 1) & 3) | (((key >> 1) & 1) << 2);
}

template <int D, int SCORE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void
history_fp4_few(const HistArgs a, int64_t slots) {
  constexpr int KS = D / 32, DB = D / 16;   // products of a score, output blocks
  constexpr int BPR = D / kFp4Block;        // blocks of a key: V's loads of a lane and stage
  constexpr int ROWB = 2 * D;               // a staged V row
  constexpr int STAGE = 32 * ROWB > kFewRows * D * 4 ? 32 * ROWB : kFewRows * D * 4;
  __shared__ __attribute__((aligned(1024))) char lds[kWaves * STAGE];
  __shared__ float pm[kWaves][kFewRows], pl[kWaves][kFewRows];
  __shared__ int odd[kWaves][kFewRows];        // by head and row: to form again
  ROCS_LDS char* const lds3 = (ROCS_LDS char*)lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  // Head groups of the same keys share cache lines: they follow each other on one XCD.
  // Parts of a history go to XCDs in turn, rotated as in history_split.
  const int HW = a.heads, KW = kWaves / HW;
  const uint32_t groups_n = (uint32_t)(a.Hk / HW), eight = kNumXcd * groups_n;
  uint32_t group = blockIdx.x % groups_n, rest = blockIdx.x / groups_n;
  if (blockIdx.x < gridDim.x / eight * eight) {
    const uint32_t i = blockIdx.x / kNumXcd, turn = i / groups_n;
    group = i % groups_n;
    rest = turn * kNumXcd + ((blockIdx.x + turn) % kNumXcd);
  }
  const int hk0 = (int)group * HW, hk = hk0 + wave % HW;
  const int split = (int)(rest % (uint32_t)a.splits);
  const HistTile t = hist_tile(a, slots - 1 - rest / (uint32_t)a.splits, kFewRows);
  if (t.rows <= 0) return;
  for (int i = tid; i < kWaves * kFewRows; i += 256) odd[i / kFewRows][i % kFewRows] = 0;

  const int row = t.row0 + min(l16, t.rows - 1);              // clamped; extra rows never stored
  const int token = row / a.G, head = hk * a.G + row % a.G;
  RowRule rr;
  score_rules<SCORE>(rr, a, head);
  rr.pos = position_of(t, token);
  rr.lim = limit_of(a, t, token);
  bf16x8 qf[KS];
  const bf16_t* q = static_cast<const bf16_t*>(a.q) + (t.q0 + token) * a.q_stride + (int64_t)head * a.D;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int d = D / 4 * g + 8 * ks;
    qf[ks] = as_bf16x8(load16(q + d, d < a.D));
  }
  const int lim_lo = limit_of(a, t, t.row0 / a.G);
  const int most = limit_of(a, t, (t.row0 + t.rows - 1) / a.G);
  const int lo = split * a.chunk, hi = split_end(a, split, most);
  const bool alone = tile_alone(a, most), direct = a.splits == 1 || alone;
  if (alone && split > 0) return;

  // This lane's block of a row. Below the kernel's own width the head's last ones stand
  // in (q is 0 there, or the result is not stored).
  const Fp4Row fr{a.Hk, a.D};
  const char* const base = static_cast<const char*>(a.k);
  const int vb = min(lane % BPR, a.D / kFp4Block - 1);
  const int k_at = fr.values(0, hk) + 16 * vb, v_at = fr.values(1, hk) + 16 * vb;
  const uint32_t row_bytes = (uint32_t)a.kv_stride;
  const uint32_t st0 = (uint32_t)(wave * STAGE);

  // A stage: 64 keys, loaded a block a lane (the n-th: key 64 / BPR n + lane / BPR); the
  // scales of lane's key, a byte a block.
  u32x4 kw[BPR], vw[BPR];
  uint32_t kse, vse, vsn;
  // (Below the kernel's width one byte ahead of the scales and their last byte instead of one
  // behind, which could lie past the pool.)
  const int ahead = a.D == D ? 0 : 1;
  const int k_byte = min(D / 4 * g / kFp4Block, a.D / kFp4Block - 1) + ahead, v_byte = vb + ahead;
  auto key_scales = [&](const char* p) __attribute__((always_inline)) -> uint32_t {
    typedef uint32_t u32u __attribute__((aligned(1)));
    typedef uint16_t u16u __attribute__((aligned(1)));
    if constexpr (D == 128) return *reinterpret_cast<const u32u*>(p - ahead);
    else return *reinterpret_cast<const u16u*>(p - ahead);
  };
  auto load_k = [&](int rows) __attribute__((always_inline)) {
    // V's with K's: they lie in the same cache lines.
    const char* p = base + (uint64_t)(uint32_t)rows * row_bytes;
    kse = key_scales(p + fr.scales(0, hk));
    vsn = key_scales(p + fr.scales(1, hk));
#pragma unroll
    for (int n = 0; n < BPR; ++n)
      kw[n] = *reinterpret_cast<const u32x4*>(
          base + (uint64_t)(uint32_t)__shfl(rows, 64 / BPR * n + lane / BPR) * row_bytes + k_at);
  };
  auto load_v = [&](int rows) __attribute__((always_inline)) {
    vse = vsn;
#pragma unroll
    for (int n = 0; n < BPR; ++n)
      vw[n] = *reinterpret_cast<const u32x4*>(
          base + (uint64_t)(uint32_t)__shfl(rows, 64 / BPR * n + lane / BPR) * row_bytes + v_at);
  };
  // Staged K codes: rows of D / 2 bytes, chunk c of `key` at c ^ k_swz: the 16 rows that a
  // quarter wave reads (or writes four chunks of) fall on distinct banks.
  auto k_swz = [](int key) { return BPR == 4 ? (key >> 2) & 3 : (key >> 3) & 1; };
  constexpr int KWW = D / 32;               // words of a lane's quarter of a key
  // The row of a stage's key `lane` in two steps: the page table's entry, a stage ahead,
  // and the row from it where it is needed (formed at once it would wait for every load
  // before it). Past the end the last key stands in, and the last stage loads one of
  // that alone: in a branch the loads could not be counted, and each wait would be for all.
  PoolKey next_key;
  auto look_up = [&](int at) __attribute__((always_inline)) { next_key = pool_key(a, t.pages, min(at + lane, hi - 1)); };

  float m = -INFINITY, l_part = 0.f;
  f32x4 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  // Transposing reads of V^T: rows 16 x + 4 g + jl / 4 of the staged 32, 16 dims.
  uint32_t va[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int key = 16 * x + 4 * g + (l16 >> 2);
    va[x] = st0 + (uint32_t)(key * ROWB + 16 * (((l16 & 3) >> 1) ^ v_swizzle<D>(key)) + 8 * (l16 & 1));
  }

  int at = lo + 64 * (wave / HW);
  int rows_now = 0;
  if (at < hi) {
    look_up(at);
    rows_now = pool_row(a, next_key);
    look_up(at + 64 * KW);
    load_k(rows_now);
    load_v(rows_now);
  }
  for (; at < hi; at += 64 * KW) {
    f32x4 s[4];
#pragma unroll
    for (int n = 0; n < BPR; ++n) {
      const int key = 64 / BPR * n + lane / BPR;
      *reinterpret_cast<ROCS_LDS u32x4*>(lds3 + st0 + key * (D / 2) + 16 * ((lane % BPR) ^ k_swz(key))) = kw[n];
    }
    uint32_t kc[4][KWW];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int key = 16 * kb + l16;
      if constexpr (D == 128) {
        const u32x4 x = *reinterpret_cast<const ROCS_LDS u32x4*>(lds3 + st0 + key * 64 + 16 * (g ^ k_swz(key)));
#pragma unroll
        for (int i = 0; i < 4; ++i) kc[kb][i] = x[i];
      } else {
        const u32x2 x = *reinterpret_cast<const ROCS_LDS u32x2*>(
            lds3 + st0 + key * 32 + 16 * ((g >> 1) ^ k_swz(key)) + 8 * (g & 1));
        kc[kb][0] = x[0];
        kc[kb][1] = x[1];
      }
    }
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const uint32_t e = (uint32_t)__shfl((int)kse, 16 * kb + l16) >> (8 * k_byte);
      const float scale = fp4_scale(e & 255u);
      s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s[kb] = mfma16(as_bf16x8(fp4_to_bf16x8(kc[kb][ks], scale)), qf[ks], s[kb]);
    }
    rows_now = pool_row(a, next_key);
    look_up(at + 128 * KW);
    load_k(rows_now);
    // V's first 32 keys, a block a lane.
    auto stage_v = [&](int half) __attribute__((always_inline)) {
#pragma unroll
      for (int n = BPR / 2 * half; n < BPR / 2 * (half + 1); ++n) {
        const int key = 64 / BPR * n + lane / BPR - 32 * half;
        const float scale = fp4_scale((uint32_t)__shfl((int)vse, 64 / BPR * n + lane / BPR) >> (8 * v_byte) & 255u);
        const uint32_t to = st0 + (uint32_t)(key * ROWB);
        const int c0 = 4 * (lane % BPR), sw = v_swizzle<D>(key);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<ROCS_LDS u32x4*>(lds3 + to + 16 * ((c0 + c) ^ sw)) = fp4_to_bf16x8(vw[n][c], scale);
      }
    };
    stage_v(0);
    uint32_t pk[4][2];
    if constexpr (SCORE != 0) {
      const float rel = (float)(rr.pos - at - 4 * g);
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float shift = (SCORE & kCap) != 0 ? rr.cap2 : 0.f;
          if constexpr ((SCORE & kBias) != 0) shift = fmaf(-rr.slope2, fabsf(rel - (float)(16 * kb + i)), shift);
          const float x = s[kb][i];
          if constexpr ((SCORE & kCap) != 0)
            s[kb][i] = fmaf(-2.0f * rr.cap2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * rr.cap_in)), shift);
          else if constexpr ((SCORE & kWideCap) != 0)
            s[kb][i] = wide_cap(x, rr) + shift;
          else
            s[kb][i] = fmaf(x, rr.scale2, shift);
        }
    }
    if (at + 64 > lim_lo) {
      const int seen = rr.lim - at - 4 * g;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * kb + i >= seen) s[kb][i] = -INFINITY;
    }
    const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
    auto weights = [&](float ms) __attribute__((always_inline)) {
      float sum = 0.f;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float e0 = s[kb][2 * w], e1 = s[kb][2 * w + 1];
          if constexpr (SCORE == 0) {
            e0 = fmaf(e0, rr.scale2, -ms);
            e1 = fmaf(e1, rr.scale2, -ms);
          } else {
            e0 -= ms;
            e1 -= ms;
          }
          pk[kb][w] = pack_bf16x2(__builtin_amdgcn_exp2f(e0), __builtin_amdgcn_exp2f(e1));
          sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[kb][w]), ones, sum, false);
        }
      return sum;
    };
    float sum = weights(m);
    if (__builtin_expect(__ballot(!(sum <= kStageBound)) != 0, 0)) {
      float mx = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[kb][i]);
      mx = max_across_rows(mx) * (SCORE == 0 ? rr.scale2 : 1.0f);
      const bool need = mx > m + kLazyMove;
      const float alpha = need ? exp2f(m - mx) : 1.0f;
      if (need) m = mx;
      l_part *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
      sum = weights(m == -INFINITY ? 0.f : m);      // no key seen yet: weights 0
    }
    l_part += sum;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half == 1) stage_v(1);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (ROCS_LDS i16x4*)(lds3 + (va[0] ^ (32u * db)))));
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (ROCS_LDS i16x4*)(lds3 + (va[1] ^ (32u * db)))));
        const bf16x8 vf = as_bf16x8(u32x4{x[0], x[1], y[0], y[1]});
        o[db] = mfma16(vf, as_bf16x8(u32x4{pk[2 * half][0], pk[2 * half][1], pk[2 * half + 1][0], pk[2 * half + 1][1]}),
                       o[db]);
      }
    }
    load_v(rows_now);
  }

  // This wave's partial softmax into its staging area, 16-byte pieces of a row
  // swizzled by the row: element i of o[db] is O[l16][16 db + 4 g + i].
  l_part = sum_across_rows(l_part);
  if (g == 0) {
    pm[wave][l16] = m;
    pl[wave][l16] = l_part;
  }
#pragma unroll
  for (int db = 0; db < DB; ++db)
    *reinterpret_cast<ROCS_LDS f32x4*>(lds3 + st0 + l16 * D * 4 + 16 * ((4 * db + g) ^ l16)) = o[db];
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
      y += *reinterpret_cast<const ROCS_LDS f32x4*>(lds3 + w * STAGE + i * D * 4 + 16 * (piece ^ i)) * f;
    }
    if (!(finite(y[0]) && finite(y[1]) && finite(y[2]) && finite(y[3])) && may_differ(l, a.D, D)) odd[hs][i] = 1;
    const int rw = t.row0 + i;
    const int64_t to_row = (t.q0 + rw / a.G) * a.H + (hk0 + hs) * a.G + rw % a.G;
    const int64_t to = (int64_t)split * a.N * a.H + to_row;
    if (a.splits > 1 && piece == 0) {
      a.part_ml[2 * to] = mx;
      a.part_ml[2 * to + 1] = alone ? kDone : l;
    }
    if (!direct) {
      if (l != 0.f) *reinterpret_cast<f32x4*>(a.part_o + to * a.D + 4 * piece) = y;
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      *reinterpret_cast<u32x2*>(static_cast<bf16_t*>(a.out) + to_row * a.D + 4 * piece) =
          u32x2{pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv)};
    }
  }
  __syncthreads();
  for (int i = wave; i < HW * t.rows; i += kWaves)        // see lone_row
    if (__builtin_amdgcn_readfirstlane(odd[i / t.rows][i % t.rows]) != 0)
      redo_row<bf16_t, true>(a, t, t.row0 + i % t.rows, hk0 + i / t.rows, lo, hi, split, direct);
}

template <int D>
hipError_t launch_few(const HistArgs& a, int64_t slots, int64_t blocks, hipStream_t s) {
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, dim3((uint32_t)blocks), dim3(256), s, a, slots);
  };
  switch (score_of(a)) {
    case kCap: return go(history_fp4_few<D, kCap>);
    case kWideCap: return go(history_fp4_few<D, kWideCap>);
    case kBias: return go(history_fp4_few<D, kBias>);
    case kCap | kBias: return go(history_fp4_few<D, kCap | kBias>);
    case kWideCap | kBias: return go(history_fp4_few<D, kWideCap | kBias>);
    default: return go(history_fp4_few<D, 0>);
  }
}

}  // namespace

hipError_t launch_history_fp4_few(const HistArgs& args, hipStream_t s) {
  HistArgs a = args;
  set_page_divisor(a);
  const int64_t slots = a.R + (a.N * a.G + kFewRows - 1) / kFewRows;
  const int64_t blocks = slots * (a.Hk / a.heads) * a.splits;
  if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
  return a.D > 64 ? launch_few<128>(a, slots, blocks, s) : launch_few<64>(a, slots, blocks, s);
}

hipError_t launch_history_fp4_tile(const HistArgs& args, hipStream_t s) {
  HistArgs a = args;
  set_page_divisor(a);
  return launch_tile<true>(a, s);
}

}  // namespace rocs
