// C ABI of the adapter linear, the rotated append and the attention over a
// cache in 4 bits (rocs_layer.h): argument checks and error reporting. Nothing
// here touches tensor data.
#include "../../include/rocs_layer.h"

#include <math.h>

#include <initializer_list>

#include "layer.h"
#include "status.h"

using namespace rocs;

namespace {

// Limits that keep the kernels' 32-bit indices in range (see rocs_history.h).
constexpr int64_t kMaxRows = int64_t(1) << 30;
// Rows of a rotation: a workgroup may have one alone, and a grid fewer than 2^24.
constexpr int64_t kMaxTurned = (int64_t(1) << 24) - 1;
constexpr int64_t kMaxKeys = (int64_t(1) << 31) - 4096;

struct Span {
  const void* p;
  size_t n;
  const char* name;
};

// Outputs (and the workspace) must not overlap an input or each other.
int32_t apart(const char* name, std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (const Span* o = outs.begin(); o != outs.end(); ++o) {
    for (const Span& i : ins)
      if (overlap(o->p, o->n, i.p, i.n))
        return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: %s overlaps %s", name, o->name, i.name);
    for (const Span* u = outs.begin(); u != o; ++u)
      if (overlap(o->p, o->n, u->p, u->n))
        return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: %s overlaps %s", name, o->name, u->name);
  }
  return ROCS_OK;
}

// Bytes that n rows of `row` elements, `stride` apart, reach over.
size_t reach(int64_t n, int64_t stride, int64_t row, size_t es) {
  return n > 0 ? (size_t)((n - 1) * stride + row) * es : 0;
}

// Positions of the rows, and the rotation. Returns ROCS_OK to go on.
int32_t check_turn(const char* name, AppendArgs& a, int32_t rot_dim, int64_t R, int64_t S,
                   int32_t dtype) {
  if (!valid_dtype(dtype)) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: unknown dtype %d", name, dtype);
  if (a.M < 0 || a.H < 0 || a.Hk < 0 || a.D < 1 || a.q_stride < 0 || a.kv_stride < 0 || R < 0 || S < 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is out of range", name);
  if (a.D > 256) return fail(ROCS_ERR_UNSUPPORTED, "%s: head_dim %d > 256", name, a.D);
  if (a.H > 65535 || a.Hk > 65535 || R > kMaxI32 || S > kMaxI32 || a.M > kMaxTurned ||
      a.M * a.H > kMaxRows || a.M * 2 * a.Hk > kMaxRows)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  if (rot_dim < 0 || rot_dim % 2 != 0 || rot_dim > a.D)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: rot_dim must be even, in 0 .. head_dim", name);
  if (a.interleaved != 0 && a.interleaved != 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: interleaved must be 0 or 1", name);
  if (a.M == 0) return ROCS_OK;
  if (rot_dim > 0 && a.freqs == nullptr)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a rotation needs freqs", name);
  if (rot_dim > 0 && a.positions == nullptr && (a.off == nullptr || a.lens == nullptr))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a rotation needs positions, or offsets and lens", name);
  if (a.off != nullptr && R == 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: rows but no requests", name);
  if (a.off == nullptr && (a.slots != nullptr || a.lens != nullptr))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: slots and lens need offsets", name);
  if (a.lens != nullptr && (S == 0 || (a.slots == nullptr && R > S)))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: without slots, request r is slot r: R <= num_slots", name);
  a.R = (int)R;
  a.S = (int)S;
  a.half = rot_dim / 2;
  a.bf16 = dtype == ROCS_DTYPE_BF16;
  return ROCS_OK;
}

}  // namespace

extern "C" {

size_t rocs_adapter_workspace_size(int64_t R, int64_t N, int64_t K, int64_t D, int32_t rank,
                                   int32_t dtype) {
  if (R <= 0 || N <= 0 || K < 1 || D < 1 || rank < 1 || rank > 256 || N > kMaxI32 ||
      !valid_dtype(dtype))
    return 0;
  return adapter_t_bytes(N, rank) + align256((size_t)N * 4);
}

int32_t rocs_adapter_linear(const void* x, int64_t x_row_stride, const void* w, const void* a,
                            const void* b, const float* scales, const float* bias,
                            const int32_t* offsets, const int32_t* adapter_ids, int64_t R,
                            int64_t N, int64_t K, int64_t D, int32_t rank, int64_t num_adapters,
                            int32_t dtype, int32_t activation, void* out, void* workspace,
                            size_t workspace_bytes, void* stream) {
  const char* name = "rocs_adapter_linear";
  if (!valid_dtype(dtype)) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: unknown dtype %d", name, dtype);
  if (activation != ROCS_ACT_NONE && activation != ROCS_ACT_RELU)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: unknown activation %d", name, activation);
  if (R < 0 || N < 0 || K < 1 || D < 1 || rank < 1 || num_adapters < 0 || x_row_stride < 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is out of range", name);
  if (rank > 256) return fail(ROCS_ERR_UNSUPPORTED, "%s: rank %d > 256", name, rank);
  if (R > kMaxI32 || N > kMaxI32 || K >= (1 << 22) || D >= (1 << 22) || num_adapters > kMaxI32 ||
      R + (N + 31) / 32 >= (1 << 23) || (N + 127) / 128 * ((D + 127) / 128) >= (1 << 24) || x_row_stride > (int64_t(1) << 31))
    return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  if (x_row_stride != 0 && x_row_stride < K)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: x_row_stride < K", name);
  if (N == 0) return ok();
  if (R == 0) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: rows but no requests", name);
  if (x == nullptr || w == nullptr || offsets == nullptr || adapter_ids == nullptr ||
      out == nullptr || (num_adapters > 0 && (a == nullptr || b == nullptr)))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  const size_t es = esize(dtype), need = rocs_adapter_workspace_size(R, N, K, D, rank, dtype);
  if (workspace == nullptr || workspace_bytes < need)
    return fail(ROCS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace needs %zu bytes, got %zu", name, need,
                workspace == nullptr ? (size_t)0 : workspace_bytes);
  if (!aligned(workspace, 256))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: workspace must be 256-byte aligned", name);
  AdapterArgs g{};
  g.x = x; g.w = w; g.a = a; g.b = b; g.scales = num_adapters > 0 ? scales : nullptr; g.bias = bias;
  g.off = offsets; g.ids = adapter_ids; g.out = out; g.t = workspace;
  g.N = N; g.x_stride = x_row_stride != 0 ? x_row_stride : K;
  g.R = (int)R; g.K = (int)K; g.D = (int)D; g.rank = rank; g.A = (int)num_adapters;
  g.bf16 = dtype == ROCS_DTYPE_BF16; g.relu = activation == ROCS_ACT_RELU;
  const int32_t st = apart(
      name, {{out, (size_t)N * D * es, "out"}, {workspace, need, "workspace"}},
      {{x, reach(N, g.x_stride, K, es), "x"}, {w, (size_t)D * K * es, "w"},
       {a, (size_t)num_adapters * rank * K * es, "a"}, {b, (size_t)num_adapters * D * rank * es, "b"},
       {scales, (size_t)num_adapters * 4, "scales"}, {bias, (size_t)D * 4, "bias"},
       {offsets, (size_t)(R + 1) * 4, "offsets"}, {adapter_ids, (size_t)R * 4, "adapter_ids"}});
  if (st != ROCS_OK) return st;
  const bool fast = dtype == ROCS_DTYPE_BF16 && K % 8 == 0 && D % 4 == 0 && rank % 8 == 0 &&
                    g.x_stride % 8 == 0 && aligned(x, 16) && aligned(w, 16) && aligned(a, 16) &&
                    aligned(b, 16) && aligned(out, 16);
  const hipError_t e = launch_adapter(g, fast, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

int32_t rocs_rotate(const void* x, int64_t x_row_stride, const float* freqs, int32_t rot_dim,
                    int32_t interleaved, const int32_t* positions, const int32_t* offsets,
                    const int32_t* slots, const int32_t* lens, int64_t R, int64_t S, int64_t M,
                    int32_t H, int32_t D, int32_t dtype, void* out, void* stream) {
  const char* name = "rocs_rotate";
  AppendArgs a{};
  a.q = x; a.q_out = out; a.freqs = freqs; a.positions = positions; a.off = offsets;
  a.slots = slots; a.lens = lens;
  a.M = M; a.H = H; a.D = D; a.interleaved = interleaved;
  a.q_stride = x_row_stride != 0 ? x_row_stride : (int64_t)H * D;
  int32_t st = check_turn(name, a, rot_dim, R, S, dtype);
  if (st != ROCS_OK) return st;
  if (H < 1 || (x_row_stride != 0 && x_row_stride < (int64_t)H * D))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: num_heads < 1, or x_row_stride < num_heads * head_dim", name);
  if (M == 0) return ok();
  if (x == nullptr || out == nullptr)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  const size_t es = esize(dtype);
  st = apart(name, {{out, (size_t)M * H * D * es, "out"}},
             {{x, reach(M, a.q_stride, (int64_t)H * D, es), "x"},
              {freqs, (size_t)a.half * 4, "freqs"}, {positions, (size_t)M * 4, "positions"},
              {offsets, (size_t)(R + 1) * 4, "offsets"}, {slots, (size_t)R * 4, "slots"},
              {lens, (size_t)S * 4, "lens"}});
  if (st != ROCS_OK) return st;
  const hipError_t e = launch_append(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

int32_t rocs_cache_append(const void* q, int64_t q_row_stride, const void* k, const void* v,
                          int64_t kv_row_stride, const int32_t* rows, const float* freqs,
                          int32_t rot_dim, int32_t interleaved, const int32_t* positions,
                          const int32_t* offsets, const int32_t* slots, const int32_t* lens,
                          int64_t R, int64_t S, int64_t M, int32_t H, int32_t Hk, int32_t D,
                          int32_t dtype, void* pool, int64_t num_pool_rows, int32_t form,
                          void* q_out, void* stream) {
  const char* name = "rocs_cache_append";
  AppendArgs a{};
  a.q = q; a.q_out = q_out; a.k = k; a.v = v; a.rows = rows; a.pool = pool; a.freqs = freqs;
  a.positions = positions; a.off = offsets; a.slots = slots; a.lens = lens;
  a.M = M; a.H = q != nullptr ? H : 0; a.Hk = Hk; a.D = D; a.interleaved = interleaved;
  a.pool_rows = num_pool_rows;
  a.q_stride = q_row_stride != 0 ? q_row_stride : (int64_t)H * D;
  a.kv_stride = kv_row_stride != 0 ? kv_row_stride : (int64_t)Hk * D;
  int32_t st = check_turn(name, a, rot_dim, R, S, dtype);
  if (st != ROCS_OK) return st;
  if (form != ROCS_POOL_ROWS && form != ROCS_POOL_FP4)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: unknown form %d of the pool", name, form);
  if (Hk < 1 || num_pool_rows < 0 || (q != nullptr && H < 1))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is out of range", name);
  if (num_pool_rows > kMaxI32) return fail(ROCS_ERR_UNSUPPORTED, "%s: cache too large", name);
  if (kv_row_stride != 0 && kv_row_stride < (int64_t)Hk * D)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: kv_row_stride < kv_heads * head_dim", name);
  if (q != nullptr && q_row_stride != 0 && q_row_stride < (int64_t)H * D)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: q_row_stride < num_heads * head_dim", name);
  const bool fp4 = form == ROCS_POOL_FP4;
  if (fp4 && D % kFp4Block != 0)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: in 4 bits head_dim must be a multiple of 32", name);
  if (M == 0) return ok();
  if (k == nullptr || v == nullptr || rows == nullptr || (num_pool_rows > 0 && pool == nullptr) ||
      (q != nullptr && q_out == nullptr))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  if (fp4 && !aligned(pool, 16))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a pool in 4 bits must be 16-byte aligned", name);
  a.fp4 = fp4;
  const size_t es = esize(dtype), kv = reach(M, a.kv_stride, (int64_t)Hk * D, es);
  const size_t row = fp4 ? rocs_fp4_row_bytes(Hk, D) : (size_t)2 * Hk * D * es;
  st = apart(name,
             {{pool, (size_t)num_pool_rows * row, "pool"},
              {q != nullptr ? q_out : nullptr, (size_t)M * a.H * D * es, "q_out"}},
             {{q, reach(M, a.q_stride, (int64_t)H * D, es), "q"}, {k, kv, "k"}, {v, kv, "v"},
              {rows, (size_t)M * 4, "rows"}, {freqs, (size_t)a.half * 4, "freqs"},
              {positions, (size_t)M * 4, "positions"}, {offsets, (size_t)(R + 1) * 4, "offsets"},
              {slots, (size_t)R * 4, "slots"}, {lens, (size_t)S * 4, "lens"}});
  if (st != ROCS_OK) return st;
  const hipError_t e = launch_append(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

size_t rocs_fp4_row_bytes(int32_t Hk, int32_t D) {
  if (Hk < 1 || Hk > 65535 || D < 1 || D > 256 || D % kFp4Block != 0) return 0;
  return (size_t)Fp4Row{Hk, D}.bytes();
}

int32_t rocs_cache_read_fp4(const int32_t* rows, int64_t M, const void* pool, int64_t num_pool_rows,
                            int32_t Hk, int32_t D, int32_t dtype, void* out, void* stream) {
  const char* name = "rocs_cache_read_fp4";
  if (!valid_dtype(dtype)) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: unknown dtype %d", name, dtype);
  if (M < 0 || num_pool_rows < 0 || Hk < 1 || D < 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is out of range", name);
  if (D > 256 || D % kFp4Block != 0)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: head_dim must be a multiple of 32 up to 256", name);
  if (Hk > 65535 || M > kMaxI32 || num_pool_rows > kMaxI32 || M * 2 * Hk > kMaxRows)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  if (M == 0) return ok();
  if (rows == nullptr || out == nullptr || (num_pool_rows > 0 && pool == nullptr))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  if (!aligned(pool, 16) || !aligned(out, 16))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: pool and out must be 16-byte aligned", name);
  const int32_t st = apart(name, {{out, (size_t)M * 2 * Hk * D * esize(dtype), "out"}},
                           {{rows, (size_t)M * 4, "rows"},
                            {pool, (size_t)num_pool_rows * rocs_fp4_row_bytes(Hk, D), "pool"}});
  if (st != ROCS_OK) return st;
  const hipError_t e = launch_read_fp4(rows, M, pool, num_pool_rows, Hk, D,
                                       dtype == ROCS_DTYPE_BF16, out, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

size_t rocs_paged_fp4_workspace_size(int64_t R, int64_t N, int32_t H, int32_t Hk, int32_t D,
                                     int64_t max_len, int32_t dtype) {
  if (R <= 0 || N <= 0 || H < 1 || Hk < 1 || H % Hk != 0 || D < 1 || D > 256 || max_len <= 0 ||
      R > kMaxI32 || N > kMaxI32 || H > 65535 || N * H > kMaxRows || max_len > kMaxI32 ||
      !valid_dtype(dtype))
    return 0;
  const HistPlan p = fp4_plan(R, N, H, Hk, D, max_len, dtype == ROCS_DTYPE_BF16);
  return p.ml_bytes + p.o_bytes;
}

int32_t rocs_paged_attention_fp4(const void* q, int64_t q_row_stride, const void* pages,
                                 const int32_t* page_table, int64_t table_width,
                                 const int32_t* kv_lens, const int32_t* slots, int64_t num_slots,
                                 const int32_t* q_offsets, const int32_t* prefix_lens,
                                 const float* slopes, int64_t R, int64_t N, int64_t num_pages,
                                 int32_t page_size, int32_t H, int32_t Hk, int32_t D,
                                 float softmax_scale, float cap, int32_t causal, int64_t max_kv_len,
                                 int32_t dtype, void* out, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  const char* name = "rocs_paged_attention_fp4";
  if (!valid_dtype(dtype)) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: unknown dtype %d", name, dtype);
  if (R < 0 || N < 0 || H < 1 || Hk < 1 || D < 1 || q_row_stride < 0 || max_kv_len < 0 ||
      table_width < 1 || num_slots < 0 || num_pages < 1 || page_size < 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is out of range", name);
  if (H % Hk != 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: num_heads %d is no multiple of kv_heads %d", name, H, Hk);
  if (causal != 0 && causal != 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: causal must be 0 or 1", name);
  if (!(cap == 0.f || cap >= 1e-30f) || cap > 3.4e38f)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: cap must be 0, or finite and at least 1e-30", name);
  if (D > 256 || D % kFp4Block != 0)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: head_dim must be a multiple of 32 up to 256", name);
  if (R > kMaxI32 || N > kMaxI32 || H > 65535 || N * H > kMaxRows || max_kv_len > kMaxI32)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  if (table_width > kMaxI32 || table_width * page_size > kMaxKeys || num_pages > kMaxI32 ||
      num_pages * page_size > kMaxI32 || num_slots > kMaxI32)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: table_width * page_size must not pass 2^31 - 4096, and "
                "num_pages * page_size be below 2^31", name);
  if (q_row_stride != 0 && q_row_stride < (int64_t)H * D)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: q_row_stride < num_heads * head_dim", name);
  if (N == 0) return ok();
  if (R == 0 || num_slots == 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: query rows but no requests or slots", name);
  if (slots == nullptr && R > num_slots)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: without slots, request r is slot r: R <= num_slots", name);
  if (q == nullptr || pages == nullptr || page_table == nullptr || kv_lens == nullptr ||
      q_offsets == nullptr || out == nullptr)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  if (!aligned(pages, 16))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: pages must be 16-byte aligned", name);
  const bool bf16 = dtype == ROCS_DTYPE_BF16;
  const size_t es = esize(dtype);
  const int64_t all = table_width * page_size;
  const int64_t most = max_kv_len > 0 && max_kv_len < all ? max_kv_len : all;
  HistArgs a{};
  a.q = q; a.k = pages; a.v = pages; a.out = out; a.q_off = q_offsets; a.table = page_table;
  a.lens = kv_lens; a.slots = slots; a.prefix = prefix_lens; a.slopes = slopes;
  a.N = N; a.width = table_width; a.pages = num_pages; a.page_size = page_size;
  a.R = (int)R; a.S = (int)num_slots; a.H = H; a.Hk = Hk; a.G = H / Hk; a.D = D; a.cap = cap;
  a.causal = causal;
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D);
  a.q_stride = q_row_stride != 0 ? q_row_stride : (int64_t)H * D;
  a.kv_stride = Fp4Row{Hk, D}.bytes();
  a.page_stride = a.kv_stride * page_size;
  const HistPlan p = fp4_plan(R, N, H, Hk, D, most, bf16);
  const size_t need = p.ml_bytes + p.o_bytes;
  if (need > 0 && (workspace == nullptr || workspace_bytes < need))
    return fail(ROCS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace needs %zu bytes, got %zu", name, need,
                workspace == nullptr ? (size_t)0 : workspace_bytes);
  if (need > 0 && !aligned(workspace, 256))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: workspace must be 256-byte aligned", name);
  const int64_t row = (int64_t)H * D;
  const int32_t st = apart(
      name, {{out, (size_t)(N * row) * es, "out"}, {need > 0 ? workspace : nullptr, need, "workspace"}},
      {{q, reach(N, a.q_stride, row, es), "q"}, {pages, (size_t)num_pages * a.page_stride, "pages"},
       {q_offsets, (size_t)(R + 1) * 4, "q_offsets"},
       {page_table, (size_t)num_slots * table_width * 4, "page_table"},
       {kv_lens, (size_t)num_slots * 4, "kv_lens"}, {slots, (size_t)R * 4, "slots"},
       {prefix_lens, (size_t)R * 4, "prefix_lens"}, {slopes, (size_t)H * 4, "slopes"}});
  if (st != ROCS_OK) return st;
  a.max_len = most;
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.heads = p.heads;
  a.part_ml = static_cast<float*>(workspace);
  a.part_o = need > 0 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + p.ml_bytes) : nullptr;
  const bool fast = bf16 && D <= 128 && a.q_stride % 8 == 0 && aligned(q, 16) && aligned(out, 16);
  const hipError_t e = launch_history_fp4(a, p.rows, bf16, fast, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

}  // extern "C"
