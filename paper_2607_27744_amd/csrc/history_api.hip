// C ABI of the history attention and the cache's pages (rocs_history.h):
// argument checks and error reporting. Nothing here touches tensor data.
#include "../../include/rocs_history.h"

#include <math.h>

#include <initializer_list>

#include "history.h"
#include "status.h"

using namespace rocs;

namespace {

// Rows (token, head) of a call: their numbers, rounded up to a tile, stay in 32 bits.
constexpr int64_t kMaxRows = int64_t(1) << 30;

// Keys of a history: the kernels step past its end in 32 bits, by less than this.
constexpr int64_t kMaxKeys = (int64_t(1) << 31) - 4096;

// The checks that both attentions share, and the launch.
int32_t attend(const char* name, HistArgs a, int64_t R, int64_t kv_rows, int64_t k_bytes,
               float scale, int64_t max_len, int32_t dtype, void* workspace, size_t workspace_bytes,
               void* stream) {
  const size_t es = esize(dtype);
  a.R = (int)R;
  a.G = a.H / a.Hk;
  a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)a.D);
  const int64_t row = (int64_t)a.H * a.D;
  const size_t out_bytes = (size_t)(a.N * row) * es;
  const size_t q_bytes = (size_t)((a.N - 1) * a.q_stride + row) * es;
  const struct { const void* p; size_t n; const char* name; } ins[] = {
      {a.q, q_bytes, "q"}, {a.k, (size_t)k_bytes, "k"}, {a.v, (size_t)k_bytes, "v"},
      {a.q_off, (size_t)(R + 1) * 4, "q_offsets"}, {a.kv_off, (size_t)(R + 1) * 4, "kv_offsets"},
      {a.table, (size_t)a.S * a.width * 4, "page_table"}, {a.lens, (size_t)a.S * 4, "kv_lens"},
      {a.slots, (size_t)R * 4, "slots"}, {a.prefix, (size_t)R * 4, "prefix_lens"},
      {a.q_docs, (size_t)a.N * 4, "q_docs"}, {a.kv_docs, (size_t)kv_rows * 4, "kv_docs"},
      {a.slopes, (size_t)a.H * 4, "slopes"}};
  const HistPlan p = history_plan(R, a.N, a.H, a.Hk, a.D, max_len, dtype == ROCS_DTYPE_BF16);
  const size_t need = p.ml_bytes + p.o_bytes;
  if (need > 0) {
    if (workspace == nullptr || workspace_bytes < need)
      return fail(ROCS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace needs %zu bytes, got %zu", name,
                  need, workspace == nullptr ? (size_t)0 : workspace_bytes);
    if (!aligned(workspace, 256))
      return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: workspace must be 256-byte aligned", name);
    if (overlap(workspace, need, a.out, out_bytes))
      return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: workspace overlaps out", name);
  }
  for (const auto& in : ins) {
    if (overlap(a.out, out_bytes, in.p, in.n))
      return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: out overlaps %s", name, in.name);
    if (need > 0 && overlap(workspace, need, in.p, in.n))
      return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: workspace overlaps %s", name, in.name);
  }
  a.max_len = max_len;
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.heads = p.heads;
  a.part_ml = static_cast<float*>(workspace);
  a.part_o = need > 0 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + p.ml_bytes)
                      : nullptr;
  const bool fast = dtype == ROCS_DTYPE_BF16 && a.D % 8 == 0 && a.D <= 128 && a.q_stride % 8 == 0 &&
                    a.kv_stride % 8 == 0 && a.page_stride % 8 == 0 && aligned(a.q, 16) &&
                    aligned(a.k, 16) && aligned(a.v, 16) && aligned(a.out, 16) &&
                    (a.table == nullptr || a.page_size % 16 == 0) && a.kv_stride < (1 << 24);
  const hipError_t e = launch_history(a, p.rows, dtype == ROCS_DTYPE_BF16, fast,
                                      static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

// Sizes and rules of both attentions. Returns ROCS_OK to go on.
int32_t check_call(const char* name, int64_t R, int64_t N, int32_t H, int32_t Hk, int32_t D,
                   int64_t q_stride, int64_t kv_stride, float cap, int32_t causal,
                   int64_t max_len, int32_t dtype) {
  if (!valid_dtype(dtype)) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: unknown dtype %d", name, dtype);
  if (R < 0 || N < 0 || H < 1 || Hk < 1 || D < 1 || q_stride < 0 || kv_stride < 0 || max_len < 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is out of range", name);
  if (H % Hk != 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: num_heads %d is no multiple of kv_heads %d", name, H, Hk);
  if (causal != 0 && causal != 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: causal must be 0 or 1", name);
  if (!(cap == 0.f || cap >= 1e-30f) || cap > 3.4e38f)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: cap must be 0, or finite and at least 1e-30", name);
  if (D > 256) return fail(ROCS_ERR_UNSUPPORTED, "%s: head_dim %d > 256", name, D);
  if (R > kMaxI32 || N > kMaxI32 || H > 65535 || N * H > kMaxRows || max_len > kMaxI32)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  if (q_stride != 0 && q_stride < (int64_t)H * D)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: q_row_stride < num_heads * head_dim", name);
  if (kv_stride != 0 && kv_stride < (int64_t)Hk * D)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: kv_row_stride < kv_heads * head_dim", name);
  return ROCS_OK;
}

// In the place of an array that an operator does not have.
const int32_t none_ = 0;
const void* const kNone = &none_;

// Entries of a call: the loops over them step by 4096 in 32 bits.
constexpr int64_t kMaxEntries = int64_t(1) << 30;

struct Cache {
  const void *table, *lens, *refs, *pool, *status, *ws;
  int64_t width, S, P, layers, row_bytes;
  int32_t page;
};

struct List {
  const void* p;
  int64_t n;               // int32 entries
};

// Sizes and pointers of a page operator; `need` bytes of workspace. lists: the
// caller's other arrays.
int32_t check_cache(const char* name, const Cache& c, std::initializer_list<List> lists,
                    size_t need, size_t have) {
  if (c.width < 1 || c.S < 1 || c.P < 1 || c.page < 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: table_width, num_slots, num_pages and page_size "
                "must be at least 1", name);
  if (c.S > (1 << 18) || c.P > kMaxI32 || c.P * c.page > kMaxI32 || c.width > kMaxI32 ||
      c.width * c.page > kMaxI32)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: cache too large (num_slots <= 2^18; num_pages * "
                "page_size and table_width * page_size < 2^31)", name);
  if (c.table == nullptr || c.refs == nullptr || c.lens == nullptr || c.pool == nullptr ||
      c.status == nullptr)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  if (c.layers < 0 || c.row_bytes < 0 || c.row_bytes > (int64_t(1) << 30) ||
      c.layers > (int64_t(1) << 20))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: num_layers or row_bytes out of range", name);
  if (need > 0) {
    if (c.ws == nullptr || have < need)
      return fail(ROCS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace needs %zu bytes, got %zu", name,
                  need, c.ws == nullptr ? (size_t)0 : have);
    if (!aligned(c.ws, 256))
      return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: workspace must be 256-byte aligned", name);
  }
  const auto bytes = [](const void* p, size_t n) { return p == kNone ? 0 : n; };
  const size_t pool = (size_t)c.layers * c.P * c.page * c.row_bytes;
  const struct { const void* p; size_t n; } parts[] = {
      {c.table, (size_t)c.S * c.width * 4}, {c.lens, bytes(c.lens, (size_t)c.S * 4)}, {c.refs, (size_t)c.P * 4},
      {c.pool, bytes(c.pool, pool)}, {c.status, bytes(c.status, 8)}, {need > 0 ? c.ws : nullptr, need}};
  for (size_t i = 0; i < 6; ++i)
    for (size_t j = 0; j < i; ++j)
      if (overlap(parts[i].p, parts[i].n, parts[j].p, parts[j].n))
        return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: the cache's arrays, status and workspace "
                    "must not overlap", name);
  for (const List& l : lists)
    for (const auto& part : parts)
      if (overlap(l.p, (size_t)l.n * 4, part.p, part.n))
        return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a list of the call overlaps the cache's arrays, "
                    "status or workspace", name);
  return ROCS_OK;
}

}  // namespace

extern "C" {

size_t rocs_history_workspace_size(int64_t R, int64_t N, int32_t H, int32_t Hk, int32_t D,
                                   int64_t max_len, int32_t dtype) {
  if (R <= 0 || N <= 0 || H < 1 || Hk < 1 || H % Hk != 0 || D < 1 || D > 256 || max_len <= 0 ||
      R > kMaxI32 || N > kMaxI32 || H > 65535 || N * H > kMaxRows || max_len > kMaxI32 ||
      !valid_dtype(dtype))
    return 0;
  const HistPlan p = history_plan(R, N, H, Hk, D, max_len, dtype == ROCS_DTYPE_BF16);
  return p.ml_bytes + p.o_bytes;
}

int32_t rocs_history_attention(const void* q, int64_t q_row_stride, const void* k, const void* v,
                               int64_t kv_row_stride, const int32_t* q_offsets,
                               const int32_t* kv_offsets, const int32_t* prefix_lens,
                               const int32_t* q_docs, const int32_t* kv_docs, const float* slopes,
                               int64_t R, int64_t N, int64_t num_kv_rows, int32_t H, int32_t Hk,
                               int32_t D, float softmax_scale, float cap, int32_t causal,
                               int64_t max_kv_len, int32_t dtype, void* out, void* workspace,
                               size_t workspace_bytes, void* stream) {
  const char* name = "rocs_history_attention";
  const int32_t st = check_call(name, R, N, H, Hk, D, q_row_stride, kv_row_stride, cap, causal,
                                max_kv_len, dtype);
  if (st != ROCS_OK) return st;
  if (num_kv_rows < 0) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: num_kv_rows < 0", name);
  if (num_kv_rows > kMaxKeys) return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  if ((q_docs == nullptr) != (kv_docs == nullptr))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: q_docs and kv_docs go together", name);
  if (N == 0) return ok();
  if (R == 0) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: query rows but no requests", name);
  if (q == nullptr || out == nullptr || q_offsets == nullptr || kv_offsets == nullptr ||
      (num_kv_rows > 0 && (k == nullptr || v == nullptr)))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  HistArgs a{};
  a.q = q; a.k = k; a.v = v; a.out = out; a.q_off = q_offsets; a.kv_off = kv_offsets;
  a.prefix = prefix_lens; a.q_docs = q_docs; a.kv_docs = kv_docs; a.slopes = slopes;
  a.N = N; a.H = H; a.Hk = Hk; a.D = D; a.cap = cap; a.causal = causal;
  a.q_stride = q_row_stride != 0 ? q_row_stride : (int64_t)H * D;
  a.kv_stride = kv_row_stride != 0 ? kv_row_stride : (int64_t)Hk * D;
  const int64_t k_bytes =
      num_kv_rows > 0 ? ((num_kv_rows - 1) * a.kv_stride + (int64_t)Hk * D) * (int64_t)esize(dtype) : 0;
  return attend(name, a, R, num_kv_rows, k_bytes, softmax_scale,
                max_kv_len > 0 ? max_kv_len : num_kv_rows, dtype, workspace, workspace_bytes, stream);
}

int32_t rocs_paged_attention(const void* q, int64_t q_row_stride, const void* k_pages,
                             const void* v_pages, int64_t page_stride, int64_t kv_row_stride,
                             const int32_t* page_table, int64_t table_width,
                             const int32_t* kv_lens, const int32_t* slots, int64_t num_slots,
                             const int32_t* q_offsets, const int32_t* prefix_lens,
                             const float* slopes, int64_t R, int64_t N, int64_t num_pages,
                             int32_t page_size, int32_t H, int32_t Hk, int32_t D,
                             float softmax_scale, float cap, int32_t causal, int64_t max_kv_len,
                             int32_t dtype, void* out, void* workspace, size_t workspace_bytes,
                             void* stream) {
  const char* name = "rocs_paged_attention";
  const int32_t st = check_call(name, R, N, H, Hk, D, q_row_stride, kv_row_stride, cap, causal,
                                max_kv_len, dtype);
  if (st != ROCS_OK) return st;
  if (table_width < 1 || num_slots < 0 || num_pages < 1 || page_size < 1 || page_stride < 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: table_width, num_pages and page_size must be at "
                "least 1", name);
  if (table_width > kMaxI32 || table_width * page_size > kMaxKeys || num_pages > kMaxI32 ||
      num_slots > kMaxI32)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: table_width * page_size must not pass 2^31 - 4096", name);
  const int64_t kv_stride = kv_row_stride != 0 ? kv_row_stride : (int64_t)Hk * D;
  const int64_t extent = (page_size - 1) * kv_stride + (int64_t)Hk * D;      // of one page
  if (page_stride != 0 && page_stride < extent)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: page_stride is smaller than a page", name);
  if (N == 0) return ok();
  if (R == 0 || num_slots == 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: query rows but no requests or slots", name);
  if (slots == nullptr && R > num_slots)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: without slots, num_requests <= num_slots", name);
  if (q == nullptr || out == nullptr || k_pages == nullptr || v_pages == nullptr ||
      q_offsets == nullptr || page_table == nullptr || kv_lens == nullptr)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  HistArgs a{};
  a.q = q; a.k = k_pages; a.v = v_pages; a.out = out; a.q_off = q_offsets; a.table = page_table;
  a.lens = kv_lens; a.slots = slots; a.prefix = prefix_lens; a.slopes = slopes;
  a.N = N; a.H = H; a.Hk = Hk; a.D = D; a.cap = cap; a.causal = causal; a.width = table_width;
  a.pages = num_pages; a.S = (int)num_slots; a.page_size = page_size;
  a.q_stride = q_row_stride != 0 ? q_row_stride : (int64_t)H * D;
  a.kv_stride = kv_stride;
  a.page_magic = page_size >= 32 ? (uint32_t)((uint64_t(1) << 32) / (uint32_t)(page_size / 16)) + 1u : 0u;
  a.page_stride = page_stride != 0 ? page_stride : page_size * kv_stride;
  const int64_t k_bytes = ((num_pages - 1) * a.page_stride + extent) * (int64_t)esize(dtype);
  const int64_t bound = table_width * page_size;
  return attend(name, a, R, 0, k_bytes, softmax_scale,
                max_kv_len > 0 && max_kv_len < bound ? max_kv_len : bound, dtype, workspace,
                workspace_bytes, stream);
}

size_t rocs_cache_workspace_size(int64_t entries, int64_t num_pages) {
  if (entries < 0 || num_pages < 1 || entries > kMaxEntries || num_pages > kMaxI32) return 0;
  // A head, then: the free pages found (reserve); three lists and the pages of
  // fork's entries; compact's counts per 4096 pages and three lists.
  const size_t n = (size_t)entries, p = (size_t)num_pages;
  const size_t compact = p / 4096 + 1 + 3 * p;
  return align256((64 + (4 * n > compact ? 4 * n : compact)) * sizeof(int32_t));
}

int32_t rocs_cache_reserve(const int32_t* slots, const int32_t* row_offsets, int64_t entries,
                           int64_t num_rows, int32_t* page_table, int64_t table_width,
                           int32_t* lens, int64_t num_slots, int32_t* refs, int64_t num_pages,
                           int32_t page_size, int32_t* rows, int32_t* status, void* workspace,
                           size_t workspace_bytes, void* stream) {
  const char* name = "rocs_cache_reserve";
  const Cache c{page_table, lens, refs, kNone, status, workspace, table_width, num_slots, num_pages,
                0, 0, page_size};
  if (entries < 0 || num_rows < 0)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is negative", name);
  if (entries > kMaxEntries || num_rows > kMaxI32)
    return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  const List from{slots, entries}, at{row_offsets, entries + 1}, to{rows, num_rows};
  const int32_t st = check_cache(name, c, {from, at, to},
                                 rocs_cache_workspace_size(entries, num_pages), workspace_bytes);
  if (st != ROCS_OK) return st;
  if ((entries > 0 && (slots == nullptr || row_offsets == nullptr)) ||
      (num_rows > 0 && (rows == nullptr || entries == 0)))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  for (const List& l : {from, at})
    if (overlap(rows, (size_t)num_rows * 4, l.p, (size_t)l.n * 4))
      return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: rows overlaps an input", name);
  const hipError_t e = launch_reserve(slots, row_offsets, entries, num_rows, page_table,
                                      table_width, lens, num_slots, refs, num_pages, page_size,
                                      rows, status, static_cast<int32_t*>(workspace),
                                      static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

int32_t rocs_cache_write(const void* x, int64_t x_row_stride, const int32_t* rows,
                         int64_t num_rows, void* pool, int64_t num_pool_rows, int64_t row_bytes,
                         void* stream) {
  const char* name = "rocs_cache_write";
  if (num_rows < 0 || num_pool_rows < 1 || row_bytes < 1 || x_row_stride < row_bytes)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: need num_rows >= 0, num_pool_rows >= 1, "
                "row_bytes >= 1 and x_row_stride >= row_bytes", name);
  if (num_rows > kMaxI32 || num_pool_rows > kMaxI32 || row_bytes > (int64_t(1) << 30))
    return fail(ROCS_ERR_UNSUPPORTED, "%s: too large", name);
  if (num_rows == 0) return ok();
  if (x == nullptr || rows == nullptr || pool == nullptr)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  const size_t pool_bytes = (size_t)num_pool_rows * row_bytes;
  if (overlap(pool, pool_bytes, x, (size_t)((num_rows - 1) * x_row_stride + row_bytes)) ||
      overlap(pool, pool_bytes, rows, (size_t)num_rows * 4))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: pool overlaps an input", name);
  const hipError_t e = launch_cache_write(x, x_row_stride, rows, num_rows, pool, num_pool_rows,
                                          row_bytes, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

int32_t rocs_cache_fork(const int32_t* parents, const int32_t* children, int64_t entries,
                        int32_t* page_table, int64_t table_width, int32_t* lens,
                        int64_t num_slots, int32_t* refs, int64_t num_pages, int32_t page_size,
                        void* pool, int64_t num_layers, int64_t row_bytes, int32_t* status,
                        void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "rocs_cache_fork";
  const Cache c{page_table, lens, refs, pool, status, workspace, table_width, num_slots, num_pages,
                num_layers, row_bytes, page_size};
  if (entries < 0 || num_layers < 1 || row_bytes < 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: need entries >= 0, num_layers >= 1 and "
                "row_bytes >= 1", name);
  if (entries > kMaxEntries) return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  const int32_t st = check_cache(name, c, {{parents, entries}, {children, entries}},
                                 rocs_cache_workspace_size(entries, num_pages), workspace_bytes);
  if (st != ROCS_OK) return st;
  if (entries > 0 && (parents == nullptr || children == nullptr))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  const hipError_t e = launch_fork(parents, children, entries, page_table, table_width, lens,
                                   num_slots, refs, num_pages, page_size, pool, num_layers,
                                   row_bytes, status, static_cast<int32_t*>(workspace),
                                   static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

int32_t rocs_cache_free(const int32_t* slots, int64_t entries, int32_t* page_table,
                        int64_t table_width, int32_t* lens, int64_t num_slots, int32_t* refs,
                        int64_t num_pages, int32_t page_size, void* stream) {
  const char* name = "rocs_cache_free";
  const Cache c{page_table, lens, refs, kNone, kNone, nullptr, table_width, num_slots, num_pages,
                0, 0, page_size};
  if (entries < 0) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is negative", name);
  if (entries >= (int64_t(1) << 24))                   // a workgroup of 256 each
    return fail(ROCS_ERR_UNSUPPORTED, "%s: batch too large", name);
  const int32_t st = check_cache(name, c, {{slots, entries}}, 0, 0);
  if (st != ROCS_OK) return st;
  if (entries == 0) return ok();
  if (slots == nullptr) return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  const hipError_t e = launch_free(slots, entries, page_table, table_width, lens, num_slots, refs,
                                   num_pages, page_size, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

int32_t rocs_cache_compact(int32_t* page_table, int64_t table_width, int64_t num_slots,
                           int32_t* refs, int64_t num_pages, int32_t page_size, void* pool,
                           int64_t num_layers, int64_t row_bytes, int32_t* status,
                           void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "rocs_cache_compact";
  const Cache c{page_table, kNone, refs, pool, status, workspace, table_width, num_slots, num_pages,
                num_layers, row_bytes, page_size};
  if (num_layers < 1 || row_bytes < 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: need num_layers >= 1 and row_bytes >= 1", name);
  const int32_t st = check_cache(name, c, {}, rocs_cache_workspace_size(0, num_pages),
                                 workspace_bytes);
  if (st != ROCS_OK) return st;
  const hipError_t e = launch_compact(page_table, table_width, num_slots, refs, num_pages, pool,
                                      num_layers, page_size * row_bytes, status,
                                      static_cast<int32_t*>(workspace),
                                      static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

int32_t rocs_cache_copy(const int32_t* src_pages, const int32_t* dst_pages, int64_t entries,
                        const void* src_pool, int64_t src_num_pages, void* dst_pool,
                        int64_t dst_num_pages, int64_t num_layers, int64_t page_bytes,
                        void* stream) {
  const char* name = "rocs_cache_copy";
  if (entries < 0 || src_num_pages < 1 || dst_num_pages < 1 || num_layers < 1 || page_bytes < 1)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: a size is out of range", name);
  if (entries > kMaxI32 || src_num_pages > kMaxI32 || dst_num_pages > kMaxI32 ||
      num_layers > (int64_t(1) << 20) || page_bytes > (int64_t(1) << 40))
    return fail(ROCS_ERR_UNSUPPORTED, "%s: too large", name);
  if (entries == 0) return ok();
  if (src_pages == nullptr || dst_pages == nullptr || src_pool == nullptr || dst_pool == nullptr)
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: null pointer argument", name);
  const size_t from = (size_t)num_layers * src_num_pages * page_bytes;
  const size_t to = (size_t)num_layers * dst_num_pages * page_bytes;
  if ((src_pool != dst_pool || src_num_pages != dst_num_pages) &&
      overlap(src_pool, from, dst_pool, to))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: the pools overlap", name);
  if (overlap(src_pages, (size_t)entries * 4, dst_pool, to) ||
      overlap(dst_pages, (size_t)entries * 4, dst_pool, to))
    return fail(ROCS_ERR_INVALID_ARGUMENT, "%s: dst_pool overlaps a list", name);
  const hipError_t e = launch_cache_copy(src_pages, dst_pages, entries, src_pool, src_num_pages,
                                         dst_pool, dst_num_pages, num_layers, page_bytes,
                                         static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return launch_failed(name, e);
  return ok();
}

}  // extern "C"
