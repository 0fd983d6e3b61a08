// The pages of the history cache: reserve, write, fork, free, compact, copy.
//
// Bookkeeping (page_table, lens, refs) stays on the device and is read and
// changed there, so no operator waits for the host. What needs an order over
// the whole cache (which pages are free, which entry gets which of them) runs
// in one workgroup with prefix sums, so that equal calls give equal tables;
// refs change by integer atomics, whose order does not matter. What moves rows
// runs over the whole chip and reads its work list from device memory.
#include "common.h"
#include "history.h"
#include "launch.h"

namespace rocs {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kSegment = 4096;             // entries of a call handled at a time
constexpr int kSlotWords = (1 << 18) / 32; // a bit per slot
constexpr int64_t kCopyUnit = 16384;       // bytes of a copy item's piece
constexpr int kCopyBlocks = 2048;          // eight workgroups a CU

// Workspace, in int32: [0] go-ahead / item count, [1] live pages below the
// border, then lists at kWsHead.
constexpr int kWsHead = 64;

// Exclusive prefix sum of v over the 1024 threads; *total gets the sum. Two
// barriers; `part` may be used again after the caller's next barrier.
__device__ __forceinline__ int block_scan(int v, int* part, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const int p = part[w];
    if (w < wave) before += p;
    sum += p;
  }
  __syncthreads();
  *total = sum;
  return before + incl - v;
}

// The first `want` pages from page `from` on with refs 0, in ascending order,
// into list; returns how many there are (at most want). All threads call it.
__device__ int free_pages(const int32_t* refs, int64_t from, int64_t P, int want, int32_t* list,
                          int* part) {
  int found = 0;
  for (int64_t base = from; base < P && found < want; base += 4 * kPlanThreads) {
    const int64_t p = base + 4 * threadIdx.x;
    bool free[4];
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      free[i] = p + i < P && refs[p + i] == 0;
      n += free[i];
    }
    int total;
    int at = found + block_scan(n, part, &total);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (free[i] && at < want) list[at] = (int)(p + i);
      at += free[i];
    }
    found += total;
  }
  return min(found, want);
}

// The largest i in [0, n) with start[i] <= v (start[0] <= v).
__device__ __forceinline__ int owner_in(const int* start, int n, int v) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= v) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// rows and page below 2^31.
__device__ __forceinline__ int pages_of(uint32_t rows, int page) {
  return (int)((rows + (uint32_t)page - 1u) / (uint32_t)page);
}

// Sets slot s's bit; whether it was set before.
__device__ __forceinline__ bool take_bit(uint32_t* bits, int s) {
  return (atomicOr(&bits[s >> 5], 1u << (s & 31)) >> (s & 31)) & 1;
}

// ---------------------------------------------------------------------------
// reserve, one workgroup. A pass over the entries checks them and adds up the
// pages; if all is well the free pages are listed and each handed to its owner
// (found by binary search in the prefix sums). A page search ends with the
// last page needed. Bound by the chain of memory latencies: what the first
// round needs (a thread's entry, the first 4096 reference counts) is in flight
// from the start and stays in registers, what was found is in LDS: 7.0 us for
// 256 entries of one row (with their pool rows), as for 16 of 2,000.
// ---------------------------------------------------------------------------
constexpr int kPagesHere = 4 * kPlanThreads;     // pages of the first round

__global__ __launch_bounds__(kPlanThreads) void reserve_kernel(
    const int32_t* __restrict__ slots, const int32_t* __restrict__ row_off, int n, int64_t M,
    int32_t* __restrict__ table, int64_t width, int32_t* __restrict__ lens, int S,
    int32_t* __restrict__ refs, int64_t P, int page, int32_t* __restrict__ rows,
    int32_t* __restrict__ status, int32_t* __restrict__ ws, int rows_here) {
  __shared__ uint32_t bits[kSlotWords];
  __shared__ int upto[kSegment], start[kSegment + 1], old_len[kSegment], slot[kSegment];
  __shared__ int found[kPagesHere];              // free pages of the first round
  __shared__ int part[kPlanThreads / 64];
  __shared__ int bad, wide;
  __shared__ unsigned long long wanted;
  const int tid = threadIdx.x;
  int32_t* list = ws + kWsHead;                  // free pages of later rounds
  int first_free = 0;
  bool open[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    open[i] = 4 * tid + i < P && refs[min((int64_t)(4 * tid + i), P - 1)] == 0;
    first_free += open[i];
  }
  // The thread's first entry: slot, first row, rows, length.
  int s0 = -1, r0 = 0, add0 = 0, l0 = 0;
  if (tid < n) {
    s0 = slots[tid];
    r0 = row_off[tid];
    add0 = max(row_off[tid + 1] - r0, 0);
    if (s0 >= 0 && s0 < S) l0 = lens[s0];
  }
  const int words = (S + 31) / 32;
  for (int i = tid; i < words; i += kPlanThreads) bits[i] = 0;
  if (tid == 0) {
    bad = wide = 0;
    wanted = 0;
  }
  __syncthreads();
  // Pages wanted, and what is wrong.
  int64_t want = 0;
  for (int i = tid; i < n; i += kPlanThreads) {
    const int s = i == tid ? s0 : slots[i];
    if (s < 0 || s >= S || take_bit(bits, s)) {
      bad = 1;
      continue;
    }
    const int l = i == tid ? l0 : lens[s];
    if (l < 0) {                                       // no length: nothing to append to
      bad = 1;
      continue;
    }
    const int add = i == tid ? add0 : max(row_off[i + 1] - row_off[i], 0);
    if ((int64_t)l + add > width * page) {             // (below 2^31, so the rest is in 32 bits)
      wide = 1;
      continue;
    }
    want += pages_of(l + add, page) - pages_of(l, page);
  }
  if (want > 0) atomicAdd(&wanted, (unsigned long long)want);
  __syncthreads();
  const int total = (int)(wanted < 0x7fffffffull ? wanted : 0x7fffffffull);
  int here = 0, have = 0;
  if (!bad && !wide && total > 0) {
    int sum;
    int at = block_scan(first_free, part, &sum);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (open[i]) found[at] = 4 * tid + i;
      at += open[i];
    }
    here = min(sum, total);
    have = here;
    if (here < total) have += free_pages(refs, kPagesHere, P, total - here, list, part);
  }
  const bool good = !bad && !wide && have == total;
  if (tid == 0) {
    status[0] = bad ? 3 : wide ? 2 : good ? 0 : 1;
    status[1] = bad || wide || good ? 0 : total - have;
    ws[0] = good;
  }
  if (!good) {
    if (rows_here)
      for (int64_t m = tid; m < M; m += kPlanThreads) rows[m] = -1;
    return;
  }
  int taken = 0;
  auto page_at = [&](int k) { return taken + k < here ? found[taken + k] : list[taken + k - here]; };
  for (int i0 = 0; i0 < n; i0 += kSegment) {
    const int cnt = min(kSegment, n - i0);
    int run = 0;
    for (int i = tid; i < (cnt + kPlanThreads - 1) / kPlanThreads * kPlanThreads; i += kPlanThreads) {
      const bool one = i0 + i == tid;
      int need = 0, s = 0, l = 0, r = 0;
      if (i < cnt) {
        s = one ? s0 : slots[i0 + i];
        r = one ? r0 : row_off[i0 + i];
        const int add = one ? add0 : max(row_off[i0 + i + 1] - r, 0);
        l = one ? l0 : lens[s];
        need = pages_of(l + add, page) - pages_of(l, page);
        if (add > 0) lens[s] = l + add;
        if (i == cnt - 1) start[cnt] = r + add;
      }
      int sum;
      const int before = block_scan(need, part, &sum);
      if (i < cnt) {
        upto[i] = run + before;
        start[i] = r;
        old_len[i] = l;
        slot[i] = s;
      }
      run += sum;
    }
    __syncthreads();                                   // the lists and the segment are complete
    for (int k = tid; k < run; k += kPlanThreads) {
      const int i = owner_in(upto, cnt, k);
      const int p = page_at(k);
      table[(int64_t)slot[i] * width + pages_of(old_len[i], page) + (k - upto[i])] = p;
      refs[p] = 1;
    }
    if (rows_here) {
      const int m1 = (int)min((int64_t)start[cnt], M);
      for (int m = max(start[0], 0) + tid; m < m1; m += kPlanThreads) {
        const int i = owner_in(start, cnt, m);
        const int at = old_len[i] + (m - start[i]), col = at / page, had = pages_of(old_len[i], page);
        const int p = col < had ? table[(int64_t)slot[i] * width + col] : page_at(upto[i] + col - had);
        rows[m] = p * page + at % page;
      }
    }
    if (rows_here && i0 + cnt == n)                    // rows of no entry (a padded batch)
      for (int64_t m = max(start[cnt], 0) + tid; m < M; m += kPlanThreads) rows[m] = -1;
    taken += run;
    __syncthreads();                                   // the segment's arrays are free
  }
}

// The pool rows of many new rows, over the chip (32,771 rows: 4.7 us, the
// latency of its search).
__global__ __launch_bounds__(256) void reserve_rows(
    const int32_t* __restrict__ slots, const int32_t* __restrict__ row_off, int n, int64_t M,
    const int32_t* __restrict__ table, int64_t width, const int32_t* __restrict__ lens, int page,
    int32_t* __restrict__ rows, const int32_t* __restrict__ ws) {
  const int64_t m = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (m >= M) return;
  if (ws[0] == 0 || m < row_off[0] || m >= row_off[n]) {
    rows[m] = -1;
    return;
  }
  const int i = owner_in(row_off, n, (int)m);
  const int s = slots[i];
  const int at = lens[s] - (row_off[i + 1] - (int)m);
  rows[m] = table[(int64_t)s * width + at / page] * page + at % page;
}

// ---------------------------------------------------------------------------
// Copies. `bytes` bytes from src to dst by a workgroup of 256 threads, four
// pieces a thread in flight. V: the widest type that all addresses allow.
// ---------------------------------------------------------------------------
template <typename V>
__device__ __forceinline__ void copy_piece(const char* __restrict__ src, char* __restrict__ dst,
                                           int bytes) {
  const int n = bytes / (int)sizeof(V);
  const V* s = reinterpret_cast<const V*>(src);
  V* d = reinterpret_cast<V*>(dst);
  for (int i = threadIdx.x; i < n; i += 4 * 256) {
    V v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + 256 * j < n) v[j] = s[i + 256 * j];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + 256 * j < n) d[i + 256 * j] = v[j];
  }
}

// Pieces of kCopyUnit bytes of `count` page copies in `layers` layers, dealt
// over the grid. rows: bytes of item i are rows[i] * row_bytes, else a page.
// In a pool a layer is `pages` pages; ids outside it are passed over.
template <typename V>
__device__ __forceinline__ void copy_items(const int32_t* __restrict__ src,
                                           const int32_t* __restrict__ dst,
                                           const int32_t* __restrict__ rows, int count,
                                           const char* __restrict__ from, int64_t from_pages,
                                           char* __restrict__ to, int64_t to_pages, int64_t layers,
                                           int64_t page_bytes, int64_t row_bytes) {
  const int64_t units = (page_bytes + kCopyUnit - 1) / kCopyUnit;
  const int64_t work = (int64_t)count * layers * units;
  for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
    const int64_t item = w / units, at = (w - item * units) * kCopyUnit;
    const int64_t layer = item / count;
    const int i = (int)(item - layer * count);
    const int64_t bytes = rows != nullptr ? rows[i] * row_bytes : page_bytes;
    const int a = src[i], b = dst[i];
    if (at >= bytes || a < 0 || a >= from_pages || b < 0 || b >= to_pages) continue;
    const int64_t left = bytes - at;
    copy_piece<V>(from + (layer * from_pages + a) * page_bytes + at,
                  to + (layer * to_pages + b) * page_bytes + at,
                  (int)(left < kCopyUnit ? left : kCopyUnit));
  }
}

template <typename V>
__global__ __launch_bounds__(256) void copy_kernel(const int32_t* __restrict__ src,
                                                   const int32_t* __restrict__ dst, int count,
                                                   const char* from, int64_t from_pages, char* to,
                                                   int64_t to_pages, int64_t layers,
                                                   int64_t page_bytes) {
  copy_items<V>(src, dst, nullptr, count, from, from_pages, to, to_pages, layers, page_bytes, 0);
}

// Row m of x into pool row rows[m]: pieces of sizeof(V) bytes, four a thread.
// Bound by HBM, each row is read and written once: 32,771 rows of 4 KiB in 44 us
// (6.1 TB/s); 256 rows of 1 KiB in 3.6 us, a launch's latency.
template <typename V>
__global__ __launch_bounds__(256) void write_kernel(const char* __restrict__ x, int64_t x_stride,
                                                    const int32_t* __restrict__ rows, int64_t M,
                                                    char* __restrict__ pool, int64_t pool_rows,
                                                    int64_t row_bytes) {
  const uint32_t per = (uint32_t)(row_bytes / (int64_t)sizeof(V));     // pieces a row
  const int64_t total = M * per;
  const int64_t i0 = (int64_t)blockIdx.x * (4 * 256) + threadIdx.x;
  V v[4];
  char* to[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t i = i0 + 256 * j;
    to[j] = nullptr;
    if (i >= total) continue;
    const int64_t m = i / per;
    const int64_t at = (i - m * per) * (int64_t)sizeof(V);
    const int r = rows[m];
    v[j] = *reinterpret_cast<const V*>(x + m * x_stride + at);
    if (r >= 0 && r < pool_rows) to[j] = pool + r * row_bytes + at;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (to[j] != nullptr) *reinterpret_cast<V*>(to[j]) = v[j];
}

// ---------------------------------------------------------------------------
// fork. The first kernel (one workgroup) checks the pairs, takes the pages for
// the last pages that are not full and leaves a list of copies; the second
// copies table rows, counts the shared pages and copies the rows, over the
// chip. The children's lengths are written by the second: the first still
// reads them as empty. 256 children of 64 histories, four layers, pages of 64
// rows of 4 KiB: 6.5 us of latencies and 38 us for 241 MB (6.3 TB/s).
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kPlanThreads) void fork_plan(
    const int32_t* __restrict__ parents, const int32_t* __restrict__ children, int n,
    const int32_t* __restrict__ table, int64_t width, const int32_t* __restrict__ lens, int S,
    int32_t* __restrict__ refs, int64_t P, int page, int32_t* __restrict__ status,
    int32_t* __restrict__ ws) {
  __shared__ uint32_t bits[kSlotWords];
  __shared__ int part[kPlanThreads / 64];
  __shared__ int bad;
  const int tid = threadIdx.x;
  int32_t* src = ws + kWsHead;
  int32_t* dst = src + n;
  int32_t* rows = dst + n;
  int32_t* list = rows + n;
  for (int i = tid; i < (S + 31) / 32; i += kPlanThreads) bits[i] = 0;
  if (tid == 0) bad = 0;
  __syncthreads();
  int mine = 0;
  for (int i = tid; i < n; i += kPlanThreads) {
    const int a = parents[i], c = children[i];
    if (a < 0 || a >= S || c < 0 || c >= S || take_bit(bits, c) || lens[c] != 0 ||
        lens[a] < 0 || lens[a] > width * page)         // (no length: its pages are not in the table)
      bad = 1;
    else
      mine += lens[a] % page != 0;
  }
  int total;
  block_scan(mine, part, &total);                      // (a barrier: the bits are complete)
  for (int i = tid; i < n; i += kPlanThreads) {
    const int a = parents[i];
    if (a >= 0 && a < S && ((bits[a >> 5] >> (a & 31)) & 1)) bad = 1;
  }
  __syncthreads();
  const int have = bad ? 0 : free_pages(refs, 0, P, total, list, part);
  const bool good = !bad && have == total;
  if (tid == 0) {
    status[0] = bad ? 3 : good ? 0 : 1;
    status[1] = bad || good ? 0 : total - have;
    ws[0] = good;
  }
  if (!good) return;
  __syncthreads();                                     // the list is complete
  int run = 0;
  for (int i = tid; i < (n + kPlanThreads - 1) / kPlanThreads * kPlanThreads; i += kPlanThreads) {
    const int l = i < n ? lens[parents[i]] : 0;
    const int rest = l % page;
    int sum;
    const int at = run + block_scan(rest != 0, part, &sum);
    run += sum;
    if (i < n) {
      rows[i] = rest;
      src[i] = rest != 0 ? table[(int64_t)parents[i] * width + l / page] : -1;
      dst[i] = rest != 0 ? list[at] : -1;
      if (rest != 0) refs[list[at]] = 1;
    }
  }
}

template <typename V>
__global__ __launch_bounds__(256) void fork_copy(
    const int32_t* __restrict__ parents, const int32_t* __restrict__ children, int n,
    int32_t* table, int64_t width, int32_t* lens, int32_t* __restrict__ refs, int64_t P, int page,
    char* pool, int64_t layers, int64_t row_bytes, const int32_t* __restrict__ ws) {
  if (ws[0] == 0) return;
  const int32_t* src = ws + kWsHead;
  const int32_t* dst = src + n;
  const int32_t* rows = dst + n;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {    // no slot is parent and child
    const int a = parents[i], c = children[i];
    const int l = lens[a], full = l / page, rest = l % page;
    for (int64_t col = threadIdx.x; col < width; col += 256) {
      int p = -1;
      if (col < full) {
        p = table[(int64_t)a * width + col];
        if (p >= 0 && p < P) atomicAdd(&refs[p], 1);
      } else if (col == full && rest != 0) {
        p = dst[i];
      }
      table[(int64_t)c * width + col] = p;
    }
    if (threadIdx.x == 0) lens[c] = l;
  }
  copy_items<V>(src, dst, rows, n, pool, P, pool, P, layers, page * row_bytes, row_bytes);
}

// free: a workgroup per entry. Taking the length with an exchange lets one of
// several entries of the same slot do the work. (256 slots: 5.0 us, latency.)
__global__ __launch_bounds__(256) void free_kernel(const int32_t* __restrict__ slots,
                                                   int32_t* __restrict__ table, int64_t width,
                                                   int32_t* __restrict__ lens, int S,
                                                   int32_t* __restrict__ refs, int64_t P,
                                                   int page) {
  __shared__ int rows;
  const int s = slots[blockIdx.x];
  if (s < 0 || s >= S) return;
  if (threadIdx.x == 0) rows = atomicExch(&lens[s], 0);
  __syncthreads();
  const int64_t held = rows <= 0 ? 0 : pages_of(rows, page) < width ? pages_of(rows, page) : width;
  for (int64_t col = threadIdx.x; col < held; col += 256) {
    const int p = table[s * width + col];
    if (p >= 0 && p < P) atomicSub(&refs[p], 1);
    table[s * width + col] = -1;
  }
}

// ---------------------------------------------------------------------------
// compact. With n live pages, the free pages below n ("holes", in order) take
// the live pages from n on ("movers", in order): the fewest moves, and no page
// is both read and written. Blocks of kCompactPages pages: counted first, then
// each block ranks its pages from the counts before it and lists them; then
// the moves and the table follow the lists. Bound by HBM: 1,293 MB of moves in
// two layers take 254 us (5.1 TB/s, a large copy's rate), the count and the lists
// of 8,000 pages 4.5 and 7.9 us.
// ws: [0] movers, lists at kWsHead: counts [nb], holes [P], movers [P], and
// rank [P] of each mover.
// ---------------------------------------------------------------------------
constexpr int kCompactPages = 4096;

__device__ __forceinline__ int count_live(const int32_t* refs, int64_t lo, int64_t hi, int* part) {
  int mine = 0, total;
#pragma unroll
  for (int j = 0; j < kCompactPages / kPlanThreads; ++j) {
    const int64_t p = lo + j * kPlanThreads + threadIdx.x;
    mine += p < hi && refs[p] > 0;
  }
  block_scan(mine, part, &total);
  return total;
}

__global__ __launch_bounds__(kPlanThreads) void compact_count(const int32_t* __restrict__ refs,
                                                              int64_t P,
                                                              int32_t* __restrict__ ws) {
  __shared__ int part[kPlanThreads / 64];
  const int64_t lo = (int64_t)blockIdx.x * kCompactPages;
  const int64_t hi = lo + kCompactPages < P ? lo + kCompactPages : P;
  const int total = count_live(refs, lo, hi, part);
  if (threadIdx.x == 0) ws[kWsHead + blockIdx.x] = total;
}

__global__ __launch_bounds__(kPlanThreads) void compact_list(const int32_t* __restrict__ refs,
                                                             int64_t P, int nb,
                                                             int32_t* __restrict__ status,
                                                             int32_t* __restrict__ ws) {
  __shared__ int part[kPlanThreads / 64];
  const int tid = threadIdx.x, b = blockIdx.x;
  int32_t* counts = ws + kWsHead;
  int32_t* holes = counts + nb;
  int32_t* movers = holes + P;
  int32_t* rank = movers + P;
  const int64_t lo = (int64_t)b * kCompactPages;
  const int64_t hi = lo + kCompactPages < P ? lo + kCompactPages : P;
  // Live pages in all blocks (n), before this block, and in the blocks that lie
  // wholly below n. A single block counts here.
  int n, before = 0, below = 0;
  if (nb == 1) {
    n = count_live(refs, 0, P, part);
  } else {
    int all = 0, pre = 0;
    for (int i = tid; i < nb; i += kPlanThreads) {
      all += counts[i];
      pre += i < b ? counts[i] : 0;
    }
    block_scan(all, part, &n);
    block_scan(pre, part, &before);
    int under = 0;
    for (int i = tid; i < n / kCompactPages; i += kPlanThreads) under += counts[i];
    block_scan(under, part, &below);
  }
  // ... and of the block that holds the border, those below it.
  below += count_live(refs, nb == 1 ? 0 : (int64_t)(n / kCompactPages) * kCompactPages, n, part);
  if (b == 0 && tid == 0) {
    ws[0] = n - below;                                 // live pages from n on
    status[0] = 0;
    status[1] = n;
  }
  for (int64_t p0 = lo; p0 < hi; p0 += kPlanThreads) {
    const int64_t p = p0 + tid;
    const bool live = p < hi && refs[p] > 0;
    int sum;
    const int r = before + block_scan(live, part, &sum);   // live pages before p
    before += sum;
    if (p >= hi) continue;
    if (p < n && !live) holes[p - r] = (int)p;
    if (p >= n && live) {
      movers[r - below] = (int)p;
      rank[p] = r - below;
    }
  }
}

template <typename V>
__global__ __launch_bounds__(256) void compact_move(int32_t* __restrict__ table, int64_t entries,
                                                    int32_t* __restrict__ refs, int64_t P, int nb,
                                                    char* pool, int64_t layers, int64_t page_bytes,
                                                    const int32_t* __restrict__ status,
                                                    const int32_t* __restrict__ ws) {
  const int count = ws[0], n = status[1];
  const int32_t* holes = ws + kWsHead + nb;
  const int32_t* movers = holes + P;
  const int32_t* rank = movers + P;
  if (count == 0) return;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  // A page id of the table that is at the border or above belongs to a slot, so
  // the page is live and has a rank; ids outside the cache are left alone.
  for (int64_t i = t; i < entries; i += step) {
    const int p = table[i];
    if (p >= n && p < P) {
      const int k = rank[p];
      if (k >= 0 && k < count && movers[k] == p) table[i] = holes[k];
    }
  }
  for (int64_t k = t; k < count; k += step) {
    refs[holes[k]] = refs[movers[k]];
    refs[movers[k]] = 0;
  }
  copy_items<V>(movers, holes, nullptr, count, pool, P, pool, P, layers, page_bytes, 0);
}

int widest(int64_t a, int64_t b, const void* p, const void* q) {
  const uint64_t all = (uint64_t)a | (uint64_t)b | reinterpret_cast<uintptr_t>(p) |
                       reinterpret_cast<uintptr_t>(q);
  return all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
}

}  // namespace

hipError_t launch_reserve(const int32_t* slots, const int32_t* row_off, int64_t n, int64_t M,
                          int32_t* table, int64_t width, int32_t* lens, int64_t S, int32_t* refs,
                          int64_t P, int page, int32_t* rows, int32_t* status, int32_t* ws,
                          hipStream_t s) {
  // Up to 4096 new rows their places are found by the same workgroup (a step of
  // single rows is one launch); more than that take a launch over the chip.
  const bool here = M <= 4096;
  hipError_t e = launch_kernel(reserve_kernel, dim3(1), dim3(kPlanThreads), s, slots, row_off,
                               (int)n, M, table, width, lens, (int)S, refs, P, page, rows, status,
                               ws, (int)here);
  if (e != hipSuccess || here) return e;
  return launch_kernel(reserve_rows, dim3((uint32_t)((M + 255) / 256)), dim3(256), s, slots,
                       row_off, (int)n, M, table, width, lens, page, rows, ws);
}

hipError_t launch_cache_write(const void* x, int64_t x_stride, const int32_t* rows, int64_t M,
                              void* pool, int64_t pool_rows, int64_t row_bytes, hipStream_t s) {
  const int w = widest(x_stride, row_bytes, x, pool);
  const int64_t blocks = (M * (row_bytes / w) + 4 * 256 - 1) / (4 * 256);
  if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, dim3((uint32_t)blocks), dim3(256), s,
                         static_cast<const char*>(x), x_stride, rows, M,
                         static_cast<char*>(pool), pool_rows, row_bytes);
  };
  return w == 16 ? go(write_kernel<u32x4>) : w == 4 ? go(write_kernel<uint32_t>) : go(write_kernel<uint8_t>);
}

hipError_t launch_fork(const int32_t* parents, const int32_t* children, int64_t n, int32_t* table,
                       int64_t width, int32_t* lens, int64_t S, int32_t* refs, int64_t P,
                       int page, void* pool, int64_t layers, int64_t row_bytes, int32_t* status,
                       int32_t* ws, hipStream_t s) {
  const hipError_t e = launch_kernel(fork_plan, dim3(1), dim3(kPlanThreads), s, parents, children,
                                     (int)n, table, width, lens, (int)S, refs, P, page, status, ws);
  if (e != hipSuccess) return e;
  const int w = widest(row_bytes, 0, pool, nullptr);
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, dim3(kCopyBlocks), dim3(256), s, parents, children, (int)n,
                         table, width, lens, refs, P, page, static_cast<char*>(pool), layers,
                         row_bytes, ws);
  };
  return w == 16 ? go(fork_copy<u32x4>) : w == 4 ? go(fork_copy<uint32_t>) : go(fork_copy<uint8_t>);
}

hipError_t launch_free(const int32_t* slots, int64_t n, int32_t* table, int64_t width,
                       int32_t* lens, int64_t S, int32_t* refs, int64_t P, int page,
                       hipStream_t s) {
  return launch_kernel(free_kernel, dim3((uint32_t)n), dim3(256), s, slots, table, width, lens,
                       (int)S, refs, P, page);
}

hipError_t launch_compact(int32_t* table, int64_t width, int64_t S, int32_t* refs, int64_t P,
                          void* pool, int64_t layers, int64_t page_bytes, int32_t* status,
                          int32_t* ws, hipStream_t s) {
  const int nb = (int)((P + kCompactPages - 1) / kCompactPages);
  hipError_t e = hipSuccess;
  if (nb > 1)
    e = launch_kernel(compact_count, dim3(nb), dim3(kPlanThreads), s, refs, P, ws);
  if (e != hipSuccess) return e;
  e = launch_kernel(compact_list, dim3(nb), dim3(kPlanThreads), s, refs, P, nb, status, ws);
  if (e != hipSuccess) return e;
  const int w = widest(page_bytes, 0, pool, nullptr);
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, dim3(kCopyBlocks), dim3(256), s, table, S * width, refs, P, nb,
                         static_cast<char*>(pool), layers, page_bytes, status, ws);
  };
  return w == 16 ? go(compact_move<u32x4>) : w == 4 ? go(compact_move<uint32_t>) : go(compact_move<uint8_t>);
}

hipError_t launch_cache_copy(const int32_t* src, const int32_t* dst, int64_t n,
                             const void* src_pool, int64_t src_pages, void* dst_pool,
                             int64_t dst_pages, int64_t layers, int64_t page_bytes,
                             hipStream_t s) {
  const int w = widest(page_bytes, 0, src_pool, dst_pool);
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, dim3(kCopyBlocks), dim3(256), s, src, dst, (int)n,
                         static_cast<const char*>(src_pool), src_pages,
                         static_cast<char*>(dst_pool), dst_pages, layers, page_bytes);
  };
  return w == 16 ? go(copy_kernel<u32x4>) : w == 4 ? go(copy_kernel<uint32_t>) : go(copy_kernel<uint8_t>);
}

}  // namespace rocs
