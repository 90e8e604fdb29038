// The pages of the 4-bit cache: taking, sharing, giving back, compacting and
// copying them (gfx950).
//
// The table is a few thousand words, and what a call decides depends on the
// rows before it (pages are taken lowest first, rows in order), so one
// workgroup decides: prefix sums over the rows and over the free pages.  The
// bytes that move, 10 to 100 KB a page and layer, are another launch over the
// whole chip that reads what was decided.  Counts are integers, so the order
// in which atomics reach them does not show.
//
// The deciding launches are bound by their trips to memory, one after the other
// (slots, lengths, last pages, counts of pages): 60 forks 7.9 us, room for 32
// rows 5.7 us, a compaction's plan 2.8 us, freeing 2 to 4 us.  The copies are
// bound by HBM: 53 MB written in 11.2 us (4.8 TB/s; what is read is 7 MB of
// shared pages and the caches), 64 MB of a compaction read and written in 23.7,
// 5.4 TB/s.  (1024 threads for any number of rows: 9.6
// and 7.0 us; the free pages of a thread handed out one after the other: 11.6.)
// Free pages are searched for from page 0 on, 4096 a pass, and a compaction's
// plan walks the pool twice: room for 64 rows 7.2 us in a pool of 1000 pages
// and 57 in one of 100000, 92 % of them in use, a compaction with nothing to
// move 4.2 and 80.

#include "q4_internal.h"

namespace tq {
namespace {

// Exclusive prefix sum of v over the workgroup's T threads; *total the sum.
template <int T>
__device__ inline int scan(int v, int* total, int* lds /*[T / 64]*/) {
  const int wave = threadIdx.x >> 6;
  const int x = wave_scan(v);
  __syncthreads();   // lds may still be read from the call before
  if ((threadIdx.x & 63) == 63) lds[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) {
    const int n = lds[w];
    before += w < wave ? n : 0;
    all += n;
  }
  *total = all;
  return x - v + before;
}

__device__ inline bool page_ok(const KvDev& c, int p) { return p >= 0 && p < c.n_pages; }
__device__ inline int pages_of(const KvDev& c, int len) { return (int)(((int64_t)len + c.page_size - 1) >> c.page_shift); }
__device__ inline int len_of(const KvDev& c, int seq) {
  // A length outside what the slot can hold is taken as the nearest one.
  return (int)min(max((int64_t)c.lens[seq], (int64_t)0), (int64_t)c.max_pages * c.page_size);
}

// Row i of the call names a slot that an earlier row names (slots: the rows'
// slots in LDS, T of them).
template <int T>
__device__ inline bool named_before(const int* slots, int i, int n_rows) {
  const int mine = slots[i];
  bool found = false;
  for (int j = 0; j < n_rows; j += 8)
#pragma unroll
    for (int e = 0; e < 8; ++e) found |= j + e < i && slots[min(j + e, T - 1)] == mine;
  return found;
}

// Hands the `total` lowest free pages out: give(k, page) for the k-th of
// them, k < total.  Returns how many there were.  Called by all T threads, each
// of which looks at 16 pages beside each other in a pass.
template <int T, class F>
__device__ int take_free(const KvDev& c, int total, int* lds, F give) {
  constexpr int kEach = 4096 / T;
  __shared__ int list[4096];
  int found = 0;
  for (int64_t p0 = 0; p0 < c.n_pages && found < total; p0 += 4096) {
    const int64_t p = p0 + threadIdx.x * kEach;
    uint32_t free = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) free |= (uint32_t)(c.refs[min(p + e, (int64_t)c.n_pages - 1)] == 0 && p + e < c.n_pages) << e;
    int all;
    int at = found + scan<T>(__popc(free), &all, lds);
    // Listed first, so that pages beside each other go to different threads.
    for (at -= found; free != 0; free &= free - 1) list[at++] = (int)p + __ffs(free) - 1;
    __syncthreads();
    for (int k = found + threadIdx.x; k < min(found + all, total); k += T) give(k, list[k - found]);
    found += all;
    __syncthreads();
  }
  return min(found, total);
}

// The row whose share [base[r], base[r+1]) of the pages holds k.
__device__ inline int row_with(const int* base, int n, int k) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (base[mid] <= k)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

template <int T>
__global__ void __launch_bounds__(T) kv_extend_kernel(KvDev c, const int32_t* __restrict__ seqs,
                                                             const int32_t* __restrict__ cu, int n_rows,
                                                             int32_t* __restrict__ starts,
                                                             int32_t* __restrict__ d_err) {
  __shared__ int lds[T / 64], slots[T], base[T], have[T];
  const int i = threadIdx.x;
  const bool row = i < n_rows;
  const int seq = row ? (seqs ? seqs[i] : i) : -1;
  slots[i] = seq;
  __syncthreads();
  bool ok = row && seq >= 0 && seq < c.n_seqs && !(seqs && named_before<T>(slots, i, n_rows));
  int len = 0, need = 0;
  int64_t want = 0;
  if (ok) {
    len = len_of(c, seq);
    const int64_t n = cu ? (int64_t)cu[i + 1] - cu[i] : 1;
    want = len + n;
    ok = n >= 0 && want <= (int64_t)c.max_pages * c.page_size && want <= INT32_MAX;
    if (ok && n > 0 && (len & (c.page_size - 1)) != 0) {
      const int last = c.pages[(int64_t)seq * c.max_pages + (len >> c.page_shift)];
      ok = page_ok(c, last) && c.refs[last] == 1;
    }
    if (ok) need = pages_of(c, (int)want) - pages_of(c, len);
  }
  int total;
  // Rows of a call ask for 2^20 pages each at most, 2^30 together.
  base[i] = scan<T>(need, &total, lds);
  have[i] = pages_of(c, len);
  __syncthreads();
  const int got = take_free<T>(c, total, lds, [&](int k, int page) {
    const int r = row_with(base, n_rows, k);
    c.pages[(int64_t)slots[r] * c.max_pages + have[r] + (k - base[r])] = page;
    c.refs[page] = 1;
  });
  __threadfence_block();
  __syncthreads();
  if (!row) return;
  if (ok && base[i] + need > got && need > 0) {
    // What was handed to a row that does not get all it asked for goes back.
    for (int k = base[i]; k < got; ++k) {
      int32_t* e = &c.pages[(int64_t)seq * c.max_pages + have[i] + (k - base[i])];
      c.refs[*e] = 0;
      *e = -1;
    }
    ok = false;
  }
  starts[i] = ok ? len : -1;
  if (ok)
    c.lens[seq] = (int)want;
  else if (d_err)
    atomicAdd(d_err, 1);
}

__global__ void __launch_bounds__(256) kv_free_kernel(KvDev c, const int32_t* __restrict__ seqs,
                                                      int32_t* __restrict__ d_err) {
  __shared__ int again;
  const int i = blockIdx.x, seq = seqs ? seqs[i] : i;
  if (threadIdx.x == 0) again = 0;
  __syncthreads();
  if (seqs)
    for (int j = threadIdx.x; j < i; j += 256)
      if (seqs[j] == seq) again = 1;
  __syncthreads();
  if (again || seq < 0 || seq >= c.n_seqs) {
    if (threadIdx.x == 0 && d_err) atomicAdd(d_err, 1);
    return;
  }
  const int n = pages_of(c, len_of(c, seq));
  int32_t* row = c.pages + (int64_t)seq * c.max_pages;
  for (int p = threadIdx.x; p < n; p += 256) {
    const int page = row[p];
    if (page_ok(c, page)) atomicSub(&c.refs[page], 1);
    row[p] = -1;
  }
  __syncthreads();
  if (threadIdx.x == 0) c.lens[seq] = 0;
}

// A fork's decisions: per row {source page, destination page} of the last
// page (-1: none to copy), {pages to share, or -1 for a refused row, length}.
struct ForkRow {
  int32_t src, dst, share, len;
};

template <int T>
__global__ void __launch_bounds__(T) kv_fork_kernel(KvDev c, const int32_t* __restrict__ parents,
                                                           const int32_t* __restrict__ children, int n_rows,
                                                           int32_t* __restrict__ d_err,
                                                           ForkRow* __restrict__ rows) {
  __shared__ int lds[T / 64], slots[T], base[T], dst[T];
  const int i = threadIdx.x;
  const bool row = i < n_rows;
  const int child = row ? children[i] : -1, parent = row ? parents[i] : -1;
  slots[i] = child;
  dst[i] = -1;
  __syncthreads();
  bool ok = row && child >= 0 && child < c.n_seqs && parent >= 0 && parent < c.n_seqs && child != parent &&
            c.lens[child] <= 0 && !named_before<T>(slots, i, n_rows);
  int len = 0, need = 0, src = -1;
  if (ok) {
    len = len_of(c, parent);
    if ((len & (c.page_size - 1)) != 0) {
      src = c.pages[(int64_t)parent * c.max_pages + (len >> c.page_shift)];
      ok = page_ok(c, src);
      need = ok;
    }
  }
  int total;
  base[i] = scan<T>(need, &total, lds);
  __syncthreads();
  // Page k goes to the last row whose share starts at or before it: of rows that
  // start there, all but the last need none.
  take_free<T>(c, total, lds, [&](int k, int page) {
    dst[row_with(base, n_rows, k)] = page;
    c.refs[page] = 1;
  });
  __syncthreads();
  if (!row) return;
  if (need && dst[i] < 0) ok = false;
  ForkRow f;
  f.src = ok && need ? src : -1;
  f.dst = ok && need ? dst[i] : -1;
  f.share = ok ? len >> c.page_shift : -1;
  f.len = len;
  rows[i] = f;
  if (!ok && d_err) atomicAdd(d_err, 1);
}

constexpr int kChunk = 16 * 1024;   // bytes of a page that a workgroup copies at a time

// `count` 16-byte words by the workgroup, four loads in flight a thread.
__device__ inline void copy_words(const u4v* __restrict__ s, u4v* __restrict__ d, int count) {
  for (int i = threadIdx.x; i < count; i += 1024) {
    u4v t[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + 256 * e < count) t[e] = s[i + 256 * e];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + 256 * e < count) d[i + 256 * e] = t[e];
  }
}

// Part `part` of `parts` of page src of `layer` to page dst.
__device__ inline void copy_part(const KvDev& c, int layer, int src, int dst, int part) {
  uint8_t* base = c.data + layer * c.layer_bytes;
  const int64_t at = (int64_t)part * kChunk;
  const int n = (int)min((int64_t)kChunk, c.page_bytes - at);
  copy_words(reinterpret_cast<const u4v*>(base + src * c.page_bytes + at),
             reinterpret_cast<u4v*>(base + dst * c.page_bytes + at), n / 16);
}

// Workgroup (part, layer, row): the row's last page; that of part 0 and layer
// 0 the row's table as well.
__global__ void __launch_bounds__(256) kv_fork_copy_kernel(KvDev c, const int32_t* __restrict__ parents,
                                                           const int32_t* __restrict__ children,
                                                           const ForkRow* __restrict__ rows) {
  const int i = blockIdx.z;
  const ForkRow f = rows[i];
  if (f.share < 0) return;
  if (f.dst >= 0) copy_part(c, blockIdx.y, f.src, f.dst, blockIdx.x);
  if (blockIdx.x != 0 || blockIdx.y != 0) return;
  const int32_t* from = c.pages + (int64_t)parents[i] * c.max_pages;
  int32_t* to = c.pages + (int64_t)children[i] * c.max_pages;
  for (int p = threadIdx.x; p < f.share; p += 256) {
    const int page = from[p];
    to[p] = page;
    if (page_ok(c, page)) atomicAdd(&c.refs[page], 1);
  }
  if (threadIdx.x == 0) {
    if (f.dst >= 0) to[f.share] = f.dst;
    c.lens[children[i]] = f.len;
  }
}

// What a compaction decides: how many pages move, from where, to where, and
// the new number of every page.
struct Compact {
  int32_t* count;
  int32_t* from;
  int32_t* to;
  int32_t* map;
};

__global__ void __launch_bounds__(1024) kv_compact_kernel(KvDev c, int32_t* __restrict__ n_live, Compact w) {
  constexpr int kThreads = 1024;
  __shared__ int lds[kThreads / 64];
  int mine = 0;
  for (int64_t p = threadIdx.x; p < c.n_pages; p += kThreads) mine += c.refs[p] > 0;
  int live;
  scan<kThreads>(mine, &live, lds);
  int holes = 0, movers = 0;
  for (int64_t p0 = 0; p0 < c.n_pages; p0 += kThreads) {
    const int64_t p = p0 + threadIdx.x;
    const bool in = p < c.n_pages, used = in && c.refs[p] > 0;
    const bool hole = in && p < live && !used, mover = used && p >= live;
    int all;
    // At most 1024 of each: both counts in one word.
    const int at = scan<kThreads>(hole | (mover << 16), &all, lds);
    if (hole) w.to[holes + (at & 0xFFFF)] = (int)p;
    if (mover) w.from[movers + (at >> 16)] = (int)p;
    if (in) w.map[p] = (int)p;
    holes += all & 0xFFFF;
    movers += all >> 16;
  }
  __threadfence_block();
  __syncthreads();
  for (int k = threadIdx.x; k < movers; k += kThreads) {
    const int f = w.from[k], t = w.to[k];
    w.map[f] = t;
    c.refs[t] = c.refs[f];
    c.refs[f] = 0;
  }
  if (threadIdx.x == 0) {
    *w.count = movers;
    if (n_live) *n_live = live;
  }
}

__global__ void __launch_bounds__(256) kv_compact_move_kernel(KvDev c, Compact w, int parts) {
  const int n = *w.count;
  if (n == 0) return;
  const int64_t entries = (int64_t)c.n_seqs * c.max_pages;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < entries; e += (int64_t)gridDim.x * 256) {
    const int p = c.pages[e];
    if (page_ok(c, p) && w.map[p] != p) c.pages[e] = w.map[p];
  }
  const int64_t jobs = (int64_t)n * c.n_layers * parts;
  for (int64_t j = blockIdx.x; j < jobs; j += gridDim.x) {
    const int part = (int)(j % parts), layer = (int)(j / parts % c.n_layers), k = (int)(j / parts / c.n_layers);
    copy_part(c, layer, w.from[k], w.to[k], part);
  }
}

__global__ void __launch_bounds__(256) kv_copy_kernel(KvDev c, const int32_t* __restrict__ src,
                                                      const int32_t* __restrict__ dst,
                                                      int32_t* __restrict__ d_err) {
  const int i = blockIdx.z, s = src[i], d = dst[i];
  if (!page_ok(c, s) || !page_ok(c, d)) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && d_err) atomicAdd(d_err, 1);
    return;
  }
  if (s != d) copy_part(c, blockIdx.y, s, d, blockIdx.x);
}

int parts_of(const KvDev& c) { return (int)((c.page_bytes + kChunk - 1) / kChunk); }

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

}  // namespace

size_t kv_workspace_bytes(const KvDev& c, int n_rows) {
  if (n_rows > 0) return sizeof(ForkRow) * (size_t)n_rows;
  return 16 + 3 * up16(4 * (size_t)c.n_pages);
}

hipError_t launch_kv_extend(const KvDev& c, const int32_t* seqs, const int32_t* cu, int n_rows, int32_t* starts,
                            int32_t* d_err, hipStream_t s) {
  if (n_rows <= 256)
    kv_extend_kernel<256><<<1, 256, 0, s>>>(c, seqs, cu, n_rows, starts, d_err);
  else
    kv_extend_kernel<TQ_KV_MAX_ROWS><<<1, TQ_KV_MAX_ROWS, 0, s>>>(c, seqs, cu, n_rows, starts, d_err);
  return hipGetLastError();
}

hipError_t launch_kv_free(const KvDev& c, const int32_t* seqs, int n_rows, int32_t* d_err, hipStream_t s) {
  kv_free_kernel<<<n_rows, 256, 0, s>>>(c, seqs, d_err);
  return hipGetLastError();
}

hipError_t launch_kv_fork(const KvDev& c, const int32_t* parents, const int32_t* children, int n_rows,
                          int32_t* d_err, void* ws, hipStream_t s) {
  ForkRow* rows = static_cast<ForkRow*>(ws);
  if (n_rows <= 256)
    kv_fork_kernel<256><<<1, 256, 0, s>>>(c, parents, children, n_rows, d_err, rows);
  else
    kv_fork_kernel<TQ_KV_MAX_ROWS><<<1, TQ_KV_MAX_ROWS, 0, s>>>(c, parents, children, n_rows, d_err, rows);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  kv_fork_copy_kernel<<<dim3(parts_of(c), c.n_layers, n_rows), 256, 0, s>>>(c, parents, children, rows);
  return hipGetLastError();
}

hipError_t launch_kv_compact(const KvDev& c, int32_t* n_live, void* ws, hipStream_t s) {
  uint8_t* p = static_cast<uint8_t*>(ws);
  const size_t list = up16(4 * (size_t)c.n_pages);
  Compact w;
  w.count = reinterpret_cast<int32_t*>(p);
  w.from = reinterpret_cast<int32_t*>(p + 16);
  w.to = reinterpret_cast<int32_t*>(p + 16 + list);
  w.map = reinterpret_cast<int32_t*>(p + 16 + 2 * list);
  kv_compact_kernel<<<1, 1024, 0, s>>>(c, n_live, w);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  kv_compact_move_kernel<<<2048, 256, 0, s>>>(c, w, parts_of(c));
  return hipGetLastError();
}

hipError_t launch_kv_copy_pages(const KvDev& c, const int32_t* src, const int32_t* dst, int n, int32_t* d_err,
                                hipStream_t s) {
  kv_copy_kernel<<<dim3(parts_of(c), c.n_layers, n), 256, 0, s>>>(c, src, dst, d_err);
  return hipGetLastError();
}

}  // namespace tq
