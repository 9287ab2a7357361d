// Pages of a cache: reserving, forking, freeing and compacting (an extension, not in the paper).  The calls move whole
// pages of bytes, whatever those hold, and keep the books: table[b][i] (page of rows i * page_rows .. of sequence b, -1
// behind the last), refs[p] (table entries that name page p; 0: free), len[b].
//
// Bookkeeping is a few thousand integers: one CTA does it, every thread a contiguous run of pages, so that one scan
// over the threads puts free pages (or pages to move) in index order; no result depends on the order of atomics.  It
// leaves a list of (source, destination) pages in scratch, which a second kernel (launched to overlap) copies for every
// pool, bound by HBM: 2 bytes moved per byte of page.
#include <algorithm>

#include "common.cuh"

namespace dl {

constexpr int kPgThreads = 1024;
constexpr int kPgCopyThreads = 256;
constexpr int kPgChunk = 16 * 1024;       // bytes a CTA copies at a time: four 16-byte loads in flight per thread
constexpr int kPgPools = 64;              // pools per copy launch

struct PgArgs {
  int32_t* table; int32_t* refs; int32_t* len;
  int32_t B, n_pages, W, shift;           // W: columns of the table; page_rows = 1 << shift
  int32_t* hdr; int32_t* src; int32_t* dst; int32_t* map; int32_t* fresh;   // scratch, see pg_scratch
  DeviceStatus* status;
};

struct PgPools { char* p[kPgPools]; };

// Two exclusive scans at once over the CTA's threads; sums: the totals.  sh: 32 int2, not used again by the caller.
__device__ __forceinline__ int2 pg_scan2(int2 v, int2* sh, int2* sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int2 run = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, run.x, o), y = __shfl_up_sync(0xffffffffu, run.y, o);
    if (lane >= o) { run.x += x; run.y += y; }
  }
  if (lane == 31) sh[warp] = run;
  __syncthreads();
  // every warp adds up the 32 warps' totals for itself
  int2 t = sh[lane], all = t;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, t.x, o), y = __shfl_up_sync(0xffffffffu, t.y, o);
    if (lane >= o) { t.x += x; t.y += y; }
  }
  *sums = make_int2(__shfl_sync(0xffffffffu, t.x, 31), __shfl_sync(0xffffffffu, t.y, 31));
  return make_int2(__shfl_sync(0xffffffffu, t.x - all.x, warp) + run.x - v.x, __shfl_sync(0xffffffffu, t.y - all.y, warp) + run.y - v.y);
}
__device__ __forceinline__ bool pg_valid(const PgArgs& a, int p) { return (unsigned)p < (unsigned)a.n_pages; }
// this thread's run of pages
__device__ __forceinline__ void pg_run(const PgArgs& a, int& from, int& to) {
  const int per = (a.n_pages + kPgThreads - 1) / kPgThreads;
  from = min(a.n_pages, (int)threadIdx.x * per);
  to = min(a.n_pages, from + per);
}
__device__ __forceinline__ int pg_pages_of(const PgArgs& a, int n) {
  return (int)min((long long)a.W, ((long long)max(n, 0) + (1 << a.shift) - 1) >> a.shift);
}

// Every sequence gets the pages for len[b] + need[b] rows, the lowest free ones in order of b; all or nothing.
__global__ void __launch_bounds__(kPgThreads)
pages_reserve_kernel(const PgArgs a, const int32_t* need) {
  extern __shared__ int sm[];
  chained_wait();
  int* have = sm;                         // [B] pages a sequence has
  int* first = sm + a.B;                  // [B + 1] pages handed out in front of it
  __shared__ int2 sh[32];
  __shared__ int too_long;
  if (threadIdx.x == 0) too_long = a.B;
  int from, to;
  pg_run(a, from, to);
  int2 mine = make_int2(0, 0), sums;      // pages wanted by this thread's sequences, free pages in its run
  for (int p = from; p < to; ++p) mine.y += a.refs[p] == 0;
  __syncthreads();
  const int per = (a.B + kPgThreads - 1) / kPgThreads, b0 = min(a.B, (int)threadIdx.x * per), b1 = min(a.B, b0 + per);
  for (int b = b0; b < b1; ++b) {
    const int32_t* row = a.table + (size_t)b * a.W;
    const int len = max(a.len[b], 0);
    // a row's pages come first, as many as its rows take at least: look there, and search if that is not so
    int lo = pg_pages_of(a, len), hi = lo;
    const bool here = lo == 0 || row[lo - 1] >= 0, end = lo == a.W || row[lo] < 0;
    if (!here) lo = 0;
    else if (!end) hi = a.W;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (row[mid] >= 0) lo = mid + 1; else hi = mid;
    }
    have[b] = lo;
    const long long rows = (long long)len + max(__ldcg(need + b), 0);
    const long long want = (rows + (1 << a.shift) - 1) >> a.shift;
    if (want > a.W) atomicMin(&too_long, b);
    first[b] = mine.x;
    mine.x += (int)max(0LL, min(want, (long long)a.W) - lo);
  }
  const int2 before = pg_scan2(mine, sh, &sums);
  const int wanted = sums.x, free_pages = sums.y;
  for (int b = b0; b < b1; ++b) first[b] += before.x;
  if (threadIdx.x == 0) first[a.B] = wanted;
  int rank = before.y;
  __syncthreads();
  if (too_long < a.B || free_pages < wanted) {
    if (threadIdx.x == 0) report_status(a.status, DL_ERR_CAPACITY, too_long < a.B ? too_long : -1);
    return;
  }
  for (int p = from; p < to && rank < wanted; ++p) {
    if (a.refs[p] != 0) continue;
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= rank) lo = mid; else hi = mid - 1;
    }
    const int at = have[lo] + rank - first[lo];
    if (DL_IN_BOUNDS(a.status, KID_PAGES, (long long)lo * a.W + at, (long long)a.B * a.W) && at < a.W) {
      a.table[(size_t)lo * a.W + at] = p;
      a.refs[p] = 1;
    }
    ++rank;
  }
}

__global__ void pages_free_kernel(const PgArgs a, const uint8_t* gone) {
  chained_go();
  chained_wait();
  const int b = blockIdx.x;
  if (!__ldcg(gone + b)) return;
  for (int i = threadIdx.x; i < a.W; i += blockDim.x) {
    const int p = a.table[(size_t)b * a.W + i];
    if (pg_valid(a, p)) atomicSub(a.refs + p, 1);
    a.table[(size_t)b * a.W + i] = -1;
  }
  if (threadIdx.x == 0) a.len[b] = 0;
}

// Sequence b becomes a fork of parent[b] as that was before the call.  Full pages are shared; of the children that need a
// parent's partly filled last page one keeps it (the parent itself if it stays, else the lowest) and each other one
// gets the lowest free page for a copy.  All or nothing.
// The counts and the table's rows, old and new, are kept in shared memory where they fit (near: 1 | 2), else in global
// memory, with a round trip for each step of the bookkeeping.
__global__ void __launch_bounds__(kPgThreads)
pages_fork_kernel(const PgArgs a, const int32_t* parent, int32_t near) {
  extern __shared__ int sm[];
  int* par = sm;                          // [B]
  int* low = sm + a.B;                    // [B] lowest child
  int* len = sm + 2 * a.B;                // [B] lengths before the call
  int* copy = sm + 3 * a.B;               // [B] the last page is to be copied
  int* mine_dst = sm + 4 * a.B;           // [B] pages handed out, in order
  int* more = sm + 5 * a.B;
  const unsigned cells = (unsigned)a.B * (unsigned)a.W;                      // below 2^31
  volatile int* refs = (near & 1) ? more : a.refs;
  if (near & 1) more += a.n_pages;
  volatile int* fresh = (near & 2) ? more : a.fresh;
  const int* old_rows = (near & 2) ? more + cells : a.table;
  __shared__ int2 sh[32];
  const int T = kPgThreads, tid = threadIdx.x;
  chained_go();
  chained_wait();
  // everything that is read, in one round trip where it fits
  if (near & 1)
    for (int p = tid; p < a.n_pages; p += T) refs[p] = a.refs[p];
  if (near & 2)
    for (unsigned i = tid; i < cells; i += T) const_cast<int*>(old_rows)[i] = a.table[i];
  for (int b = tid; b < a.B; b += T) {
    int p = __ldcg(parent + b);
    if (p < -1 || p >= a.B) {
      report_status(a.status, DL_ERR_INVALID_ARG, b);
      p = b;                              // left as it is
    }
    par[b] = p;
    low[b] = a.B;
    len[b] = a.len[b];
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += T)
    if (par[b] >= 0) atomicMin(&low[par[b]], b);
  __syncthreads();
  auto rows_of = [&](int b) { return par[b] >= 0 ? len[par[b]] : 0; };       // new length
  for (int b = tid; b < a.B; b += T) {
    const int p = par[b], n = rows_of(b);
    bool c = false;
    if (p >= 0 && (n & ((1 << a.shift) - 1)) != 0 && (par[p] == p ? p : low[p]) != b) {
      const int used = pg_pages_of(a, n);
      c = used > 0 && pg_valid(a, old_rows[(size_t)p * a.W + used - 1]);
    }
    copy[b] = c;
  }
  __syncthreads();
  // new rows, counts of the pages that come and go
  for (unsigned i = tid; i < cells; i += T) {
    const int b = (int)(i / (unsigned)a.W), c = (int)(i - (unsigned)b * a.W), p = par[b];
    if (p == b) continue;
    const int used = pg_pages_of(a, rows_of(b));
    const int old = old_rows[i], now = p >= 0 && c < used ? old_rows[(size_t)p * a.W + c] : -1;
    fresh[i] = now;
    if (pg_valid(a, old)) atomicSub(const_cast<int*>(refs) + old, 1);
    if (pg_valid(a, now) && !(copy[b] && c == used - 1)) atomicAdd(const_cast<int*>(refs) + now, 1);
  }
  if (!(near & 1)) __threadfence();
  __syncthreads();
  // copies in order of b, free pages in order of index
  const int per = (a.B + T - 1) / T, b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
  int from, to;
  int2 mine = make_int2(0, 0), sums;
  for (int b = b0; b < b1; ++b) mine.x += copy[b];
  pg_run(a, from, to);
  for (int p = from; p < to; ++p) mine.y += refs[p] == 0;
  const int2 before = pg_scan2(mine, sh, &sums);
  const int copies = sums.x;
  int at = before.x, rank = before.y;
  if (sums.y < copies) {
    if (!(near & 1))                      // put the counts back
      for (unsigned i = tid; i < cells; i += T) {
        const int b = (int)(i / (unsigned)a.W), col = (int)(i - (unsigned)b * a.W);
        if (par[b] == b) continue;
        const int old = old_rows[i], now = fresh[i];
        if (pg_valid(a, old)) atomicAdd(const_cast<int*>(refs) + old, 1);
        if (pg_valid(a, now) && !(copy[b] && col == pg_pages_of(a, rows_of(b)) - 1)) atomicSub(const_cast<int*>(refs) + now, 1);
      }
    if (tid == 0) { a.hdr[0] = 0; report_status(a.status, DL_ERR_CAPACITY, -1); }
    return;
  }
  for (int p = from; p < to && rank < copies; ++p)
    if (refs[p] == 0) mine_dst[rank++] = p;
  __syncthreads();
  for (int b = b0; b < b1; ++b)
    if (copy[b]) {
      const unsigned cell = (unsigned)b * a.W + pg_pages_of(a, rows_of(b)) - 1;
      const int d = mine_dst[at];
      a.src[at] = fresh[cell];
      a.dst[at++] = d;
      fresh[cell] = d;
      refs[d] = 1;
    }
  __syncthreads();
  for (unsigned i = tid; i < cells; i += T) {
    const int b = (int)(i / (unsigned)a.W);
    if (par[b] != b) a.table[i] = fresh[i];
  }
  if (near & 1)
    for (int p = tid; p < a.n_pages; p += T) a.refs[p] = refs[p];
  for (int b = tid; b < a.B; b += T)
    if (par[b] != b) a.len[b] = rows_of(b);
  if (tid == 0) a.hdr[0] = copies;
}

// Pages in use behind the first `live` ids move into the free ids below, both in index order.
__global__ void __launch_bounds__(kPgThreads)
pages_compact_kernel(const PgArgs a, int32_t* live_out) {
  __shared__ int2 sh[32], sh2[32];
  chained_go();
  chained_wait();
  int from, to;
  int2 c = make_int2(0, 0), sums;
  pg_run(a, from, to);
  for (int p = from; p < to; ++p) c.x += a.refs[p] != 0;
  pg_scan2(c, sh, &sums);
  const int live = sums.x;
  c = make_int2(0, 0);                    // pages to move, free pages below
  for (int p = from; p < to; ++p) {
    const bool used = a.refs[p] != 0;
    c.x += used && p >= live;
    c.y += !used && p < live;
  }
  const int2 at = pg_scan2(c, sh2, &sums);
  int m = at.x, h = at.y;
  const int moves = sums.x;               // == sums.y
  for (int p = from; p < to; ++p) {
    const bool used = a.refs[p] != 0;
    if (used && p >= live) a.src[m++] = p;
    if (!used && p < live) a.dst[h++] = p;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < moves; i += kPgThreads) {
    const int s = a.src[i], d = a.dst[i];
    a.map[s] = d;
    a.refs[d] = a.refs[s];
    a.refs[s] = 0;
  }
  if (threadIdx.x == 0) {
    a.hdr[0] = moves;
    a.hdr[1] = live;
    if (live_out) *live_out = live;
  }
}

// Copies hdr[0] pages of every pool; with remap, also gives the table's entries of moved pages their new numbers.
__global__ void __launch_bounds__(kPgCopyThreads)
pages_copy_kernel(const PgArgs a, const __grid_constant__ PgPools pools, int32_t n_pools, long long page_bytes, int32_t remap) {
  chained_go();
  chained_wait();
  const int n = __ldcg(a.hdr);
  if (remap) {
    const int live = __ldcg(a.hdr + 1);
    const long long cells = (long long)a.B * a.W;
    for (long long i = (long long)blockIdx.x * kPgCopyThreads + threadIdx.x; i < cells; i += (long long)gridDim.x * kPgCopyThreads) {
      const int p = a.table[i];
      if (p >= live && p < a.n_pages) a.table[i] = __ldcg(a.map + p);
    }
  }
  const int chunks = (int)((page_bytes + kPgChunk - 1) / kPgChunk);
  const long long all = (long long)n * chunks * n_pools;
  for (long long w = blockIdx.x; w < all; w += gridDim.x) {
    const int l = (int)(w / ((long long)n * chunks));
    const long long rest = w - (long long)l * n * chunks;
    const int i = (int)(rest / chunks), ch = (int)(rest - (long long)i * chunks);
    const long long off = (long long)ch * kPgChunk;
    const char* s = pools.p[l] + (long long)__ldcg(a.src + i) * page_bytes + off;
    char* d = pools.p[l] + (long long)__ldcg(a.dst + i) * page_bytes + off;
    const int units = (int)(min((long long)kPgChunk, page_bytes - off) >> 4);
    uint4 v[kPgChunk / 16 / kPgCopyThreads];
#pragma unroll
    for (int k = 0; k < kPgChunk / 16 / kPgCopyThreads; ++k) {
      const int u = threadIdx.x + k * kPgCopyThreads;
      if (u < units) v[k] = __ldcs(reinterpret_cast<const uint4*>(s) + u);
    }
#pragma unroll
    for (int k = 0; k < kPgChunk / 16 / kPgCopyThreads; ++k) {
      const int u = threadIdx.x + k * kPgCopyThreads;
      if (u < units) __stcs(reinterpret_cast<uint4*>(d) + u, v[k]);
    }
  }
}

// Scratch: 4 ints of counts, src and dst lists, new numbers of moved pages, new table rows.
int64_t pages_scratch_bytes(const dl_pages* p) {
  const int64_t list = std::max(p->B, p->n_pages);
  return 4 * (4 + 2 * list + p->n_pages + (int64_t)p->B * p->max_pages);
}

static PgArgs pg_args(const dl_ctx* ctx, const dl_pages* p, void* scratch) {
  PgArgs a = {};
  a.table = p->table; a.refs = p->refs; a.len = p->len;
  a.B = p->B; a.n_pages = p->n_pages; a.W = p->max_pages;
  a.shift = p->page_rows == 16 ? 4 : p->page_rows == 32 ? 5 : p->page_rows == 64 ? 6 : 7;
  a.status = ctx->ws.base ? ctx->ws.status : nullptr;
  if (scratch) {
    const int64_t list = std::max(p->B, p->n_pages);
    a.hdr = static_cast<int32_t*>(scratch);
    a.src = a.hdr + 4;
    a.dst = a.src + list;
    a.map = a.dst + list;
    a.fresh = a.map + p->n_pages;
  }
  return a;
}

static cudaError_t pg_copy(const dl_ctx* ctx, const PgArgs& a, int32_t n_pools, void* const* pools, int64_t page_bytes,
                           bool remap, cudaStream_t s) {
  for (int at = 0; at < n_pools || (at == 0 && remap); at += kPgPools) {
    PgPools pp = {};
    const int n = std::min(kPgPools, n_pools - at);
    for (int i = 0; i < n; ++i) pp.p[i] = static_cast<char*>(pools[at + i]);
    const cudaError_t e = launch_chained(pages_copy_kernel, dim3(ctx->sm_count * 8), dim3(kPgCopyThreads), 0, s, a, pp, n,
                                         (long long)page_bytes, (int32_t)(remap && at == 0));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_pages_reserve(const dl_ctx* ctx, const dl_pages* p, const int32_t* need, cudaStream_t s) {
  const size_t smem = (size_t)(2 * p->B + 1) * 4;
  return launch_chained(pages_reserve_kernel, dim3(1), dim3(kPgThreads), smem, s, pg_args(ctx, p, nullptr), need);
}

cudaError_t launch_pages_free(const dl_ctx* ctx, const dl_pages* p, const uint8_t* gone, cudaStream_t s) {
  return launch_chained(pages_free_kernel, dim3(p->B), dim3(128), 0, s, pg_args(ctx, p, nullptr), gone);
}

cudaError_t launch_pages_fork(const dl_ctx* ctx, const dl_pages* p, const int32_t* parent, int32_t n_pools,
                              void* const* pools, int64_t page_bytes, void* scratch, cudaStream_t s) {
  const PgArgs a = pg_args(ctx, p, scratch);
  // shared memory: five lists of B, and the counts and the rows where 160 KB hold them
  constexpr size_t kMost = 160 * 1024;
  size_t smem = (size_t)5 * p->B * 4;
  int near = 0;
  if (smem + (size_t)p->n_pages * 4 <= kMost) { near |= 1; smem += (size_t)p->n_pages * 4; }
  const size_t rows = 2 * (size_t)p->B * p->max_pages * 4;
  if (smem + rows <= kMost) { near |= 2; smem += rows; }
  cudaError_t e = cudaSuccess;
  // (asked for whatever this call takes: the 48 KB that a kernel has without asking also hold its static arrays)
  static int attr_set[64];
  if (!attr_set[ctx->device & 63]) {
    e = cudaFuncSetAttribute(pages_fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMost);
    if (e != cudaSuccess) return e;
    attr_set[ctx->device & 63] = 1;
  }
  e = launch_chained(pages_fork_kernel, dim3(1), dim3(kPgThreads), smem, s, a, parent, near);
  return e != cudaSuccess ? e : pg_copy(ctx, a, n_pools, pools, page_bytes, false, s);
}

cudaError_t launch_pages_compact(const dl_ctx* ctx, const dl_pages* p, int32_t n_pools, void* const* pools,
                                 int64_t page_bytes, int32_t* live, void* scratch, cudaStream_t s) {
  const PgArgs a = pg_args(ctx, p, scratch);
  const cudaError_t e = launch_chained(pages_compact_kernel, dim3(1), dim3(kPgThreads), 0, s, a, live);
  return e != cudaSuccess ? e : pg_copy(ctx, a, n_pools, pools, page_bytes, true, s);
}

}  // namespace dl
