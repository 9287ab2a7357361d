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

// Exclusive scan over the CTA's threads; *sum gets the total.  sh: 33 ints.
__device__ __forceinline__ int pg_scan(int v, int* sh, int* sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int run = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += x;
  }
  if (lane == 31) sh[warp] = run;
  __syncthreads();
  if (warp == 0) {
    int x = sh[lane], y = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int z = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) y += z;
    }
    sh[lane] = y - x;
    if (lane == 31) sh[32] = y;
  }
  __syncthreads();
  const int before = sh[warp] + run - v;
  *sum = sh[32];
  __syncthreads();
  return before;
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
pages_reserve_kernel(const PgArgs a, const int32_t* __restrict__ need) {
  extern __shared__ int sm[];
  int* have = sm;                         // [B] pages a sequence has
  int* first = sm + a.B;                  // [B + 1] pages handed out in front of it
  __shared__ int sh[33], too_long;
  if (threadIdx.x == 0) too_long = a.B;
  __syncthreads();
  const int per = (a.B + kPgThreads - 1) / kPgThreads, b0 = min(a.B, (int)threadIdx.x * per), b1 = min(a.B, b0 + per);
  int mine = 0;
  for (int b = b0; b < b1; ++b) {
    const int32_t* row = a.table + (size_t)b * a.W;
    int lo = 0, hi = a.W;                 // a row's pages come first: the first -1 by bisection
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (row[mid] >= 0) lo = mid + 1; else hi = mid;
    }
    have[b] = lo;
    const long long rows = (long long)max(a.len[b], 0) + max(need[b], 0);
    const long long want = (rows + (1 << a.shift) - 1) >> a.shift;
    if (want > a.W) atomicMin(&too_long, b);
    first[b] = mine;
    mine += (int)max(0LL, min(want, (long long)a.W) - lo);
  }
  int wanted;
  const int before = pg_scan(mine, sh, &wanted);
  for (int b = b0; b < b1; ++b) first[b] += before;
  if (threadIdx.x == 0) first[a.B] = wanted;
  int from, to, c = 0, free_pages;
  pg_run(a, from, to);
  for (int p = from; p < to; ++p) c += a.refs[p] == 0;
  int rank = pg_scan(c, sh, &free_pages);
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

__global__ void pages_free_kernel(const PgArgs a, const uint8_t* __restrict__ gone) {
  const int b = blockIdx.x;
  if (!gone[b]) return;
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
__global__ void __launch_bounds__(kPgThreads)
pages_fork_kernel(const PgArgs a, const int32_t* __restrict__ parent) {
  extern __shared__ int sm[];
  int* par = sm;                          // [B]
  int* low = sm + a.B;                    // [B] lowest child
  int* rows = sm + 2 * a.B;               // [B] new length
  int* copy = sm + 3 * a.B;               // [B] the last page is to be copied
  __shared__ int sh[33];
  const int T = kPgThreads, tid = threadIdx.x;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int b = tid; b < a.B; b += T) {
    int p = parent[b];
    if (p < -1 || p >= a.B) {
      report_status(a.status, DL_ERR_INVALID_ARG, b);
      p = b;                              // left as it is
    }
    par[b] = p;
    low[b] = a.B;
    rows[b] = p >= 0 ? a.len[p] : 0;
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += T)
    if (par[b] >= 0) atomicMin(&low[par[b]], b);
  __syncthreads();
  for (int b = tid; b < a.B; b += T) {
    const int p = par[b];
    bool c = false;
    if (p >= 0 && (rows[b] & ((1 << a.shift) - 1)) != 0 && (par[p] == p ? p : low[p]) != b) {
      const int used = pg_pages_of(a, rows[b]);
      c = used > 0 && pg_valid(a, a.table[(size_t)p * a.W + used - 1]);
    }
    copy[b] = c;
  }
  __syncthreads();
  // new rows into scratch, counts of the pages that come and go
  const long long cells = (long long)a.B * a.W;
  for (long long i = tid; i < cells; i += T) {
    const int b = (int)(i / a.W), c = (int)(i - (long long)b * a.W), p = par[b];
    if (p == b) continue;
    const int used = pg_pages_of(a, rows[b]);
    const int old = a.table[i], now = p >= 0 && c < used ? a.table[(size_t)p * a.W + c] : -1;
    a.fresh[i] = now;
    if (pg_valid(a, old)) atomicSub(a.refs + old, 1);
    if (pg_valid(a, now) && !(copy[b] && c == used - 1)) atomicAdd(a.refs + now, 1);
  }
  __threadfence();
  __syncthreads();
  // copies in order of b, free pages in order of index
  const int per = (a.B + T - 1) / T, b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
  int mine = 0, copies, free_pages, c = 0, from, to;
  for (int b = b0; b < b1; ++b) mine += copy[b];
  int at = pg_scan(mine, sh, &copies);
  pg_run(a, from, to);
  for (int p = from; p < to; ++p) c += __ldcg(a.refs + p) == 0;
  int rank = pg_scan(c, sh, &free_pages);
  if (free_pages < copies) {
    for (long long i = tid; i < cells; i += T) {
      const int b = (int)(i / a.W), col = (int)(i - (long long)b * a.W);
      if (par[b] == b) continue;
      const int old = a.table[i], now = a.fresh[i];
      if (pg_valid(a, old)) atomicAdd(a.refs + old, 1);
      if (pg_valid(a, now) && !(copy[b] && col == pg_pages_of(a, rows[b]) - 1)) atomicSub(a.refs + now, 1);
    }
    if (tid == 0) { a.hdr[0] = 0; report_status(a.status, DL_ERR_CAPACITY, -1); }
    return;
  }
  for (int p = from; p < to && rank < copies; ++p)
    if (__ldcg(a.refs + p) == 0) a.dst[rank++] = p;
  __syncthreads();
  for (int b = b0; b < b1; ++b)
    if (copy[b]) {
      const size_t cell = (size_t)b * a.W + pg_pages_of(a, rows[b]) - 1;
      const int d = a.dst[at];
      a.src[at++] = a.fresh[cell];
      a.fresh[cell] = d;
      a.refs[d] = 1;
    }
  __syncthreads();
  for (long long i = tid; i < cells; i += T) {
    const int b = (int)(i / a.W);
    if (par[b] != b) a.table[i] = a.fresh[i];
  }
  for (int b = tid; b < a.B; b += T)
    if (par[b] != b) a.len[b] = rows[b];
  if (tid == 0) a.hdr[0] = copies;
}

// Pages in use behind the first `live` ids move into the free ids below, both in index order.
__global__ void __launch_bounds__(kPgThreads)
pages_compact_kernel(const PgArgs a, int32_t* live_out) {
  __shared__ int sh[33];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int from, to, c = 0, live, moves, holes;
  pg_run(a, from, to);
  for (int p = from; p < to; ++p) c += a.refs[p] != 0;
  pg_scan(c, sh, &live);
  int movers = 0, free_below = 0;
  for (int p = from; p < to; ++p) {
    const bool used = a.refs[p] != 0;
    movers += used && p >= live;
    free_below += !used && p < live;
  }
  int m = pg_scan(movers, sh, &moves), h = pg_scan(free_below, sh, &holes);   // moves == holes
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
  asm volatile("griddepcontrol.wait;" ::: "memory");
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
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctx->sm_count * 8);
    cfg.blockDim = dim3(kPgCopyThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = at == 0 ? 1 : 0;    // the first copy follows the bookkeeping kernel
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, pages_copy_kernel, a, (const PgPools)pp, n, (long long)page_bytes,
                                             (int32_t)(remap && at == 0));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_pages_reserve(const dl_ctx* ctx, const dl_pages* p, const int32_t* need, cudaStream_t s) {
  const size_t smem = (size_t)(2 * p->B + 1) * 4;
  pages_reserve_kernel<<<1, kPgThreads, smem, s>>>(pg_args(ctx, p, nullptr), need);
  return cudaGetLastError();
}

cudaError_t launch_pages_free(const dl_ctx* ctx, const dl_pages* p, const uint8_t* gone, cudaStream_t s) {
  pages_free_kernel<<<p->B, 128, 0, s>>>(pg_args(ctx, p, nullptr), gone);
  return cudaGetLastError();
}

cudaError_t launch_pages_fork(const dl_ctx* ctx, const dl_pages* p, const int32_t* parent, int32_t n_pools,
                              void* const* pools, int64_t page_bytes, void* scratch, cudaStream_t s) {
  const PgArgs a = pg_args(ctx, p, scratch);
  const size_t smem = (size_t)4 * p->B * 4;
  pages_fork_kernel<<<1, kPgThreads, smem, s>>>(a, parent);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : pg_copy(ctx, a, n_pools, pools, page_bytes, false, s);
}

cudaError_t launch_pages_compact(const dl_ctx* ctx, const dl_pages* p, int32_t n_pools, void* const* pools,
                                 int64_t page_bytes, int32_t* live, void* scratch, cudaStream_t s) {
  const PgArgs a = pg_args(ctx, p, scratch);
  pages_compact_kernel<<<1, kPgThreads, 0, s>>>(a, live);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : pg_copy(ctx, a, n_pools, pools, page_bytes, true, s);
}

}  // namespace dl
