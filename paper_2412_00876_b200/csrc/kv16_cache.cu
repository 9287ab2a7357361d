// Rows into the paged 16-bit K/V cache: appended with the position rotation on the way, and kept or dropped once drafts are
// verified.  An extension, not in the paper: the append of Eq. 6 for rows that are not position-encoded yet.
//
//   plan   : (with a keep mask or a commit) per sequence, count the kept rows and list them in front of the others, check that
//            their pages are there, note the first destination row, advance the length: one CTA per sequence;
//   append : a CTA takes a few packed rows; cos and sin of those that are kept or asked for go to shared memory once and serve all
//            heads; then every thread moves 32 bytes at a time (both halves of 8 pairs), two such units in flight, q to q_out, k to
//            k_out and the cache, v to the cache;
//   commit : accepted rows move up; a thread stays at one 16-byte column of one pool, tensor and head and walks the rows in
//            order, so that no row is overwritten before it has been read;
//   tree   : ancestors' bits and depths of tree nodes.
//
// The append is bound by memory: 23 thousand rows of 32 + 2 x 8 heads 104.5 us, 5.8 TB/s moved; a batch of which a mask keeps a part
// (22 thousand rows of 32 + 32 heads, 8 thousand kept) 60 us with its plan of 6 us, and there the rows kept are far apart.  Between
// the first load and the last store lie the row's place, the angles and the rotation, so what counts is how many CTAs are at
// different points of that: (rows a CTA, units in flight, CTAs a multiprocessor), both batches in us: 16, 4, 4: 78.5 and 124;
// 8, 4, 4: 74, 116; 8, 2, 8: 77, 129; 12, 10, 8, 6, 5, 4, 3, 2 with 2, 6: 66, 64, 64.5, 62, 60, 60, 62, 67 and 117, 112, 110.5, 107,
// 107, 104.5, 107, 111; 4, 3, 5: 66, 114; 4, 1, 8: 58.5, 106.5; 4, 2, 7 (spills): 67, 119.  A fixed unit per thread: 64-72 and 117-137, a
// grid of resident CTAs that take rows in turn: 70-98 and 111-122.  Flags counted by every CTA instead of listed by the plan: 77, 120.
// Moving accepted rows takes 7 us for 32 sequences of four layers, launch and two dependent looks at the books included.
#include <algorithm>

#include "kv16.cuh"

namespace dl {

constexpr int kK16Threads = 256;
constexpr int kK16Rows = 4;              // most packed rows per CTA of the append
constexpr int kK16Batch = 2;             // units of 32 bytes a thread has in flight
constexpr int kK16Ctas = 6;              // CTAs of it a multiprocessor holds
constexpr int kK16PlanThreads = 1024;

// Whether rows [base, base + count) of sequence b have pages: a sequence's pages come first in its table row, so the last one
// tells.  (Every row's own page is looked at again where it is written.)
__device__ __forceinline__ bool k16_fits(const K16Pages& pg, int b, int base, int count) {
  return base >= 0 && (count == 0 || k16_page(pg, b, (long long)base + count - 1) >= 0);
}

// With a mask: order[starts[b] ..] gets the sequence's rows, the kept ones first, both kinds in their order.
__global__ void __launch_bounds__(kK16PlanThreads)
kv16_plan_kernel(const K16Pages pg, const int32_t* starts, const uint8_t* keep, int32_t total, int32_t commit,
                 int32_t* plan_base, int32_t* plan_count, int32_t* order) {
  static_assert(kK16PlanThreads == 32 * 32, "a lane per warp");
  __shared__ int sh[2][32];
  chained_go();
  chained_wait();
  const int b = blockIdx.x, base = __ldcg(pg.len + b), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int from = k16_start(starts, b, total), to = max(from, k16_start(starts, b + 1, total));
  int count = to - from;
  if (keep) {
    // four flags a thread, from a 4-byte boundary on; those of other rows are 0
    constexpr int kStep = 4 * kK16PlanThreads;
    const int first = from - (int)(reinterpret_cast<uintptr_t>(keep + from) & 3);
    auto flags = [&](int at) {
      uint32_t m = 0;
      if (at >= from && at + 4 <= to) {
        const uint32_t b = __vcmpne4(__ldcg(reinterpret_cast<const uint32_t*>(keep + at)), 0) & 0x01010101u;
        m = (b * 0x01020408u) >> 24;                               // the four bytes' lowest bits side by side
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at + i >= from && at + i < to && __ldcg(keep + at + i) != 0) m |= 1u << i;
      }
      return m;
    };
    const bool once = to - first <= kStep;                         // all flags at a time: their number comes with the places
    if (!once) {
      int c = 0;
      for (int at = first + 4 * (int)threadIdx.x; at < to; at += kStep) c += __popc(flags(at));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
      if (lane == 0) sh[0][warp] = c;
      __syncthreads();
      c = sh[0][lane];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
      count = c;
    }
    int kept = from, turn = 1;                                     // place of the next kept row
    for (int i0 = first; i0 < to; i0 += kStep, turn ^= 1) {
      const int at = i0 + 4 * (int)threadIdx.x;
      const uint32_t m = flags(at);
      const int n = __popc(m);
      int run = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += v;
      }
      if (lane == 31) sh[turn][warp] = run;
      __syncthreads();
      // every warp adds up the warps' totals for itself
      const int mine = sh[turn][lane];
      int all = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, all, o);
        if (lane >= o) all += v;
      }
      const int of_step = __shfl_sync(0xffffffffu, all, 31);
      if (once) count = of_step;
      int front = kept + run - n + __shfl_sync(0xffffffffu, all - mine, warp);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (at + i < from || at + i >= to) continue;
        const bool f = (m >> i) & 1;
        order[f ? front : from + count + (at + i - from) - (front - from)] = at + i;
        front += f;
      }
      kept += of_step;
    }
  }
  if (threadIdx.x == 0) {
    const bool ok = k16_fits(pg, b, base, count);
    plan_base[b] = base;
    plan_count[b] = ok ? count : -1 - count;
    if (ok && commit) pg.len[b] = base + count;
  }
}

struct K16Append {
  const __nv_bfloat16* q; const __nv_bfloat16* k; const __nv_bfloat16* v;
  __nv_bfloat16* q_out; __nv_bfloat16* k_out; __nv_bfloat16* pool;
  long long q_stride, kv_stride, q_out_stride, k_out_stride;
  const int32_t* pos; const double* freqs; const int32_t* starts;
  const int32_t* plan_base; const int32_t* plan_count;             // NULL: lengths as they are; count: -1 - it where pages lack
  const int32_t* order;                                            // NULL: nothing is dropped
  int32_t H, Hk, total, rows, rot, interleaved;
  uint32_t per_row, per_row_inv;                                   // units of a row, 2^32 / units rounded up
  float amplitude;
  DeviceStatus* status;
};

// Eight pairs: x = their first values, y = their second; cs = cos and sin of each, in order.
__device__ __forceinline__ void k16_turn(float (&x)[8], float (&y)[8], const float2* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 w = cs[i];
    const float a = x[i] * w.x - y[i] * w.y;
    y[i] = y[i] * w.x + x[i] * w.y;
    x[i] = a;
  }
}
__device__ __forceinline__ uint32_t k16_pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void k16_rotate(uint4& a, uint4& b, bool interleaved, const float2* cs) {
  float x[8], y[8];
  const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
  uint32_t ra[4], rb[4];
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = bf16lo(wa[i]); y[i] = bf16hi(wa[i]);
      x[4 + i] = bf16lo(wb[i]); y[4 + i] = bf16hi(wb[i]);
    }
    k16_turn(x, y, cs);
#pragma unroll
    for (int i = 0; i < 4; ++i) { ra[i] = k16_pack(x[i], y[i]); rb[i] = k16_pack(x[4 + i], y[4 + i]); }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16lo(wa[i]); x[2 * i + 1] = bf16hi(wa[i]);
      y[2 * i] = bf16lo(wb[i]); y[2 * i + 1] = bf16hi(wb[i]);
    }
    k16_turn(x, y, cs);
#pragma unroll
    for (int i = 0; i < 4; ++i) { ra[i] = k16_pack(x[2 * i], x[2 * i + 1]); rb[i] = k16_pack(y[2 * i], y[2 * i + 1]); }
  }
  a = make_uint4(ra[0], ra[1], ra[2], ra[3]);
  b = make_uint4(rb[0], rb[1], rb[2], rb[3]);
}

template <int D>
__global__ void __launch_bounds__(kK16Threads, kK16Ctas)
kv16_append_kernel(const K16Pages pg, const K16Append a) {
  extern __shared__ int seq_start[];
  __shared__ uint64_t step[D / 2];                                 // turns per position, 64 bits of the fraction
  __shared__ float2 cs[kK16Rows][D / 2];
  __shared__ int row_of[kK16Rows];                                 // rows that have something to do
  __shared__ long long row_at[kK16Rows];                           // K row of head 0 in the pool; -1: not cached
  __shared__ int n_rows;
  chained_go();
  chained_wait();
  const int t0 = blockIdx.x * a.rows, n = min(a.rows, a.total - t0), half = a.rot >> 1;
  if ((int)threadIdx.x < half) {
    double turns = __ldcg(a.freqs + threadIdx.x) * 0.15915494309189533577;
    turns -= floor(turns);
    step[threadIdx.x] = (uint64_t)__double2ull_rn(turns * 18446744073709551616.0);
  }
  if (a.pool) {
    for (int b = threadIdx.x; b <= pg.B; b += kK16Threads) seq_start[b] = k16_start(a.starts, b, a.total);
    __syncthreads();
  }
  if (threadIdx.x < 32) {
    const int t = threadIdx.x, x = t0 + t;                         // place in the order of rows
    const bool in = t < n;
    const int b = in && a.pool ? k16_sequence(seq_start, pg.B, x) : -1;
    int r = x;
    long long at = -1;
    if (b >= 0) {
      const int rank = x - seq_start[b], number = seq_start[b + 1] - seq_start[b];
      const int base = a.plan_base ? __ldcg(a.plan_base + b) : __ldcg(pg.len + b);
      const int planned = a.plan_count ? __ldcg(a.plan_count + b) : 0;
      if (a.order) r = min(max(__ldcg(a.order + x), 0), a.total - 1);
      const bool fits = a.plan_count ? planned >= 0 : k16_fits(pg, b, base, number);
      if (!fits && rank == 0 && blockIdx.y == 0) report_status(a.status, DL_ERR_CAPACITY, b);
      if (fits && rank < (a.order ? planned : number)) {
        const int page = k16_page(pg, b, (long long)base + rank);
        if (page >= 0) at = k16_row(pg, a.Hk, page, 0, 0, (long long)base + rank);
      }
    }
    const bool work = in && (at >= 0 || ((b >= 0 || a.pool == nullptr) && (a.q_out || a.k_out)));
    const unsigned w = __ballot_sync(0xffffffffu, work);
    if (work) {
      const int i = __popc(w & ((1u << t) - 1u));
      row_of[i] = r;
      row_at[i] = at;
    }
    if (t == 0) n_rows = __popc(w);
  }
  __syncthreads();
  const int n_work = n_rows;
  for (int i = threadIdx.x; i < n_work * half; i += kK16Threads) {
    const int w = i / half, f = i - w * half;
    // the angle as a fraction of a turn, 64 bits of it: products with positions wrap around by themselves
    const int64_t angle = (int64_t)((uint64_t)(int64_t)__ldcg(a.pos + row_of[w]) * step[f]);
    float s, c;
    sincospif((float)angle * 1.0842021724855044e-19f, &s, &c);     // half turns: 2^-63
    cs[w][f] = make_float2(c * a.amplitude, s * a.amplitude);
  }
  __syncthreads();
  // All units of all rows in one row of indices, kK16Batch of them per thread in flight (a thread writes what it has read alone, so
  // in-place outputs are safe).
  constexpr int C = D / 16;                                        // units of 32 bytes per head
  const int uq = a.q_out ? a.H * C : 0, uk = a.Hk * C;
  const int rot_units = a.rot >> 4, all = n_work * (int)a.per_row;
  const long long v_rows = (long long)a.Hk << pg.shift;            // rows from K to V of a page
  for (int i0 = (blockIdx.y * kK16Threads) * kK16Batch + threadIdx.x; i0 < all; i0 += gridDim.y * kK16Threads * kK16Batch) {
    uint4 w0[kK16Batch], w1[kK16Batch];
    int row[kK16Batch], part[kK16Batch], d0[kK16Batch], d1[kK16Batch], head[kK16Batch];
#pragma unroll
    for (int k = 0; k < kK16Batch; ++k) {
      const int i = i0 + k * kK16Threads;
      part[k] = -1;
      if (i >= all) continue;
      row[k] = (int)__umulhi((uint32_t)i, a.per_row_inv);
      const int u = i - row[k] * (int)a.per_row, p = u < uq ? 0 : u < uq + uk ? 1 : 2;
      const int x = u - (p == 0 ? 0 : p == 1 ? uq : uq + uk), c = x % C;
      head[k] = x / C;
      if (p > 0 && row_at[row[k]] < 0 && !(p == 1 && a.k_out)) continue;
      part[k] = p;
      const bool pairs = p < 2 && c < rot_units && !a.interleaved;  // halves apart
      d0[k] = pairs ? 8 * c : 16 * c;
      d1[k] = pairs ? 8 * c + half : 16 * c + 8;
      const long long r = row_of[row[k]];
      const __nv_bfloat16* src = (p == 0 ? a.q + r * a.q_stride : (p == 1 ? a.k : a.v) + r * a.kv_stride) + head[k] * D;
      w0[k] = *reinterpret_cast<const uint4*>(src + d0[k]);
      w1[k] = *reinterpret_cast<const uint4*>(src + d1[k]);
    }
#pragma unroll
    for (int k = 0; k < kK16Batch; ++k) {
      if (part[k] < 0) continue;
      const int c = (i0 + k * kK16Threads - row[k] * (int)a.per_row - (part[k] == 0 ? 0 : part[k] == 1 ? uq : uq + uk)) % C;
      if (part[k] < 2 && c < rot_units) k16_rotate(w0[k], w1[k], a.interleaved != 0, &cs[row[k]][8 * c]);
      const long long r = row_of[row[k]], at = row_at[row[k]];
      if (part[k] == 0 || (part[k] == 1 && a.k_out)) {
        __nv_bfloat16* o = (part[k] == 0 ? a.q_out + r * a.q_out_stride : a.k_out + r * a.k_out_stride) + head[k] * D;
        *reinterpret_cast<uint4*>(o + d0[k]) = w0[k];
        *reinterpret_cast<uint4*>(o + d1[k]) = w1[k];
      }
      if (part[k] > 0 && at >= 0) {
        const long long dst = (at + (part[k] == 2 ? v_rows : 0) + ((long long)head[k] << pg.shift)) * D;
        if (DL_IN_BOUNDS(a.status, KID_KV16, dst + D - 1, (((long long)pg.n_pages * 2 * a.Hk) << pg.shift) * D)) {
          *reinterpret_cast<uint4*>(a.pool + dst + d0[k]) = w0[k];
          *reinterpret_cast<uint4*>(a.pool + dst + d1[k]) = w1[k];
        }
      }
    }
  }
}

// ---- accepted rows ----------------------------------------------------------------------------------------------------
constexpr int kK16Pools = 64;            // pools per launch
struct K16Pools { char* p[kK16Pools]; };

// grid: (sequence, slices of the pools' 16-byte columns).  `ticket` (one per sequence, zero between launches; NULL: lengths stay): the
// last of a sequence's CTAs, all of which have read its length by then, advances it.
template <int D>
__global__ void __launch_bounds__(kK16Threads)
kv16_move_kernel(const K16Pages pg, const __grid_constant__ K16Pools pools, int32_t n_pools, int32_t Hk, const int32_t* starts,
                 const uint8_t* keep, int32_t total, int32_t* ticket, DeviceStatus* st) {
  __shared__ int sh[kK16Threads / 32], warp_sum[kK16Threads / 32];
  __shared__ long long src_row[kK16Threads], dst_row[kK16Threads];  // K row of head 0 in the pool; -1: no page
  chained_go();
  chained_wait();
  const int b = blockIdx.x, base = __ldcg(pg.len + b);
  const int from = k16_start(starts, b, total), to = max(from, k16_start(starts, b + 1, total));
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // the last kept row must have a page
  int last = -1;
  for (int i = from + threadIdx.x; i < to; i += kK16Threads)
    if (__ldcg(keep + i) != 0) last = i - from;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) last = max(last, __shfl_xor_sync(0xffffffffu, last, o));
  if (lane == 0) sh[warp] = last;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kK16Threads / 32; ++w) last = max(last, sh[w]);
  if (last < 0) return;
  if (!k16_fits(pg, b, base, last + 1)) {
    if (blockIdx.y == 0 && threadIdx.x == 0) report_status(st, DL_ERR_CAPACITY, b);
    return;
  }
  constexpr int C = D / 8;
  const int columns = n_pools * 2 * Hk * C;
  const long long v_off = (long long)Hk << pg.shift;               // rows from K to V of a page
  int rank0 = 0;                                                   // kept rows of earlier rounds
  for (int i0 = 0; i0 <= last; i0 += kK16Threads) {
    const int i = i0 + threadIdx.x;
    const bool f = i <= last && __ldcg(keep + from + i) != 0;
    const unsigned m = __ballot_sync(0xffffffffu, f);
    if (lane == 0) warp_sum[warp] = __popc(m);
    __syncthreads();
    int rank = __popc(m & ((1u << lane) - 1u)), count = 0;
#pragma unroll
    for (int w = 0; w < kK16Threads / 32; ++w) {
      if (w < warp) rank += warp_sum[w];
      count += warp_sum[w];
    }
    if (f) {
      const long long s = (long long)base + i, d = (long long)base + rank0 + rank;
      const int ps = k16_page(pg, b, s), pd = k16_page(pg, b, d);
      const bool there = ps >= 0 && pd >= 0 && s != d;
      src_row[rank] = there ? k16_row(pg, Hk, ps, 0, 0, s) : -1;
      dst_row[rank] = there ? k16_row(pg, Hk, pd, 0, 0, d) : -1;
    }
    __syncthreads();
    for (int u = blockIdx.y * kK16Threads + threadIdx.x; u < columns; u += gridDim.y * kK16Threads) {
      const int c = u % C, h = (u / C) % Hk, kv = (u / (C * Hk)) & 1, l = u / (2 * C * Hk);
      __nv_bfloat16* pool = reinterpret_cast<__nv_bfloat16*>(pools.p[l]) + (kv * v_off + ((long long)h << pg.shift)) * D + 8 * c;
      for (int j = 0; j < count; j += 4) {
        uint4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j + k < count && src_row[j + k] >= 0) w[k] = *reinterpret_cast<const uint4*>(pool + src_row[j + k] * D);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j + k < count && dst_row[j + k] >= 0 &&
              DL_IN_BOUNDS(st, KID_KV16, dst_row[j + k], ((long long)pg.n_pages * 2 * Hk) << pg.shift))
            *reinterpret_cast<uint4*>(pool + dst_row[j + k] * D) = w[k];
      }
    }
    rank0 += count;
    __syncthreads();
  }
  if (ticket && threadIdx.x == 0 && atomicAdd(ticket + b, 1) == (int)gridDim.y - 1) {
    ticket[b] = 0;
    pg.len[b] = base + rank0;
  }
}

// ---- trees ------------------------------------------------------------------------------------------------------------
// One CTA per sequence: parents in shared memory, a thread per node walks up; ancestors have lower numbers, so it passes the words
// of its mask once, from the last to the first.
__global__ void __launch_bounds__(kK16Threads)
tree_plan_kernel(const int32_t* parent, const int32_t* starts, const int32_t* pos0, int32_t total, int32_t words,
                 int32_t* mask, int32_t* pos, DeviceStatus* st) {
  extern __shared__ int up[];
  chained_go();
  chained_wait();
  const int b = blockIdx.x;
  const int from = k16_start(starts, b, total), to = max(from, k16_start(starts, b + 1, total));
  const int n = min(to - from, 32 * words);
  bool bad = to - from > n;
  for (int i = threadIdx.x; i < n; i += kK16Threads) {
    int p = i == 0 ? -1 : __ldcg(parent + from + i);
    if (p < -1 || p >= i) { bad = true; p = -1; }
    up[i] = p;
  }
  if (bad) report_status(st, DL_ERR_INVALID_ARG, b);
  __syncthreads();
  const int first = pos0 ? __ldcg(pos0 + b) : 0;
  for (int i = threadIdx.x; i < n; i += kK16Threads) {
    int32_t* row = mask + (size_t)(from + i) * words;
    uint32_t bits = 0;
    int depth = -1, w = words - 1;
    for (int j = i; j >= 0; j = up[j]) {
      ++depth;
      for (; w > (j >> 5); --w) { row[w] = (int32_t)bits; bits = 0; }
      bits |= 1u << (j & 31);
    }
    for (; w >= 0; --w) { row[w] = (int32_t)bits; bits = 0; }
    if (pos) pos[from + i] = (int32_t)((uint32_t)first + (uint32_t)depth);
  }
}

// ---- launchers --------------------------------------------------------------------------------------------------------
cudaError_t launch_kv16_append(const dl_ctx* ctx, const dl_pages* p, int32_t Hk, void* pool, const void* q, int64_t q_stride,
                               const void* k, const void* v, int64_t kv_stride, const int32_t* pos, const dl_rope* rope,
                               const int32_t* starts, const uint8_t* keep, int32_t total, void* q_out, int64_t q_out_stride,
                               void* k_out, int64_t k_out_stride, int32_t commit, cudaStream_t s) {
  const int D = ctx->desc.head_dim, H = ctx->desc.n_heads;
  const K16Pages pg = k16_pages(p);
  K16Append a = {};
  a.q = static_cast<const __nv_bfloat16*>(q); a.k = static_cast<const __nv_bfloat16*>(k); a.v = static_cast<const __nv_bfloat16*>(v);
  a.q_out = static_cast<__nv_bfloat16*>(q_out); a.k_out = static_cast<__nv_bfloat16*>(k_out); a.pool = static_cast<__nv_bfloat16*>(pool);
  a.q_stride = q_stride; a.kv_stride = kv_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
  a.pos = pos; a.starts = starts;
  a.H = H; a.Hk = Hk; a.total = total;
  a.amplitude = 1.f;
  if (rope) { a.freqs = rope->freqs; a.rot = rope->rot_dim; a.interleaved = rope->interleaved; a.amplitude = rope->amplitude; }
  a.status = ctx->ws.base ? ctx->ws.status : nullptr;
  if (pool && (keep || commit)) {
    a.plan_base = ctx->ws.plan_base;
    a.plan_count = ctx->ws.plan_count;
    int32_t* order = reinterpret_cast<int32_t*>(ctx->ws.kv4_partial);
    if (keep) a.order = order;
    const cudaError_t e = launch_chained(kv16_plan_kernel, dim3(pg.B), dim3(kK16PlanThreads), 0, s, pg, starts, keep, total, commit,
                                         ctx->ws.plan_base, ctx->ws.plan_count, order);
    if (e != cudaSuccess) return e;
  }
  const int units = ((q_out ? H : 0) + (pool ? 2 : 1) * Hk) * (D / 16);
  static_assert(kK16Rows <= 4, "units of a call's widest rows (2^15) would not be told apart: see the check of the arguments");
  a.per_row = (uint32_t)units;
  a.per_row_inv = (uint32_t)(((1ull << 32) + units - 1) / units);
  // Rows per CTA: as many as leave four CTAs a multiprocessor; fewer rows than that are shared by several CTAs (grid y).  With 32
  // heads and 32 of K/V, 1280, 1600, 2000 rows: 22.6, 24.8, 28.2 us; if two or one CTA a multiprocessor are left 24.9, 26.7, 29.0;
  // always four rows a CTA 24.9, 26.7, 29.0 (fewer rows wait for the host's call, 22 us with a plan of the tree, in every form).
  a.rows = std::min(kK16Rows, std::max(1, total / (4 * ctx->sm_count)));
  const int slices = a.rows > 1 ? 1 : std::min((units + kK16Threads - 1) / kK16Threads, std::max(1, 8 * ctx->sm_count / total));
  const dim3 grid((total + a.rows - 1) / a.rows, slices);
  const size_t smem = pool ? (size_t)(pg.B + 1) * 4 : 0;
  return D == 128 ? launch_chained(kv16_append_kernel<128>, grid, dim3(kK16Threads), smem, s, pg, a)
                  : launch_chained(kv16_append_kernel<64>, grid, dim3(kK16Threads), smem, s, pg, a);
}

cudaError_t launch_kv16_commit(const dl_ctx* ctx, const dl_pages* p, int32_t Hk, int32_t n_pools, void* const* pools,
                               const int32_t* starts, const uint8_t* keep, int32_t total, cudaStream_t s) {
  const K16Pages pg = k16_pages(p);
  DeviceStatus* st = ctx->ws.base ? ctx->ws.status : nullptr;
  const int D = ctx->desc.head_dim;
  for (int at = 0; at < n_pools || at == 0; at += kK16Pools) {
    K16Pools pp = {};
    const int n = std::min(kK16Pools, n_pools - at);
    for (int i = 0; i < n; ++i) pp.p[i] = static_cast<char*>(pools[at + i]);
    const int slices = (int)std::min<long long>(std::max(1LL, ((long long)n * 2 * Hk * (D / 8) + kK16Threads - 1) / kK16Threads), 4096);
    int32_t* ticket = at + kK16Pools >= n_pools ? ctx->ws.dec_ticket : nullptr;        // with the last pools
    const dim3 grid(pg.B, slices);
    const cudaError_t e = D == 128 ? launch_chained(kv16_move_kernel<128>, grid, dim3(kK16Threads), 0, s, pg, pp, n, Hk, starts, keep, total, ticket, st)
                                   : launch_chained(kv16_move_kernel<64>, grid, dim3(kK16Threads), 0, s, pg, pp, n, Hk, starts, keep, total, ticket, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_tree_plan(const dl_ctx* ctx, const int32_t* parent, const int32_t* starts, const int32_t* pos0, int32_t B,
                             int32_t total, int32_t words, int32_t* mask, int32_t* pos, cudaStream_t s) {
  const size_t smem = (size_t)std::min(32 * words, total) * 4;
  return launch_chained(tree_plan_kernel, dim3(B), dim3(kK16Threads), smem, s, parent, starts, pos0, total, words, mask, pos,
                        ctx->ws.base ? ctx->ws.status : nullptr);
}

}  // namespace dl
