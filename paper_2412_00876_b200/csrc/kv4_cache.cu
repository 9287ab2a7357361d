// Rows into and out of the paged 4-bit K/V cache (format: kv4.cuh).  An extension, not in the paper: the append of Eq. 6
// and the set builder of Eq. 5 / Eq. 11 (kept rows only, in order), with the rows held in 4 bits.
//
//   plan   : per sequence, count the kept rows, check that the pages for them are there, note the first destination
//            row and (optionally) advance the length: one CTA per sequence;
//   append : a CTA takes 32 packed source rows, ranks the kept ones and quantises them, 8 values per lane, 8 lanes per
//            group; dropped rows are not read;
//   read   : the same walk the other way, codes to bf16.
// Both are bound by HBM: a kept row costs 2 D bytes in and 9 D / 16 out per head and tensor.
#include <algorithm>

#include "kv4.cuh"

namespace dl {

constexpr int kK4Threads = 256;
constexpr int kK4Rows = 32;              // packed rows per CTA

__device__ __forceinline__ int k4_block_sum(int v, int* sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0) sh[warp] = v;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int w = 0; w < kK4Threads / 32; ++w) t += sh[w];
  __syncthreads();
  return t;
}

// Start of sequence b among `total` packed rows; a start outside them is brought back inside, so that no list of starts
// leads out of a buffer.
__device__ __forceinline__ int k4_start(const int32_t* starts, int b, int total) { return min(max(__ldg(starts + b), 0), total); }

// The sequence that packed row r belongs to: the last b whose start is <= r (so empty sequences own nothing), or -1.
__device__ __forceinline__ int k4_sequence(const int32_t* starts, int B, int total, int r) {
  int lo = -1, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (k4_start(starts, mid, total) <= r) lo = mid; else hi = mid - 1;
  }
  return (lo >= 0 && r < k4_start(starts, lo + 1, total)) ? lo : -1;
}

// kept rows among packed rows [from, to), counted by the whole CTA
__device__ __forceinline__ int k4_count(const uint8_t* keep, int from, int to, int* sh) {
  int c = 0;
  for (int i = from + threadIdx.x; i < to; i += kK4Threads) c += keep[i] != 0;
  return k4_block_sum(c, sh);
}

__global__ void __launch_bounds__(kK4Threads)
kv4_plan_kernel(const PagesArg pg, int32_t* len, const int32_t* __restrict__ starts, const uint8_t* __restrict__ keep,
                int32_t total, int32_t commit, int32_t* plan_base, int32_t* plan_count, DeviceStatus* st) {
  __shared__ int sh[kK4Threads / 32];
  const int b = blockIdx.x;
  const int from = k4_start(starts, b, total), to = max(from, k4_start(starts, b + 1, total));
  const int count = keep ? k4_count(keep, from, to, sh) : to - from;
  const int base = len[b];
  const long long rows = (long long)pg.max_pages * (kKv4Rows << pg.tile_shift);
  bool ok = base >= 0 && (long long)base + count <= rows;
  if (ok && count > 0) {
    const int shift = pg.tile_shift + 4;
    int bad = 0;
    for (int i = (base >> shift) + threadIdx.x; i <= (base + count - 1) >> shift; i += kK4Threads)
      bad += (unsigned)pg.table[(size_t)b * pg.max_pages + i] >= (unsigned)pg.n_pages;
    ok = k4_block_sum(bad, sh) == 0;
  }
  if (threadIdx.x == 0) {
    plan_base[b] = base;
    plan_count[b] = ok ? count : -1;
    if (!ok) report_status(st, DL_ERR_CAPACITY, b);
    else if (commit) len[b] = base + count;
  }
}

// k, v: packed rows [total] of Hk * D values, `stride` values apart.
template <int D>
__global__ void __launch_bounds__(kK4Threads)
kv4_append_kernel(const PagesArg pg, uint8_t* __restrict__ pool, int32_t Hk, const __nv_bfloat16* __restrict__ k,
                  const __nv_bfloat16* __restrict__ v, long long stride, const int32_t* __restrict__ starts,
                  const uint8_t* __restrict__ keep, int32_t total, const int32_t* __restrict__ plan_base,
                  const int32_t* __restrict__ plan_count, DeviceStatus* st) {
  __shared__ int sh[kK4Threads / 32];
  __shared__ int row_src[kK4Rows], row_dst[kK4Rows], row_page[kK4Rows], n_kept;
  const int t0 = blockIdx.x * kK4Rows;
  const int b0 = k4_sequence(starts, pg.B, total, t0);
  int before = 0;                                                  // kept rows of the first row's sequence in front of it
  if (b0 >= 0) {
    const int from = k4_start(starts, b0, total);
    before = keep ? k4_count(keep, from, t0, sh) : t0 - from;
  }
  if (threadIdx.x < 32) {
    const int r = t0 + threadIdx.x;
    const int b = r < total ? k4_sequence(starts, pg.B, total, r) : -1;
    const bool f = b >= 0 && (keep == nullptr || keep[r] != 0);
    const unsigned m = __ballot_sync(0xffffffffu, f);
    int dst = -1, page = -1;
    if (f && plan_count[b] >= 0) {
      const int head = max(k4_start(starts, b, total) - t0, 0);   // first lane of this sequence
      dst = plan_base[b] + (b == b0 ? before : 0) + __popc(m & ((1u << threadIdx.x) - 1u) & ~((1u << head) - 1u));
      if ((dst >> (pg.tile_shift + 4)) < pg.max_pages)
        page = __ldg(pg.table + (size_t)b * pg.max_pages + (dst >> (pg.tile_shift + 4)));
      if ((unsigned)page >= (unsigned)pg.n_pages) dst = -1;       // the plan has checked this; never a wild store
    }
    const unsigned w = __ballot_sync(0xffffffffu, dst >= 0);
    if (dst >= 0) {
      const int i = __popc(w & ((1u << threadIdx.x) - 1u));
      row_src[i] = r; row_dst[i] = dst; row_page[i] = page;
    }
    if (threadIdx.x == 0) n_kept = __popc(w);
  }
  __syncthreads();
  constexpr int LR = D / 8;                                       // lanes per row of one head and tensor
  const int half = Hk * LR, U = 2 * half, n = n_kept * U;
  const int n_up = (n + 31) & ~31;                                // whole warps stay together for the shuffles
  for (int i = blockIdx.y * kK4Threads + threadIdx.x; i < n_up; i += gridDim.y * kK4Threads) {
    const bool on = i < n;
    const int j = on ? i : n - 1;
    const int row = j / U, rem = j - row * U;
    const bool is_v = rem >= half;
    const int l = is_v ? rem - half : rem;
    const uint4 raw = __ldg(reinterpret_cast<const uint4*>((is_v ? v : k) + row_src[row] * stride + (long long)l * 8));
    uint32_t word;
    const uint32_t code = kv4_quantise8(raw, word);
    const int hk = l / LR, R = row_dst[row];
    const long long tile = kv4_tile_index(pg, row_page[row], Hk, hk, R >> 4);
    if (on && DL_IN_BOUNDS(st, KID_KV4_APPEND, tile, (long long)pg.n_pages * Hk << pg.tile_shift))
      kv4_store8<D>(pool + tile * Kv4<D>::TILE, R & 15, l - hk * LR, is_v, code, word);
  }
}

// Rows row0[b], row0[b] + 1, ... of every sequence as bf16, packed by `starts`.  A row without a page reads as zero and is
// reported.
template <int D>
__global__ void __launch_bounds__(kK4Threads)
kv4_read_kernel(const PagesArg pg, const uint8_t* __restrict__ pool, int32_t Hk, const int32_t* __restrict__ row0,
                const int32_t* __restrict__ starts, int32_t total, __nv_bfloat16* __restrict__ k_out,
                __nv_bfloat16* __restrict__ v_out, DeviceStatus* st) {
  __shared__ int row_pos[kK4Rows], row_page[kK4Rows];
  const int t0 = blockIdx.x * kK4Rows;
  if (threadIdx.x < 32) {
    const int r = t0 + threadIdx.x;
    const int b = r < total ? k4_sequence(starts, pg.B, total, r) : -1;
    int pos = -1, page = -1;                                      // -1: a packed row of no sequence, left as it is
    if (b >= 0) {
      const long long at = (long long)__ldg(row0 + b) + (r - k4_start(starts, b, total));
      pos = 0;
      if (at >= 0 && (at >> (pg.tile_shift + 4)) < pg.max_pages) {
        pos = (int)at;
        page = __ldg(pg.table + (size_t)b * pg.max_pages + (pos >> (pg.tile_shift + 4)));
      }
      if ((unsigned)page >= (unsigned)pg.n_pages) {
        page = -1;
        report_status(st, DL_ERR_INVALID_ARG, b);
      }
    }
    row_pos[threadIdx.x] = pos;
    row_page[threadIdx.x] = page;
  }
  __syncthreads();
  constexpr int LR = D / 8;
  const int half = Hk * LR, U = 2 * half, n = min(kK4Rows, total - t0) * U;
  for (int i = blockIdx.y * kK4Threads + threadIdx.x; i < n; i += gridDim.y * kK4Threads) {
    const int row = i / U, rem = i - row * U;
    const bool is_v = rem >= half;
    const int l = is_v ? rem - half : rem;
    const int R = row_pos[row];
    if (R < 0) continue;
    const int hk = l / LR, lr = l - hk * LR, g = lr >> 3;
    uint4 o = make_uint4(0u, 0u, 0u, 0u);
    if (row_page[row] >= 0) {
      const uint8_t* tile = pool + (long long)kv4_tile_index(pg, row_page[row], Hk, hk, R >> 4) * Kv4<D>::TILE;
      const uint32_t c = __ldg(reinterpret_cast<const uint32_t*>(tile + (is_v ? Kv4<D>::V : 0) +
                                                                 kv4_group_off<D>(R & 15, g) + 4 * (lr & 7)));
      const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(tile + (is_v ? Kv4<D>::VM : Kv4<D>::KM) +
                                                                 ((R & 15) * Kv4<D>::NG + g) * 4));
      const float s = bf16lo(w), z = bf16hi(w);
      uint32_t p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x0 = fmaf((float)((c >> (8 * e)) & 15u), s, z), x1 = fmaf((float)((c >> (8 * e + 4)) & 15u), s, z);
        p[e] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x0)) |
               ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x1)) << 16);
      }
      o = make_uint4(p[0], p[1], p[2], p[3]);
    }
    const long long at = (long long)(t0 + row) * half + l;
    if (DL_IN_BOUNDS(st, KID_KV4_READ, at, (long long)total * half))
      reinterpret_cast<uint4*>(is_v ? v_out : k_out)[at] = o;
  }
}

// CTAs along y: the units of a row tile are shared by several CTAs where the rows alone would not fill the GPU
static int k4_split(const dl_ctx* ctx, int tiles, int Hk) {
  const int most = std::max(1, kK4Rows * 2 * Hk * ctx->desc.head_dim / 8 / kK4Threads);
  return std::max(1, std::min(most, 8 * ctx->sm_count / std::max(tiles, 1)));
}

cudaError_t launch_kv4_append(const dl_ctx* ctx, const dl_pages* p, int32_t Hk, void* pool, const void* k, const void* v,
                              int64_t stride, const int32_t* starts, const uint8_t* keep, int32_t total, int32_t commit,
                              cudaStream_t s) {
  const PagesArg pg = pages_arg(p);
  kv4_plan_kernel<<<p->B, kK4Threads, 0, s>>>(pg, p->len, starts, keep, total, commit, ctx->ws.plan_base,
                                               ctx->ws.plan_count, ctx->ws.status);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || total == 0) return e;
  const int tiles = (total + kK4Rows - 1) / kK4Rows;
  const dim3 grid(tiles, k4_split(ctx, tiles, Hk));
  auto kernel = ctx->desc.head_dim == 128 ? kv4_append_kernel<128> : kv4_append_kernel<64>;
  kernel<<<grid, kK4Threads, 0, s>>>(pg, static_cast<uint8_t*>(pool), Hk, static_cast<const __nv_bfloat16*>(k),
                                     static_cast<const __nv_bfloat16*>(v), stride, starts, keep, total,
                                     ctx->ws.plan_base, ctx->ws.plan_count, ctx->ws.status);
  return cudaGetLastError();
}

cudaError_t launch_kv4_read(const dl_ctx* ctx, const dl_pages* p, int32_t Hk, const void* pool, const int32_t* row0,
                            const int32_t* starts, int32_t total, void* k_out, void* v_out, cudaStream_t s) {
  if (total == 0) return cudaSuccess;
  const int tiles = (total + kK4Rows - 1) / kK4Rows;
  const dim3 grid(tiles, k4_split(ctx, tiles, Hk));
  auto kernel = ctx->desc.head_dim == 128 ? kv4_read_kernel<128> : kv4_read_kernel<64>;
  kernel<<<grid, kK4Threads, 0, s>>>(pages_arg(p), static_cast<const uint8_t*>(pool), Hk, row0, starts, total,
                                     static_cast<__nv_bfloat16*>(k_out), static_cast<__nv_bfloat16*>(v_out),
                                     ctx->ws.status);
  return cudaGetLastError();
}

}  // namespace dl
