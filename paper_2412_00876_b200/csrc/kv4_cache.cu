// Rows into and out of the paged 4-bit K/V cache (format: kv4.cuh).  An extension, not in the paper: the append of Eq. 6
// and the set builder of Eq. 5 / Eq. 11 (kept rows only, in order), with the rows held in 4 bits.
//
//   plan   : per sequence, count the kept rows, check that the pages for them are there, note the first destination
//            row and (optionally) advance the length: one CTA per sequence;
//   append : a CTA takes up to 32 packed source rows, ranks the kept ones and quantises them, 16 values per lane, 4
//            lanes per group; dropped rows are not read.  A thread stays at one place of the row (head, tensor, 16 dims)
//            and walks the kept rows; wide rows are shared by several CTAs (grid y);
//   read   : the same walk the other way, codes to bf16.
// Floor: HBM, a kept row costs 2 D bytes in and 9 D / 16 out per head and tensor.  What the kernels run into is issue: 200
// (append) and 150 (read) instructions per 16 values a lane, 69 and 57 % of the issue slots, so a row's place in its tile is
// worked out once per CTA, not per lane.  97 MB to 27 (23.7k rows of 8 heads) and back: 29.5 and 27.4 us, 4.2 and 4.5 TB/s.
// Measured and not better: two or four rows at a time, the next row's loads ahead, a product and a sum on fp32 pairs, the
// two rows that share V bytes in the halves of a warp or joined by one thread (0-8 % slower).
// With a mask every CTA of the append counts the flags in front of its rows, from its sequence's start: nothing at 700 rows, but
// it grows with the square of the length (one sequence of 8 heads, all rows kept, with a mask and without: 8k rows 24 and 21 us,
// 32k 58 and 38, 131k 189 and 123).
#include <algorithm>

#include "kv4.cuh"

namespace dl {

constexpr int kK4Threads = 256;
constexpr int kK4Rows = 32;              // most packed rows per CTA
constexpr int kK4CtasSm = 8;             // CTAs an SM holds, by threads

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

// All of them into shared memory (B + 1 ints): a search there costs no round trips to L2.
__device__ __forceinline__ void k4_load_starts(const int32_t* starts, int B, int total, int* st) {
  for (int b = threadIdx.x; b <= B; b += kK4Threads) st[b] = k4_start(starts, b, total);
  __syncthreads();
}

// The sequence that packed row r belongs to: the last b whose start is <= r (so empty sequences own nothing), or -1.
__device__ __forceinline__ int k4_sequence(const int* st, int B, int r) {
  int lo = -1, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (st[mid] <= r) lo = mid; else hi = mid - 1;
  }
  return (lo >= 0 && r < st[lo + 1]) ? lo : -1;
}

// A thread's place in a row of U units (16 values of one head and tensor each): unit `rem`, starting at the CTA's row
// `first` and going on by `step` rows; rem >= U: no place.
struct K4Place { int rem, first, step; };
__device__ __forceinline__ K4Place k4_place(int U) {
  K4Place p;
  if (U >= kK4Threads) {
    p.rem = blockIdx.y * kK4Threads + threadIdx.x;
    p.first = 0;
    p.step = 1;
  } else {
    p.step = kK4Threads / U;
    p.first = threadIdx.x / U;
    p.rem = p.first < p.step ? threadIdx.x - p.first * U : U;
  }
  return p;
}

// 32 bytes: in one access where the addresses are multiples of 32 (kWide), else in two (a selected batch appended and read:
// 94.7 against 100.6 us; half a sector at a time, a warp's access takes twice the passes)
template <bool kWide> __device__ __forceinline__ void k4_load32(const void* p, uint32_t (&r)[8]) {
  if (kWide) {
    asm("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p));
  } else {
    const uint4 x = __ldg(static_cast<const uint4*>(p)), y = __ldg(static_cast<const uint4*>(p) + 1);
    r[0] = x.x; r[1] = x.y; r[2] = x.z; r[3] = x.w; r[4] = y.x; r[5] = y.y; r[6] = y.z; r[7] = y.w;
  }
}
template <bool kWide> __device__ __forceinline__ void k4_store32(void* p, const uint32_t (&r)[8]) {
  if (kWide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 :: "l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(r[0], r[1], r[2], r[3]);
    static_cast<uint4*>(p)[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
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
  chained_go();                                                    // the append kernel may start
  const int b = blockIdx.x, base = len[b];
  const int from = k4_start(starts, b, total), to = max(from, k4_start(starts, b + 1, total));
  const int count = keep ? k4_count(keep, from, to, sh) : to - from;
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

// k, v: packed rows [total] of Hk * D values, `stride` values apart; `rows` of them per CTA.
template <int D, bool kWide>
__global__ void __launch_bounds__(kK4Threads, kK4CtasSm)
kv4_append_kernel(const PagesArg pg, uint8_t* __restrict__ pool, int32_t Hk, const __nv_bfloat16* __restrict__ k,
                  const __nv_bfloat16* __restrict__ v, long long stride, const int32_t* __restrict__ starts,
                  const uint8_t* __restrict__ keep, int32_t total, int32_t rows, const int32_t* plan_base,
                  const int32_t* plan_count, DeviceStatus* st) {
  extern __shared__ int seq_start[];
  __shared__ int sh[kK4Threads / 32];
  __shared__ long long row_src[kK4Rows], row_tile[kK4Rows];       // offset of a kept row's source, of its tile in head 0
  __shared__ Kv4Row row_at[2][kK4Rows];                           // its place in the tile, in K and in V
  __shared__ int n_kept;
  const int t0 = blockIdx.x * rows;
  k4_load_starts(starts, pg.B, total, seq_start);
  const int b0 = k4_sequence(seq_start, pg.B, t0);
  int before = 0;                                                  // kept rows of the first row's sequence in front of it
  if (b0 >= 0) before = keep ? k4_count(keep, seq_start[b0], t0, sh) : t0 - seq_start[b0];
  chained_wait();                                                  // the plan
  if (threadIdx.x < 32) {
    const int r = t0 + threadIdx.x;
    const int b = (int)threadIdx.x < rows && r < total ? k4_sequence(seq_start, pg.B, r) : -1;
    const bool f = b >= 0 && (keep == nullptr || keep[r] != 0);
    const unsigned m = __ballot_sync(0xffffffffu, f);
    int dst = -1, page = -1;
    if (f && __ldcg(plan_count + b) >= 0) {
      const int head = max(seq_start[b] - t0, 0);                 // first lane of this sequence
      dst = __ldcg(plan_base + b) + (b == b0 ? before : 0) + __popc(m & ((1u << threadIdx.x) - 1u) & ~((1u << head) - 1u));
      if ((dst >> (pg.tile_shift + 4)) < pg.max_pages)
        page = __ldg(pg.table + (size_t)b * pg.max_pages + (dst >> (pg.tile_shift + 4)));
      if ((unsigned)page >= (unsigned)pg.n_pages) dst = -1;       // the plan has checked this; never a wild store
    }
    const unsigned w = __ballot_sync(0xffffffffu, dst >= 0);
    if (dst >= 0) {
      const int i = __popc(w & ((1u << threadIdx.x) - 1u));
      row_src[i] = r * stride;
      row_tile[i] = (long long)kv4_tile_index(pg, page, Hk, 0, dst >> 4) * Kv4<D>::TILE;
      row_at[0][i] = kv4_row<D>(dst & 15, false);
      row_at[1][i] = kv4_row<D>(dst & 15, true);
    }
    if (threadIdx.x == 0) n_kept = __popc(w);
  }
  __syncthreads();
  constexpr int LR = D / 16;                                      // units per row of one head and tensor
  const int half = Hk * LR, U = 2 * half, n = n_kept;
  const K4Place at = k4_place(U);
  const bool on = at.rem < U;
  const bool is_v = at.rem >= half;
  const int l = on ? (is_v ? at.rem - half : at.rem) : 0, hk = l / LR, lr = l - hk * LR;
  const __nv_bfloat16* src = (is_v ? v : k) + l * 16;
  uint8_t* head = pool + ((long long)hk << pg.tile_shift) * Kv4<D>::TILE;
  const Kv4Row* places = row_at[is_v];
  for (int base = 0; base < n; base += at.step) {                 // the same trips for all lanes: they shuffle together
    // (rows behind the last kept one, and places behind the row's last, take another's values and store nothing)
    const int row = base + at.first;
    uint32_t raw[8];
    k4_load32<kWide>(src + row_src[min(row, n - 1)], raw);
    uint32_t word;
    const uint2 code = kv4_quantise16(raw, word);
    if (on && row < n) {
      uint8_t* tile = head + row_tile[row];
      if (DL_IN_BOUNDS(st, KID_KV4_APPEND, (tile - pool) / Kv4<D>::TILE, (long long)pg.n_pages * Hk << pg.tile_shift))
        kv4_store16(tile, places[row], lr, is_v, code, word);
    }
  }
}

// Rows row0[b], row0[b] + 1, ... of every sequence as bf16, packed by `starts`.  A row without a page reads as zero and is
// reported.
template <int D, bool kWide>
__global__ void __launch_bounds__(kK4Threads, kK4CtasSm)
kv4_read_kernel(const PagesArg pg, const uint8_t* __restrict__ pool, int32_t Hk, const int32_t* __restrict__ row0,
                const int32_t* __restrict__ starts, int32_t total, int32_t rows, __nv_bfloat16* __restrict__ k_out,
                __nv_bfloat16* __restrict__ v_out, DeviceStatus* st) {
  extern __shared__ int seq_start[];
  __shared__ long long row_tile[kK4Rows];                         // -1: no page, -2: a packed row of no sequence, left as it is
  __shared__ Kv4Row row_at[2][kK4Rows];
  const int t0 = blockIdx.x * rows;
  k4_load_starts(starts, pg.B, total, seq_start);
  if (threadIdx.x < 32) {
    const int r = t0 + threadIdx.x;
    const int b = (int)threadIdx.x < rows && r < total ? k4_sequence(seq_start, pg.B, r) : -1;
    long long tile = -2;
    int in = 0;
    if (b >= 0) {
      const long long pos = (long long)__ldg(row0 + b) + (r - seq_start[b]);
      tile = -1;
      if (pos >= 0 && (pos >> (pg.tile_shift + 4)) < pg.max_pages) {
        const int page = __ldg(pg.table + (size_t)b * pg.max_pages + (pos >> (pg.tile_shift + 4)));
        tile = kv4_tile_index(pg, page, Hk, 0, (int)(pos >> 4));
        in = (int)pos & 15;
      }
      if (tile < 0) report_status(st, DL_ERR_INVALID_ARG, b);
    }
    row_tile[threadIdx.x] = tile < 0 ? tile : tile * Kv4<D>::TILE;
    row_at[0][threadIdx.x] = kv4_row<D>(in, false);
    row_at[1][threadIdx.x] = kv4_row<D>(in, true);
  }
  __syncthreads();
  constexpr int LR = D / 16;
  const int half = Hk * LR, U = 2 * half, n = min(rows, total - t0);
  const K4Place at = k4_place(U);
  if (at.rem >= U) return;
  const bool is_v = at.rem >= half;
  const int l = is_v ? at.rem - half : at.rem, hk = l / LR, lr = l - hk * LR;
  const uint8_t* head = pool + ((long long)hk << pg.tile_shift) * Kv4<D>::TILE;
  const Kv4Row* places = row_at[is_v];
  __nv_bfloat16* out = (is_v ? v_out : k_out) + l * 16;
  const uint64_t magic = kv4_pack2(-8388608.f, -8388608.f);
  for (int row = at.first; row < n; row += at.step) {
    const long long at_tile = row_tile[row];
    if (at_tile == -2) continue;
    uint2 code = make_uint2(0u, 0u);
    uint32_t word = 0u;
    if (at_tile >= 0) {
      const Kv4Row place = places[row];
      code = kv4_load16(head + at_tile, place, lr, is_v);
      word = __ldg(reinterpret_cast<const uint32_t*>(head + at_tile + place.word + (lr & ~3)));
    }
    const float s = bf16lo(word), z = bf16hi(word);
    const uint64_t s2 = kv4_pack2(s, s), z2 = kv4_pack2(z, z);
    uint32_t p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // a code in the low byte of 2^23, less 2^23
      const uint32_t even = (e < 4 ? code.x : code.y) & 0x0F0F0F0Fu, odd = ((e < 4 ? code.x : code.y) >> 4) & 0x0F0F0F0Fu;
      const uint64_t v = kv4_add2(kv4_pack2(__uint_as_float(__byte_perm(even, 0x4B000000u, 0x7540 | (e & 3))),
                                            __uint_as_float(__byte_perm(odd, 0x4B000000u, 0x7540 | (e & 3)))), magic);
      const uint64_t y = kv4_fma2(v, s2, z2);
      const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float((uint32_t)y), __uint_as_float((uint32_t)(y >> 32)));
      p[e] = *reinterpret_cast<const uint32_t*>(&b);
    }
    const long long to = (long long)(t0 + row) * (half * 16);
    if (DL_IN_BOUNDS(st, KID_KV4_READ, to + l * 16 + 15, 16LL * total * half))
      k4_store32<kWide>(out + to, p);
  }
}

// Packed rows per CTA (at most kK4Rows) and the grid: as many CTAs as the GPU holds `waves` times, or a whole multiple.
// Rows that all count make even CTAs, so that one full wave is best (23.7k rows of 8 heads, append or read: 1, 2, 3, 4
// waves 33, 33.7, 35.5, 37 us); with a mask the kept rows are spread unevenly and four are (a third kept of 21.9k rows of 32
// heads, appended and read: 3, 4, 5, 6 waves 92.7, 91.6, 91.5, 91.9 us; 2 waves about 95).
static dim3 k4_grid(const dl_ctx* ctx, int total, int Hk, int waves, int* rows) {
  const int U = 2 * Hk * ctx->desc.head_dim / 16, slabs = (U + kK4Threads - 1) / kK4Threads;
  do {
    const long long ctas = std::max(1LL, (long long)waves++ * kK4CtasSm * ctx->sm_count / slabs);
    *rows = (int)((total + ctas - 1) / ctas);
  } while (*rows > kK4Rows);
  return dim3((total + *rows - 1) / *rows, slabs);
}

cudaError_t launch_kv4_append(const dl_ctx* ctx, const dl_pages* p, int32_t Hk, void* pool, const void* k, const void* v,
                              int64_t stride, const int32_t* starts, const uint8_t* keep, int32_t total, int32_t commit,
                              cudaStream_t s) {
  const PagesArg pg = pages_arg(p);
  kv4_plan_kernel<<<p->B, kK4Threads, 0, s>>>(pg, p->len, starts, keep, total, commit, ctx->ws.plan_base,
                                               ctx->ws.plan_count, ctx->ws.status);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || total == 0) return e;
  int rows;
  const dim3 grid = k4_grid(ctx, total, Hk, keep ? 4 : 1, &rows);
  const bool wide = ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | (uintptr_t)stride * 2) & 31u) == 0;
  auto kernel = ctx->desc.head_dim == 128 ? (wide ? kv4_append_kernel<128, true> : kv4_append_kernel<128, false>)
                                          : (wide ? kv4_append_kernel<64, true> : kv4_append_kernel<64, false>);
  return launch_chained(kernel, grid, dim3(kK4Threads),
                        (size_t)(p->B + 1) * sizeof(int), s, pg, static_cast<uint8_t*>(pool), Hk,
                        static_cast<const __nv_bfloat16*>(k), static_cast<const __nv_bfloat16*>(v), stride, starts, keep,
                        total, rows, ctx->ws.plan_base, ctx->ws.plan_count, ctx->ws.status);
}

cudaError_t launch_kv4_read(const dl_ctx* ctx, const dl_pages* p, int32_t Hk, const void* pool, const int32_t* row0,
                            const int32_t* starts, int32_t total, void* k_out, void* v_out, cudaStream_t s) {
  if (total == 0) return cudaSuccess;
  int rows;
  const dim3 grid = k4_grid(ctx, total, Hk, 1, &rows);
  const bool wide = ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 31u) == 0;
  auto kernel = ctx->desc.head_dim == 128 ? (wide ? kv4_read_kernel<128, true> : kv4_read_kernel<128, false>)
                                          : (wide ? kv4_read_kernel<64, true> : kv4_read_kernel<64, false>);
  kernel<<<grid, kK4Threads, (size_t)(p->B + 1) * sizeof(int), s>>>(pages_arg(p), static_cast<const uint8_t*>(pool), Hk, row0, starts, total, rows,
                                     static_cast<__nv_bfloat16*>(k_out), static_cast<__nv_bfloat16*>(v_out),
                                     ctx->ws.status);
  return cudaGetLastError();
}

}  // namespace dl
