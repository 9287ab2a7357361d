// Attention over a paged cache in 16 bits for up to 64 rows an item (nodes times query heads of a K/V head): small trees of drafted
// tokens, single tokens.  An extension, not in the paper.  bf16, head_dim 64 or 128.
//
// With so few rows the matrix unit is used the other way round: keys across its 128 rows, the item's N rows (16, 32 or 64) across
// the columns.
//   S^T [128 keys][N] = K Q^T;   P^T = 2^(S^T scale - m), one key per thread;   O^T [D dims][N] += V^T P^T
// K and V are read from shared memory as they come (V^T is V with the roles of its indices exchanged), P^T goes through shared
// memory as 64-byte rows of keys.  So a tile costs a thread N / 2 exponentials instead of 128, all eight warps have work however few
// the rows are, the masked form of the pass is the same code with N selects in front, S^T and O^T take so few columns of tensor
// memory that both are kept twice: K Q^T of the next tile, across the ends of items, too, runs beside the exponentials.
// What a row needs across keys is across threads here: its maximum is looked for in a share's first tile only (and again if a
// score passes it by far: the threads vote), its sum is added up per thread and joined at the share's end.  P^T is rounded to bf16
// once, as 16-bit matrix products take it (at most 2^-8 of a weight); sums are of the unrounded weights, in fp32.
//   warps 0-7 : exponentials and epilogue; thread = key of the tile (lane of tensor memory), later = dim of the output; warps 0-3
//               the first half of the rows, 4-7 the second: rows have nothing to do with one another
//   warp 8    : the producer: Q tiles, then K and V tiles through one ring, K a tile ahead
//   warp 9    : issues the MMAs
//   warp 10   : allocates tensor memory (256 columns: S^T, S^T, O^T, O^T)
// Every wait is bounded (pipeline.cuh); an abort leaves DL_ERR_TIMEOUT in the status word.
//
// Bound by memory where there is much of it: 48 single tokens over 500 to 9000 rows, 8 K/V heads, 137 us (6.1 TB/s in all, 7 while it
// streams).  32 trees of 20-26 nodes, 32 heads of their own, over 272 to 1296 rows: 82 us for 396 MB; what comes on top of the
// 61 us of copying is fixed: 6 us until the first tiles are there, the uneven end, the joining of parts (6 us cold).
// N = 16 and 32 beside 64: a tile costs N exponentials and N columns of P^T whatever the rows are.  The trees take 83 us with N = 32
// and 118 with 64; trees of 5-16 nodes 79 with 16, 80.5 with 32, 107 with 64; the single tokens 138, 139, 144.5.
// Up to 64 rows: from 33 on this and attn_tree_tc.cu are even over much memory (32 trees of 33-64 nodes 121 and 118 us, 32 of 5-8 nodes
// with 8 heads 88 both, 4 of those over 60-131 thousand rows 130 and 126), and where a few items share all CTAs this is
// faster (2 trees of 16 nodes over 4000 rows 17.2 and 19.5, 32 tokens with 64 heads a group 32 and 35).
// The trees with rows on M, one lane and two CTAs a multiprocessor: 101 us instead of 82.
// Four warps of exponentials instead of eight 110 (90 then), the sums of an item's end behind the next one's first tile
// 89 (83 then), the next item's page numbers requested early: no change.
#include <algorithm>

#include "attn_prefill_softmax.cuh"
#include "attn_tree.cuh"

namespace dl {

constexpr int kRwProducer = 8, kRwIssuer = 9, kRwAlloc = 10, kRwCheck = 11;
// A thread's sum of exponentials above which the maxima are looked for again: far enough that it is rare; P in bf16 and sums in
// fp32 keep their relative accuracy at that size as at any other.
constexpr float kRwFar = 1048576.f;

template <int D, int N> struct Rw {
  static constexpr int HALF = 128 * 128;               // 128 rows of 64 dims
  static constexpr int TILE = (D / 64) * HALF;         // one operand tile
  static constexpr int SLOTS = D == 128 ? 6 : 12;
  static constexpr int P = SLOTS * TILE;               // P^T: blocks of 128 keys x 32 rows (behind the ring: with 64 dims the MMAs read
                                                       // a second block of dims behind V, which goes nowhere)
  static constexpr int P_ROW = N == 16 ? 32 : 64;      // bytes of a key's row of a block, which is also the width of the swizzle
  static constexpr int P_BLOCK = 128 * 64;
  static constexpr int P_BUFS = N <= 32 ? 2 : 1;
  static constexpr int Q = P + 2 * P_BLOCK;
  static constexpr int Q_HALF = 64 * 128;              // 64 rows of 64 dims
  static constexpr int Q_PLACES = D == 64 || N <= 32 ? 2 : 1;
  static constexpr int Q_STEP = D == 64 ? Q_HALF : Q_HALF / 2;   // from one place to the next
  static constexpr int RED = Q + 2 * Q_HALF;           // [4][64] of the warps, [64] maxima, [64] sums, [2][64][2] mask words
  static constexpr int BAR = RED + 1024 + 256 + 256 + 1024;
  static constexpr int SMEM = BAR + 512;
};

// Shared-memory matrix descriptor of an MN-major bf16 tile of rows of 32 elements along MN (64 bytes; or 16, 32 bytes), one row per k,
// stored with the swizzle of that width: 8-k groups follow one another, the next elements along MN start `mn_block_bytes` further on.
template <int kRow> __device__ __forceinline__ uint64_t rw_desc_mn(uint32_t addr, uint32_t mn_block_bytes) {
  static_assert(kRow == 32 || kRow == 64, "width of the swizzle");
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((mn_block_bytes >> 4) & 0x3FFF) << 16;
  d |= (uint64_t)(8 * kRow >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)(kRow == 64 ? 4 : 6) << 61;
  return d;
}

__device__ __forceinline__ void rw_tmem_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void rw_tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               :: "r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
template <int W> __device__ __forceinline__ void rw_tmem_ld(uint32_t addr, uint32_t* r) {
  if (W == 8) rw_tmem_ld8(addr, r);
  else if (W == 16) tmem_ld16(addr, r);
  else tmem_ld32(addr, r);
}
template <int W> __device__ __forceinline__ void rw_tmem_st(uint32_t addr, const uint32_t* r) {
  if (W == 8) rw_tmem_st8(addr, r);
  else if (W == 16) tmem_st16(addr, r);
  else tmem_st32(addr, r);
}
// one lane of the (whole) warp, always the same one
__device__ __forceinline__ bool rw_elect() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// the four warps that work on one half of the rows
__device__ __forceinline__ void rw_sync(int half) { asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory"); }
__device__ __forceinline__ bool rw_any(int half, bool v) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((uint32_t)v), "r"(1 + half) : "memory");
  return r != 0;
}
__device__ __forceinline__ float rw_warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// Sums of W values over the warp's lanes: lane i returns that of value i % W.
template <int W> __device__ __forceinline__ float rw_column_sums(float (&v)[W], int lane) {
#pragma unroll
  for (int o = 16; o >= W; o >>= 1)
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) {
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float keep = up ? v[o + i] : v[i], give = up ? v[i] : v[o + i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  return v[0];
}

template <int D, int N>
__global__ void __launch_bounds__(kTrRowsThreads, 1)
attn_tree_rows_kernel(const __grid_constant__ TrMaps maps, const K16Pages pg, const TrArgs a) {
  using S = Rw<D, N>;
  constexpr int F = kTrRows;
  extern __shared__ __align__(1024) char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (smem_u32(smem) & 1023u) {                        // the swizzled tiles need 1024-byte alignment
    if (tid == 0) report_status(a.status, DL_ERR_ALIGNMENT, -1);
    chained_wait();
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::BAR);
  auto kv_full = [&](int i) { return smem_u32(bars + i); };
  auto kv_empty = [&](int i) { return smem_u32(bars + S::SLOTS + i); };
  enum { Q_FULL = 0, Q_EMPTY, S_FULL, S_EMPTY, P_FULL, P_EMPTY, O_FULL, O_FREE, N_BAR };       // two of each
  auto bar = [&](int i, int x) { return smem_u32(bars + 2 * S::SLOTS + 2 * i + x); };
  static_assert(2 * S::SLOTS + 2 * N_BAR <= 40, "barriers");
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 40);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 41);
  volatile uint8_t* seen = reinterpret_cast<volatile uint8_t*>(bars + 42);   // [kTrSeen]: which 16-row parts of a tile have pages
  TrHead* hd = reinterpret_cast<TrHead*>(bars + 44);
  static_assert(44 * 8 + sizeof(TrHead) <= 512, "shared memory behind the barriers");

  if (tid == 0) {
    *abort_flag = 0;
    for (int i = 0; i < S::SLOTS; ++i) { mbar_init(kv_full(i), 1); mbar_init(kv_empty(i), 1); }
    for (int i = 0; i < N_BAR; ++i)
      for (int x = 0; x < 2; ++x) mbar_init(bar(i, x), i == S_EMPTY || i == P_FULL || i == O_FREE ? 8 : 1);
    fence_mbar_init();
  }
  // rows of Q that no box fills are zero
  for (int i = tid; i < 2 * S::Q_HALF / 16; i += kTrRowsThreads) reinterpret_cast<uint4*>(smem + S::Q)[i] = make_uint4(0, 0, 0, 0);
  // Tensor memory is only asked for when the kernels in front are done, and nothing behind comes up before it is there: none
  // of them can wait for the other's with tensor memory in hand.
  chained_wait();
  if (warp == kRwAlloc) { tmem_alloc(smem_u32(tmem_slot), 256); tmem_relinquish(); }
  tr_find<F>(pg, a, hd, reinterpret_cast<long long*>(smem));                 // (the ring is not in use yet)
  fence_proxy_async();
  if (tid == 0) a.heads[blockIdx.x] = *hd;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  chained_go();
  const uint32_t tmem = *tmem_slot;
  // Places of the g-th K and V in the order through the ring: K_0, K_1, V_0, K_2, V_1, ...; last: there is no next tile
  auto pos_k = [&](int g) { return g == 0 ? 0 : 2 * g - 1; };
  auto pos_v = [&](int g, bool last) { return last ? 2 * g + 1 : 2 * g + 2; };

  if (warp == kRwProducer) {
    // ---------------------------------------------------------------- producer
    const CUtensorMap* mq = reinterpret_cast<const CUtensorMap*>(maps.q);
    const CUtensorMap* mkv = reinterpret_cast<const CUtensorMap*>(maps.kv);
    if (lane == 0) { tma_prefetch_desc(mq); tma_prefetch_desc(mkv); }
    TrWalker<F> W(pg, a, *hd);
    TrItem I, J;
    int n_q = 0, ring = 0, g = 0;                      // Q tiles, ring tiles, key tiles so far
    bool ok = true, stop = false;
    const int page_rows = 1 << pg.shift, ppt = kTrBN >> pg.shift;            // pages per tile
    const uint32_t page_bytes = (uint32_t)page_rows * 128u;                  // of 64 dims
    auto wait = [&](uint32_t b, uint32_t parity) { ok = mbar_wait_spin(b, parity & 1u, abort_flag) && ok; };
    auto load_q = [&](const TrItem& X) {               // whole warp
      const int place = n_q % S::Q_PLACES;
      wait(bar(Q_EMPTY, place), ((uint32_t)(n_q / S::Q_PLACES) & 1u) ^ 1u);
      if (!warp_agreed(ok)) { stop = true; return; }
      ++n_q;
      if (lane == 0) {
        mbar_expect_tx(bar(Q_FULL, place), (uint32_t)(D / 64) * 128u * (uint32_t)(a.box_rows * a.G));
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf)
          tma_load_3d(smem_u32(smem + S::Q + place * S::Q_STEP + hf * S::Q_HALF), mq, 64 * hf, X.h * a.G, X.row0 + X.q0, bar(Q_FULL, place));
      }
      __syncwarp();
    };
    // K (kv = 0) or V of a tile: this lane's page of it, `pages` in all
    auto load = [&](int kv, int h, int entry, int pages) {                   // whole warp
      const int slot = ring % S::SLOTS;
      wait(kv_empty(slot), ((uint32_t)(ring / S::SLOTS) & 1u) ^ 1u);
      if (!warp_agreed(ok)) { stop = true; return; }
      ++ring;
      if (lane == 0) mbar_expect_tx(kv_full(slot), (uint32_t)(D / 64) * page_bytes * (uint32_t)pages);
      __syncwarp();
      if (lane < pages) {
        // (a page that is not there: rows behind the pool, which read as zero)
        int y = (unsigned)entry < (unsigned)pg.n_pages ? (int)k16_row(pg, a.Hk, entry, kv, h, 0) : (int)a.pool_rows;
        if (!DL_IN_BOUNDS(a.status, KID_TREE, y, (long long)a.pool_rows + 1)) y = (int)a.pool_rows;
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf)
          tma_load_2d(smem_u32(smem + slot * S::TILE + hf * S::HALF) + (uint32_t)lane * page_bytes, mkv, 64 * hf, y, kv_full(slot));
      }
      __syncwarp();
    };
    bool more = W.next(J);
    if (more && S::Q_PLACES == 2) load_q(J);
    int v_entry = -1, v_pages = 0, v_h = 0;            // the tile whose V is still to come
    while (!stop && more) {
      I = J;
      more = W.next(J);
      // page numbers of the share, 32 at a time in the warp's lanes
      const int32_t* row = pg.table + (size_t)I.b * pg.W;
      const int first_page = I.t * ppt, rows_all = I.held + I.n, limit = min(pg.W, (rows_all + page_rows - 1) >> pg.shift);
      auto block = [&](int k) {
        const int i = first_page + 32 * k + lane;
        return i < limit ? __ldcg(row + i) : -1;
      };
      int blk = 0, cur = block(0), after = block(1);
      for (int j = 0; j < I.nt && !stop; ++j) {
        const int k = (j * ppt) >> 5;
        if (k > blk) { cur = after; ++blk; after = block(blk + 1); }
        const int entry = __shfl_sync(0xffffffffu, cur, ((j * ppt) & 31) + (lane < ppt ? lane : 0));
        const int pages = min(ppt, (rows_all - (I.t + j) * kTrBN + page_rows - 1) >> pg.shift);
        // 16-row parts with a page, for the exponentials
        const bool lost = lane < pages && (unsigned)entry >= (unsigned)pg.n_pages;
        const unsigned miss = __ballot_sync(0xffffffffu, lost);
        const unsigned parts = __ballot_sync(0xffffffffu, lane < 8 && !((miss >> (lane >> (pg.shift - 4))) & 1));
        if (lane == 0) seen[g % kTrSeen] = (uint8_t)parts;
        if (lost) report_status(a.status, DL_ERR_INVALID_ARG, I.b);
        __syncwarp();
        load(0, I.h, entry, pages);
        if (!stop && g > 0) load(1, v_h, v_entry, v_pages);
        v_entry = entry; v_pages = pages; v_h = I.h;
        // the next item's Q beside this one's tiles; with one place for it, this one's
        if (j == 0 && !stop) {
          if (S::Q_PLACES == 1) load_q(I);
          else if (more) load_q(J);
        }
        ++g;
      }
    }
    if (!stop && g > 0) load(1, v_h, v_entry, v_pages);
    if (stop && lane == 0) {
      // what was requested must land before the CTA's shared memory is released
      for (int i = max(0, ring - S::SLOTS); i < ring; ++i)
        for (int k = 0; k < kSpinLimit && !mbar_try_wait(kv_full(i % S::SLOTS), (uint32_t)(i / S::SLOTS) & 1u); ++k) __nanosleep(40);
      for (int i = max(0, n_q - S::Q_PLACES); i < n_q; ++i)
        for (int k = 0; k < kSpinLimit && !mbar_try_wait(bar(Q_FULL, i % S::Q_PLACES), (uint32_t)(i / S::Q_PLACES) & 1u); ++k) __nanosleep(40);
    }
  } else if (warp == kRwIssuer) {
    // ---------------------------------------------------------------- MMA issuer
    // The whole warp walks the loop, so that counters and descriptors stay warp-uniform, and one elected lane issues.  Its lanes
    // wait each for itself, so the warp agrees before it goes on or stops.
    constexpr uint32_t idesc_s = idesc_bf16(128, N), idesc_o = idesc_bf16(128, N, 1, 1);       // O^T: both operands MN-major
    const uint32_t t_s = uniform32(tmem), t_o = uniform32(tmem + 128);
    const uint64_t k_base = uniform64(smem_desc_sw128(smem_u32(smem))), q_base = uniform64(smem_desc_sw128(smem_u32(smem + S::Q)));
    const uint64_t v_base = uniform64(smem_desc_sw128_mn(smem_u32(smem), S::HALF));
    const uint64_t p_base = uniform64(rw_desc_mn<S::P_ROW>(smem_u32(smem + S::P), S::P_BLOCK));
    TrWalker<F> W(pg, a, *hd);
    TrItem I;
    int g = 0, run = 0;                                // key tiles, items so far
    bool ok = true, stop = false;                      // this lane's waits so far; the warp has agreed to stop
    auto wait = [&](uint32_t b, uint32_t parity) { ok = mbar_wait_spin(b, parity & 1u, abort_flag) && ok; };
    auto full = [&](int pos) { wait(kv_full(pos % S::SLOTS), (uint32_t)(pos / S::SLOTS)); return pos % S::SLOTS; };
    struct { int ksteps, run; bool first, last; } v = {0, 0, false, false};  // the tile whose P V is still to come
    auto issue_o = [&](int t, bool at_end) {           // O^T += V^T P^T of tile t
      const int sv = full(pos_v(t, at_end)), pb = t % S::P_BUFS, ob = v.run & 1;
      if (v.first) wait(bar(O_FREE, ob), ((uint32_t)(v.run >> 1) & 1u) ^ 1u);
      wait(bar(P_FULL, pb), (uint32_t)(t / S::P_BUFS));
      if (!warp_agreed(ok)) { stop = true; return; }
      tc_fence_after();
      const uint64_t vd = v_base + (uint64_t)uniform32((uint32_t)sv * (S::TILE >> 4));
      const uint64_t pd = p_base + (uint64_t)uniform32((uint32_t)pb * (S::P_BLOCK >> 4));
      const uint32_t ksteps = uniform32((uint32_t)v.ksteps), acc = uniform32(!v.first), d = t_o + uniform32((uint32_t)ob * 64);
      const bool last = uniform32(v.last) != 0;
      if (rw_elect()) {
#pragma unroll
        for (uint32_t ks = 0; ks < 8; ++ks)
          if (ks < ksteps) mma_ss(d, vd + ks * (2048 >> 4), pd + ks * (16 * S::P_ROW >> 4), idesc_o, ks == 0 ? acc : 1u);
        mma_commit(kv_empty(sv));
        mma_commit(bar(P_EMPTY, pb));
        if (last) mma_commit(bar(O_FULL, ob));
      }
      __syncwarp();
    };
    while (!stop && W.next(I)) {
      for (int j = 0; j < I.nt && !stop; ++j) {
        // (with one place for Q the last item's P V does not wait for this one's Q)
        const bool before = j == 0 && S::Q_PLACES == 1;
        if (before && g > 0) issue_o(g - 1, false);
        if (stop) break;
        const int place = run % S::Q_PLACES, sb = g & 1;
        if (j == 0) wait(bar(Q_FULL, place), (uint32_t)(run / S::Q_PLACES));
        const int sk = full(pos_k(g));
        wait(bar(S_EMPTY, sb), ((uint32_t)(g >> 1) & 1u) ^ 1u);
        if (!warp_agreed(ok)) { stop = true; break; }
        tc_fence_after();
        const uint64_t kd = k_base + (uint64_t)uniform32((uint32_t)sk * (S::TILE >> 4));
        const uint64_t qd = q_base + (uint64_t)uniform32((uint32_t)place * (S::Q_STEP >> 4));
        const uint32_t d = t_s + uniform32((uint32_t)sb * 64);
        const bool last = uniform32(j == I.nt - 1) != 0;
        if (rw_elect()) {
#pragma unroll
          for (uint32_t ks = 0; ks < D / 16; ++ks)     // the second 64 dims are a tile of their own
            mma_ss(d, kd + (ks >> 2) * (S::HALF >> 4) + 2 * (ks & 3), qd + (ks >> 2) * (S::Q_HALF >> 4) + 2 * (ks & 3), idesc_s, ks != 0);
          mma_commit(bar(S_FULL, sb));
          mma_commit(kv_empty(sk));
          if (last) mma_commit(bar(Q_EMPTY, place));
        }
        __syncwarp();
        if (!before && g > 0) issue_o(g - 1, false);
        v.ksteps = (min(kTrBN, I.held + I.n - (I.t + j) * kTrBN) + 15) >> 4;
        v.run = run;
        v.first = j == 0;
        v.last = j == I.nt - 1;
        ++g;
      }
      ++run;
    }
    if (!stop && g > 0) issue_o(g - 1, true);
  } else if (warp < 8) {
    // ---------------------------------------------------------------- exponentials, epilogue
    constexpr int kW = N / 2;                                                // rows of one half
    const int half = warp >> 2, quad = warp & 3, t = tid & 127;              // t: this thread's key in a tile, and its dim
    const int col0 = half * kW;                                              // the half's first row
    const uint32_t lane_off = (uint32_t)(quad * 32) << 16;
    float* red = reinterpret_cast<float*>(smem + S::RED) + col0;             // [4][64]
    float* m_s = reinterpret_cast<float*>(smem + S::RED) + 4 * 64 + col0;    // [64] maxima in use, times scale
    float* l_s = m_s + 64;                                                   // [64]
    uint32_t* mask_s = reinterpret_cast<uint32_t*>(smem + S::RED + 1536) + half * 128;       // [64][2]
    const uint64_t sc2 = pack2(a.scale_log2, a.scale_log2);
    TrWalker<F> W(pg, a, *hd);
    TrItem I;
    int g = 0, run = 0;
    while (W.next(I)) {
      const int rows = min(I.n, a.PB) * a.G - col0;                          // of this half (a sequence's nodes are one tile of rows here)
      const int ob = run & 1, keys = I.held + I.n;
      const uint32_t o_addr = tmem + lane_off + 128 + ob * 64 + col0;
      // the mask's words, two a node (no more than 64 nodes): one per thread, kept until a tile needs them
      uint32_t mask_word = 0;
      if (a.mask && (t >> 1) < I.n && (t & 1) < a.words)
        mask_word = (uint32_t)__ldcg(a.mask + (size_t)(I.row0 + (t >> 1)) * a.words + (t & 1));
      uint64_t nm2[kW / 2], l2[kW / 2];                                      // minus the maxima, sums of this thread's keys
#pragma unroll
      for (int c = 0; c < kW / 2; ++c) nm2[c] = l2[c] = 0ull;
      for (int j = 0; j < I.nt; ++j, ++g) {
        const int c0 = (I.t + j) * kTrBN, key = c0 + t, sb = g & 1;
        const uint32_t s_addr = tmem + lane_off + sb * 64 + col0;
        mbar_wait_spin(bar(S_FULL, sb), (uint32_t)(g >> 1) & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
        // rows that see this thread's key
        const uint32_t parts = seen[g % kTrSeen];
        const bool masked = c0 + kTrBN > I.held || parts != 0xFF;
        uint32_t vis = 0xFFFFFFFFu;
        if (masked) {
          if (a.mask && c0 + kTrBN > I.held) {
            mask_s[t] = mask_word;
            rw_sync(half);
          }
          const int node = key - I.held;
          if (node >= I.n || !((parts >> (t >> 4)) & 1)) {
            vis = 0u;
          } else if (node >= 0) {
            if (a.mask) {
              vis = 0u;
              const uint64_t group = a.G >= 64 ? ~0ull : (1ull << a.G) - 1ull;
              const int i1 = min(I.n, (col0 + kW - 1) / a.G + 1);
#pragma unroll 4
              for (int i = col0 / a.G; i < i1; ++i) {
                const int lo = i * a.G - col0;
                const uint32_t bits = (uint32_t)(lo >= 0 ? group << lo : group >> -lo);
                vis |= ((mask_s[2 * i + (node >> 5)] >> (node & 31)) & 1) ? bits : 0u;
              }
            } else {
              const int lo = node * a.G - col0;
              vis = lo <= 0 ? 0xFFFFFFFFu : lo >= 32 ? 0u : 0xFFFFFFFFu << lo;
            }
          }
        }
        uint32_t s[kW];
        bool look = j == 0;
        for (;;) {
          __syncwarp();
          rw_tmem_ld<kW>(s_addr, s);
          tmem_ld_wait();
          if (masked) {
#pragma unroll
            for (int c = 0; c < kW; ++c)
              if (!((vis >> c) & 1)) s[c] = 0xFF800000u;           // -inf
          }
          if (look) {
            // The rows' maxima: over the warp's keys, then over the warps.  What a share has summed up so far follows.
            float mine = -INFINITY;
#pragma unroll
            for (int c = 0; c < kW; ++c) {
              const float top = rw_warp_max(__uint_as_float(s[c]));
              if (lane == c) mine = top;
            }
            if (lane < kW) red[quad * 64 + lane] = mine;
            rw_sync(half);
            if (t < kW) {
              const float top = fmaxf(fmaxf(red[t], red[64 + t]), fmaxf(red[128 + t], red[192 + t])) * a.scale_log2;
              // (below every score but -inf, and finite: keys that score -inf weigh 0 against it, were they all that came so far)
              const float old = j == 0 ? -3.402823466e38f : m_s[t];
              m_s[t] = fmaxf(old, top);
            }
            rw_sync(half);
            if (j > 0) {
              // everything up to the last tile is in O^T
              mbar_wait_spin(bar(P_EMPTY, (g - 1) % S::P_BUFS), (uint32_t)((g - 1) / S::P_BUFS) & 1u, abort_flag);
              __syncwarp();
              tc_fence_after();
              uint32_t o[kW];
              rw_tmem_ld<kW>(o_addr, o);
              tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < kW; c += 2) {
                float o0, o1;
                unpack2(nm2[c / 2], o0, o1);
                const uint64_t f = pack2(fast_exp2(-o0 - m_s[c]), fast_exp2(-o1 - m_s[c + 1]));
                l2[c / 2] = fmul2(l2[c / 2], f);
                unpack2(fmul2(pack2(__uint_as_float(o[c]), __uint_as_float(o[c + 1])), f), o0, o1);
                o[c] = __float_as_uint(o0);
                o[c + 1] = __float_as_uint(o1);
              }
              rw_tmem_st<kW>(o_addr, o);
              tmem_st_wait();
              tc_fence_before();
            }
#pragma unroll
            for (int c = 0; c < kW; c += 2) nm2[c / 2] = pack2(-m_s[c], -m_s[c + 1]);
          }
          float sum = 0.f, sum2 = 0.f;
#pragma unroll
          for (int c = 0; c < kW; c += 2) {
            float e0, e1;
            unpack2(ffma2(pack2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), sc2, nm2[c / 2]), e0, e1);
            e0 = fast_exp2(e0);
            e1 = fast_exp2(e1);
            sum += e0;
            sum2 += e1;
            s[c] = __float_as_uint(e0);
            s[c + 1] = __float_as_uint(e1);
          }
          // (the sum is over the half's rows, those of nobody among them: a NaN in one must not hide that another one's is too large)
          if (!rw_any(half, !look && !(sum + sum2 <= kRwFar))) break;
          look = true;                                             // the tile is done over under its own maxima
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(S_EMPTY, sb));
        const int pb = g % S::P_BUFS;
        uint32_t p[kW / 2];
#pragma unroll
        for (int c = 0; c < kW; c += 2) {
          const float e0 = __uint_as_float(s[c]), e1 = __uint_as_float(s[c + 1]);
          l2[c / 2] = fadd2(l2[c / 2], pack2(e0, e1));
          p[c / 2] = cvt_bf16x2(e0, e1);
        }
        mbar_wait_spin(bar(P_EMPTY, pb), ((uint32_t)(g / S::P_BUFS) & 1u) ^ 1u, abort_flag);
#pragma unroll
        for (int u = 0; u < kW / 8; ++u) {                         // 16-byte units of this key's row, XOR-swizzled
          const int unit = half * (kW / 8) + u;
          *reinterpret_cast<uint4*>(smem + S::P + (pb + (unit >> 2)) * S::P_BLOCK + t * S::P_ROW +
                                    (((unit & 3) ^ (N == 16 ? (t >> 2) & 1 : (t >> 1) & 3)) << 4)) =
              make_uint4(p[4 * u], p[4 * u + 1], p[4 * u + 2], p[4 * u + 3]);
        }
        if (half == 0 && key >= keys && t < ((keys - c0 + 15) & ~15)) {
          // a row behind the sequence's last that V^T P^T covers: 0 * x must stay 0 for any bit pattern of it
          const int pos = pos_v(g, j == I.nt - 1 && W.left <= 0), slot = pos % S::SLOTS;
          mbar_wait_spin(kv_full(slot), (uint32_t)(pos / S::SLOTS) & 1u, abort_flag);
#pragma unroll
          for (int u = 0; u < D / 8; ++u)
            *reinterpret_cast<uint4*>(smem + slot * S::TILE + (u >> 3) * S::HALF + t * 128 + (u & 7) * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(P_FULL, pb));
      }
      // ---- epilogue: the rows' sums over all keys, then O^T, a dim per thread
      {
        float l[kW];
#pragma unroll
        for (int c = 0; c < kW; c += 2) unpack2(l2[c / 2], l[c], l[c + 1]);
        const float v = rw_column_sums<kW>(l, lane);
        if (lane < kW) red[quad * 64 + lane] = v;
      }
      rw_sync(half);
      const bool whole = I.t == 0 && I.nt == I.T;                      // not cut by a border
      constexpr int kPartFloats = TrPart<D, F>::FLOATS;
      float* part = a.parts + ((size_t)blockIdx.x * 2 + (I.first ? 0 : 1)) * kPartFloats;
      if (t < kW) {
        const float l = (red[t] + red[64 + t]) + (red[128 + t] + red[192 + t]);
        l_s[t] = l != 0.f ? 1.0f / l : 0.f;                            // (a NaN sum is the row's)
        if (!whole && t < rows) reinterpret_cast<float2*>(part)[col0 + t] = make_float2(m_s[t], l);
      }
      rw_sync(half);
      mbar_wait_spin(bar(O_FULL, ob), (uint32_t)(run >> 1) & 1u, abort_flag);
      __syncwarp();
      tc_fence_after();
      uint32_t o[kW];
      rw_tmem_ld<kW>(o_addr, o);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(O_FREE, ob));
      if (t < D) {                                                     // (whole warps)
        if (whole) {
          // two rows at a time: even lanes store two dims of the first, odd lanes of the second
          const bool odd = lane & 1;
          const int node0 = col0 / a.G;
          int head = col0 - node0 * a.G;                               // row c: node c / G, head c % G
          size_t at = ((size_t)(I.row0 + node0) * a.H + I.h * a.G + head) * D;
          auto advance = [&] {
            at += D;
            if (++head == a.G) { head = 0; at += (size_t)(a.H - a.G) * D; }
          };
#pragma unroll
          for (int c = 0; c < kW; c += 2) {
            if (c >= rows) break;
            const float v0 = __uint_as_float(o[c]) * l_s[c], v1 = __uint_as_float(o[c + 1]) * l_s[c + 1];
            const float got = __shfl_xor_sync(0xffffffffu, odd ? v0 : v1, 1);
            const size_t at0 = at;
            advance();
            const size_t mine = (odd ? at : at0) + (t & ~1);
            if (c + (odd ? 1 : 0) < rows && DL_IN_BOUNDS(a.status, KID_TREE, mine + 1, (size_t)a.total * a.H * D))
              *reinterpret_cast<uint32_t*>(a.out + mine) = odd ? cvt_bf16x2(got, v1) : cvt_bf16x2(v0, got);
            advance();
          }
        } else {
#pragma unroll
          for (int c = 0; c < kW; ++c)
            if (c < rows) {
              float* po = part + 2 * TrPart<D, F>::ROWS + (size_t)(col0 + c) * D + t;
              if (DL_IN_BOUNDS(a.status, KID_TREE, po - a.parts, (long long)gridDim.x * 2 * kPartFloats)) *po = __uint_as_float(o[c]);
            }
        }
      }
      ++run;
    }
    if (*abort_flag && tid == 0) report_status(a.status, DL_ERR_TIMEOUT, blockIdx.x);
  } else if (warp == kRwCheck) {
    // starts that lead out of the tensors (they are clamped wherever they are used) and sequences with more nodes than were
    // said (cut off there) are reported
    if (blockIdx.x == 0)
      for (int b = lane; b < pg.B; b += 32) {
        const int s0 = __ldcg(a.starts + b), s1 = __ldcg(a.starts + b + 1);
        if (s0 < 0 || s1 < s0 || s1 > a.total || s1 - s0 > a.said_rows) report_status(a.status, DL_ERR_INVALID_ARG, b);
      }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kRwAlloc) { tc_fence_after(); tmem_dealloc(tmem, 256); }
}

bool attn_tree_rows_supported(const dl_ctx* ctx) {
  return ctx->smem_optin >= std::max(Rw<128, 64>::SMEM, Rw<64, 64>::SMEM);
}

template <int D, int N>
static cudaError_t rw_launch(const dl_ctx* ctx, const TrMaps& maps, const K16Pages& pg, const TrArgs& a, int ranges, cudaStream_t s) {
  static int attr_set[64];                             // (all calls ask for the same: two threads may)
  if (!attr_set[ctx->device & 63]) {
    const cudaError_t e = cudaFuncSetAttribute(attn_tree_rows_kernel<D, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, Rw<D, N>::SMEM);
    if (e != cudaSuccess) return e;
    attr_set[ctx->device & 63] = 1;
  }
  return launch_chained(attn_tree_rows_kernel<D, N>, dim3(ranges), dim3(kTrRowsThreads), Rw<D, N>::SMEM, s, maps, pg, a);
}

cudaError_t launch_attn_tree_rows(const dl_ctx* ctx, const TrMaps& maps, const K16Pages& pg, const TrArgs& a, int ranges, cudaStream_t s) {
  const int rows = a.box_rows * a.G;
  auto launch = ctx->desc.head_dim == 128 ? (rows <= 16 ? rw_launch<128, 16> : rows <= 32 ? rw_launch<128, 32> : rw_launch<128, 64>)
                                          : (rows <= 16 ? rw_launch<64, 16> : rows <= 32 ? rw_launch<64, 32> : rw_launch<64, 64>);
  return launch(ctx, maps, pg, a, ranges, s);
}

}  // namespace dl
