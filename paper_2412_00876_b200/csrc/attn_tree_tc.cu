// Attention of new rows (trees of drafted tokens, chunks of a prompt, single tokens) over a paged cache in 16 bits, on the tensor
// cores: more than 64 rows an item, the joining of parts, and the launcher.  An extension, not in the paper.  bf16, head_dim 64 or 128.
//
// Sequence b's n new rows (nodes) attend the cache's rows [0, held) and, by a mask or causally, the n rows behind them, which hold
// the nodes' own K and V.  The G query heads of a K/V head and the nodes make one matrix: row = (node, head), 128 / G nodes a
// tile of 128 rows (one TMA box [nodes][G heads][64 dims] is just that).  Keys come in tiles of 128 rows, a TMA box per page.
// How the work is cut into ranges: attn_tree.cuh.
//   warp 8        : the producer: Q tiles, then K and V tiles through a ring
//   warps 9, 10   : issue the MMAs of lane A / B: S = Q K^T into tensor memory, O += P V with P read from tensor memory
//   warps 0-3/4-7 : softmax and epilogue of lane A / B, one row per thread
//   warp 11       : allocates tensor memory (512 columns: O_A | S_A | O_B | S_B)
// A lane is a chain (softmax, P V and Q K^T, softmax); two of them keep the pipes busy.  What the lanes share is the template's
// choice.  Up to 128 rows (kTrSplit): both work on the same rows, lane A the even key tiles, B the odd ones, each through a ring
// of its own, and an item's end adds the two up.  More rows (kTrPair): each lane has a tile of rows, and a K/V tile serves both.
// Up to 64 rows go the other way round, keys across the matrix unit's rows: attn_tree_rows.cu.
// Every wait is bounded (pipeline.cuh); an abort leaves DL_ERR_TIMEOUT in the status word.
//
// P is rounded to bf16, as 16-bit matrix products take it, and once only: at most 2^-8 of a weight.  Sums are of the unrounded weights;
// scores, maxima, sums and the joining are fp32.
//
// Bound by a lane's chain of about 2.3 us a tile.  Chunks of 900-1100 nodes over 3000-8000 rows (32 heads, 8 of K/V): 380 GFLOP in 372 us
// cold and on its own, 1.03 PFLOP/s, and 22 us of joining; 421-429 us a call among others, 0.89 PFLOP/s.  Four trees of 32-48 nodes, 8
// heads each, over 60-131 thousand rows: three tiles of rows in two passes over K and V (1.45 GB), 385 us, 15 of them of joining.
// Two lanes through ONE ring, each waiting for its own tiles only, lose data: see Tr.  Odd last tiles of rows given to both lanes
// inside the kernel for pairs made those trees 321-360 us, but chunks 433-474 and short contexts 5 to 15 % slower; in a launch of their
// own: 368 instead of 375, and trees without such a tile 3 to 5 % slower.  The producer telling the others its items instead of
// everyone's own walk: 1 to 3 us more an item.
// The masked form of the pass unrolled like the other one: 101 -> 119 us where it matters most (instruction cache).  Visible keys looked up
// before the wait for scores: no gain.  Extra units of an item 1 instead of 4: 40.8 -> 42.6 us (100 nodes, 16 thousand rows), 61 -> 66.
// Joining: by arithmetic on the ranges instead of a search through their heads 4 us less; three or four CTAs of it a
// multiprocessor instead of two no change.
#include <algorithm>

#include "attn_packed_softmax.cuh"
#include "attn_tree.cuh"

namespace dl {

constexpr int kTrPatience = 4000, kTrTurnTiles = 4;                // polls for a turn, tiles from which lanes take turns (attn_packed_tc.cu)
// Registers per thread (the kernel starts every thread at 168): the warps that issue and load walk the items, for which 40 are too
// few (spilled, they hold up every hand-over: 1024 items of five key tiles 112 us, with 72 103, with 88 101; chunks of 1000 rows
// 432, 411, 417; four trees of 17-32 nodes with 8 heads over 95 thousand rows 225, 204, 217); the softmax warps do with 216.
constexpr int kTrRegsSmall = 72, kTrRegsSoftmax = 216;
static_assert(128 * kTrRegsSmall + 256 * kTrRegsSoftmax <= kTrThreads * 168, "more registers than the launch has");
template <int F> static constexpr int tr_whole_tiles() { return F == kTrRows ? 6 : 12; }      // key tiles up to which items are not cut

template <int D, int F> struct Tr {
  static constexpr bool kPair = F == kTrPair;
  static constexpr int HALF = 128 * 128;               // 128 rows of 64 dims
  static constexpr int TILE = (D / 64) * HALF;         // one operand tile
  static constexpr int Q_TILES = kPair ? 2 : 1;
  static constexpr int SLOTS = D == 128 ? 7 - Q_TILES : 12;
  // Slots of a ring.  A wait by parity only tells one use of a slot from the next: whoever waits for a slot's uses has to wait for
  // every one of them.  So lanes that take different tiles have a ring each.
  static constexpr int RING = kPair ? SLOTS : SLOTS / 2;
  static constexpr int KV = Q_TILES * TILE;            // offset of the rings (behind the Q tiles)
  static constexpr int EXCH = KV + SLOTS * TILE;       // [2][128] row maximum and sum of the lanes
  static constexpr int BAR = EXCH + (kPair ? 0 : 2 * 128 * 8);
  static constexpr int SMEM = BAR + 512;
};

// One lane's share of that: rows of nodes [q0, q_hi), `keys` of which it may see, tiles j = lane's first, + step, ...
struct TrLane { int q0, q_hi, keys, n_tiles; };

template <int F>
__device__ __forceinline__ TrLane tr_lane(const TrArgs& a, const TrItem& I, int x) {
  TrLane L;
  L.q0 = I.q0 + (F == kTrPair ? x * a.PB : 0);
  L.q_hi = min(I.n, L.q0 + a.PB);
  L.keys = I.held + (a.mask ? I.n : L.q_hi);
  if (F == kTrPair) L.n_tiles = L.q0 < I.n ? min(max((L.keys + kTrBN - 1) / kTrBN - I.t, 0), I.nt) : 0;
  else L.n_tiles = (I.nt + 1 - x) >> 1;
  return L;
}
// the lane's i-th tile, counted from the share's first
template <int F> __device__ __forceinline__ int tr_tile(int i, int x) { return F == kTrSplit ? 2 * i + x : i; }
// keys of the share's tile j that a lane's MMAs cover
__device__ __forceinline__ int tr_cols(const TrItem& I, const TrLane& L, int j) {
  return min(kTrBN, (L.keys - (I.t + j) * kTrBN + 15) & ~15);
}
// 32 bits of a row's mask from bit j0 on (zeros come in front and behind); m0, m1: its first two words.
__device__ __forceinline__ uint32_t tr_mask_bits(const int32_t* row, int words, uint32_t m0, uint32_t m1, int j0) {
  const int w = j0 >> 5;
  auto word = [&](int i) { return i == 0 ? m0 : i == 1 ? m1 : i > 0 && i < words ? (uint32_t)__ldcg(row + i) : 0u; };
  return __funnelshift_r(word(w), word(w + 1), j0 & 31);
}
__device__ __forceinline__ uint32_t tr_low(int n) { return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u; }

// The softmax of a tile of which a row sees the columns whose bits are set in vis (bit c of word q: column 32 q + c): 32 columns at a
// time in a rolled loop; otherwise as in attn_prefill_softmax.cuh, but for the step by which a row's maximum is raised: whole powers of
// two, so that what the tile has stored as bf16 already keeps its bits when it is scaled down, and P is rounded once only.  (By the
// difference itself P was rounded twice in such rows, 2.8 half steps of the output in all instead of 2.)
__device__ __forceinline__ void tr_softmax_words(uint32_t s_addr, uint32_t o_addr, int n_ch, const uint32_t (&vis)[4], bool owned,
                                                 int o_blocks, float scale_log2, float& m_used, float& l_run) {
  const uint64_t sc2 = pack2(scale_log2, scale_log2);
  uint32_t v0 = vis[0], v1 = vis[1], v2 = vis[2], v3 = vis[3];
#pragma unroll 1
  for (int q = 0; q < 4; ++q) {
    uint32_t pk[16];
    if (q < n_ch) {
      uint32_t buf[32];
      tmem_ld32(s_addr + 32 * q, buf);
      tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (!((v0 >> c) & 1)) buf[c] = 0xFF800000u;                // -inf
      float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int c = 0; c < 32; c += 8) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
          mx4[w] = fmax3(mx4[w], __uint_as_float(buf[c + 2 * w]), __uint_as_float(buf[c + 2 * w + 1]));
      }
      const float mc = fmax3(mx4[0], mx4[1], fmaxf(mx4[2], mx4[3])) * scale_log2;
      const bool need = owned && mc > m_used + kRescaleStep;
      if (__any_sync(0xffffffffu, need)) {
        const float m_old = m_used;
        if (need) m_used = m_old < -1e38f ? mc : m_old + ceilf(mc - m_old);              // (a first maximum has nothing in front of it)
        const float corr = need ? fast_exp2(m_old - m_used) : 1.0f;
        l_run *= corr;
        at_rescale_row(o_addr, s_addr, q, corr, o_blocks);
      }
      const uint64_t nm2 = pack2(-m_used, -m_used);
      float la = 0.f, lb = 0.f;
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        float e0, e1;
        unpack2(ffma2(pack2(__uint_as_float(buf[2 * c]), __uint_as_float(buf[2 * c + 1])), sc2, nm2), e0, e1);
        e0 = fast_exp2(e0);
        e1 = fast_exp2(e1);
        la += e0;
        lb += e1;
        pk[c] = cvt_bf16x2(e0, e1);
      }
      l_run += la + lb;
    } else {
#pragma unroll
      for (int c = 0; c < 16; ++c) pk[c] = 0u;
    }
    tmem_st16(s_addr + 16 * q, pk);
    v0 = v1; v1 = v2; v2 = v3;
  }
  tmem_st_wait();
}

template <int D, int F>
__global__ void __launch_bounds__(kTrThreads, 1)
attn_tree_kernel(const __grid_constant__ TrMaps maps, const K16Pages pg, const TrArgs a) {
  using S = Tr<D, F>;
  constexpr bool kPair = S::kPair;
  constexpr int kProducer = 8, kIssuer = 9, kLast = 11;
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
  // Q_*: of a Q tile (kPair: the lane's; else tile 0); the others of a lane
  enum { Q_FULL = 0, Q_EMPTY, S_FULL, P_HALF, P_FULL, O_FULL, O_FREE, N_BAR };
  auto bar = [&](int x, int i) { return smem_u32(bars + 2 * S::SLOTS + x * N_BAR + i); };
  static_assert(2 * S::SLOTS + 2 * N_BAR <= 40, "barriers");
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 40);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 41);
  volatile int* passes = reinterpret_cast<volatile int*>(bars + 42);         // [lane x][warp quad]: softmax passes behind it
  volatile uint8_t* seen = reinterpret_cast<volatile uint8_t*>(bars + 46);   // [kTrSeen]: which 16-row parts of a tile have pages
  TrHead* hd = reinterpret_cast<TrHead*>(bars + 48);
  static_assert(48 * 8 + sizeof(TrHead) <= 512, "shared memory behind the barriers");

  if (tid == 0) {
    *abort_flag = 0;
    for (int i = 0; i < 8; ++i) passes[i] = 0;
    for (int i = 0; i < S::SLOTS; ++i) { mbar_init(kv_full(i), 1); mbar_init(kv_empty(i), kPair ? 2 : 1); }
    for (int x = 0; x < 2; ++x)
      for (int i = 0; i < N_BAR; ++i)
        mbar_init(bar(x, i), i == P_HALF || i == P_FULL ? 4 : i == O_FREE ? (F == kTrSplit ? 8 : 4) : i == Q_EMPTY ? (F == kTrSplit ? 2 : 1) : 1);
    fence_mbar_init();
  }
  // Tensor memory is only asked for when the kernels in front are done, and nothing behind comes up before it is there: none
  // of them can wait for the other's with tensor memory in hand.
  chained_wait();
  if (warp == kLast) { tmem_alloc(smem_u32(tmem_slot), 512); tmem_relinquish(); }
  tr_find<F>(pg, a, hd, reinterpret_cast<long long*>(smem));             // (the ring is not in use yet)
  fence_proxy_async();
  if (tid == 0) a.heads[blockIdx.x] = *hd;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  chained_go();
  const uint32_t tmem = *tmem_slot;

  if (warp == kProducer) {
    // ---------------------------------------------------------------- producer
    reg_dec<kTrRegsSmall>();
    const CUtensorMap* mq = reinterpret_cast<const CUtensorMap*>(maps.q);
    const CUtensorMap* mkv = reinterpret_cast<const CUtensorMap*>(maps.kv);
    if (lane == 0) { tma_prefetch_desc(mq); tma_prefetch_desc(mkv); }
    TrWalker<F> W(pg, a, *hd);
    TrItem I;
    int n_q[2] = {0, 0}, ring[2] = {0, 0}, tiles = 0;  // Q tiles per place, tiles per ring, key tiles so far
    bool ok = true, stop = false;
    const int page_rows = 1 << pg.shift, ppt = kTrBN >> pg.shift;            // pages per tile
    const uint32_t page_bytes = (uint32_t)page_rows * 128u;                  // of 64 dims
    auto wait = [&](uint32_t b, uint32_t parity) { ok = mbar_wait_spin(b, parity & 1u, abort_flag) && ok; };
    auto load_q = [&](int buf, int q0) {               // whole warp; true: the warp goes on
      wait(bar(buf, Q_EMPTY), ((uint32_t)n_q[buf] & 1u) ^ 1u);
      if (!warp_agreed(ok)) { stop = true; return; }
      ++n_q[buf];
      if (lane == 0) {
        mbar_expect_tx(bar(buf, Q_FULL), (uint32_t)(D / 64) * 128u * (uint32_t)(a.box_rows * a.G));
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf)
          tma_load_3d(smem_u32(smem + buf * S::TILE + hf * S::HALF), mq, 64 * hf, I.h * a.G, I.row0 + q0, bar(buf, Q_FULL));
      }
      __syncwarp();
    };
    while (!stop && W.next(I)) {
      // page numbers of the share, 32 at a time in the warp's lanes: those of K's tile, and of the block in front for V's
      const int32_t* row = pg.table + (size_t)I.b * pg.W;
      const int first_page = I.t * ppt, limit = min(pg.W, (I.held + I.n + page_rows - 1) >> pg.shift);
      auto block = [&](int k) {
        const int i = first_page + 32 * k + lane;
        return i < limit ? __ldcg(row + i) : -1;
      };
      int blk = 0, cur = block(0), before = -1, after = block(1);
      const int rows_all = I.held + I.n;
      auto load = [&](int kv, int j) {                 // whole warp
        const int x = F == kTrSplit ? j & 1 : 0, use = ring[x] / S::RING, slot = x * S::RING + ring[x] % S::RING;
        wait(kv_empty(slot), ((uint32_t)use & 1u) ^ 1u);
        if (!warp_agreed(ok)) { stop = true; return; }
        ++ring[x];
        const int k = (j * ppt) >> 5;
        if (k > blk) { before = cur; cur = after; ++blk; after = block(blk + 1); }
        const int entry = __shfl_sync(0xffffffffu, k == blk ? cur : before, ((j * ppt) & 31) + (lane < ppt ? lane : 0));
        const int c0 = (I.t + j) * kTrBN;
        const int pages = min(ppt, (rows_all - c0 + page_rows - 1) >> pg.shift);
        const bool mine = lane < pages, there = (unsigned)entry < (unsigned)pg.n_pages;
        if (kv == 0) {                                 // 16-row parts with a page, for the softmax
          const int part = lane >> (pg.shift - 4);      // this lane's part lies in that page
          const unsigned miss = __ballot_sync(0xffffffffu, mine && !there);
          const unsigned parts = __ballot_sync(0xffffffffu, lane < 8 && !((miss >> part) & 1));
          if (lane == 0) seen[tiles % kTrSeen] = (uint8_t)parts;
          ++tiles;
          if (mine && !there) report_status(a.status, DL_ERR_INVALID_ARG, I.b);
        }
        if (lane == 0) mbar_expect_tx(kv_full(slot), (uint32_t)(D / 64) * page_bytes * (uint32_t)pages);
        __syncwarp();
        if (mine) {
          // (a page that is not there: rows behind the pool, which read as zero)
          int y = there ? (int)k16_row(pg, a.Hk, entry, kv, I.h, 0) : (int)a.pool_rows;
          if (!DL_IN_BOUNDS(a.status, KID_TREE, y, (long long)a.pool_rows + 1)) y = (int)a.pool_rows;
#pragma unroll
          for (int hf = 0; hf < D / 64; ++hf)
            tma_load_2d(smem_u32(smem + S::KV + slot * S::TILE + hf * S::HALF) + (uint32_t)lane * page_bytes, mkv, 64 * hf, y, kv_full(slot));
        }
        __syncwarp();
      };
      // (the first K tiles in front of Q, whose place is the last item's until that one's last Q K^T)
      load(0, 0);
      if (F == kTrSplit && !stop && I.nt > 1) load(0, 1);
      if (!stop && tr_lane<F>(a, I, 0).n_tiles > 0) load_q(0, I.q0);
      if (kPair && !stop && tr_lane<F>(a, I, 1).n_tiles > 0) load_q(1, I.q0 + a.PB);
      constexpr int kAhead = F == kTrSplit ? 2 : 1;    // K runs ahead of V by the tiles that the ring's users work on
      for (int j = 0; j < I.nt && !stop; ++j) {
        load(1, j);
        if (!stop && j + kAhead < I.nt) load(0, j + kAhead);
      }
    }
    if (stop && lane == 0) {
      // what was requested must land before the CTA's shared memory is released
      for (int x = 0; x < 2; ++x)
        for (int i = max(0, ring[x] - S::RING); i < ring[x]; ++i)
          for (int k = 0; k < kSpinLimit && !mbar_try_wait(kv_full(x * S::RING + i % S::RING), (uint32_t)(i / S::RING) & 1u); ++k) __nanosleep(40);
      for (int x = 0; x < 2; ++x)
        if (n_q[x] > 0)
          for (int k = 0; k < kSpinLimit && !mbar_try_wait(bar(x, Q_FULL), (uint32_t)(n_q[x] - 1) & 1u); ++k) __nanosleep(40);
    }
  } else if (warp >= kIssuer && warp < kIssuer + 2) {
    // ---------------------------------------------------------------- MMA issuer of one lane
    // The whole warp walks the loop, so that counters and descriptors stay warp-uniform, and one elected lane issues.  Its lanes
    // wait each for itself, so the warp agrees before it goes on or stops.
    reg_dec<kTrRegsSmall>();
    const int x = warp - kIssuer;
    const uint32_t t_o = uniform32(tmem + x * kAtLaneCols + kAtColO), t_s = uniform32(tmem + x * kAtLaneCols + kAtColS);
    constexpr uint32_t idesc_pv = idesc_bf16(kTrBM, D, 0, 1);          // B (= V) is MN-major
    const uint64_t q_base = uniform64(smem_desc_sw128(smem_u32(smem)));
    const uint64_t kv_desc = uniform64(smem_desc_sw128(smem_u32(smem + S::KV)));
    const uint64_t v_desc = uniform64(smem_desc_sw128_mn(smem_u32(smem + S::KV), S::HALF));
    TrWalker<F> W(pg, a, *hd);
    TrItem I;
    int n_item = 0, n_mine = 0, g0 = 0, ring0 = 0;     // items, those with tiles of this lane, its tiles, its ring's tiles so far
    bool ok = true, stop = false;                      // this lane's waits so far; the warp has agreed to stop
    auto wait = [&](uint32_t b, uint32_t parity) { ok = mbar_wait_spin(b, parity & 1u, abort_flag) && ok; };
    while (!stop && W.next(I)) {
      const TrLane L = tr_lane<F>(a, I, x);
      const int n_sub = L.n_tiles;
      auto full = [&](int u, int is_v) {               // waits for K or V of tile u of the ring's share; returns its slot
        const int t = ring0 + 2 * u + is_v, slot = (F == kTrSplit ? x * S::RING : 0) + t % S::RING;
        wait(kv_full(slot), (uint32_t)(t / S::RING));
        return slot;
      };
      const int qb = kPair ? x : 0;                    // Q tile
      const uint32_t q_use = (uint32_t)(kPair ? n_mine : n_item);
      const uint64_t q_desc = q_base + (uint64_t)uniform32((uint32_t)qb * (S::TILE >> 4));
      for (int u = -1; u < n_sub; ++u) {
        if (n_sub == 0) break;
        const bool has_pv = u >= 0, has_qk = u + 1 < n_sub;
        const int g = g0 + u, j = tr_tile<F>(max(u, 0), x), jn = tr_tile<F>(min(u + 1, n_sub - 1), x);
        int sv = 0, sk = 0;
        if (!has_pv) wait(bar(qb, Q_FULL), q_use);
        if (has_pv) sv = full(u, 1);
        if (has_qk) sk = full(u + 1, 0);
        if (u == 0) wait(bar(x, O_FREE), (uint32_t)n_mine ^ 1u);            // previous item's O has been read
        if (has_pv) wait(bar(x, P_HALF), (uint32_t)g);
        if (!warp_agreed(ok)) { stop = true; break; }
        tc_fence_after();
        const uint64_t vd = v_desc + (uint64_t)uniform32((uint32_t)sv * (S::TILE >> 4));
        const uint64_t kd = kv_desc + (uint64_t)uniform32((uint32_t)sk * (S::TILE >> 4));
        const uint32_t ksteps = has_pv ? uniform32((uint32_t)tr_cols(I, L, j) >> 4) : 0u, acc = uniform32(u != 0);
        const uint32_t idesc_qk = uniform32(idesc_bf16(kTrBM, (uint32_t)tr_cols(I, L, jn)));
        if (has_pv) {
          if (pk_elect()) {
#pragma unroll
            for (uint32_t ks = 0; ks < 4; ++ks)
              if (ks < ksteps) mma_ts(t_o, t_s + ks * 8, vd + ks * (2048 >> 4), idesc_pv, ks == 0 ? acc : 1u);
          }
          __syncwarp();
          wait(bar(x, P_FULL), (uint32_t)g);           // (agreed on at the next turn)
          __syncwarp();
          tc_fence_after();
        }
        if (pk_elect()) {
          if (has_pv) {
#pragma unroll
            for (uint32_t ks = 4; ks < 8; ++ks)
              if (ks < ksteps) mma_ts(t_o, t_s + ks * 8, vd + ks * (2048 >> 4), idesc_pv, 1u);
            mma_commit(kv_empty(sv));
            if (!has_qk) mma_commit(bar(x, O_FULL));
          }
          if (has_qk) {
#pragma unroll
            for (uint32_t ks = 0; ks < D / 16; ++ks) {
              constexpr uint64_t half = S::HALF >> 4;                  // the second 64 dims are a tile of their own
              mma_ss(t_s, q_desc + (ks >> 2) * half + 2 * (ks & 3), kd + (ks >> 2) * half + 2 * (ks & 3), idesc_qk, ks != 0);
            }
            mma_commit(bar(x, S_FULL));
            mma_commit(kv_empty(sk));
            if (u + 2 == n_sub) mma_commit(bar(qb, Q_EMPTY));
          }
        }
        __syncwarp();
      }
      if (F == kTrSplit && n_sub == 0) {                      // nothing of this item: its share of the Q tile's release
        wait(bar(qb, Q_FULL), q_use);
        stop = !warp_agreed(ok);
        if (!stop && lane == 0) mbar_arrive(bar(qb, Q_EMPTY));
      }
      if (kPair)                                       // tiles that only the other lane uses, in the ring's order
        for (int j = n_sub; j < I.nt && !stop; ++j) {
          const int s0 = full(j, 0);
          if (lane == 0 && ok) mbar_arrive(kv_empty(s0));
          const int s1 = full(j, 1);
          if (lane == 0 && ok) mbar_arrive(kv_empty(s1));
          stop = !warp_agreed(ok);
        }
      ring0 += 2 * (F == kTrSplit ? n_sub : I.nt);
      g0 += n_sub;
      ++n_item;
      if (n_sub > 0) ++n_mine;
    }
  } else if (warp < kProducer) {
    // ---------------------------------------------------------------- softmax / epilogue warps of one lane
    reg_inc<kTrRegsSoftmax>();
    const int x = warp >> 2, quad = warp & 3;
    const int row = quad * 32 + lane;                                  // row within the tile
    const uint32_t lane_off = (uint32_t)(quad * 32) << 16;
    const uint32_t s_addr = tmem + lane_off + x * kAtLaneCols + kAtColS;
    const uint32_t o_addr = tmem + lane_off + x * kAtLaneCols + kAtColO;
    float2* exch = reinterpret_cast<float2*>(smem + S::EXCH);
    const int my_node = row / a.G, my_head = row - my_node * a.G, warp_node = (quad * 32) / a.G;
    constexpr int kItemRows = TrPart<D, F>::ROWS, kPartFloats = TrPart<D, F>::FLOATS;
    TrWalker<F> W(pg, a, *hd);
    TrItem I;
    int g0 = 0, g_twin = 0, ring0 = 0, n_mine[2] = {0, 0}, tiles = 0;  // (n_mine: of both lanes)
    while (W.next(I)) {
      const TrLane L = tr_lane<F>(a, I, x), Lt = tr_lane<F>(a, I, x ^ 1);
      const int n_sub = L.n_tiles;
      const int node = L.q0 + my_node;
      const bool owned = my_node < a.PB && node < L.q_hi;
      const bool active = L.q0 + warp_node < L.q_hi && warp_node < a.PB;     // some row of the warp is a node's
      float m_used = -3.402823466e38f, l_run = 0.f;
      const int twin0 = kPair && n_sub >= kTrTurnTiles ? g_twin : -(1 << 30);
      const int32_t* mask_row = a.mask ? a.mask + (size_t)(I.row0 + min(node, I.n - 1)) * a.words : nullptr;
      uint32_t m0 = 0, m1 = 0;
      if (a.mask && active) {
        m0 = (uint32_t)__ldcg(mask_row);
        if (a.words > 1) m1 = (uint32_t)__ldcg(mask_row + 1);
      }
      for (int u = 0; u < n_sub; ++u) {
        const int j = tr_tile<F>(u, x), c0 = (I.t + j) * kTrBN;
        mbar_wait_spin(bar(x, S_FULL), (uint32_t)(g0 + u) & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
        auto turn = [&] {
          if (!kPair) return;
          if (lane == 0) {
            const int before = twin0 + min(u + x, Lt.n_tiles);
            for (int i = 0; i < kTrPatience && passes[4 * (x ^ 1) + quad] < before; ++i) { }
          }
          __syncwarp();
        };
        auto pass_on = [&] { if (kPair && lane == 0) passes[4 * x + quad] = g0 + u + 1; };
        auto hand_over = [&](int which) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(x, which));
        };
        const uint32_t parts = seen[(tiles + j) % kTrSeen];
        const int sees = a.mask ? I.held : I.held + L.q0 + warp_node + 1;      // keys that every row of the warp sees
        if (active && c0 + kTrBN <= sees && parts == 0xFF) {
          pk_softmax_full(s_addr, o_addr, owned, u > 0 ? D / 32 : 0, a.scale_log2, m_used, l_run, turn,
                          [&] { hand_over(P_HALF); }, pass_on);
          hand_over(P_FULL);
          continue;
        }
        turn();
        if (active) {
          uint32_t vis[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int base = c0 + 32 * w;
            uint32_t v;
            if (a.mask) {
              v = tr_low(I.held - base);
              if (base + 32 > I.held) v |= tr_mask_bits(mask_row, a.words, m0, m1, base - I.held);
              v &= tr_low(I.held + I.n - base);
            } else {
              v = tr_low(I.held + node + 1 - base);
            }
            if (!((parts >> (2 * w)) & 1)) v &= 0xFFFF0000u;
            if (!((parts >> (2 * w + 1)) & 1)) v &= 0x0000FFFFu;
            vis[w] = v;
          }
          const int n_ch = min(4, (L.keys - c0 + 31) >> 5);
          tr_softmax_words(s_addr, o_addr, n_ch, vis, owned, u > 0 ? D / 32 : 0, a.scale_log2, m_used, l_run);
        }
        pass_on();
        const int valid = I.held + I.n - c0;                           // V's rows behind them that P V covers are zeroed
        if (tr_cols(I, L, j) > valid) {
          const int t = ring0 + 2 * u + 1, slot = (F == kTrSplit ? x * S::RING : 0) + t % S::RING;
          mbar_wait_spin(kv_full(slot), (uint32_t)(t / S::RING) & 1u, abort_flag);
          char* v_s = smem + S::KV + slot * S::TILE;
          const int pad = tr_cols(I, L, j) - valid;
          for (int w = row; w < pad * (D / 8); w += 128) {
            const int rr = valid + w / (D / 8), c = w % (D / 8);
            *reinterpret_cast<uint4*>(v_s + (c >> 3) * S::HALF + rr * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async();
        }
        hand_over(P_HALF);
        hand_over(P_FULL);
      }
      // ---- epilogue
      const bool whole = I.t == 0 && I.nt == I.T;                      // not cut by a border
      const int slot = I.first ? 0 : 1;
      float* part = a.parts + ((size_t)blockIdx.x * 2 + slot) * kPartFloats;
      const size_t out_row = ((size_t)(I.row0 + node) * a.H + I.h * a.G + my_head) * D;
      if (F != kTrSplit) {
        const int part_row = x * 128 + row;
        if (n_sub > 0) {
          mbar_wait_spin(bar(x, O_FULL), (uint32_t)n_mine[x] & 1u, abort_flag);
          __syncwarp();
          tc_fence_after();
        }
        if (!whole && owned) reinterpret_cast<float2*>(part)[part_row] = make_float2(m_used, l_run);
        const float inv = l_run != 0.f ? 1.0f / l_run : 0.f;             // (a NaN sum is the row's)
        if (n_sub > 0) {
          if (active) {
#pragma unroll 1
            for (int rd = 0; rd < D / 64; ++rd) {
              uint32_t o[64];
              __syncwarp();
              tmem_ld64(o_addr + rd * 64, o);
              tmem_ld_wait();
              if (owned && whole) {
#pragma unroll
                for (int i = 0; i < 64; i += 16) {
                  uint32_t w[8];
#pragma unroll
                  for (int k = 0; k < 8; ++k) w[k] = cvt_bf16x2(__uint_as_float(o[i + 2 * k]) * inv, __uint_as_float(o[i + 2 * k + 1]) * inv);
                  if (DL_IN_BOUNDS(a.status, KID_TREE, out_row + rd * 64 + i + 15, (size_t)a.total * a.H * D))
                    tr_store32_any(a.out + out_row + rd * 64 + i, w, a.wide);
                }
              } else if (owned) {
                float* po = part + 2 * kItemRows + (size_t)part_row * D + rd * 64;
                if (DL_IN_BOUNDS(a.status, KID_TREE, po + 63 - a.parts, (long long)gridDim.x * 2 * kPartFloats)) {
#pragma unroll
                  for (int i = 0; i < 64; i += 8) tr_store32(po + i, o + i);
                }
              }
            }
            __syncwarp();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(x, O_FREE));
        }
      } else {
        // both lanes hold sums of the same rows: each takes half of the columns of both
#pragma unroll
        for (int y = 0; y < 2; ++y)
          if (tr_lane<F>(a, I, y).n_tiles > 0) mbar_wait_spin(bar(y, O_FULL), (uint32_t)n_mine[y] & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
        if (active) {
          exch[x * 128 + row] = make_float2(m_used, l_run);
          asm volatile("bar.sync %0, 64;" ::"r"(1 + quad) : "memory");
          const float2 twin = exch[(x ^ 1) * 128 + row];
          asm volatile("bar.sync %0, 64;" ::"r"(1 + quad) : "memory");       // read before the next item writes
          const float m = fmaxf(m_used, twin.x);
          const float w_me = l_run != 0.f ? fast_exp2(m_used - m) : 0.f, w_tw = twin.y != 0.f ? fast_exp2(twin.x - m) : 0.f;
          const float l = l_run * w_me + twin.y * w_tw;
          const float inv = whole ? (l != 0.f ? 1.0f / l : 0.f) : 1.f;
          const float f_me = w_me * inv, f_tw = w_tw * inv;
          const uint32_t base = tmem + lane_off + kAtColO + x * (D / 2);
          if (!whole && owned && x == 0) reinterpret_cast<float2*>(part)[row] = make_float2(m, l);
#pragma unroll 1
          for (int c = 0; c < D / 2; c += 32) {
            uint32_t p[32], q[32];
            __syncwarp();
            tmem_ld32(base + x * kAtLaneCols + c, p);
            tmem_ld32(base + (x ^ 1) * kAtLaneCols + c, q);
            tmem_ld_wait();
            // (a lane without a sum has left whatever was in tensor memory: not 0 times that, but nothing; NaN weights stay)
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const float u0 = w_me != 0.f ? __uint_as_float(p[i]) * f_me : 0.f, u1 = w_tw != 0.f ? __uint_as_float(q[i]) * f_tw : 0.f;
              p[i] = __float_as_uint(u0 + u1);
            }
            if (owned && whole) {
#pragma unroll
              for (int i = 0; i < 32; i += 16) {
                uint32_t w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = cvt_bf16x2(__uint_as_float(p[i + 2 * k]), __uint_as_float(p[i + 2 * k + 1]));
                if (DL_IN_BOUNDS(a.status, KID_TREE, out_row + x * (D / 2) + c + i + 15, (size_t)a.total * a.H * D))
                  tr_store32_any(a.out + out_row + x * (D / 2) + c + i, w, a.wide);
              }
            } else if (owned) {
              float* po = part + 2 * kItemRows + (size_t)row * D + x * (D / 2) + c;
              if (DL_IN_BOUNDS(a.status, KID_TREE, po + 31 - a.parts, (long long)gridDim.x * 2 * kPartFloats)) {
#pragma unroll
                for (int i = 0; i < 32; i += 8) tr_store32(po + i, p + i);
              }
            }
          }
          __syncwarp();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0)
          for (int y = 0; y < 2; ++y)
            if (tr_lane<F>(a, I, y).n_tiles > 0) mbar_arrive(bar(y, O_FREE));
      }
#pragma unroll
      for (int y = 0; y < 2; ++y)
        if (tr_lane<F>(a, I, y).n_tiles > 0) ++n_mine[y];
      g0 += n_sub;
      g_twin += Lt.n_tiles;
      ring0 += 2 * (F == kTrSplit ? n_sub : I.nt);
      tiles += I.nt;
    }
    if (*abort_flag && row == 0) report_status(a.status, DL_ERR_TIMEOUT, blockIdx.x);
  } else {
    reg_dec<kTrRegsSmall>();                             // same budget as the rest of its warpgroup
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
  if (warp == kLast) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

// Joins the parts of items that borders of ranges cut.  CTA (c, y) belongs to the border in front of range c; the CTAs of all
// borders that cut an item share its rows out between them, so that an item of many parts has many CTAs.  A warp takes two rows
// at a time, a lane D / 32 dims of each, with four parts of both in flight; where there are many parts a CTA takes a row at a
// time, and its warps share the parts.
constexpr int kTrJoinThreads = 256, kTrJoinWarps = kTrJoinThreads / 32;
constexpr int kTrJoinMany = 16;                                    // parts from which on a CTA takes a row at a time

// Sums of a row: relative to the maximum m, over parts.
template <int E> struct TrSum { float m, l, o[E]; };
template <int E> __device__ __forceinline__ void tr_add(TrSum<E>& s, float m, float l, const float* o) {
  if (l == 0.f) return;                                            // (a part without a sum has no values either; a NaN stays one)
  const float top = fmaxf(s.m, m), c = exp2f(s.m - top), w = exp2f(m - top);
  s.m = top;
  s.l = s.l * c + l * w;
#pragma unroll
  for (int e = 0; e < E; ++e) s.o[e] = s.o[e] * c + o[e] * w;
}
template <int E> __device__ __forceinline__ void tr_load(const float* p, float (&o)[E]) {
  if (E == 4) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
    o[0] = v.x; o[1] = v.y; o[2 % E] = v.z; o[3 % E] = v.w;
  } else {
    const float2 v = __ldcg(reinterpret_cast<const float2*>(p));
    o[0] = v.x; o[1] = v.y;
  }
}

template <int D, int F>
__global__ void __launch_bounds__(kTrJoinThreads)
attn_tree_join_kernel(const TrArgs a, int32_t ranges) {
  constexpr bool kPair = F == kTrPair;
  constexpr int kItemRows = TrPart<D, F>::ROWS, kPartFloats = TrPart<D, F>::FLOATS;
  constexpr int E = D / 32;
  __shared__ float far_m[kTrJoinWarps], far_l[kTrJoinWarps], far_o[kTrJoinWarps][D];
  const int c = blockIdx.x + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  chained_go();
  chained_wait();
  const TrHead hd = a.heads[c];
  if (hd.units == 0 || hd.t == 0) return;                          // the border falls between items (or there is none)
  constexpr int kExtra = tr_extra<F>();
  const long long W = hd.all, item = hd.first - hd.t - kExtra;     // the item's units begin there, its key tiles at tiles
  const long long tiles = item + kExtra, end = tiles + hd.T;
  // Range c holds units [W c / ranges, W (c + 1) / ranges), so unit u is range_of(u)'s; with fewer units than ranges each is a
  // range of its own, and others are empty between them.
  auto range_of = [&](long long u) { return (int)(((u + 1) * ranges - 1) / W); };
  const bool dense = W >= ranges;
  const int c_lo = range_of(tiles);
  const int n_parts = dense ? range_of(end - 1) - c_lo + 1 : hd.T;
  const int group = dense ? c - c_lo - 1 : (int)(hd.first - tiles) - 1, groups = n_parts - 1;  // this border among the item's
  const int slot0 = W * c_lo / ranges < item ? 1 : 0;              // where the first part lies
  const int rows = min(hd.n - hd.q0, (kPair ? 2 : 1) * a.PB) * a.G;
  const int me = blockIdx.y * groups + group, all = gridDim.y * groups;      // this CTA among the item's
  auto part = [&](int i) {
    const int r = dense ? c_lo + i : range_of(tiles + i);
    return a.parts + (size_t)(2 * r + (i == 0 ? slot0 : 0)) * kPartFloats;
  };
  auto row_in_part = [&](int r) { return kPair && r >= a.PB * a.G ? 128 + r - a.PB * a.G : r; };
  auto store = [&](int r, const TrSum<E>& s) {
    const int node = r / a.G, head = r - node * a.G;
    const float inv = s.l != 0.f ? 1.f / s.l : 0.f;
    const size_t at = ((size_t)(hd.row0 + hd.q0 + node) * a.H + hd.h * a.G + head) * D + lane * E;
    if (!DL_IN_BOUNDS(a.status, KID_TREE, at + E - 1, (size_t)a.total * a.H * D)) return;
#pragma unroll
    for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t*>(a.out + at + e) = cvt_bf16x2(s.o[e] * inv, s.o[e + 1] * inv);
  };
  auto none = [] {
    TrSum<E> s;
    s.m = -3.402823466e38f;
    s.l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s.o[e] = 0.f;
    return s;
  };
  if (n_parts >= kTrJoinMany) {
    for (int r = me; r < rows; r += all) {
      const int pr = row_in_part(r);
      TrSum<E> s = none();
      for (int i0 = warp; i0 < n_parts; i0 += 4 * kTrJoinWarps) {
        float2 ml[4];
        float o[4][E];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = i0 + k * kTrJoinWarps;
          if (i >= n_parts) continue;
          ml[k] = __ldcg(reinterpret_cast<const float2*>(part(i)) + pr);
          tr_load<E>(part(i) + 2 * kItemRows + (size_t)pr * D + lane * E, o[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i0 + k * kTrJoinWarps < n_parts) tr_add<E>(s, ml[k].x, ml[k].y, o[k]);
      }
      if (lane == 0) { far_m[warp] = s.m; far_l[warp] = s.l; }
#pragma unroll
      for (int e = 0; e < E; ++e) far_o[warp][lane * E + e] = s.o[e];
      __syncthreads();
      if (warp == 0) {
        TrSum<E> all = none();
#pragma unroll
        for (int w = 0; w < kTrJoinWarps; ++w) tr_add<E>(all, far_m[w], far_l[w], &far_o[w][lane * E]);
        store(r, all);
      }
      __syncthreads();
    }
    return;
  }
  for (int r = 2 * (me * kTrJoinWarps + warp); r < rows; r += 2 * all * kTrJoinWarps) {
    TrSum<E> s[2] = {none(), none()};
    const bool two = r + 1 < rows;
    const int pr[2] = {row_in_part(r), row_in_part(two ? r + 1 : r)};
    for (int i0 = 0; i0 < n_parts; i0 += 4) {
      float2 ml[4][2];
      float o[4][2][E];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i0 + k >= n_parts) continue;
        const float* p = part(i0 + k);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          ml[k][y] = __ldcg(reinterpret_cast<const float2*>(p) + pr[y]);
          tr_load<E>(p + 2 * kItemRows + (size_t)pr[y] * D + lane * E, o[k][y]);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i0 + k < n_parts) {
          tr_add<E>(s[0], ml[k][0].x, ml[k][0].y, o[k][0]);
          tr_add<E>(s[1], ml[k][1].x, ml[k][1].y, o[k][1]);
        }
    }
    store(r, s[0]);
    if (two) store(r + 1, s[1]);
  }
}

static int64_t tr_head_floats(int32_t sm_count) { return ((int64_t)sm_count * (sizeof(TrHead) / 4) + 63) & ~(int64_t)63; }

// Scratch: the ranges' heads, two parts a range of up to 256 rows.
int64_t attn_tree_scratch_floats(int32_t sm_count, const dl_model_desc& d) {
  return tr_head_floats(sm_count) + (int64_t)sm_count * 2 * 256 * (d.head_dim + 2);
}

template <int D> static constexpr int tr_smem() { return std::max(Tr<D, kTrSplit>::SMEM, Tr<D, kTrPair>::SMEM); }

bool attn_tree_supported(const dl_ctx* ctx) {
  return ctx->desc.dtype == DL_BF16 && ctx->tmap_encode != nullptr && ctx->smem_optin >= std::max(tr_smem<128>(), tr_smem<64>()) &&
         attn_tree_rows_supported(ctx);
}

template <int D, int F>
static cudaError_t tr_launch(dl_ctx* ctx, const TrMaps& maps, const K16Pages& pg, TrArgs a, cudaStream_t s) {
  // As many ranges as multiprocessors, but no more than there can be key tiles (or items, where those are not cut: where a table
  // row's pages hold few key tiles, a join would cost more than the CTA that has a tile more than others).
  const long long row_tiles = std::min(std::min<long long>((long long)pg.B * ((a.max_rows + a.PB - 1) / a.PB), (long long)a.total), 1LL << 20);
  const long long key_tiles = (((long long)pg.W << pg.shift) + a.max_rows + kTrBN - 1) / kTrBN;
  a.whole = key_tiles <= tr_whole_tiles<F>();
  const int ranges = (int)std::min<long long>(ctx->sm_count, std::max(1LL, row_tiles * a.Hk * (a.whole ? 1 : key_tiles + tr_extra<F>())));
  cudaError_t e;
  if constexpr (F == kTrRows) {
    e = launch_attn_tree_rows(ctx, maps, pg, a, ranges, s);
  } else {
    static int attr_set[64];                           // (all calls ask for the same: two threads may)
    if (!attr_set[ctx->device & 63]) {
      e = cudaFuncSetAttribute(attn_tree_kernel<D, F>, cudaFuncAttributeMaxDynamicSharedMemorySize, Tr<D, F>::SMEM);
      if (e != cudaSuccess) return e;
      attr_set[ctx->device & 63] = 1;
    }
    e = launch_chained(attn_tree_kernel<D, F>, dim3(ranges), dim3(kTrThreads), Tr<D, F>::SMEM, s, maps, pg, a);
  }
  if (e != cudaSuccess || ranges == 1 || a.whole) return e;
  const int rows = std::min((F == kTrPair ? 2 : 1) * a.PB, a.max_rows) * a.G;
  return launch_chained(attn_tree_join_kernel<D, F>, dim3(ranges - 1, (rows + 2 * kTrJoinWarps - 1) / (2 * kTrJoinWarps)),
                        dim3(kTrJoinThreads), 0, s, a, ranges);
}

cudaError_t launch_attn_tree(dl_ctx* ctx, const dl_pages* p, int32_t Hk, const void* pool, const void* q, int64_t q_stride,
                             const int32_t* starts, int32_t total, int32_t max_rows, const int32_t* mask, int32_t words,
                             float scale, void* out, cudaStream_t s) {
  const K16Pages pg = k16_pages(p);
  const int D = ctx->desc.head_dim, H = ctx->desc.n_heads;
  TrArgs a = {};
  a.starts = starts; a.mask = mask; a.out = static_cast<__nv_bfloat16*>(out);
  a.status = ctx->ws.status;
  a.heads = reinterpret_cast<TrHead*>(ctx->ws.kv4_partial);
  a.parts = ctx->ws.kv4_partial + tr_head_floats(ctx->sm_count);
  a.H = H; a.Hk = Hk; a.G = H / Hk; a.total = total; a.words = words;
  a.said_rows = mask ? (int)std::min<long long>(max_rows, 32LL * words) : max_rows;
  a.max_rows = std::min(a.said_rows, total);
  const int rows = (int)std::min<long long>((long long)a.max_rows * a.G, 1 << 20);
  // The largest sequence decides for all (the host knows no other).  A chunk of 1000 nodes over 4000 rows (32 heads, 8 of K/V) with 47
  // single tokens over 500-9000: 261 us, in two calls 96 + 144; with 15 tokens over 500-4000: 134, in two calls 109 + 42.
  const int form = rows <= kTrFewRows ? kTrRows : a.max_rows <= kTrBM / a.G ? kTrSplit : kTrPair;
  a.PB = (form == kTrRows ? kTrFewRows : kTrBM) / a.G;
  a.box_rows = std::min(a.PB, a.max_rows);
  a.scale_log2 = scale * 1.4426950408889634f;
  const uint64_t pool_rows = (2ull * Hk * pg.n_pages) << pg.shift;
  a.pool_rows = (uint32_t)pool_rows;
  a.wide = (reinterpret_cast<uintptr_t>(out) & 31u) == 0;
  TrMaps maps;
  const uint64_t dq[3] = {(uint64_t)D, (uint64_t)H, (uint64_t)total}, sq[2] = {2ull * D, 2ull * q_stride};
  const uint64_t dkv[2] = {(uint64_t)D, pool_rows}, skv[1] = {2ull * D};
  const uint32_t bq[3] = {64u, (uint32_t)a.G, (uint32_t)a.box_rows}, bkv[2] = {64u, 1u << pg.shift};
  if (!encode_bf16_map(ctx->tmap_encode, reinterpret_cast<CUtensorMap*>(maps.q), q, 3, dq, sq, bq) ||
      !encode_bf16_map(ctx->tmap_encode, reinterpret_cast<CUtensorMap*>(maps.kv), pool, 2, dkv, skv, bkv))
    return cudaErrorInvalidValue;
  auto launch = D == 128 ? (form == kTrRows ? tr_launch<128, kTrRows> : form == kTrSplit ? tr_launch<128, kTrSplit> : tr_launch<128, kTrPair>)
                         : (form == kTrRows ? tr_launch<64, kTrRows> : form == kTrSplit ? tr_launch<64, kTrSplit> : tr_launch<64, kTrPair>);
  return launch(ctx, maps, pg, a, s);
}

}  // namespace dl
