// Causal attention over packed prompts with grouped heads, on the tensor cores (Eq. 1 on whole prompts: what the layers in
// front of the token selection compute).  bf16, head_dim 64 or 128.
//
// Rows [starts[b], starts[b+1]) of q [total][H][D] and k, v [total][Hkv][D] are sequence b.  Query head h reads K/V
// head h / G, G = H / Hkv.  A query tile is 128 rows of (position, head): 128 / P positions of P heads of one group, P the
// largest power of two that divides G (one TMA box [positions][P heads][64 dims] is just that), so that a group's heads
// share every K/V tile and short prompts fill a tile sooner.  A work item is (sequence, P heads, PAIR of query tiles),
// pairs counted from the sequence's end (aligned to its start they measured 4 % slower on 700 tokens); the two tiles are
// the CTA's two lanes, the later positions lane A.  One persistent CTA per SM walks the items, longest first.
//   warp 8        : the producer: Q tiles, then K and V tiles of 128 rows through one ring of four slots, used by both
//                   lanes (a K/V tile crosses from L2 once per 256 query rows)
//   warps 9, 10   : issue the MMAs of lane A / B: S = Q K^T (128 x N) into tensor memory, O += P V with P read from
//                   tensor memory; block u = P_u V_u (its first half as soon as half of P is there), then Q K_{u+1}^T over
//                   P in order behind it
//   warps 0-3/4-7 : softmax and epilogue of lane A / B, one row per thread
//   warp 11       : allocates tensor memory (512 columns: O_A | S_A | O_B | S_B); the first CTA's checks `starts`
// A lane is a chain: softmax, P V and Q K^T, softmax; with head_dim 128 tensor memory has no room for a second score buffer
// (with 64, whose O takes half of its columns, a quarter of it is unused).  So the two
// lanes have to be half a period apart, and every link counts.  On 8192 tokens (32 heads, 8 of K/V), TFLOP/s: 611 with
// the MMAs issued by a single lane's code (operands moved to uniform registers one by one, 135 cycles an MMA), 800 with the
// issuing warp uniform, 930 without cubics for a part of the exponentials (the special-function unit is not what is
// short), 1055 with the passes taking turns, the maximum only looked for where a sum shows that it is needed, and an
// elected lane issuing, 1112 with the first half of P handed over early (two such sequences 1170, eight, over 4 ms, 1025;
// four with head_dim 64: 669).  Without any softmax the same kernel reaches 1635.  Two threads per row (16 softmax warps): 900.
// The last tile of a lane uses N = its keys rounded up to 16; where that reaches past the sequence's end, the softmax
// warps zero those V rows in shared memory first (0 * x must stay 0 for any bit pattern of a neighbour's rows).
// Every wait is bounded (pipeline.cuh); an abort leaves DL_ERR_TIMEOUT in the status word.
#include <algorithm>

#include "attn_prefill.cuh"
#include "attn_packed_softmax.cuh"
#include "common.cuh"
#include "tc05.cuh"

namespace dl {

constexpr int kPkThreads = 384;
constexpr int kPkSlots = 4;                            // K/V ring: two K and two V tiles
constexpr int kPkBM = 128, kPkBN = 128;
// Registers per thread (the kernel starts every thread at 168): a softmax warp holds a whole score row.  With 216 it spilled.
constexpr int kPkRegsSmall = 40, kPkRegsSoftmax = 232;
static_assert(128 * kPkRegsSmall + 256 * kPkRegsSoftmax <= 384 * 168, "more registers than the launch has");
// Polls a softmax warp waits for its turn (300 and 60000 take the same time within 2 %), and the key tiles from which on an
// item takes turns: 24k rows of 32 / 8 heads in sequences of 700, 1024 and 2048 take 196, 240 and 398 us from 1, 2 or 4 on,
// 206, 252 and 410 from 8 on, 206, 260 and 450 without; two of 8192 1050 - 1120 and 1225 without; of 256 and 384, 1 % more with 4
// than with 1.
constexpr int kPkPatience = 4000;
constexpr int kPkTurnTiles = 4;

template <int D> struct Pk {
  static constexpr int HALF = 128 * 128;               // 128 rows of 64 dims
  static constexpr int TILE = (D / 64) * HALF;         // one operand tile
  static constexpr int KV = 2 * TILE;                  // offset of the ring (behind the two Q tiles)
  static constexpr int STAGE = KV + kPkSlots * TILE;   // output staging, 4 KB per softmax warp
  static constexpr int BAR = STAGE + 8 * 4096;
  static constexpr int SMEM = BAR + 512;
};

struct PkMaps { alignas(64) unsigned char q[128]; alignas(64) unsigned char k[128]; alignas(64) unsigned char v[128]; alignas(64) unsigned char o[128]; };

struct PkArgs {
  const int32_t* starts; __nv_bfloat16* out; DeviceStatus* status;
  int32_t B, H, G, total, max_rows, said_rows;         // max_rows: the caller's said_rows, or total if that is less
  int32_t p_shift;                                     // P = 1 << p_shift heads per tile
  int32_t n_hs;                                        // H / P
  int32_t pairs;                                       // pairs of tiles of a sequence of max_rows rows
  int32_t by_column;                                   // columns that a CTA takes one at a time, see PkWalker
  float scale_log2;
};

// A pair of tiles: the 256 / P positions in front of q_hi (clipped at 0); n_kv: key tiles of its later tile.
struct PkItem { int b, h0, row0, n, q_hi, n_kv; };
struct PkLane { int q0, q_hi, n_tiles; bool exists; };   // rows of positions q0 .. q_hi - 1 are the lane's own

__device__ __forceinline__ PkLane pk_lane(const PkArgs& a, const PkItem& I, int x) {
  const int PB = kPkBM >> a.p_shift;                   // positions per tile
  PkLane L;
  L.q_hi = I.q_hi - x * PB;
  L.exists = L.q_hi > 0;
  L.q0 = max(L.q_hi - PB, 0);
  L.n_tiles = (L.q_hi + kPkBN - 1) / kPkBN;
  return L;
}
// keys of tile j that a lane's MMAs cover
__device__ __forceinline__ int pk_cols(const PkLane& L, int j) { return min(kPkBN, (L.q_hi - j * kPkBN + 15) & ~15); }

// Items in the order every role walks them.  Where sequences are of much the same length and there are several (sequence,
// heads) columns for every CTA (`by_column`, a multiple of the grid: how many of them go this way), a CTA takes a column
// at a time, all its pairs, the last one first: K and V of the column stay in L2.  The rest goes pair by pair over all
// columns, the last pairs first, which spreads a long sequence over all CTAs.  (All of a batch of 32 prompts of 700 tokens
// with 32 heads pair by pair: 930 MB read from DRAM instead of 560.)
// The rule (the longest at most 1.5 times the mean, four columns a CTA), 32 heads of 128, by columns and pair by pair: 640, 1024
// and 2048 columns of 624-743 rows 149 / 145, 230 / 242, 444 / 472 us, 512 the same; 32 sequences of up to 1100 rows whose
// longest is 1.07, 1.3, 1.45 and 1.6 times the mean 407 / 441, 355 / 365, 330 / 337 and 318 / 307; 24 of up to 4000,
// 1.2 times 2700 / 2650.
struct PkWalker {
  const PkArgs& a;
  int p, col, s0, s1, n_col, grid;                     // next: pair, column, its start and end (in flight)
  __device__ __forceinline__ explicit PkWalker(const PkArgs& a_) : a(a_) {
    n_col = a.B * a.n_hs;
    grid = (int)gridDim.x;
    p = 0;
    col = (int)blockIdx.x;
    if (a.by_column == 0) wrap();
    fetch();
  }
  __device__ __forceinline__ void wrap() {
    while (col >= n_col && p < a.pairs) { col -= n_col - a.by_column; ++p; }
  }
  __device__ __forceinline__ void fetch() {
    s0 = s1 = 0;
    if (p < a.pairs && col < n_col) {
      const int b = col / a.n_hs;
      s0 = ld_early(a.starts + b);
      s1 = ld_early(a.starts + b + 1);
    }
  }
  __device__ __forceinline__ bool next(PkItem& I) {
    for (;;) {
      if (p >= a.pairs) return false;
      const int cp = p, cc = col, c0 = min(max(s0, 0), a.total), c1 = min(max(s1, c0), a.total);
      I.b = cc / a.n_hs;
      I.h0 = (cc - I.b * a.n_hs) << a.p_shift;
      I.row0 = c0;
      I.n = min(c1 - c0, a.max_rows);
      I.q_hi = I.n - cp * (2 * kPkBM >> a.p_shift);
      I.n_kv = (I.q_hi + kPkBN - 1) / kPkBN;
      if (cc < a.by_column) {
        if (I.q_hi > (2 * kPkBM >> a.p_shift)) {
          ++p;                                         // the column's next pair: start and end stay
        } else {
          p = 0;
          col += grid;
          if (col >= a.by_column) wrap();
          fetch();
        }
      } else {
        col += grid;
        wrap();
        fetch();
      }
      if (I.q_hi > 0) return true;
    }
  }
};

template <int D>
__global__ void __launch_bounds__(kPkThreads, 1)
attn_packed_kernel(const __grid_constant__ PkMaps maps, const PkArgs a) {
  using S = Pk<D>;
  extern __shared__ __align__(1024) char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (smem_u32(smem) & 1023u) {                        // the swizzled tiles need 1024-byte alignment
    if (tid == 0) report_status(a.status, DL_ERR_ALIGNMENT, -1);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::BAR);
  auto kv_full = [&](int i) { return smem_u32(bars + i); };
  auto kv_empty = [&](int i) { return smem_u32(bars + kPkSlots + i); };
  enum { Q_FULL = 0, Q_EMPTY, S_FULL, P_HALF, P_FULL, O_FULL, O_FREE, N_BAR };
  auto bar = [&](int x, int i) { return smem_u32(bars + 2 * kPkSlots + x * N_BAR + i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 32);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 33);
  volatile int* passes = reinterpret_cast<volatile int*>(bars + 34);         // [lane x][warp quad]: softmax passes behind it

  if (tid == 0) {
    *abort_flag = 0;
    for (int i = 0; i < 8; ++i) passes[i] = 0;
    for (int i = 0; i < kPkSlots; ++i) { mbar_init(kv_full(i), 1); mbar_init(kv_empty(i), 2); }
    for (int x = 0; x < 2; ++x)
      for (int i = 0; i < N_BAR; ++i) mbar_init(bar(x, i), (i == P_HALF || i == P_FULL || i == O_FREE) ? 4 : 1);
    fence_mbar_init();
  }
  if (warp == 11) { tmem_alloc(smem_u32(tmem_slot), 512); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 8) {
    // ---------------------------------------------------------------- producer
    reg_dec<kPkRegsSmall>();
    if (lane == 0) {
      const CUtensorMap* mq = reinterpret_cast<const CUtensorMap*>(maps.q);
      const CUtensorMap* mk = reinterpret_cast<const CUtensorMap*>(maps.k);
      const CUtensorMap* mv = reinterpret_cast<const CUtensorMap*>(maps.v);
      tma_prefetch_desc(mq);
      tma_prefetch_desc(mk);
      tma_prefetch_desc(mv);
      PkWalker W(a);
      PkItem I;
      int n_q[2] = {0, 0}, t = 0;                      // Q tiles per lane, ring tiles so far
      auto load_q = [&](int x) {
        const PkLane L = pk_lane(a, I, x);
        if (!L.exists) return;
        mbar_wait_spin(bar(x, Q_EMPTY), ((uint32_t)n_q[x] & 1u) ^ 1u, abort_flag);
        if (*abort_flag) return;
        ++n_q[x];
        mbar_expect_tx(bar(x, Q_FULL), S::TILE);
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf)
          tma_load_3d(smem_u32(smem + x * S::TILE + hf * S::HALF), mq, 64 * hf, I.h0, I.row0 + L.q0, bar(x, Q_FULL));
      };
      auto load_kv = [&](const CUtensorMap* m, int j) {
        const int slot = t % kPkSlots;
        mbar_wait_spin(kv_empty(slot), ((uint32_t)(t / kPkSlots) & 1u) ^ 1u, abort_flag);
        if (*abort_flag) return;
        ++t;
        mbar_expect_tx(kv_full(slot), S::TILE);
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf)
          tma_load_3d(smem_u32(smem + S::KV + slot * S::TILE + hf * S::HALF), m, 64 * hf, I.h0 / a.G, I.row0 + j * kPkBN, kv_full(slot));
      };
      // (Bringing the next item's first tiles into L2 ahead of time measured 1-10 % slower.)
      while (!*abort_flag && W.next(I)) {
        load_q(0);
        load_kv(mk, 0);
        load_q(1);
        load_kv(mv, 0);
        for (int u = 1; u < I.n_kv && !*abort_flag; ++u) { load_kv(mk, u); load_kv(mv, u); }
      }
      if (*abort_flag) {
        // what was requested must land before the CTA's shared memory is released
        for (int i = max(0, t - kPkSlots); i < t; ++i)
          for (int k = 0; k < kSpinLimit && !mbar_try_wait(kv_full(i % kPkSlots), (uint32_t)(i / kPkSlots) & 1u); ++k) __nanosleep(40);
        for (int x = 0; x < 2; ++x)
          if (n_q[x] > 0)
            for (int k = 0; k < kSpinLimit && !mbar_try_wait(bar(x, Q_FULL), (uint32_t)(n_q[x] - 1) & 1u); ++k) __nanosleep(40);
      }
    }
  } else if (warp == 9 || warp == 10) {
    // ---------------------------------------------------------------- MMA issuer of one lane
    // The whole warp walks the loop, so that counters and descriptors stay warp-uniform, and one elected lane issues: an MMA
    // is then an instruction or two.  Its lanes wait each for itself, so the warp agrees before it goes on or stops.
    reg_dec<kPkRegsSmall>();
    {
      const int x = warp - 9;
      const uint32_t t_o = uniform32(tmem + x * kAtLaneCols + kAtColO), t_s = uniform32(tmem + x * kAtLaneCols + kAtColS);
      constexpr uint32_t idesc_pv = idesc_bf16(kPkBM, D, 0, 1);        // B (= V) is MN-major
      const uint64_t q_desc = uniform64(smem_desc_sw128(smem_u32(smem + x * S::TILE)));
      const uint64_t kv_desc = uniform64(smem_desc_sw128(smem_u32(smem + S::KV)));
      const uint64_t v_desc = uniform64(smem_desc_sw128_mn(smem_u32(smem + S::KV), S::HALF));
      PkWalker W(a);
      PkItem I;
      int n_item = 0, g0 = 0, ring0 = 0;               // this lane's items and key tiles, the ring's tiles so far
      bool ok = true, stop = false;                    // this lane's waits so far; the warp has agreed to stop
      auto wait = [&](uint32_t b, uint32_t parity) { ok = mbar_wait_spin(b, parity & 1u, abort_flag) && ok; };
      while (!stop && W.next(I)) {
        const PkLane L = pk_lane(a, I, x);
        const int n_sub = L.exists ? L.n_tiles : 0;
        auto full = [&](int u, int is_v) {             // waits for K_u or V_u; returns its slot
          const int t = ring0 + 2 * u + is_v;
          wait(kv_full(t % kPkSlots), (uint32_t)(t / kPkSlots));
          return t % kPkSlots;
        };
        for (int u = -1; u < n_sub; ++u) {
          if (n_sub == 0) break;
          const bool has_pv = u >= 0, has_qk = u + 1 < n_sub;
          const int g = g0 + u;
          int sv = 0, sk = 0;
          if (!has_pv) wait(bar(x, Q_FULL), (uint32_t)n_item);
          if (has_pv) sv = full(u, 1);
          if (has_qk) sk = full(u + 1, 0);
          if (u == 0) wait(bar(x, O_FREE), (uint32_t)n_item ^ 1u);            // previous item's O has been read
          if (has_pv) wait(bar(x, P_HALF), (uint32_t)g);
          if (!warp_agreed(ok)) { stop = true; break; }
          tc_fence_after();
          const uint64_t vd = v_desc + (uint64_t)uniform32((uint32_t)sv * (S::TILE >> 4));
          const uint64_t kd = kv_desc + (uint64_t)uniform32((uint32_t)sk * (S::TILE >> 4));
          const uint32_t ksteps = has_pv ? uniform32((uint32_t)pk_cols(L, u) >> 4) : 0u, acc = uniform32(u != 0);
          const uint32_t idesc_qk = uniform32(idesc_bf16(kPkBM, (uint32_t)pk_cols(L, min(u + 1, n_sub - 1))));
          if (has_pv) {
            if (pk_elect()) {
#pragma unroll
              for (uint32_t ks = 0; ks < 4; ++ks)
                if (ks < ksteps) mma_ts(t_o, t_s + ks * 8, vd + ks * (2048 >> 4), idesc_pv, ks == 0 ? acc : 1u);
            }
            __syncwarp();
            wait(bar(x, P_FULL), (uint32_t)g);         // (agreed on at the next turn: a vote here costs 0.5 % of long prompts)
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
                constexpr uint64_t half = S::HALF >> 4;                // the second 64 dims are a tile of their own
                mma_ss(t_s, q_desc + (ks >> 2) * half + 2 * (ks & 3), kd + (ks >> 2) * half + 2 * (ks & 3), idesc_qk, ks != 0);
              }
              mma_commit(bar(x, S_FULL));
              mma_commit(kv_empty(sk));
              if (u + 2 == n_sub) mma_commit(bar(x, Q_EMPTY));
            }
          }
          __syncwarp();
        }
        // tiles that only the other lane uses: this lane's share of the release, in the ring's order
        for (int u = n_sub; u < I.n_kv && !stop; ++u) {
          const int sk = full(u, 0);
          if (lane == 0 && ok) mbar_arrive(kv_empty(sk));
          const int sv = full(u, 1);
          if (lane == 0 && ok) mbar_arrive(kv_empty(sv));
          stop = !warp_agreed(ok);
        }
        ring0 += 2 * I.n_kv;
        g0 += n_sub;
        if (n_sub > 0) ++n_item;
      }
    }
  } else if (warp < 8) {
    // ---------------------------------------------------------------- softmax / epilogue warps of one lane
    reg_inc<kPkRegsSoftmax>();
    const int x = warp >> 2, quad = warp & 3;
    const int row = quad * 32 + lane;                                  // row within the query tile
    const uint32_t lane_off = (uint32_t)(quad * 32) << 16;
    const uint32_t s_addr = tmem + lane_off + x * kAtLaneCols + kAtColS;
    const uint32_t o_addr = tmem + lane_off + x * kAtLaneCols + kAtColO;
    const CUtensorMap* mo = reinterpret_cast<const CUtensorMap*>(maps.o);
    char* so = smem + S::STAGE + warp * 4096;                          // this warp's 4 KB: two 32 x 32 blocks
    const int P = 1 << a.p_shift, w_pos = (quad * 32) >> a.p_shift;    // this warp's first position in the tile
    const int w_last = (quad * 32 + 31) >> a.p_shift;
    PkWalker W(a);
    PkItem I;
    int g0 = 0, g_twin = 0, ring0 = 0, n_item = 0;                     // g_twin: the other lane's key tiles so far
    while (W.next(I)) {
      const PkLane L = pk_lane(a, I, x), Lt = pk_lane(a, I, x ^ 1);
      const int n_twin = Lt.exists ? Lt.n_tiles : 0;
      if (!L.exists) { ring0 += 2 * I.n_kv; g_twin += n_twin; continue; }
      const int pos = L.q0 + (row >> a.p_shift);                       // this thread's position
      const int r0 = L.q0 + w_pos;                                     // the warp's first position
      // (below every score but -inf, and finite: keys that score -inf weigh 0 against it, were they all that came so far)
      float m_used = -3.402823466e38f, l_run = 0.f;
      const int n_sub = L.n_tiles;
      const int twin0 = n_sub >= kPkTurnTiles ? g_twin : -(1 << 30);   // short items do not wait
      for (int u = 0; u < n_sub; ++u) {
        const int c0 = u * kPkBN;
        mbar_wait_spin(bar(x, S_FULL), (uint32_t)(g0 + u) & 1u, abort_flag);
        // The lanes' softmax passes take turns, A, B, A, B (warp by warp: the twin is the warp of the same scheduler).  Left
        // alone they fall into step: both softmax together, tensor pipe idle, then both wait for their MMAs.  Only a
        // matter of speed: the wait gives up after a while.
        auto turn = [&] {
          if (lane == 0) {
            const int before = twin0 + min(u + x, n_twin);
            for (int i = 0; i < kPkPatience && passes[4 * (x ^ 1) + quad] < before; ++i) { }
          }
          __syncwarp();
        };
        __syncwarp();
        tc_fence_after();
        auto pass_on = [&] { if (lane == 0) passes[4 * x + quad] = g0 + u + 1; };
        auto hand_over = [&](int which) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(x, which));
        };
        if (c0 + kPkBN - 1 <= r0) {
          pk_softmax_full(s_addr, o_addr, pos < L.q_hi, u > 0 ? D / 32 : 0, a.scale_log2, m_used, l_run, turn,
                          [&] { hand_over(P_HALF); }, pass_on);
          hand_over(P_FULL);
          continue;
        }
        // The causal edge or the sequence's end crosses the tile: 32 columns at a time in a rolled loop, those that some row of
        // the warp may see.  (A second unrolled pass for such tiles is faster by itself and slower in the kernel, by 12 %
        // on long prompts and 10 % on 700 tokens: the two no longer fit the instruction cache together.)
        const int n_ch = min(4, (min(L.q_hi, L.q0 + w_last + 1) - c0 + 31) >> 5);
        turn();
        at_softmax_chunks<0>(s_addr, o_addr, n_ch, pos - c0, c0 - r0, pos < L.q_hi, u > 0 ? D / 32 : 0, a.scale_log2, m_used, l_run);
        pass_on();
        const int pad = c0 + pk_cols(L, u) - I.n;                      // rows past the sequence's end that P V covers
        if (pad > 0) {
          const int t = ring0 + 2 * u + 1;
          mbar_wait_spin(kv_full(t % kPkSlots), (uint32_t)(t / kPkSlots) & 1u, abort_flag);
          char* v_s = smem + S::KV + (t % kPkSlots) * S::TILE;
          const int valid = I.n - c0;
          for (int w = row; w < pad * (D / 8); w += 128) {
            const int rr = valid + w / (D / 8), c = w % (D / 8);
            *reinterpret_cast<uint4*>(v_s + (c >> 3) * S::HALF + rr * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async();
        }
        hand_over(P_HALF);
        hand_over(P_FULL);
      }
      // ---- epilogue: O / l -> bf16 -> out, 64 columns per round through this warp's staging (16-byte units XOR-swizzled
      // by row pair: the 64-byte swizzle of the tensor map)
      mbar_wait_spin(bar(x, O_FULL), (uint32_t)n_item & 1u, abort_flag);
      __syncwarp();
      tc_fence_after();
      const float inv = 1.0f / l_run;
      const bool whole = L.q0 + w_last < L.q_hi;                       // warp-uniform
#pragma unroll 1
      for (int rd = 0; rd < D / 64; ++rd) {
        uint32_t o[64];
        tmem_ld64(o_addr + rd * 64, o);
        if (lane == 0) bulk_wait_read<0>();              // earlier stores must have read the staging
        tmem_ld_wait();
        if (rd == D / 64 - 1) tc_fence_before();         // all of O is in registers: the next item may overwrite it
        __syncwarp();
        if (rd == D / 64 - 1 && lane == 0) mbar_arrive(bar(x, O_FREE));
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint32_t* ob = o + 32 * blk + 8 * u;
            uint4 w;
            w.x = cvt_bf16x2(__uint_as_float(ob[0]) * inv, __uint_as_float(ob[1]) * inv);
            w.y = cvt_bf16x2(__uint_as_float(ob[2]) * inv, __uint_as_float(ob[3]) * inv);
            w.z = cvt_bf16x2(__uint_as_float(ob[4]) * inv, __uint_as_float(ob[5]) * inv);
            w.w = cvt_bf16x2(__uint_as_float(ob[6]) * inv, __uint_as_float(ob[7]) * inv);
            *reinterpret_cast<uint4*>(so + blk * 2048 + lane * 64 + ((u ^ ((lane >> 1) & 3)) << 4)) = w;
          }
        }
        if (whole) {
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            tma_store_4d(mo, smem_u32(so), rd * 64, I.h0, I.row0 + r0, 0);
            tma_store_4d(mo, smem_u32(so + 2048), rd * 64 + 32, I.h0, I.row0 + r0, 0);
            bulk_commit();
          }
        } else {
          __syncwarp();
#pragma unroll
          for (int blk = 0; blk < 2; ++blk) {
#pragma unroll
            for (int it = 0; it < 4; ++it) {
              const int r = it * 8 + (lane >> 2), u = lane & 3;
              const uint4 w = *reinterpret_cast<const uint4*>(so + blk * 2048 + r * 64 + ((u ^ ((r >> 1) & 3)) << 4));
              const int rp = L.q0 + ((quad * 32 + r) >> a.p_shift);
              const size_t at = ((size_t)(I.row0 + rp) * a.H + I.h0 + ((quad * 32 + r) & (P - 1))) * D + (2 * rd + blk) * 32 + u * 8;
              if (rp < L.q_hi && DL_IN_BOUNDS(a.status, KID_PACKED, at + 7, (size_t)a.total * a.H * D))
                *reinterpret_cast<uint4*>(a.out + at) = w;
            }
          }
          __syncwarp();                                  // the next round overwrites what these loads read
        }
      }
      g0 += n_sub;
      g_twin += n_twin;
      ring0 += 2 * I.n_kv;
      ++n_item;
    }
    if (lane == 0) bulk_wait_read<0>();                  // staged data must be read before shared memory goes
    if (*abort_flag && row == 0) report_status(a.status, DL_ERR_TIMEOUT, blockIdx.x);
  } else {
    reg_dec<kPkRegsSmall>();                             // same budget as the rest of its warpgroup
    // starts that lead out of the tensors (they are clamped wherever they are used) and sequences longer than max_rows
    // (cut off there) are reported
    if (blockIdx.x == 0)
      for (int b = lane; b < a.B; b += 32) {
        const int s0 = __ldg(a.starts + b), s1 = __ldg(a.starts + b + 1);
        if (s0 < 0 || s1 < s0 || s1 > a.total || s1 - s0 > a.said_rows) report_status(a.status, DL_ERR_INVALID_ARG, b);
      }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 11) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

template <int D>
static cudaError_t pk_launch(dl_ctx* ctx, const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride,
                             int32_t Hk, PkArgs& a, cudaStream_t s) {
  const int P = 1 << a.p_shift;
  PkMaps maps;
  const uint64_t dq[3] = {(uint64_t)D, (uint64_t)a.H, (uint64_t)a.total}, sq[2] = {2ull * D, 2ull * q_stride};
  const uint64_t dk[3] = {(uint64_t)D, (uint64_t)Hk, (uint64_t)a.total}, sk[2] = {2ull * D, 2ull * kv_stride};
  const uint64_t dout[4] = {(uint64_t)D, (uint64_t)a.H, (uint64_t)a.total, 1}, so[3] = {2ull * D, 2ull * D * a.H, 2ull * D * a.H * a.total};
  const uint32_t bq[3] = {64u, (uint32_t)P, (uint32_t)(kPkBM / P)}, bk[3] = {64u, 1u, (uint32_t)kPkBN};
  const uint32_t bo[4] = {32u, (uint32_t)P, (uint32_t)(32 / P), 1u};
  if (!encode_bf16_map(ctx->tmap_encode, reinterpret_cast<CUtensorMap*>(maps.q), q, 3, dq, sq, bq) ||
      !encode_bf16_map(ctx->tmap_encode, reinterpret_cast<CUtensorMap*>(maps.k), k, 3, dk, sk, bk) ||
      !encode_bf16_map(ctx->tmap_encode, reinterpret_cast<CUtensorMap*>(maps.v), v, 3, dk, sk, bk) ||
      !encode_bf16_map(ctx->tmap_encode, reinterpret_cast<CUtensorMap*>(maps.o), a.out, 4, dout, so, bo, CU_TENSOR_MAP_SWIZZLE_64B))
    return cudaErrorInvalidValue;
  const long long columns = (long long)a.B * a.n_hs, items = columns * a.pairs;
  if (items >= (1LL << 31) - ctx->sm_count) return cudaErrorInvalidValue;
  a.by_column = 0;
  if (2LL * a.B * a.max_rows <= 3LL * a.total && columns >= 4LL * ctx->sm_count)
    a.by_column = (int)(columns / ctx->sm_count) * ctx->sm_count;
  static int attr_set[64];
  if (!attr_set[ctx->device & 63]) {
    const cudaError_t e = cudaFuncSetAttribute(attn_packed_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Pk<D>::SMEM);
    if (e != cudaSuccess) return e;
    attr_set[ctx->device & 63] = 1;
  }
  attn_packed_kernel<D><<<(int)std::min<long long>(items, ctx->sm_count), kPkThreads, Pk<D>::SMEM, s>>>(maps, a);
  return cudaGetLastError();
}

bool attn_packed_supported(const dl_ctx* ctx) {
  const dl_model_desc& d = ctx->desc;
  return d.dtype == DL_BF16 && ctx->tmap_encode != nullptr && (size_t)ctx->smem_optin >= (size_t)Pk<128>::SMEM;
}

cudaError_t launch_attn_packed(dl_ctx* ctx, const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride,
                               const int32_t* starts, int32_t B, int32_t Hk, int32_t total, int32_t max_rows, float scale,
                               void* out, cudaStream_t s) {
  const dl_model_desc& d = ctx->desc;
  PkArgs a;
  a.starts = starts;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.status = ctx->ws.base ? ctx->ws.status : nullptr;
  a.B = B; a.H = d.n_heads; a.G = d.n_heads / Hk; a.total = total; a.max_rows = std::min(max_rows, total);
  a.said_rows = max_rows;
  a.p_shift = 0;
  while (a.p_shift < 4 && a.G % (2 << a.p_shift) == 0) ++a.p_shift;
  a.n_hs = a.H >> a.p_shift;
  const int pair_rows = 2 * kPkBM >> a.p_shift;
  a.pairs = (a.max_rows + pair_rows - 1) / pair_rows;
  a.scale_log2 = scale * 1.4426950408889634f;
  return d.head_dim == 128 ? pk_launch<128>(ctx, q, k, v, q_stride, kv_stride, Hk, a, s)
                           : pk_launch<64>(ctx, q, k, v, q_stride, kv_stride, Hk, a, s);
}

}  // namespace dl
