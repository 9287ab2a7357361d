// What the kernels of attention over the paged 16-bit cache share (attn_tree_tc.cu, attn_tree_rows.cu): the cut of a call's work into
// even ranges and the walk through a range.
//
// Few rows and many keys is the usual shape, so the work is (sequence, tile of rows, K/V head) items of T key tiles each, and ALL
// key tiles of a call are cut into as many even ranges as there are CTAs, whatever the lengths are: a CTA's range covers the end
// of one item, some whole ones, the start of another.  Items cut by a border leave their parts (sums, row maxima) in
// scratch, and a second kernel joins them in order: no result depends on timing.
// An item costs more than its key tiles (its masked tile, the hand-over to the next one, its outputs): it counts tr_extra() units
// more, in front of its tiles, so that a range of many short items holds fewer tiles.
// Short contexts (TrArgs::whole) are not cut: a range holds whole items, as many as the others or one more, and nothing is
// joined.  The host decides, by what a row of the table has columns for: a wide table is cut whatever the lengths are.  With up to 64
// rows an item that goes up to 6 key tiles.  4 nodes with 32 heads, 8 key heads: 8 sequences of 60, 200 and
// 400 rows 10.3, 12.7 and 14.9 us cut, 7.8, 8.8 and 10.7 whole; 32 sequences 12.4, 20.0 and 24.8 cut, 11.3, 15.3 and 20.4 whole.
// 40 uneven sequences of up to 400 rows with 32 key heads, where a CTA has nine items, lose 63.5 -> 67.6, those of up to 200 win
// 54.5 -> 51.4; up to 10 tiles 85 -> 90, up to 12 82 -> 95.  More rows leave larger parts, so there it is 12: 32 heads, 50-100 nodes
// over up to 600, 800, 1100 rows, 6 sequences 34.1, 38.4, 40.9 cut, 30.0, 33.7, 39.0 whole; 32 sequences 98, 112, 118 and 89, 106, 119.
#pragma once

#include "attn_prefill.cuh"
#include "kv16.cuh"
#include "tc05.cuh"

namespace dl {

constexpr int kTrBM = 128, kTrBN = 128;
// How an item's rows are laid out: see attn_tree_tc.cu (kTrSplit, kTrPair) and attn_tree_rows.cu (kTrRows)
enum TrForm { kTrRows = 0, kTrSplit = 1, kTrPair = 2 };
constexpr int kTrFewRows = 64;                                     // rows up to which kTrRows takes an item
constexpr int kTrSeen = 16;                                        // key tiles whose page flags are kept
// rows that a part of an item has room for, and its floats
template <int D, int F> struct TrPart {
  static constexpr int ROWS = F == kTrPair ? 256 : F == kTrSplit ? 128 : kTrFewRows;
  static constexpr int FLOATS = ROWS * (D + 2);
};
constexpr int kTrThreads = 384, kTrRowsThreads = 384;
template <int F> __host__ __device__ constexpr int tr_threads() { return F == kTrRows ? kTrRowsThreads : kTrThreads; }

struct TrMaps { alignas(64) unsigned char q[128]; alignas(64) unsigned char kv[128]; };

// What a CTA's range begins with, for the joining kernel.
//   (b, q0, h), t: its first item and key tile; units: what the walk has left, without extra units in front of the first tile
//   (0: no tile); first, all: its first unit among all units, and their number
struct TrHead { int b, q0, h, t; int T, n, row0, held; long long units, first, all; };

struct TrArgs {
  const int32_t* starts; const int32_t* mask; __nv_bfloat16* out; DeviceStatus* status;
  TrHead* heads; float* parts;                         // [grid], [grid][2 slots][rows of an item][D + 2]
  int32_t H, Hk, G, PB, total, max_rows, said_rows, words;   // PB: nodes per tile of rows
  int32_t box_rows;                                    // nodes per Q box
  uint32_t pool_rows;                                  // rows of the pool's tensor map
  int32_t wide;                                        // out is 32-byte aligned
  int32_t whole;                                       // ranges are of whole items, each of them a unit
  float scale_log2;
};

// Key tiles of an item: nodes [q0, ...) of a sequence.
template <int F>
__device__ __forceinline__ int tr_reach(const TrArgs& a, int q0) { return q0 + (F == kTrPair ? 2 : 1) * a.PB; }
template <int F>
__device__ __forceinline__ int tr_tiles(const TrArgs& a, int held, int n, int q0) {
  return (held + (a.mask ? n : min(n, tr_reach<F>(a, q0))) + kTrBN - 1) / kTrBN;
}

// Extra units of an item, as measured: a serving batch of trees (kTrRows) 83, 82.4, 81.9 us with 2, 3, 4 and 90 without, single tokens 143
// without and 138; pairs see attn_tree_tc.cu.
template <int F> __host__ __device__ constexpr int tr_extra() { return F == kTrRows ? 3 : 4; }

struct TrSeq { int row0, n, held; };
__device__ __forceinline__ TrSeq tr_seq(const K16Pages& pg, const TrArgs& a, int b) {
  TrSeq s;
  s.row0 = k16_start(a.starts, b, a.total);
  s.n = min(max(k16_start(a.starts, b + 1, a.total) - s.row0, 0), a.max_rows);
  s.held = (int)min((long long)max(__ldcg(pg.len + b), 0), (long long)pg.W << pg.shift);
  return s;
}

// A CTA's share of an item: key tiles [t, t + nt) of T.
struct TrItem { int b, h, row0, n, held, q0, T, t, nt; bool first; };
// Walks a CTA's items; every role does so for itself.
template <int F>
struct TrWalker {
  const K16Pages& pg; const TrArgs& a;
  TrSeq s, ahead;                                      // the sequence, the one behind it (requested early)
  int b, h, q0, t; long long left; bool first;
  __device__ __forceinline__ TrWalker(const K16Pages& pg_, const TrArgs& a_, const TrHead& hd) : pg(pg_), a(a_) {
    b = hd.b; h = hd.h; q0 = hd.q0; t = hd.t; left = hd.units; first = true;
    s.row0 = hd.row0; s.n = hd.n; s.held = hd.held;
    if (left > 0) fetch();
  }
  __device__ __forceinline__ void fetch() {
    ahead.row0 = ahead.n = ahead.held = 0;
    if (b + 1 < pg.B) ahead = tr_seq(pg, a, b + 1);
  }
  __device__ __forceinline__ bool next(TrItem& I) {
    if (left <= 0) return false;
    I.b = b; I.h = h; I.row0 = s.row0; I.n = s.n; I.held = s.held; I.q0 = q0; I.t = t; I.first = first;
    I.T = tr_tiles<F>(a, s.held, s.n, q0);
    I.nt = a.whole ? I.T : (int)min((long long)(I.T - t), left);
    left -= a.whole ? 1 : I.nt;
    first = false;
    t = 0;
    if (left > 0 && !a.whole) left = max(left - tr_extra<F>(), 0ll);   // the next item's extra units
    if (left > 0 && ++h == a.Hk) {
      h = 0;
      q0 = tr_reach<F>(a, q0);
      if (q0 >= s.n) {
        q0 = 0;
        do { ++b; s = ahead; fetch(); } while (s.n == 0 && b + 1 < pg.B);
        if (s.n == 0) left = 0;                        // (the ranges end with the last sequence that has nodes)
      }
    }
    return true;
  }
};

// 32 bytes from registers; where the address is a multiple of 32, in one access
__device__ __forceinline__ void tr_store32(void* p, const uint32_t* r) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               :: "l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}

__device__ __forceinline__ void tr_store32_any(void* p, const uint32_t* r, int wide) {
  if (wide) { tr_store32(p, r); return; }
  static_cast<uint4*>(p)[0] = make_uint4(r[0], r[1], r[2], r[3]);
  static_cast<uint4*>(p)[1] = make_uint4(r[4], r[5], r[6], r[7]);
}

// Where the CTA's even range of all key tiles begins: found by the whole CTA, left in *hd (shared); scratch: shared.
template <int F>
__device__ __forceinline__ void tr_find(const K16Pages& pg, const TrArgs& a, TrHead* hd, long long* scratch) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int T = tr_threads<F>();
  const int per = (pg.B + T - 1) / T, b0 = min(pg.B, tid * per), b1 = min(pg.B, b0 + per);
  auto units = [&](const TrSeq& s) {
    long long u = 0;
    for (int q0 = 0; q0 < s.n; q0 = tr_reach<F>(a, q0)) u += a.whole ? 1 : tr_tiles<F>(a, s.held, s.n, q0) + tr_extra<F>();
    return u * a.Hk;
  };
  long long mine = 0;
  TrSeq s0 = {0, 0, 0};                                // the thread's first sequence (its only one, up to as many as threads)
  if (b0 < b1) s0 = tr_seq(pg, a, b0);
  for (int b = b0; b < b1; ++b) mine += units(b == b0 ? s0 : tr_seq(pg, a, b));
  long long run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += v;
  }
  if (lane == 31) scratch[warp] = run;
  if (tid == 0) hd->units = 0;
  __syncthreads();
  long long front = 0, all = 0;
#pragma unroll
  for (int w = 0; w < T / 32; ++w) {
    if (w < warp) front += scratch[w];
    all += scratch[w];
  }
  const long long u0 = all * blockIdx.x / gridDim.x, u1 = all * (blockIdx.x + 1) / gridDim.x;
  long long at = front + run - mine;                   // units in front of this thread's sequences
  if (u0 < u1 && at <= u0 && u0 < at + mine) {
    for (int b = b0; b < b1; ++b) {
      const TrSeq s = b == b0 ? s0 : tr_seq(pg, a, b);
      const long long u = units(s);
      if (u0 >= at + u) { at += u; continue; }
      int rest_q0 = 0;
      long long rest = u0 - at;
      for (; rest_q0 < s.n; rest_q0 = tr_reach<F>(a, rest_q0)) {
        const long long x = (long long)(a.whole ? 1 : tr_tiles<F>(a, s.held, s.n, rest_q0) + tr_extra<F>()) * a.Hk;
        if (rest < x) break;
        rest -= x;
      }
      hd->b = b; hd->q0 = rest_q0; hd->n = s.n; hd->row0 = s.row0; hd->held = s.held;
      hd->T = tr_tiles<F>(a, s.held, s.n, rest_q0);
      const int extra = a.whole ? 0 : tr_extra<F>(), cost = a.whole ? 1 : hd->T + extra;
      hd->h = (int)(rest / cost);
      const int x = (int)(rest - (long long)hd->h * cost);
      hd->t = max(x - extra, 0);
      hd->units = max(u1 - u0 - max(extra - x, 0), 0ll);
      hd->first = u0;
      hd->all = all;
      break;
    }
  }
  __syncthreads();
}

// The kernel for up to kTrFewRows rows an item (attn_tree_rows.cu): launches it over `ranges` ranges.
cudaError_t launch_attn_tree_rows(const dl_ctx* ctx, const TrMaps& maps, const K16Pages& pg, const TrArgs& a, int ranges, cudaStream_t s);
bool attn_tree_rows_supported(const dl_ctx* ctx);

}  // namespace dl
