// Decode attention over a paged 4-bit K/V cache with grouped heads (an extension of Eq. 6; NOT in the paper).
//
// One new token per sequence: its G = H / Hkv query heads of a K/V head attend the rows the sequence's pages hold
// (kv4.cuh: value = s * code + z per 64 values) and the token's own k_t, v_t in bf16.  bf16 models, D = 64 or 128.
//
// Bound by the bytes of the cache: 18 D bytes per 16 rows and K/V head.  The codes are never turned into values:
//   scores   q . k = sum over groups of  s * (q . codes) + z * (sum of q over the group)
//   outputs  O     = sum over keys of (p s) codes + p z
// so the matrix instructions work on the codes themselves, and s and z are applied once per key and group.
// A code in bits 0-3 or 4-7 of a half word IS an fp16 number (a subnormal: code * 2^-24 or code * 2^-20), so eight codes
// become four operand registers of mma.sync m16n8k16 with one shift and four ANDs; the powers of two are taken out in q
// (an exact scaling by 1/16 of the dims concerned) and at the end.  (As e4m3 bytes, where a code is code * 2^-9, they
// would take one shift and two ANDs, but the 8-bit m16n8k32 is made of conversions and two 16-bit products on this GPU: an
// earlier form of the kernel took 364 instead of 250 instructions a tile with it.)  q is divided by a power of two into fp16's range (exact down to 2^-28 of a head's
// largest value).  P s is rounded to fp16 after multiplication by a power of two `fd` of its head and group of dims, which puts
// the largest P s that they have met so far at 2^9 .. 2^15 (2^-7 .. for values below 2^-110): 2^-11 of every P s down to 2^-23
// of that one, and no more than 2^-34 of it for any below, however the scores and the sizes of V's rows are spread.  (P alone is held relative to a maximum
// that lags by up to 2^8.  One power of two for all, following the largest s, takes 57.1 instead of 57.9 us for
// 4 x 100k rows and 43.4 instead of 45.2 us for 16 heads a K/V head on 16 x 20k; but a row of large values that nobody attends,
// or a leading score with a value of zero, then pushed the others out of fp16.)
// The query heads are the N side and 16 keys (scores) or 16 dims (outputs) the M side, so that up to 8 heads of a group
// cost one pass over the codes:
//   S^T[key][head] = K codes [16 keys][16 dims] x q^T          A straight from shared memory, B = q (registers)
//   O^T[dim][head] += V^T codes [16 dims][16 keys] x P^T       A straight from shared memory, B: P through movmatrix
// (An operand of V that keeps the high dims' bits above its own, their sum taken off at the end, is one operation less per
// word and 1 % faster, but sums 17 times as large lose too many bits on long rows: 0.0088 instead of 0.0018 of the outputs.)
// With one query head per K/V head the eight columns hold the same q, so that the four lanes of a row of the products can
// take one key each of a unit's four instead of all the same four: 230 instructions a tile where the general form takes 294
// (32 x 784 rows of 32 heads of 128: 36.9 -> 32.8 us).
//
// Work: the units (32 rows: two tiles) of all (sequence, K/V head) pairs in one line, cut into equal ranges, one per warp:
// every warp streams the same number of units whatever the lengths are, through its own ring (one bulk copy per
// tile).  A pair that lies within one range is finished there; the parts of the others go to scratch and are joined by a second
// kernel, in order and without atomics: the same call gives the same bits.  (Joined by the warp that delivers the last
// part, few parts took as long, and many, 100 and more a pair, four times as long as all the rest.)  Page numbers are fetched
// 16 units ahead, a tile per lane; the lane that holds a tile's number copies it.
#include <algorithm>

#include "kv4.cuh"
#include "pipeline.cuh"

namespace dl {

struct K4Args {
  const __nv_bfloat16* q; const __nv_bfloat16* k_t; const __nv_bfloat16* v_t;   // [B][H][D], [B][Hk][D]
  uint8_t* pool; PagesArg pg; const uint8_t* keep; __nv_bfloat16* out;
  float* partial; float* sums; DeviceStatus* status;
  int32_t H, Hk, G, grid_warps, stages;
  float scale_log2;
};

constexpr int kK4Warps = 4;              // warps per CTA
// CTAs per SM by blocks of 8 query heads: what their registers allow.  (16 heads take 70 ps a row and K/V head where 8 take 36: as
// much as two passes of 8 would, at half of their bytes.)
__host__ __device__ constexpr int k4_ctas(int nt) { return nt == 1 ? 3 : 2; }
constexpr int kK4Lag = 8;                // log2 units by which the maximum in use may lag
constexpr int kK4Unit = 32;              // rows of a unit: two tiles
constexpr int kK4MergeWarps = 16;        // most warps of a joining CTA

// Units after which a part's sums leave the matrix accumulators: those cut every addition off (at 2^-23 of the sum), so a
// sum of many positive terms comes out too small, in proportion to their number.  (600k rows, 8 heads: an error of 0.0040 of
// the outputs without, 0.0018 with this; 4 x 60-131k rows 57.6 -> 57.8 us, every 16 units 59.2.)
constexpr int kK4Flush = 32;
// floats a lane keeps of them: the accumulators, the maxima in use, the powers of two in use
template <int D> __host__ __device__ constexpr int k4_keep(int nt) { return nt * (D / 4 + 8); }
// P s times its power of two: where the largest goes when it passes the limit, the limit (half of fp16's), and the power of two
// to begin with, the most there is (times P, at most 2^kK4Lag, it is finite)
constexpr int kK4Put = 9, kK4Most = 15, kK4Begin = 119;
static_assert(kK4Begin + kK4Lag < 128, "0 * infinity");

// floats of a part: D sums per head, then the head's maximum and its sum of exponentials (16-byte steps)
template <int D> __host__ __device__ constexpr int k4_slot(int G) { return G * (D + 4); }

__device__ __forceinline__ int k4_rows(const PagesArg& p, int b) {
  return (int)min((long long)max(__ldg(p.len + b), 0), (long long)p.max_pages * (kKv4Rows << p.tile_shift));
}
// units of one K/V head of a sequence of n rows; an empty one counts 1, so that somebody writes its output
__device__ __forceinline__ int k4_units(int n) { return max(1, (n + kK4Unit - 1) / kK4Unit); }

// pre[b] = units in front of sequence b, pre[B] = all, rows[b] its rows; called by the whole CTA
__device__ __forceinline__ void k4_prefix(const PagesArg& p, int Hk, int* pre, int* rows, int* sums) {
  const int T = blockDim.x, per = (p.B + T - 1) / T, from = min(p.B, (int)threadIdx.x * per), to = min(p.B, from + per);
  int c = 0;
  for (int b = from; b < to; ++b) {
    const int n = k4_rows(p, b);
    rows[b] = n;
    c += k4_units(n) * Hk;
    pre[b + 1] = c;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int run = c;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += v;
  }
  if (lane == 31) sums[warp] = run;
  __syncthreads();
  int base = run - c;
  for (int w = 0; w < warp; ++w) base += sums[w];
  for (int b = from; b < to; ++b) pre[b + 1] += base;
  if (threadIdx.x == 0) pre[0] = 0;
  __syncthreads();
}
__device__ __forceinline__ int k4_find(const int* pre, int B, int u) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= u) lo = mid; else hi = mid - 1;
  }
  return lo;
}
// the line of `total` units as W ranges
__device__ __forceinline__ int k4_width(int total, int grid_warps) { return max(1, min(grid_warps, total)); }
__device__ __forceinline__ int k4_range(int w, int total, int W) { return (int)((long long)w * total / W); }
__device__ __forceinline__ int k4_owner(int u, int total, int W) { return (int)((((long long)u + 1) * W - 1) / total); }

__device__ __forceinline__ void k4_mma(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same into fresh accumulators
__device__ __forceinline__ void k4_mma_first(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t k4_transpose(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t k4_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float k4_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float k4_pow2(int e) { return __int_as_float((e + 127) << 23); }     // -126 <= e <= 127
__device__ __forceinline__ int k4_exponent(float x) { return (int)((uint32_t)__float_as_int(x) >> 23) - 127; }   // x > 0
// the larger ones of two pairs of fp16 values; a NaN loses
__device__ __forceinline__ uint32_t k4_max2(uint32_t x, uint32_t y) {
  uint32_t r;
  asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}
// one of two fp16 values, neither below zero, is 2^kK4Most or more
__device__ __forceinline__ bool k4_beyond(uint32_t x) {
  constexpr uint32_t kAdd = 0x8000u - ((kK4Most + 15u) << 10);      // carries into the sign from there on
  return ((x + (kAdd | kAdd << 16)) & 0x80008000u) != 0u;
}
__device__ __forceinline__ uint32_t k4_lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 k4_lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}

// 16 values of a query or key row from dim `d` on, as floats (zeros where !on)
__device__ __forceinline__ void k4_load16(const __nv_bfloat16* p, bool on, float* x) {
  uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
  if (on) { a = __ldg(reinterpret_cast<const uint4*>(p)); b = __ldg(reinterpret_cast<const uint4*>(p) + 1); }
  const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) { x[2 * i] = bf16lo(u[i]); x[2 * i + 1] = bf16hi(u[i]); }
}

template <int D, int NT, bool kOne>                               // NT: blocks of 8 query heads; kOne: one head per K/V head
__global__ void __launch_bounds__(kK4Warps * 32, k4_ctas(NT))
attn_decode_kv4_kernel(const K4Args a) {
  using F = Kv4<D>;
  constexpr int NG = F::NG;
  constexpr int NC = kOne ? 1 : 2, KL = kOne ? 1 : 4;             // heads a lane keeps of a block; keys of a unit
  extern __shared__ __align__(128) char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, j = lane & 3;
  const int NS = a.stages;
  char* ring = smem + (size_t)warp * NS * (2 * F::TILE);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + (size_t)kK4Warps * NS * (2 * F::TILE)) + warp * NS;
  int* pre = reinterpret_cast<int*>(smem + (size_t)kK4Warps * NS * (2 * F::TILE + 8));
  int* rows = pre + a.pg.B + 1;
  __shared__ int sh_sums[kK4Warps];
  __shared__ int sh_abort;
  volatile int* abort_flag = &sh_abort;
  chained_go();                                                   // the joining kernel may come up
  if (tid == 0) sh_abort = 0;
  if (lane == 0) {
    for (int s = 0; s < NS; ++s) mbar_init(smem_u32(&bars[s]), 1);
    fence_mbar_init();
  }
  k4_prefix(a.pg, a.Hk, pre, rows, sh_sums);                      // (its barriers also publish the above)
  const int total = pre[a.pg.B], W = k4_width(total, a.grid_warps);
  const int gw = warp * gridDim.x + blockIdx.x;                   // few ranges go to as many SMs as there are
  if (gw >= W) return;
  const int u0 = k4_range(gw, total, W), u1 = k4_range(gw + 1, total, W);

  // ---- page numbers: lane 2 i + h holds that of tile h of unit base + i, for this block of 16 units and (requested
  //      ahead) the next
  int nx_page = -1, nx_b = -1, nx_hk = 0, nx_t = 0;               // nx_b < 0: nothing to copy
  auto request = [&](int base) {
    const int u = base + (lane >> 1);
    nx_b = -1;
    if (u < u1) {
      const int b = k4_find(pre, a.pg.B, u), rem = u - pre[b], units = k4_units(rows[b]);
      nx_hk = rem / units;
      nx_t = 2 * (rem - nx_hk * units) + (lane & 1);
      if (nx_t * kKv4Rows < rows[b]) {
        nx_b = b;
        nx_page = __ldg(a.pg.table + (size_t)b * a.pg.max_pages + (nx_t >> a.pg.tile_shift));
      }
    }
  };
  auto resolve = [&]() {
    int idx = -1;
    if (nx_b >= 0) {
      idx = kv4_tile_index(a.pg, nx_page, a.Hk, nx_hk, nx_t);
      if (idx < 0) report_status(a.status, DL_ERR_INVALID_ARG, nx_b);
    }
    return idx;
  };
  request(u0);
  int cur_idx = resolve(), p_at = 0;                              // p_at: place of the next unit in this block
  uint32_t here = 0;                                              // bits 2 s, 2 s + 1: which tiles of slot s were fetched
  int p_u = u0, p_slot = 0;
  auto produce = [&]() {
    if (p_at == 16) {
      cur_idx = resolve();
      p_at = 0;
      request(p_u + 16);
    }
    const bool mine = (lane >> 1) == p_at && cur_idx >= 0;
    const uint32_t got = (__ballot_sync(0xffffffffu, mine) >> (2 * p_at)) & 3u;
    const uint32_t bar = smem_u32(&bars[p_slot]);
    if (lane == 0) {
      if (got) mbar_expect_tx(bar, got == 3u ? 2 * F::TILE : F::TILE);
      else mbar_arrive(bar);
    }
    __syncwarp();
    if (mine)
      bulk_g2s(smem_u32(ring + (size_t)(2 * p_slot + (lane & 1)) * F::TILE), a.pool + (long long)cur_idx * F::TILE, F::TILE, bar);
    here = (here & ~(3u << (2 * p_slot))) | (got << (2 * p_slot));
    ++p_u;
    ++p_at;
    if (++p_slot == NS) p_slot = 0;
  };
  // One unit each first, the rest of the ring behind the query's preparation: asked for all at once, the rings of the
  // whole GPU take 5 us to fill and the first units arrive in the middle of that.
  produce();
  request(u0 + 16);

  // ---- where the consumer is
  int b = k4_find(pre, a.pg.B, u0);
  int units = k4_units(rows[b]), hk = (u0 - pre[b]) / units, t = (u0 - pre[b]) - hk * units;
  int slot = 0, phase = 0;
  bool gave_up = false;                                           // a wait ran out (the lane's own, until the warp has agreed)
  for (int u = u0; u < u1;) {
    // ================ one (sequence, K/V head), or the part of it that lies in this range
    const int n = rows[b], seg0 = u - t, seg1 = seg0 + units, part_end = min(seg1, u1);
    uint32_t qb[NT][NG][4][2];                                    // B operand: head r of block nt, 16 dims per step
    float qs[NT][NG][NC], fq[NT][NC], se[NT][NC];                   // of heads 2j, 2j + 1: sum of q * scale, score factor, own score
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const bool on = kOne || nt * 8 + r < a.G;
      const __nv_bfloat16* qp = a.q + ((size_t)b * a.H + hk * a.G + (kOne ? 0 : nt * 8 + r)) * D;
      float x[NG][16], dot = 0.f, sum[NG], mx = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float y[16];
        k4_load16(qp + 64 * g + 16 * j, on, x[g]);
        k4_load16(a.k_t + ((size_t)b * a.Hk + hk) * D + 64 * g + 16 * j, true, y);
        sum[g] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          dot = fmaf(x[g][i], y[i], dot);
          sum[g] += x[g][i];
          mx = fmaxf(mx, fabsf(x[g][i]));
        }
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
#pragma unroll
        for (int g = 0; g < NG; ++g) sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], o);
      }
      const int e = max(-100, min(110, (int)(__float_as_uint(mx) >> 23) - 127));   // |q| < 2^(e + 1)
      const float down = k4_pow2(13 - e), down16 = down * 0.0625f;
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const float* y = x[g] + 8 * w;
          qb[nt][g][2 * w][0] = k4_f16x2(y[0] * down, y[4] * down);
          qb[nt][g][2 * w][1] = k4_f16x2(y[1] * down16, y[5] * down16);
          qb[nt][g][2 * w + 1][0] = k4_f16x2(y[2] * down, y[6] * down);
          qb[nt][g][2 * w + 1][1] = k4_f16x2(y[3] * down16, y[7] * down16);
        }
      const float fr = a.scale_log2 * k4_pow2(e + 11);            // 2^24 of the codes, 2^(e - 13) of q
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int from = (2 * j + c) * 4;
        fq[nt][c] = __shfl_sync(0xffffffffu, fr, from);
        se[nt][c] = __shfl_sync(0xffffffffu, dot, from) * a.scale_log2;
#pragma unroll
        for (int g = 0; g < NG; ++g) qs[nt][g][c] = __shfl_sync(0xffffffffu, sum[g], from) * a.scale_log2;
      }
    }
    if (u == u0)
      for (int i = 1; i < NS && p_u < u1; ++i) produce();
    // ---- Eq. 6's append, by the warp that has the pair's first unit: lanes 0 .. D/16-1 hold k_t, the next D/16 v_t
    if (t == 0 && a.keep != nullptr && a.keep[b] != 0) {
      constexpr int LR = D / 16;
      const int l = lane % LR;
      const bool is_v = lane >= LR, on = lane < 2 * LR;
      const uint4* from = reinterpret_cast<const uint4*>((is_v ? a.v_t : a.k_t) + ((size_t)b * a.Hk + hk) * D) + 2 * l;
      const uint4 lo = __ldg(from), hi = __ldg(from + 1);
      const uint32_t raw[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      uint32_t word;
      const uint2 code = kv4_quantise16(raw, word);
      const int pi = n >> (a.pg.tile_shift + 4);
      const int idx = pi < a.pg.max_pages
                          ? kv4_tile_index(a.pg, __ldg(a.pg.table + (size_t)b * a.pg.max_pages + pi), a.Hk, hk, n >> 4) : -1;
      if (idx < 0) {
        if (lane == 0 && hk == 0) report_status(a.status, DL_ERR_CAPACITY, b);
      } else if (on && DL_IN_BOUNDS(a.status, KID_DECODE_KV4, idx, ((long long)a.pg.n_pages * a.Hk) << a.pg.tile_shift)) {
        kv4_store16(a.pool + (long long)idx * F::TILE, kv4_row<D>(n & 15, is_v), l, is_v, code, word);
      }
    }

    float m[NT][NC], l_run[NT][NC], zacc[NT][NG][NC], acc[NT][NG][4][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        m[nt][c] = l_run[nt][c] = 0.f;                            // (not a maximum yet: see `seen`)
#pragma unroll
        for (int g = 0; g < NG; ++g) zacc[nt][g][c] = 0.f;
      }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[nt][g][i][0] = acc[nt][g][i][1] = acc[nt][g][i][2] = acc[nt][g][i][3] = 0.f;
      }
    }
    uint32_t seen = 0;                                            // heads (bit 2 nt + c) whose maximum in use has been set
    float fd[NT][NG][NC];                                         // P s is held as P s fd, a power of two
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int c = 0; c < NC; ++c) fd[nt][g][c] = k4_pow2(kK4Begin);

    // ================ units.  The products of the next unit's keys stand beside the current unit's exponentials and values, so
    // that a warp has two independent chains to work on.
    float d[2][NT][NG][4], vs[KL][NG], vz[KL][NG], s[NT][KL][NC];
    auto key_products = [&](uint32_t unit) {                      // codes times query: lane's keys r and r + 8 of both tiles
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const uint32_t ka = unit + h * F::TILE + kv4_k_off<D>(r, g) + 8 * j;
          const uint2 w0 = k4_lds64(ka), w1 = k4_lds64(ka + 8 * F::RB);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t x = w ? w0.y : w0.x, y = w ? w1.y : w1.x, x8 = x >> 8, y8 = y >> 8;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              if (w == 0) k4_mma_first(d[h][nt][g], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, qb[nt][g][0][0], qb[nt][g][0][1]);
              else k4_mma(d[h][nt][g], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, qb[nt][g][2][0], qb[nt][g][2][1]);
              k4_mma(d[h][nt][g], x8 & 0x000F000Fu, y8 & 0x000F000Fu, x8 & 0x00F000F0u, y8 & 0x00F000F0u, qb[nt][g][2 * w + 1][0], qb[nt][g][2 * w + 1][1]);
            }
          }
        }
    };
    // Scores less the maximum in use, from the products and the words of the lane's keys (index 2 h + i: key r + 8 i of
    // tile h; with one head every column of the products is the same, and a lane keeps the key whose index is j); nr: rows of the unit that are there, got: tiles that are.
    auto scores = [&](uint32_t unit, int nr, uint32_t got) {
#pragma unroll
      for (int k = 0; k < KL; ++k) {
        uint32_t kw[NG], vw[NG];
        const int kk = kOne ? j : k;
        const uint32_t at = unit + (kk >> 1) * F::TILE + (r + 8 * (kk & 1)) * 4 * NG;
        if (NG == 2) {
          const uint2 x = k4_lds64(at + F::KM), y = k4_lds64(at + F::VM);
          kw[0] = x.x; kw[NG - 1] = x.y; vw[0] = y.x; vw[NG - 1] = y.y;
        } else {
          kw[0] = k4_lds32(at + F::KM); vw[0] = k4_lds32(at + F::VM);
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) { vs[k][g] = bf16lo(vw[g]); vz[k][g] = bf16hi(vw[g]); }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            float dot = 0.f, off = -m[nt][c];
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              const float x = kOne ? ((j & 1) ? (j >> 1 ? d[1][nt][g][2] : d[0][nt][g][2]) : (j >> 1 ? d[1][nt][g][0] : d[0][nt][g][0]))
                                   : d[k >> 1][nt][g][2 * (k & 1) + c];
              dot = fmaf(bf16lo(kw[g]), x, dot);
              off = fmaf(bf16hi(kw[g]), qs[nt][g][c], off);
            }
            s[nt][k][c] = fmaf(fq[nt][c], dot, off);
          }
      }
      if (nr < kK4Unit || got != 3u) {
        // the last unit of a sequence, or one with a page missing: whatever stands in rows that are not there counts nothing
#pragma unroll
        for (int k = 0; k < KL; ++k) {
          const int kk = kOne ? j : k;
          if (16 * (kk >> 1) + r + 8 * (kk & 1) >= nr || !((got >> (kk >> 1)) & 1u)) {
#pragma unroll
            for (int g = 0; g < NG; ++g) vs[k][g] = vz[k][g] = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int c = 0; c < NC; ++c) s[nt][k][c] = -INFINITY;
          }
        }
      }
    };
    // Adds to the accumulators what has been kept of them (rounded sums), with the maxima and powers of two it was kept at
    // brought to those in use; `out`: keeps the result and clears the accumulators.
    auto flush = [&](bool in, bool out) {
      float4* keep = reinterpret_cast<float4*>(a.sums + (size_t)gw * (32 * k4_keep<D>(NT))) + lane;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float4* mine = keep + nt * 8 * k4_keep<D>(1);
        float4 was_m = make_float4(0.f, 0.f, 0.f, 0.f), was_fd = was_m;
        if (in) {
          was_m = __ldcg(mine + 32 * 4 * NG);
          was_fd = __ldcg(mine + 32 * (4 * NG + 1));
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          float f[2] = {0.f, 0.f};
          if (in) {
            // (a power of two goes up by less than its maximum does; a head without a score had sums of zero, whatever its
            // maximum)
            const int e0 = k4_exponent(fd[nt][g][0]) - k4_exponent(g == 0 ? was_fd.x : was_fd.y);
            const int e1 = k4_exponent(fd[nt][g][NC - 1]) - k4_exponent(g == 0 ? was_fd.z : was_fd.w);
            f[0] = fminf(1.f, k4_exp2(was_m.x - m[nt][0] + (float)e0));
            f[1] = kOne ? f[0] : fminf(1.f, k4_exp2(was_m.y - m[nt][NC - 1] + (float)e1));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float* x = acc[nt][g][i];
            if (in) {
              const float4 y = __ldcg(mine + 32 * (4 * g + i));
              x[0] = fmaf(y.x, f[0], x[0]); x[1] = fmaf(y.y, f[1], x[1]);
              x[2] = fmaf(y.z, f[0], x[2]); x[3] = fmaf(y.w, f[1], x[3]);
            }
            if (out) {
              __stcg(mine + 32 * (4 * g + i), make_float4(x[0], x[1], x[2], x[3]));
              x[0] = x[1] = x[2] = x[3] = 0.f;
            }
          }
        }
        if (out) {
          __stcg(mine + 32 * 4 * NG, make_float4(m[nt][0], m[nt][NC - 1], 0.f, 0.f));
          __stcg(mine + 32 * (4 * NG + 1), make_float4(fd[nt][0][0], fd[nt][NG - 1][0], fd[nt][0][NC - 1], fd[nt][NG - 1][NC - 1]));
        }
      }
    };
    auto arrived = [&](int sl, int ph) {                          // false: the wait ran out
      return mbar_try_wait(smem_u32(&bars[sl]), ph) || mbar_wait(smem_u32(&bars[sl]), ph, abort_flag);
    };
    auto slot_addr = [&](int sl) { return smem_u32(ring + (size_t)sl * (2 * F::TILE)); };
    // (After a wait that ran out the products are of whatever the slot holds, up to the vote.)
    gave_up = !arrived(slot, phase);
    key_products(slot_addr(slot));
    scores(slot_addr(slot), n - t * kK4Unit, (here >> (2 * slot)) & 3u);
    for (;; ++u, ++t) {
      int next = slot + 1, next_phase = phase;
      if (next == NS) { next = 0; next_phase ^= 1; }
      const bool more = u + 1 < part_end;
      if (more && !arrived(next, next_phase)) gave_up = true;
      const uint32_t unit = slot_addr(slot), next_unit = slot_addr(more ? next : slot);
      auto most = [](const float* x, int step) {                  // over the lane's keys
        return kOne ? x[0] : fmaxf(fmaxf(x[0], x[(KL > 1) * step]), fmaxf(x[(KL > 1) * 2 * step], x[(KL > 1) * 3 * step]));
      };
      // P, and P s in fp16: of heads 2j and 2j + 1 for each key and group, with one head of both groups
      float p[NT][KL][NC];
      uint32_t y[NT][kOne ? 1 : NG][KL];
      auto weigh = [&] {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < KL; ++k)
#pragma unroll
            for (int c = 0; c < NC; ++c) p[nt][k][c] = k4_exp2(s[nt][k][c]);
      };
      auto products = [&] {                                       // returns the largest two
        uint32_t top = 0u;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int g = 0; g < (kOne ? 1 : NG); ++g)
#pragma unroll
            for (int k = 0; k < KL; ++k) {
              y[nt][g][k] = kOne ? k4_f16x2(p[nt][k][0] * fd[nt][0][0] * vs[k][0], NG == 2 ? p[nt][k][0] * fd[nt][NG - 1][0] * vs[k][NG - 1] : 0.f)
                                 : k4_f16x2(p[nt][k][0] * fd[nt][g][0] * vs[k][g], p[nt][k][NC - 1] * fd[nt][g][NC - 1] * vs[k][g]);
              top = k4_max2(top, y[nt][g][k]);
            }
        return top;
      };
      weigh();
      bool raise = gave_up || seen != (kOne ? 1u : (1u << (2 * NT)) - 1u) || k4_beyond(products());
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          raise |= most(&s[nt][0][c], NC) > (float)kK4Lag;
      if (__any_sync(0xffffffffu, raise)) {
        if (!warp_agreed(!gave_up)) { gave_up = true; break; }
        // rare: the maxima in use go up to what has been seen, and powers of two come down from what they make too large
        float fix[NT][NG][NC];                                    // what that makes of the accumulators
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            float mx = most(&s[nt][0][c], NC);
#pragma unroll
            for (int o = kOne ? 1 : 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            // up by mx (the first time: to it, wherever it is); a head without a finite score yet stays
            const bool known = (seen >> (2 * nt + c)) & 1u, finite = mx > -INFINITY && mx < INFINITY;
            const float by = finite && (!known || mx > 0.f) ? mx : 0.f, up = known ? by : 0.f;
            const float corr = k4_exp2(-up);
            if (finite) seen |= 1u << (2 * nt + c);
            m[nt][c] += by;
#pragma unroll
            for (int k = 0; k < KL; ++k) s[nt][k][c] -= by;
            l_run[nt][c] *= corr;
            // the weights met so far are that much smaller from now on: their power of two makes up for it as far as it may, so
            // that their likes keep their bits, and the sums take the rest
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              zacc[nt][g][c] *= corr;
              const int e = k4_exponent(fd[nt][g][c]), go = min((int)fminf(up, 250.f), kK4Begin - e);
              fix[nt][g][c] = k4_exp2((float)go - up);
              fd[nt][g][c] = k4_pow2(e + go);
            }
          }
        weigh();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int g = 0; g < NG; ++g) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              float w = 0.f;                                      // the largest P s (a NaN is none)
#pragma unroll
              for (int k = 0; k < KL; ++k) w = fmaxf(w, p[nt][k][c] * vs[k][g]);
#pragma unroll
              for (int o = kOne ? 1 : 4; o < 32; o <<= 1) w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, o));
              // (an infinite one that is not p's fault is 2^128 and a little more, which fits, too)
              const int e = k4_exponent(fd[nt][g][c]), to = w * fd[nt][g][c] >= k4_pow2(kK4Most) ? kK4Put - k4_exponent(w) : e;
              fix[nt][g][c] *= k4_pow2(max(-126, to - e));
              fd[nt][g][c] = k4_pow2(to);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              acc[nt][g][i][0] *= fix[nt][g][0];
              acc[nt][g][i][1] *= fix[nt][g][NC - 1];             // (with one head all columns are its own)
              acc[nt][g][i][2] *= fix[nt][g][0];
              acc[nt][g][i][3] *= fix[nt][g][NC - 1];
            }
          }
        products();
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < KL; ++k)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            l_run[nt][c] += p[nt][k][c];
#pragma unroll
            for (int g = 0; g < NG; ++g) zacc[nt][g][c] = fmaf(p[nt][k][c], vz[k][g], zacc[nt][g][c]);
          }
      // ---- O^T += V^T (P s)^T tile by tile: lane's row pairs j and j + 4, its dims 64 g + 8 r .. + 7
      // With one head, the lanes of row r hold P s of keys 0 r, r + 8, 16 + r and 24 + r, one pair (the two groups) each, in
      // columns 4 h + 2 i + g.  For tile h the columns of the other tile are made zero; what the rest of them add up to
      // nobody reads: the sums of group g are in columns g (tile 0) and 4 + g (tile 1).
      uint32_t one[2] = {0u, 0u};
      if (kOne) {
        one[0] = k4_transpose(y[0][0][0]);
        one[1] = k4_transpose(__shfl_xor_sync(0xffffffffu, y[0][0][0], 1));
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t pb[NT][NG][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              pb[nt][g][i] = kOne ? ((r >> 2) == h ? one[i] : 0u) : k4_transpose(y[nt][g % (kOne ? 1 : NG)][(2 * h + i) % KL]);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const uint32_t va = unit + h * F::TILE;
          const uint2 wx = k4_lds64(va + kv4_v_off<D>(j, 64 * g + 8 * r)), wy = k4_lds64(va + kv4_v_off<D>(j + 4, 64 * g + 8 * r));
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t x = w ? wx.y : wx.x, y = w ? wy.y : wy.x, x8 = x >> 8, y8 = y >> 8;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              k4_mma(acc[nt][g][2 * w], x & 0x000F000Fu, x & 0x00F000F0u, y & 0x000F000Fu, y & 0x00F000F0u, pb[nt][g][0], pb[nt][g][1]);
              k4_mma(acc[nt][g][2 * w + 1], x8 & 0x000F000Fu, x8 & 0x00F000F0u, y8 & 0x000F000Fu, y8 & 0x00F000F0u, pb[nt][g][0], pb[nt][g][1]);
            }
          }
        }
      }
      const int done = u + 1 - max(seg0, u0);                     // units of this part
      if (done % kK4Flush == 0 && more) flush(done > kK4Flush, true);
      // (without a next unit these are products nobody reads)
      key_products(next_unit);
      __syncwarp();
      if (p_u < u1) produce();
      slot = next;
      phase = next_phase;
      if (!more) { ++u; ++t; break; }
      scores(next_unit, n - (t + 1) * kK4Unit, (here >> (2 * next)) & 3u);
    }
    if (gave_up) break;                                           // (the whole warp)

    // ================ finish the part
    if (u - max(seg0, u0) > kK4Flush) flush(true, false);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int o = kOne ? 1 : 4; o < 32; o <<= 1) {
          l_run[nt][c] += __shfl_xor_sync(0xffffffffu, l_run[nt][c], o);
#pragma unroll
          for (int g = 0; g < NG; ++g) zacc[nt][g][c] += __shfl_xor_sync(0xffffffffu, zacc[nt][g][c], o);
        }
        if (kOne) {
          // both tiles' columns, in one
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              acc[nt][g][i][0] = acc[nt][g][i][g] + __shfl_xor_sync(0xffffffffu, acc[nt][g][i][g], 2);
              acc[nt][g][i][2] = acc[nt][g][i][2 + g] + __shfl_xor_sync(0xffffffffu, acc[nt][g][i][2 + g], 2);
            }
        }
        const int head = nt * 8 + 2 * j + c;
        if (head >= a.G) continue;                                // (after the shuffles of this pair)
        const float top = l_run[nt][c] == 0.f ? -INFINITY : m[nt][c];   // nothing attended: no maximum
        const bool whole = seg0 >= u0 && seg1 <= u1;
        // this lane's dims 64 g + 8 r + 0 .. 7 of the head
        float o[NG][8];
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float up = k4_pow2(-k4_exponent(fd[nt][g][c]));
            o[g][2 * i] = fmaf(acc[nt][g][i][c] * 16777216.f, up, zacc[nt][g][c]);
            o[g][2 * i + 1] = fmaf(acc[nt][g][i][2 + c] * 1048576.f, up, zacc[nt][g][c]);
          }
        if (whole) {
          const float mine = se[nt][c], M = fmaxf(top, mine);
          const float wc = top == -INFINITY ? 0.f : k4_exp2(top - M), we = k4_exp2(mine - M);
          const float inv = 1.f / fmaf(l_run[nt][c], wc, we);
          const __nv_bfloat16* vt = a.v_t + ((size_t)b * a.Hk + hk) * D;
          const size_t at = ((size_t)b * a.H + hk * a.G + head) * D;
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const uint4 vw = __ldg(reinterpret_cast<const uint4*>(vt + 64 * g + 8 * r));
            const uint32_t v[4] = {vw.x, vw.y, vw.z, vw.w};
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const __nv_bfloat162 y = __floats2bfloat162_rn(fmaf(o[g][2 * i], wc, we * bf16lo(v[i])) * inv,
                                                             fmaf(o[g][2 * i + 1], wc, we * bf16hi(v[i])) * inv);
              w[i] = *reinterpret_cast<const uint32_t*>(&y);
            }
            if (DL_IN_BOUNDS(a.status, KID_DECODE_KV4, at + 64 * g + 8 * r + 7, (size_t)a.pg.B * a.H * D))
              *reinterpret_cast<uint4*>(a.out + at + 64 * g + 8 * r) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else {
          // slot 0 of a range: the pair that began before it; slot 1: the one that goes on behind it
          float* pp = a.partial + ((size_t)gw * 2 + (seg0 < u0 ? 0 : 1)) * k4_slot<D>(a.G) + (size_t)head * (D + 4);
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            *reinterpret_cast<float4*>(pp + 64 * g + 8 * r) = make_float4(o[g][0], o[g][1], o[g][2], o[g][3]);
            *reinterpret_cast<float4*>(pp + 64 * g + 8 * r + 4) = make_float4(o[g][4], o[g][5], o[g][6], o[g][7]);
          }
          if (r == 0) { pp[D] = top; pp[D + 1] = l_run[nt][c]; }
        }
      }
    if (t == units) {
      t = 0;
      if (++hk == a.Hk) {
        hk = 0;
        if (++b < a.pg.B) units = k4_units(rows[b]);
      }
    }
  }
  if (gave_up) {
    if (lane == 0) report_status(a.status, DL_ERR_TIMEOUT, blockIdx.x);
    // copies still in flight must land before the CTA's shared memory goes: the last NS tiles requested
    for (int v = max(u0, p_u - NS); v < p_u; ++v)
      for (int i = 0; i < kSpinLimit && !mbar_try_wait(smem_u32(&bars[(v - u0) % NS]), ((v - u0) / NS) & 1); ++i) __nanosleep(40);
  }
}

// Joins the parts of a pair that several ranges share: one CTA per query head, parts dealt to its warps in order, four
// dims per lane.
template <int D>
__global__ void __launch_bounds__(kK4MergeWarps * 32)
attn_merge_kv4_kernel(const K4Args a) {
  constexpr int PL = D / 32;                                      // dims per lane
  const int NW = blockDim.x >> 5;
  extern __shared__ __align__(128) char smem[];
  int* pre = reinterpret_cast<int*>(smem);
  int* rows = pre + a.pg.B + 1;
  __shared__ int sh_sums[kK4MergeWarps];
  __shared__ float sh_o[kK4MergeWarps][D], sh_l[kK4MergeWarps], sh_m[kK4MergeWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.x / a.H, head = blockIdx.x - b * a.H, hk = head / a.G, hg = head - hk * a.G;
  k4_prefix(a.pg, a.Hk, pre, rows, sh_sums);
  const int total = pre[a.pg.B], W = k4_width(total, a.grid_warps);
  const int units = k4_units(rows[b]), s0 = pre[b] + hk * units;
  const int first = k4_owner(s0, total, W), last = k4_owner(s0 + units - 1, total, W);
  if (first == last) {
    // this grid must not retire before its predecessor has: what follows in the stream relies on both
    chained_wait();
    return;
  }
  // the token's own score (every warp for itself)
  const __nv_bfloat16* qp = a.q + ((size_t)b * a.H + head) * D + lane * PL;
  const __nv_bfloat16* kp = a.k_t + ((size_t)b * a.Hk + hk) * D + lane * PL;
  float own = 0.f;
#pragma unroll
  for (int i = 0; i < PL; ++i) own = fmaf(__bfloat162float(qp[i]), __bfloat162float(kp[i]), own);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) own += __shfl_xor_sync(0xffffffffu, own, o);
  own *= a.scale_log2;
  chained_wait();                                                 // the parts have been written from here on
  const int first_slot = k4_range(first, total, W) <= s0 ? 1 : 0; // the pair begins inside that range
  auto part = [&](int w) {
    return a.partial + ((size_t)w * 2 + (w == first ? first_slot : 0)) * k4_slot<D>(a.G) + (size_t)hg * (D + 4);
  };
  float M = -INFINITY, o[PL], l = 0.f;                            // of this warp's parts
#pragma unroll
  for (int i = 0; i < PL; ++i) o[i] = 0.f;
  constexpr int NB = 5;                                           // parts in flight
  for (int w0 = first + warp; w0 <= last; w0 += NB * NW) {
    float mw[NB], lw[NB], x[NB][PL], top = M;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int w = w0 + k * NW;
      mw[k] = -INFINITY;
      lw[k] = 0.f;
#pragma unroll
      for (int i = 0; i < PL; ++i) x[k][i] = 0.f;
      if (w <= last) {
        const float* pp = part(w);
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(pp + D));
        mw[k] = ml.x;
        lw[k] = ml.y;
        if (PL == 4) {
          const float4 y = __ldcg(reinterpret_cast<const float4*>(pp + lane * PL));
          x[k][0] = y.x; x[k][1] = y.y; x[k][PL - 2] = y.z; x[k][PL - 1] = y.w;
        } else {
          const float2 y = __ldcg(reinterpret_cast<const float2*>(pp + lane * PL));
          x[k][0] = y.x; x[k][1] = y.y;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < NB; ++k) top = fmaxf(top, mw[k]);
    const float corr = M == -INFINITY ? 0.f : k4_exp2(M - top);
    M = top;
    l *= corr;
#pragma unroll
    for (int i = 0; i < PL; ++i) o[i] *= corr;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const float wt = mw[k] == -INFINITY ? 0.f : k4_exp2(mw[k] - M);
      l = fmaf(lw[k], wt, l);
#pragma unroll
      for (int i = 0; i < PL; ++i) o[i] = fmaf(x[k][i], wt, o[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < PL; ++i) sh_o[warp][lane * PL + i] = o[i];
  if (lane == 0) { sh_l[warp] = l; sh_m[warp] = M; }
  __syncthreads();
  const int dim = threadIdx.x;
  if (dim < D) {
    float top = own;
    for (int w = 0; w < NW; ++w) top = fmaxf(top, sh_m[w]);
    const float we = k4_exp2(own - top);
    float num = we * __bfloat162float(a.v_t[((size_t)b * a.Hk + hk) * D + dim]), den = we;
    for (int w = 0; w < NW; ++w) {
      const float wt = sh_m[w] == -INFINITY ? 0.f : k4_exp2(sh_m[w] - top);
      num = fmaf(sh_o[w][dim], wt, num);
      den = fmaf(sh_l[w], wt, den);
    }
    const size_t at = ((size_t)b * a.H + head) * D + dim;
    if (DL_IN_BOUNDS(a.status, KID_DECODE_KV4, at, (size_t)a.pg.B * a.H * D)) a.out[at] = __float2bfloat16_rn(num / den);
  }
}

template <int D, int NT, bool kOne>
static cudaError_t k4_launch(const dl_ctx* ctx, K4Args& a, cudaStream_t s) {
  constexpr int kCtas = k4_ctas(NT);
  const size_t pre_bytes = (size_t)(2 * a.pg.B + 1) * sizeof(int);
  const int per_cta = (ctx->smem_optin + 1024) / kCtas - 1024;
  int ns = (int)((per_cta - (int)pre_bytes - 256) / (kK4Warps * (2 * Kv4<D>::TILE + 8)));
  ns = std::min(ns, 8);
  if (ns < 2) return cudaErrorInvalidConfiguration;
  a.stages = ns;
  const size_t smem = (size_t)kK4Warps * ns * (2 * Kv4<D>::TILE + 8) + pre_bytes;
  auto kernel = attn_decode_kv4_kernel<D, NT, kOne>;
  cudaError_t e = cudaSuccess;
  static int attr_set[64];                                        // (all calls ask for the same: two threads may)
  if (!attr_set[ctx->device & 63]) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, per_cta - 256);
    if (e != cudaSuccess) return e;
    attr_set[ctx->device & 63] = 1;
  }
  const int grid = ctx->sm_count * kCtas;
  a.grid_warps = grid * kK4Warps;
  kernel<<<grid, kK4Warps * 32, smem, s>>>(a);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  // 16 warps where a pair has 32 parts or more, else four (pairs share the ranges evenly when there are few of them)
  const int threads = a.grid_warps / ((long long)a.pg.B * a.Hk) >= 32 ? kK4MergeWarps * 32 : 128;
  return launch_chained(attn_merge_kv4_kernel<D>, dim3(a.pg.B * a.H), dim3(threads), pre_bytes, s, a);
}

// floats of scratch: two parts for each range; a warp's kept sums
static int64_t k4_part_floats(int32_t sm_count, const dl_model_desc& d) {
  const int64_t G = std::min(d.n_heads, 16);
  return std::max((int64_t)sm_count * k4_ctas(1) * kK4Warps * 2 * std::min<int64_t>(G, 8),
                  (int64_t)sm_count * k4_ctas(2) * kK4Warps * 2 * G) * (d.head_dim + 4);
}
int64_t kv4_scratch_floats(int32_t sm_count, const dl_model_desc& d) {
  return k4_part_floats(sm_count, d) + (int64_t)sm_count * kK4Warps * 32 * std::max(k4_ctas(1) * k4_keep<128>(1), k4_ctas(2) * k4_keep<128>(2));
}

cudaError_t launch_attn_decode_kv4(const dl_ctx* ctx, const dl_pages* p, int32_t Hk, void* pool, const void* q,
                                   const void* k_t, const void* v_t, const uint8_t* keep, float scale, void* out,
                                   cudaStream_t s) {
  const dl_model_desc& d = ctx->desc;
  K4Args a;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k_t = static_cast<const __nv_bfloat16*>(k_t);
  a.v_t = static_cast<const __nv_bfloat16*>(v_t);
  a.pool = static_cast<uint8_t*>(pool);
  a.pg = pages_arg(p);
  a.keep = keep;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.partial = ctx->ws.kv4_partial;
  a.sums = a.partial + k4_part_floats(ctx->sm_count, d);          // (parts are multiples of 16 bytes)
  a.status = ctx->ws.status;
  a.H = d.n_heads; a.Hk = Hk; a.G = d.n_heads / Hk;
  a.scale_log2 = scale * 1.4426950408889634f;
  if (a.G == 1) return d.head_dim == 128 ? k4_launch<128, 1, true>(ctx, a, s) : k4_launch<64, 1, true>(ctx, a, s);
  if (d.head_dim == 128) return a.G <= 8 ? k4_launch<128, 1, false>(ctx, a, s) : k4_launch<128, 2, false>(ctx, a, s);
  return a.G <= 8 ? k4_launch<64, 1, false>(ctx, a, s) : k4_launch<64, 2, false>(ctx, a, s);
}

}  // namespace dl
