// Verification of drafted trees against the target's distributions (rejection sampling along the tree, or greedily), with given
// random numbers.  An extension, not in the paper.
//
// Nodes are tested in the order of their numbers; a node counts if its parent is the node reached so far.  With p, q the target's
// and the draft's rows there, what is left of p once some children were rejected is r_s(v) = max(p(v) - s q(v), 0) for ONE
// number s per node: rejecting a child replaces r by max(r - (R / a) q, 0), R = sum of r, a = the draft's mass not yet rejected,
// and that is r under s + R / a, since r is p - s q wherever it is not 0 (and a rejected token has r = 0 already).  So a
// rejection costs one sum over the row, an acceptance none: it takes p and q at one token, and those are fetched for all nodes at the
// start, before it is known which of them will count.
// Sums are taken over trunc(r 2^44) in 64-bit integers, so that neither their order nor the way the row is split matters and
// the token drawn at the end is the same bit for bit wherever it is computed.
//
// A cluster of eight CTAs shares a sequence: each walks the tree on its own (same numbers, same decisions) and sums its part of a
// row; a warp tells its sum to all CTAs through distributed shared memory, then the cluster's barrier, and all of them know it.
// Vocabularies of up to 32768 leave 8 values a thread, which stay in registers as long as the node is the one reached.  What bounds a
// call is the chain of passes of its unluckiest sequence; 40 registers let three CTAs share a multiprocessor, so that 55 sequences
// go at once (48 trees of 40-64 nodes: 26 us, greedily 20-26 nodes 16; side by side 24.4, read anew in every pass, as larger vocabularies
// are, 26.6; with 69 registers, the values kept as 64-bit floats, 34 us; with 64 26 us).
// Measured and not better: bringing rows into L2 when a node is reached (26 us), or those of its children (greedily 15.4 -> 19.7).
#include <algorithm>

#include "kv16.cuh"

namespace dl {

constexpr int kTvThreads = 512;
constexpr int kTvCluster = 8;
constexpr int kTvNodes = 2048;           // most nodes of a sequence
constexpr int kTvBlock = 8;              // values a thread takes at a time
constexpr double kTvUnit = 17592186044416.0;                       // 2^44; up to 2^18 values of at most that: sums below 2^63

struct TvArgs {
  const void* target; const float* draft; const float* u; const int32_t* tokens; const int32_t* parent; const int32_t* starts;
  uint8_t* keep; int32_t* count; int32_t* next;
  long long target_stride, draft_stride;
  int32_t B, total, vocab, cap;          // cap: nodes that shared memory has room for
  int32_t wide;                          // rows begin on 16 bytes: bit 0 the target's, bit 1 the draft's
  DeviceStatus* status;
};

__device__ __forceinline__ uint32_t tv_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void tv_cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// writes v to the same shared-memory word of the cluster's CTA `rank`
__device__ __forceinline__ void tv_tell(unsigned long long* word, uint32_t rank, unsigned long long v) {
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(word);
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(rank));
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there), "l"(v) : "memory");
}

// a child's random number, held to [0, 1): below 0 and NaN as 0, from 1 on as the last number in front of it
__device__ __forceinline__ float tv_number(float u) { return fminf(fmaxf(u, 0.f), 0x1.fffffep-1f); }
__device__ __forceinline__ double tv_held(double x) { return x > 0.0 ? (x < 1.0 ? x : 1.0) : 0.0; }
// (p - s q held to 0..1) in units of 2^-44, cut off: from p 2^44 and s 2^44, which round as p and s do; NaN converts to the least
// number, what is too large to the largest
__device__ __forceinline__ unsigned long long tv_units(double p, double q, double s) {
  const long long r = __double2ll_rz(__dsub_rn(p, __dmul_rn(s, q)));
  return (unsigned long long)min(max(r, 0ll), (long long)kTvUnit);
}

// order of values as integers: NaN as -infinity, -0 as +0
__device__ __forceinline__ uint32_t tv_order(float v) {
  v = isnan(v) ? -INFINITY : v + 0.0f;
  const uint32_t w = __float_as_uint(v);
  return (w & 0x80000000u) ? ~w : (w | 0x80000000u);
}

struct TvShared {
  unsigned long long each[2][kTvCluster * kTvThreads / 32];        // what the cluster's warps told this CTA, two rounds
  unsigned long long from[2][kTvCluster];                          // what its CTAs did
  unsigned long long warp[kTvThreads / 32];
};

// sum over the warp of values below 2^57
__device__ __forceinline__ unsigned long long tv_warp_sum(unsigned long long v) {
  constexpr uint32_t kLimb = (1u << 26) - 1u;
  const uint32_t a = __reduce_add_sync(0xffffffffu, (uint32_t)v & kLimb), b = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 26) & kLimb),
                 c = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 52));
  return (unsigned long long)a + ((unsigned long long)b << 26) + ((unsigned long long)c << 52);
}
__device__ __forceinline__ unsigned long long tv_warp_max(unsigned long long v) {
  const uint32_t top = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32));
  const uint32_t low = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32) == top ? (uint32_t)v : 0u);
  return ((unsigned long long)top << 32) | low;
}
// Sum (or largest) over the cluster of what every warp has found: each tells all CTAs, and every warp puts the numbers together for
// itself.  Two sets of words, so that one barrier of the cluster per round is enough.
template <bool kMax>
__device__ __forceinline__ unsigned long long tv_all(unsigned long long of_warp, TvShared* sh, uint32_t rank, int& round) {
  constexpr int kWarps = kTvThreads / 32;
  const int lane = threadIdx.x & 31;
  unsigned long long* box = sh->each[round & 1];
  ++round;
  if (lane < kTvCluster) tv_tell(box + rank * kWarps + (threadIdx.x >> 5), lane, of_warp);
  tv_cluster_sync();
  unsigned long long v = 0;
#pragma unroll
  for (int i = 0; i < kTvCluster * kWarps / 32; ++i) {
    const unsigned long long x = box[32 * i + lane];
    v = kMax ? (x > v ? x : v) : v + x;
  }
  return kMax ? tv_warp_max(v) : tv_warp_sum(v);
}
// Sum over the cluster; `before` gets the sum over the threads in front of this one, in the order of CTAs and threads.
__device__ __forceinline__ unsigned long long tv_scan(unsigned long long v, TvShared* sh, uint32_t rank, int& round, unsigned long long* before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long run = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long x = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += x;
  }
  if (lane == 31) sh->warp[warp] = run;
  __syncthreads();
  unsigned long long mine = 0, front = 0;
#pragma unroll
  for (int w = 0; w < kTvThreads / 32; ++w) {
    const unsigned long long x = sh->warp[w];
    if (w < warp) front += x;
    mine += x;
  }
  unsigned long long* box = sh->from[round & 1];
  ++round;
  if (threadIdx.x < kTvCluster) tv_tell(box + rank, threadIdx.x, mine);
  tv_cluster_sync();
  unsigned long long all = 0;
#pragma unroll
  for (int c = 0; c < kTvCluster; ++c) {
    const unsigned long long x = box[c];
    if (c < (int)rank) front += x;
    all += x;
  }
  *before = front + run - v;
  return all;
}

// Eight values of a row from v on, those behind its end 0 (or -infinity).
template <typename T> __device__ __forceinline__ void tv_load(const T* row, int v, int vocab, bool wide, float fill, float (&x)[kTvBlock]) {
  if (wide && v + kTvBlock <= vocab) {
    if (sizeof(T) == 4) {
      const float4 a = __ldcg(reinterpret_cast<const float4*>(row + v)), b = __ldcg(reinterpret_cast<const float4*>(row + v) + 1);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
      const uint4 a = __ldcg(reinterpret_cast<const uint4*>(row + v));
      x[0] = bf16lo(a.x); x[1] = bf16hi(a.x); x[2] = bf16lo(a.y); x[3] = bf16hi(a.y);
      x[4] = bf16lo(a.z); x[5] = bf16hi(a.z); x[6] = bf16lo(a.w); x[7] = bf16hi(a.w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kTvBlock; ++i) x[i] = v + i < vocab ? to_f32<T>(row[v + i]) : fill;
  }
}

// kNear: a thread's part of a row is one block.
template <int MODE, typename T, bool kNear>
__global__ void __launch_bounds__(kTvThreads, 3)
tree_verify_kernel(const TvArgs a) {
  extern __shared__ int nodes[];
  __shared__ TvShared sh;
  chained_go();
  chained_wait();
  constexpr bool kGreedy = MODE == DL_VERIFY_GREEDY, kPoint = MODE == DL_VERIFY_POINT;
  constexpr bool kDraft = MODE == DL_VERIFY_SAMPLE || MODE == DL_VERIFY_REPLACED;
  const uint32_t rank = tv_rank();
  const int b = blockIdx.x / kTvCluster, tid = threadIdx.x, lane = tid & 31;
  const int from = k16_start(a.starts, b, a.total), to = max(from, k16_start(a.starts, b + 1, a.total));
  const int n = min(to - from, a.cap);
  int* up = nodes;                                                 // parent; -2: never reached
  int* tok = nodes + a.cap;
  float* un = reinterpret_cast<float*>(nodes + 2 * a.cap);
  float* pc = reinterpret_cast<float*>(nodes + 3 * a.cap);          // the target's and the draft's value at the token, behind the parent
  float* qc = reinterpret_cast<float*>(nodes + 4 * a.cap);
  const T* target = static_cast<const T*>(a.target);
  if (n == 0) {
    if (rank == 0 && tid == 0) { a.count[b] = 0; a.next[b] = -1; }
    return;
  }
  bool bad = to - from > n;
  for (int i = tid; i < n; i += kTvThreads) {
    int p = i == 0 ? -1 : __ldcg(a.parent + from + i);
    const int t = i == 0 ? 0 : __ldcg(a.tokens + from + i);
    const float u = kGreedy ? 0.f : __ldcg(a.u + from + i);
    if (i > 0 && (p < 0 || p >= i)) { bad = bad || p != -1; p = -2; }
    if (i > 0 && (unsigned)t >= (unsigned)a.vocab) { bad = true; p = -2; }
    up[i] = p;
    tok[i] = t;
    if (!kGreedy) {
      un[i] = i > 0 ? tv_number(u) : u;                            // (the root's is held where the token is drawn)
      pc[i] = p >= 0 ? to_f32<T>(target[(from + p) * a.target_stride + t]) : 0.f;
      qc[i] = kDraft && p >= 0 ? __ldcg(a.draft + (from + p) * a.draft_stride + t) : 0.f;
    }
  }
  if (bad && rank == 0) report_status(a.status, DL_ERR_INVALID_ARG, b);
  if (rank == 0)
    for (int i = tid; i < to - from; i += kTvThreads) a.keep[from + i] = i == 0;
  tv_cluster_sync();                                               // (and every CTA is there before anybody tells it something)
  // this thread's part of a row
  const int blocks = kNear ? 1 : (a.vocab + kTvCluster * kTvThreads * kTvBlock - 1) / (kTvCluster * kTvThreads * kTvBlock);
  const int v0 = ((int)rank * kTvThreads + tid) * blocks * kTvBlock;
  const bool wide_p = a.wide & 1, wide_q = a.wide & 2;
  int at = 0, accepted = 1, round = 0, round2 = 0;
  double s = 0.0, R = 1.0, left = 1.0;
  // the next child of `at` behind node i, or n: 32 nodes at a time
  auto next_child = [&](int i) {
    for (int base = (i + 1) & ~31; base < n; base += 32) {
      const int j = base + lane;
      const unsigned m = __ballot_sync(0xffffffffu, j < n && j > i && up[j] == at);
      if (m) return base + __ffs(m) - 1;
    }
    return n;
  };
  auto best_of = [&](int node) {
    const T* row = target + (long long)(from + node) * a.target_stride;
    uint32_t best = 0u, index = 0xFFFFFFFFu;                       // (every value's order is above 0)
    for (int k = 0; k < blocks; ++k) {
      const int v = v0 + k * kTvBlock;
      if (v >= a.vocab) break;
      float x[kTvBlock];
      tv_load<T>(row, v, a.vocab, wide_p, 0.f, x);
#pragma unroll
      for (int i = 0; i < kTvBlock; ++i) {
        const uint32_t o = tv_order(x[i]);
        if (v + i < a.vocab && o > best) { best = o; index = (uint32_t)(v + i); }
      }
    }
    const uint32_t top = __reduce_max_sync(0xffffffffu, best);
    const uint32_t first = __reduce_min_sync(0xffffffffu, best == top ? index : 0xFFFFFFFFu);
    return (int)(0xFFFFFFFFu - (uint32_t)tv_all<true>(((unsigned long long)top << 32) | (0xFFFFFFFFu - first), &sh, rank, round));
  };
  // the row of the node reached: p 2^44 and q of this thread's block, if it has one only
  float pr[kTvBlock], qr[kTvBlock];
  bool here = false;
  auto fetch = [&](int v, float (&p)[kTvBlock], float (&q)[kTvBlock]) {
    float x[kTvBlock], y[kTvBlock];
    if (v < a.vocab) {
      tv_load<T>(target + (long long)(from + at) * a.target_stride, v, a.vocab, wide_p, 0.f, x);
      if (kDraft) tv_load<float>(a.draft + (long long)(from + at) * a.draft_stride, v, a.vocab, wide_q, 0.f, y);
    }
#pragma unroll
    for (int i = 0; i < kTvBlock; ++i) {
      p[i] = v < a.vocab ? x[i] : 0.f;
      q[i] = kDraft && v < a.vocab ? y[i] : 0.f;
    }
    if (kPoint)                                                    // tokens that this node's children have had rejected count 0
      for (int j = next_child(at); j < n; j = next_child(j)) {
        const int d = tok[j] - v;
#pragma unroll
        for (int i = 0; i < kTvBlock; ++i)
          if (d == i) p[i] = 0.f;
      }
  };
  // weights of the thread's values, in their order: f(value's index, its weight); true ends it
  auto weigh = [&](bool plain, auto f) {
    const double s44 = s * kTvUnit;
    for (int k = 0; k < blocks; ++k) {
      const int v = v0 + k * kTvBlock;
      if (!kPoint && v >= a.vocab) break;                          // (POINT: whole warps look for children)
      if (plain) {
        float x[kTvBlock];
        if (v < a.vocab) tv_load<T>(target + (long long)(from + at) * a.target_stride, v, a.vocab, wide_p, 0.f, x);
#pragma unroll
        for (int i = 0; i < kTvBlock; ++i)
          if (v < a.vocab && f(v + i, tv_units((double)x[i] * kTvUnit, 0.0, 0.0))) return;
        continue;
      }
      if (!kNear || !here) fetch(v, pr, qr);
      here = kNear;
#pragma unroll
      for (int i = 0; i < kTvBlock; ++i)
        if (f(v + i, tv_units((double)pr[i] * kTvUnit, (double)qr[i], s44))) return;
    }
  };
  auto sum_of = [&](bool plain) {
    unsigned long long sum = 0;
    weigh(plain, [&](int, unsigned long long w) { sum += w; return false; });
    return sum;
  };
  int best = kGreedy ? best_of(0) : 0;
  for (int i = next_child(0); i < n; i = next_child(i)) {
    bool yes;
    if (kGreedy) {
      yes = tok[i] == best;
    } else {
      const double u = (double)un[i], p = (double)pc[i], q = (double)qc[i];
      if (kPoint) {
        bool gone = false;                                         // the same token has been rejected here already
        for (int j = next_child(at); j < i; j = next_child(j)) gone = gone || tok[j] == tok[i];
        const double pl = gone ? 0.0 : p;
        yes = __dmul_rn(u, R) < pl;
        if (!yes) R = __dsub_rn(R, pl);
      } else {
        yes = left > 0.0 && __dmul_rn(__dmul_rn(u, q), R) < __dmul_rn(tv_held(__dsub_rn(p, __dmul_rn(s, q))), left);
        if (!yes && left > 0.0) {
          s = __dadd_rn(s, __ddiv_rn(R, left));
          R = __ull2double_rn(tv_all<false>(tv_warp_sum(sum_of(false)), &sh, rank, round)) / kTvUnit;
          if (MODE == DL_VERIFY_SAMPLE) left = __dsub_rn(left, q);
        }
      }
    }
    if (yes) {
      at = i;
      ++accepted;
      s = 0.0;
      R = left = 1.0;
      here = false;
      if (rank == 0 && tid == 0) a.keep[from + i] = 1;
      if (kGreedy) best = best_of(i);
    }
  }
  if (!kGreedy) {
    unsigned long long before, sum = sum_of(false);
    unsigned long long all = tv_scan(sum, &sh, rank, round2, &before);
    const bool plain = all == 0;                                   // nothing is left of r
    if (plain) {
      sum = sum_of(true);
      all = tv_scan(sum, &sh, rank, round2, &before);
    }
    const unsigned long long k = (unsigned long long)min(max(__double2ll_rz((double)un[0] * 2147483648.0), 0ll), 0x7FFFFFFFll);
    const unsigned long long bound = k * (all >> 31) + ((k * (all & 0x7FFFFFFFull)) >> 31);
    const bool mine = all > 0 && before <= bound && bound < before + sum;
    if (kPoint ? __any_sync(0xffffffffu, mine) : mine) {
      int token = -1;
      weigh(plain, [&](int v, unsigned long long w) {
        before += w;
        if (token < 0 && before > bound) token = v;
        return !kPoint && token >= 0;
      });
      if (mine) a.next[b] = token;
    }
    if (all == 0 && rank == 0 && tid == 0) {
      a.next[b] = -1;
      report_status(a.status, DL_ERR_INVALID_ARG, b);
    }
  } else if (rank == 0 && tid == 0) {
    a.next[b] = best;
  }
  if (rank == 0 && tid == 0) a.count[b] = accepted;
  tv_cluster_sync();                                               // no CTA leaves while others may still write its words
}

template <int MODE, typename T>
static cudaError_t tv_launch(const TvArgs& a, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.B * kTvCluster);
  cfg.blockDim = dim3(kTvThreads);
  cfg.dynamicSmemBytes = (size_t)5 * a.cap * 4;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kTvCluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return a.vocab <= kTvCluster * kTvThreads * kTvBlock ? cudaLaunchKernelEx(&cfg, tree_verify_kernel<MODE, T, true>, a)
                                                        : cudaLaunchKernelEx(&cfg, tree_verify_kernel<MODE, T, false>, a);
}

cudaError_t launch_tree_verify(const dl_ctx* ctx, const void* target, int32_t dtype, int64_t target_stride, const float* draft,
                               int64_t draft_stride, const float* u, const int32_t* tokens, const int32_t* parent,
                               const int32_t* starts, int32_t B, int32_t total, int32_t vocab, int32_t mode, uint8_t* keep,
                               int32_t* count, int32_t* next, cudaStream_t s) {
  TvArgs a = {};
  a.target = target; a.draft = draft; a.u = u; a.tokens = tokens; a.parent = parent; a.starts = starts;
  a.keep = keep; a.count = count; a.next = next;
  a.target_stride = target_stride; a.draft_stride = draft_stride;
  a.B = B; a.total = total; a.vocab = vocab; a.cap = std::min(std::max(total, 1), kTvNodes);
  a.wide = (target_stride % (dtype == DL_F32 ? 4 : 8) == 0 ? 1 : 0) | (draft_stride % 4 == 0 ? 2 : 0);   // (the tensors do)
  a.status = ctx->ws.base ? ctx->ws.status : nullptr;
  switch (mode) {
    case DL_VERIFY_GREEDY:
      return dtype == DL_F32 ? tv_launch<DL_VERIFY_GREEDY, float>(a, s) : tv_launch<DL_VERIFY_GREEDY, __nv_bfloat16>(a, s);
    case DL_VERIFY_SAMPLE: return tv_launch<DL_VERIFY_SAMPLE, float>(a, s);
    case DL_VERIFY_REPLACED: return tv_launch<DL_VERIFY_REPLACED, float>(a, s);
    default: return tv_launch<DL_VERIFY_POINT, float>(a, s);
  }
}

}  // namespace dl
