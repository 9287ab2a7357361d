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
// A cluster of CTAs shares a sequence: each walks the tree on its own (same numbers, same decisions), sums its part of
// a row, and tells the others its sum through distributed shared memory.
#include <algorithm>

#include "kv16.cuh"

namespace dl {

constexpr int kTvThreads = 512;
constexpr int kTvCluster = 8;
constexpr int kTvNodes = 2048;           // most nodes of a sequence
constexpr double kTvUnit = 17592186044416.0;                       // 2^44; up to 2^18 values of at most that: sums below 2^63

struct TvArgs {
  const void* target; const float* draft; const float* u; const int32_t* tokens; const int32_t* parent; const int32_t* starts;
  uint8_t* keep; int32_t* count; int32_t* next;
  long long target_stride, draft_stride;
  int32_t B, total, vocab, cap;          // cap: nodes that shared memory has room for
  DeviceStatus* status;
};

__device__ __forceinline__ uint32_t tv_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void tv_cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// writes v to the same shared-memory word of the cluster's CTA `rank`
__device__ __forceinline__ void tv_tell(unsigned long long* word, uint32_t rank, unsigned long long v) {
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(word);
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(rank));
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there), "l"(v) : "memory");
}

__device__ __forceinline__ double tv_held(double x) { return x > 0.0 ? (x < 1.0 ? x : 1.0) : 0.0; }
// r in units of 2^-44, cut off: p - s q without a fused step
__device__ __forceinline__ unsigned long long tv_units(float p, float q, double s) {
  const double r = __dsub_rn((double)p, __dmul_rn(s, (double)q));
  return (unsigned long long)__double2ll_rz(tv_held(r) * kTvUnit);
}

// order of values as integers: NaN as -infinity, -0 as +0; ties go to the lower index
__device__ __forceinline__ unsigned long long tv_key(float v, uint32_t index) {
  v = isnan(v) ? -INFINITY : v + 0.0f;
  const uint32_t w = __float_as_uint(v);
  const uint32_t o = (w & 0x80000000u) ? ~w : (w | 0x80000000u);
  return ((unsigned long long)o << 32) | (0xFFFFFFFFu - index);
}

struct TvShared {
  unsigned long long from[2][kTvCluster];                          // what the cluster's CTAs told this one, two rounds
  unsigned long long warp[kTvThreads / 32];
};

// Sum (or largest) over the cluster of every thread's v; `before` gets the sum over the threads in front of this one, in the order
// of CTAs and threads.  Two sets of words, so that one barrier of the cluster per round is enough.
template <bool kMax, bool kScan>
__device__ __forceinline__ unsigned long long tv_join(unsigned long long v, TvShared* sh, uint32_t rank, int& round,
                                                      unsigned long long* before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long run = v;
  if (kScan) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long x = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += x;
    }
    if (lane == 31) sh->warp[warp] = run;
  } else {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long x = __shfl_xor_sync(0xffffffffu, run, o);
      run = kMax ? (x > run ? x : run) : run + x;
    }
    if (lane == 0) sh->warp[warp] = run;
  }
  __syncthreads();
  unsigned long long mine = 0, front = 0;
#pragma unroll
  for (int w = 0; w < kTvThreads / 32; ++w) {
    const unsigned long long x = sh->warp[w];
    if (kScan && w < warp) front += x;
    mine = kMax ? (x > mine ? x : mine) : mine + x;
  }
  unsigned long long* box = sh->from[round & 1];
  ++round;
  if (threadIdx.x < kTvCluster) tv_tell(box + rank, threadIdx.x, mine);
  tv_cluster_sync();
  unsigned long long all = 0;
#pragma unroll
  for (int c = 0; c < kTvCluster; ++c) {
    const unsigned long long x = box[c];
    if (kScan && c < (int)rank) front += x;
    all = kMax ? (x > all ? x : all) : all + x;
  }
  if (kScan) *before = front + run - v;
  return all;
}

template <int MODE, typename T>
__global__ void __launch_bounds__(kTvThreads)
tree_verify_kernel(const TvArgs a) {
  extern __shared__ int nodes[];
  __shared__ TvShared sh;
  chained_go();
  chained_wait();
  constexpr bool kGreedy = MODE == DL_VERIFY_GREEDY, kPoint = MODE == DL_VERIFY_POINT;
  constexpr bool kDraft = MODE == DL_VERIFY_SAMPLE || MODE == DL_VERIFY_REPLACED;
  const uint32_t rank = tv_rank();
  const int b = blockIdx.x / kTvCluster, tid = threadIdx.x;
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
    if (i > 0 && (p < 0 || p >= i)) { bad = bad || p != -1; p = -2; }
    if (i > 0 && (unsigned)t >= (unsigned)a.vocab) { bad = true; p = -2; }
    up[i] = p;
    tok[i] = t;
    if (!kGreedy) {
      un[i] = __ldcg(a.u + from + i);
      pc[i] = p >= 0 ? to_f32<T>(target[(from + p) * a.target_stride + t]) : 0.f;
      qc[i] = kDraft && p >= 0 ? __ldcg(a.draft + (from + p) * a.draft_stride + t) : 0.f;
    }
  }
  if (bad && rank == 0) report_status(a.status, DL_ERR_INVALID_ARG, b);
  __syncthreads();
  // this thread's part of a row
  const int per = (a.vocab + kTvCluster * kTvThreads - 1) / (kTvCluster * kTvThreads);
  const int v0 = min(a.vocab, ((int)rank * kTvThreads + tid) * per), v1 = min(a.vocab, v0 + per);
  int at = 0, accepted = 1, round = 0;
  double s = 0.0, R = 1.0, left = 1.0;
  auto best_of = [&](int node) {
    const T* row = target + (long long)(from + node) * a.target_stride;
    unsigned long long best = 0;
    for (int v = v0; v < v1; ++v) {
      const unsigned long long k = tv_key(to_f32<T>(row[v]), (uint32_t)v);
      best = k > best ? k : best;
    }
    return (int)(0xFFFFFFFFu - (uint32_t)tv_join<true, false>(best, &sh, rank, round, nullptr));
  };
  // a token that this node's children have had rejected already (POINT)
  auto gone = [&](int token, int until) {
    for (int j = at + 1; j < until; ++j)
      if (up[j] == at && tok[j] == token) return true;
    return false;
  };
  auto units = [&](int v) {
    const float p = to_f32<T>(target[(long long)(from + at) * a.target_stride + v]);
    if (kPoint) return gone(v, n) ? 0ull : tv_units(p, 0.f, 0.0);
    return tv_units(p, kDraft ? __ldcg(a.draft + (long long)(from + at) * a.draft_stride + v) : 0.f, s);
  };
  int best = kGreedy ? best_of(0) : 0;
  if (rank == 0)
    for (int i = tid; i < n; i += kTvThreads) a.keep[from + i] = i == 0;
  for (int i = 1; i < n; ++i) {
    if (up[i] != at) continue;
    bool yes;
    if (kGreedy) {
      yes = tok[i] == best;
    } else {
      const double u = (double)un[i], p = (double)pc[i], q = (double)qc[i];
      if (kPoint) {
        const double pl = gone(tok[i], i) ? 0.0 : p;
        yes = __dmul_rn(u, R) < pl;
        if (!yes) R = __dsub_rn(R, pl);
      } else {
        yes = left > 0.0 && __dmul_rn(__dmul_rn(u, q), R) < __dmul_rn(tv_held(__dsub_rn(p, __dmul_rn(s, q))), left);
        if (!yes && left > 0.0) {
          s = __dadd_rn(s, __ddiv_rn(R, left));
          unsigned long long sum = 0;
          for (int v = v0; v < v1; ++v) sum += units(v);
          R = __ull2double_rn(tv_join<false, false>(sum, &sh, rank, round, nullptr)) / kTvUnit;
          if (MODE == DL_VERIFY_SAMPLE) left = __dsub_rn(left, q);
        }
      }
    }
    if (yes) {
      at = i;
      ++accepted;
      s = 0.0;
      R = left = 1.0;
      if (rank == 0) {
        __syncthreads();                                           // the flags' zeros are written
        if (tid == 0) a.keep[from + i] = 1;
      }
      if (kGreedy) best = best_of(i);
    }
  }
  int token = best;
  if (!kGreedy) {
    unsigned long long sum = 0, before;
    for (int v = v0; v < v1; ++v) sum += units(v);
    unsigned long long all = tv_join<false, true>(sum, &sh, rank, round, &before);
    const bool plain = all == 0;                                   // nothing is left of r
    auto weight = [&](int v) {
      return plain ? tv_units(to_f32<T>(target[(long long)(from + at) * a.target_stride + v]), 0.f, 0.0) : units(v);
    };
    if (plain) {
      sum = 0;
      for (int v = v0; v < v1; ++v) sum += weight(v);
      all = tv_join<false, true>(sum, &sh, rank, round, &before);
    }
    const unsigned long long k = (unsigned long long)min(max(__double2ll_rz((double)un[0] * 2147483648.0), 0ll), 0x7FFFFFFFll);
    const unsigned long long bound = k * (all >> 31) + ((k * (all & 0x7FFFFFFFull)) >> 31);
    token = -1;
    if (all > 0 && before <= bound && bound < before + sum) {
      for (int v = v0; v < v1; ++v) {
        before += weight(v);
        if (before > bound) { token = v; break; }
      }
      a.next[b] = token;
    }
    if (all == 0 && rank == 0 && tid == 0) {
      a.next[b] = -1;
      report_status(a.status, DL_ERR_INVALID_ARG, b);
    }
  } else if (rank == 0 && tid == 0) {
    a.next[b] = token;
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
  return cudaLaunchKernelEx(&cfg, tree_verify_kernel<MODE, T>, a);
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
