// Attention of tree nodes (drafted tokens, chunks of a prompt, single tokens) over a paged cache in 16 bits.  An extension, not in
// the paper.  Plain form on the CUDA cores: a warp per (node, query head), keys one after the other with a running maximum.
#include <algorithm>

#include "kv16.cuh"

namespace dl {

struct AtTreeArgs {
  const __nv_bfloat16* q; const __nv_bfloat16* pool; const int32_t* starts; const int32_t* mask; __nv_bfloat16* out;
  long long q_stride;
  int32_t H, Hk, total, max_rows, words;
  float scale_log2;
  DeviceStatus* status;
};

template <int D>
__global__ void __launch_bounds__(128)
attn_tree_kernel(const K16Pages pg, const AtTreeArgs a) {
  extern __shared__ int seq_start[];
  for (int b = threadIdx.x; b <= pg.B; b += blockDim.x) seq_start[b] = k16_start(a.starts, b, a.total);
  __syncthreads();
  const int lane = threadIdx.x & 31, r = blockIdx.x, h = blockIdx.y * 4 + (threadIdx.x >> 5);
  if (h >= a.H) return;
  const int b = k16_sequence(seq_start, pg.B, r);
  if (b < 0) return;
  const int i = r - seq_start[b], n = seq_start[b + 1] - seq_start[b];
  if (i >= a.max_rows) {
    report_status(a.status, DL_ERR_INVALID_ARG, b);
    return;
  }
  constexpr int E = D / 32;
  const int hk = h / (a.H / a.Hk), held = max(__ldcg(pg.len + b), 0);
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = __bfloat162float(a.q[r * a.q_stride + h * D + lane * E + e]) * a.scale_log2;
    o[e] = 0.f;
  }
  for (int t = 0; t < held + n; ++t) {
    if (t >= held) {
      const int j = t - held;
      if (a.mask ? !((a.mask[(size_t)r * a.words + (j >> 5)] >> (j & 31)) & 1) : j > i) continue;
    }
    const int page = k16_page(pg, b, t);
    if (page < 0) {
      report_status(a.status, DL_ERR_INVALID_ARG, b);
      continue;
    }
    const __nv_bfloat16* k = a.pool + k16_row(pg, a.Hk, page, 0, hk, t) * D + lane * E;
    const __nv_bfloat16* v = a.pool + k16_row(pg, a.Hk, page, 1, hk, t) * D + lane * E;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += q[e] * __bfloat162float(k[e]);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    const float top = fmaxf(m, s);
    if (top == -INFINITY) continue;
    const float c = exp2f(m - top), p = exp2f(s - top);
    m = top;
    l = l * c + p;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * c + p * __bfloat162float(v[e]);
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) a.out[((size_t)r * a.H + h) * D + lane * E + e] = __float2bfloat16_rn(o[e] * inv);
}

cudaError_t launch_attn_tree(dl_ctx* ctx, const dl_pages* p, int32_t Hk, const void* pool, const void* q, int64_t q_stride,
                             const int32_t* starts, int32_t total, int32_t max_rows, const int32_t* mask, int32_t words,
                             float scale, void* out, cudaStream_t s) {
  const K16Pages pg = k16_pages(p);
  AtTreeArgs a = {};
  a.q = static_cast<const __nv_bfloat16*>(q); a.pool = static_cast<const __nv_bfloat16*>(pool);
  a.starts = starts; a.mask = mask; a.out = static_cast<__nv_bfloat16*>(out);
  a.q_stride = q_stride;
  a.H = ctx->desc.n_heads; a.Hk = Hk; a.total = total; a.words = words;
  a.max_rows = mask ? std::min(max_rows, 32 * words) : max_rows;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.status = ctx->ws.base ? ctx->ws.status : nullptr;
  const dim3 grid(total, (a.H + 3) / 4);
  const size_t smem = (size_t)(pg.B + 1) * 4;
  if (ctx->desc.head_dim == 128) attn_tree_kernel<128><<<grid, 128, smem, s>>>(pg, a);
  else attn_tree_kernel<64><<<grid, 128, smem, s>>>(pg, a);
  return cudaGetLastError();
}

}  // namespace dl
