// The paged K/V cache in 16 bits, shared by the kernels that write and read it: page = [K, V][Hk][page_rows][D] bf16.
#pragma once

#include "common.cuh"

namespace dl {

struct K16Pages {
  const int32_t* table; int32_t* len;
  int32_t B, n_pages, W, shift;           // W: columns of the table; page_rows = 1 << shift
};

inline K16Pages k16_pages(const dl_pages* p) {
  K16Pages a = {};
  if (!p) return a;
  a.table = p->table; a.len = p->len;
  a.B = p->B; a.n_pages = p->n_pages; a.W = p->max_pages;
  a.shift = p->page_rows == 16 ? 4 : p->page_rows == 32 ? 5 : p->page_rows == 64 ? 6 : 7;
  return a;
}

// Page of row t of sequence b, or -1.  (.cg loads: the books may be written by the launch in front.)
__device__ __forceinline__ int k16_page(const K16Pages& pg, int b, long long t) {
  const long long i = t >> pg.shift;
  if (t < 0 || i >= pg.W) return -1;
  const int p = __ldcg(pg.table + (size_t)b * pg.W + i);
  return (unsigned)p < (unsigned)pg.n_pages ? p : -1;
}

// Row of the pool (of D values) that holds K (kv = 0) or V (1) of row t, which lies in `page`, for K/V head h.
__device__ __forceinline__ long long k16_row(const K16Pages& pg, int Hk, int page, int kv, int h, long long t) {
  return ((((long long)page * 2 + kv) * Hk + h) << pg.shift) + (t & ((1 << pg.shift) - 1));
}

// Start of sequence b among `total` packed rows, brought back inside them.
__device__ __forceinline__ int k16_start(const int32_t* starts, int b, int total) { return min(max(__ldcg(starts + b), 0), total); }

// The sequence that packed row r belongs to (st: all B + 1 starts, brought back inside): the last whose start is <= r, or -1.
__device__ __forceinline__ int k16_sequence(const int* st, int B, int r) {
  int lo = -1, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (st[mid] <= r) lo = mid; else hi = mid - 1;
  }
  return (lo >= 0 && r < st[lo + 1]) ? lo : -1;
}

}  // namespace dl
