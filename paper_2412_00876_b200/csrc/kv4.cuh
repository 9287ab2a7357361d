// The 4-bit K/V cache: how a page is laid out and how a row becomes codes (shared by kv4_cache.cu and
// attn_decode_kv4.cu).
//
// A row of D values (D = 64 or 128) is cut into groups of 64.  Per group: z = min, s = bf16((max - min) / 15),
// code = nearest-even((x - z) * (1 / s)) clipped to 0 .. 15, each operation rounded to fp32; the value held is
// s * code + z.  The inputs are bf16, so z is exact in bf16; where s is below 2^-126 (a constant group, say) all codes
// are 0.  A group with a NaN or an infinity in it, or with a range beyond fp32, holds NaN.
//
// A page of page_rows rows holds, per K/V head, page_rows / 16 tiles of 16 rows; a tile is 18 D consecutive bytes:
//   K codes [16][D/2] | V codes [8][D] | K words [16][D/64] | V words [16][D/64]       word = s | z << 16 (bf16 bits)
// K: a 32-bit unit holds 8 consecutive dims of a row, lowest dim in the lowest 4 bits; for D = 128 the two 32-byte halves of
// a row (its two groups) are swapped in rows with bit 1 set.  V: the rows 2i, 2i + 1 share D bytes; a 32-bit unit holds 4
// consecutive dims, of row 2i in its lower half and of row 2i + 1 in its upper half (what one fp16 operand register of
// P V wants); the 16-byte steps of a pair are XORed with 2 (i & 3) (D = 64: 2 (i >> 1 & 1)).  With both orders the decode
// kernel's fragment loads touch every bank once.  One tile is one bulk copy, so a cache is read in pieces of 2304
// (1152) bytes.
#pragma once

#include "common.cuh"

namespace dl {

constexpr int kKv4Rows = 16;            // rows per tile
constexpr int kKv4Group = 64;           // values per scale

template <int D> struct Kv4 {
  static constexpr int NG = D / kKv4Group;            // groups per row
  static constexpr int RB = D / 2;                    // bytes of a row's codes
  static constexpr int V = kKv4Rows * RB;             // offset of the V codes
  static constexpr int KM = 2 * kKv4Rows * RB;        // K words
  static constexpr int VM = KM + kKv4Rows * 4 * NG;   // V words
  static constexpr int TILE = VM + kKv4Rows * 4 * NG;
  static_assert(TILE == 18 * D, "tile size");
};

// byte offset, inside a tile, of the 32 bytes that hold group g of `row`'s K codes
template <int D> __device__ __forceinline__ int kv4_k_off(int row, int g) {
  return row * Kv4<D>::RB + (D == 128 ? 32 * (g ^ ((row >> 1) & 1)) : 0);
}
// byte offset, inside a tile, of the 8 bytes (two units: dims d .. d + 7, d a multiple of 8) of row pair i's V codes
template <int D> __device__ __forceinline__ int kv4_v_off(int i, int d) {
  const int step = (d >> 4) ^ (D == 128 ? 2 * (i & 3) : 2 * ((i >> 1) & 1));
  return Kv4<D>::V + i * D + 16 * step + (d & 8);
}

// bf16 pairs: minimum and maximum that keep a NaN
__device__ __forceinline__ uint32_t kv4_min2(uint32_t x, uint32_t y) {
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}
__device__ __forceinline__ uint32_t kv4_max2(uint32_t x, uint32_t y) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}
// two fp32 operations, each rounded by itself
__device__ __forceinline__ uint64_t kv4_pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint64_t kv4_add2(uint64_t x, uint64_t y) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  return r;
}
__device__ __forceinline__ uint64_t kv4_fma2(uint64_t x, uint64_t y, uint64_t z) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
  return r;
}

// range / 15, correctly rounded (range normal): the product with the rounded reciprocal, corrected once with the exact
// remainder (Markstein's scheme).
__device__ __forceinline__ float kv4_div15(float range) {
  constexpr float c = 1.f / 15.f;
  const float q = __fmul_rn(range, c);
  return __fmaf_rn(__fmaf_rn(-15.f, q, range), c, q);
}
// 1 / s, correctly rounded, for a normal s of eight significant bits (bf16) up to 2^125: one Newton step from the
// approximation leaves an error below 2^-44 of the result, and 1 / s, a power of two over an odd number below 256, is never
// nearer than 2^-33 to the middle between two floats.
__device__ __forceinline__ float kv4_recip(float s) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s));
  return __fmaf_rn(y, __fmaf_rn(-s, y, 1.f), y);
}

// Sixteen consecutive values per lane (`u`: bf16 pairs), four lanes per group (lanes 4i .. 4i + 3): this lane's codes, and
// the group's word.  All 32 lanes take part.  The extremes are found on bf16 pairs; from the first reduction on a lane
// holds (min, -max) in one register.
__device__ __forceinline__ uint2 kv4_quantise16(const uint32_t (&u)[8], uint32_t& word) {
  uint32_t mn = u[0], mx = u[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) { mn = kv4_min2(mn, u[i]); mx = kv4_max2(mx, u[i]); }
  mx ^= 0x80008000u;                                                        // -max
  uint32_t ext = kv4_min2(__byte_perm(mn, mx, 0x5410), __byte_perm(mn, mx, 0x7632));
  ext = kv4_min2(ext, __shfl_xor_sync(0xffffffffu, ext, 1));
  ext = kv4_min2(ext, __shfl_xor_sync(0xffffffffu, ext, 2));
  const float lo = bf16lo(ext), range = __fsub_rn(-bf16hi(ext), lo);
  const bool odd = !(range <= 3.402823466e38f);                             // a NaN, an infinity, a range beyond fp32
  const __nv_bfloat16 sb = __float2bfloat16_rn(kv4_div15(range));
  const float s = __bfloat162float(sb);
  // s >= 2^-126 has eight significant bits, so (x - z) / s is at most 15 (1 + 2^-8): no code above 15
  const bool flat = odd || !(s >= 1.17549435e-38f);
  const float inv = flat ? 0.f : kv4_recip(s);
  uint32_t c[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // + 2^23: the nearest integer ends up in the low bits (the product is rounded first, as the definition says)
      const uint32_t w = u[4 * h + i];
      t[2 * i] = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(bf16lo(w), lo), inv), 8388608.f));
      t[2 * i + 1] = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(bf16hi(w), lo), inv), 8388608.f));
    }
    uint32_t acc = t[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) acc = acc * 16u + t[i];
    c[h] = acc - 0x4B000000u * 0x11111111u;                                 // what the bits of 2^23 have added up to
  }
  word = odd ? 0x7FC00000u : (uint32_t)__bfloat16_as_ushort(sb) | (ext << 16);
  return flat ? make_uint2(0u, 0u) : make_uint2(c[0], c[1]);
}

// Where row `row` of a tile has its codes and words, in a form that is cheap per lane: the codes of lane l (0 .. D/16 - 1:
// dims 16 l .. 16 l + 15) begin at code + (place ^ turn) with place = 8 l in K, 16 l in V, its group's word at word + 4 (l / 4).
struct Kv4Row { int code, turn, word, upper; };          // upper (V): the row has the upper halves of its pair's units
template <int D> __device__ __forceinline__ Kv4Row kv4_row(int row, bool is_v) {
  Kv4Row r;
  const int i = row >> 1;
  r.code = is_v ? kv4_v_off<D>(0, 0) + i * D : row * Kv4<D>::RB;
  r.turn = is_v ? kv4_v_off<D>(i, 0) - r.code : kv4_k_off<D>(row, 0) - r.code;
  r.word = (is_v ? Kv4<D>::VM : Kv4<D>::KM) + row * Kv4<D>::NG * 4;
  r.upper = row & 1;
  return r;
}
// Stores what kv4_quantise16 gave for lane `l` of a row of the tile at `tile`; is_v picks the tensor.  No byte of another row
// is written.
__device__ __forceinline__ void kv4_store16(uint8_t* tile, const Kv4Row& r, int l, bool is_v, uint2 code, uint32_t word) {
  if (is_v) {
    uint16_t* to = reinterpret_cast<uint16_t*>(tile + (r.code + 2 * r.upper + ((16 * l) ^ r.turn)));
    to[0] = (uint16_t)code.x;
    to[2] = (uint16_t)(code.x >> 16);
    to[4] = (uint16_t)code.y;
    to[6] = (uint16_t)(code.y >> 16);
  } else {
    *reinterpret_cast<uint2*>(tile + (r.code + ((8 * l) ^ r.turn))) = code;
  }
  if ((l & 3) == 0) *reinterpret_cast<uint32_t*>(tile + r.word + l) = word;
}
// The codes that it stored.
__device__ __forceinline__ uint2 kv4_load16(const uint8_t* tile, const Kv4Row& r, int l, bool is_v) {
  if (!is_v) return __ldg(reinterpret_cast<const uint2*>(tile + (r.code + ((8 * l) ^ r.turn))));
  const uint4 w = __ldg(reinterpret_cast<const uint4*>(tile + (r.code + ((16 * l) ^ r.turn))));
  const uint32_t pick = r.upper ? 0x7632u : 0x5410u;
  return make_uint2(__byte_perm(w.x, w.y, pick), __byte_perm(w.z, w.w, pick));
}

// What a paged call knows of the pages, by value.
struct PagesArg {
  const int32_t* table; const int32_t* len;
  int32_t B, n_pages, max_pages, tile_shift;          // page_rows = 16 << tile_shift
};

inline PagesArg pages_arg(const dl_pages* p) {
  return PagesArg{p->table, p->len, p->B, p->n_pages, p->max_pages,
                  p->page_rows == 16 ? 0 : p->page_rows == 32 ? 1 : p->page_rows == 64 ? 2 : 3};
}

// Tile index in the pool of tile t (16 rows) of sequence b and K/V head hk, or -1 where the table names no page.
__device__ __forceinline__ int kv4_tile_index(const PagesArg& p, int page, int Hk, int hk, int t) {
  if ((unsigned)page >= (unsigned)p.n_pages) return -1;
  return ((page * Hk + hk) << p.tile_shift) + (t & ((1 << p.tile_shift) - 1));
}

}  // namespace dl
