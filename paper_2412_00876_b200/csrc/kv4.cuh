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

// Eight consecutive values per lane (`raw`: bf16), eight lanes per group (lanes 8i .. 8i + 7): this lane's codes, and the
// group's word.  All 32 lanes take part.
__device__ __forceinline__ uint32_t kv4_quantise8(uint4 raw, uint32_t& word) {
  const uint32_t u[4] = {raw.x, raw.y, raw.z, raw.w};
  float x[8];
  bool odd = false;                                   // a NaN or an infinity
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16lo(u[i]);
    x[2 * i + 1] = bf16hi(u[i]);
    odd |= (u[i] & 0x7F80u) == 0x7F80u || (u[i] & 0x7F800000u) == 0x7F800000u;
  }
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) { lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]); }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const float range = __fsub_rn(hi, lo);
  odd |= !(range <= 3.402823466e38f);
  const uint32_t lane = threadIdx.x & 31;
  odd = ((__ballot_sync(0xffffffffu, odd) >> (lane & 24)) & 0xFFu) != 0;
  const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(range, 15.f));
  const float s = __bfloat162float(sb);
  const bool flat = odd || !(s >= 1.17549435e-38f);
  const float inv = flat ? 0.f : __frcp_rn(s);
  uint32_t code = 0;
  if (!flat) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // t = nearest integer in the low bits of (v + 2^23); v >= 0, and above 15 only by the rounding of s
      const float v = fminf(__fmul_rn(__fsub_rn(x[i], lo), inv), 15.f);
      code |= (__float_as_uint(__fadd_rn(v, 8388608.f)) & 15u) << (4 * i);
    }
  }
  word = odd ? 0x7FC00000u
             : (uint32_t)__bfloat16_as_ushort(sb) | ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(lo)) << 16);
  return code;
}

// Stores what kv4_quantise8 gave for lane `l` (0 .. D/8 - 1: dims 8 l .. 8 l + 7) of row `row` of the tile at `tile`;
// is_v picks the tensor.  No byte of another row is written.
template <int D> __device__ __forceinline__ void kv4_store8(uint8_t* tile, int row, int l, bool is_v, uint32_t code, uint32_t word) {
  const int g = l >> 3;
  if (is_v) {
    uint16_t* to = reinterpret_cast<uint16_t*>(tile + kv4_v_off<D>(row >> 1, 8 * l)) + (row & 1);
    to[0] = (uint16_t)code;
    to[2] = (uint16_t)(code >> 16);
  } else {
    *reinterpret_cast<uint32_t*>(tile + kv4_k_off<D>(row, g) + 4 * (l & 7)) = code;
  }
  if ((l & 7) == 0)
    *reinterpret_cast<uint32_t*>(tile + (is_v ? Kv4<D>::VM : Kv4<D>::KM) + (row * Kv4<D>::NG + g) * 4) = word;
}
// The codes that it stored.
template <int D> __device__ __forceinline__ uint32_t kv4_load8(const uint8_t* tile, int row, int l, bool is_v) {
  if (!is_v) return __ldg(reinterpret_cast<const uint32_t*>(tile + kv4_k_off<D>(row, l >> 3) + 4 * (l & 7)));
  const uint2 w = __ldg(reinterpret_cast<const uint2*>(tile + kv4_v_off<D>(row >> 1, 8 * l)));
  return __byte_perm(w.x, w.y, (row & 1) ? 0x7632 : 0x5410);
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
