// The softmax of a score tile in which a thread holds a whole row in registers, and what the warps around it use: shared by the
// tensor-core attention kernels over packed prompts (attn_packed_tc.cu) and over a paged cache (attn_tree_tc.cu).
#pragma once

#include "attn_prefill_softmax.cuh"

namespace dl {

constexpr float kPkFar = 1048576.f, kPkFarLog2 = 14.f; // a half row's sum, and a score's lead, above which the maximum is looked for again
constexpr int kPkNext = 16;                            // pair of columns (of 64) behind which the other lane's pass may start
constexpr int kPkAhead = 4, kPkBehind = 6, kPkRing = 12;   // pairs between the stages of the exponentials
static_assert(kPkRing > kPkAhead + kPkBehind, "a pair's place is taken again before it is done");

// True in one lane of the (whole) warp, always the same one; code under it counts as warp-uniform for the compiler.
__device__ __forceinline__ bool pk_elect() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

// Maximum of three that stays where it stands: as plain arithmetic on loop-invariant scores the compiler moves the search
// for the maximum in front of the loop it is a rare part of, and every tile pays for it.
__device__ __forceinline__ float pk_max3(float x, float y, float z) {
  float r;
  asm volatile("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}

// Waits for this warp's tensor-memory loads; the 64 registers are operands, so that nothing that reads them can move in
// front of the wait.
__device__ __forceinline__ void pk_ld_wait64(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]), "+r"(r[32]), "+r"(r[33]), "+r"(r[34]), "+r"(r[35]), "+r"(r[36]), "+r"(r[37]), "+r"(r[38]), "+r"(r[39]), "+r"(r[40]), "+r"(r[41]), "+r"(r[42]), "+r"(r[43]), "+r"(r[44]), "+r"(r[45]), "+r"(r[46]), "+r"(r[47]), "+r"(r[48]), "+r"(r[49]), "+r"(r[50]), "+r"(r[51]), "+r"(r[52]), "+r"(r[53]), "+r"(r[54]), "+r"(r[55]), "+r"(r[56]), "+r"(r[57]), "+r"(r[58]), "+r"(r[59]), "+r"(r[60]), "+r"(r[61]), "+r"(r[62]), "+r"(r[63]) :: "memory");
}

// The softmax of a score tile that every row of the warp sees whole: one row per thread, its 128 scores in registers, P (as
// bf16 pairs) over the first half of the score buffer; `half` is called when the first 64 columns of P are there, so that
// their products may start, `next` when the other lane's pass may.  A row's maximum takes a warp as long as a third of the
// exponentials, so it is only looked for in an item's first tile.  After that the exponentials are taken relative to the
// maximum in use, and the tile is done over with a new one only if a score has passed it by far: the sum of the first half
// shows that (an overflow is an infinite sum), and the second half's maximum, found beside the first half's exponentials.
// P keeps its relative accuracy at any size.
template <typename Turn, typename Half, typename Next>
__device__ __forceinline__ void pk_softmax_full(uint32_t s_addr, uint32_t o_addr, bool owned, int o_blocks, float scale_log2,
                                                float& m_used, float& l_run, Turn turn, Half half, Next next) {
  uint32_t s[128];
  tmem_ld64(s_addr, s);
  tmem_ld64(s_addr + 64, s + 64);
  pk_ld_wait64(s);
  pk_ld_wait64(s + 64);
  turn();
  bool look = o_blocks == 0;
  float t[2 * kPkRing];
  const uint64_t sc2 = pack2(scale_log2, scale_log2);
redo:
  if (look) {
    float mx[8];
#pragma unroll
    for (int w = 0; w < 8; ++w) mx[w] = pk_max3(-INFINITY, __uint_as_float(s[2 * w]), __uint_as_float(s[2 * w + 1]));
#pragma unroll
    for (int c = 16; c < 128; c += 16)
#pragma unroll
      for (int w = 0; w < 8; ++w) mx[w] = pk_max3(mx[w], __uint_as_float(s[c + 2 * w]), __uint_as_float(s[c + 2 * w + 1]));
    const float mc = pk_max3(pk_max3(mx[0], mx[1], mx[2]), pk_max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * scale_log2;
    const bool need = owned && mc > m_used;
    const float corr = need ? fast_exp2(m_used - mc) : 1.0f;
    if (need) m_used = mc;
    l_run *= corr;
    if (o_blocks > 0) at_rescale_row(o_addr, s_addr, 0, corr, o_blocks);
  }
  const uint64_t nm2 = pack2(-m_used, -m_used);
  uint64_t l2[4] = {0ull, 0ull, 0ull, 0ull};
  float far[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  uint32_t pk[16];
  // Three stages, pair by pair and a few pairs apart, so that the special-function unit (8 cycles for a warp's
  // exponential) does not wait for the arithmetic in front of it or behind it.
#pragma unroll
  for (int i = 0; i < 64 + kPkAhead + kPkBehind; ++i) {
    if (i < 64) {
      float y0, y1;
      unpack2(ffma2(pack2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), sc2, nm2), y0, y1);
      t[(2 * i) % (2 * kPkRing)] = y0;
      t[(2 * i + 1) % (2 * kPkRing)] = y1;
    }
    if (i < 32) far[i & 3] = pk_max3(far[i & 3], __uint_as_float(s[64 + 2 * i]), __uint_as_float(s[64 + 2 * i + 1]));
    const int e = i - kPkAhead;
    if (e >= 0 && e < 64) {
      float& e0 = t[(2 * e) % (2 * kPkRing)];
      float& e1 = t[(2 * e + 1) % (2 * kPkRing)];
      e0 = fast_exp2(e0);
      e1 = fast_exp2(e1);
    }
    const int c = e - kPkBehind;
    if (c >= 0) {
      const float e0 = t[(2 * c) % (2 * kPkRing)], e1 = t[(2 * c + 1) % (2 * kPkRing)];
      l2[c & 3] = fadd2(l2[c & 3], pack2(e0, e1));
      pk[c & 15] = cvt_bf16x2(e0, e1);
      if ((c & 15) == 15) tmem_st16(s_addr + (c & ~15), pk);
      if (c == 32) {
        float la, lb;
        unpack2(fadd2(fadd2(l2[0], l2[1]), fadd2(l2[2], l2[3])), la, lb);
        const float ahead = fmaxf(fmaxf(far[0], far[1]), fmaxf(far[2], far[3])) * scale_log2 - m_used;
        if (__any_sync(0xffffffffu, owned && !look && (la + lb > kPkFar || ahead > kPkFarLog2))) {
          look = true;
          goto redo;
        }
      }
      if (c == 38) { tmem_st_wait(); half(); }
      if (c == kPkNext) next();
    }
  }
  float la, lb;
  unpack2(fadd2(fadd2(l2[0], l2[1]), fadd2(l2[2], l2[3])), la, lb);
  l_run += la + lb;
  tmem_st_wait();
}

}  // namespace dl
