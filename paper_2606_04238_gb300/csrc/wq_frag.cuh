// wq_frag.cuh -- MMA fragments of cached rows: how a lane of an mma.sync attention kernel
// holds the bytes of K and V rows of 16, 8 or 4 bits, and the binary16 (bf16) operands that
// it makes of them in registers.
#pragma once

#include <cstdint>

#include "wq_cvt.cuh"

namespace wq {

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const void *p) {
  static_assert(N == 1 || N == 2 || N == 4, "");
  if constexpr (N == 4) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    w[0] = v.x, w[1] = v.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t *>(p);
  }
}

// How a lane holds a cached row.  K: lane t of a position's four holds KI
// pieces of KW words, piece i at byte i * 64 + t * 4 KW.  V: lane n of a
// position's eight holds VI pieces of VW words, piece i at byte i * 128 + n * 4 VW.
template <int HD, int BITS>
struct RowLay {
  static constexpr int ROW = HD * BITS / 8;                     // bytes a row
  static constexpr int KW = ROW / 4 >= 16 ? 4 : ROW / 16, KI = ROW / (16 * KW);
  static constexpr int VW = ROW / 8 >= 16 ? 4 : ROW / 32, VI = ROW / (32 * VW);
  static constexpr int KS = HD / 16;                            // MMA steps along HD
  static constexpr int NJ = HD / 8;                             // 8-column tiles of the output
  // first of the four values that lane t gives MMA step ks
  static __device__ __forceinline__ int q_at(int ks, int t) {
    constexpr int PER = KW * 4 * 8 / BITS;                      // values a piece
    return (4 * ks / PER) * (4 * PER) + t * PER + 4 * ks % PER;
  }
  // value of column n of output tile j
  static __device__ __forceinline__ int v_at(int j, int n) {
    constexpr int PER = VW * 4 * 8 / BITS;
    return (j / PER) * (8 * PER) + n * PER + j % PER;
  }
};

// The codes of MASK in x as binary16 1024 + code (64 + code in bits 4 to 7).  One instruction: a second constant would be
// a second one, so 1024 is a register that the compiler does not know the value of.
template <uint32_t MASK>
__device__ __forceinline__ uint32_t plus1024(uint32_t x) {
  uint32_t k, v;
  asm("mov.b32 %0, 0x64006400;" : "=r"(k));
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(v) : "r"(x), "n"(MASK), "r"(k));  // (x & MASK) | k
  return v;
}
// The fragments (b0, b1) of MMA step ks from a lane's words of one K row; zk: z
// in both halves, as 1024 + z (8 bits, low), and 64 + z (4 bits, high).
template <int HD, int BITS>
__device__ __forceinline__ void k_frag(const uint32_t (&w)[RowLay<HD, BITS>::KI * RowLay<HD, BITS>::KW], int ks, uint32_t z1024,
                                       uint32_t z64, uint32_t &b0, uint32_t &b1) {
  if constexpr (BITS == 16) {
    b0 = w[2 * ks];
    b1 = w[2 * ks + 1];
  } else if constexpr (BITS == 8) {
    b0 = hsub2_u(__byte_perm(w[ks], 0x64646464u, 0x4140), z1024);
    b1 = hsub2_u(__byte_perm(w[ks], 0x64646464u, 0x4342), z1024);
  } else {
    const uint32_t x = ks % 2 ? w[ks / 2] >> 8 : w[ks / 2];
    b0 = hsub2_u(plus1024<0x000f000fu>(x), z1024);
    b1 = hfma16_u(plus1024<0x00f000f0u>(x), z64);
  }
}

// Output tile j's fragment half from a lane's words of two V rows (the lower
// position in the low halves); z1024, z64 hold their two zeros.
template <int HD, int BITS>
__device__ __forceinline__ uint32_t v_frag(const uint32_t (&wa)[RowLay<HD, BITS>::VI * RowLay<HD, BITS>::VW],
                                           const uint32_t (&wb)[RowLay<HD, BITS>::VI * RowLay<HD, BITS>::VW], int j,
                                           uint32_t z1024, uint32_t z64) {
  if constexpr (BITS == 16) {
    return __byte_perm(wa[j / 2], wb[j / 2], j % 2 ? 0x7632 : 0x5410);
  } else if constexpr (BITS == 8) {
    const uint32_t x = __byte_perm(wa[j / 4], wb[j / 4], j % 4 / 2 ? 0x7362 : 0x5140);
    return hsub2_u(__byte_perm(x, 0x64646464u, j % 2 ? 0x4342 : 0x4140), z1024);
  } else {
    // value e of a word: bits 4 (e / 2) + 16 (e % 2)
    uint32_t x = __byte_perm(wa[j / 8], wb[j / 8], j % 2 ? 0x7632 : 0x5410);
    const int nib = j % 8 / 2;
    if (nib >= 2) x >>= 8;
    return nib % 2 ? hfma16_u(plus1024<0x00f000f0u>(x), z64) : hsub2_u(plus1024<0x000f000fu>(x), z1024);
  }
}

__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace wq
