// wq_tc.cuh -- what the tcgen05 attention kernels share: TMEM stores, products with an
// operand from TMEM, their descriptors, and codes converted for shared memory.
#pragma once

#include <cuda_fp16.h>

#include <cstdint>

#include "wq_cvt.cuh"
#include "wq_frag.cuh"
#include "wq_ptx.cuh"

namespace wq {

// Barrier `id` over `count` threads: whether `v` holds for all of them.
__device__ __forceinline__ bool barrier_and(int id, int count, bool v) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %3, 0;\n barrier.cta.red.and.pred q, %1, %2, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"(id), "r"(count), "r"((uint32_t)v)
      : "memory");
  return r != 0;
}
// 2^e, -126 <= e <= 127
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// 32 lanes x 16 consecutive 32-bit TMEM columns, written.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
// 32 lanes x 8 columns.
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]),
               "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// Waits for this thread's loads from TMEM; v, of one of them, is not used before.
__device__ __forceinline__ void tmem_ld_wait16(float (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                 "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D (TMEM) = A (TMEM) * B (+ D when `accumulate`), issued by one thread.
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The products and their commit for a warp that runs its loop as one, issued by the lane with `lead` set (elect_one, once):
// descriptors are then the warp's, and held in uniform registers.
__device__ __forceinline__ void umma_ss_lead(uint32_t lead, uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void umma_ts_lead(uint32_t lead, uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void umma_commit_lead(uint32_t lead, uint64_t *bar) {
  asm volatile(
      "{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n"
      " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(smem_addr(bar)),
      "r"(lead)
      : "memory");
}
// B operand [k][n] with n contiguous (MN-major), 128-byte swizzle: blocks of 64 n
// `lbo` bytes apart, groups of 8 k 1024 bytes apart.
__device__ __forceinline__ uint64_t umma_desc_mnmajor_sw128(uint32_t saddr, uint32_t lbo) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// fp32 accumulator, A and B binary16 or bf16, A K-major, B K-major or MN-major.
__host__ __device__ constexpr uint32_t attn_idesc(int N, bool bf16, bool b_mn) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(128 >> 4) << 24);
}

// 2^(m - mn) for a maximum raised from m to mn (whole numbers, or infinite).
__device__ __forceinline__ float raise_factor(float m, float mn) {
  const float d = m - mn;
  return mn == m ? 1.f : d < -126.f ? 0.f : pow2i((int)d);
}
// 8 codes as 8 binary16 values code - z; z1024: 1024 + z in both halves.
template <int BITS>
__device__ __forceinline__ uint4 convert8(const uint2 &c, uint32_t z1024) {
  uint4 o;
  if constexpr (BITS == 8) {
    o.x = hsub2_u(__byte_perm(c.x, 0x64646464u, 0x4140), z1024);
    o.y = hsub2_u(__byte_perm(c.x, 0x64646464u, 0x4342), z1024);
    o.z = hsub2_u(__byte_perm(c.y, 0x64646464u, 0x4140), z1024);
    o.w = hsub2_u(__byte_perm(c.y, 0x64646464u, 0x4342), z1024);
  } else {
    // 64 + z from 1024 + z: exact (z <= 15)
    const uint32_t z64 = hsub2_u(z1024, 0x63806380u);  // 960
    const uint32_t x = c.x >> 8;
    o.x = hsub2_u(plus1024<0x000f000fu>(c.x), z1024);
    o.y = hfma16_u(plus1024<0x00f000f0u>(c.x), z64);
    o.z = hsub2_u(plus1024<0x000f000fu>(x), z1024);
    o.w = hfma16_u(plus1024<0x00f000f0u>(x), z64);
  }
  return o;
}

}  // namespace wq
