// wq_rows.cuh -- rows of a KV cache (one position's K or V of one kv head) as the
// kernels that write and read them share them: the quantizer, the codes' packing, a row
// read back; and launches of one row a few lanes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "wq_cvt.cuh"
#include "wq_kv.h"
#include "wq_ptx.cuh"

namespace wq {

// Quotients by a divisor of the whole launch: x d' >> (31 + l), l = ceil(log2 d), d' the
// whole number above 2^(31 + l) / d, too large by at most 1: exact for x below 2^31.
struct Divisor {
  unsigned d, mul;
  int shift;
  explicit Divisor(int by) : d((unsigned)by), shift(31) {
    while ((1u << (shift - 31)) < d) ++shift;
    mul = (unsigned)((1ull << shift) / d + 1);
  }
  __device__ __forceinline__ unsigned divide(unsigned x) const { return (unsigned)((unsigned long long)x * mul >> shift); }
};

// 16 values of a row whose range around 0 is mn .. mx: the row's scale and zero as a
// cache holds them, the values' codes, two a word.
//   With M = 1.5 2^23, v r + M rounded is M + a whole number, held in its low bits.
// r is 1 / sf made 2^-22 larger and 2^-22 smaller: v / sf and its rounding to fp32 lie
// between the two products, so that where both give the same whole number it is the
// quotient's; else (a half, or within 2^-21 of its size of one: in 5% of rows of normal
// bf16 values in 4 bits, for 8 bits 0.2%) the pair is divided.
// A product is below 2^9, since sf is at least two thirds of range / qmax.
template <int BITS>
__device__ __forceinline__ uint32_t quantize16(const float (&v)[16], float mn, float mx, uint32_t (&c)[8]) {
  constexpr float qmax = (float)((1 << BITS) - 1), M = 12582912.f;
  __half sh = __float2half_rn(__fdiv_rn(__fsub_rn(mx, mn), qmax));
  if (__half2float(sh) == 0.f) {  // no value is above 2^-25 qmax: codes and zero point 0
#pragma unroll
    for (int k = 0; k < 8; ++k) c[k] = 0;
    return kZeroRow;
  }
  const float sf = __half2float(sh);
  if (!isfinite(sf)) {  // also infinite or NaN values: mx - mn is then too
#pragma unroll
    for (int k = 0; k < 8; ++k) c[k] = 0;
    return 0x7fffu;
  }
  const float zf = __fadd_rn(fminf(fmaxf(rintf(__fdiv_rn(-mn, sf)), 0.f), qmax), 0.f);
  const float rcp = __frcp_rn(sf), up = __fmul_rn(rcp, 1.f + 0x1p-22f), dn = __fmul_rn(rcp, 1.f - 0x1p-22f);
  const uint64_t up2 = pack_f32x2(up, up), dn2 = pack_f32x2(dn, dn), M2 = pack_f32x2(M, M);
  const uint32_t z2 = (uint32_t)zf * 0x10001u, q2 = (uint32_t)qmax * 0x10001u;
  uint32_t differ = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint64_t x = pack_f32x2(v[2 * k], v[2 * k + 1]), t = fma_f32x2(x, up2, M2), u = fma_f32x2(x, dn2, M2);
    const uint32_t t0 = (uint32_t)t, t1 = (uint32_t)(t >> 32);
    differ |= t0 ^ (uint32_t)u;
    differ |= t1 ^ (uint32_t)(u >> 32);
    c[k] = __viaddmin_s16x2_relu(__byte_perm(t0, t1, 0x5410), z2, q2);  // max(min(t + z, qmax), 0)
  }
  if (differ != 0) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint64_t x = pack_f32x2(v[2 * k], v[2 * k + 1]);
      if (fma_f32x2(x, up2, M2) != fma_f32x2(x, dn2, M2)) {  // (both are near 1.5 2^23: equal as numbers if as bits)
        const float t0 = __fadd_rn(rintf(__fdiv_rn(v[2 * k], sf)), zf);
        const float t1 = __fadd_rn(rintf(__fdiv_rn(v[2 * k + 1], sf)), zf);
        c[k] = (uint32_t)fminf(fmaxf(t0, 0.f), qmax) | (uint32_t)fminf(fmaxf(t1, 0.f), qmax) << 16;
      }
    }
  }
  return (uint32_t)__half_as_ushort(sh) | (uint32_t)__half_as_ushort(__float2half_rn(zf)) << 16;
}

// The codes of quantize16 as a row holds them: 8 bits in 4 words, 4 bits in 2 (value e of a
// word of 8 at bits 4 (e / 2) + 16 (e % 2)).
template <int BITS>
__device__ __forceinline__ void pack_codes(const uint32_t (&c)[8], uint32_t (&w)[BITS / 2]) {
  if constexpr (BITS == 8) {
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __byte_perm(c[2 * k], c[2 * k + 1], 0x6420);
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) w[k] = (c[4 * k] + (c[4 * k + 1] << 4)) + ((c[4 * k + 2] + (c[4 * k + 3] << 4)) << 8);
  }
}

// Row `row` of a cache as HD bf16 or fp32 values at dst + out, zeros where not `get`: lane l
// of its HD / 16.  A lane takes the values of one 16-byte store at a time (8 of bf16, 4 of
// fp32), chunks l, l + HD / 16, .. of the row, so that a row's stores are whole lines.
template <int HD, int BITS, bool F32>
__device__ __forceinline__ void read_row(const void *rows, const uint32_t *meta, size_t row, int lane, bool get, void *dst,
                                         size_t out) {
  constexpr int LPR = HD / 16, N = F32 ? 4 : 8, CH = 16 / N;  // lanes a row, values a chunk, chunks a lane
  const uint8_t *src = reinterpret_cast<const uint8_t *>(rows) + row * (HD * BITS / 8);
  float v[CH][N];
  uint32_t m = 0;
  uint32_t w[CH][4];  // a chunk's bytes (4 bits: the word it lies in)
  if (get) {
    if (BITS != 16) m = __ldcs(meta + row);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = lane + i * LPR;
      if (BITS == 16 && N == 8) {
        const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(src) + c);
        w[i][0] = q.x, w[i][1] = q.y, w[i][2] = q.z, w[i][3] = q.w;
      } else if ((BITS == 16 && N == 4) || (BITS == 8 && N == 8)) {
        const uint2 q = __ldcs(reinterpret_cast<const uint2 *>(src) + c);
        w[i][0] = q.x, w[i][1] = q.y;
      } else {
        w[i][0] = __ldcs(reinterpret_cast<const uint32_t *>(src) + (BITS == 4 && N == 4 ? c / 2 : c));
      }
    }
  }
  // code - z exactly in binary16, as (1024 + code) - (1024 + z)
  const float s = __half2float(__ushort_as_half((unsigned short)(m & 0xffffu)));
  const __half2 z = __hadd2(__half2half2(__ushort_as_half((unsigned short)(m >> 16))), __float2half2_rn(1024.f));
  auto pair = [&](uint32_t codes, float *to) {
    const uint32_t c = codes | 0x64006400u;
    const float2 f = __half22float2(__hsub2(*reinterpret_cast<const __half2 *>(&c), z));
    to[0] = __fmul_rn(s, f.x);
    to[1] = __fmul_rn(s, f.y);
  };
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      if (!get) {
        v[i][e] = v[i][e + 1] = 0.f;
      } else if (BITS == 16) {
        v[i][e] = bf_lo(w[i][e / 2]);
        v[i][e + 1] = bf_hi(w[i][e / 2]);
      } else if (BITS == 8) {
        pair(__byte_perm(w[i][e / 4], 0, e % 4 ? 0x4342 : 0x4140), &v[i][e]);
      } else {
        // value x of a word of 8 at bits 4 (x / 2) + 16 (x % 2)
        const int half = N == 4 ? lane % 2 * 8 : 0;  // (LPR is even: a lane's chunks are all first or all second halves)
        pair(w[i][0] >> (half + 2 * e) & 0x000f000fu, &v[i][e]);
      }
    }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const size_t at = out + (size_t)(lane + i * LPR) * N;
    if constexpr (F32)
      *reinterpret_cast<float4 *>(reinterpret_cast<float *>(dst) + at) = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]);
    else
      *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(dst) + at) =
          make_uint4(pack_bf2(v[i][0], v[i][1]), pack_bf2(v[i][2], v[i][3]), pack_bf2(v[i][4], v[i][5]),
                     pack_bf2(v[i][6], v[i][7]));
  }
}

// A launch that may begin while the one before it ends (the kernel waits by pdl_wait).
template <class... Params, class... Args>
cudaError_t launch_pdl(void (*k)(Params...), unsigned grid, int threads, cudaStream_t s, const Args &...args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  return cudaLaunchKernelEx(&cfg, k, args...);
}

// CTAs of a launch of one row (of hd values) per hd / 16 lanes.
inline unsigned row_ctas(long long rows, int hd, int threads) {
  const long long per = threads / (hd / 16);
  return (unsigned)((rows + per - 1) / per);
}

}  // namespace wq
