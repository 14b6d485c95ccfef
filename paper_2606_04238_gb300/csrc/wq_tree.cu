// wq_tree.cu -- attention of a tree of drafted tokens over a KV cache (sm_103a):
// the verify step of speculative decoding, and with one draft a decode step over
// a quantized cache.
//
// Per sequence b and kv head g, row r = t rep + h stands for draft t and query
// head g rep + h (rep = H / Hkv).  It attends to the cached positions 0 ..
// lens[b] - 1 and to the drafts j with bit j of mask[b][t] (their K and V are
// bf16 rows of their own and not in the cache yet):
//   x_j = scale log2(e) (q . k_j),  o = sum_j 2^(x_j - m) v_j / sum_j 2^(x_j - m).
// A cached row of 8 or 4 bits is s (code - z) with one scale and one whole zero
// point (wq_kv.cu), and code - z is exact in binary16.  So K's scale multiplies
// the score, and V's scale is taken into the exponent:
//   y_j = x_j + log2 s_j,  p_j = 2^(y_j - m),  o = sum_j p_j (code - z)_j / sum_j p_j / s_j,
// with m the running maximum of y.  p_j then fills binary16's range whatever V's
// scales are; p_j (bf16 for a bf16 cache) and q (bf16 given; for a quantized
// cache binary16 with an exact power of two a row) are the products' only other
// 16-bit operands, all sums and softmax statistics fp32.  Rounding p costs 2^-11
// (binary16) or 2^-8 (bf16) of each term at most, of either sign; the bf16 store of
// o costs as much of their sum.
//
// A CTA of 4 warps takes one (b, g), 16 rows and one split of the context; each
// warp takes chunks of 16 (4 bits: 32) positions with mma.sync m16n8k16, rows as
// M.  Codes go from global memory to the MMA fragments through registers alone:
// the contraction over HD and the order of V's columns are free, so a lane takes
// 16 consecutive bytes of its position's row, and two prmt or and-or build the
// binary16 value 1024 + code, from which 1024 + z is subtracted (exact).  The
// next chunk's K is loaded when the current one's has been converted, V likewise.
// The drafts' chunks run first, in bf16.  The splits' partial results are merged
// in a fixed order by a second kernel (none with one split).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "wq_internal.h"
#include "wq_kv.h"
#include "wq_ptx.cuh"

namespace wq {

// Status word: WQ_OK (0), or WQ_ERR_ARG (-1) after a length outside [0,
// max_len] or a count outside [0, T] was met (that sequence is skipped).
__device__ int g_tree_status = 0;

namespace {

constexpr int kTreeWarps = 4;
constexpr int kRows = 16;  // rows a CTA takes

__device__ __forceinline__ uint32_t pack_bf2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack_h2(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t hsub2_u(uint32_t a, uint32_t b) {
  const __half2 v = __hsub2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&v);
}
// a / 16 - b
__device__ __forceinline__ uint32_t hfma16_u(uint32_t a, uint32_t b) {
  const uint32_t k = 0x2c002c00u;  // 1/16, 1/16
  const __half2 v = __hfma2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&k),
                            __hneg2(*reinterpret_cast<const __half2 *>(&b)));
  return *reinterpret_cast<const uint32_t *>(&v);
}
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const void *p) {
  static_assert(N == 1 || N == 2 || N == 4, "");
  if constexpr (N == 4) {
    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else if constexpr (N == 2) {
    const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
    w[0] = v.x, w[1] = v.y;
  } else {
    w[0] = __ldg(reinterpret_cast<const uint32_t *>(p));
  }
}

// How a lane holds a cached row.  K: lane t of a position's four holds KI
// pieces of KW words, piece i at byte i * 64 + t * 4 KW.  V: lane n of a
// position's eight holds VI pieces of VW words, piece i at byte i * 128 + n * 4 VW.
template <int HD, int BITS>
struct Lay {
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

// The fragments (b0, b1) of MMA step ks from a lane's words of one K row; zk: z
// in both halves, as 1024 + z (8 bits, low), and 64 + z (4 bits, high).
template <int HD, int BITS>
__device__ __forceinline__ void k_frag(const uint32_t (&w)[Lay<HD, BITS>::KI * Lay<HD, BITS>::KW], int ks, uint32_t z1024,
                                       uint32_t z64, uint32_t &b0, uint32_t &b1) {
  if constexpr (BITS == 16) {
    b0 = w[2 * ks];
    b1 = w[2 * ks + 1];
  } else if constexpr (BITS == 8) {
    b0 = hsub2_u(__byte_perm(w[ks], 0x64646464u, 0x4140), z1024);
    b1 = hsub2_u(__byte_perm(w[ks], 0x64646464u, 0x4342), z1024);
  } else {
    const uint32_t x = ks % 2 ? w[ks / 2] >> 8 : w[ks / 2];
    b0 = hsub2_u((x & 0x000f000fu) | 0x64006400u, z1024);
    b1 = hfma16_u((x & 0x00f000f0u) | 0x64006400u, z64);
  }
}

// Output tile j's fragment half from a lane's words of two V rows (the lower
// position in the low halves); z1024, z64 hold their two zeros.
template <int HD, int BITS>
__device__ __forceinline__ uint32_t v_frag(const uint32_t (&wa)[Lay<HD, BITS>::VI * Lay<HD, BITS>::VW],
                                           const uint32_t (&wb)[Lay<HD, BITS>::VI * Lay<HD, BITS>::VW], int j,
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
    return nib % 2 ? hfma16_u((x & 0x00f000f0u) | 0x64006400u, z64) : hsub2_u((x & 0x000f000fu) | 0x64006400u, z1024);
  }
}

// What a warp accumulates: rows gr and gr + 8 of its 16, columns v_at(j, 2 tc),
// v_at(j, 2 tc + 1); m the rows' maximum of y, l this lane's part of their sums.
template <int HD>
struct Acc {
  float o[HD / 8][4];
  float m[2], l[2];
};

// y[u][e]: scores of positions 8 u + 2 tc + e % 2 and row gr + 8 (e / 2), -inf
// where masked.  Leaves p (fp32) in y and the accumulators rescaled.
template <int HD, int NT>
__device__ __forceinline__ void softmax_step(Acc<HD> &acc, float (&y)[NT][4]) {
  float mc[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) mc[e / 2] = fmaxf(mc[e / 2], y[u][e]);
  float ms[2], al[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    mc[i] = fmaxf(mc[i], __shfl_xor_sync(0xffffffffu, mc[i], 1));
    mc[i] = fmaxf(mc[i], __shfl_xor_sync(0xffffffffu, mc[i], 2));
    const float mn = fmaxf(acc.m[i], mc[i]);
    ms[i] = mn == -INFINITY ? 0.f : mn;
    al[i] = exp2f(acc.m[i] - ms[i]);  // 0 at first (m = -inf)
    acc.m[i] = mn;
  }
  if (__any_sync(0xffffffffu, al[0] != 1.f || al[1] != 1.f)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) acc.l[i] *= al[i];
#pragma unroll
    for (int j = 0; j < HD / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc.o[j][e] *= al[e / 2];
  }
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) y[u][e] = exp2f(y[u][e] - ms[e / 2]);
}

// q's fragments: rows gr, gr + 8 of the CTA's 16; -1: a row of zeros.
template <int HD, int BITS>
__device__ __forceinline__ void load_q(uint32_t (&qa)[HD / 16][4], float (&qf)[2], const __nv_bfloat16 *q0,
                                       const __nv_bfloat16 *q1, int tc, float scale) {
  using L = Lay<HD, BITS>;
  float mx[2] = {0.f, 0.f};
#pragma unroll
  for (int ks = 0; ks < L::KS; ++ks) {
    const int at = L::q_at(ks, tc);
    const uint2 a = q0 ? __ldg(reinterpret_cast<const uint2 *>(q0 + at)) : make_uint2(0, 0);
    const uint2 b = q1 ? __ldg(reinterpret_cast<const uint2 *>(q1 + at)) : make_uint2(0, 0);
    qa[ks][0] = a.x, qa[ks][1] = b.x, qa[ks][2] = a.y, qa[ks][3] = b.y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mx[i % 2] = fmaxf(mx[i % 2], fabsf(bf_lo(qa[ks][i])));
      mx[i % 2] = fmaxf(mx[i % 2], fabsf(bf_hi(qa[ks][i])));
    }
  }
  qf[0] = qf[1] = scale;
  if constexpr (BITS != 16) {
    // an exact power of two puts the row's largest value in [2^14, 2^15): what
    // binary16 then loses is below 2^-38 of it
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
      mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
    }
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // exponent of mx, kept where 2^e and 2^-e are normal; 0 and inf: 1
      const int e = (int)(__float_as_uint(mx[i]) >> 23) - 127;
      const int sh = e == 128 || mx[i] == 0.f ? 0 : min(126, max(-100, 14 - e));
      f[i] = __uint_as_float((uint32_t)(127 + sh) << 23);
      qf[i] = scale * __uint_as_float((uint32_t)(127 - sh) << 23);
    }
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i) qa[ks][i] = pack_h2(bf_lo(qa[ks][i]) * f[i % 2], bf_hi(qa[ks][i]) * f[i % 2]);
  }
}

}  // namespace

// Where lane tc's output columns go: Lay<HD, BITS> of the context's V for the
// cache's chunks, Lay<HD, 16> for the drafts'.  Both orders differ for a
// quantized cache, so a draft's V is fetched in the cache's order (value by
// value: at most T rows).
template <int HD, int BITS>
__global__ void __launch_bounds__(kTreeWarps * 32, 2) attn_tree_kernel(const TreeArgs a) {
  using L = Lay<HD, BITS>;
  using L16 = Lay<HD, 16>;
  constexpr int NC = BITS == 4 ? 2 : 1, CHP = 16 * NC;  // 16-position groups a chunk
  constexpr int OS = HD + 4;
  __shared__ __align__(16) float so[kTreeWarps][kRows][OS];
  __shared__ float sm[kTreeWarps][kRows], sl[kTreeWarps][kRows];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gr = lane >> 2, tc = lane & 3;
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, split = blockIdx.y, r0 = blockIdx.z * kRows;
  const int rep = a.H / a.Hkv, R = a.T * rep;
  const int len = a.lens[b], cnt = a.counts ? a.counts[b] : a.T;
  if (len < 0 || len > a.max_len || cnt < 0 || cnt > a.T) {
    if (tid == 0 && g == 0 && split == 0 && r0 == 0) atomicExch(&g_tree_status, -1);
    return;
  }
  // units of this split: chunks of drafts, then of the context
  const int ndr = (cnt + 15) / 16, U = ndr + (len + CHP - 1) / CHP;
  const int u0 = (int)((long long)U * split / a.S), u1 = (int)((long long)U * (split + 1) / a.S);
  const int ra = r0 + gr, rb = ra + 8;
  const int ta = ra / rep, tb = rb / rep;  // the rows' drafts
  const bool ina = ra < R && ta < cnt, inb = rb < R && tb < cnt;
  const __nv_bfloat16 *qbase = reinterpret_cast<const __nv_bfloat16 *>(a.q);
  const __nv_bfloat16 *qa_p = ina ? qbase + (((size_t)b * a.T + ta) * a.H + g * rep + ra % rep) * HD : nullptr;
  const __nv_bfloat16 *qb_p = inb ? qbase + (((size_t)b * a.T + tb) * a.H + g * rep + rb % rep) * HD : nullptr;

  Acc<HD> acc;
#pragma unroll
  for (int j = 0; j < HD / 8; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc.o[j][e] = 0.f;
  acc.m[0] = acc.m[1] = -INFINITY;
  acc.l[0] = acc.l[1] = 0.f;
  uint32_t qa[L::KS][4];
  float qf[2];

  // ---- drafts
  int u = u0 + warp;
  const size_t dstride = (size_t)a.Hkv * HD;
  const __nv_bfloat16 *kd = reinterpret_cast<const __nv_bfloat16 *>(a.kn) + ((size_t)b * a.T * a.Hkv + g) * HD;
  const __nv_bfloat16 *vd = reinterpret_cast<const __nv_bfloat16 *>(a.vn) + ((size_t)b * a.T * a.Hkv + g) * HD;
  if (u < min(u1, ndr)) {
    load_q<HD, 16>(qa, qf, qa_p, qb_p, tc, a.scale);
    for (; u < min(u1, ndr); u += kTreeWarps) {
      const int j0 = u * 16, n = min(16, cnt - j0);
      float y[2][4];
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        uint32_t w[L16::KI * L16::KW];
        const int j = min(j0 + 8 * v + gr, cnt - 1);
#pragma unroll
        for (int i = 0; i < L16::KI; ++i)
          load_words(*reinterpret_cast<uint32_t(*)[4]>(&w[4 * i]), kd + j * dstride + i * 32 + tc * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[v][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < L::KS; ++ks) mma_bf16_16816(y[v], qa[ks], w[2 * ks], w[2 * ks + 1]);
      }
      uint32_t see[2] = {0, 0};  // bits: drafts j0 .. j0 + 15 that rows gr, gr + 8 see
      const uint32_t have = n >= 16 ? 0xffffu : (1u << n) - 1u;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int t = i ? tb : ta;
        if (!(i ? inb : ina)) continue;
        if (a.mask)
          see[i] = a.mask[((size_t)b * a.T + t) * a.words + j0 / 32] >> (j0 % 32) & have;
        else
          see[i] = t >= j0 + 15 ? have : t < j0 ? 0u : ((2u << (t - j0)) - 1u) & have;
      }
#pragma unroll
      for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          y[v][e] = see[e / 2] >> (8 * v + 2 * tc + e % 2) & 1 ? y[v][e] * qf[e / 2] : -INFINITY;
      softmax_step<HD, 2>(acc, y);
      uint32_t pf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) pf[i] = pack_bf2(y[i / 2][2 * (i % 2)], y[i / 2][2 * (i % 2) + 1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) acc.l[i] += (y[0][2 * i] + y[0][2 * i + 1]) + (y[1][2 * i] + y[1][2 * i + 1]);
      bool odd = false;
#pragma unroll
      for (int j = 0; j < L::NJ; ++j) {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = 8 * (i / 2) + 2 * tc + i % 2;
          uint32_t x = 0;
          if (p < n) x = __bfloat16_as_ushort(vd[(size_t)(j0 + p) * dstride + L::v_at(j, gr)]);
          if ((x & 0x7f80u) == 0x7f80u) {
            x = 0;
            odd = true;
          }
          h[i] = x;
        }
        mma_bf16_16816(acc.o[j], pf, h[0] | h[1] << 16, h[2] | h[3] << 16);
      }
      if (__any_sync(0xffffffffu, odd)) {
        for (int p = 0; p < n; ++p)
#pragma unroll
          for (int j = 0; j < L::NJ; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float x = __bfloat162float(vd[(size_t)(j0 + p) * dstride + L::v_at(j, 2 * tc + e)]);
              if (isfinite(x)) continue;
              if (see[0] >> p & 1) acc.o[j][e] += x;
              if (see[1] >> p & 1) acc.o[j][2 + e] += x;
            }
      }
    }
  }

  // ---- context
  if (u < u1) {
    load_q<HD, BITS>(qa, qf, qa_p, qb_p, tc, a.scale);
    const size_t base = ((size_t)b * a.Hkv + g) * a.max_len;
    const uint8_t *kc = reinterpret_cast<const uint8_t *>(a.kc) + base * L::ROW;
    const uint8_t *vc = reinterpret_cast<const uint8_t *>(a.vc) + base * L::ROW;
    uint32_t kw[NC][2][L::KI * L::KW], vw[NC][4][L::VI * L::VW], meta[NC];
    auto load_k = [&](int p0) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int p = min(p0 + 16 * c + 8 * v + gr, len - 1);
#pragma unroll
          for (int i = 0; i < L::KI; ++i)
            load_words(*reinterpret_cast<uint32_t(*)[L::KW]>(&kw[c][v][L::KW * i]),
                       kc + (size_t)p * L::ROW + i * 64 + tc * 4 * L::KW);
        }
    };
    auto load_v = [&](int p0) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int p = min(p0 + 16 * c + 8 * (v / 2) + 2 * tc + v % 2, len - 1);
#pragma unroll
          for (int i = 0; i < L::VI; ++i)
            load_words(*reinterpret_cast<uint32_t(*)[L::VW]>(&vw[c][v][L::VW * i]),
                       vc + (size_t)p * L::ROW + i * 128 + gr * 4 * L::VW);
        }
    };
    auto load_meta = [&](int p0) {  // lanes 0-15: K's, 16-31: V's
      if constexpr (BITS != 16)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          meta[c] = __ldg((lane < 16 ? a.km : a.vm) + base + min(p0 + 16 * c + (lane & 15), len - 1));
    };
    int p0 = (u - ndr) * CHP;
    load_k(p0);
    load_meta(p0);
    load_v(p0);
    for (; u < u1; u += kTreeWarps, p0 += kTreeWarps * CHP) {
      const int pn = u + kTreeWarps < u1 ? p0 + kTreeWarps * CHP : p0;  // past the end: the same rows again
      float y[2 * NC][4];
      uint32_t mk[NC], mv[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) mk[c] = mv[c] = meta[c];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          uint32_t z1 = 0, z6 = 0;
          if constexpr (BITS != 16) {
            const uint32_t m = __shfl_sync(0xffffffffu, mk[c], 8 * v + gr);
            const __half z = __ushort_as_half((unsigned short)(m >> 16));
            const __half2 zz = __half2half2(z);
            const __half2 k1 = __hadd2(zz, __float2half2_rn(1024.f)), k6 = __hadd2(zz, __float2half2_rn(64.f));
            z1 = *reinterpret_cast<const uint32_t *>(&k1);
            z6 = *reinterpret_cast<const uint32_t *>(&k6);
          }
          float *yy = y[2 * c + v];
#pragma unroll
          for (int e = 0; e < 4; ++e) yy[e] = 0.f;
#pragma unroll
          for (int ks = 0; ks < L::KS; ++ks) {
            uint32_t b0, b1;
            k_frag<HD, BITS>(kw[c][v], ks, z1, z6, b0, b1);
            if constexpr (BITS == 16)
              mma_bf16_16816(y[2 * c + v], qa[ks], b0, b1);
            else
              mma_f16_16816(y[2 * c + v], qa[ks], b0, b1);
          }
        }
      load_k(pn);
      float rs[NC][4];
      uint32_t zv[NC][2][2];  // [.][positions 2 tc, + 1 of 8 v ..][1024 + z, 64 + z]
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int at = 8 * (v / 2) + 2 * tc + v % 2;  // of the group's 16 positions
          const bool in = p0 + 16 * c + at < len;
          float *yy = y[2 * c + v / 2];
          if constexpr (BITS == 16) {
            yy[v % 2] = in ? yy[v % 2] * qf[0] : -INFINITY;
            yy[2 + v % 2] = in ? yy[2 + v % 2] * qf[1] : -INFINITY;
          } else {
            const uint32_t m = __shfl_sync(0xffffffffu, mk[c], at), mm = __shfl_sync(0xffffffffu, mv[c], 16 + at);
            const float sk = __half2float(__ushort_as_half((unsigned short)(m & 0xffffu)));
            float sv = __half2float(__ushort_as_half((unsigned short)(mm & 0xffffu)));
            if (sv == 0.f) sv = 1.f;  // a zero-filled cache's row: code - z is 0
            const float lg = in ? __log2f(sv) : -INFINITY;
            rs[c][v] = __frcp_rn(sv);
            yy[v % 2] = fmaf(yy[v % 2] * qf[0], sk, lg);
            yy[2 + v % 2] = fmaf(yy[2 + v % 2] * qf[1], sk, lg);
            if (!in) yy[v % 2] = yy[2 + v % 2] = -INFINITY, rs[c][v] = 0.f;
            const uint32_t zh = mm >> 16;
            if (v % 2 == 0)
              zv[c][v / 2][0] = zh;
            else
              zv[c][v / 2][0] |= zh << 16;
          }
        }
      if constexpr (BITS != 16)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const __half2 zz = *reinterpret_cast<const __half2 *>(&zv[c][v][0]);
            const __half2 k1 = __hadd2(zz, __float2half2_rn(1024.f)), k6 = __hadd2(zz, __float2half2_rn(64.f));
            zv[c][v][0] = *reinterpret_cast<const uint32_t *>(&k1);
            zv[c][v][1] = *reinterpret_cast<const uint32_t *>(&k6);
          }
      load_meta(pn);
      softmax_step<HD, 2 * NC>(acc, y);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        uint32_t pf[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = y[2 * c + i / 2][2 * (i % 2)], q = y[2 * c + i / 2][2 * (i % 2) + 1];
          pf[i] = BITS == 16 ? pack_bf2(p, q) : pack_h2(p, q);
          if constexpr (BITS == 16)
            acc.l[i % 2] += p + q;
          else
            acc.l[i % 2] += fmaf(p, rs[c][2 * (i / 2)], q * rs[c][2 * (i / 2) + 1]);
        }
#pragma unroll
        for (int j = 0; j < L::NJ; ++j) {
          uint32_t b0 = v_frag<HD, BITS>(vw[c][0], vw[c][1], j, zv[c][0][0], zv[c][0][1]);
          uint32_t b1 = v_frag<HD, BITS>(vw[c][2], vw[c][3], j, zv[c][1][0], zv[c][1][1]);
          if constexpr (BITS == 16)
            mma_bf16_16816(acc.o[j], pf, b0, b1);
          else
            mma_f16_16816(acc.o[j], pf, b0, b1);
        }
      }
      load_v(pn);
    }
  }

  // ---- the warps' results merged in warp order
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    acc.l[i] += __shfl_xor_sync(0xffffffffu, acc.l[i], 1);
    acc.l[i] += __shfl_xor_sync(0xffffffffu, acc.l[i], 2);
    if (tc == 0) {
      sm[warp][gr + 8 * i] = acc.m[i];
      sl[warp][gr + 8 * i] = acc.l[i];
    }
  }
#pragma unroll
  for (int j = 0; j < L::NJ; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) so[warp][gr + 8 * (e / 2)][L::v_at(j, 2 * tc + e % 2)] = acc.o[j][e];
  __syncthreads();
  for (int i = tid; i < kRows * HD / 2; i += kTreeWarps * 32) {
    const int r = i / (HD / 2), e = 2 * (i % (HD / 2)), row = r0 + r;
    if (row >= R) break;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kTreeWarps; ++w) M = fmaxf(M, sm[w][r]);
    float Ls = 0.f, O0 = 0.f, O1 = 0.f;
#pragma unroll
    for (int w = 0; w < kTreeWarps; ++w) {
      const float f = sm[w][r] == -INFINITY ? 0.f : exp2f(sm[w][r] - M);
      Ls = fmaf(sl[w][r], f, Ls);
      O0 = fmaf(so[w][r][e], f, O0);
      O1 = fmaf(so[w][r][e + 1], f, O1);
    }
    if (a.S == 1) {
      const int t = row / rep, h = g * rep + row % rep;
      const bool none = (M == -INFINITY && Ls == 0.f) || t >= cnt;  // sees nothing, or is padding
      *reinterpret_cast<uint32_t *>(reinterpret_cast<__nv_bfloat16 *>(a.o) + (((size_t)b * a.T + t) * a.H + h) * HD + e) =
          none ? 0u : pack_bf2(O0 / Ls, O1 / Ls);
    } else {
      float *pt = a.part + (((size_t)blockIdx.x * R + row) * a.S + split) * (HD + 2);
      *reinterpret_cast<float2 *>(pt + e) = make_float2(O0, O1);
      if (e == 0) *reinterpret_cast<float2 *>(pt + HD) = make_float2(M, Ls);
    }
  }
}

// o of one row: its splits' parts added in a fixed order by WPR warps (warp w:
// splits w, w + WPR, .. in order, then the warps in order).  grid: rows / (8 / WPR).
constexpr int kCombineWarps = 8;

template <int HD, int WPR>
__global__ void __launch_bounds__(kCombineWarps * 32) attn_tree_combine_kernel(const TreeArgs a) {
  constexpr int E = HD / 32, CU = WPR == 1 ? 4 : 8;  // splits loaded in one round trip
  __shared__ float wm[kCombineWarps], wl[kCombineWarps], wo[kCombineWarps][HD];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rep = a.H / a.Hkv, R = a.T * rep;
  const long long rows = (long long)a.batch * a.Hkv * R;
  const long long row = (long long)blockIdx.x * (kCombineWarps / WPR) + warp / WPR;
  const int sub = warp % WPR;
  pdl_wait();
  pdl_launch_dependents();
  const bool in = row < rows;
  const int bg = (int)(row / R), r = (int)(row - (long long)bg * R), b = bg / a.Hkv, g = bg % a.Hkv;
  bool skip = !in;
  int cnt = a.T;
  if (in) {
    const int len = a.lens[b];
    if (a.counts) cnt = a.counts[b];
    skip = len < 0 || len > a.max_len || cnt < 0 || cnt > a.T;
  }
  float M = -INFINITY, Ls = 0.f, O[E];
#pragma unroll
  for (int e = 0; e < E; ++e) O[e] = 0.f;
  if (!skip) {
    const float *pt = a.part + (size_t)row * a.S * (HD + 2);
    for (int s0 = sub; s0 < a.S; s0 += CU * WPR) {
      float2 ml[CU], ov[CU][E / 2];
      float mn = M;
#pragma unroll
      for (int c = 0; c < CU; ++c) {
        const int s = s0 + c * WPR;
        const float *ps = pt + (size_t)s * (HD + 2);
        ml[c] = s < a.S ? *reinterpret_cast<const float2 *>(ps + HD) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int e = 0; e < E / 2; ++e)
          ov[c][e] = s < a.S ? *reinterpret_cast<const float2 *>(ps + lane * E + 2 * e) : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int c = 0; c < CU; ++c) mn = fmaxf(mn, ml[c].x);
      const float f0 = M == -INFINITY ? 0.f : exp2f(M - mn);
      M = mn;
      Ls *= f0;
#pragma unroll
      for (int e = 0; e < E; ++e) O[e] *= f0;
#pragma unroll
      for (int c = 0; c < CU; ++c) {
        const float f = ml[c].x == -INFINITY ? 0.f : exp2f(ml[c].x - M);
        Ls = fmaf(ml[c].y, f, Ls);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          O[2 * e] = fmaf(ov[c][e].x, f, O[2 * e]);
          O[2 * e + 1] = fmaf(ov[c][e].y, f, O[2 * e + 1]);
        }
      }
    }
  }
  if constexpr (WPR > 1) {
    if (lane == 0) {
      wm[warp] = M;
      wl[warp] = Ls;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) wo[warp][lane * E + e] = O[e];
    __syncthreads();
    if (sub != 0) return;
    M = -INFINITY;
    Ls = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) O[e] = 0.f;
    for (int w = warp; w < warp + WPR; ++w) M = fmaxf(M, wm[w]);
    for (int w = warp; w < warp + WPR; ++w) {
      const float f = wm[w] == -INFINITY ? 0.f : exp2f(wm[w] - M);
      Ls = fmaf(wl[w], f, Ls);
#pragma unroll
      for (int e = 0; e < E; ++e) O[e] = fmaf(wo[w][lane * E + e], f, O[e]);
    }
  }
  if (skip) return;
  const int t = r / rep, h = g * rep + r % rep;
  __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(a.o) + (((size_t)b * a.T + t) * a.H + h) * HD + lane * E;
#pragma unroll
  for (int e = 0; e < E / 2; ++e)
    reinterpret_cast<uint32_t *>(dst)[e] = (M == -INFINITY && Ls == 0.f) || t >= cnt ? 0u : pack_bf2(O[2 * e] / Ls, O[2 * e + 1] / Ls);
}

int tree_splits(int batch, int T, int H, int Hkv, int max_len, int num_sms) {
  // as many CTAs as the SMs hold at once (2 each), at least 64 positions a split
  const long long row_tiles = ((long long)T * (H / Hkv) + kRows - 1) / kRows;
  const long long want = std::max(1ll, 2ll * num_sms / (batch * (long long)Hkv * row_tiles));
  return (int)std::max(1ll, std::min(want, ((long long)max_len + T + 63) / 64));
}

size_t tree_part_floats(int batch, int T, int H, int Hkv, int hd, int max_len, int num_sms) {
  // more than one split only where the CTAs are at most two an SM, of 16 rows each
  const long long most = (long long)batch * T * H * (((long long)max_len + T + 63) / 64);
  return (size_t)std::min(most, 2ll * kRows * num_sms) * (hd + 2);
}

namespace {

template <int HD, int BITS>
cudaError_t launch_tree_t(const TreeArgs &a, cudaStream_t s) {
  const int R = a.T * (a.H / a.Hkv);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(a.batch * a.Hkv, a.S, (R + kRows - 1) / kRows);
  cfg.blockDim = dim3(kTreeWarps * 32);
  cudaError_t e = cudaLaunchKernelEx(&cfg, attn_tree_kernel<HD, BITS>, a);
  if (e != cudaSuccess || a.S == 1) return e;
  const long long rows = (long long)a.batch * a.Hkv * R;
  cfg.blockDim = dim3(kCombineWarps * 32);
  if (a.S <= 8) {
    cfg.gridDim = dim3((unsigned)((rows + kCombineWarps - 1) / kCombineWarps));
    return cudaLaunchKernelEx(&cfg, attn_tree_combine_kernel<HD, 1>, a);
  }
  cfg.gridDim = dim3((unsigned)rows);
  return cudaLaunchKernelEx(&cfg, attn_tree_combine_kernel<HD, kCombineWarps>, a);
}

}  // namespace

cudaError_t launch_attn_tree(const TreeArgs &a, int hd, int bits, cudaStream_t s) {
#define WQ_TREE(HD, BITS) \
  if (hd == HD && bits == BITS) return launch_tree_t<HD, BITS>(a, s);
  WQ_TREE(128, 16) WQ_TREE(128, 8) WQ_TREE(128, 4) WQ_TREE(64, 16) WQ_TREE(64, 8) WQ_TREE(64, 4)
#undef WQ_TREE
  return cudaErrorInvalidValue;
}

cudaError_t read_tree_status(int *status) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(status, g_tree_status, sizeof(int));
  if (e != cudaSuccess) return e;
  const int zero = 0;
  return cudaMemcpyToSymbol(g_tree_status, &zero, sizeof(int));
}

}  // namespace wq
