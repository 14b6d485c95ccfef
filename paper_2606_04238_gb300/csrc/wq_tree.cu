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
// with m the running maximum of y.  The terms being p_j times a whole number, p_j then
// fills binary16's range whatever V's scales are.  The drafts' terms come first, V as it
// is, and their sum's size is taken into m before the context's.  p_j (bf16 for a bf16
// cache and for drafts) and q (bf16 given; for a quantized cache binary16 with an
// exact power of two a row) are the products' only other 16-bit operands, all sums and
// softmax statistics fp32.  Rounding p costs 2^-11 (binary16) or 2^-8 (bf16) of each
// term at most, of either sign; the bf16 store of o costs 2^-8 of their sum.  p is bf16
// where V is (one product's operands have one type, and V's values need bf16's range);
// keeping p's other bits, in further bf16 parts as wq_attn.cu does, takes as many more
// products.  Measured against 64 bits: 0.0023 of the norm over a bf16 cache where the
// store alone is 0.0017; over 8 and 4 bits 0.0017.
//
// A CTA of 4 warps takes one (b, g), 16 rows and one split of the context, in tiles
// of 64 positions that bulk copies bring into a ring of 64 KB of shared memory; a
// warp takes 16 positions of a tile with mma.sync m16n8k16, rows as M.  Codes go
// from there to the MMA fragments through registers alone: the contraction over HD
// and the order of V's columns are free, so a lane takes 16 consecutive bytes of its
// position's row, and two prmt or and-or build the binary16 value 1024 + code, from
// which 1024 + z is subtracted (exact).  The drafts' chunks run first, in bf16,
// straight from global memory, while the first tiles are on their way.  Few
// splits are a cluster, whose CTAs add up the splits' results (each a share of the
// rows) from one another's shared memory; else a second kernel does.  Both add in a
// fixed order.
//
// Measured (device time): one token over 500 positions of 8 bits, 32 query heads over
// 8 kv heads of 128, 6.8 us, all latency: launch, the lengths, one round of loads, the
// cluster's exchange.  Four drafts over 32,767 positions of 4 bits 24.3 us, 1.5 TB/s: 3
// until queries and first tile are there, 1.5 a tile after that, 2.5 for a CTA's results
// and 3.5 for the second kernel.  A warp's 16 positions of a tile take 550 instructions,
// of which 200 make fragments and products; three warps a scheduler issue 0.6 a clock.
// Scales fetched three tiles ahead and V rows that meet in fewer banks changed nothing.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "wq_cvt.cuh"
#include "wq_internal.h"
#include "wq_kv.h"
#include "wq_ptx.cuh"

namespace wq {

namespace cg = cooperative_groups;

// Status word: WQ_OK (0), WQ_ERR_ARG (-1) after a length outside [0, max_len] or a
// count outside [0, T] was met (that sequence is skipped), WQ_ERR_TIMEOUT (-6)
// after a wait ran out.
__device__ int g_tree_status = 0;

namespace {

constexpr int kTreeWarps = 4;
constexpr int kRows = 16;     // rows a CTA takes
constexpr int kTreeTile = 64;  // positions a tile
constexpr int kRing = 65536;   // bytes of the ring at most
constexpr int kTreeCluster = 8;  // splits that a cluster can be
// Exponents that the drafts' sums can bring into a row's maximum.  The least is that of zeros, below what the smallest
// scale (2^-24) gives; with the most, probabilities of the context are still normal numbers in l.
constexpr int kLeastSize = -40, kMostSize = 64;

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
struct Lay {
  static constexpr int ROW = HD * BITS / 8;                     // bytes a row
  static constexpr int KW = ROW / 4 >= 16 ? 4 : ROW / 16, KI = ROW / (16 * KW);
  static constexpr int VW = ROW / 8 >= 16 ? 4 : ROW / 32, VI = ROW / (32 * VW);
  static constexpr int KS = HD / 16;                            // MMA steps along HD
  static constexpr int NJ = HD / 8;                             // 8-column tiles of the output
  static constexpr int STAGE = 2 * kTreeTile * ROW;             // bytes of a tile
  static constexpr int NS = kRing / STAGE < 8 ? kRing / STAGE : 8;
  static constexpr int OUT = kTreeWarps * kRows * (HD + 4) * 4; // the warps' results, over the ring
  static constexpr int SMEM = NS * STAGE > OUT ? NS * STAGE : OUT;
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

// What a warp accumulates: rows gr and gr + 8 of its 16, columns v_at(j, 2 tc),
// v_at(j, 2 tc + 1); m the rows' maximum of y, l this lane's part of their sums.
template <int HD>
struct Acc {
  float o[HD / 8][4];
  float m[2], l[2];
};

// y[u][e]: scores of positions 8 u + 2 tc + e % 2 and row gr + 8 (e / 2), -inf
// where masked.  Leaves p (fp32) in y and the accumulators rescaled.
//   TOP > 0, the first step after the drafts': what those gave a row is o 2^m and l 2^m with V as it is, and y has log2 s in
// it from here on.  So m takes in the exponent of the row's largest |o| over 2^TOP, a code's size, and o and l the inverse:
// o is then what a p of about 1 gives over codes, whatever V's unit.
template <int HD, int NT, int TOP = 0>
__device__ __forceinline__ void softmax_step(Acc<HD> &acc, float (&y)[NT][4], bool after_drafts = false) {
  float mc[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) mc[e / 2] = fmaxf(mc[e / 2], y[u][e]);
  // Nothing is rescaled until a score passes its row's maximum so far by 2^8 (p stays below that)
  if (__any_sync(0xffffffffu, mc[0] > acc.m[0] + 8.f || mc[1] > acc.m[1] + 8.f || (TOP > 0 && after_drafts))) {
    float al[2], f[2] = {1.f, 1.f};
    if (TOP > 0 && after_drafts) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float big = 0.f;
#pragma unroll
        for (int j = 0; j < HD / 8; ++j) big = fmaxf(fmaxf(big, fabsf(acc.o[j][2 * i])), fabsf(acc.o[j][2 * i + 1]));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
        const int e = min(max((int)(__float_as_uint(big) >> 23) - 127 - TOP, kLeastSize), isinf(big) ? 0 : kMostSize);
        acc.m[i] += (float)e;
        f[i] = __uint_as_float((uint32_t)(127 - e) << 23);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mc[i] = fmaxf(mc[i], __shfl_xor_sync(0xffffffffu, mc[i], 1));
      mc[i] = fmaxf(mc[i], __shfl_xor_sync(0xffffffffu, mc[i], 2));
      const float mn = fmaxf(acc.m[i], mc[i]);
      al[i] = mn == -INFINITY ? 1.f : ex2(acc.m[i] - mn) * f[i];  // 0 at first (m = -inf)
      acc.m[i] = mn;
      acc.l[i] *= al[i];
    }
#pragma unroll
    for (int j = 0; j < HD / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc.o[j][e] *= al[e / 2];
  }
  const float ms[2] = {acc.m[0] == -INFINITY ? 0.f : acc.m[0], acc.m[1] == -INFINITY ? 0.f : acc.m[1]};
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) y[u][e] = ex2(y[u][e] - ms[e / 2]);
}

// q's fragments: rows gr, gr + 8 of the CTA's 16; -1: a row of zeros.
template <int HD, int BITS>
__device__ __forceinline__ void load_q(uint32_t (&qa)[HD / 16][4], float (&qf)[2], const __nv_bfloat16 *q0,
                                       const __nv_bfloat16 *q1, int tc, float scale) {
  using L = Lay<HD, BITS>;
  uint32_t big[2] = {0, 0};  // the rows' largest |q|, as bf16 bits
#pragma unroll
  for (int ks = 0; ks < L::KS; ++ks) {
    const int at = L::q_at(ks, tc);
    const uint2 a = q0 ? __ldg(reinterpret_cast<const uint2 *>(q0 + at)) : make_uint2(0, 0);
    const uint2 b = q1 ? __ldg(reinterpret_cast<const uint2 *>(q1 + at)) : make_uint2(0, 0);
    qa[ks][0] = a.x, qa[ks][1] = b.x, qa[ks][2] = a.y, qa[ks][3] = b.y;
    if constexpr (BITS != 16)
#pragma unroll
      for (int i = 0; i < 4; ++i) big[i % 2] = __vmaxu2(big[i % 2], qa[ks][i] & 0x7fff7fffu);
  }
  qf[0] = qf[1] = scale;
  if constexpr (BITS != 16) {
    // an exact power of two puts the row's largest value in [2^14, 2^15): what
    // binary16 then loses is below 2^-38 of it
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      big[i] = max(big[i] & 0xffffu, big[i] >> 16);
      big[i] = max(big[i], __shfl_xor_sync(0xffffffffu, big[i], 1));
      big[i] = max(big[i], __shfl_xor_sync(0xffffffffu, big[i], 2));
      // its exponent, kept where 2^e and 2^-e are normal; 0 and inf: 1
      const int e = (int)(big[i] >> 7) - 127;
      const int sh = e == 128 || big[i] == 0 ? 0 : min(126, max(-100, 14 - e));
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

template <int HD, int BITS>
__global__ void __launch_bounds__(kTreeWarps * 32, 3) attn_tree_kernel(const TreeArgs a) {
  using L = Lay<HD, BITS>;
  using L16 = Lay<HD, 16>;
  constexpr int OS = HD + 4;
  extern __shared__ __align__(128) uint8_t tree_ring[];
  __shared__ uint64_t full[L::NS], empty[L::NS];
  __shared__ float sm[kTreeWarps][kRows], sl[kTreeWarps][kRows];
  __shared__ int late;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gr = lane >> 2, tc = lane & 3;
  if (tid == 0) {
    for (int i = 0; i < L::NS; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], kTreeWarps);
    }
    fence_barrier_init();
    late = 0;
  }
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, split = blockIdx.y, r0 = blockIdx.z * kRows;
  const int rep = a.H / a.Hkv, R = a.T * rep;
  const int len = a.lens[b], cnt = a.counts ? a.counts[b] : a.T;
  if (len < 0 || len > a.max_len || cnt < 0 || cnt > a.T) {  // the whole cluster alike
    if (tid == 0 && g == 0 && split == 0 && r0 == 0) atomicExch(&g_tree_status, -1);
    return;
  }
  // what this split takes, in units of 16: drafts, then the context
  const int ndr = (cnt + 15) / 16, U = ndr + (len + 15) / 16;
  const int u0 = (int)((long long)U * split / a.S), u1 = (int)((long long)U * (split + 1) / a.S);
  const bool rows = r0 < cnt * rep;  // rows of drafts that exist
  const int c0 = rows ? (max(u0, ndr) - ndr) * 16 : 0, c1 = rows ? min(len, (u1 - ndr) * 16) : 0;  // positions
  const int nt = c1 > c0 ? (c1 - c0 + kTreeTile - 1) / kTreeTile : 0;
  const size_t base = ((size_t)b * a.Hkv + g) * a.max_len;
  const uint8_t *kc = reinterpret_cast<const uint8_t *>(a.kc) + base * L::ROW;
  const uint8_t *vc = reinterpret_cast<const uint8_t *>(a.vc) + base * L::ROW;
  auto copy_tile = [&](int i) {  // one thread
    const int p = c0 + i * kTreeTile, st = i % L::NS;
    const uint32_t bytes = (uint32_t)min(kTreeTile, c1 - p) * L::ROW;
    mbar_arrive_expect_tx(&full[st], 2 * bytes);
    bulk_g2s(tree_ring + st * L::STAGE, kc + (size_t)p * L::ROW, bytes, &full[st]);
    bulk_g2s(tree_ring + st * L::STAGE + L::STAGE / 2, vc + (size_t)p * L::ROW, bytes, &full[st]);
  };
  // (the ring's other tiles are asked for once the queries are here, which would else wait behind all CTAs' tiles: four
  // drafts over 32,767 positions of 4 bits 27.3 -> 23.5 us)
  if (tid == 0 && nt > 0) copy_tile(0);
  const int ra = r0 + gr, rb = ra + 8;
  const int ta = ra / rep, tb = rb / rep;  // the rows' drafts
  const bool ina = ra < R && ta < cnt, inb = rb < R && tb < cnt;
  const __nv_bfloat16 *qbase = reinterpret_cast<const __nv_bfloat16 *>(a.q);
  const __nv_bfloat16 *qa_p = ina ? qbase + (((size_t)b * a.T + ta) * a.H + g * rep + ra % rep) * HD : nullptr;
  const __nv_bfloat16 *qb_p = inb ? qbase + (((size_t)b * a.T + tb) * a.H + g * rep + rb % rep) * HD : nullptr;
  uint32_t meta = 0;
  auto load_meta = [&](int i) {  // lanes 0-15: K's, 16-31: V's of the warp's 16 positions of tile i
    if constexpr (BITS != 16)
      meta = __ldg((lane < 16 ? a.km : a.vm) + base + min(c0 + i * kTreeTile + warp * 16 + (lane & 15), len - 1));
  };
  if (nt > 0) load_meta(0);

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
  if (rows && u < min(u1, ndr)) {
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
      // V's rows in the order of the cache's columns (8 in a row lie together in all of them)
      bool odd = false;
      uint32_t vw[4][HD / 16];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = 8 * (i / 2) + 2 * tc + i % 2;
#pragma unroll
        for (int k = 0; k < HD / 64; ++k) {
          const uint4 x = p < n ? __ldg(reinterpret_cast<const uint4 *>(vd + (size_t)(j0 + p) * dstride + L::v_at(8 * k, gr)))
                                : make_uint4(0, 0, 0, 0);
          vw[i][4 * k] = x.x, vw[i][4 * k + 1] = x.y, vw[i][4 * k + 2] = x.z, vw[i][4 * k + 3] = x.w;
        }
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          uint32_t &x = vw[i][k];
          if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u, odd = true;
          if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu, odd = true;
        }
      }
#pragma unroll
      for (int j = 0; j < L::NJ; ++j)
        mma_bf16_16816(acc.o[j], pf, __byte_perm(vw[0][j / 2], vw[1][j / 2], j % 2 ? 0x7632 : 0x5410),
                       __byte_perm(vw[2][j / 2], vw[3][j / 2], j % 2 ? 0x7632 : 0x5410));
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
  bool ok = true;
  if (nt > 0) {
    load_q<HD, BITS>(qa, qf, qa_p, qb_p, tc, a.scale);
    if (tid == 0)
      for (int i = 1; i < min(nt, L::NS); ++i) copy_tile(i);
    for (int i = 0; i < nt && ok; ++i) {
      const int st = i % L::NS, p0 = c0 + i * kTreeTile + warp * 16, n = c1 - p0;  // n: positions of the warp's 16
      ok = __all_sync(0xffffffffu, mbar_wait(&full[st], (i / L::NS) & 1));
      if (!ok) break;
      // rows of zeros, those of a zero-filled cache too: code - z is 0, and the least scale (kLeastScale) does as well
      const uint32_t mw = (meta & 0xffffu) == 0 || meta == kZeroRow ? (meta & 0xffff0000u) | 1u : meta;
      if (i + 1 < nt) load_meta(i + 1);
      if (n > 0) {
        const uint8_t *kt = tree_ring + st * L::STAGE + warp * 16 * L::ROW, *vt = kt + L::STAGE / 2;
        float y[2][4];
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          uint32_t kw[L::KI * L::KW], z1 = 0, z6 = 0;
#pragma unroll
          for (int k = 0; k < L::KI; ++k)
            load_words(*reinterpret_cast<uint32_t(*)[L::KW]>(&kw[L::KW * k]), kt + (8 * v + gr) * L::ROW + k * 64 + tc * 4 * L::KW);
          if constexpr (BITS != 16) {
            const uint32_t m = __shfl_sync(0xffffffffu, mw, 8 * v + gr);
            const __half2 zz = __half2half2(__ushort_as_half((unsigned short)(m >> 16)));
            const __half2 k1 = __hadd2(zz, __float2half2_rn(1024.f)), k6 = __hadd2(zz, __float2half2_rn(64.f));
            z1 = *reinterpret_cast<const uint32_t *>(&k1);
            z6 = *reinterpret_cast<const uint32_t *>(&k6);
          }
          // two chains of MMAs
          float y2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 4; ++e) y[v][e] = 0.f;
#pragma unroll
          for (int ks = 0; ks < L::KS; ++ks) {
            uint32_t b0, b1;
            k_frag<HD, BITS>(kw, ks, z1, z6, b0, b1);
            if constexpr (BITS == 16)
              mma_bf16_16816(ks % 2 ? y2 : y[v], qa[ks], b0, b1);
            else
              mma_f16_16816(ks % 2 ? y2 : y[v], qa[ks], b0, b1);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) y[v][e] += y2[e];
        }
        float rs[4];
        uint32_t zv[2][2];  // [positions 2 tc, + 1 of 8 v ..][1024 + z, 64 + z]
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          float *yy = y[v / 2];
          if constexpr (BITS == 16) {
            yy[v % 2] *= qf[0];
            yy[2 + v % 2] *= qf[1];
          } else {
            const int at = 8 * (v / 2) + 2 * tc + v % 2;  // of the 16 positions
            const uint32_t m = __shfl_sync(0xffffffffu, mw, at), mm = __shfl_sync(0xffffffffu, mw, 16 + at);
            const float sk = __half2float(__ushort_as_half((unsigned short)(m & 0xffffu)));
            const float sv = __half2float(__ushort_as_half((unsigned short)(mm & 0xffffu)));
            const float lg = lg2(sv);
            rs[v] = rcp(sv);
            yy[v % 2] = fmaf(yy[v % 2] * qf[0], sk, lg);
            yy[2 + v % 2] = fmaf(yy[2 + v % 2] * qf[1], sk, lg);
            if (v % 2 == 0)
              zv[v / 2][0] = mm >> 16;
            else
              zv[v / 2][0] |= mm & 0xffff0000u;
          }
        }
        if (n < 16)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (8 * (v / 2) + 2 * tc + v % 2 >= n) {
              y[v / 2][v % 2] = y[v / 2][2 + v % 2] = -INFINITY;
              rs[v] = 0.f;
            }
        if constexpr (BITS != 16)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const __half2 zz = *reinterpret_cast<const __half2 *>(&zv[v][0]);
            const __half2 k1 = __hadd2(zz, __float2half2_rn(1024.f)), k6 = __hadd2(zz, __float2half2_rn(64.f));
            zv[v][0] = *reinterpret_cast<const uint32_t *>(&k1);
            zv[v][1] = *reinterpret_cast<const uint32_t *>(&k6);
          }
        uint32_t vw[4][L::VI * L::VW];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int at = 8 * (v / 2) + 2 * tc + v % 2;
#pragma unroll
          for (int k = 0; k < L::VI; ++k)
            load_words(*reinterpret_cast<uint32_t(*)[L::VW]>(&vw[v][L::VW * k]), vt + at * L::ROW + k * 128 + gr * 4 * L::VW);
        }
        if (BITS == 16 && n < 16)  // what the ring held before may not be finite
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (8 * (v / 2) + 2 * tc + v % 2 >= n)
#pragma unroll
              for (int k = 0; k < L::VI * L::VW; ++k) vw[v][k] = 0;
        softmax_step<HD, 2, BITS == 16 ? 0 : BITS - 1>(acc, y, i == 0 && u0 + warp < min(u1, ndr));
        uint32_t pf[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float p = y[k / 2][2 * (k % 2)], q = y[k / 2][2 * (k % 2) + 1];
          pf[k] = BITS == 16 ? pack_bf2(p, q) : pack_h2(p, q);
          if constexpr (BITS == 16)
            acc.l[k % 2] += p + q;
          else
            acc.l[k % 2] += fmaf(p, rs[2 * (k / 2)], q * rs[2 * (k / 2) + 1]);
        }
#pragma unroll
        for (int j = 0; j < L::NJ; ++j) {
          const uint32_t b0 = v_frag<HD, BITS>(vw[0], vw[1], j, zv[0][0], zv[0][1]);
          const uint32_t b1 = v_frag<HD, BITS>(vw[2], vw[3], j, zv[1][0], zv[1][1]);
          if constexpr (BITS == 16)
            mma_bf16_16816(acc.o[j], pf, b0, b1);
          else
            mma_f16_16816(acc.o[j], pf, b0, b1);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[st]);
      // the tile NS after the one before this, whose warps have had a tile's time
      if (warp == 0 && i > 0 && i - 1 + L::NS < nt) {
        const int e = (i - 1) % L::NS;
        ok = __all_sync(0xffffffffu, mbar_wait(&empty[e], ((i - 1) / L::NS) & 1));
        if (ok && lane == 0) copy_tile(i - 1 + L::NS);
      }
    }
    if (!ok && lane == 0) late = 1;
  }
  __syncthreads();
  if (late) {  // copies in flight are given time to land
    if (tid == 0) atomicExch(&g_tree_status, -6);
    const unsigned long long t0 = global_timer_ns();
    for (int i = 0; i < (1 << 20) && global_timer_ns() - t0 < 2000000ull; ++i) __nanosleep(1000);
    __syncthreads();
  }
  float(*so)[kRows][OS] = reinterpret_cast<float(*)[kRows][OS]>(tree_ring);

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
      const float f = sm[w][r] == -INFINITY ? 0.f : ex2(sm[w][r] - M);
      Ls = fmaf(sl[w][r], f, Ls);
      O0 = fmaf(so[w][r][e], f, O0);
      O1 = fmaf(so[w][r][e + 1], f, O1);
    }
    if (a.S == 1) {
      const int t = row / rep, h = g * rep + row % rep;
      const bool none = (M == -INFINITY && Ls == 0.f) || t >= cnt;  // sees nothing, or is padding
      *reinterpret_cast<uint32_t *>(reinterpret_cast<__nv_bfloat16 *>(a.o) + (((size_t)b * a.T + t) * a.H + h) * HD + e) =
          none ? 0u : pack_bf2(O0 / Ls, O1 / Ls);
    } else if (a.cluster) {
      // (this thread alone reads these places: the warps' results, whose first takes the CTA's)
      so[0][r][e] = O0;
      so[0][r][e + 1] = O1;
      if (e == 0) {
        so[0][r][HD] = M;
        so[0][r][HD + 1] = Ls;
      }
    } else {
      float *pt = a.part + (((size_t)blockIdx.x * R + row) * a.S + split) * (HD + 2);
      *reinterpret_cast<float2 *>(pt + e) = make_float2(O0, O1);
      if (e == 0) *reinterpret_cast<float2 *>(pt + HD) = make_float2(M, Ls);
    }
  }
  if (a.cluster) {
    // the cluster's CTAs are the splits: CTA `split` adds up its share of the outputs
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
    const float *of[kTreeCluster];
#pragma unroll
    for (int k = 0; k < kTreeCluster; ++k) of[k] = k < a.S ? cl.map_shared_rank(&so[0][0][0], k) : nullptr;
    for (int i = split * kTreeWarps * 32 + tid; i < kRows * HD / 2; i += a.S * kTreeWarps * 32) {
      const int r = i / (HD / 2), e = 2 * (i % (HD / 2)), row = r0 + r;
      if (row >= R) break;
      float2 ml[kTreeCluster], ov[kTreeCluster];
      float M = -INFINITY, Ls = 0.f, O0 = 0.f, O1 = 0.f;
#pragma unroll
      for (int k = 0; k < kTreeCluster; ++k) {
        ml[k] = k < a.S ? *reinterpret_cast<const float2 *>(of[k] + r * OS + HD) : make_float2(-INFINITY, 0.f);
        ov[k] = k < a.S ? *reinterpret_cast<const float2 *>(of[k] + r * OS + e) : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < kTreeCluster; ++k) M = fmaxf(M, ml[k].x);
#pragma unroll
      for (int k = 0; k < kTreeCluster; ++k) {
        const float f = ml[k].x == -INFINITY ? 0.f : ex2(ml[k].x - M);
        Ls = fmaf(ml[k].y, f, Ls);
        O0 = fmaf(ov[k].x, f, O0);
        O1 = fmaf(ov[k].y, f, O1);
      }
      const int t = row / rep, h = g * rep + row % rep;
      const bool none = (M == -INFINITY && Ls == 0.f) || t >= cnt;
      *reinterpret_cast<uint32_t *>(reinterpret_cast<__nv_bfloat16 *>(a.o) + (((size_t)b * a.T + t) * a.H + h) * HD + e) =
          none ? 0u : pack_bf2(O0 / Ls, O1 / Ls);
    }
    cl.sync();  // no CTA leaves while another reads from it
  }
}

// o of one row: its splits' parts added in a fixed order (warp w: splits w, w + 8, .. in order, then the warps in
// order).  grid: rows.
constexpr int kCombineWarps = 8;

template <int HD>
__global__ void __launch_bounds__(kCombineWarps * 32) attn_tree_combine_kernel(const TreeArgs a) {
  constexpr int E = HD / 32, CU = 8;  // splits loaded in one round trip
  __shared__ float wm[kCombineWarps], wl[kCombineWarps], wo[kCombineWarps][HD];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rep = a.H / a.Hkv, R = a.T * rep;
  const size_t row = blockIdx.x;
  const int bg = (int)(row / R), r = (int)(row - (size_t)bg * R), b = bg / a.Hkv, g = bg % a.Hkv;
  pdl_wait();
  pdl_launch_dependents();
  const int len = a.lens[b], cnt = a.counts ? a.counts[b] : a.T;
  float M = -INFINITY, Ls = 0.f, O[E];
#pragma unroll
  for (int e = 0; e < E; ++e) O[e] = 0.f;
  const float *pt = a.part + row * a.S * (HD + 2);
  for (int s0 = warp; s0 < a.S; s0 += CU * kCombineWarps) {
    float2 ml[CU], ov[CU][E / 2];
    float mn = M;
#pragma unroll
    for (int c = 0; c < CU; ++c) {
      const int s = s0 + c * kCombineWarps;
      const float *ps = pt + (size_t)s * (HD + 2);
      ml[c] = s < a.S ? *reinterpret_cast<const float2 *>(ps + HD) : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int e = 0; e < E / 2; ++e)
        ov[c][e] = s < a.S ? *reinterpret_cast<const float2 *>(ps + lane * E + 2 * e) : make_float2(0.f, 0.f);
    }
#pragma unroll
    for (int c = 0; c < CU; ++c) mn = fmaxf(mn, ml[c].x);
    const float f0 = M == -INFINITY ? 0.f : ex2(M - mn);
    M = mn;
    Ls *= f0;
#pragma unroll
    for (int e = 0; e < E; ++e) O[e] *= f0;
#pragma unroll
    for (int c = 0; c < CU; ++c) {
      const float f = ml[c].x == -INFINITY ? 0.f : ex2(ml[c].x - M);  // (a NaN of a part stays NaN)
      Ls = fmaf(ml[c].y, f, Ls);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        O[2 * e] = fmaf(ov[c][e].x, f, O[2 * e]);
        O[2 * e + 1] = fmaf(ov[c][e].y, f, O[2 * e + 1]);
      }
    }
  }
  if (len < 0 || len > a.max_len || cnt < 0 || cnt > a.T) return;  // skipped (the whole CTA alike)
  if (lane == 0) {
    wm[warp] = M;
    wl[warp] = Ls;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) wo[warp][lane * E + e] = O[e];
  __syncthreads();
  if (threadIdx.x >= HD / 2) return;
  const int e = 2 * threadIdx.x;
  M = -INFINITY;
  Ls = 0.f;
  float O0 = 0.f, O1 = 0.f;
#pragma unroll
  for (int w = 0; w < kCombineWarps; ++w) M = fmaxf(M, wm[w]);
#pragma unroll
  for (int w = 0; w < kCombineWarps; ++w) {
    const float f = wm[w] == -INFINITY ? 0.f : ex2(wm[w] - M);
    Ls = fmaf(wl[w], f, Ls);
    O0 = fmaf(wo[w][e], f, O0);
    O1 = fmaf(wo[w][e + 1], f, O1);
  }
  const int t = r / rep, h = g * rep + r % rep;
  const bool none = (M == -INFINITY && Ls == 0.f) || t >= cnt;
  *reinterpret_cast<uint32_t *>(reinterpret_cast<__nv_bfloat16 *>(a.o) + (((size_t)b * a.T + t) * a.H + h) * HD + e) =
      none ? 0u : pack_bf2(O0 / Ls, O1 / Ls);
}

int tree_splits(int batch, int T, int H, int Hkv, int max_len, int num_sms) {
  // as many CTAs as the SMs hold at once (3 each), at least 64 positions a split
  const long long row_tiles = ((long long)T * (H / Hkv) + kRows - 1) / kRows;
  const long long want = std::max(1ll, 3ll * num_sms / (batch * (long long)Hkv * row_tiles));
  return (int)std::max(1ll, std::min(want, ((long long)max_len + T + 63) / 64));
}

// Whether the splits are a cluster each.  Three at most always are (32 rows over 512 positions, 16 sequences: 13.7 us
// against 16.1 with a second kernel); more only where every CTA has an SM of its own, since clusters of several CTAs that
// share SMs wait for places together (4 sequences, 8 drafts, 1024 positions, 7 splits: 19.0 against 16.3; one sequence,
// one draft, 500 positions, 8 splits: the same time on the GPU, one launch less for the host).
bool tree_cluster(int batch, int T, int H, int Hkv, int S, int num_sms) {
  const long long row_tiles = ((long long)T * (H / Hkv) + kRows - 1) / kRows;
  return S > 1 && (S <= 3 || (S <= kTreeCluster && batch * (long long)Hkv * row_tiles * S <= num_sms));
}

size_t tree_part_floats(int batch, int T, int H, int Hkv, int hd, int max_len, int num_sms) {
  // more than one split only where the CTAs are at most three an SM, of 16 rows each
  const long long most = (long long)batch * T * H * (((long long)max_len + T + 63) / 64);
  return (size_t)std::min(most, 3ll * kRows * num_sms) * (hd + 2);
}

namespace {

// Once a device: the kernel's shared memory.
template <int HD, int BITS>
cudaError_t prepare_tree() {
  static std::atomic<bool> done[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < 64 && done[dev].load(std::memory_order_acquire)) return cudaSuccess;
  e = cudaFuncSetAttribute(attn_tree_kernel<HD, BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay<HD, BITS>::SMEM);
  if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
  return e;
}

template <int HD, int BITS>
cudaError_t launch_tree_t(const TreeArgs &a, cudaStream_t s) {
  const int R = a.T * (a.H / a.Hkv);
  cudaError_t e = prepare_tree<HD, BITS>();
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = a.S;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = a.cluster ? 2 : 1;
  cfg.gridDim = dim3(a.batch * a.Hkv, a.S, (R + kRows - 1) / kRows);
  cfg.blockDim = dim3(kTreeWarps * 32);
  cfg.dynamicSmemBytes = Lay<HD, BITS>::SMEM;
  e = cudaLaunchKernelEx(&cfg, attn_tree_kernel<HD, BITS>, a);
  if (e != cudaSuccess || a.S == 1 || a.cluster) return e;
  const long long rows = (long long)a.batch * a.Hkv * R;
  cfg.numAttrs = 1;
  cfg.blockDim = dim3(kCombineWarps * 32);
  cfg.dynamicSmemBytes = 0;
  cfg.gridDim = dim3((unsigned)rows);
  return cudaLaunchKernelEx(&cfg, attn_tree_combine_kernel<HD>, a);
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
