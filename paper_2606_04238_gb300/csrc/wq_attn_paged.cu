// wq_attn_paged.cu -- causal attention of a ragged batch over a paged KV cache of 16, 8 or 4
// bits (sm_103a) on mma.sync, for sequences of few query rows: decode steps and short runs
// of drafts.
//
// Query i of a sequence of nq stands at position kv_len - nq + i and sees the positions up to
// its own.  Row r = i rep + h stands for token i and query head g rep + h of kv head g:
//   x_j = scale log2(e) (q . k_j),  o = sum_j 2^(x_j - m) v_j / sum_j 2^(x_j - m).
// Positions are the products' M and rows their N: S^T = K Q^T and O^T = V^T P^T, so that
// 8 rows take what 16 would as M, and a lane's softmax values are half as many.  A cached row
// of 8 or 4 bits is s (code - z), and code - z is exact in binary16: K's scale multiplies the
// score, V's is taken into the exponent,
//   p_j = 2^(x_j + log2 s_j - m),  o = sum_j p_j (code - z)_j / sum_j p_j / s_j,
// with m the running maximum of x_j + log2 s_j.  (Codes as they lie there are binary16 too,
// subnormal numbers code 2^-24, and the zero points could come off the sums: a third of the
// instructions less.  But the tensor cores add products of subnormal numbers with 2^-14 of
// their size lost, a 4-bit column's error then 2^-14 of its codes and not of their difference.)
// p_j is rounded to binary16 (2^6 larger than above, so that it is a normal number, off by 2^-11
// of its term at most, down to 2^-20 of the largest; below that by 2^-31 of the largest) or over a bf16
// cache to bf16 (2^-8); everything else is fp32.
//
// The blocks of 64 positions (128 of 4 bits) of all (sequence, row tile, kv head) are laid end to end and
// every CTA takes an equal run of them, found from the lengths themselves; what it has of an
// (item) that other CTAs share is left in the workspace, and the last of them to arrive adds
// up all parts in their order.  A warp takes 16 positions (32 of 4 bits) at a time, 16 of which
// always lie in one page, through a ring of its own that cp.async fills: no warp waits for another.
// The maximum is only raised, and sums and O rescaled, where a score passes it by 8.
//   64 tokens over 4k to 8k positions of 4 bits (8 kv heads of 128, 4 query heads each) take 91
// to 94 us for 426 MB, 0.69 of the copy's rate: 311 instructions a warp for 16 positions at
// 0.58 a clock and scheduler, with the three warps that 168 registers leave room for.  One
// token over 500 positions of 8 bits takes 9, over 32,767 of 4 bits 19: the chain of one
// launch and one block, and the sum of the parts.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "wq_cvt.cuh"
#include "wq_frag.cuh"
#include "wq_internal.h"
#include "wq_kv.h"
#include "wq_paged.h"
#include "wq_ptx.cuh"
#include "wq_ragged.cuh"

namespace wq {

// Status word: WQ_OK (0), or WQ_ERR_ARG (-1) after a row offset, length or page outside its
// range was met (that sequence is skipped; a page outside the pool is read as page 0).
__device__ int g_attn_paged_status = 0;

namespace {

constexpr int kWarps = 4;
constexpr int kSub = 16;             // positions of an MMA step, always of one page
constexpr int kCtasPerSm = 3;        // at most
constexpr int kMostRows = 16;        // rows of an item at most

__device__ __forceinline__ uint32_t hadd2_u(uint32_t a, uint32_t b) {
  const __half2 v = __hadd2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float v;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ float half_of(uint32_t m) { return __half2float(__ushort_as_half((unsigned short)(m & 0xffffu))); }
// An 8 x 8 matrix of 16-bit values (row lane / 4, columns 2 (lane % 4) ..) transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// cp.async of 16 and of 4 bytes, and loads, at a shared-memory address.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
template <int N>
__device__ __forceinline__ void lds_words(uint32_t (&w)[N], uint32_t at) {
  static_assert(N == 1 || N == 2 || N == 4, "");
  if constexpr (N == 4)
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
  else if constexpr (N == 2)
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
  else
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
}
// How a warp holds 16 positions.  K: lane (gr, tc) takes 16-byte pieces tc, tc + 4, .. of the
// row in place gr and of that in place gr + 8 (KW words each: half or a quarter of a piece
// where rows are shorter than 128 bytes).  V: lane (gr, tc) takes pieces gr, gr + 8, .. of the
// rows tc, tc + 4, tc + 8 and tc + 12.  Row p lies in place 2 (p % 4) + p / 4 % 2 of its eight
// for K, so that place j of the product's order is row j / 2 + 4 (j % 2) for both.  Pieces are
// permuted within a row by what keeps a quarter warp's lanes in different banks.
template <int HD, int BITS>
struct Lay : RowLay<HD, BITS> {
  static constexpr int ROW = RowLay<HD, BITS>::ROW;
  static constexpr int CHR = ROW / 16, COPIES = kSub * CHR / 32;  // pieces a row; copies a lane of K, and of V, of 16 positions
  // positions a warp takes in one step: 32 of 4 bits, whose bytes are few for a step's fixed instructions
  static constexpr int SUBS = BITS == 4 ? 2 : 1, UNIT = kSub * SUBS, BLOCK = kWarps * UNIT;
  static constexpr int SUB = 2 * kSub * ROW + (BITS == 16 ? 0 : 128), STAGE = SUBS * SUB;
  static constexpr int NS = BITS == 16 && HD == 128 ? 3 : BITS == 4 ? 3 : 16 * 1024 / STAGE < 6 ? 16 * 1024 / STAGE : 6;
  static_assert(NS >= 2, "a stage in flight beside the one that is read");
  static constexpr int RING = kWarps * NS * STAGE;
  static __device__ __forceinline__ int k_swz(int place) { return ROW >= 128 ? 4 * (place & 1) : 0; }
  static __device__ __forceinline__ int v_swz(int row) { return ROW >= 128 ? 2 * (row & 3) : ROW == 64 ? 2 * (row / 2 & 1) : 0; }
};

// CTAs an SM holds: 168 registers a thread (with 128 and four CTAs 64 tokens over 4k to 8k positions of 4 bits take 100 us
// for 92, over 2k to 4k of a bf16 pool, heads of 64, 78 for 68); a bf16 ring of heads of 128 takes 96 KB.
constexpr int occupancy(int hd, int bits, int nt) { return bits == 16 && hd == 128 ? 2 : kCtasPerSm; }

// A sequence; the blocks of positions of each of its items, and its tiles of rows.
struct Item : Seq {
  int blocks, tiles;
};
template <int BLOCK>
__device__ __forceinline__ Item get_item(const AttnPagedArgs &a, int b, int rep, int rows, bool &bad) {
  Item s;
  static_cast<Seq &>(s) = get_seq(a, b, bad);
  s.tiles = (s.nq * rep + rows - 1) / rows;
  s.blocks = max(1, (s.len + BLOCK - 1) / BLOCK);
  return s;
}

}  // namespace

template <int HD, int BITS, int NT>
__global__ void __launch_bounds__(kWarps * 32, occupancy(HD, BITS, NT)) attn_paged_kernel(const AttnPagedArgs a) {
  using L = Lay<HD, BITS>;
  constexpr int ROWS = 8 * NT, OS = HD + 4, PS = HD + 4;  // (a part's row: its sums, maximum and sum of p)
  extern __shared__ __align__(128) uint8_t paged_ring[];
  __shared__ float sm[kWarps][ROWS], sl[kWarps][ROWS];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gr = lane >> 2, tc = lane & 3;
  const uint32_t ring_at = smem_addr(paged_ring) + warp * (L::NS * L::STAGE);
  const int rep = a.H / a.Hkv, page = 1 << a.shift;
  pdl_wait();
  pdl_launch_dependents();

  // ---- this CTA's run of blocks: every warp the same sums
  bool bad = false;
  long long total = 0;
  for (int b = lane; b < a.batch; b += 32) {
    const Item s = get_item<L::BLOCK>(a, b, rep, ROWS, bad);
    total += (long long)s.blocks * s.tiles;
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  total *= a.Hkv;
  if (bad && blockIdx.x == 0) atomicExch(&g_attn_paged_status, -1);
  const long long N = min((long long)gridDim.x, total), c = blockIdx.x;
  if (c >= N) return;
  const long long x0 = total * c / N, x1 = total * (c + 1) / N;
  // the sequence that x0 falls into
  int b = 0;
  long long base = 0;
  Item s{};
  for (int b0 = 0;; b0 += 32) {
    long long mine = 0;
    if (b0 + lane < a.batch) {
      s = get_item<L::BLOCK>(a, b0 + lane, rep, ROWS, bad);
      mine = (long long)s.blocks * s.tiles * a.Hkv;
    }
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, x0 < base + incl);
    if (hit) {
      const int src = __ffs(hit) - 1;
      b = b0 + src;
      base += __shfl_sync(0xffffffffu, incl - mine, src);
      break;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  s = get_item<L::BLOCK>(a, b, rep, ROWS, bad);

  for (long long x = x0; x < x1;) {
    while (x >= base + (long long)s.blocks * s.tiles * a.Hkv) {
      base += (long long)s.blocks * s.tiles * a.Hkv;
      s = get_item<L::BLOCK>(a, ++b, rep, ROWS, bad);
    }
    const int local = (int)((x - base) / s.blocks), blk0 = (int)((x - base) - (long long)local * s.blocks);
    const int g = local % a.Hkv, r0 = local / a.Hkv * ROWS;
    const int blk1 = (int)min((long long)s.blocks, blk0 + (x1 - x));
    const long long item = x - blk0;  // the item's first block
    x += blk1 - blk0;
    const int R = s.nq * rep, before = s.len - s.nq;  // positions that every row sees, less its own
    const int most = s.len == 0 ? 0 : before + min(R - 1, r0 + ROWS - 1) / rep + 1;  // positions that the tile's last row sees
    const int least = s.len == 0 ? 0 : before + r0 / rep + 1;                       // ... and its first
    const int u0 = blk0 * kWarps + warp, c1 = min(most, blk1 * L::BLOCK);
    const int nu = u0 * L::UNIT < c1 ? ((c1 - u0 * L::UNIT + L::UNIT - 1) / L::UNIT + kWarps - 1) / kWarps : 0;  // this warp's units

    // the pool's first rows of 16 positions each: lane i has those of unit i / SUBS of the next 32 / SUBS (a pool has fewer
    // than 2^32 rows: host check; what lies behind the last position is some row of it)
    uint32_t rows = 0;
    auto load_rows = [&](int k) {
      // (lanes ahead of the last position may be 2016 past it: above 2^31 where it is the largest that tables may have)
      const uint32_t p = (uint32_t)(u0 + kWarps * (k + lane / L::SUBS)) * L::UNIT + lane % L::SUBS * kSub;
      int id = a.tables[(size_t)b * a.max_pages + (min(p, (uint32_t)c1 - 1) >> a.shift)];
      if ((unsigned)id >= (unsigned)a.n_pages) {
        id = 0;
        atomicExch(&g_attn_paged_status, -1);
      }
      rows = (((uint32_t)id * a.Hkv + g) << a.shift) + (p & (page - 1));
    };
    auto copy_unit = [&](int k, int stage) {
      constexpr int PER = 32 / L::SUBS;
      if (k % PER == 0 && k < nu) load_rows(k);
#pragma unroll
      for (int u = 0; u < L::SUBS; ++u) {
        const size_t row = __shfl_sync(0xffffffffu, rows, k % PER * L::SUBS + u);
        if (k >= nu) continue;
        const uint32_t st = ring_at + stage * L::STAGE + u * L::SUB;
        const uint8_t *ks = reinterpret_cast<const uint8_t *>(a.kc) + row * L::ROW + lane * 16;
        const uint8_t *vs = reinterpret_cast<const uint8_t *>(a.vc) + row * L::ROW + lane * 16;
#pragma unroll
        for (int i = 0; i < L::COPIES; ++i) {
          const int p = (lane + 32 * i) / L::CHR, ch = (lane + 32 * i) % L::CHR;
          const int place = (p & 8) + 2 * (p & 3) + (p >> 2 & 1);
          copy16(st + place * L::ROW + ((ch ^ L::k_swz(place)) << 4), ks + 512 * i);
          copy16(st + (kSub + p) * L::ROW + ((ch ^ L::v_swz(p)) << 4), vs + 512 * i);
        }
        if constexpr (BITS != 16)  // scales and zero points of rows p and p + 8 beside each other
          copy4(st + 2 * kSub * L::ROW + ((lane & 16) + 2 * (lane & 7) + (lane >> 3 & 1)) * 4,
                    (lane < 16 ? a.km : a.vm) + row + (lane & 15));
      }
      cp_async_commit();
    };
#pragma unroll 1
    for (int k = 0; k < L::NS - 1; ++k) copy_unit(k, k);

    // ---- the rows' queries: lane (gr, tc) has row gr's operands, rows 2 tc and 2 tc + 1 its scores
    uint32_t qb[NT][L::KS][2];
    float A[NT][2];            // x = s A acc
    int limit[NT][2];          // positions that the rows see
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = r0 + 8 * n + gr;
      const bool in = r < R;
      const __nv_bfloat16 *qp = reinterpret_cast<const __nv_bfloat16 *>(a.q) +
                                ((size_t)(s.q0 + (in ? r / rep : 0)) * a.H + g * rep + (in ? r % rep : 0)) * HD;
      uint32_t big = 0;
#pragma unroll
      for (int ks = 0; ks < L::KS; ++ks) {
        const uint2 v = in ? __ldg(reinterpret_cast<const uint2 *>(qp + L::q_at(ks, tc))) : make_uint2(0, 0);
        qb[n][ks][0] = v.x, qb[n][ks][1] = v.y;
        big = __vmaxu2(big, __vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu));
      }
      float qf = a.scale;
      if constexpr (BITS != 16) {
        // an exact power of two puts the row's largest value in [2^14, 2^15): what binary16 then
        // loses is below 2^-38 of it
        big = max(big & 0xffffu, big >> 16);
        big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
        const int e = (int)(big >> 7) - 127;
        const int sh = e == 128 || big == 0 ? 0 : min(126, max(-100, 14 - e));
        const float f = __uint_as_float((uint32_t)(127 + sh) << 23);
        qf = a.scale * __uint_as_float((uint32_t)(127 - sh) << 23);
#pragma unroll
        for (int ks = 0; ks < L::KS; ++ks)
#pragma unroll
          for (int i = 0; i < 2; ++i) qb[n][ks][i] = pack_h2(bf_lo(qb[n][ks][i]) * f, bf_hi(qb[n][ks][i]) * f);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = r0 + 8 * n + 2 * tc + e;
        A[n][e] = __shfl_sync(0xffffffffu, qf, 8 * tc + 4 * e);
        limit[n][e] = rr < R && s.len > 0 ? before + rr / rep + 1 : 0;
      }
    }

    float o[NT][L::NJ / 2][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; j < L::NJ / 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][j][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) m[n][e] = -INFINITY, l[n][e] = 0.f;
    }

    // what a score is less before 2^x: the rows' maxima (less kLift: p is 2^kLift times larger, so that small ones are normal
    // numbers), 0 while there is none; a score above the limit raises them, so that p stays below 2^(8 + kLift)
    constexpr float kLift = BITS == 16 ? 0.f : 6.f;
    float base_m[NT][2], most_y[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) base_m[n][e] = -kLift, most_y[n][e] = -INFINITY;
    const int pa = (gr >> 1) + 4 * (gr & 1);  // the lane's positions of the scores: pa and pa + 8 of 16

    auto highest = [](const float (&y)[L::SUBS][NT][4], int n, int e) {  // of the lane's scores of row e
      float t = fmaxf(y[0][n][e], y[0][n][2 + e]);
#pragma unroll
      for (int u = 1; u < L::SUBS; ++u) t = fmaxf(t, fmaxf(y[u][n][e], y[u][n][2 + e]));
      return t;
    };
    // One step's positions, from p0 on.  SOME: some row does not see them all, and behind the last position they may hold
    // anything.
    auto unit = [&](uint32_t st0, int p0, auto is_some) {
      constexpr bool SOME = decltype(is_some)::value;
      float y[L::SUBS][NT][4];
      [[maybe_unused]] float rs[L::SUBS][2];
#pragma unroll
      for (int u = 0; u < L::SUBS; ++u) {
        const uint32_t st = st0 + u * L::SUB;
        uint32_t ka[L::KI * L::KW], kb[L::KI * L::KW];
#pragma unroll
        for (int i = 0; i < L::KI; ++i) {
          const int off = L::ROW >= 64 ? (((tc + 4 * i) ^ L::k_swz(gr)) << 4) : tc * 4 * L::KW;
          lds_words(*reinterpret_cast<uint32_t(*)[L::KW]>(&ka[L::KW * i]), st + gr * L::ROW + off);
          lds_words(*reinterpret_cast<uint32_t(*)[L::KW]>(&kb[L::KW * i]), st + (gr + 8) * L::ROW + off);
        }
        uint32_t za = 0, zb = 0, za6 = 0, zb6 = 0;
        float sk[2] = {1.f, 1.f}, lg[2] = {0.f, 0.f};
        if constexpr (BITS != 16) {
          const uint32_t meta = st + 2 * kSub * L::ROW;
          uint32_t mk[2], mv[2];
          lds_words(mk, meta + 8 * pa);
          lds_words(mv, meta + 64 + 8 * pa);
          const uint32_t k1024 = 0x64006400u;
          za = hadd2_u(__byte_perm(mk[0], 0, 0x3232), k1024), zb = hadd2_u(__byte_perm(mk[1], 0, 0x3232), k1024);
          za6 = hsub2_u(za, 0x63806380u), zb6 = hsub2_u(zb, 0x63806380u);  // less 960: 64 + z, exact
          sk[0] = half_of(mk[0]), sk[1] = half_of(mk[1]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            // rows of zeros, those of a zero-filled cache too: code - z is 0, and the least scale does as well
            const uint32_t m = i ? mv[1] : mv[0];
            const float s = max_nan((int)m < 0 ? 0.f : half_of(m), kLeastScale);  // (kZeroRow: the one zero point below 0)
            lg[i] = lg2(s);
            rs[u][i] = rcp(s);
          }
        }
#pragma unroll
        for (int ks = 0; ks < L::KS; ++ks) {
          uint32_t f[4];
          k_frag<HD, BITS>(ka, ks, za, za6, f[0], f[2]);
          k_frag<HD, BITS>(kb, ks, zb, zb6, f[1], f[3]);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if (ks == 0)
#pragma unroll
              for (int e = 0; e < 4; ++e) y[u][n][e] = 0.f;
            if constexpr (BITS == 16)
              mma_bf16_16816(y[u][n], f, qb[n][ks][0], qb[n][ks][1]);
            else
              mma_f16_16816(y[u][n], f, qb[n][ks][0], qb[n][ks][1]);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[u][n][e] = BITS == 16 ? y[u][n][e] * A[n][e % 2] : fmaf(y[u][n][e], A[n][e % 2] * sk[e / 2], lg[e / 2]);
            if (SOME && p0 + kSub * u + pa + 8 * (e / 2) >= limit[n][e % 2]) y[u][n][e] = -INFINITY;
          }
      }
      // ---- softmax
      bool up = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          up |= highest(y, n, e) > most_y[n][e];
        }
      if (__any_sync(0xffffffffu, up)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float al[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float t = highest(y, n, e);
#pragma unroll
            for (int d = 4; d <= 16; d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
            t = fmaxf(t, m[n][e]);
            al[e] = t == -INFINITY ? 1.f : ex2(m[n][e] - t);
            m[n][e] = t;
            base_m[n][e] = t == -INFINITY ? -kLift : t - kLift;
            most_y[n][e] = t + 8.f;
            l[n][e] *= al[e];
          }
#pragma unroll
          for (int j = 0; j < L::NJ / 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][j][e] *= al[e % 2];
        }
      }
#pragma unroll
      for (int u = 0; u < L::SUBS; ++u) {
        const uint32_t sv = st0 + u * L::SUB + kSub * L::ROW;
        const int q0 = p0 + kSub * u;
        uint32_t vw[4][L::VI * L::VW];
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int i = 0; i < L::VI; ++i) {
            const int off = L::ROW >= 128 ? (((gr + 8 * i) ^ L::v_swz(tc)) << 4)
                                          : (((gr * 4 * L::VW >> 4) ^ L::v_swz(tc)) << 4) + (gr * 4 * L::VW & 15);
            lds_words(*reinterpret_cast<uint32_t(*)[L::VW]>(&vw[v][L::VW * i]), sv + (tc + 4 * v) * L::ROW + off);
          }
        uint32_t zv[2] = {0, 0}, z6[2] = {0, 0};  // 1024 + z of rows tc and tc + 4, tc + 8 and tc + 12
        if constexpr (BITS != 16) {
          const uint32_t meta = sv + kSub * L::ROW + 64;
          uint32_t x[2], w[2];
          lds_words(x, meta + 8 * tc);
          lds_words(w, meta + 8 * tc + 32);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t z = __byte_perm(x[i], w[i], 0x7632);
            if (SOME) z &= (q0 + tc + 8 * i < most ? 0xffffu : 0u) | (q0 + tc + 4 + 8 * i < most ? 0xffff0000u : 0u);
            zv[i] = hadd2_u(z, 0x64006400u);
            z6[i] = hsub2_u(zv[i], 0x63806380u);
          }
        }
        bool odd = false;
        if (SOME && BITS == 16)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const bool behind = q0 + tc + 4 * v >= most;
#pragma unroll
            for (int i = 0; i < L::VI * L::VW; ++i) {
              uint32_t &w = vw[v][i];
              if (behind) w = 0;
              // values that are not finite are taken out, and added to the rows that see them
              if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u, odd = true;
              if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu, odd = true;
            }
          }
        uint32_t pb[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float p0 = ex2(y[u][n][2 * i] - base_m[n][0]), p1 = ex2(y[u][n][2 * i + 1] - base_m[n][1]);
            pb[n][i] = transpose8(BITS == 16 ? pack_bf2(p0, p1) : pack_h2(p0, p1));
            if constexpr (BITS == 16) {
              l[n][0] += p0;
              l[n][1] += p1;
            } else {  // (a masked row's scale may be NaN)
              if (!SOME || p0 != 0.f) l[n][0] = fmaf(p0, rs[u][i], l[n][0]);
              if (!SOME || p1 != 0.f) l[n][1] = fmaf(p1, rs[u][i], l[n][1]);
            }
          }
#pragma unroll
        for (int j = 0; j < L::NJ / 2; ++j) {
          uint32_t f[4];
          f[0] = v_frag<HD, BITS>(vw[0], vw[1], 2 * j, zv[0], z6[0]);
          f[1] = v_frag<HD, BITS>(vw[0], vw[1], 2 * j + 1, zv[0], z6[0]);
          f[2] = v_frag<HD, BITS>(vw[2], vw[3], 2 * j, zv[1], z6[1]);
          f[3] = v_frag<HD, BITS>(vw[2], vw[3], 2 * j + 1, zv[1], z6[1]);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if constexpr (BITS == 16)
              mma_bf16_16816(o[n][j], f, pb[n][0], pb[n][1]);
            else
              mma_f16_16816(o[n][j], f, pb[n][0], pb[n][1]);
          }
        }
        if (SOME && BITS == 16 && __any_sync(0xffffffffu, odd)) {
          for (int p = 0; p < kSub && q0 + p < most; ++p)
#pragma unroll
            for (int j = 0; j < L::NJ; ++j) {
              const int at = L::v_at(j, gr) * 2;
              uint32_t w[1];
              lds_words(w, sv + p * L::ROW + (((at >> 4) ^ L::v_swz(p)) << 4) + (at & 12));
              const float f = at & 2 ? bf_hi(w[0]) : bf_lo(w[0]);
              if (isfinite(f)) continue;
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if (q0 + p < limit[n][e]) o[n][j / 2][2 * (j % 2) + e] += f;
            }
        }
      }
    };

    int stage = 0, into = L::NS - 1;
    for (int k = 0; k < nu; ++k) {
      cp_async_wait_group<L::NS - 2>();
      __syncwarp();
      // (every lane has read what this stage held, the one before)
      copy_unit(k + L::NS - 1, into);
      into = into + 1 == L::NS ? 0 : into + 1;
      const uint32_t st = ring_at + stage * L::STAGE;
      stage = stage + 1 == L::NS ? 0 : stage + 1;
      const int p0 = (u0 + kWarps * k) * L::UNIT;
      if (p0 + L::UNIT > least)
        unit(st, p0, std::true_type());
      else
        unit(st, p0, std::false_type());
    }
    cp_async_wait_all();
    __syncthreads();  // the rings are read to their end

    // ---- the warps' results, over the rings
    float(*so)[ROWS][OS] = reinterpret_cast<float(*)[ROWS][OS]>(paged_ring);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int d = 4; d <= 16; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
        const int r = 8 * n + 2 * tc + e;
        if (gr == 0) {
          sm[warp][r] = m[n][e];
          sl[warp][r] = l[n][e];
        }
#pragma unroll
        for (int j = 0; j < L::NJ; ++j) so[warp][r][L::v_at(j, gr)] = o[n][j / 2][2 * (j % 2) + e];
      }
    __syncthreads();
    const bool whole = blk0 == 0 && blk1 == s.blocks;
    // the warps' results added up in their order: the rows' outputs, or this CTA's part of them
    auto add_up = [&](bool all, float *part) {
      for (int i = tid; i < ROWS * HD / 2; i += kWarps * 32) {
        const int r = i / (HD / 2), e = 2 * (i % (HD / 2)), row = r0 + r;
        if (row >= R) break;
        float M = -INFINITY, Ls = 0.f, O0 = 0.f, O1 = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm[w][r]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = sm[w][r] == -INFINITY ? 0.f : ex2(sm[w][r] - M);
          Ls = fmaf(sl[w][r], f, Ls);
          O0 = fmaf(so[w][r][e], f, O0);
          O1 = fmaf(so[w][r][e + 1], f, O1);
        }
        if (all) {
          if (Ls == 0.f) Ls = NAN;  // scores that are all -inf have no softmax
          *reinterpret_cast<uint32_t *>(reinterpret_cast<__nv_bfloat16 *>(a.o) +
                                        ((size_t)(s.q0 + row / rep) * a.H + g * rep + row % rep) * HD + e) =
              s.len == 0 ? 0u : pack_bf2(O0 / Ls, O1 / Ls);  // (not served: zeros)
        } else {
          float *pt = part + (size_t)r * PS;
          *reinterpret_cast<float2 *>(pt + e) = make_float2(O0, O1);
          if (e == 0) *reinterpret_cast<float2 *>(pt + HD) = make_float2(M, Ls);
        }
      }
    };
    // of the CTAs that share the item, c0 has its begin (in its place 1), the others their first blocks (0)
    auto part_of = [&](long long cta, bool begin) { return a.part + ((size_t)cta * 2 + begin) * kMostRows * PS; };
    add_up(whole, part_of(c, blk0 == 0));
    if (!whole) {
      const int c0 = (int)(((item + 1) * N - 1) / total), parts = (int)(((item + s.blocks) * N - 1) / total) - c0 + 1;
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        last = atomicAdd(&a.counters[c0], 1) == parts - 1;
        if (last) a.counters[c0] = 0;
      }
      __syncthreads();
      if (last) {
        // all parts: warp w adds up w, w + 4, .. in order, a row's HD / 4 lanes 16 bytes each, then the warps in order
        __threadfence();
        constexpr int LPR = HD / 4, RPW = 32 / LPR, CU = 8;
        const int e = 4 * (lane % LPR);
        for (int rr = 0; rr < min(ROWS, R - r0); rr += RPW) {
          const int r = min(rr + lane / LPR, ROWS - 1);
          float M = -INFINITY, Ls = 0.f;
          float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int k0 = warp; k0 < parts; k0 += CU * kWarps) {
            float2 ml[CU];
            float4 ov[CU];
            float mn = M;
#pragma unroll
            for (int j = 0; j < CU; ++j) {
              const int k = k0 + j * kWarps;
              const float *pt = part_of(c0 + min(k, parts - 1), k == 0) + (size_t)r * PS;
              ml[j] = k < parts ? __ldcg(reinterpret_cast<const float2 *>(pt + HD)) : make_float2(-INFINITY, 0.f);
              ov[j] = k < parts ? __ldcg(reinterpret_cast<const float4 *>(pt + e)) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int j = 0; j < CU; ++j) mn = fmaxf(mn, ml[j].x);
            const float f0 = M == -INFINITY ? 0.f : ex2(M - mn);
            M = mn;
            Ls *= f0;
            O.x *= f0, O.y *= f0, O.z *= f0, O.w *= f0;
#pragma unroll
            for (int j = 0; j < CU; ++j) {
              const float f = ml[j].x == -INFINITY ? 0.f : ex2(ml[j].x - M);  // (a NaN of a part stays NaN)
              Ls = fmaf(ml[j].y, f, Ls);
              O.x = fmaf(ov[j].x, f, O.x), O.y = fmaf(ov[j].y, f, O.y), O.z = fmaf(ov[j].z, f, O.z), O.w = fmaf(ov[j].w, f, O.w);
            }
          }
          if (lane % LPR == 0) sm[warp][r] = M, sl[warp][r] = Ls;
          so[warp][r][e] = O.x, so[warp][r][e + 1] = O.y, so[warp][r][e + 2] = O.z, so[warp][r][e + 3] = O.w;
        }
        __syncthreads();
        add_up(true, nullptr);
      }
    }
    __syncthreads();  // the rings take the next item's positions
  }
}

int attn_paged_ctas(int num_sms) { return kCtasPerSm * num_sms; }

size_t attn_paged_part_floats(int hd, int num_sms) {
  return (size_t)attn_paged_ctas(num_sms) * 2 * kMostRows * (hd + 4);
}

namespace {

template <int HD, int BITS, int NT>
cudaError_t launch_t(const AttnPagedArgs &a, int num_sms, cudaStream_t s) {
  using L = Lay<HD, BITS>;
  constexpr int out = kWarps * 8 * NT * (HD + 4) * 4, smem = L::RING > out ? L::RING : out;
  static std::atomic<bool> done[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  auto k = attn_paged_kernel<HD, BITS, NT>;
  if (dev < 0 || dev >= 64 || !done[dev].load(std::memory_order_acquire)) {
    if ((e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
  }
  // as many CTAs as the SMs hold at once, and no more than blocks there can be
  const long long tiles = ((long long)a.m * (a.H / a.Hkv) + 8 * NT - 1) / (8 * NT) + a.batch;
  const long long blocks = (((long long)a.max_pages << a.shift) + L::BLOCK - 1) / L::BLOCK;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)std::min((long long)occupancy(HD, BITS, NT) * num_sms, std::min(tiles, (long long)1 << 30) * blocks * a.Hkv));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  return cudaLaunchKernelEx(&cfg, k, a);
}

}  // namespace

cudaError_t launch_attn_paged(const AttnPagedArgs &a, int hd, int bits, int num_sms, cudaStream_t s) {
  const bool one = (long long)std::min(a.max_q, a.most_q) * (a.H / a.Hkv) <= 8;
#define WQ_PAGED(HD, BITS) \
  if (hd == HD && bits == BITS) return one ? launch_t<HD, BITS, 1>(a, num_sms, s) : launch_t<HD, BITS, 2>(a, num_sms, s);
  WQ_PAGED(128, 16) WQ_PAGED(128, 8) WQ_PAGED(128, 4) WQ_PAGED(64, 16) WQ_PAGED(64, 8) WQ_PAGED(64, 4)
#undef WQ_PAGED
  return cudaErrorInvalidValue;
}

cudaError_t read_attn_paged_status(int *status) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(status, g_attn_paged_status, sizeof(int));
  if (e != cudaSuccess) return e;
  const int zero = 0;
  return cudaMemcpyToSymbol(g_attn_paged_status, &zero, sizeof(int));
}

}  // namespace wq
