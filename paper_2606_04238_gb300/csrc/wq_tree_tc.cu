// wq_tree_tc.cu -- attention of a tree of drafted tokens over a KV cache on the
// tcgen05 tensor cores (sm_103a): the mathematics of wq_tree.cu for calls with
// more rows (drafts x query heads of a kv head) than one m16 tile.
//
// A CTA takes one (b, g), a block of 128 rows and a range of 128-position tiles:
//   S = Q K^T   128 x 128 in TMEM, Q and K in shared memory (K-major);
//   P           binary16 (bf16 cache: bf16) over S's own TMEM columns, rounded from
//               the fp32 softmax of one thread a row;
//   O += P V    128 x HD in TMEM, P as the A operand from TMEM, V [position][HD] in
//               shared memory as it lies in the cache (MN-major).
// Thirteen warps: 0-3 softmax (thread = row), 4-11 load a tile's codes into registers
// one tile ahead, convert them and store them in the 128-byte swizzled layout, 12 issues
// the MMAs.  K's operands are code - z, exact, its scales factors of the scores.  V's are
// (code - z) s 2^-t rounded to binary16, t one for a tile: 2^-11 of each term at most, for
// which the rows' threads, the longest chain, need no factor a position.  P rounds like
// wq_tree.cu's.  Two CTAs an SM (256 TMEM columns and ~100 KB
// each) fill each other's waits: a tile's products, softmax and products again are
// one chain.  A draft tile's rows are brought into binary16 by an exact power of two
// a row, V's taken into the exponent of the row's p (a masked draft then has no say in the
// others' steps, whatever it holds); so are V's rows of a context tile whose scales are far
// apart.  The running maximum is raised, and O rescaled in TMEM, only when 32 of a
// row's probabilities add up to 2^8: p stays below that, and no maximum is searched.
//
// The tiles of all (b, g, row block) are dealt to the CTAs in nearly equal
// ranges: every CTA finds the tiles a range takes from the lengths themselves.
// Ranges of one row block that is split are merged by a second kernel.
//
// Measured (device time): 4 sequences of 9,400 to 15,600 positions in 4 bits, 47 to 61
// drafts, 40 query heads over 8 kv heads of 128: 89 us, 450 TFLOP/s of products that
// count.  8 sequences of 1,300 to 3,900 positions in bf16, 33 to 60 drafts, 64 heads over
// 8 of 64: 55 us.  16 sequences of 580 to 1,950 positions in 8 bits, 4 to 8 drafts: 34 us,
// of which 7 until the queries are in place and 8 from the last tile to the merged rows.
// A tile of 128 positions takes a CTA 1.8 us (bf16, 64) to 2.9 us (4 bits, 128) with two
// CTAs an SM, 1.6 and 2.3 alone.  No one part bounds it: about half the issue slots, half
// the tensor rate (whole tiles) and 60% of shared memory's bandwidth are in use, and copies
// that leave out the exponentials, the conversion or either product are at most 8% faster.
// Scores and outputs in halves of 64 positions, so that a half's softmax runs beside the
// other's products, gained nothing (57 -> 56 and 92 -> 96 us): a row's thread then never
// waits, and its own instructions, ~4 clocks each, are the chain.  64 columns a thread at
// a time (one wait for the scores, no branch between) took 134 us for 92: K's scales then
// come from shared memory one load after the other.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cstdint>

#include "wq_cvt.cuh"
#include "wq_internal.h"
#include "wq_kv.h"
#include "wq_ptx.cuh"

namespace wq {

// Status word: WQ_OK (0), WQ_ERR_ARG (-1) after a length or count outside its
// range (that sequence is skipped), WQ_ERR_TIMEOUT (-6) after a wait ran out.
__device__ int g_tree_tc_status = 0;

namespace {

constexpr int kTcRows = 128;      // rows a CTA takes
constexpr int kTile = 128;        // positions a tile
constexpr int kConv = 256;        // converting threads
constexpr int kTcThreads = 128 + kConv + 32;
constexpr int kMmaWarp = 4 + kConv / 32;
constexpr int kBlk = kTile * 128;  // bytes of a 64-value block of Q, K or V: [row][128 bytes], swizzled
constexpr int kTmemCols = 256;    // S / P 0..127, O 128..
// Queries enter binary16 times 2^7, which keeps a row with its largest |q| in [2^-4, 2^8) whole but for values
// below 2^-27 of that; other rows by a power of two of their own.
constexpr int kQueryShift = 7;
// Exponents that a draft's V can bring into its score over a quantized cache.  The least is that of zeros, below what the
// smallest scale gives; with the most, the context's probabilities are still normal numbers in the sums.
constexpr int kLeastSize = -40, kMostSize = 64;
// Exponents that V's scales of a tile may span with one power of two for all: a small row's terms then have steps of up to
// 2^8 times 2^-25 of the largest.  Beyond it each row has its own, as drafts have (4 x 64 drafts over 13,000 positions of
// 4 bits: 124 us with no such tile, 170 with such tiles alone).
constexpr int kSpread = 8;
// registers a thread: the launch's 72 x 416 shared out as 104 x 128 + 56 x 256 + 72 x 32
constexpr int kRegsSoftmax = 104, kRegsConv = 56;

__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
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
// The exact power of two 2^e that puts a row's largest value mx (not 0) in [2^top,
// 2^(top + 1)); kept where 2^e and 2^-e are normal.  An infinite mx: 2^(top - 128),
// which keeps every finite value in range.
__device__ __forceinline__ int f16_shift(float mx, int top) {
  const int e = (int)(__float_as_uint(mx) >> 23) - 127;
  return mx == 0.f ? 0 : min(126, top - e);
}

// 32 lanes x 16 consecutive 32-bit TMEM columns, written.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
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
// B operand [k][n] with n contiguous (MN-major), 128-byte swizzle: blocks of 64 n
// `lbo` bytes apart, groups of 8 k 1024 bytes apart.
__device__ __forceinline__ uint64_t umma_desc_mnmajor_sw128(uint32_t saddr, uint32_t lbo) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// fp32 accumulator, A and B binary16 or bf16, A K-major, B K-major or MN-major.
__host__ __device__ constexpr uint32_t tree_idesc(int N, bool bf16, bool b_mn) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(kTcRows >> 4) << 24);
}

// 2^(m - mn) for a maximum raised from m to mn (whole numbers, or infinite).
__device__ __forceinline__ float raise_factor(float m, float mn) {
  const float d = m - mn;
  return mn == m ? 1.f : d < -126.f ? 0.f : pow2i((int)d);
}
// What a row has so far, times al: its probabilities of the tile's first 32 pc columns, and 16 oc columns of O.
template <bool BF>
__device__ __noinline__ void rescale(uint32_t tw, int pc, int oc, float al) {
  tmem_st_wait();
#pragma unroll 1
  for (int c = 0; c < pc; ++c) {
    uint32_t p[16];
    tmem_ld16(tw + 16 * c, p);
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 16; ++e)
      p[e] = BF ? pack_bf2(bf_lo(p[e]) * al, bf_hi(p[e]) * al) : hmul2_u(p[e], pack_h2(al, al));
    tmem_st16(tw + 16 * c, p);
  }
#pragma unroll 1
  for (int c = 0; c < oc; ++c) {
    uint32_t o[16];
    tmem_ld16(tw + 128 + 16 * c, o);
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * al);
    tmem_st16(tw + 128 + 16 * c, o);
  }
}

// Infinities and NaN among four columns of a bf16 cache's V, n positions from vp on: every row sees them, so a column that
// has any is their sum; a copy's p of 0 for the others' positions made it NaN.  (A quantized cache has NaN rows only.)
template <int HD>
__device__ __noinline__ float4 column_infinities(const __nv_bfloat16 *vp, int n, float4 o) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < n; ++p) {
    const uint2 x = __ldg(reinterpret_cast<const uint2 *>(vp + (size_t)p * HD));
    const float f[4] = {bf_lo(x.x), bf_hi(x.x), bf_lo(x.y), bf_hi(x.y)};
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += isfinite(f[e]) ? 0.f : f[e];
  }
  if (s[0] != 0.f) o.x = s[0];
  if (s[1] != 0.f) o.y = s[1];
  if (s[2] != 0.f) o.z = s[2];
  if (s[3] != 0.f) o.w = s[3];
  return o;
}

// What a CTA takes: row block rb of (b, g), tiles t0 .. t1 - 1 (drafts' tiles
// first); n splits of the row block, this is `split`, its partial results at `slot`.
struct Work {
  int b, g, rb, t0, t1, split, n, slot, len, cnt;
  bool any;
};

// Tiles of sequence b, and its row blocks; 0 tiles where a length or count is out
// of range.
__device__ __forceinline__ void seq_tiles(const TreeArgs &a, int b, int rep, int &len, int &cnt, int &tiles, int &blocks) {
  len = a.lens[b];
  cnt = a.counts ? a.counts[b] : a.T;
  const bool bad = len < 0 || len > a.max_len || cnt < 0 || cnt > a.T;
  tiles = bad ? 0 : cnt == 0 ? 1 : (cnt + kTile - 1) / kTile + (len + kTile - 1) / kTile;
  blocks = bad ? 0 : max(1, (cnt * rep + kTcRows - 1) / kTcRows);
}

// a / b rounded up, 0 <= a < 2^22, by the reciprocal: the product is within 1 of the quotient.
__device__ __forceinline__ int ceil_div(int a, int b, float rb) {
  int q = (int)(__int2float_rn(a) * rb);
  q -= q * b > a;
  q += (q + 1) * b <= a;
  return q + (q * b < a);
}

// One warp, every CTA the same sums.  Ranges of W tiles: W the least of 32 candidates, from the tiles a CTA of an even
// split would take up to what certainly gives no more than `target` ranges; then this CTA's range.
// Whole row blocks, W the most tiles, where they are `target` already or the host launches no merge.
__device__ Work find_work(const TreeArgs &a, int rep, int cta) {
  const int lane = threadIdx.x & 31;
  int len = 0, cnt = 0, tiles = 0, blocks = 0;
  unsigned total = 0, many = 0;  // (32 bits: tiles x kv heads x row blocks of what fits in memory)
  const unsigned target = (unsigned)a.target;
  int most = 1;
  for (int b = lane; b < a.batch; b += 32) {
    seq_tiles(a, b, rep, len, cnt, tiles, blocks);
    total += tiles * blocks;
    many += blocks;
    most = max(most, tiles);
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    total += __shfl_xor_sync(0xffffffffu, total, o);
    many += __shfl_xor_sync(0xffffffffu, many, o);
  }
  most = __reduce_max_sync(0xffffffffu, most);
  total *= a.Hkv;
  many *= a.Hkv;
  int W = most;
  if (a.split && many < target && most > 1) {
    // sum ceil(tiles / W) <= total / W + many: no more than `target` at hi
    const int lo = max(1, (int)((total + target - 1) / target));
    const int hi = min(most, max(lo, (int)((total + (target - many) - 1) / (target - many))));
    const int cand = lo + (hi - lo) / 31 * lane + (hi - lo) % 31 * lane / 31;
    const float rc = __frcp_rn((float)cand);
    unsigned n = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
      if (a.batch > 32) {
        tiles = blocks = 0;
        if (b0 + lane < a.batch) seq_tiles(a, b0 + lane, rep, len, cnt, tiles, blocks);
      }
      const int m = min(32, a.batch - b0);
#pragma unroll 4
      for (int j = 0; j < m; ++j)
        n += ceil_div(__shfl_sync(0xffffffffu, tiles, j), cand, rc) * __shfl_sync(0xffffffffu, blocks, j);
    }
    const unsigned fits = __ballot_sync(0xffffffffu, n * a.Hkv <= target);
    W = __shfl_sync(0xffffffffu, cand, fits ? __ffs(fits) - 1 : 31);
  }
  if (cta == 0 && lane == 0) a.table[a.batch] = make_int4(W < most, 0, 0, 0);
  const float rw = __frcp_rn((float)W);
  // the sequence this CTA falls into
  Work w;
  w.any = false;
  unsigned base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    const int b = b0 + lane;
    if (a.batch > 32) {
      tiles = blocks = len = cnt = 0;
      if (b < a.batch) seq_tiles(a, b, rep, len, cnt, tiles, blocks);
    }
    const int n = ceil_div(tiles, W, rw), mine = n * blocks * a.Hkv;
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, cta < (int)(base + incl));
    if (cta == 0 && b < a.batch) {
      a.table[b] = make_int4((int)(base + incl - mine), n, blocks, cnt);
      if (tiles == 0) atomicExch(&g_tree_tc_status, -1);
    }
    if (hit && !w.any) {
      const int src = __ffs(hit) - 1;
      const int first = (int)(base + __shfl_sync(0xffffffffu, incl - mine, src));
      w.any = true;
      w.b = b0 + src;
      w.n = __shfl_sync(0xffffffffu, n, src);
      const int rbs = __shfl_sync(0xffffffffu, blocks, src), nt = __shfl_sync(0xffffffffu, tiles, src);
      w.len = __shfl_sync(0xffffffffu, len, src);
      w.cnt = __shfl_sync(0xffffffffu, cnt, src);
      const int i = cta - first;  // (split, g, row block), the row block fastest
      w.rb = i % rbs;
      w.g = i / rbs % a.Hkv;
      w.split = i / (rbs * a.Hkv);
      const int each = nt / w.n, more = nt - each * w.n;  // nt split / n = each split + more split / n
      w.t0 = each * w.split + more * w.split / w.n;
      w.t1 = each * (w.split + 1) + more * (w.split + 1) / w.n;
      w.slot = cta;
      if (cta != 0) break;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  return w;
}

template <int HD, int BITS>
struct Cfg {
  static constexpr int NB = HD / 64;             // 64-value blocks
  static constexpr int KB = NB * kBlk;           // bytes of one operand tile
  static constexpr int CH = HD / 8;              // 16-byte chunks a row of 16-bit values
  static constexpr int IT = kTile * CH / kConv;  // chunks a converting thread takes
  static constexpr int RS = kConv / CH;          // rows between them
  static constexpr int SMEM = 1024 + 3 * KB;     // Q, K, V
};

struct Shared {
  uint64_t k_full, k_empty, v_full, v_empty, s_full, p_full;
  uint32_t tmem;
  int fail;
  uint32_t odd[4];  // drafts whose V has values that are not finite
  int wide;         // a draft's V is beyond binary16 with its exponent at kMostSize: V of the tile is bf16, and p too
  Work work;
  // of a tile: K's scales (times the score scale and the queries' 2^-kQueryShift) and the exponent t of V's operands, which are values
  // times 2^-t.  Two tiles of each: the next tile's are written while this one's are read
  __align__(16) float sk[2][kTile];
  int te[2], spread[2];  // spread: V's scales span more than kSpread exponents, and each row has a t of its own
  uint32_t zk[kTile];                        // 1024 + z of K, twice
  __align__(16) uint2 zsv[kTile];            // 1024 + z of V, twice; its scale times 2^-t, twice
  __align__(16) uint32_t top[2][8];          // four warps' shares of the least and of the largest V scale of a tile (bits)
  __align__(16) float td[2][kTile], tw[2][kTile];  // rows' own exponents t of V (drafts, spread), 2^-t
};

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
    o.x = hsub2_u((c.x & 0x000f000fu) | 0x64006400u, z1024);
    o.y = hfma16_u((c.x & 0x00f000f0u) | 0x64006400u, z64);
    o.z = hsub2_u((x & 0x000f000fu) | 0x64006400u, z1024);
    o.w = hfma16_u((x & 0x00f000f0u) | 0x64006400u, z64);
  }
  return o;
}

}  // namespace

template <int HD, int BITS>
__global__ void __launch_bounds__(kTcThreads, 2) attn_tree_tc_kernel(const TreeArgs a) {
  using C = Cfg<HD, BITS>;
  constexpr bool BF = BITS == 16;
  constexpr int ROW = HD * BITS / 8;
  extern __shared__ uint8_t tree_dyn[];
  __shared__ Shared sh;
  uint8_t *qbuf = tree_dyn + (1024 - (smem_addr(tree_dyn) & 1023)) % 1024, *kbuf = qbuf + C::KB, *vbuf = kbuf + C::KB;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rep = a.H / a.Hkv;
  if (warp == kMmaWarp) {
    tmem_alloc(&sh.tmem, kTmemCols);
    if (lane == 0) {
      mbar_init(&sh.k_full, kConv / 32);
      mbar_init(&sh.v_full, kConv / 32);
      mbar_init(&sh.k_empty, 1);
      mbar_init(&sh.v_empty, 1);
      mbar_init(&sh.s_full, 1);
      mbar_init(&sh.p_full, 4);
      fence_barrier_init();
      sh.fail = 0;
    }
  } else if (warp == 4 && lane < 4) {
    sh.odd[lane] = 0;
    sh.wide = 0;
  }
  pdl_wait();
  pdl_launch_dependents();
  if (warp == 0) {
    const Work w = find_work(a, rep, blockIdx.x);
    if (lane == 0) sh.work = w;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const Work w = sh.work;
  const uint32_t tm = sh.tmem;
  const int row0 = w.any ? w.rb * kTcRows : 0;
  const int R = a.T * rep, live = w.any ? min(w.cnt * rep - row0, kTcRows) : 0;  // rows of drafts that exist
  const int nt = live > 0 ? w.t1 - w.t0 : 0;
  const int ndr = w.any && w.cnt > 0 ? 1 : 0;  // the drafts are one tile
  auto draft_of = [&](int row) { return row * a.rep_magic >> 16; };  // row / rep
  // a warp's arrival, its shared-memory writes made visible to the tensor cores
  auto hand_over = [&](uint64_t *bar) {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
  };
  // all lanes alike: a warp leaves its loop as one after a timeout
  auto wait = [&](uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)) != 0; };

  if (nt > 0 && warp == kMmaWarp) {
    // ---- MMAs
    constexpr uint32_t idqk = tree_idesc(kTile, BF, false), idpv = tree_idesc(HD, BF, true);
    const uint64_t qd = umma_desc_kmajor_sw128(smem_addr(qbuf), 1024), kd = umma_desc_kmajor_sw128(smem_addr(kbuf), 1024);
    const uint64_t vd = umma_desc_mnmajor_sw128(smem_addr(vbuf), kBlk);
    if (elect_one()) {
      bool ok = mbar_wait(&sh.p_full, 0);  // Q is in place
      for (int i = 0; i < nt && ok; ++i) {
        ok = mbar_wait(&sh.k_full, i & 1);
        // P V of the tile before has read P, which S overwrites
        if (ok && i > 0) ok = mbar_wait(&sh.v_empty, (i - 1) & 1);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks) {
          const uint64_t off = (uint64_t)(((ks / 4) * kBlk + (ks % 4) * 32) >> 4);
          umma_f16(tm, qd + off, kd + off, idqk, ks > 0);
        }
        umma_commit(&sh.s_full);
        umma_commit(&sh.k_empty);
        ok = mbar_wait(&sh.v_full, i & 1) && mbar_wait(&sh.p_full, (i + 1) & 1);
        if (!ok) break;
        tc_fence_after();
        const uint32_t id = !BF && i == 0 && w.t0 < ndr && sh.wide ? tree_idesc(HD, true, true) : idpv;
#pragma unroll
        for (int ks = 0; ks < kTile / 16; ++ks)
          umma_ts(tm + 128, tm + 8 * ks, vd + (uint64_t)((ks * 2048) >> 4), id, i > 0 || ks > 0);
        umma_commit(&sh.v_empty);
      }
      if (!ok) sh.fail = 1;
    }
    __syncwarp();
  } else if (nt > 0 && warp >= 4) {
    // ---- loads and conversion: chunk c of rows r0 + it RS
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsConv));
    const int ct = tid - 128, c = ct % C::CH, r0 = ct / C::CH;
    const uint32_t dst0 = (c / 8) * kBlk + r0 * 128 + (((c & 7) ^ (r0 & 7)) << 4);
    const size_t base = ((size_t)w.b * a.Hkv + w.g) * a.max_len;
    const uint8_t *kc = reinterpret_cast<const uint8_t *>(a.kc) + base * ROW + c * BITS;
    const uint8_t *vc = reinterpret_cast<const uint8_t *>(a.vc) + base * ROW + c * BITS;
    uint2 kr[C::IT], vr[C::IT];
    uint32_t meta = 0;
    auto fetch = [&](const uint8_t *src, uint2 (&r)[C::IT], int p0) {
#pragma unroll
      for (int it = 0; it < C::IT; ++it) {
        const uint8_t *p = src + (size_t)(uint32_t)min(p0 + r0 + it * C::RS, w.len - 1) * ROW;
        if (BITS == 8)
          r[it] = __ldg(reinterpret_cast<const uint2 *>(p));
        else if (BITS == 4)
          r[it].x = __ldg(reinterpret_cast<const uint32_t *>(p));
      }
    };
    auto fetch_meta = [&](int p0) {
      if (!BF) meta = __ldg((ct < kTile ? a.km : a.vm) + base + min(p0 + (ct & (kTile - 1)), w.len - 1));
    };
    // copies of a bf16 tile, straight to its place; zeros past the length
    auto copy = [&](const uint8_t *src, uint8_t *to, int p0) {
#pragma unroll
      for (int it = 0; it < C::IT; ++it) {
        const int p = p0 + r0 + it * C::RS;
        cp_async16_zfill(to + dst0 + it * C::RS * 128, src + (size_t)(uint32_t)min(p, w.len - 1) * ROW,
                         p < w.len ? 16u : 0u);
      }
      cp_async_commit();
    };
    const __nv_bfloat16 *kd = reinterpret_cast<const __nv_bfloat16 *>(a.kn) + ((size_t)w.b * a.T * a.Hkv + w.g) * HD + c * 8;
    const __nv_bfloat16 *vd = reinterpret_cast<const __nv_bfloat16 *>(a.vn) + ((size_t)w.b * a.T * a.Hkv + w.g) * HD + c * 8;
    // chunk it of the drafts' rows; V's values that are not finite are noted and taken out
    auto draft_chunk = [&](const __nv_bfloat16 *src, int it, bool is_v, uint32_t (&x)[4]) {
      const int j = r0 + it * C::RS;
      const uint4 v = j < w.cnt ? __ldg(reinterpret_cast<const uint4 *>(src + (size_t)j * a.Hkv * HD)) : make_uint4(0, 0, 0, 0);
      x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
      if (!is_v) return;
      bool odd = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u, odd = true;
        if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu, odd = true;
      }
      if (odd) atomicOr(&sh.odd[j / 32], 1u << (j % 32));
    };
    auto largest = [&](const uint32_t (&x)[4]) {
      float mx = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, fmaxf(fabsf(bf_lo(x[e])), fabsf(bf_hi(x[e]))));
      return mx;
    };
    auto scaled = [&](uint32_t (&x)[4], float f) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = pack_h2(bf_lo(x[e]) * f, bf_hi(x[e]) * f);
    };
    const float qscale = a.scale * pow2i(-kQueryShift);  // of K's scales
    // The drafts' tile: K and V in binary16 by a power of two a row (bf16 cache: as they are).  V's brings its largest
    // value to [2^(BITS + 5), 2^(BITS + 6)), where a code times a scale is at most.
    auto draft_tile = [&]() {
      const int its = min(C::IT, (w.cnt + C::RS - 1) / C::RS);  // chunks with drafts in them
#pragma unroll 1
      for (int it = 0; it < its; ++it) {
        uint32_t x[4], y[4];
        draft_chunk(kd, it, false, x);
        draft_chunk(vd, it, true, y);
        if constexpr (!BF) {
          float mx = largest(x), mv = largest(y);
#pragma unroll
          for (int o = C::CH / 2; o >= 1; o >>= 1) {
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, o));
          }
          const int e2 = f16_shift(mx, 14);
          scaled(x, pow2i(e2));
          if (c == 0) {
            const int r = r0 + it * C::RS, ev = (int)(__float_as_uint(mv) >> 23) - 127 - (BITS + 5);
            const int t = min(max(ev, kLeastSize), kMostSize);
            sh.sk[0][r] = qscale * pow2i(-e2);
            sh.td[0][r] = (float)t;
            sh.tw[0][r] = pow2i(-t);
            if (ev > kMostSize) sh.wide = 1;
          }
        } else {
          *reinterpret_cast<uint4 *>(vbuf + dst0 + it * C::RS * 128) = make_uint4(y[0], y[1], y[2], y[3]);
        }
        *reinterpret_cast<uint4 *>(kbuf + dst0 + it * C::RS * 128) = make_uint4(x[0], x[1], x[2], x[3]);
      }
      // (K's other rows hold what they held: their scores are not looked at)
      if constexpr (!BF) {
        if (c == 0)
#pragma unroll 1
          for (int it = its; it < C::IT; ++it) sh.td[0][r0 + it * C::RS] = sh.tw[0][r0 + it * C::RS] = 0.f;
        if (ct == 0) sh.te[0] = 0;
        hand_over(&sh.k_full);
        named_barrier_sync(1, kConv);
        const bool wide = sh.wide != 0;
#pragma unroll 1
        for (int it = 0; it < its; ++it) {
          uint32_t y[4];
          draft_chunk(vd, it, true, y);
          if (!wide) scaled(y, sh.tw[0][r0 + it * C::RS]);
          *reinterpret_cast<uint4 *>(vbuf + dst0 + it * C::RS * 128) = make_uint4(y[0], y[1], y[2], y[3]);
        }
      } else {
        hand_over(&sh.k_full);
      }
#pragma unroll 1
      for (int it = its; it < C::IT; ++it)
        *reinterpret_cast<uint4 *>(vbuf + dst0 + it * C::RS * 128) = make_uint4(0, 0, 0, 0);
      hand_over(&sh.v_full);
    };
    auto pos_of = [&](int i) { return (w.t0 + i - ndr) * kTile; };
    const int i_ctx = max(0, ndr - w.t0);  // first tile of the context
    bool ok = true;
    if (i_ctx < nt && !BF) {
      fetch_meta(pos_of(i_ctx));
      fetch(kc, kr, pos_of(i_ctx));
      fetch(vc, vr, pos_of(i_ctx));
    }
    if (i_ctx > 0) draft_tile();
    // the warps' least and largest V scale of the tile whose scales this thread holds (bits; a NaN counts as the least)
    auto note_top = [&](int which) {
      if (ct < kTile) return;
      uint32_t v = (meta & 0xffffu) > 0x7c00u ? 0u : meta & 0xffffu;
      if (v == 0 || meta == kZeroRow) v = 1;  // kLeastScale
      const uint32_t lo = __reduce_min_sync(0xffffffffu, v);
      v = __reduce_max_sync(0xffffffffu, v);
      if (lane == 0) sh.top[which][warp - 8] = lo, sh.top[which][warp - 4] = v;
    };
    if (!BF && i_ctx < nt) {
      note_top(i_ctx & 1);
      named_barrier_sync(1, kConv);
    }
    for (int i = i_ctx; i < nt; ++i) {
      const int p0 = pos_of(i);
      if constexpr (BF) {
        // K's place is free once the scores of tile i - 1 are done, V's once its outputs are
        if (i > 0) ok = wait(&sh.k_empty, (i - 1) & 1);
        if (!ok) break;
        copy(kc, kbuf, p0);
        if (i > i_ctx) {  // V of tile i - 1 has landed meanwhile
          cp_async_wait_group1();
          hand_over(&sh.v_full);
        }
        cp_async_wait_all();
        hand_over(&sh.k_full);
        if (i > 0) ok = wait(&sh.v_empty, (i - 1) & 1);
        if (!ok) break;
        copy(vc, vbuf, p0);
      } else {
        const int par = i & 1, pn = i + 1 < nt ? p0 + kTile : p0;
        if (i > 0) ok = wait(&sh.k_empty, (i - 1) & 1);
        // V's operands (code - z) s 2^-t: t puts the tile's largest s in [2^5, 2^6), or where they span too much each
        // row's own, which then counts in the row's score
        const uint4 tops = *reinterpret_cast<const uint4 *>(&sh.top[par][4]), lows = *reinterpret_cast<const uint4 *>(&sh.top[par][0]);
        auto exponent = [](uint32_t h) {
          return (int)(__float_as_uint(__half2float(__ushort_as_half((unsigned short)h))) >> 23) - 127 - 5;
        };
        const int te = exponent(max(max(tops.x, tops.y), max(tops.z, tops.w)));
        const bool spread = te - exponent(min(min(lows.x, lows.y), min(lows.z, lows.w))) > kSpread;
        {
          const float s0 = __half2float(__ushort_as_half((unsigned short)(meta & 0xffffu)));
          const __half2 z = __hadd2(__half2half2(__ushort_as_half((unsigned short)(meta >> 16))), __float2half2_rn(1024.f));
          const uint32_t zz = *reinterpret_cast<const uint32_t *>(&z);
          const int r = ct & (kTile - 1);
          if (ct < kTile) {
            sh.sk[par][r] = s0 * qscale;
            sh.zk[r] = zz;
            if (ct == 0) sh.te[par] = spread ? 0 : te, sh.spread[par] = spread;
          } else {
            float sv = s0 == 0.f || meta == kZeroRow ? kLeastScale : s0;  // (then code - z is 0)
            const int t = spread ? min((int)(__float_as_uint(sv) >> 23) - 127 - 5, te) : te;  // (a NaN scale's: te)
            if (spread) sh.td[par][r] = (float)t, sh.tw[par][r] = pow2i(-t);
            sv *= pow2i(-t);
            sh.zsv[r] = make_uint2(zz, pack_h2(sv, sv));
          }
        }
        ok = barrier_and(1, kConv, ok);  // the warps leave together after a timeout
        if (!ok) break;
        fetch_meta(pn);
#pragma unroll
        for (int it = 0; it < C::IT; ++it)
          *reinterpret_cast<uint4 *>(kbuf + dst0 + it * C::RS * 128) = convert8<BITS>(kr[it], sh.zk[r0 + it * C::RS]);
        hand_over(&sh.k_full);
        fetch(kc, kr, pn);
        if (i > 0) ok = wait(&sh.v_empty, (i - 1) & 1);
#pragma unroll
        for (int it = 0; it < C::IT; ++it) {
          const uint2 zs = sh.zsv[r0 + it * C::RS];
          uint4 v = convert8<BITS>(vr[it], zs.x);
          v.x = hmul2_u(v.x, zs.y), v.y = hmul2_u(v.y, zs.y), v.z = hmul2_u(v.z, zs.y), v.w = hmul2_u(v.w, zs.y);
          *reinterpret_cast<uint4 *>(vbuf + dst0 + it * C::RS * 128) = v;
        }
        hand_over(&sh.v_full);
        fetch(vc, vr, pn);
        note_top(par ^ 1);
        // every warp has read this tile's zeros before the next one's are written
        ok = barrier_and(1, kConv, ok);
        if (!ok) break;
      }
    }
    if constexpr (BF) {
      cp_async_wait_all();
      if (ok && i_ctx < nt) hand_over(&sh.v_full);  // the last tile's V
    }
    if (!ok && lane == 0) sh.fail = 1;
  } else if (nt > 0) {
    // ---- softmax: thread = row.  Up to 64 (32) rows stand twice (four times) in the 128, each copy with its own
    // half (quarter) of a tile's positions, so that all four warps work on them; the copies are merged at the end.
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int rpc = live <= 32 ? 32 : live <= 64 ? 64 : 128, copies = kTcRows / rpc, copy = tid / rpc;
    const int lr = tid & (rpc - 1), t = draft_of(row0 + lr);
    const bool in = lr < live;
    const bool busy = (warp * 32 & (rpc - 1)) < live;  // warps without rows only keep the barriers going
    const uint32_t tw = tm + ((uint32_t)(warp * 32) << 16);
    // c1, of the raw products: bf16 the score scale (its sign in Q); else what a row's own power of two differs from
    // the common one, which K's scales take in
    float c1 = BF ? fabsf(a.scale) : 1.f;
    bool own = false;
    uint32_t see[4] = {0, 0, 0, 0};
    if (busy) {
      // a warp's 32 rows, CH lanes a row: copied to their place, then worked on there
      constexpr int RI = 32 / C::CH;  // rows an instruction
      const int ch = lane % C::CH;
      auto place = [&](int row) { return qbuf + (ch / 8) * kBlk + row * 128 + (((ch & 7) ^ (row & 7)) << 4); };
      const __nv_bfloat16 *q0 = reinterpret_cast<const __nv_bfloat16 *>(a.q) + ((size_t)w.b * a.T * a.H + w.g * rep) * HD + ch * 8;
#pragma unroll 1
      for (int row = warp * 32 + lane / C::CH; row < warp * 32 + 32; row += RI) {
        const int q = row & (rpc - 1), rq = row0 + min(q, live - 1), tq = draft_of(rq);
        cp_async16_zfill(place(row), q0 + ((size_t)tq * a.H + rq - tq * rep) * HD, q < live ? 16u : 0u);
      }
      if (w.t0 < ndr && in) {  // the drafts that the row sees
#pragma unroll
        for (int h = 0; h < 4; ++h)
          if (32 * h < w.cnt)
            see[h] = a.mask ? a.mask[((size_t)w.b * a.T + t) * a.words + h]
                            : t >= 32 * h + 31 ? 0xffffffffu : t < 32 * h ? 0u : (2u << (t - 32 * h)) - 1u;
      }
      cp_async_wait_all();
      __syncwarp();
      // thread = row
      auto chunk = [&](int c) { return reinterpret_cast<uint4 *>(qbuf + (c / 8) * kBlk + tid * 128 + (((c & 7) ^ (tid & 7)) << 4)); };
      if constexpr (BF) {
        if (a.scale < 0.f)
#pragma unroll 4
          for (int c = 0; c < C::CH; ++c) {
            uint4 v = *chunk(c);
            *chunk(c) = make_uint4(v.x ^ 0x80008000u, v.y ^ 0x80008000u, v.z ^ 0x80008000u, v.w ^ 0x80008000u);
          }
      } else {
        uint32_t big = 0;  // the row's largest |q|, as bf16 bits
#pragma unroll
        for (int c = 0; c < C::CH; ++c) {
          const uint4 v = *chunk(c);
          big = __vmaxu2(big, __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
        }
        big = max(big & 0xffffu, big >> 16);
        const int e = (int)(big >> 7) - 127;
        int mine = kQueryShift;
        if (big != 0 && (e < -4 || e >= 8)) mine = max(min(min(126, 14 - e), kQueryShift + 126), -114);
        c1 = pow2i(kQueryShift - mine);
        const float f = pow2i(mine);
        own = __any_sync(0xffffffffu, c1 != 1.f);
#pragma unroll 4
        for (int c = 0; c < C::CH; ++c) {
          const uint4 v = *chunk(c);
          *chunk(c) = make_uint4(pack_h2(bf_lo(v.x) * f, bf_hi(v.x) * f), pack_h2(bf_lo(v.y) * f, bf_hi(v.y) * f),
                                 pack_h2(bf_lo(v.z) * f, bf_hi(v.z) * f), pack_h2(bf_lo(v.w) * f, bf_hi(v.w) * f));
        }
      }
    }
    hand_over(&sh.p_full);  // phase 0: Q
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int i = 0; i < nt; ++i) {
      const int par = i & 1, tile = w.t0 + i;
      // (the scales were written before K was handed to the MMA warp, which issued S after that)
      ok = wait(&sh.s_full, i & 1);
      if (!ok) break;
      tc_fence_after();
      if (busy) {
        // which of the tile's positions count: the drafts the row sees, those before the length
        const bool drafts = tile < ndr, search = i == 0 || (i == 1 && w.t0 < ndr);
        const int left = drafts ? w.cnt : w.len - (tile - ndr) * kTile;
        const bool some = drafts || left < kTile;
        auto seen = [&](int h) {
          const int n = left - 32 * h;
          const uint32_t have = n >= 32 ? 0xffffffffu : (1u << n) - 1u;  // (n > 0: works(h))
          return drafts ? have & (h == 0 ? see[0] : h == 1 ? see[1] : h == 2 ? see[2] : see[3]) : have;
        };
        const bool own_t = !BF && (drafts || sh.spread[par]);  // V's rows have exponents of their own
        const int ti = BF ? 0 : sh.te[par];
        const float te = (float)ti;
        // the 32 columns that this copy works on, where any count
        auto works = [&](int h) { return (h * copies) / 4 == copy && 32 * h < left; };
        // u = the scores of 32 columns less m, from their raw products, where they count
        auto exponents = [&](float (&u)[32], int h, float ms, bool masks) {
          float4 k4[BF ? 1 : 8];
          tmem_ld32(tw + 32 * h, *reinterpret_cast<uint32_t(*)[32]>(&u));
          if constexpr (!BF)
#pragma unroll
            for (int j = 0; j < 8; ++j) k4[j] = *reinterpret_cast<const float4 *>(&sh.sk[par][32 * h + 4 * j]);
          tmem_ld_wait();
          if (!BF && own)
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] *= c1;
          const uint64_t mm = pack_f32x2(ms, ms), cc = pack_f32x2(c1, c1);
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            uint64_t k0 = cc, k1 = cc;
            if constexpr (!BF) k0 = pack_f32x2(k4[j / 4].x, k4[j / 4].y), k1 = pack_f32x2(k4[j / 4].z, k4[j / 4].w);
            unpack_f32x2(fma_f32x2(pack_f32x2(u[j], u[j + 1]), k0, mm), u[j], u[j + 1]);
            unpack_f32x2(fma_f32x2(pack_f32x2(u[j + 2], u[j + 3]), k1, mm), u[j + 2], u[j + 3]);
          }
          if (masks && own_t)
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] += sh.td[par][32 * h + j];
          if (masks && some) {
            const uint32_t bits = seen(h);
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] = bits >> j & 1 ? u[j] : -INFINITY;
          }
        };
        auto largest = [&](const float (&u)[32]) {
          float top[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            top[j] = fmaxf(u[j], u[j + 4]);
#pragma unroll
            for (int e = 8; e < 32; e += 8) top[j] = fmaxf(fmaxf(top[j], u[j + e]), u[j + e + 4]);
          }
          return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        };
        // 32 columns at a time: probabilities with the row's maximum so far.  Where a row's 32 add up to 2^8 (or it
        // has no maximum yet), the maximum is raised first, to a whole number, so that what was computed with the
        // old one is rescaled by exact powers of two.
        float total = 0.f;
        auto probabilities = [&](int h, bool masks) {
          float u[32], part = 0.f;
          uint32_t p[16];
          const float ms = m == -INFINITY ? 0.f : te - m;
          exponents(u, h, ms, masks);
#pragma unroll 1
          for (int again = 0; again < 2; ++again) {
            uint64_t sum[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float e0 = ex2(u[j]), e1 = ex2(u[j + 1]);
              sum[j / 2 % 2] = add_f32x2(sum[j / 2 % 2], pack_f32x2(e0, e1));
              p[j / 2] = BF ? pack_bf2(e0, e1) : pack_h2(e0, e1);
            }
            float s0, s1;
            unpack_f32x2(add_f32x2(sum[0], sum[1]), s0, s1);
            part = s0 + s1;
            const bool up = part >= 256.f || (m == -INFINITY && part > 0.f);
            if (again || !__any_sync(0xffffffffu, up)) break;
            const float mn = up ? ceilf(largest(u) - ms + te) : m;
            const float al = raise_factor(m, mn);
            rescale<BF>(tw, h, i > 0 ? HD / 16 : 0, al);
            m = mn;
            l *= al;
            total *= al;
            const float now = m == -INFINITY ? 0.f : te - m;
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] += now - ms;
          }
          if (masks && own_t) {  // each p stands for 2^-t of itself with a t of its own
            const bool wide = drafts && sh.wide != 0;
            part = 0.f;
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float e0 = ex2(u[j]) * sh.tw[par][32 * h + j], e1 = ex2(u[j + 1]) * sh.tw[par][32 * h + j + 1];
              part += e0 + e1;
              if (wide) p[j / 2] = pack_bf2(e0, e1);
            }
          }
          total += part;
          // columns 16 h ..: S's there have been read
          tmem_st16(tw + 16 * h, p);
        };
        if (!search && copies == 1 && !some && !own_t) {
          // four times in a row: a row's work is bound by latency, which the next columns' loads then overlap
#pragma unroll
          for (int h = 0; h < 4; ++h) probabilities(h, false);
        } else {
          // A range's first tile, the drafts' and the first of the context set the maximum from all their scores (with
          // the drafts' alone to go by, raises in the tiles after it took 6 us of 61).
          if (search) {
            float mx = -INFINITY;
#pragma unroll 1
            for (int h = 0; h < 4; ++h) {
              if (!works(h)) continue;
              float u[32];
              exponents(u, h, te, true);
              mx = fmaxf(mx, largest(u));
            }
            if (__any_sync(0xffffffffu, mx > m)) {
              const float mn = fmaxf(m, ceilf(mx)), al = raise_factor(m, mn);
              if (i > 0 && __any_sync(0xffffffffu, al != 1.f && m > -INFINITY)) rescale<BF>(tw, 0, HD / 16, al);
              m = mn;
              l *= al;
            }
          }
#pragma unroll 1
          for (int h = 0; h < 4; ++h) {
            if (works(h)) {
              probabilities(h, true);
            } else {
              const uint32_t none[16] = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
              tmem_st16(tw + 16 * h, none);
            }
          }
        }
        l = fmaf(total, BF ? 1.f : pow2i(-ti), l);  // p stands for 2^-t of itself
        tmem_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full);
    }
    if (ok) ok = wait(&sh.v_empty, (nt - 1) & 1);
    if (!ok && lane == 0) sh.fail = 1;
    ok = barrier_and(2, 128, ok);
    tc_fence_after();
    if (ok) {
      // ---- the rows' outputs, or their partial results, over shared memory (Q's and K's place): row tid's 16-byte
      // chunk c at c ^ (tid % chunks), so that neither rows nor chunks meet in a bank
      constexpr int CK = HD / 4;
      float4 *stage = reinterpret_cast<float4 *>(qbuf);
      if (busy) {
#pragma unroll 1
        for (int h = 0; h < HD / 32; ++h) {
          uint32_t v[32];
          tmem_ld32(tw + 128 + 32 * h, v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 8; ++j)
            stage[tid * CK + ((8 * h + j) ^ (tid & (CK - 1)))] =
                make_float4(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1]), __uint_as_float(v[4 * j + 2]),
                            __uint_as_float(v[4 * j + 3]));
        }
      }
      float *sm = sh.sk[0], *sl = sh.sk[1];
      sm[tid] = m;
      sl[tid] = l;
      named_barrier_sync(2, 128);
      const bool whole = w.n == 1;
      const bool odd = w.t0 < ndr && (sh.odd[0] | sh.odd[1] | sh.odd[2] | sh.odd[3]) != 0;
      // CK lanes a row (one row a turn: four took 2.5 us more at 64 drafts, code that every CTA fetches once)
      const int c = tid % CK;
#pragma unroll 1
      for (int lrow = tid / CK; lrow < live; lrow += 128 / CK) {
        float M = sm[lrow], L = sl[lrow];
        float4 o = stage[lrow * CK + (c ^ (lrow & (CK - 1)))];
        if (copies > 1) {
#pragma unroll 1
          for (int k = 1; k < copies; ++k) M = fmaxf(M, sm[k * rpc + lrow]);
          float f = sm[lrow] == -INFINITY ? 0.f : ex2(sm[lrow] - M);  // (a NaN of a copy stays NaN)
          L *= f;
          o.x *= f, o.y *= f, o.z *= f, o.w *= f;
#pragma unroll 1
          for (int k = 1; k < copies; ++k) {
            const int row = k * rpc + lrow;
            f = sm[row] == -INFINITY ? 0.f : ex2(sm[row] - M);
            const float4 x = stage[row * CK + (c ^ (row & (CK - 1)))];
            L = fmaf(sl[row], f, L);
            o.x = fmaf(x.x, f, o.x), o.y = fmaf(x.y, f, o.y), o.z = fmaf(x.z, f, o.z), o.w = fmaf(x.w, f, o.w);
          }
          if (BF && !(fabsf((o.x + o.y) + (o.z + o.w)) < INFINITY)) {
            const int p0 = max(0, w.t0 - ndr) * kTile;
            o = column_infinities<HD>(reinterpret_cast<const __nv_bfloat16 *>(a.vc) +
                                          (((size_t)w.b * a.Hkv + w.g) * a.max_len + p0) * HD + 4 * c,
                                      min(w.len, (w.t1 - ndr) * kTile) - p0, o);
          }
        }
        const int ro = row0 + lrow, to = draft_of(ro);
        if (odd) {
#pragma unroll 1
          for (int j = 0; j < w.cnt; ++j) {
            if (!(sh.odd[j / 32] >> (j % 32) & 1)) continue;
            if (!(a.mask ? a.mask[((size_t)w.b * a.T + to) * a.words + j / 32] >> (j % 32) & 1 : j <= to)) continue;
            const __nv_bfloat16 *vj = reinterpret_cast<const __nv_bfloat16 *>(a.vn) +
                                      (((size_t)w.b * a.T + j) * a.Hkv + w.g) * HD + 4 * c;
            float f[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              f[e] = __bfloat162float(vj[e]);
              f[e] = isfinite(f[e]) ? 0.f : f[e];
            }
            o.x += f[0], o.y += f[1], o.z += f[2], o.w += f[3];
          }
        }
        if (whole) {
          const bool none = M == -INFINITY && L == 0.f;  // (all scores NaN: L is NaN)
          const float inv = none ? 0.f : 1.f / L;
          *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(a.o) +
                                     (((size_t)w.b * a.T + to) * a.H + w.g * rep + ro - to * rep) * HD + 4 * c) =
              none ? make_uint2(0, 0) : make_uint2(pack_bf2(o.x * inv, o.y * inv), pack_bf2(o.z * inv, o.w * inv));
        } else {
          float *pt = a.part + ((size_t)w.slot * a.part_rows + lrow) * (HD + 4);
          *reinterpret_cast<float4 *>(pt + 4 * c) = o;
          if (c == 0) *reinterpret_cast<float2 *>(pt + HD) = make_float2(M, L);
        }
      }
    }
  }
  // rows of drafts that do not exist: 0, by the last row block's first split
  if (w.any && w.split == 0 && w.cnt * rep - row0 <= kTcRows) {
    const int z0 = max(row0, w.cnt * rep);
#pragma unroll 1
    for (int i = z0 * (HD / 8) + tid; i < R * (HD / 8); i += kTcThreads) {
      const int row = i / (HD / 8), e = i % (HD / 8), to = draft_of(row);
      *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(a.o) +
                                 (((size_t)w.b * a.T + to) * a.H + w.g * rep + row - to * rep) * HD + 8 * e) =
          make_uint4(0, 0, 0, 0);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (sh.fail) {
    // what the MMA warp issued last is given time to end before its memory goes
    if (tid == 0) atomicExch(&g_tree_tc_status, -6);
    const unsigned long long t0 = global_timer_ns();
    for (int i = 0; i < (1 << 20) && global_timer_ns() - t0 < 2000000ull; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tm, kTmemCols);
  }
}

// o of the rows whose block was split: HD / 4 lanes a row, its parts in split order,
// CU of them loaded in one round trip.  TURNS: a launch that most likely has nothing to
// merge, of few CTAs that take the rows in turn.
template <int HD, int CU, bool TURNS>
__global__ void __launch_bounds__(256) attn_tree_merge_kernel(const TreeArgs a) {
  constexpr int LPR = HD / 4;
  const int rep = a.H / a.Hkv, R = a.T * rep;
  const int c = threadIdx.x % LPR;
  auto merge = [&](int bg, int r, int b, int g) {
    const int4 tab = a.table[b];  // first range, splits, row blocks, drafts
    if (tab.y <= 1 || r >= tab.w * rep) return;  // written by the first kernel, or skipped
    const size_t step = (size_t)a.Hkv * tab.z * a.part_rows * (HD + 4);
    const float *pt = a.part + ((size_t)(tab.x + g * tab.z + r / kTcRows) * a.part_rows + r % kTcRows) * (HD + 4);
    float M = -INFINITY, L = 0.f;
    float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < tab.y; s0 += CU) {
      float2 ml[CU];
      float4 ov[CU];
      float mn = M;
#pragma unroll
      for (int j = 0; j < CU; ++j) {
        const float *ps = pt + (size_t)(s0 + j) * step;
        const bool in = s0 + j < tab.y;
        ml[j] = in ? *reinterpret_cast<const float2 *>(ps + HD) : make_float2(-INFINITY, 0.f);
        ov[j] = in ? *reinterpret_cast<const float4 *>(ps + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int j = 0; j < CU; ++j) mn = fmaxf(mn, ml[j].x);
      const float f0 = M == -INFINITY ? 0.f : ex2(M - mn);
      M = mn;
      L *= f0;
      O.x *= f0, O.y *= f0, O.z *= f0, O.w *= f0;
#pragma unroll
      for (int j = 0; j < CU; ++j) {
        const float f = ml[j].x == -INFINITY ? 0.f : ex2(ml[j].x - M);  // (a NaN of a part stays NaN)
        L = fmaf(ml[j].y, f, L);
        O.x = fmaf(ov[j].x, f, O.x), O.y = fmaf(ov[j].y, f, O.y), O.z = fmaf(ov[j].z, f, O.z), O.w = fmaf(ov[j].w, f, O.w);
      }
    }
    const bool none = M == -INFINITY && L == 0.f;
    *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(a.o) +
                               (((size_t)b * a.T + r / rep) * a.H + g * rep + r % rep) * HD + 4 * c) =
        none ? make_uint2(0, 0) : make_uint2(pack_bf2(O.x / L, O.y / L), pack_bf2(O.z / L, O.w / L));
  };
  long long row = (long long)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  int bg = (int)(row / R), r = (int)(row - (long long)bg * R), b = bg / a.Hkv, g = bg % a.Hkv;
  pdl_wait();
  pdl_launch_dependents();
  if (TURNS && a.table[a.batch].x == 0) return;  // nothing was split
  while (row < (long long)a.batch * a.Hkv * R) {
    merge(bg, r, b, g);
    if (!TURNS) return;
    row += (long long)gridDim.x * (256 / LPR);
    bg = (int)(row / R), r = (int)(row - (long long)bg * R), b = bg / a.Hkv, g = bg % a.Hkv;
  }
}

namespace {

// Once a device: the kernel's shared memory; and whether the warps' shares of
// registers fit into what a block is launched with (their exchange would wait
// forever otherwise).
template <int HD, int BITS>
cudaError_t prepare_tc() {
  static std::atomic<bool> done[64];
  auto k = attn_tree_tc_kernel<HD, BITS>;
  constexpr int smem = Cfg<HD, BITS>::SMEM;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < 64 && done[dev].load(std::memory_order_acquire)) return cudaSuccess;
  cudaFuncAttributes f;
  if ((e = cudaFuncGetAttributes(&f, k)) != cudaSuccess) return e;
  if (kRegsSoftmax * 128 + kRegsConv * kConv > f.numRegs * (128 + kConv)) return cudaErrorInvalidConfiguration;
  if ((e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
  if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
  return cudaSuccess;
}

template <int HD, int BITS>
cudaError_t launch_tree_tc_t(const TreeArgs &a, unsigned grid, bool turns, bool many, cudaStream_t s) {
  constexpr int sm = Cfg<HD, BITS>::SMEM;
  cudaError_t e = prepare_tc<HD, BITS>();
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kTcThreads);
  cfg.dynamicSmemBytes = sm;
  e = cudaLaunchKernelEx(&cfg, attn_tree_tc_kernel<HD, BITS>, a);
  if (e != cudaSuccess || !a.split) return e;
  const long long rows = (long long)a.batch * a.H * a.T;
  cfg.gridDim = dim3((unsigned)std::min((rows * (HD / 4) + 255) / 256, turns ? 2ll * a.target : LLONG_MAX));
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg,
                            turns  ? attn_tree_merge_kernel<HD, 2, true>
                            : many ? attn_tree_merge_kernel<HD, 8, false>
                                   : attn_tree_merge_kernel<HD, 2, false>,
                            a);
}

}  // namespace

// CTAs that the device holds at once.
int tree_tc_target(int num_sms) { return 2 * num_sms; }

size_t tree_tc_part_floats(int batch, int T, int H, int Hkv, int hd, int max_len, int num_sms) {
  // a range of its own for every split, of which there are at most `target`, and at most one a tile
  const long long rows = std::min((long long)T * (H / Hkv), (long long)kTcRows);
  const long long tiles = ((long long)max_len + kTile - 1) / kTile + (T + kTile - 1) / kTile;
  const long long blocks = ((long long)T * (H / Hkv) + kTcRows - 1) / kTcRows;
  return (size_t)(std::min((long long)tree_tc_target(num_sms), (long long)batch * Hkv * blocks * tiles) * rows * (hd + 4));
}

cudaError_t launch_attn_tree_tc(TreeArgs a, int hd, int bits, int num_sms, cudaStream_t s) {
  const int rep = a.H / a.Hkv;
  if (a.scale == 0.f) return cudaErrorInvalidValue;
  const long long blocks = (long long)a.batch * a.Hkv * (((long long)a.T * rep + kTcRows - 1) / kTcRows);
  a.target = tree_tc_target(num_sms);
  a.part_rows = std::min(a.T * rep, kTcRows);
  a.rep_magic = (65536 + rep - 1) / rep;  // row / rep = row rep_magic >> 16 for row < 65536 / (rep - 1)
  const long long tiles = ((long long)a.max_len + kTile - 1) / kTile + (a.T + kTile - 1) / kTile;
  const unsigned grid = (unsigned)std::max(blocks, std::min((long long)a.target, blocks * tiles));
  // Few row blocks are split often and are few rows: eight parts in one round trip (38 parts a block: a call 39.0 us
  // for 45.3); else two, as more warps then fit (2 parts of 488 rows, 64 heads: 1.2 us less).
  const bool many = blocks * 8 <= a.target;
  // Row blocks are split where those of the drafts that exist are fewer than `target`: the device knows the counts, the
  // host only whether there are any.  Without them a call of `target` row blocks is never split and has no merge
  // to launch.  With them it may be, and where the counts are full the merge finds nothing to do (1.3 us: 20 sequences
  // of 61 drafts over 500 positions 53.4 for 52.1; of 15 in the same places 22.2).
  a.split = tiles > 1 && (blocks < a.target || a.counts != nullptr);
#define WQ_TREE(HD, BITS) \
  if (hd == HD && bits == BITS) return launch_tree_tc_t<HD, BITS>(a, grid, blocks >= a.target, many, s);
  WQ_TREE(128, 16) WQ_TREE(128, 8) WQ_TREE(128, 4) WQ_TREE(64, 16) WQ_TREE(64, 8) WQ_TREE(64, 4)
#undef WQ_TREE
  return cudaErrorInvalidValue;
}

cudaError_t read_tree_tc_status(int *status) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(status, g_tree_tc_status, sizeof(int));
  if (e != cudaSuccess) return e;
  const int zero = 0;
  return cudaMemcpyToSymbol(g_tree_tc_status, &zero, sizeof(int));
}

}  // namespace wq
