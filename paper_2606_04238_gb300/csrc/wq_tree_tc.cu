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
// one tile ahead, convert them (code - z, exact) and store them in the 128-byte
// swizzled layout, 12 issues the MMAs.  Two CTAs an SM (256 TMEM columns and ~100 KB
// each) fill each other's waits: a tile's products, softmax and products again are
// one chain.  A draft tile's rows are brought into binary16 by an exact power of two
// a row.  The running maximum is raised, and O rescaled in TMEM, only when a row's
// scores pass it by 2^8: p stays below 2^8.
//
// The tiles of all (b, g, row block) are dealt to the CTAs in nearly equal
// ranges: every CTA finds the tiles a range takes from the lengths themselves.
// Ranges of one row block that is split are merged by a second kernel.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

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
constexpr float kRaise = 8.f;
constexpr int kTmemCols = 256;    // S / P 0..127, O 128..
// registers a thread: the launch's 72 x 416 shared out as 88 x 128 + 64 x 256 + 72 x 32
constexpr int kRegsSoftmax = 88, kRegsConv = 64;

__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack_h2(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
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
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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

// 32 lanes x 32 consecutive 32-bit TMEM columns, written.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(
          taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
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

// One warp (every CTA the same sums): the least number W of tiles a range for which
// the ranges are at most `target` (or the longest sequence's tiles), then this
// CTA's range.  W >= a.min_tiles.
__device__ Work find_work(const TreeArgs &a, int rep, int cta) {
  const int lane = threadIdx.x & 31;
  int len, cnt, tiles, blocks;
  auto ranges = [&](int W) {  // ranges of all sequences with W tiles each
    long long s = 0;
    for (int b = lane; b < a.batch; b += 32) {
      seq_tiles(a, b, rep, len, cnt, tiles, blocks);
      s += (long long)((tiles + W - 1) / W) * blocks;
    }
    for (int o = 16; o >= 1; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s * a.Hkv;
  };
  long long total = 0;
  int most = 1;
  for (int b = lane; b < a.batch; b += 32) {
    seq_tiles(a, b, rep, len, cnt, tiles, blocks);
    total += (long long)tiles * blocks;
    most = max(most, tiles);
  }
  for (int o = 16; o >= 1; o >>= 1) {
    total += __shfl_xor_sync(0xffffffffu, total, o);
    most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
  }
  total *= a.Hkv;
  int lo = max(a.min_tiles, (int)min((long long)most, (total + a.target - 1) / a.target)), hi = max(most, lo);
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (ranges(mid) <= a.target)
      hi = mid;
    else
      lo = mid + 1;
  }
  const int W = lo;
  // the sequence this CTA falls into
  Work w;
  w.any = false;
  long long base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    const int b = b0 + lane;
    tiles = blocks = len = cnt = 0;
    if (b < a.batch) seq_tiles(a, b, rep, len, cnt, tiles, blocks);
    const int n = (tiles + W - 1) / W, mine = n * blocks * a.Hkv;
    int incl = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, cta < base + incl);
    if (cta == 0 && b < a.batch) {
      if (a.table) a.table[b] = make_int2((int)(base + incl - mine), n);
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
      w.t0 = (int)((long long)nt * w.split / w.n);
      w.t1 = (int)((long long)nt * (w.split + 1) / w.n);
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
  Work work;
  // K's scale (times the score scale), log2 of V's scale, its reciprocal; 1024 + z twice.  Two tiles
  // of each: the next tile's are written while this one's are read
  __align__(16) float sk[2][kTile];
  __align__(16) float lg[2][kTile];
  __align__(16) float rs[2][kTile];
  uint32_t zk[kTile], zv[kTile];
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
  pdl_wait();
  pdl_launch_dependents();
  if (warp == 0) {
    const Work w = find_work(a, rep, blockIdx.x);
    if (lane == 0) sh.work = w;
  } else if (warp == kMmaWarp) {
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
    bool ok = wait(&sh.p_full, 0);  // Q is in place
    for (int i = 0; i < nt && ok; ++i) {
      ok = wait(&sh.k_full, i & 1);
      // P V of the tile before has read P, which S overwrites
      if (ok && i > 0) ok = wait(&sh.v_empty, (i - 1) & 1);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks) {
          const uint64_t off = (uint64_t)(((ks / 4) * kBlk + (ks % 4) * 32) >> 4);
          umma_f16(tm, qd + off, kd + off, idqk, ks > 0);
        }
        umma_commit(&sh.s_full);
        umma_commit(&sh.k_empty);
      }
      __syncwarp();
      ok = wait(&sh.p_full, (i + 1) & 1) && wait(&sh.v_full, i & 1);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
#pragma unroll
        for (int ks = 0; ks < kTile / 16; ++ks)
          umma_ts(tm + 128, tm + 8 * ks, vd + (uint64_t)((ks * 2048) >> 4), idpv, i > 0 || ks > 0);
        umma_commit(&sh.v_empty);
      }
      __syncwarp();
    }
    if (!ok && lane == 0) sh.fail = 1;
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
    // the drafts' K or V: in binary16 by a power of two a row, or as it is
    auto draft = [&](const void *rows, uint8_t *to, bool is_v) {
      const __nv_bfloat16 *src = reinterpret_cast<const __nv_bfloat16 *>(rows) + ((size_t)w.b * a.T * a.Hkv + w.g) * HD + c * 8;
#pragma unroll 1
      for (int it = 0; it < C::IT; ++it) {
        const int j = r0 + it * C::RS;
        const uint4 v = j < w.cnt ? __ldg(reinterpret_cast<const uint4 *>(src + (size_t)j * a.Hkv * HD)) : make_uint4(0, 0, 0, 0);
        uint32_t x[4] = {v.x, v.y, v.z, v.w};
        if (is_v) {
          bool odd = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u, odd = true;
            if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu, odd = true;
          }
          if (odd) atomicOr(&sh.odd[j / 32], 1u << (j % 32));
        }
        if constexpr (!BF) {
          float mx = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, fmaxf(fabsf(bf_lo(x[e])), fabsf(bf_hi(x[e]))));
#pragma unroll
          for (int o = C::CH / 2; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          // V as large as codes are, so that p times the row's scale is as large as theirs
          const int e2 = f16_shift(mx, is_v ? BITS - 1 : 14);
          const float f = pow2i(e2);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = pack_h2(bf_lo(x[e]) * f, bf_hi(x[e]) * f);
          if (c == 0) {
            if (is_v) {
              sh.lg[0][j] = (float)-e2;
              sh.rs[0][j] = f;
            } else {
              sh.sk[0][j] = a.scale * pow2i(-e2);
            }
          }
        }
        *reinterpret_cast<uint4 *>(to + dst0 + it * C::RS * 128) = make_uint4(x[0], x[1], x[2], x[3]);
      }
    };
    auto pos_of = [&](int i) { return (w.t0 + i - ndr) * kTile; };
    const int i_ctx = max(0, ndr - w.t0);  // first tile of the context
    bool ok = true;
    if (i_ctx < nt && !BF) {
      fetch_meta(pos_of(i_ctx));
      fetch(kc, kr, pos_of(i_ctx));
      fetch(vc, vr, pos_of(i_ctx));
    }
    if (i_ctx > 0) {
      draft(a.kn, kbuf, false);
      draft(a.vn, vbuf, true);
      hand_over(&sh.k_full);
      hand_over(&sh.v_full);
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
        {
          const float s0 = __half2float(__ushort_as_half((unsigned short)(meta & 0xffffu)));
          const __half2 z = __hadd2(__half2half2(__ushort_as_half((unsigned short)(meta >> 16))), __float2half2_rn(1024.f));
          const uint32_t zz = *reinterpret_cast<const uint32_t *>(&z);
          const int r = ct & (kTile - 1);
          if (ct < kTile) {
            sh.sk[par][r] = s0 * a.scale;
            sh.zk[r] = zz;
          } else {
            const float sv = s0 == 0.f ? 1.f : s0;  // a zero-filled cache's row: code - z is 0
            const bool in = p0 + r < w.len;
            sh.lg[par][r] = in ? __log2f(sv) : -INFINITY;
            sh.rs[par][r] = in ? __frcp_rn(sv) : 0.f;
            sh.zv[r] = zz;
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
        for (int it = 0; it < C::IT; ++it)
          *reinterpret_cast<uint4 *>(vbuf + dst0 + it * C::RS * 128) = convert8<BITS>(vr[it], sh.zv[r0 + it * C::RS]);
        hand_over(&sh.v_full);
        fetch(vc, vr, pn);
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
    // ---- softmax: thread = row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int r = row0 + tid, t = r / rep;
    const bool in = tid < live;
    const bool busy = warp * 32 < live;  // warps without rows only keep the barriers going
    const uint32_t tw = tm + ((uint32_t)(warp * 32) << 16);
    float c1 = a.scale;  // of the raw products: bf16 the score scale (its sign in Q), else 2^-e of the row
    if (busy) {
      const uint4 *q = reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(a.q) +
                                                       (((size_t)w.b * a.T + (in ? t : 0)) * a.H + w.g * rep + (in ? r % rep : 0)) * HD);
      float f = 1.f;
      if constexpr (BF) {
        c1 = fabsf(a.scale);
      } else {
        float mx = 0.f;
#pragma unroll 4
        for (int i = 0; i < HD / 8; ++i) {
          const uint4 v = in ? __ldg(q + i) : make_uint4(0, 0, 0, 0);
          mx = fmaxf(mx, fmaxf(fmaxf(fmaxf(fabsf(bf_lo(v.x)), fabsf(bf_hi(v.x))), fmaxf(fabsf(bf_lo(v.y)), fabsf(bf_hi(v.y)))),
                               fmaxf(fmaxf(fabsf(bf_lo(v.z)), fabsf(bf_hi(v.z))), fmaxf(fabsf(bf_lo(v.w)), fabsf(bf_hi(v.w))))));
        }
        const int e = f16_shift(mx, 14);
        f = pow2i(e);
        c1 = pow2i(-e);
      }
#pragma unroll 4
      for (int i = 0; i < HD / 8; ++i) {
        const uint4 v = in ? __ldg(q + i) : make_uint4(0, 0, 0, 0);
        uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (BF)
            x[e] ^= a.scale < 0.f ? 0x80008000u : 0u;
          else
            x[e] = pack_h2(bf_lo(x[e]) * f, bf_hi(x[e]) * f);
        }
        *reinterpret_cast<uint4 *>(qbuf + (i / 8) * kBlk + tid * 128 + (((i & 7) ^ (tid & 7)) << 4)) =
            make_uint4(x[0], x[1], x[2], x[3]);
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
        const bool some = tile < ndr || w.len - (tile - ndr) * kTile < kTile;
        uint32_t see[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
        if (some)
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const int n = (tile < ndr ? w.cnt : w.len - (tile - ndr) * kTile) - 32 * h;
            uint32_t have = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
            if (tile < ndr) {
              if (!in || n <= 0)
                have = 0;
              else if (a.mask)
                have &= a.mask[((size_t)w.b * a.T + t) * a.words + h];
              else
                have &= t >= 32 * h + 31 ? 0xffffffffu : t < 32 * h ? 0u : (2u << (t - 32 * h)) - 1u;
            }
            see[h] = have;
          }
        // 1. scores (over the raw products where they differ) and their maximum
        float mx = -INFINITY;
        const uint64_t cc = pack_f32x2(c1, c1);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t s[32];
          tmem_ld32(tw + 32 * h, s);
          tmem_ld_wait();
          float *y = reinterpret_cast<float *>(s);
          if constexpr (!BF) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const float4 k4 = *reinterpret_cast<const float4 *>(&sh.sk[par][32 * h + j]);
              const float4 g4 = *reinterpret_cast<const float4 *>(&sh.lg[par][32 * h + j]);
              uint64_t u = fma_f32x2(mul_f32x2(pack_f32x2(y[j], y[j + 1]), cc), pack_f32x2(k4.x, k4.y), pack_f32x2(g4.x, g4.y));
              unpack_f32x2(u, y[j], y[j + 1]);
              u = fma_f32x2(mul_f32x2(pack_f32x2(y[j + 2], y[j + 3]), cc), pack_f32x2(k4.z, k4.w), pack_f32x2(g4.z, g4.w));
              unpack_f32x2(u, y[j + 2], y[j + 3]);
            }
          }
          if (some)
#pragma unroll
            for (int j = 0; j < 32; ++j) y[j] = see[h] >> j & 1 ? y[j] : -INFINITY;
#pragma unroll
          for (int j = 0; j < 32; j += 2) mx = fmaxf(mx, fmaxf(y[j], y[j + 1]));
          if (!BF || some) tmem_st32(tw + 32 * h, s);
        }
        if (BF) mx = mx == -INFINITY ? mx : mx * c1;
        if (__any_sync(0xffffffffu, mx > m + kRaise)) {
          const float mn = fmaxf(m, mx), al = mn == -INFINITY ? 1.f : ex2(m - mn);
          l *= al;
          m = mn;
          if (i > 0)  // P V of the tiles before is complete (S was issued after it)
#pragma unroll 1
            for (int h = 0; h < HD / 32; ++h) {
              uint32_t o[32];
              tmem_ld32(tw + 128 + 32 * h, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * al);
              tmem_st32(tw + 128 + 32 * h, o);
            }
        }
        tmem_st_wait();
        // 2. probabilities
        const float ms = m == -INFINITY ? 0.f : m;
        uint64_t sum = 0;
        const uint64_t mm = pack_f32x2(-ms, -ms), by = BF ? cc : pack_f32x2(1.f, 1.f);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t s[32], p[16];
          tmem_ld32(tw + 32 * h, s);
          tmem_ld_wait();
          const float *y = reinterpret_cast<const float *>(s);
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            float4 r4 = make_float4(1.f, 1.f, 1.f, 1.f);
            if (!BF) r4 = *reinterpret_cast<const float4 *>(&sh.rs[par][32 * h + j]);
            float e[4];
            uint64_t u = fma_f32x2(pack_f32x2(y[j], y[j + 1]), by, mm);
            unpack_f32x2(u, e[0], e[1]);
            u = fma_f32x2(pack_f32x2(y[j + 2], y[j + 3]), by, mm);
            unpack_f32x2(u, e[2], e[3]);
#pragma unroll
            for (int k = 0; k < 4; ++k) e[k] = ex2(e[k]);
            sum = fma_f32x2(pack_f32x2(e[0], e[1]), pack_f32x2(r4.x, r4.y), sum);
            sum = fma_f32x2(pack_f32x2(e[2], e[3]), pack_f32x2(r4.z, r4.w), sum);
            p[j / 2] = BF ? pack_bf2(e[0], e[1]) : pack_h2(e[0], e[1]);
            p[j / 2 + 1] = BF ? pack_bf2(e[2], e[3]) : pack_h2(e[2], e[3]);
          }
          // columns 16 h ..: S's there have been read
          tmem_st16(tw + 16 * h, p);
        }
        float l0, l1;
        unpack_f32x2(sum, l0, l1);
        l += l0 + l1;
        tmem_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full);
    }
    if (ok) ok = wait(&sh.v_empty, (nt - 1) & 1);
    if (!ok && lane == 0) sh.fail = 1;
    tc_fence_after();
    if (busy && ok) {
      // ---- the row's output, or its partial result
      const bool whole = w.n == 1, none = m == -INFINITY && l == 0.f;  // (all scores NaN: l is NaN)
      const float inv = whole ? (none ? 0.f : 1.f / l) : 1.f;
      const bool odd = w.t0 < ndr && (sh.odd[0] | sh.odd[1] | sh.odd[2] | sh.odd[3]) != 0;
      float *pt = a.part + ((size_t)w.slot * a.part_rows + tid) * (HD + 2);
      __nv_bfloat16 *o = reinterpret_cast<__nv_bfloat16 *>(a.o) +
                         (((size_t)w.b * a.T + t) * a.H + w.g * rep + r % rep) * HD;
#pragma unroll 1
      for (int h = 0; h < HD / 32; ++h) {
        uint32_t v[32];
        tmem_ld32(tw + 128 + 32 * h, v);
        tmem_ld_wait();
        if (!in) continue;
        if (odd) {
#pragma unroll 1
          for (int j = 0; j < w.cnt; ++j) {
            if (!(sh.odd[j / 32] >> (j % 32) & 1)) continue;
            const bool see = a.mask ? a.mask[((size_t)w.b * a.T + t) * a.words + j / 32] >> (j % 32) & 1 : j <= t;
            if (!see) continue;
            const __nv_bfloat16 *vj = reinterpret_cast<const __nv_bfloat16 *>(a.vn) +
                                      (((size_t)w.b * a.T + j) * a.Hkv + w.g) * HD + 32 * h;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float f = __bfloat162float(vj[e]);
              if (!isfinite(f)) v[e] = __float_as_uint(__uint_as_float(v[e]) + f);
            }
          }
        }
        if (whole) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint32_t u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              u[k] = none ? 0u : pack_bf2(__uint_as_float(v[e + 2 * k]) * inv, __uint_as_float(v[e + 2 * k + 1]) * inv);
            *reinterpret_cast<uint4 *>(o + 32 * h + e) = make_uint4(u[0], u[1], u[2], u[3]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 32; e += 2)
            *reinterpret_cast<float2 *>(pt + 32 * h + e) = make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1]));
        }
      }
      if (in && !whole) *reinterpret_cast<float2 *>(pt + HD) = make_float2(m, l);
    }
  }
  // rows of drafts that do not exist: 0, by the last row block's first split
  if (w.any && w.split == 0 && w.cnt * rep - row0 <= kTcRows) {
    const int z0 = max(row0, w.cnt * rep);
    for (int i = z0 * (HD / 8) + tid; i < R * (HD / 8); i += kTcThreads) {
      const int row = i / (HD / 8), e = i % (HD / 8);
      *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(a.o) +
                                 (((size_t)w.b * a.T + row / rep) * a.H + w.g * rep + row % rep) * HD + 8 * e) =
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

// o of the rows whose block was split: a warp a row, its parts in split order.
template <int HD>
__global__ void __launch_bounds__(256) attn_tree_merge_kernel(const TreeArgs a) {
  constexpr int E = HD / 32, CU = 4;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, rep = a.H / a.Hkv, R = a.T * rep;
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= (long long)a.batch * a.Hkv * R) return;
  const int bg = (int)(row / R), r = (int)(row - (long long)bg * R), b = bg / a.Hkv, g = bg % a.Hkv;
  const int2 tab = a.table[b];
  int len, cnt, tiles, blocks;
  seq_tiles(a, b, rep, len, cnt, tiles, blocks);
  if (tab.y <= 1 || r >= cnt * rep) return;  // written by the first kernel, or skipped
  const size_t step = (size_t)a.Hkv * blocks * a.part_rows * (HD + 2);
  const float *pt = a.part + ((size_t)(tab.x + g * blocks + r / kTcRows) * a.part_rows + r % kTcRows) * (HD + 2);
  float M = -INFINITY, L = 0.f, O[E];
#pragma unroll
  for (int e = 0; e < E; ++e) O[e] = 0.f;
  for (int s0 = 0; s0 < tab.y; s0 += CU) {
    float2 ml[CU], ov[CU][E / 2];
    float mn = M;
#pragma unroll
    for (int c = 0; c < CU; ++c) {
      const float *ps = pt + (size_t)(s0 + c) * step;
      const bool in = s0 + c < tab.y;
      ml[c] = in ? *reinterpret_cast<const float2 *>(ps + HD) : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int e = 0; e < E / 2; ++e)
        ov[c][e] = in ? *reinterpret_cast<const float2 *>(ps + lane * E + 2 * e) : make_float2(0.f, 0.f);
    }
#pragma unroll
    for (int c = 0; c < CU; ++c) mn = fmaxf(mn, ml[c].x);
    const float f0 = M == -INFINITY ? 0.f : ex2(M - mn);
    M = mn;
    L *= f0;
#pragma unroll
    for (int e = 0; e < E; ++e) O[e] *= f0;
#pragma unroll
    for (int c = 0; c < CU; ++c) {
      if (s0 + c >= tab.y) break;
      const float f = ml[c].x == -INFINITY ? 0.f : ex2(ml[c].x - M);  // (a NaN of a part stays NaN)
      L = fmaf(ml[c].y, f, L);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        O[2 * e] = fmaf(ov[c][e].x, f, O[2 * e]);
        O[2 * e + 1] = fmaf(ov[c][e].y, f, O[2 * e + 1]);
      }
    }
  }
  const bool none = M == -INFINITY && L == 0.f;
  __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(a.o) +
                       (((size_t)b * a.T + r / rep) * a.H + g * rep + r % rep) * HD + lane * E;
#pragma unroll
  for (int e = 0; e < E / 2; ++e)
    reinterpret_cast<uint32_t *>(dst)[e] = none ? 0u : pack_bf2(O[2 * e] / L, O[2 * e + 1] / L);
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
cudaError_t launch_tree_tc_t(const TreeArgs &a, unsigned grid, bool merge, cudaStream_t s) {
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
  if (e != cudaSuccess || !merge) return e;
  const long long rows = (long long)a.batch * a.H * a.T;
  cfg.gridDim = dim3((unsigned)((rows + 7) / 8));
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, attn_tree_merge_kernel<HD>, a);
}

}  // namespace

// CTAs that the device holds at once.
int tree_tc_target(int num_sms) { return 2 * num_sms; }

size_t tree_tc_part_floats(int batch, int T, int H, int Hkv, int hd, int max_len, int num_sms) {
  // a range of its own for every split, of which there are at most `target`, and at most one a tile
  const long long rows = std::min((long long)T * (H / Hkv), (long long)kTcRows);
  const long long tiles = ((long long)max_len + kTile - 1) / kTile + (T + kTile - 1) / kTile;
  const long long blocks = ((long long)T * (H / Hkv) + kTcRows - 1) / kTcRows;
  return (size_t)(std::min((long long)tree_tc_target(num_sms), (long long)batch * Hkv * blocks * tiles) * rows * (hd + 2));
}

cudaError_t launch_attn_tree_tc(TreeArgs a, int hd, int bits, int num_sms, cudaStream_t s) {
  const int rep = a.H / a.Hkv;
  if (a.scale == 0.f) return cudaErrorInvalidValue;
  const long long blocks = (long long)a.batch * a.Hkv * (((long long)a.T * rep + kTcRows - 1) / kTcRows);
  a.target = tree_tc_target(num_sms);
  a.min_tiles = 1;
  a.part_rows = std::min(a.T * rep, kTcRows);
  const long long tiles = ((long long)a.max_len + kTile - 1) / kTile + (a.T + kTile - 1) / kTile;
  const unsigned grid = (unsigned)std::max(blocks, std::min((long long)a.target, blocks * tiles));
  const bool merge = blocks < a.target && tiles > a.min_tiles;  // else every row block is one range
#define WQ_TREE(HD, BITS) \
  if (hd == HD && bits == BITS) return launch_tree_tc_t<HD, BITS>(a, grid, merge, s);
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
