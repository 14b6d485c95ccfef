// wq_attn_paged_tc.cu -- causal attention of a ragged batch over a paged KV cache on the
// tcgen05 tensor cores (sm_103a): the mathematics of wq_attn_paged.cu for sequences of more
// query rows (tokens x query heads of a kv head), chunks of prompts above all.
//
// A CTA (one an SM) takes a block of 256 rows of a sequence and kv head, as two streams of
// 128, and tiles of 128 positions:
//   S = Q K^T   128 x 128 a stream in TMEM, Q and K in shared memory (K-major);
//   P           binary16 (bf16 pool: bf16) over S's own columns, from the fp32 softmax of two
//               threads a row, half the tile's positions each (a half's p over its own scores);
//   O += P V    128 x HD a stream in TMEM, P as the A operand from TMEM, V [position][HD]
//               in shared memory as it lies in a page (MN-major).
// The MMA warp issues P V of one stream and its next S while the other's softmax runs (heads
// of 64: S of the step after that, a third buffer being free).  Up to
// 128 rows (a block's rest, short chunks) both streams have the same rows and take the tiles
// in turn; their results are added up at the end.  28 warps: 0-15 softmax; 16-23 the block's
// queries, then K and V, 16 positions of a tile each (codes through registers to binary16 in the
// 128-byte swizzled layout; a bf16 pool by cp.async); 24 the MMAs; 25 the runs of tiles, four
// ahead; 26-27 only hold the registers that the softmax warps take over.
//
// K's operands are code - z, exact, its scales factors of the scores; V's are (code - z) s 2^-t
// rounded to binary16, t one for 16 positions, or, where their scales span more than 2^8, one for
// each, taken into the score.  The maximum is not searched in every tile: a row's first is that
// of the first 16 scores that it sees; from there on p is taken with the maximum that the row has,
// which is raised, and what was computed with it rescaled in TMEM by a power of two, only where
// 16 p add up to 2^15 (p is 2^6 at most where it is raised).
//
// The tiles of all blocks are laid end to end and every CTA takes an equal run, found from the
// lengths themselves; blocks are paired, the first with the last and so on inward, so that
// a causal prompt's pairs are about equally long.  What a CTA has of a block that others
// share is left in the workspace, and the last of them to arrive adds up all parts in their order.
//
// Bound by the softmax warps' chains (scores from TMEM, 2^x, conversion, P to TMEM: four
// times 16 columns a tile), which the other stream's and the products' round trip overlap in
// part: 2000 tokens over 14,000 positions of 4 bits, 40 heads of 128, take 529 us, 0.53 of the
// measured dense rate for the products alone; a prompt of 4000 over a bf16 pool, 64 heads of
// 64, takes 213, 0.32 (half as many products a 2^x).  Tried and slower: tiles of 64 positions
// with S twice (718 us for 572), a row's 64 scores before any is stored (227 for 219), 32
// columns at a time.  Short runs are bound by their ends: what 14 decode steps and two chunks
// of 250 tokens take (96 us) is in the larger part Q's and the first tile's way in, and parts
// of 132 KB written and added up.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "wq_cvt.cuh"
#include "wq_internal.h"
#include "wq_kv.h"
#include "wq_paged.h"
#include "wq_ptx.cuh"
#include "wq_ragged.cuh"
#include "wq_rows.cuh"
#include "wq_tc.cuh"

namespace wq {

// Status word: WQ_OK (0), WQ_ERR_ARG (-1) after a row offset, length or page outside its range
// (that sequence is skipped; such a page is read as page 0), WQ_ERR_TIMEOUT (-6) after
// a wait ran out.
__device__ int g_attn_paged_tc_status = 0;

namespace {

constexpr int kStream = 128;               // rows of a stream
constexpr int kBlockRows = 2 * kStream;
constexpr int kTile = 128;                 // positions a tile
constexpr int kSoft = 512;                 // softmax threads
constexpr int kConv = 256;                 // converting threads
constexpr int kConvWarp = kSoft / 32, kMmaWarp = kConvWarp + kConv / 32;
constexpr int kThreads = kSoft + kConv + 128;  // the MMA warp, one that plans, and two that registers are allotted with
// registers a thread: the launch's 72 x 896 shared out as 80 x 512 + 64 x 256 + 56 x 128
constexpr int kRegsSoftmax = 80, kRegsConv = 64, kRegsMma = 56;
constexpr int kBlk = kTile * 128;          // bytes of a 64-value block of Q, K or V: [row][128 bytes], swizzled
constexpr int kTmemCols = 512;             // S / P: a buffer each 128; O behind them, a stream each HD
// Queries enter binary16 times 2^7, which keeps a row with its largest |q| in [2^-4, 2^8) whole
// but for values below 2^-27 of that; other rows by a power of two of their own.
constexpr int kQueryShift = 7;
constexpr int kSpread = 8;                 // exponents that V's scales of 16 positions may span with one power of two for all
constexpr int kOwn = 1 << 16;
constexpr int kRing = 8;
constexpr float kMostSum = 32768.f;        // of 16 p; binary16 ends at 65504

template <int HD, int BITS>
struct Cfg {
  static constexpr int NB = HD / 64;             // 64-value blocks
  static constexpr int KB = NB * kBlk;           // bytes of one operand tile
  static constexpr int CH = HD / 8;              // 16-byte chunks a row of 16-bit values
  static constexpr int ROW = HD * BITS / 8;
  // stages of K and V tiles: heads of 64 leave room for four (the next tiles' conversion then waits for no product)
  static constexpr unsigned STAGES = HD == 64 ? 4 : 2;
  static constexpr int SMEM = 1024 + (2 + 2 * (int)STAGES) * KB;  // Q of both streams, K and V
  // codes: 16-byte pieces a row, pieces of a row in one load of a warp, rows of it, loads a row, loads of a warp's 16 rows
  static constexpr int PPR = ROW / 16, PP = PPR < 4 ? PPR : 4, RPI = 32 / PP, SPR = PPR / PP, NI = 16 * PPR / 32;
  static_assert(RPI > 0 && SPR > 0 && NI > 0, "");
  // Steps (a tile of a stream each) take the S buffers in turn.  Heads of 64 leave room for three: the MMA warp is then
  // three steps ahead, and S of a stream's next tile is there when its softmax comes to it.
  static constexpr int BUFS = HD == 64 ? 3 : 2, O_AT = BUFS * kTile;
  static_assert(O_AT + 2 * HD <= kTmemCols, "");
  static constexpr float LIFT = BITS == 16 ? 0.f : 6.f;  // of p: small ones are then normal numbers
};


// A run of tiles of one block of rows.
struct Run {
  int b, g, q0, len, before, r0, live, t0, n;  // live: rows of the block; tiles t0 .. t0 + n - 1
  int least;                                   // positions that its first row sees
  int c0, cl;                                  // the first and last CTA that have tiles of the block
  bool any, split, whole;
};

struct Shared {
  uint64_t q_full, q_empty, k_full[4], k_empty[4], v_full[4], v_empty[4], s_full[3], p_full[3];
  uint64_t o_full[2][2];  // by stream and parity of its tile (two of a stream's products may be under way)
  uint64_t run_full[4], run_empty[4];
  Run run[4];
  uint32_t tmem;
  int fail, last;
  // of a tile, eight tiles deep (a tile's are written when S of the one STAGES tiles before is done, whose softmax has then
  // ended for the tile two before that): K's scales times the score scale and 2^-kQueryShift, V's exponents t
  __align__(16) float sk[kRing][kTile];
  __align__(16) int te[kRing][8];  // by 16 positions; kOwn: their rows have their own
  __align__(16) float td[kRing][kTile], tw[kRing][kTile];
  float qf[4][kBlockRows];         // what a row's own power of two differs from 2^kQueryShift
  // of a block, by converting warp: positions from its first masked tile on (384 at most) whose V is not finite, and whether
  // there are any
  uint32_t odd[4][8][16];
  float pm[2][2][kStream], pl[2][2][kStream];  // the halves' maxima and sums
  int limit[2][kStream];                       // positions that a stream's rows see
};

// The line of tiles: sequences in order, in a sequence pairs of blocks, the kv head fastest.  A pair has C places, as many
// as any has tiles; those behind its two blocks are empty.
struct Walk {
  long long x, x1, base, T, N, total;
  int b, R, nb, before, C;
  Seq s;

  __device__ __forceinline__ int tiles(const Divisor &by_rep, int k, bool full) const {
    if (s.len == 0) return 1;
    const int r = k * kBlockRows + kBlockRows - 1;
    return (before + (int)by_rep.divide(full ? r : min(r, R - 1)) + 1 + kTile - 1) / kTile;
  }
  __device__ __forceinline__ void load(const AttnPagedArgs &a, const Divisor &by_rep, int to, bool &bad) {
    b = to;
    s = get_seq(a, b, bad);
    R = s.nq * (int)by_rep.d;
    nb = (R + kBlockRows - 1) / kBlockRows;
    before = s.len - s.nq;
    // (tiles(k) + tiles(nb - 1 - k) is at most this: quotients and their rounding up differ by one at most)
    C = nb == 0 ? 0 : nb == 1 ? tiles(by_rep, 0, false) : tiles(by_rep, 0, false) + tiles(by_rep, nb - 1, true) + 1;
    total = (long long)a.Hkv * ((nb + 1) / 2) * C;
  }
  // One warp, all lanes alike: this CTA's part of the line.
  __device__ __forceinline__ void start(const AttnPagedArgs &a, const Divisor &by_rep, bool &bad) {
    const int lane = threadIdx.x & 31;
    T = 0;
    for (int i = lane; i < a.batch; i += 32) {
      load(a, by_rep, i, bad);
      T += total;
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) T += __shfl_xor_sync(0xffffffffu, T, o);
    N = min((long long)gridDim.x, T);
    const long long c = blockIdx.x;
    x = x1 = base = 0;
    if (c >= N) return;
    x = T * c / N;
    x1 = T * (c + 1) / N;
    for (int b0 = 0;; b0 += 32) {
      long long mine = 0;
      if (b0 + lane < a.batch) {
        load(a, by_rep, b0 + lane, bad);
        mine = total;
      }
      long long incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, x < base + incl);
      if (hit) {
        const int src = __ffs(hit) - 1;
        base += __shfl_sync(0xffffffffu, incl - mine, src);
        load(a, by_rep, b0 + src, bad);
        return;
      }
      base += __shfl_sync(0xffffffffu, incl, 31);
    }
  }
  // One thread: the next run; false at the end.
  __device__ __forceinline__ bool next(const AttnPagedArgs &a, const Divisor &by_rep, Run &o) {
    bool bad = false;
    while (x < x1) {
      while (x >= base + total) {
        base += total;
        load(a, by_rep, b + 1, bad);
      }
      const long long local = x - base, item = local / C;
      const int y = (int)(local - item * C), p = (int)(item / a.Hkv), p2 = nb - 1 - p;
      const int t1 = tiles(by_rep, p, false), t2 = p2 != p ? tiles(by_rep, p2, false) : 0;
      if (y >= t1 + t2) {  // an empty place
        x += C - y;
        continue;
      }
      const int k = y < t1 ? p : p2, off = y < t1 ? y : y - t1, all = y < t1 ? t1 : t2;
      const int n = (int)min((long long)(all - off), x1 - x);
      o.b = b, o.g = (int)(item % a.Hkv), o.q0 = s.q0, o.len = s.len, o.before = before;
      o.r0 = k * kBlockRows, o.live = min(kBlockRows, R - o.r0);
      o.t0 = off, o.n = s.len == 0 ? 0 : n;
      o.split = o.live <= kStream;
      o.whole = n == all;
      o.least = before + (int)by_rep.divide(o.r0) + 1;
      o.c0 = (int)(((x - off + 1) * N - 1) / T);
      o.cl = (int)(((x - off + all) * N - 1) / T);
      x += n;
      return o.any = true;
    }
    return o.any = false;
  }
};

// A half row's p of 16 c columns, and 16 c columns of O, times al.
template <bool BF>
__device__ __noinline__ void rescale_p(uint32_t at, int c, float al) {
  tmem_st_wait();
#pragma unroll 1
  for (int i = 0; i < (c + 1) / 2; ++i) {  // (a place behind the last may hold scores that are not read yet: put back as they are)
    uint32_t p[16];
    tmem_ld16(at + 16 * i, p);
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e < 8 || 2 * i + 1 < c) p[e] = BF ? pack_bf2(bf_lo(p[e]) * al, bf_hi(p[e]) * al) : hmul2_u(p[e], pack_h2(al, al));
    tmem_st16(at + 16 * i, p);
  }
  tmem_st_wait();
}
template <int N>
__device__ __noinline__ void rescale_o(uint32_t at, float al) {
#pragma unroll 1
  for (int c = 0; c < N; ++c) {
    uint32_t o[16];
    tmem_ld16(at + 16 * c, o);
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * al);
    tmem_st16(at + 16 * c, o);
  }
}

// Lane `at` of four has v[i], 16 bytes i of its row: after, 16 bytes `at` of the rows of lane i.
__device__ __forceinline__ void transpose4(uint4 (&v)[4], int at) {
  auto swap = [](uint4 &a, uint4 &b, bool up, int by) {  // a of the upper lane for b of the lower one
    const uint4 give = up ? a : b;
    uint4 got;
    got.x = __shfl_xor_sync(0xffffffffu, give.x, by), got.y = __shfl_xor_sync(0xffffffffu, give.y, by);
    got.z = __shfl_xor_sync(0xffffffffu, give.z, by), got.w = __shfl_xor_sync(0xffffffffu, give.w, by);
    if (up)
      a = got;
    else
      b = got;
  };
  swap(v[0], v[1], at & 1, 1);
  swap(v[2], v[3], at & 1, 1);
  swap(v[0], v[2], at & 2, 2);
  swap(v[1], v[3], at & 2, 2);
}

__device__ __forceinline__ float half_lo(uint32_t m) { return __half2float(__ushort_as_half((unsigned short)(m & 0xffffu))); }

}  // namespace

template <int HD, int BITS>
__global__ void __launch_bounds__(kThreads, 1) attn_paged_tc_kernel(const AttnPagedArgs a, const Divisor by_rep) {
  using C = Cfg<HD, BITS>;
  constexpr bool BF = BITS == 16;
  extern __shared__ uint8_t paged_dyn[];
  __shared__ Shared sh;
  uint8_t *qbuf = paged_dyn + (1024 - (smem_addr(paged_dyn) & 1023)) % 1024, *kbuf = qbuf + 2 * C::KB, *vbuf = kbuf + C::STAGES * C::KB;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int page = 1 << a.shift;
  if (warp == kMmaWarp) {
    tmem_alloc(&sh.tmem, kTmemCols);
    if (lane == 0) {
      mbar_init(&sh.q_full, kConv / 32);
      mbar_init(&sh.q_empty, 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(&sh.o_full[i][0], 1);
        mbar_init(&sh.o_full[i][1], 1);
      }
      for (int i = 0; i < 3; ++i) {
        mbar_init(&sh.s_full[i], 1);
        mbar_init(&sh.p_full[i], 8);
      }
      for (int i = 0; i < 4; ++i) {
        mbar_init(&sh.k_full[i], kConv / 32);
        mbar_init(&sh.v_full[i], kConv / 32);
        mbar_init(&sh.k_empty[i], 1);
        mbar_init(&sh.v_empty[i], 1);
        mbar_init(&sh.run_full[i], 1);
        mbar_init(&sh.run_empty[i], kMmaWarp + 1);
      }
      fence_barrier_init();
      sh.fail = 0;
    }
  }
  pdl_wait();
  pdl_launch_dependents();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = sh.tmem;
  const int rep = (int)by_rep.d;
  // all lanes alike: a warp leaves its loop as one after a timeout
  auto wait = [&](uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)) != 0; };
  // a warp is done with a run
  auto done = [&](int turn) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.run_empty[turn & 3]);
  };
  // a warp's arrival, its shared-memory writes made visible to the tensor cores
  auto hand_over = [&](uint64_t *bar) {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
  };

  if (warp >= kMmaWarp) {
    // ---- MMAs.  T: tiles so far, cs: tiles of a stream so far
    constexpr uint32_t idqk = attn_idesc(kTile, BF, false), idpv = attn_idesc(HD, BF, true);
    const uint64_t qd = umma_desc_kmajor_sw128(smem_addr(qbuf), 1024), kd = umma_desc_kmajor_sw128(smem_addr(kbuf), 1024);
    const uint64_t vd = umma_desc_mnmajor_sw128(smem_addr(vbuf), kBlk);
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsMma));
    if (warp == kMmaWarp + 1) {
      // the runs, for all warps
      bool bad = false, ok = true;
      Walk walk;
      walk.start(a, by_rep, bad);
      if (bad && blockIdx.x == 0) atomicExch(&g_attn_paged_tc_status, -1);
      if (lane == 0)
        for (int turn = 0; ok; ++turn) {
          if (turn >= 4) ok = mbar_wait(&sh.run_empty[turn & 3], (turn >> 2) + 1 & 1);
          if (!ok) break;
          const bool any = walk.next(a, by_rep, sh.run[turn & 3]);
          mbar_arrive(&sh.run_full[turn & 3]);
          if (!any) break;
        }
      if (!ok) sh.fail = 1;
    } else if (warp == kMmaWarp) {
      const uint32_t lead = elect_one();
      const uint32_t tm0 = __shfl_sync(0xffffffffu, tm, 0);
      bool ok = true;
      int seg = 0;
      unsigned T = 0, K = 0, odd = 0;  // K: steps of the runs before; bit s of odd: the parity of stream s's tiles
      for (int turn = 0; ok; ++turn) {
        const Run &w = sh.run[turn & 3];
        ok = wait(&sh.run_full[turn & 3], turn >> 2 & 1);
        if (!ok || !w.any) break;
        const int n = __shfl_sync(0xffffffffu, w.n, 0), split = __shfl_sync(0xffffffffu, (int)w.split, 0);
        const int steps = split ? n : 2 * n, ahead = split ? 2 : C::BUFS;
        // step k is tile k of split blocks, tile k / 2 of others, stream k % 2
        auto k_there = [&](int k) {
          const unsigned x = T + (split ? k : k >> 1);
          return wait(&sh.k_full[x % C::STAGES], x / C::STAGES & 1);
        };
        auto scores = [&](int k) {
          const unsigned x = T + (split ? k : k >> 1), s = k & 1, buf = (K + k) % C::BUFS;
          const uint64_t q = qd + (uint64_t)(((split ? 0 : s) * C::KB) >> 4), kt = kd + (uint64_t)((x % C::STAGES * C::KB) >> 4);
#pragma unroll
          for (int ks = 0; ks < HD / 16; ++ks) {
            const uint64_t off = (uint64_t)(((ks / 4) * kBlk + (ks % 4) * 32) >> 4);
            umma_ss_lead(lead, tm0 + buf * 128, q + off, kt + off, idqk, ks > 0);
          }
          umma_commit_lead(lead, &sh.s_full[buf]);
          if (split || s == 1) umma_commit_lead(lead, &sh.k_empty[x % C::STAGES]);
          if (k == steps - 1) umma_commit_lead(lead, &sh.q_empty);
        };
        if (n > 0) ok = wait(&sh.q_full, seg & 1);
        for (int k = 0; k < min(ahead, steps) && ok; ++k) {
          ok = k_there(k);
          tc_fence_after();
          if (ok) scores(k);
        }
        for (int k = 0; k < steps && ok; ++k) {
          const unsigned x = T + (split ? k : k >> 1), s = k & 1, st = x % C::STAGES, buf = (K + k) % C::BUFS;
          // (of split blocks the converting warps may wait for this tile's products before they hand K over)
          if (!split && k + ahead < steps) ok = k_there(k + ahead);
          ok = ok && wait(&sh.v_full[st], x / C::STAGES & 1) && wait(&sh.p_full[buf], (K + k) / C::BUFS & 1);
          if (!ok) break;
          tc_fence_after();
          const uint64_t v = vd + (uint64_t)((st * C::KB) >> 4);
#pragma unroll
          for (int ks = 0; ks < kTile / 16; ++ks)
            umma_ts_lead(lead, tm0 + C::O_AT + s * HD, tm0 + buf * 128 + 8 * ks + (ks < 4 ? 0 : 32), v + (uint64_t)((ks * 2048) >> 4), idpv, k > 1 || ks > 0);
          if (C::BUFS > 2 || k + ahead >= steps) umma_commit_lead(lead, &sh.o_full[s][C::BUFS > 2 ? odd >> s & 1 : 0]);
          odd ^= 1u << s;
          if (split || s == 1) umma_commit_lead(lead, &sh.v_empty[st]);
          if (k + ahead < steps) {
            if (split) {
              ok = k_there(k + ahead);
              tc_fence_after();
            }
            if (ok) scores(k + ahead);
          }
        }
        K += steps;
        T += n;
        seg += n > 0;
        done(turn);
      }
      if (!ok && lane == 0) sh.fail = 1;
    }
    __syncwarp();
  } else if (warp >= kConvWarp) {
    // ---- queries, K and V: warp cw has rows 16 cw .. of every tile, which lie in one page
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsConv));
    const int ct = tid - 32 * kConvWarp, cw = ct >> 5;
    const uint8_t *const kc = reinterpret_cast<const uint8_t *>(a.kc), *const vc = reinterpret_cast<const uint8_t *>(a.vc);
    bool ok = true;
    int seg = 0;
    unsigned T = 0;
    for (int turn = 0; ok; ++turn) {
      const Run &w = sh.run[turn & 3];
      ok = wait(&sh.run_full[turn & 3], turn >> 2 & 1);
      if (!ok || !w.any) break;
      if (w.n == 0) {
        done(turn);
        continue;
      }
      const int n = w.n, len = w.len, p1 = w.t0 * kTile + 16 * cw;  // the warp's first position of the first tile
      const int first_odd = w.least / kTile * kTile;  // positions from w.least on are not seen by all rows
      const int *const table = a.tables + (size_t)w.b * a.max_pages;
      // the page of the warp's rows of tile ti, and the pool's row of the first (a pool has fewer than 2^32: host check);
      // rows behind the length are some row of the pool
      auto load_id = [&](int ti) { return table[min(p1 + ti * kTile, len - 1) >> a.shift]; };
      auto base_of = [&](int id, int ti) {
        if ((unsigned)id >= (unsigned)a.n_pages) {
          id = 0;
          if (lane == 0) atomicExch(&g_attn_paged_tc_status, -1);
        }
        return (((uint32_t)id * a.Hkv + w.g) << a.shift) + ((p1 + ti * kTile) & (page - 1));
      };
      int id0 = load_id(0), id1 = load_id(1);
      if (lane < 16) sh.odd[seg & 3][cw][lane] = 0;

      // the block's queries
      if (seg > 0) ok = wait(&sh.q_empty, (seg - 1) & 1);
      if (!ok) break;
      {
        const int c = ct % C::CH;
        const __nv_bfloat16 *q0 = reinterpret_cast<const __nv_bfloat16 *>(a.q) + ((size_t)w.q0 * a.H + w.g * rep) * HD + c * 8;
        constexpr int STEP = kConv / C::CH, QU = 4;  // rows a pass, passes on their way
        const int rows = (w.live + 31) / 32 * 32;
#pragma unroll 1
        for (int r0 = ct / C::CH; r0 < rows; r0 += QU * STEP) {
          uint4 x[QU];
#pragma unroll
          for (int u = 0; u < QU; ++u) {
            const int row = w.r0 + min(r0 + u * STEP, w.live - 1), tok = (int)by_rep.divide(row);
            x[u] = __ldg(reinterpret_cast<const uint4 *>(q0 + ((size_t)tok * a.H + row - tok * rep) * HD));
          }
#pragma unroll
          for (int u = 0; u < QU; ++u) {
            const int r = r0 + u * STEP;
            if (r >= rows) break;  // (a warp's lanes alike: rows is a multiple of 32)
            const uint4 v = x[u];
            uint4 *dst = reinterpret_cast<uint4 *>(qbuf + (r / kStream) * C::KB + (c / 8) * kBlk + r % kStream * 128 + (((c & 7) ^ (r & 7)) << 4));
            if constexpr (BF) {
              *dst = v;
            } else {
              uint32_t big = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
              big = max(big & 0xffffu, big >> 16);  // the row's largest |q|, as bf16 bits
#pragma unroll
              for (int o = C::CH / 2; o >= 1; o >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
              const int e = (int)(big >> 7) - 127;
              int mine = kQueryShift;
              if (big != 0 && (e < -4 || e >= 8)) mine = max(min(min(126, 14 - e), kQueryShift + 126), -114);
              const float f = pow2i(mine);
              if (c == 0) sh.qf[seg & 3][r] = pow2i(kQueryShift - mine);
              *dst = make_uint4(pack_h2(bf_lo(v.x) * f, bf_hi(v.x) * f), pack_h2(bf_lo(v.y) * f, bf_hi(v.y) * f),
                                pack_h2(bf_lo(v.z) * f, bf_hi(v.z) * f), pack_h2(bf_lo(v.w) * f, bf_hi(v.w) * f));
            }
          }
        }
      }
      hand_over(&sh.q_full);

      if constexpr (BF) {
        // a lane's 16-byte chunks lane, lane + 32, .. of the 16 rows
        constexpr int NC = 16 * C::CH / 32;
        auto place = [&](uint8_t *tile, int i) {
          const int r = (lane + 32 * i) / C::CH, c = lane % C::CH;
          return tile + (c / 8) * kBlk + (16 * cw + r) * 128 + (((c & 7) ^ (r & 7)) << 4);
        };
        auto copy = [&](const uint8_t *src, uint8_t *tile, uint32_t base, int ti) {
          const uint8_t *p = src + (size_t)base * C::ROW + lane * 16;
          const int left = len - p1 - ti * kTile;  // rows before the length
#pragma unroll
          for (int i = 0; i < NC; ++i) cp_async16_zfill(place(tile, i), p + 512 * i, (lane + 32 * i) / C::CH < left ? 16u : 0u);
          cp_async_commit();
        };
        auto clean = [&](uint8_t *tile, int ti) {
          // V's values that are not finite are taken out and noted: rows that do not see them must not meet them
          if ((w.t0 + ti + 1) * kTile <= w.least) return;
#pragma unroll 1
          for (int i = 0; i < NC; ++i) {
            uint4 *p = reinterpret_cast<uint4 *>(place(tile, i));
            const uint4 v = *p;
            uint32_t x[4] = {v.x, v.y, v.z, v.w};
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u, odd = true;
              if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu, odd = true;
            }
            if (odd) {
              *p = make_uint4(x[0], x[1], x[2], x[3]);
              const int at = p1 + ti * kTile + (lane + 32 * i) / C::CH - first_odd;
              atomicOr(&sh.odd[seg & 3][cw][at / 32], 1u << (at % 32));
              sh.odd[seg & 3][cw][15] = 1;
            }
          }
        };
        for (int ti = 0; ti < n; ++ti) {
          const unsigned st = (T + ti) % C::STAGES, last = (T + ti - 1) % C::STAGES;
          const uint32_t base = base_of(id0, ti);
          id0 = id1;
          id1 = load_id(ti + 2);
          if (T + ti >= C::STAGES) ok = wait(&sh.k_empty[st], (T + ti) / C::STAGES + 1 & 1);
          if (!ok) break;
          copy(kc, kbuf + st * C::KB, base, ti);
          if (ti > 0) {  // K of the tile before has landed, all but the last two groups have
            cp_async_wait_group<2>();
            hand_over(&sh.k_full[last]);
          }
          if (T + ti >= C::STAGES) ok = wait(&sh.v_empty[st], (T + ti) / C::STAGES + 1 & 1);
          if (!ok) break;
          copy(vc, vbuf + st * C::KB, base, ti);
          if (ti > 0) {
            cp_async_wait_group<2>();
            clean(vbuf + last * C::KB, ti - 1);
            hand_over(&sh.v_full[last]);
          }
        }
        const unsigned st = (T + n - 1) % C::STAGES;
        if (ok) {
          cp_async_wait_group<1>();
          hand_over(&sh.k_full[st]);
        }
        cp_async_wait_all();
        if (ok) {
          clean(vbuf + st * C::KB, n - 1);
          hand_over(&sh.v_full[st]);
        }
      } else {
        const float qscale = a.scale * pow2i(-kQueryShift);  // of K's scales
        const int lr = lane % 8 + 8 * (lane / 8 / C::PP), lp = lane / 8 % C::PP;  // a lane's row and piece of a load
        // where chunk i of the lane's first piece goes (rows 8 further lie 1024 bytes further, and are swizzled alike)
        constexpr int CPP = BITS == 4 ? 4 : 2;  // 8-value chunks a piece
        uint32_t to[CPP];
#pragma unroll
        for (int i = 0; i < CPP; ++i) {
          const int c = CPP * lp + i;
          to[i] = (c / 8) * kBlk + (16 * cw + lr) * 128 + (((c & 7) ^ (lr & 7)) << 4);
        }
        uint4 rk[C::NI], rv[C::NI];
        auto fetch = [&](const uint8_t *src, uint4 (&r)[C::NI], uint32_t base) {
          const uint8_t *p = src + (size_t)base * C::ROW + lr * C::ROW + lp * 16;
#pragma unroll
          for (int k = 0; k < C::NI; ++k)
            r[k] = __ldg(reinterpret_cast<const uint4 *>(p + (k / C::SPR) * C::RPI * C::ROW + (k % C::SPR) * C::PP * 16));
        };
        // lanes 0-15: K's, 16-31: V's scale and zero point of the warp's rows
        auto fetch_meta = [&](uint32_t base) { return __ldg((lane < 16 ? a.km : a.vm) + base + (lane & 15)); };
        uint32_t m0, b1 = base_of(id0, 0);
        m0 = fetch_meta(b1);
        fetch(kc, rk, b1);
        fetch(vc, rv, b1);
        for (int ti = 0; ti < n; ++ti) {
          const unsigned st = (T + ti) % C::STAGES, ring = (T + ti) % kRing, p0 = p1 + ti * kTile;
          b1 = base_of(id1, ti + 1);
          const uint32_t m1 = fetch_meta(b1);
          id1 = load_id(ti + 2);
          // V's exponent: the largest scale at 2^5 .., or each row's own where they span too much (a NaN counts as the least)
          uint32_t v = (m0 & 0xffffu) > 0x7c00u ? 0u : m0 & 0xffffu;
          if (v == 0 || m0 == kZeroRow) v = 1;  // kLeastScale
          const bool in = p0 + (lane & 15) < len;
          const uint32_t hi = __reduce_max_sync(0xffffffffu, lane >= 16 && in ? v : 1u);
          const uint32_t lo = __reduce_min_sync(0xffffffffu, lane >= 16 && in ? v : 0x7c00u);
          auto exponent = [](float s) { return (int)(__float_as_uint(s) >> 23) - 127 - 5; };
          const int te = exponent(half_lo(hi));
          const bool spread = te - exponent(half_lo(lo)) > kSpread;
          // of the lane's row: 1024 + z; V: its scale times 2^-t too
          const int pl = lane & 15;
          const float s0 = half_lo(m0);
          const __half2 z = __hadd2(__half2half2(__ushort_as_half((unsigned short)(in ? m0 >> 16 : 0u))), __float2half2_rn(1024.f));
          uint32_t zs = *reinterpret_cast<const uint32_t *>(&z);
          if (T + ti >= C::STAGES) ok = wait(&sh.k_empty[st], (T + ti) / C::STAGES + 1 & 1);
          if (!ok) break;
          if (lane < 16) {
            sh.sk[ring][16 * cw + pl] = s0 * qscale;
          } else {
            float v = s0 == 0.f || m0 == kZeroRow ? kLeastScale : s0;
            const int t = spread ? min(exponent(v), te) : te;  // (a NaN's: te)
            if (spread) sh.td[ring][16 * cw + pl] = (float)t, sh.tw[ring][16 * cw + pl] = pow2i(-t);
            v *= pow2i(-t);
            if (in && v != v && p0 - 16 * cw + kTile > w.least) {  // a NaN row that not all rows see
              const int x = p0 + pl - first_odd;
              atomicOr(&sh.odd[seg & 3][cw][x / 32], 1u << (x % 32));
              sh.odd[seg & 3][cw][15] = 1;
              v = 0.f;
            }
            zs = __byte_perm(zs, in ? (uint32_t)__half_as_ushort(__float2half_rn(v)) : 0u, 0x5410);
          }
          if (lane == 0) sh.te[ring][cw] = spread ? kOwn : te;
          uint8_t *const tk = kbuf + st * C::KB, *const tv = vbuf + st * C::KB;
#pragma unroll
          for (int k = 0; k < C::NI; ++k) {
            const uint32_t z = __shfl_sync(0xffffffffu, zs, lr + C::RPI * (k / C::SPR));
            const uint32_t x[4] = {rk[k].x, rk[k].y, rk[k].z, rk[k].w};
#pragma unroll
            for (int i = 0; i < CPP; ++i)
              *reinterpret_cast<uint4 *>(tk + to[i] + (k / C::SPR) * C::RPI * 128 + (k % C::SPR) * (CPP * C::PP / 8) * kBlk) =
                  convert8<BITS>(BITS == 4 ? make_uint2(x[i], 0) : make_uint2(x[2 * i % 4], x[(2 * i + 1) % 4]), z);
          }
          hand_over(&sh.k_full[st]);
          fetch(kc, rk, b1);
          if (T + ti >= C::STAGES) ok = wait(&sh.v_empty[st], (T + ti) / C::STAGES + 1 & 1);
          if (!ok) break;
#pragma unroll
          for (int k = 0; k < C::NI; ++k) {
            const uint32_t both = __shfl_sync(0xffffffffu, zs, 16 + lr + C::RPI * (k / C::SPR));
            const uint32_t z = __byte_perm(both, 0, 0x1010), s2 = __byte_perm(both, 0, 0x3232);
            const uint32_t x[4] = {rv[k].x, rv[k].y, rv[k].z, rv[k].w};
#pragma unroll
            for (int i = 0; i < CPP; ++i) {
              uint4 o = convert8<BITS>(BITS == 4 ? make_uint2(x[i], 0) : make_uint2(x[2 * i % 4], x[(2 * i + 1) % 4]), z);
              o.x = hmul2_u(o.x, s2), o.y = hmul2_u(o.y, s2), o.z = hmul2_u(o.z, s2), o.w = hmul2_u(o.w, s2);
              *reinterpret_cast<uint4 *>(tv + to[i] + (k / C::SPR) * C::RPI * 128 + (k % C::SPR) * (CPP * C::PP / 8) * kBlk) = o;
            }
          }
          hand_over(&sh.v_full[st]);
          fetch(vc, rv, b1);
          m0 = m1;
        }
      }
      T += n;
      ++seg;
      done(turn);
    }
    if (!ok && lane == 0) sh.fail = 1;
  } else {
    // ---- softmax: stream s, half h of a tile's positions, thread = row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int s = warp / 8, h = warp / 4 % 2, row = tid % kStream;
    const uint32_t tw = tm + ((uint32_t)(warp % 4 * 32) << 16), to = tw + C::O_AT + s * HD;
    bool ok = true;
    int seg = 0, cs = 0, os = 0;  // cs: tiles of the stream, os: blocks
    unsigned T = 0, K = 0;        // K: steps of the runs before
    // the two warps of a row's halves
    auto sync_pair = [&](bool v) { return barrier_and(4 + warp / 8 * 4 + warp % 4, 64, v); };
    for (int turn = 0; ok; ++turn) {
      const Run &w = sh.run[turn & 3];
      ok = wait(&sh.run_full[turn & 3], turn >> 2 & 1);
      ok = barrier_and(3, kSoft, ok);
      if (!ok || !w.any) break;
      const int lr = w.split ? row : s * kStream + row;  // the block's row
      const bool in = lr < w.live, busy = lr - lane < w.live;
      auto token = [&]() { return (int)by_rep.divide(w.r0 + min(lr, w.live - 1)); };
      sh.limit[s][row] = in && w.len > 0 ? w.before + token() + 1 : 0;  // (by both halves' threads, the same)
      const int first = w.split ? s : 0, step = w.split ? 2 : 1;
      auto out_row = [&](int tok) {
        return reinterpret_cast<__nv_bfloat16 *>(a.o) + ((size_t)(w.q0 + tok) * a.H + w.g * rep + w.r0 + lr - tok * rep) * HD;
      };
      float m = -INFINITY, l = 0.f, c1 = 1.f;
      bool own = false;
      for (int ti = first; ti < w.n; ti += step) {
        const int ring = (T + ti) % kRing, p0 = (w.t0 + ti) * kTile + 64 * h;
        const unsigned k = K + (w.split ? ti : 2 * ti + s), buf = k % C::BUFS;
        const uint32_t ts = tw + buf * 128;
        ok = wait(&sh.s_full[buf], k / C::BUFS & 1);
        ++cs;
        tc_fence_after();
        if (ti == first) {
          c1 = BF ? a.scale : in ? sh.qf[seg & 3][lr] : 1.f;
          own = !BF && __any_sync(0xffffffffu, c1 != 1.f);
        }
        // V's exponents of the half's four times 16 positions
        const bool some = p0 + 64 > w.least;
        bool plain = !some && !own;
        if constexpr (!BF) {
          const int4 te4 = *reinterpret_cast<const int4 *>(&sh.te[ring][4 * h]);
          plain = plain && max(max(te4.x, te4.y), max(te4.z, te4.w)) < kOwn;
        }
        // u = the scores of columns 16 c .. (raw in u) plus ms (and V's exponents), -inf where they are not seen
        auto exponents = [&](float (&u)[16], int c, float ms, bool spread, bool plain) {
          const uint64_t mm = pack_f32x2(ms, ms), cc = pack_f32x2(c1, c1);
          if (!BF && !plain && own)
#pragma unroll
            for (int j = 0; j < 16; ++j) u[j] *= c1;
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            uint64_t k0 = cc, k1 = cc;
            if constexpr (!BF) {
              const float4 k4 = *reinterpret_cast<const float4 *>(&sh.sk[ring][64 * h + 16 * c + j]);
              k0 = pack_f32x2(k4.x, k4.y), k1 = pack_f32x2(k4.z, k4.w);
            }
            unpack_f32x2(fma_f32x2(pack_f32x2(u[j], u[j + 1]), k0, mm), u[j], u[j + 1]);
            unpack_f32x2(fma_f32x2(pack_f32x2(u[j + 2], u[j + 3]), k1, mm), u[j + 2], u[j + 3]);
          }
          if (plain) return;
          if (spread)
#pragma unroll
            for (int j = 0; j < 16; ++j) u[j] += sh.td[ring][64 * h + 16 * c + j];
          if (some) {
            const int n = sh.limit[s][row] - p0 - 16 * c;
#pragma unroll
            for (int j = 0; j < 16; ++j) u[j] = j < n ? u[j] : -INFINITY;
          }
        };
        // The half row's p with maximum m, into the columns whose scores have been read, and their sum (p stands for 2^-t).
        // 16 columns at a time: where those add up to kMostSum, or are the first that the row sees, m is raised first, to a whole
        // number, so that what has been computed with the old one is rescaled by an exact power of two.  (The first maximum is
        // the scores' own: powers of scores below -126 are zeros, and say nothing.)
        const float m0 = m;
        float part = 0.f;
        auto probabilities = [&](auto is_plain) {
          constexpr bool PLAIN = decltype(is_plain)::value;
          const int sees = PLAIN || !some ? 64 : sh.limit[s][row] - p0;  // of the half's columns
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int t = BF ? 0 : sh.te[ring][4 * h + c];
            const bool spread = !PLAIN && t == kOwn;
            const float te = spread ? 0.f : (float)t;
            uint32_t p[8];
            float sum, sum_l;
#pragma unroll 1
            for (bool raised = false;; raised = true) {
              float u[16];
              tmem_ld16(ts + 64 * h + 16 * c, *reinterpret_cast<uint32_t(*)[16]>(&u));
              tmem_ld_wait16(u);
              exponents(u, c, m == -INFINITY ? 0.f : te - m, spread, PLAIN);
              uint64_t s2[2] = {0, 0};
              sum_l = 0.f;
#pragma unroll
              for (int j = 0; j < 16; j += 2) {
                const float e0 = ex2(u[j]), e1 = ex2(u[j + 1]);
                p[j / 2] = BF ? pack_bf2(e0, e1) : pack_h2(e0, e1);
                s2[j / 2 % 2] = add_f32x2(s2[j / 2 % 2], pack_f32x2(e0, e1));
                if (spread)
                  sum_l += fmaf(e0, sh.tw[ring][64 * h + 16 * c + j], e1 * sh.tw[ring][64 * h + 16 * c + j + 1]);
              }
              float x, y;
              unpack_f32x2(add_f32x2(s2[0], s2[1]), x, y);
              sum = x + y;
              const bool up = sum >= kMostSum || (m == -INFINITY && sees > 16 * c);
              if (raised || !__any_sync(0xffffffffu, up)) break;
              // (rare: the scores once more)
              tmem_ld16(ts + 64 * h + 16 * c, *reinterpret_cast<uint32_t(*)[16]>(&u));
              tmem_ld_wait16(u);
              exponents(u, c, te, spread, false);
              float mx = -INFINITY;
#pragma unroll
              for (int j = 0; j < 16; ++j) mx = fmaxf(mx, u[j]);
              const float mn = up ? ceilf(mx) - C::LIFT : m, al = raise_factor(m, mn);  // (all scores -inf: no maximum yet)
              if (c > 0) rescale_p<BF>(ts + 64 * h, c, al);
              part *= al;
              m = mn;
            }
            part = spread ? part + sum_l : BF ? part + sum : fmaf(sum, pow2i(-t), part);
            tmem_st8(ts + 64 * h + 8 * c, p);
          }
        };
        if (busy && ok) {
          if (plain)
            probabilities(std::true_type());
          else
            probabilities(std::false_type());
        }
        // the halves of a row go by the larger maximum
        if (!sync_pair(ok && m == m0)) {
          sh.pm[s][h][row] = m;
          // O of the tiles before (S of this one may be older than their products)
          if (C::BUFS > 2 && ti != first && !wait(&sh.o_full[s][cs & 1], (cs - 2) >> 1 & 1)) ok = false;
          tc_fence_after();
          ok = sync_pair(ok);
          if (!ok) break;
          if (busy) {
            const float mn = fmaxf(m, sh.pm[s][h ^ 1][row]), al = raise_factor(m, mn), old = raise_factor(m0, mn);
            if (__any_sync(0xffffffffu, al != 1.f)) {
              tmem_st_wait();
              rescale_p<BF>(ts + 64 * h, 4, al);
              part *= al;
            }
            if (ti != first && __any_sync(0xffffffffu, old != 1.f)) rescale_o<HD / 32>(to + h * (HD / 2), old);
            m = mn;
            l *= old;
          }
          sync_pair(true);  // pm is read
        }
        if (busy) {
          l += part;
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[buf]);
      }

      // ---- the rows' outputs, or their parts
      const int tok = token();
      if (w.n == 0) {  // not served
        if (in && (s == 0 || !w.split))
#pragma unroll 1
          for (int e = 0; e < HD / 16; ++e)
            *reinterpret_cast<uint4 *>(out_row(tok) + h * (HD / 2) + 8 * e) = make_uint4(0, 0, 0, 0);
        done(turn);
        continue;
      }
      const bool has = first < w.n;
      if (has && ok) {
        ok = C::BUFS > 2 ? wait(&sh.o_full[s][(cs - 1) & 1], (cs - 1) >> 1 & 1) : wait(&sh.o_full[s][0], os & 1);
        ++os;
        sh.pl[s][h][row] = l;
      }
      ok = barrier_and(3, kSoft, ok);  // (both streams leave together after a timeout)
      if (!ok) break;
      tc_fence_after();
      const float L = has ? sh.pl[s][0][row] + sh.pl[s][1][row] : 0.f;
      const bool alone = w.whole && !w.split;
      // (every row of a block with tiles sees a position: a sum of 0 is that of scores that are all -inf, which have no softmax)
      const float inv = !alone ? 1.f : L == 0.f ? NAN : 1.f / L;
      const int c0 = w.c0, cl = w.cl;
      float *pt = a.part + (((size_t)blockIdx.x * 2 + (w.t0 == 0)) * kBlockRows + s * kStream + row) * (HD + 4);
      if (has && busy) {
        const int least = w.least, first_odd = least / kTile * kTile, limit = sh.limit[s][row];
        uint32_t odd = 0;
        if ((w.t0 + w.n) * kTile > least)
#pragma unroll 1
          for (int i = 0; i < 8; ++i) odd |= sh.odd[seg & 3][i][15];
#pragma unroll 1
        for (int c = 0; c < HD / 64; ++c) {
          float o[32];
          tmem_ld32(to + h * (HD / 2) + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(&o));
          tmem_ld_wait();
          if (odd != 0) {  // V rows that are not finite, added where they are seen
#pragma unroll 1
            for (int x = 0; x < 384 && first_odd + x < limit; ++x) {
              if ((sh.odd[seg & 3][x % kTile / 16][x / 32] >> (x % 32) & 1) == 0) continue;
              // (in split blocks the other stream's tiles are the other stream's to add)
              if (w.split && ((first_odd + x) / kTile - w.t0 - first) % 2 != 0) continue;
              const int p = first_odd + x, id = min(max(a.tables[(size_t)w.b * a.max_pages + (p >> a.shift)], 0), a.n_pages - 1);
              const size_t at = (((size_t)id * a.Hkv + w.g) << a.shift) + (p & (page - 1));
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                const float f = BF ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(a.vc)[at * HD + h * (HD / 2) + 32 * c + e])
                                   : __int_as_float(0x7fffffff);
                if (!isfinite(f)) o[e] += f;
              }
            }
          }
          // four lanes write 64 bytes of a row together: lane i of four has rows i' = 0 .. 3's 16 bytes i
          const int quad = lane & ~3, at = lane & 3;
          if (alone) {
            uint4 v[4];
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              v[e / 8] = make_uint4(pack_bf2(o[e] * inv, o[e + 1] * inv), pack_bf2(o[e + 2] * inv, o[e + 3] * inv),
                                    pack_bf2(o[e + 4] * inv, o[e + 5] * inv), pack_bf2(o[e + 6] * inv, o[e + 7] * inv));
            transpose4(v, at);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int other = lr - at + i, ot = __shfl_sync(0xffffffffu, tok, quad + i);
              if (other < w.live)
                *reinterpret_cast<uint4 *>(out_row(ot) + (ptrdiff_t)(other - lr) * HD + h * (HD / 2) + 32 * c + 8 * at) = v[i];
            }
          } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint4 v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                v[e] = make_uint4(__float_as_uint(o[16 * k + 4 * e]), __float_as_uint(o[16 * k + 4 * e + 1]),
                                  __float_as_uint(o[16 * k + 4 * e + 2]), __float_as_uint(o[16 * k + 4 * e + 3]));
              transpose4(v, at);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (lr - at + i < w.live)
                  *reinterpret_cast<uint4 *>(pt + (i - at) * (HD + 4) + h * (HD / 2) + 32 * c + 16 * k + 4 * at) = v[i];
            }
          }
        }
      }
      tc_fence_before();
      if (!alone) {
        if (in && h == 0) *reinterpret_cast<float2 *>(pt + HD) = make_float2(m, L);
        __threadfence();
        named_barrier_sync(3, kSoft);
        if (!w.whole) {
          if (tid == 0) {
            sh.last = atomicAdd(&a.counters[c0], 1) == cl - c0;
            if (sh.last) a.counters[c0] = 0;
          }
          named_barrier_sync(3, kSoft);
        }
        if (w.whole || sh.last) {
          // all parts of the block in their order: CTA c0 has its begin (in its place 1), the others their first blocks
          // (0); a split block's streams one after the other
          __threadfence();
          constexpr int LPR = HD / 4, RU = 4, STEP = kSoft / LPR, ROW = HD + 4, PART = kBlockRows * ROW;  // lanes a row, rows of a thread in flight
          // (the run's numbers by value: stores of results might otherwise be stores to them)
          const int e = 4 * (tid % LPR), split = w.split, parts = (cl - c0 + 1) << split, live = w.live, r0 = w.r0, h0 = w.g * rep;
          const float *const p0 = a.part + (size_t)c0 * 2 * PART;
          __nv_bfloat16 *const o0 = reinterpret_cast<__nv_bfloat16 *>(a.o) + ((size_t)w.q0 * a.H + h0) * HD + e;
#pragma unroll 1
          for (int r = tid / LPR; r < live; r += RU * STEP) {
            float M[RU], S[RU];
            float4 O[RU];
            int at[RU];
#pragma unroll
            for (int j = 0; j < RU; ++j) {
              M[j] = -INFINITY, S[j] = 0.f, O[j] = make_float4(0.f, 0.f, 0.f, 0.f);
              at[j] = min(r + j * STEP, live - 1) * ROW;
            }
#pragma unroll 1
            for (int k = 0; k < parts; ++k) {
              const int cta = k >> split;
              const float *const ps = p0 + (size_t)(cta == 0 ? 1 : 2 * cta) * PART + (k & split) * (kStream * ROW);
              float2 ml[RU];
              float4 ov[RU];
#pragma unroll
              for (int j = 0; j < RU; ++j) {
                ml[j] = __ldcg(reinterpret_cast<const float2 *>(ps + at[j] + HD));
                ov[j] = __ldcg(reinterpret_cast<const float4 *>(ps + at[j] + e));
              }
#pragma unroll
              for (int j = 0; j < RU; ++j) {
                const bool none = ml[j].x == -INFINITY;  // (then its values were not written, or its sum alone counts)
                const float mn = fmaxf(M[j], ml[j].x);
                const float f0 = M[j] == -INFINITY ? 0.f : ex2(M[j] - mn), f = none ? 0.f : ex2(ml[j].x - mn);
                S[j] = fmaf(S[j], M[j] == -INFINITY ? 1.f : f0, none ? ml[j].y : ml[j].y * f);  // (a NaN of a part stays NaN)
                M[j] = mn;
                O[j].x = fmaf(none ? 0.f : ov[j].x, f, O[j].x * f0), O[j].y = fmaf(none ? 0.f : ov[j].y, f, O[j].y * f0);
                O[j].z = fmaf(none ? 0.f : ov[j].z, f, O[j].z * f0), O[j].w = fmaf(none ? 0.f : ov[j].w, f, O[j].w * f0);
              }
            }
#pragma unroll
            for (int j = 0; j < RU; ++j) {
              const int rr = r0 + r + j * STEP, t = (int)by_rep.divide(rr);
              const float inv = S[j] == 0.f ? NAN : 1.f / S[j];
              if (r + j * STEP < live)
                *reinterpret_cast<uint2 *>(o0 + ((ptrdiff_t)t * a.H + rr - t * rep) * HD) =
                    make_uint2(pack_bf2(O[j].x * inv, O[j].y * inv), pack_bf2(O[j].z * inv, O[j].w * inv));
            }
          }
        }
      }
      T += w.n;
      K += w.split ? w.n : 2 * w.n;
      ++seg;
      done(turn);
    }
    if (!ok && lane == 0) sh.fail = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (sh.fail) {
    // what the MMA warp issued last is given time to end before its memory goes
    if (tid == 0) atomicExch(&g_attn_paged_tc_status, -6);
    const unsigned long long t0 = global_timer_ns();
    for (int i = 0; i < (1 << 20) && global_timer_ns() - t0 < 2000000ull; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tm, kTmemCols);
  }
}

size_t attn_paged_tc_part_floats(int hd, int num_sms) { return (size_t)num_sms * 2 * kBlockRows * (hd + 4); }

namespace {

template <int HD, int BITS>
cudaError_t launch_t(const AttnPagedArgs &a, int num_sms, cudaStream_t s) {
  constexpr int smem = Cfg<HD, BITS>::SMEM;
  static std::atomic<bool> done[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  auto k = attn_paged_tc_kernel<HD, BITS>;
  if (dev < 0 || dev >= 64 || !done[dev].load(std::memory_order_acquire)) {
    // whether the warps' shares of registers fit into what a block is launched with (their exchange would wait forever)
    cudaFuncAttributes f;
    if ((e = cudaFuncGetAttributes(&f, k)) != cudaSuccess) return e;
    if (kRegsSoftmax * kSoft + kRegsConv * kConv + kRegsMma * 128 > f.numRegs * kThreads) return cudaErrorInvalidConfiguration;
    if ((e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
  }
  const long long blocks = ((long long)a.m * (a.H / a.Hkv) + kBlockRows - 1) / kBlockRows + a.batch;
  const long long tiles = (((long long)a.max_pages << a.shift) + kTile - 1) / kTile;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)std::min((long long)num_sms, blocks * tiles * a.Hkv));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  return cudaLaunchKernelEx(&cfg, k, a, Divisor(a.H / a.Hkv));
}

}  // namespace

cudaError_t launch_attn_paged_tc(const AttnPagedArgs &a, int hd, int bits, int num_sms, cudaStream_t s) {
#define WQ_PAGED(HD, BITS) \
  if (hd == HD && bits == BITS) return launch_t<HD, BITS>(a, num_sms, s);
  WQ_PAGED(128, 16) WQ_PAGED(128, 8) WQ_PAGED(128, 4) WQ_PAGED(64, 16) WQ_PAGED(64, 8) WQ_PAGED(64, 4)
#undef WQ_PAGED
  return cudaErrorInvalidValue;
}

cudaError_t read_attn_paged_tc_status(int *status) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(status, g_attn_paged_tc_status, sizeof(int));
  if (e != cudaSuccess) return e;
  const int zero = 0;
  return cudaMemcpyToSymbol(g_attn_paged_tc_status, &zero, sizeof(int));
}

}  // namespace wq
