// wq_kv.cu -- what feeds tree attention (sm_103a): rows quantized into the KV
// cache as they are written, cached rows read back, and the head norm and
// rotary positions of drafted tokens' projections.
//
// A cached row is one position's K or V of one kv head (HD values):
//   s = fp16((mx - mn) / qmax), mn = min(0, row), mx = max(0, row)  (1 if zero, z then -0),
//   z = clamp(rint(-mn / s), 0, qmax), code = clamp(rint(v / s) + z, 0, qmax),
// value s (code - z), in fp32 with explicit round-to-nearest.  0 lies in the
// range, so z needs no sign and code - z is a whole number of 9 bits: an exact
// binary16 operand, with one scale a row, for the attention's matrix products.
// A row with a value that is not finite, or a scale beyond binary16, is held as
// scale NaN, codes 0: it reads back as NaN.
//
// A row is taken by 8 lanes (HD 128) or 4 (HD 64), 16 values a lane: 3 or 2
// shuffles for the row's range, and the lane's codes are one 16-byte (8 bits)
// or 8-byte (4 bits) store.  A lane takes a K row and the V row beside it (one row
// a lane: less in flight, 28.8 us for 26.6 below).  8191 tokens of 8 kv heads are
// written to 4 bits and read back to bf16 in 21.6 us, 3.5 TB/s; written alone, in 14.1
// us, to 8 bits 13.6, to a bf16 cache 13.1 (5.1 TB/s), and from fp32 17.7, 17.3 and
// 18.7.  Neither issue slots (55% of them at 4 bits, 17 instructions a value; with a
// division a value and codes clamped one by one 24, 31.5 us the pair) nor memory is full:
// a CTA loads its rows once and then works on them, and at 80 registers a thread 20 of
// an SM's warps cannot hide that.  Reads are bound by HBM: 12,000 tokens of 8 bits 11.0
// us, 6.8 TB/s; 32,768 of 4 bits to fp32 49.8 us, 6.1 TB/s.  Decode steps are bound by
// launches: 16 tokens written and read back 4.4 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "wq_cvt.cuh"
#include "wq_internal.h"
#include "wq_kv.h"
#include "wq_ptx.cuh"
#include "wq_rows.cuh"

namespace wq {

// Status word of these kernels: WQ_OK (0), or WQ_ERR_ARG (-1) after a start,
// count, index or position outside its range was met on the device (what it
// names is skipped).  Read and cleared by read_kv_status.
__device__ int g_kv_status = 0;

namespace {

constexpr int kAppendThreads = 128, kReadThreads = 256;

}  // namespace

// Slot i of the launch: sequence, head and step n, the step fastest, so that
// neighbouring rows of the cache are written together (tokens in groups with their
// other heads beside them took the same time).
// Lane l of a slot holds values 16 l .. 16 l + 15 of its K row and of its V row.
template <int HD, int BITS, bool F32>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const KvAppendArgs a, const Divisor by_n, const Divisor by_kv) {
  constexpr int LPR = HD / 16;  // lanes a row
  pdl_wait();
  pdl_launch_dependents();
  const unsigned slot = blockIdx.x * (kAppendThreads / LPR) + threadIdx.x / LPR;
  const int lane = threadIdx.x % LPR;
  bool put = slot < (unsigned)a.batch * a.n_kv * a.n;  // below 2^30 (host check)
  const unsigned bh = by_n.divide(slot);
  const int n = (int)(slot - bh * (unsigned)a.n);
  const int b = (int)by_kv.divide(bh), h = (int)(bh - (unsigned)b * (unsigned)a.n_kv);
  int t = n;
  long long pos = 0;
  if (put) {
    const int start = a.start[b], cnt = a.counts ? a.counts[b] : a.n;
    if (a.index) t = a.index[(size_t)b * a.n + n];
    if (cnt < 0 || cnt > a.n || start < 0 || (long long)start + cnt > a.max_len) {
      if (lane == 0) atomicExch(&g_kv_status, -1);
      put = false;
    } else if (n >= cnt) {
      put = false;
    } else if (t < 0 || t >= a.n_src) {
      if (lane == 0) atomicExch(&g_kv_status, -1);
      put = false;
    }
    pos = (long long)start + n;
  }
  float v[2][16];
  uint4 raw[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const long long *st = i ? a.v_stride : a.k_stride;
    const long long off = put ? (long long)b * st[0] + (long long)t * st[1] + (long long)h * st[2] + lane * 16 : 0;
    if (F32) {
      const float4 *src = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(i ? a.v : a.k) + off);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 f = put ? __ldcs(src + k) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[i][4 * k] = f.x, v[i][4 * k + 1] = f.y, v[i][4 * k + 2] = f.z, v[i][4 * k + 3] = f.w;
      }
    } else {
      const uint4 *src = reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(i ? a.v : a.k) + off);
      raw[i][0] = put ? __ldcs(src) : make_uint4(0, 0, 0, 0);
      raw[i][1] = put ? __ldcs(src + 1) : make_uint4(0, 0, 0, 0);
    }
  }
  const size_t row = ((size_t)b * a.n_kv + h) * a.max_len + pos;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (BITS == 16) {
      if (!put) continue;
      uint4 *dst = reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(i ? a.vc : a.kc) + row * HD + lane * 16);
      if (F32) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          raw[i][k] = make_uint4(pack_bf2(v[i][8 * k], v[i][8 * k + 1]), pack_bf2(v[i][8 * k + 2], v[i][8 * k + 3]),
                                 pack_bf2(v[i][8 * k + 4], v[i][8 * k + 5]), pack_bf2(v[i][8 * k + 6], v[i][8 * k + 7]));
      }
      dst[0] = raw[i][0];
      dst[1] = raw[i][1];
    } else {
      // the row's range around 0 (a NaN is kept in mx)
      float mn = 0.f, mx = 0.f;
      if (F32) {
        bool nan = false;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          mn = fminf(mn, v[i][e]);
          mx = fmaxf(mx, v[i][e]);
          nan |= v[i][e] != v[i][e];
        }
        if (nan) mx = __int_as_float(0x7fffffff);
#pragma unroll
        for (int o = LPR / 2; o >= 1; o >>= 1) {
          const float x = __shfl_xor_sync(0xffffffffu, mn, o), y = __shfl_xor_sync(0xffffffffu, mx, o);
          mn = fminf(mn, x);
          mx = y > mx || y != y ? y : mx;
        }
      } else {
        __nv_bfloat162 lo = __float2bfloat162_rn(0.f), hi = lo;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t w[4] = {raw[i][k].x, raw[i][k].y, raw[i][k].z, raw[i][k].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&w[j]);
            lo = __hmin2_nan(lo, x);
            hi = __hmax2_nan(hi, x);
            v[i][8 * k + 2 * j] = bf_lo(w[j]), v[i][8 * k + 2 * j + 1] = bf_hi(w[j]);
          }
        }
        // (the most, minus the least) go through the lanes together
        __nv_bfloat162 r = __halves2bfloat162(__hmax_nan(__low2bfloat16(hi), __high2bfloat16(hi)),
                                              __hneg(__hmin_nan(__low2bfloat16(lo), __high2bfloat16(lo))));
#pragma unroll
        for (int o = LPR / 2; o >= 1; o >>= 1) r = __hmax2_nan(r, __shfl_xor_sync(0xffffffffu, r, o));
        mx = __low2float(r);
        mn = -__high2float(r);
      }
      uint32_t c[8];
      const uint32_t meta = quantize16<BITS>(v[i], mn, mx, c);
      if (!put) continue;
      uint8_t *dst = reinterpret_cast<uint8_t *>(i ? a.vc : a.kc) + row * (HD * BITS / 8) + lane * (2 * BITS);
      uint32_t w[BITS / 2];
      pack_codes<BITS>(c, w);
      if constexpr (BITS == 8)
        *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
      else
        *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
      if (lane == 0) (i ? a.vm : a.km)[row] = meta;
    }
  }
}

template <int HD, int BITS, bool F32>
__global__ void __launch_bounds__(kReadThreads) kv_read_kernel(const KvReadArgs a, const Divisor by_n, const Divisor by_kv) {
  constexpr int LPR = HD / 16;  // lanes a row
  pdl_wait();
  pdl_launch_dependents();
  const unsigned slot = blockIdx.x * (kReadThreads / LPR) + threadIdx.x / LPR;
  const int lane = threadIdx.x % LPR;
  const unsigned per_cache = (unsigned)a.batch * a.n_kv * a.n;  // below 2^30 (host check)
  if (slot >= 2 * per_cache) return;
  const bool is_v = slot >= per_cache;
  const unsigned rest = is_v ? slot - per_cache : slot;
  const unsigned bh = by_n.divide(rest);
  const int n = (int)(rest - bh * (unsigned)a.n);
  const int b = (int)by_kv.divide(bh), h = (int)(bh - (unsigned)b * (unsigned)a.n_kv);
  const int start = a.start[b], cnt = a.counts ? a.counts[b] : a.n;
  if (cnt < 0 || cnt > a.n || start < 0 || (long long)start + cnt > a.max_len) {
    if (lane == 0) atomicExch(&g_kv_status, -1);
    return;
  }
  const size_t row = ((size_t)b * a.n_kv + h) * a.max_len + start + n;
  const size_t out = (((size_t)b * a.n + n) * a.n_kv + h) * HD;
  const bool get = n < cnt;
  read_row<HD, BITS, F32>(is_v ? a.vc : a.kc, is_v ? a.vm : a.km, row, lane, get, is_v ? a.v : a.k, out);
}

// Query, key and value rows of a token from its fp32 projections: all scaled by
// the layer input's RMSNorm 1 / sqrt(mean(x^2) + eps) (x given), queries and
// keys normed per head and rotated by the table's cosines and sines at the
// token's position (value i with i + HD/2), each rounded once to bf16.  A CTA
// takes one token; LPR lanes take a head, 4 values of each half a lane, and a
// lane's heads are loaded before the sum over x is waited for.  10 tokens of 48 heads
// of 128 take 2.8 us, launch latency; 1220 tokens of 56 heads 14.4 us, 4.6 TB/s: loads
// in flight bound it (72 registers a thread leave 7 CTAs of 128 threads an SM, and a CTA's
// loads start when one before it has left).

template <int HD, int THREADS>
__global__ void __launch_bounds__(THREADS, 896 / THREADS) qkv_rope_kernel(const QkvRopeArgs a) {
  constexpr int LPR = HD / 8, GROUPS = THREADS / LPR, MAXU = 4;  // lanes a head, heads a pass, passes in registers
  __shared__ float red[THREADS / 32];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid % LPR, grp = tid / LPR;
  const int heads = a.n_heads + 2 * a.n_kv;
  const size_t tok = blockIdx.x;
  const int pos = a.positions[tok];
  if (pos < 0 || pos >= a.n_pos) {
    if (tid == 0) atomicExch(&g_kv_status, -1);
    return;
  }
  const float *src = a.qkv + tok * heads * HD;
  float4 lo[MAXU], hi[MAXU];
  auto fetch = [&](int h0) {
#pragma unroll
    for (int u = 0; u < MAXU; ++u) {
      const int h = h0 + u * GROUPS + grp;
      if (h < heads) {
        lo[u] = __ldcs(reinterpret_cast<const float4 *>(src + (size_t)h * HD + 4 * lane));
        hi[u] = __ldcs(reinterpret_cast<const float4 *>(src + (size_t)h * HD + HD / 2 + 4 * lane));
      }
    }
  };
  fetch(0);
  // cos, sin of the lane's four angles
  const float4 *tab = reinterpret_cast<const float4 *>(a.table + ((size_t)pos * (HD / 2) + 4 * lane) * 2);
  const float4 cs0 = tab[0], cs1 = tab[1];
  const float co[4] = {cs0.x, cs0.z, cs1.x, cs1.z}, si[4] = {cs0.y, cs0.w, cs1.y, cs1.w};
  float rs = 1.f;
  if (a.x) {
    float ss = 0.f;
    const uint4 *xs = reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(a.x) + tok * a.d);
    for (int i = tid; i < a.d / 8; i += THREADS) {
      const uint4 q = xs[i];
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ss = fmaf(bf_lo(w[e]), bf_lo(w[e]), ss);
        ss = fmaf(bf_hi(w[e]), bf_hi(w[e]), ss);
      }
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (tid % 32 == 0) red[tid / 32] = ss;
    __syncthreads();
    float tot = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) tot += red[w];
    rs = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fdiv_rn(tot, (float)a.d), kRmsEps)));
  }
  for (int h0 = 0; h0 < heads; h0 += MAXU * GROUPS) {
    if (h0 > 0) fetch(h0);
#pragma unroll
    for (int u = 0; u < MAXU; ++u) {
      const int h = h0 + u * GROUPS + grp;
      if (h0 + u * GROUPS >= heads) break;  // uniform in the CTA
      const bool in = h < heads;
      float x0[4] = {lo[u].x * rs, lo[u].y * rs, lo[u].z * rs, lo[u].w * rs};
      float x1[4] = {hi[u].x * rs, hi[u].y * rs, hi[u].z * rs, hi[u].w * rs};
      if (!in)
#pragma unroll
        for (int e = 0; e < 4; ++e) x0[e] = x1[e] = 0.f;
      const bool turns = h < a.n_heads + a.n_kv;
      float hn = 1.f;
      if (a.head_norm) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sq = fmaf(x0[e], x0[e], fmaf(x1[e], x1[e], sq));
#pragma unroll
        for (int o = LPR / 2; o >= 1; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
        hn = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sq, (float)HD), kRmsEps)));
      }
      if (turns)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = x0[e] * hn, q = x1[e] * hn;
          x0[e] = p * co[e] - q * si[e];
          x1[e] = q * co[e] + p * si[e];
        }
      if (!in) continue;
      __nv_bfloat16 *dst = h < a.n_heads ? reinterpret_cast<__nv_bfloat16 *>(a.q) + (tok * a.n_heads + h) * HD
                           : turns       ? reinterpret_cast<__nv_bfloat16 *>(a.k) + (tok * a.n_kv + h - a.n_heads) * HD
                                         : reinterpret_cast<__nv_bfloat16 *>(a.v) +
                                         (tok * a.n_kv + h - a.n_heads - a.n_kv) * HD;
      *reinterpret_cast<uint2 *>(dst + 4 * lane) = make_uint2(pack_bf2(x0[0], x0[1]), pack_bf2(x0[2], x0[3]));
      *reinterpret_cast<uint2 *>(dst + HD / 2 + 4 * lane) = make_uint2(pack_bf2(x1[0], x1[1]), pack_bf2(x1[2], x1[3]));
    }
  }
}

cudaError_t launch_kv_append(const KvAppendArgs &a, int hd, int bits, bool f32, cudaStream_t s) {
  const unsigned grid = row_ctas((long long)a.batch * a.n_kv * a.n, hd, kAppendThreads);
#define WQ_APPEND(HD, BITS)                                                               \
  if (hd == HD && bits == BITS)                                                           \
    return f32 ? launch_pdl(kv_append_kernel<HD, BITS, true>, grid, kAppendThreads, s, a, Divisor(a.n), Divisor(a.n_kv))     \
               : launch_pdl(kv_append_kernel<HD, BITS, false>, grid, kAppendThreads, s, a, Divisor(a.n), Divisor(a.n_kv));
  WQ_APPEND(128, 16) WQ_APPEND(128, 8) WQ_APPEND(128, 4) WQ_APPEND(64, 16) WQ_APPEND(64, 8) WQ_APPEND(64, 4)
#undef WQ_APPEND
  return cudaErrorInvalidValue;
}

cudaError_t launch_kv_read(const KvReadArgs &a, int hd, int bits, bool f32, cudaStream_t s) {
  const unsigned grid = row_ctas(2ll * a.batch * a.n_kv * a.n, hd, kReadThreads);
#define WQ_READ(HD, BITS)                                                               \
  if (hd == HD && bits == BITS)                                                         \
    return f32 ? launch_pdl(kv_read_kernel<HD, BITS, true>, grid, kReadThreads, s, a, Divisor(a.n), Divisor(a.n_kv))     \
               : launch_pdl(kv_read_kernel<HD, BITS, false>, grid, kReadThreads, s, a, Divisor(a.n), Divisor(a.n_kv));
  WQ_READ(128, 16) WQ_READ(128, 8) WQ_READ(128, 4) WQ_READ(64, 16) WQ_READ(64, 8) WQ_READ(64, 4)
#undef WQ_READ
  return cudaErrorInvalidValue;
}

cudaError_t launch_qkv_rope(const QkvRopeArgs &a, int m, int hd, int num_sms, cudaStream_t s) {
  // Up to two tokens an SM 256 threads a token, whose heads are then all in flight (304
  // tokens of 48 heads 4.4 us, with 128 threads 5.5), above that 128, of which seven
  // CTAs fit an SM where of 256 only three do (1220 tokens of 56 heads 14.5 us for 20.9).
  const bool few = m <= 2 * num_sms;
  if (hd == 128)
    return few ? launch_pdl(qkv_rope_kernel<128, 256>, (unsigned)m, 256, s, a)
               : launch_pdl(qkv_rope_kernel<128, 128>, (unsigned)m, 128, s, a);
  if (hd == 64)
    return few ? launch_pdl(qkv_rope_kernel<64, 256>, (unsigned)m, 256, s, a)
               : launch_pdl(qkv_rope_kernel<64, 128>, (unsigned)m, 128, s, a);
  return cudaErrorInvalidValue;
}

cudaError_t read_kv_status(int *status) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(status, g_kv_status, sizeof(int));
  if (e != cudaSuccess) return e;
  const int zero = 0;
  return cudaMemcpyToSymbol(g_kv_status, &zero, sizeof(int));
}

}  // namespace wq
