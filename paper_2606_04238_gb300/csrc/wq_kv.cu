// wq_kv.cu -- what feeds tree attention (sm_103a): rows quantized into the KV
// cache as they are written, cached rows read back, and the head norm and
// rotary positions of drafted tokens' projections.
//
// A cached row is one position's K or V of one kv head (HD values):
//   s = fp16((mx - mn) / qmax), mn = min(0, row), mx = max(0, row)  (1 if zero),
//   z = clamp(rint(-mn / s), 0, qmax), code = clamp(rint(v / s) + z, 0, qmax),
// value s (code - z), in fp32 with explicit round-to-nearest.  0 lies in the
// range, so z needs no sign and code - z is a whole number of 9 bits: an exact
// binary16 operand, with one scale a row, for the attention's matrix products.
// A row with a value that is not finite, or a scale beyond binary16, is held as
// scale NaN, codes 0: it reads back as NaN.
//
// A row is taken by 8 lanes (HD 128) or 4 (HD 64), 16 values a lane: 3 or 2
// shuffles for the row's range, and the lane's codes are one 16-byte (8 bits)
// or 8-byte (4 bits) store.  Bound by HBM for prompts, by launch latency for
// decode steps.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "wq_internal.h"
#include "wq_kv.h"
#include "wq_ptx.cuh"
#include "wq_quant.cuh"

namespace wq {

// Status word of these kernels: WQ_OK (0), or WQ_ERR_ARG (-1) after a start,
// count, index or position outside its range was met on the device (what it
// names is skipped).  Read and cleared by read_kv_status.
__device__ int g_kv_status = 0;

namespace {

constexpr int kKvThreads = 256;

__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}

}  // namespace

// Slot i of the launch: cache (K, V), sequence, head and step n, the step
// fastest, so that neighbouring rows of the cache are written together.  Lane l
// of a row holds its values 16 l .. 16 l + 15.
template <int HD, int BITS, bool F32>
__global__ void __launch_bounds__(kKvThreads) kv_append_kernel(const KvAppendArgs a) {
  constexpr int LPR = HD / 16;  // lanes a row
  pdl_wait();
  pdl_launch_dependents();
  const long long slot = (long long)blockIdx.x * (kKvThreads / LPR) + threadIdx.x / LPR;
  const int lane = threadIdx.x % LPR;
  const long long per_cache = (long long)a.batch * a.n_kv * a.n;
  const bool in = slot < 2 * per_cache;
  const bool is_v = slot >= per_cache;
  const unsigned rest = (unsigned)(is_v ? slot - per_cache : slot);  // below 2^31 (host check)
  const unsigned bh = rest / (unsigned)a.n;
  const int n = (int)(rest - bh * (unsigned)a.n);
  const int b = (int)(bh / (unsigned)a.n_kv), h = (int)(bh - (unsigned)b * (unsigned)a.n_kv);
  bool put = in;
  int t = n;
  long long pos = 0;
  if (in) {
    const int start = a.start[b], cnt = a.counts ? a.counts[b] : a.n;
    if (cnt < 0 || cnt > a.n || start < 0 || (long long)start + cnt > a.max_len) {
      if (lane == 0) atomicExch(&g_kv_status, -1);
      put = false;
    } else if (n >= cnt) {
      put = false;
    } else {
      pos = (long long)start + n;
      if (a.index) t = a.index[(size_t)b * a.n + n];
      if (t < 0 || t >= a.n_src) {
        if (lane == 0) atomicExch(&g_kv_status, -1);
        put = false;
      }
    }
  }
  float v[16];
  uint4 raw[2];
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = 0.f;
  raw[0] = raw[1] = make_uint4(0, 0, 0, 0);
  if (put) {
    const long long *st = is_v ? a.v_stride : a.k_stride;
    const long long off = (long long)b * st[0] + (long long)t * st[1] + (long long)h * st[2] + lane * 16;
    if (F32) {
      const float4 *src = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(is_v ? a.v : a.k) + off);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 f = __ldcs(src + i);
        v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
      }
    } else {
      const uint4 *src = reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(is_v ? a.v : a.k) + off);
      raw[0] = __ldcs(src);
      raw[1] = __ldcs(src + 1);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[8 * i + 2 * j] = bf_lo(w[j]), v[8 * i + 2 * j + 1] = bf_hi(w[j]);
      }
    }
  }
  const size_t row = ((size_t)b * a.n_kv + h) * a.max_len + pos;
  if constexpr (BITS == 16) {
    if (!put) return;
    uint4 *dst = reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(is_v ? a.vc : a.kc) + row * HD + lane * 16);
    if (F32) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        raw[i] = make_uint4(pack_bf2(v[8 * i], v[8 * i + 1]), pack_bf2(v[8 * i + 2], v[8 * i + 3]),
                            pack_bf2(v[8 * i + 4], v[8 * i + 5]), pack_bf2(v[8 * i + 6], v[8 * i + 7]));
    }
    dst[0] = raw[0];
    dst[1] = raw[1];
  } else {
    constexpr float qmax = (float)((1 << BITS) - 1);
    float mn = 0.f, mx = 0.f;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      mn = fminf(mn, v[e]);
      mx = fmaxf(mx, v[e]);
      bad |= !isfinite(v[e]);
    }
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) {
      mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      bad |= __shfl_xor_sync(0xffffffffu, (int)bad, o) != 0;
    }
    __half sh = __float2half_rn(__fdiv_rn(__fsub_rn(mx, mn), qmax));
    if (__half2float(sh) == 0.f) sh = __float2half_rn(1.f);
    const float sf = __half2float(sh);
    bad |= !isfinite(sf);
    const float zf = bad ? 0.f : __fadd_rn(fminf(fmaxf(rintf(__fdiv_rn(-mn, sf)), 0.f), qmax), 0.f);
    const float rcp = __frcp_rn(sf);
    uint32_t c[16];
#pragma unroll
    for (int e = 0; e < 16; ++e)
      c[e] = bad ? 0u : (uint32_t)fminf(fmaxf(__fadd_rn(rint_div(v[e], sf, rcp), zf), 0.f), qmax);
    if (!put) return;
    uint8_t *dst = reinterpret_cast<uint8_t *>(is_v ? a.vc : a.kc) + row * (HD * BITS / 8) + lane * (2 * BITS);
    if (BITS == 8) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = c[4 * i] | c[4 * i + 1] << 8 | c[4 * i + 2] << 16 | c[4 * i + 3] << 24;
      *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      // value e of a word of 8 at bits 4 (e / 2) + 16 (e % 2)
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 16; ++e) w[e / 8] |= c[e] << (4 * (e % 8 / 2) + 16 * (e % 2));
      *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
    }
    if (lane == 0)
      (is_v ? a.vm : a.km)[row] = (bad ? 0x7fffu : (uint32_t)__half_as_ushort(sh)) |
                                  (uint32_t)__half_as_ushort(__float2half_rn(zf)) << 16;
  }
}

// A lane takes 8 values at a time, chunks l and l + LPR of its row, so that a
// row's stores are whole 128-byte lines.
template <int HD, int BITS, bool F32>
__global__ void __launch_bounds__(kKvThreads) kv_read_kernel(const KvReadArgs a) {
  constexpr int LPR = HD / 16;
  pdl_wait();
  pdl_launch_dependents();
  const long long slot = (long long)blockIdx.x * (kKvThreads / LPR) + threadIdx.x / LPR;
  const int lane = threadIdx.x % LPR;
  const long long per_cache = (long long)a.batch * a.n_kv * a.n;
  if (slot >= 2 * per_cache) return;
  const bool is_v = slot >= per_cache;
  const unsigned rest = (unsigned)(is_v ? slot - per_cache : slot);
  const unsigned bh = rest / (unsigned)a.n;
  const int n = (int)(rest - bh * (unsigned)a.n);
  const int b = (int)(bh / (unsigned)a.n_kv), h = (int)(bh - (unsigned)b * (unsigned)a.n_kv);
  const int start = a.start[b], cnt = a.counts ? a.counts[b] : a.n;
  if (cnt < 0 || cnt > a.n || start < 0 || (long long)start + cnt > a.max_len) {
    if (lane == 0) atomicExch(&g_kv_status, -1);
    return;
  }
  const size_t row = ((size_t)b * a.n_kv + h) * a.max_len + start + n;
  const size_t out = (((size_t)b * a.n + n) * a.n_kv + h) * HD;
  const bool get = n < cnt;
  const void *cache = is_v ? a.vc : a.kc;
  float v[2][8];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
  if (get) {
    float s = 0.f, z = 0.f;
    if (BITS != 16) {
      const uint32_t m = (is_v ? a.vm : a.km)[row];
      s = __half2float(__ushort_as_half((unsigned short)(m & 0xffffu)));
      z = __half2float(__ushort_as_half((unsigned short)(m >> 16)));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = lane + i * LPR;  // chunk of 8 values
      if (BITS == 16) {
        const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(cache) + row * HD + c * 8));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][2 * j] = bf_lo(w[j]), v[i][2 * j + 1] = bf_hi(w[j]);
      } else if (BITS == 8) {
        const uint2 q = __ldcs(reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(cache) + row * HD + c * 8));
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[i][e] = __fmul_rn(s, (float)((e < 4 ? q.x : q.y) >> (8 * (e % 4)) & 0xffu) - z);
      } else {
        const uint32_t q = __ldcs(reinterpret_cast<const uint32_t *>(reinterpret_cast<const uint8_t *>(cache) + row * (HD / 2) + c * 4));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = __fmul_rn(s, (float)(q >> (4 * (e / 2) + 16 * (e % 2)) & 0xfu) - z);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const size_t at = out + (lane + i * LPR) * 8;
    if (F32) {
      float4 *dst = reinterpret_cast<float4 *>(reinterpret_cast<float *>(is_v ? a.v : a.k) + at);
      dst[0] = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]);
      dst[1] = make_float4(v[i][4], v[i][5], v[i][6], v[i][7]);
    } else {
      *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(is_v ? a.v : a.k) + at) =
          make_uint4(pack_bf2(v[i][0], v[i][1]), pack_bf2(v[i][2], v[i][3]), pack_bf2(v[i][4], v[i][5]),
                     pack_bf2(v[i][6], v[i][7]));
    }
  }
}

// Query, key and value rows of a token from its fp32 projections: all scaled by
// the layer input's RMSNorm 1 / sqrt(mean(x^2) + eps) (x given), queries and
// keys normed per head and rotated by the table's cosines and sines at the
// token's position (value i with i + HD/2), each rounded once to bf16.  A CTA
// takes one token; LPR lanes take a head, 4 values of each half a lane, and a
// lane's heads are loaded before the sum over x is waited for.
constexpr int kRopeThreads = 256;

template <int HD>
__global__ void __launch_bounds__(kRopeThreads) qkv_rope_kernel(const QkvRopeArgs a) {
  constexpr int LPR = HD / 8, GROUPS = kRopeThreads / LPR, MAXU = 4;  // lanes a head, heads a pass, passes in registers
  __shared__ float red[kRopeThreads / 32];
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
    for (int i = tid; i < a.d / 8; i += kRopeThreads) {
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
    for (int w = 0; w < kRopeThreads / 32; ++w) tot += red[w];
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

namespace {

template <class Kernel, class Args>
cudaError_t launch_pdl(Kernel k, const Args &a, unsigned grid, int threads, cudaStream_t s) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  return cudaLaunchKernelEx(&cfg, k, a);
}

// CTAs of a launch of one row (of hd values) per hd / 16 lanes.
unsigned row_ctas(long long rows, int hd) {
  const long long per = kKvThreads / (hd / 16);
  return (unsigned)((rows + per - 1) / per);
}

}  // namespace

cudaError_t launch_kv_append(const KvAppendArgs &a, int hd, int bits, bool f32, cudaStream_t s) {
  const unsigned grid = row_ctas(2ll * a.batch * a.n_kv * a.n, hd);
#define WQ_APPEND(HD, BITS)                                                               \
  if (hd == HD && bits == BITS)                                                           \
    return f32 ? launch_pdl(kv_append_kernel<HD, BITS, true>, a, grid, kKvThreads, s)     \
               : launch_pdl(kv_append_kernel<HD, BITS, false>, a, grid, kKvThreads, s);
  WQ_APPEND(128, 16) WQ_APPEND(128, 8) WQ_APPEND(128, 4) WQ_APPEND(64, 16) WQ_APPEND(64, 8) WQ_APPEND(64, 4)
#undef WQ_APPEND
  return cudaErrorInvalidValue;
}

cudaError_t launch_kv_read(const KvReadArgs &a, int hd, int bits, bool f32, cudaStream_t s) {
  const unsigned grid = row_ctas(2ll * a.batch * a.n_kv * a.n, hd);
#define WQ_READ(HD, BITS)                                                               \
  if (hd == HD && bits == BITS)                                                         \
    return f32 ? launch_pdl(kv_read_kernel<HD, BITS, true>, a, grid, kKvThreads, s)     \
               : launch_pdl(kv_read_kernel<HD, BITS, false>, a, grid, kKvThreads, s);
  WQ_READ(128, 16) WQ_READ(128, 8) WQ_READ(128, 4) WQ_READ(64, 16) WQ_READ(64, 8) WQ_READ(64, 4)
#undef WQ_READ
  return cudaErrorInvalidValue;
}

cudaError_t launch_qkv_rope(const QkvRopeArgs &a, int m, int hd, cudaStream_t s) {
  if (hd == 128) return launch_pdl(qkv_rope_kernel<128>, a, (unsigned)m, kRopeThreads, s);
  if (hd == 64) return launch_pdl(qkv_rope_kernel<64>, a, (unsigned)m, kRopeThreads, s);
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
