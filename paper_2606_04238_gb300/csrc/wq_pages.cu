// wq_pages.cu -- the pages of a KV cache (sm_103a): the plan of a step of a continuous
// batch (which pages each request takes and gives back, where its tokens go), projections
// normed, rotated and written to the slots of their tokens, and rows read back by slot.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "wq_cvt.cuh"
#include "wq_internal.h"
#include "wq_paged.h"
#include "wq_ptx.cuh"
#include "wq_rows.cuh"

namespace wq {

namespace cg = cooperative_groups;

// Status word of these kernels: WQ_OK (0), or WQ_ERR_ARG (-1) after a length, count, page,
// position or slot outside its range was met (what it names is skipped).
__device__ int g_pages_status = 0;

namespace {

constexpr int kPlanThreads = 512, kPutThreads = 128;
constexpr int kPagedReadThreads = 256;

struct Sums {
  int tokens, want, back;
};

// The first of n ascending sums that is above x (n: none).
__device__ __forceinline__ int above(const int *sums, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (sums[mid] > x)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

// Inclusive sums over the CTA's threads, on top of `carry`, which becomes the total.  (All
// the tables' entries are fewer than 2^31: host check.)
__device__ __forceinline__ int scan(int v, int *warps, int &carry) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += up;
  }
  __syncthreads();  // the sums of the scan before have been read
  if (lane == 31) warps[warp] = v;
  __syncthreads();
  int before = carry, total = carry;
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    before += w < warp ? warps[w] : 0;
    total += warps[w];
  }
  carry = total;
  return v + before;
}

}  // namespace

// One step's plan.  With have = ceil(lens / page) and need = ceil((keep + n_new) / page), a
// request gives back its pages need .. have - 1 or takes need - have more.  Pages given
// back go on the stack of free pages in request order, then pages are taken from its top in
// request order: both places are sums over the requests before, so nothing depends on the
// order of threads and no atomics are needed.
//   Every CTA of the cluster takes the same sums over all requests (at most 2048, a few
// shuffles each), then a share of the rows, of the pages taken and of those given back.  No
// entry is read that another CTA writes: a request either takes or gives, only entries from
// `have` on are written, and the stack is written above n_free and read below it.  The
// cluster's barrier stands between the reads of lens and n_free and the writes of kv_lens
// and n_free_out, which may be the same arrays.
//   Bound by latency, not by its few kB: 32 requests of a token each take 4.1 us from launch
// to launch, 256 requests with 20 new prompts among them 7.0.
__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PagePlanArgs a) {
  extern __shared__ int plan_smem[];
  __shared__ int warps[kPlanThreads / 32];
  int *const s_end = plan_smem, *const s_want = s_end + a.batch, *const s_back = s_want + a.batch,
            *const s_have = s_back + a.batch, *const s_keep = s_have + a.batch;
  cg::cluster_group cl = cg::this_cluster();
  pdl_wait();
  pdl_launch_dependents();
  const int page = 1 << a.shift, most = a.max_pages << a.shift;  // below 2^31 (host check)
  const int tid = threadIdx.x;
  bool bad = false;
  const int nf_in = *a.n_free, nf = min(max(nf_in, 0), a.n_pages);
  bad |= nf != nf_in;
  int tokens = 0, wants = 0, backs = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kPlanThreads) {
    const int b = b0 + tid;
    const bool in = b < a.batch;
    const int len = in ? a.lens[b] : 0, keep = in && a.keep ? a.keep[b] : len, n = in ? a.n_new[b] : 0;
    const bool valid = len >= 0 && len <= most && keep >= 0 && keep <= len && n >= 0 && (long long)keep + n <= most;
    const int end = scan(min(max(n, 0), a.m + 1), warps, tokens);
    const bool fits = valid && (end <= a.m || n == 0);
    bad |= in && !fits;
    const int have = (len + page - 1) >> a.shift, need = (keep + n + page - 1) >> a.shift;
    const int want = scan(fits ? max(need - have, 0) : 0, warps, wants);
    const int back = scan(fits ? max(have - need, 0) : 0, warps, backs);
    if (in) {
      s_end[b] = end;
      s_want[b] = want;
      s_back[b] = back;
      s_have[b] = fits ? have : -1;
      s_keep[b] = keep;
    }
  }
  // (more pages than there are: some were given back twice)
  bad |= backs > a.n_pages - nf;
  backs = min(backs, a.n_pages - nf);
  const int top = nf + backs;
  __syncthreads();
  // served: all, but for requests that want pages where they and those before them want more than there are
  const int last = above(s_want, a.batch, top);  // the first that is not served for want of pages
  const int taken = last > 0 ? s_want[last - 1] : 0;
  auto served = [&](int b) {
    if (s_have[b] < 0) return false;
    return b < last || s_want[b] == (b > 0 ? s_want[b - 1] : 0);
  };
  // page i given back
  auto given = [&](int i) {
    const int b = above(s_back, a.batch, i), first = b > 0 ? s_back[b - 1] : 0;
    return a.tables[(size_t)b * a.max_pages + s_have[b] - (s_back[b] - first) + i - first];
  };
  // page i taken
  auto pop = [&](int i) {
    const int at = top - 1 - i;
    return at >= nf ? given(at - nf) : a.free_pages[at];
  };
  cl.sync();
  const int gid = (int)cl.block_rank() * kPlanThreads + tid, step = (int)cl.num_blocks() * kPlanThreads;
  if (gid == 0) *a.n_free_out = top - taken;
  for (int b = gid; b < a.batch; b += step) {
    const int first = b > 0 ? s_end[b - 1] : 0;
    if (b == 0) a.cu[0] = 0;
    a.cu[b + 1] = min(s_end[b], a.m);
    a.kv_lens[b] = served(b) ? s_keep[b] + s_end[b] - first : -1;
  }
  for (int j = gid; j < a.m; j += step) {
    const int b = above(s_end, a.batch, j);
    int pos = 0, slot = -1;
    if (b < a.batch && served(b)) {
      pos = s_keep[b] + j - (b > 0 ? s_end[b - 1] : 0);
      const int p = pos >> a.shift;
      const int id = p < s_have[b] ? a.tables[(size_t)b * a.max_pages + p] : pop((b > 0 ? s_want[b - 1] : 0) + p - s_have[b]);
      if (id >= 0 && id < a.n_pages)
        slot = (id << a.shift) + (pos & (page - 1));
      else
        bad = true;
    }
    a.positions[j] = pos;
    a.slots[j] = slot;
  }
  for (int i = gid; i < taken; i += step) {
    const int b = above(s_want, a.batch, i);
    a.tables[(size_t)b * a.max_pages + s_have[b] + i - (b > 0 ? s_want[b - 1] : 0)] = pop(i);
  }
  for (int i = gid; i < backs - taken; i += step) a.free_pages[nf + i] = given(i);
  if (bad) atomicExch(&g_pages_status, -1);
}

// Query, key and value rows of a token: all scaled by 1 / sqrt(mean(x^2) + eps) (x given),
// queries and keys normed per head, times the norm's weights, and rotated (value i with i +
// HD/2); queries rounded to bf16, K and V quantized to the token's slot from fp32.  Sums,
// products and roundings are separate and in one order (a row's squares: its halves, a
// lane's eight pairwise, the lanes pairwise), so that equal rows have equal codes.
//   A CTA takes a token.  HD / 16 lanes take a row, values 8 l .. and HD/2 + 8 l .., so that
// a value and the one it is rotated with are one lane's.  Bound by instructions and loads in
// flight together: 4093 tokens of 40 + 16 bf16 heads of 128 to 4 bits take 26.7 us, 3.9 TB/s
// (one value an instruction and without the next heads on their way 37); 16 tokens 4.0, a
// launch's latency.
template <int HD, int BITS, bool F32>
__global__ void __launch_bounds__(kPutThreads, F32 && BITS != 16 ? 4 : 5) qkv_paged_kernel(const QkvPagedArgs a) {
  constexpr int THREADS = kPutThreads, LPR = HD / 16, GROUPS = THREADS / LPR, U = 2;  // lanes a row, rows a pass, passes in flight
  __shared__ float red[THREADS / 32];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid % LPR, grp = tid / LPR;
  const int heads = a.n_heads + 2 * a.n_kv, passes = (heads + GROUPS - 1) / GROUPS;
  const size_t tok = blockIdx.x;
  const int pos = a.positions ? a.positions[tok] : 0, slot = a.slots[tok];
  uint4 raw[U][F32 ? 4 : 2];
  auto fetch = [&](int pass, uint4 (&r)[F32 ? 4 : 2]) {
    const int h = pass * GROUPS + grp;
    if (h >= heads) return;
    const size_t at = (tok * heads + h) * HD + 8 * lane;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (F32) {
        const uint4 *p = reinterpret_cast<const uint4 *>(reinterpret_cast<const float *>(a.qkv) + at + i * (HD / 2));
        r[2 * i] = __ldcs(p), r[2 * i + 1] = __ldcs(p + 1);
      } else {
        r[i] = __ldcs(reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(a.qkv) + at + i * (HD / 2)));
      }
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u) fetch(u, raw[u]);
  const bool bad = a.positions && (pos < 0 || pos >= a.n_pos), out = slot < -1 || (slot >> a.shift) >= a.n_pages;
  if (bad || out) {
    if (tid == 0) atomicExch(&g_pages_status, -1);
    if (bad && !a.bad_zeros) return;
  }
  const bool put = slot >= 0 && !out;
  // (two values an instruction; each of its operations is rounded as by itself)
  uint64_t co[4], si[4];  // of the lane's eight angles
  if (a.positions) {
    const float4 *tab = reinterpret_cast<const float4 *>(a.table + ((size_t)(bad ? 0 : pos) * (HD / 2) + 8 * lane) * 2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 t = __ldg(tab + e);
      co[e] = pack_f32x2(t.x, t.z), si[e] = pack_f32x2(t.y, t.w);
    }
  }
  uint64_t rs = 0;
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
    const float r = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fdiv_rn(tot, (float)a.d), kRmsEps)));
    rs = bad ? 0 : pack_f32x2(r, r);  // (x may hold anything there)
  }
  auto work = [&](int pass, uint4 (&r)[F32 ? 4 : 2]) {
    const int h = pass * GROUPS + grp;
    const bool in = h < heads, is_q = h < a.n_heads, turns = h < a.n_heads + a.n_kv, has = in && !bad;
    uint64_t w[8];  // values 8 l .., then HD/2 + 8 l ..
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[2 * i] = has ? (uint64_t)r[i].y << 32 | r[i].x : 0, w[2 * i + 1] = has ? (uint64_t)r[i].w << 32 | r[i].z : 0;
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t x[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * i + e] = has ? pack_f32x2(bf_lo(x[e]), bf_hi(x[e])) : 0;
      }
    }
    fetch(pass + U, r);
    if (a.x)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = mul_f32x2(w[e], rs);
    // heads of a warp's rows ascend: whether any of them is Q or K, or K or V, is known to all its lanes
    if (a.head_norm && __any_sync(0xffffffffu, in && turns)) {
      uint64_t sq[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) sq[e] = add_f32x2(mul_f32x2(w[e], w[e]), mul_f32x2(w[4 + e], w[4 + e]));
      float s, s1;
      unpack_f32x2(add_f32x2(add_f32x2(sq[0], sq[2]), add_f32x2(sq[1], sq[3])), s, s1);
      s = __fadd_rn(s, s1);
#pragma unroll
      for (int o = LPR / 2; o >= 1; o >>= 1) s = __fadd_rn(s, __shfl_xor_sync(0xffffffffu, s, o));
      const float hn = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fmul_rn(s, 1.f / HD), kRmsEps)));
      if (turns) {
        const void *norm = is_q ? a.q_norm : a.k_norm;
        const uint64_t hn2 = pack_f32x2(hn, hn);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = mul_f32x2(w[e], hn2);
        if (norm) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4 g = __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(norm) + i * (HD / 2) + 8 * lane));
            const uint32_t x[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) w[4 * i + e] = mul_f32x2(w[4 * i + e], pack_f32x2(bf_lo(x[e]), bf_hi(x[e])));
          }
        }
      }
    }
    if (turns && a.positions) {
      const uint64_t minus = pack_f32x2(-1.f, -1.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint64_t lo = w[e], hi = w[4 + e];
        w[e] = fma_f32x2(mul_f32x2(hi, si[e]), minus, mul_f32x2(lo, co[e]));  // (the product with -1 is exact)
        w[4 + e] = add_f32x2(mul_f32x2(hi, co[e]), mul_f32x2(lo, si[e]));
      }
    }
    float v[16];
#pragma unroll
    for (int e = 0; e < 8; ++e) unpack_f32x2(w[e], v[2 * e], v[2 * e + 1]);
    auto rounded = [&](int i) {
      return make_uint4(pack_bf2(v[8 * i], v[8 * i + 1]), pack_bf2(v[8 * i + 2], v[8 * i + 3]), pack_bf2(v[8 * i + 4], v[8 * i + 5]),
                        pack_bf2(v[8 * i + 6], v[8 * i + 7]));
    };
    if (in && is_q) {
      __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(a.q) + (tok * a.n_heads + h) * HD + 8 * lane;
      *reinterpret_cast<uint4 *>(dst) = rounded(0);
      *reinterpret_cast<uint4 *>(dst + HD / 2) = rounded(1);
    }
    if (!put || __all_sync(0xffffffffu, is_q || !in)) return;
    const int g = turns ? h - a.n_heads : h - a.n_heads - a.n_kv;
    const bool mine = in && !is_q;
    const size_t row = mine ? (((size_t)(slot >> a.shift) * a.n_kv + g) << a.shift) + (slot & ((1 << a.shift) - 1)) : 0;
    uint8_t *dst = reinterpret_cast<uint8_t *>(turns ? a.kc : a.vc) + row * (HD * BITS / 8) + lane * BITS;
    if constexpr (BITS == 16) {
      if (!mine) return;
      *reinterpret_cast<uint4 *>(dst) = rounded(0);
      *reinterpret_cast<uint4 *>(dst + HD) = rounded(1);
    } else {
      float mn = 0.f, mx = 0.f;
      bool nan = false;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        mn = fminf(mn, v[e]);
        mx = fmaxf(mx, v[e]);
        nan |= v[e] != v[e];
      }
      if (nan) mx = __int_as_float(0x7fffffff);
#pragma unroll
      for (int o = LPR / 2; o >= 1; o >>= 1) {
        const float x = __shfl_xor_sync(0xffffffffu, mn, o), y = __shfl_xor_sync(0xffffffffu, mx, o);
        mn = fminf(mn, x);
        mx = y > mx || y != y ? y : mx;
      }
      uint32_t c[8], p[BITS / 2];
      const uint32_t meta = quantize16<BITS>(v, mn, mx, c);
      if (!mine) return;
      pack_codes<BITS>(c, p);
      if constexpr (BITS == 8) {
        *reinterpret_cast<uint2 *>(dst) = make_uint2(p[0], p[1]);
        *reinterpret_cast<uint2 *>(dst + HD / 2) = make_uint2(p[2], p[3]);
      } else {
        *reinterpret_cast<uint32_t *>(dst) = p[0];
        *reinterpret_cast<uint32_t *>(dst + HD / 4) = p[1];
      }
      if (lane == 0) (turns ? a.km : a.vm)[row] = meta;
    }
  };
  for (int pass = 0; pass < passes; pass += U) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (pass + u < passes) work(pass + u, raw[u]);  // uniform in the CTA
  }
}

// Rows at the slots, zeros where a slot is -1.  Place i of the launch: token and head, K's
// before V's.  Bound by memory: 20,000 tokens of 8 heads of 128 from 4 bits to bf16 take
// 18.8 us, 104 MB at 5.5 TB/s.
template <int HD, int BITS, bool F32>
__global__ void __launch_bounds__(kPagedReadThreads) paged_read_kernel(const PagedReadArgs a, const Divisor by_kv) {
  constexpr int LPR = HD / 16;
  pdl_wait();
  pdl_launch_dependents();
  const unsigned at = blockIdx.x * (kPagedReadThreads / LPR) + threadIdx.x / LPR;
  const int lane = threadIdx.x % LPR;
  const unsigned per_cache = (unsigned)a.m * a.n_kv;  // below 2^30 (host check)
  if (at >= 2 * per_cache) return;
  const bool is_v = at >= per_cache;
  const unsigned rest = is_v ? at - per_cache : at;
  const unsigned t = by_kv.divide(rest);
  const int g = (int)(rest - t * (unsigned)a.n_kv), slot = a.slots[t];
  if (slot < -1 || (slot >> a.shift) >= a.n_pages) {
    if (lane == 0) atomicExch(&g_pages_status, -1);
    return;
  }
  const size_t row = slot < 0 ? 0 : (((size_t)(slot >> a.shift) * a.n_kv + g) << a.shift) + (slot & ((1 << a.shift) - 1));
  read_row<HD, BITS, F32>(is_v ? a.vc : a.kc, is_v ? a.vm : a.km, row, lane, slot >= 0, is_v ? a.v : a.k, (size_t)rest * HD);
}

cudaError_t launch_page_plan(const PagePlanArgs &a, cudaStream_t s) {
  // CTAs of a cluster: 2 rows a thread, and at most the 8 that every cluster may have
  const int ctas = std::min(8, std::max(1, (a.m + 2 * kPlanThreads - 1) / (2 * kPlanThreads)));
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.dynamicSmemBytes = sizeof(int) * 5 * (size_t)a.batch;
  return cudaLaunchKernelEx(&cfg, page_plan_kernel, a);
}

cudaError_t launch_qkv_paged(const QkvPagedArgs &a, int m, int hd, int bits, bool f32, cudaStream_t s) {
#define WQ_PAGED(HD, BITS)                                                              \
  if (hd == HD && bits == BITS)                                                         \
    return f32 ? launch_pdl(qkv_paged_kernel<HD, BITS, true>, (unsigned)m, kPutThreads, s, a)   \
               : launch_pdl(qkv_paged_kernel<HD, BITS, false>, (unsigned)m, kPutThreads, s, a);
  WQ_PAGED(128, 16) WQ_PAGED(128, 8) WQ_PAGED(128, 4) WQ_PAGED(64, 16) WQ_PAGED(64, 8) WQ_PAGED(64, 4)
#undef WQ_PAGED
  return cudaErrorInvalidValue;
}

cudaError_t launch_paged_read(const PagedReadArgs &a, int hd, int bits, bool f32, cudaStream_t s) {
  const unsigned grid = row_ctas(2ll * a.m * a.n_kv, hd, kPagedReadThreads);
#define WQ_READ(HD, BITS)                                                                                           \
  if (hd == HD && bits == BITS)                                                                                     \
    return f32 ? launch_pdl(paged_read_kernel<HD, BITS, true>, grid, kPagedReadThreads, s, a, Divisor(a.n_kv))      \
               : launch_pdl(paged_read_kernel<HD, BITS, false>, grid, kPagedReadThreads, s, a, Divisor(a.n_kv));
  WQ_READ(128, 16) WQ_READ(128, 8) WQ_READ(128, 4) WQ_READ(64, 16) WQ_READ(64, 8) WQ_READ(64, 4)
#undef WQ_READ
  return cudaErrorInvalidValue;
}

cudaError_t read_pages_status(int *status) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(status, g_pages_status, sizeof(int));
  if (e != cudaSuccess) return e;
  const int zero = 0;
  return cudaMemcpyToSymbol(g_pages_status, &zero, sizeof(int));
}

}  // namespace wq
