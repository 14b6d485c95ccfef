// wq_paged.h -- launchers of the operators of a paged KV cache: step plans, rows written to
// and read from pages (wq_pages.cu), attention over pages (wq_attn_paged.cu).
// Arguments have been validated by the C ABI; every launcher returns the launch status.
//
// A pool of pages is a cache [n_pages][n_kv][page][HD], page a power of two: position
// `slot` of it is place slot % page of page slot / page.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace wq {

constexpr int kMaxRequests = 2048;     // of a step plan
constexpr int kMaxPlanRows = 1 << 18;  // query rows of a step plan

struct PagePlanArgs {
  const int *lens, *keep, *n_new;  // [batch]; keep null: lens
  int *tables, *free_pages;        // [batch][max_pages], [n_pages]
  const int *n_free;
  int *n_free_out;
  int batch, shift, max_pages, n_pages, m;  // page = 1 << shift
  int *cu, *kv_lens, *positions, *slots;
};
cudaError_t launch_page_plan(const PagePlanArgs &a, cudaStream_t s);

struct QkvPagedArgs {
  const void *qkv;       // fp32 or bf16 [m][(n_heads + 2 n_kv) HD]
  const void *x;         // bf16 [m][d] or null
  const int *positions;  // [m] or null: no rotation
  const float *table;    // [n_pos][HD / 2][2]
  const void *q_norm, *k_norm;  // bf16 [HD] or null: ones
  const int *slots;
  void *kc, *vc;
  uint32_t *km, *vm;
  void *q;  // bf16 [m][n_heads][HD]
  int d, n_heads, n_kv, n_pos, head_norm, n_pages, shift;
  int bad_zeros;  // rows of a token whose position is not in the table: 1 zeros, 0 not written
};
cudaError_t launch_qkv_paged(const QkvPagedArgs &a, int m, int hd, int bits, bool f32, cudaStream_t s);

struct PagedReadArgs {
  const void *kc, *vc;
  const uint32_t *km, *vm;
  const int *slots;
  void *k, *v;  // [m][n_kv][HD]
  int m, n_kv, n_pages, shift;
};
cudaError_t launch_paged_read(const PagedReadArgs &a, int hd, int bits, bool f32, cudaStream_t s);
// Reads and clears the status word of the three kernels above.
cudaError_t read_pages_status(int *status);

struct AttnPagedArgs {
  const void *q;            // bf16 [m][H][HD]
  const void *kc, *vc;      // pages
  const uint32_t *km, *vm;  // scales and zeros of rows (8 and 4 bits)
  const int *cu, *kv_lens;  // [batch + 1], [batch]
  const int *tables;        // [batch][max_pages]
  int m, max_q, batch, H, Hkv, n_pages, shift, max_pages;
  int least_q, most_q;      // query rows of the sequences that the launch takes
  float scale;              // of the scores, times log2(e)
  float *part;              // [CTA][2][16][HD + 4]
  int *counters;            // [CTA], zero between calls
  void *o;                  // bf16 [m][H][HD]
};
// CTAs of a launch at most, and what they leave for one another in floats.
int attn_paged_ctas(int num_sms);
size_t attn_paged_part_floats(int hd, int num_sms);
cudaError_t launch_attn_paged(const AttnPagedArgs &a, int hd, int bits, int num_sms, cudaStream_t s);
cudaError_t read_attn_paged_status(int *status);
// The same on the tcgen05 tensor cores (wq_attn_paged_tc.cu); part: [CTA][2][256][HD + 4].
size_t attn_paged_tc_part_floats(int hd, int num_sms);
cudaError_t launch_attn_paged_tc(const AttnPagedArgs &a, int hd, int bits, int num_sms, cudaStream_t s);
cudaError_t read_attn_paged_tc_status(int *status);

}  // namespace wq
