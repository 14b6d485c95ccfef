// wq_kv.h -- launchers of the KV-cache operators (wq_kv.cu) and of attention
// over a tree of drafted tokens (wq_tree.cu).  Arguments have been validated by
// the C ABI; every launcher returns the launch status.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace wq {

// Scale and zero of a cached row of zeros: 1 and -0 (the zero point of any other row is +0 or above).  Attention takes such
// a V row, like one of a zero-filled cache (scale 0), for one of the least scale: its codes are its zero point, so any
// scale gives its values, and 1 would make small rows beside it look small.
constexpr uint32_t kZeroRow = 0x80003c00u;
constexpr float kLeastScale = 0x1p-24f;  // of binary16, bits 0x0001

// Rows k, v [batch][n_src][n_kv][HD] (strides in values: sequence, token, head)
// into the caches [batch][n_kv][max_len][HD] at start[b] + n, n < counts[b]
// (null: n), row n taken from token index[b][n] (null: n).
struct KvAppendArgs {
  const void *k, *v;
  long long k_stride[3], v_stride[3];
  void *kc, *vc;
  uint32_t *km, *vm;
  const int *start, *counts, *index;
  int batch, n_kv, max_len, n_src, n;
};
cudaError_t launch_kv_append(const KvAppendArgs &a, int hd, int bits, bool f32, cudaStream_t s);

// Positions start[b] .. start[b] + n - 1 of the caches as rows [batch][n][n_kv][HD],
// zeros from counts[b] (null: n) on.
struct KvReadArgs {
  const void *kc, *vc;
  const uint32_t *km, *vm;
  void *k, *v;
  const int *start, *counts;
  int batch, n_kv, max_len, n;
};
cudaError_t launch_kv_read(const KvReadArgs &a, int hd, int bits, bool f32, cudaStream_t s);

struct QkvRopeArgs {
  const float *qkv;   // [m][(n_heads + 2 n_kv) HD]
  const void *x;      // bf16 [m][d] or null
  const int *positions;
  const float *table;  // [n_pos][HD / 2][2]
  void *q, *k, *v;
  int d, n_heads, n_kv, n_pos, head_norm;
};
cudaError_t launch_qkv_rope(const QkvRopeArgs &a, int m, int hd, int num_sms, cudaStream_t s);
// Reads and clears the status word of the three kernels above.
cudaError_t read_kv_status(int *status);

struct TreeArgs {
  const void *q;                // bf16 [batch][T][H][HD]
  const void *kn, *vn;          // bf16 [batch][T][Hkv][HD]
  const void *kc, *vc;          // caches
  const uint32_t *km, *vm;      // scales and zeros of cached rows (8 and 4 bits)
  const int *lens, *counts;     // [batch]; counts null: T
  const uint32_t *mask;         // [batch][T][words] or null: each draft sees itself and the earlier ones
  int batch, T, H, Hkv, max_len, words;
  float scale;                  // of the scores, times log2(e)
  float *part;                  // [batch Hkv][rows][S][HD + 2] (S > 1)
  void *o;                      // bf16 [batch][T][H][HD]
  int S, cluster;               // splits of the context; whether they are a cluster
  // tcgen05 kernel: ranges of tiles wanted, whether row blocks may be split (only then the merge is
  // launched), rows of a range's partial results, and per sequence its first range, splits, row
  // blocks and drafts; after the sequences whether any was split (.x)
  int target, split, part_rows, rep_magic;
  int4 *table;
};
// Splits of the context a launch takes, and its partial results in floats.
int tree_splits(int batch, int T, int H, int Hkv, int max_len, int num_sms);
bool tree_cluster(int batch, int T, int H, int Hkv, int S, int num_sms);
size_t tree_part_floats(int batch, int T, int H, int Hkv, int hd, int max_len, int num_sms);
cudaError_t launch_attn_tree(const TreeArgs &a, int hd, int bits, cudaStream_t s);
cudaError_t read_tree_status(int *status);
// The same on the tcgen05 tensor cores (wq_tree_tc.cu); part: [range][part_rows][HD + 4].
size_t tree_tc_part_floats(int batch, int T, int H, int Hkv, int hd, int max_len, int num_sms);
cudaError_t launch_attn_tree_tc(TreeArgs a, int hd, int bits, int num_sms, cudaStream_t s);
cudaError_t read_tree_tc_status(int *status);

}  // namespace wq
