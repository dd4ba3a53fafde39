// Host-side launchers of the block operators' kernels (internal; the public ABI is include/sk_block.h).
#pragma once
#include "sk_launch.h"

namespace sk {

// A HIP error under the calling thread's sk_last_hip_error (sk_api.hip).
void note_hip_error(hipError_t e, const char* what);

// Arguments of the attention kernels.  Rows of o, dO and dq are dense [batch, q_len, heads, D], lse and the like
// [batch, heads, q_len], dk and dv dense [batch, k_len, kv_heads, D].
struct AttentionArgs {
  const void *q, *k, *v, *d_o;
  const void* o_in;             // backward: the forward pass's result
  void *o, *dq, *dk, *dv;
  float* lse;                   // forward: written unless null; backward: read
  void* o_rest;                 // bf16: what o's rounding left off, or null; as lse
  float *lse2, *delta;          // backward: lse log2(e) and -sum_d dO o of every row, left by dq's kernel for dk's and dv's
  const int32_t *q_lengths, *k_lengths;
  int64_t qs[3], ks[3], vs[3];  // batch, token, head strides in elements
  int batch, q_len, k_len, heads, kv_heads, group, D;
  int causal;
  float scale;
  void* workspace;              // forward
  // backward: parts that dk and dv are summed in, and room for [parts][dk, dv] in fp32 where there are several
  int parts;
  float* partial;
  // ... shares of the keys that dq is summed in (bf16), and room for [shares][dq]
  int q_shares;
  float* q_partial;
};
int attention_parts(const AttentionArgs& a, bool f32);
int attention_query_shares(const AttentionArgs& a);
// Sums up what is in parts (nothing where nothing is).
hipError_t launch_attention_sum_parts(const AttentionArgs& a, bool f32, hipStream_t s);

size_t attention_fwd_bytes_bf16(const AttentionArgs& a);
hipError_t launch_attention_fwd(const AttentionArgs& a, bool f32, hipStream_t s);
// dq and delta, then dk and dv
hipError_t launch_attention_bwd(const AttentionArgs& a, bool f32, hipStream_t s);

hipError_t launch_attention_fwd_bf16(const AttentionArgs& a, hipStream_t s);
hipError_t launch_attention_bwd_bf16(const AttentionArgs& a, hipStream_t s);

struct NormRopeArgs {
  const void *q, *k, *wq, *wk;
  const float *cos, *sin;
  const void* positions;
  void *q_out, *k_out;                    // forward: the results; backward: dq, dk
  const void *dq_out, *dk_out;            // backward
  float* partial;                         // backward: [groups][2][D] sums of dwq, dwk
  void *dwq, *dwk;
  int64_t qs[2], ks[2], qos[2], kos[2];
  int64_t tokens, table_rows;
  int heads, kv_heads, D, rotary, interleaved, pos64;
  float eps;
};
constexpr int NORM_ROPE_MAX_GROUPS = 1024;
hipError_t launch_norm_rope_fwd(const NormRopeArgs& a, bool f32, hipStream_t s);
hipError_t launch_norm_rope_bwd(const NormRopeArgs& a, bool f32, hipStream_t s);

struct EmbeddingArgs {
  const void* ids;
  const void* table;     // forward
  const void* dy;        // backward
  void* out;             // y, or dtable
  int64_t tokens, rows;
  int width, ids64;
  int run;               // backward: tokens of a sorted run
  float scale;
  // backward: the tokens sorted by id (stable), and the fp32 sums of runs that are cut
  unsigned *keys, *order, *keys_runs, *order_runs;
  float* partial;        // [chunks][2][width]
};
constexpr int EMBEDDING_RUN = 16384;   // tokens one work-group sorts at most
// Sorted tokens summed at a stretch (backward): 32 where that gives two waves a SIMD, else 16.  The whole backward pass with 32 and with 16: 4001 tokens of 768
// features in f32 31.7 and 28.1 us, 8192 of them 40.2 and 37.9; in bf16 16384 of 1024 features 46.2 and 43.9, 32768 (the line) 59.5 and 60.3, 16384 of 4096 153.9 and 159.3.
inline int embedding_chunk(int64_t tokens, int64_t width, int esize) {
  return (tokens + 31) / 32 * ((width * esize / 16 + 63) / 64) >= 8 * NUM_CUS ? 32 : 16;
}
// Tokens of a sorted run: all that fit one work-group's LDS where the gradient's fill, in the same launch, takes longer than their sort (16384 take 30
// us, at 6.7 TB/s as long as 200 MB), or there are many runs to put in order, else 4096 (10 us) and a launch that orders up to eight runs (8 us).
inline int embedding_run(int64_t tokens, int64_t rows, int64_t width, int esize) {
  return tokens <= 8192 || tokens > 8 * 4096 || rows * width * esize >= (int64_t)128 << 20 ? EMBEDDING_RUN : 4096;
}
hipError_t launch_embedding_fwd(const EmbeddingArgs& a, bool f32, hipStream_t s);
hipError_t launch_embedding_bwd(const EmbeddingArgs& a, bool f32, hipStream_t s);

struct DropoutArgs {
  const void *x, *residual;
  void* y;
  int64_t n;
  unsigned drop;         // of 65536 words, those below it
  float scale;           // 65536 / (65536 - drop), 0 if that has no value
  unsigned key[2], offset[2];
};
hipError_t launch_dropout(const DropoutArgs& a, bool f32, hipStream_t s);

// Runs of rows that column sums are formed in: of groups of 512 columns about four work-groups to a CU, 16 rows at least.  (Two, three and eight: a dense layer's dz of
// 4096 x 4096 behind gelu 24.0, 20.8 and 19.2 us for 19.7, of 16384 x 11008 behind silu 265, 250 and 252 for 257; the sums' launch level.)
struct ColumnRuns {
  int groups, runs, rows;   // rows of a run
  ColumnRuns(int64_t of_rows, int64_t columns) {
    groups = (int)((columns + 511) / 512);
    const int64_t wanted = (4 * NUM_CUS + groups - 1) / groups, most = (of_rows + 15) / 16;
    const int64_t n = wanted < most ? wanted : most;
    rows = (int)(((of_rows + n - 1) / n + 15) / 16 * 16);
    runs = (int)((of_rows + rows - 1) / rows);
  }
};

struct LayerNormArgs {
  const void *x, *residual, *weight, *bias;   // forward: x and the residual (or null); backward: x is what was normed
  void *y, *s;                                // forward: the result, and the sum (or null)
  unsigned* rest;                             // [rows][width / 8] what a bf16 sum's rounding left off, or null: forward written, backward read
  float* stats;                               // [rows][mean, 1 / deviation]: forward written unless null, backward read
  const void *dy, *ds;                        // backward; ds or null
  void *dx, *dweight, *dbias;                 // backward; weights' or null
  float* partial;                             // backward: [groups][dweight, dbias][width], null where neither is wanted
  int64_t rows, x_stride, residual_stride;
  int width;
  float eps;
};
// Lanes to a row: eight values a lane and piece, a row on part of a wave, a work-group's four, or sixteen waves.
inline int layer_norm_lanes(int width) {
  const int pieces = width / 8;
  return pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 32 ? 32 : pieces <= 128 ? 64 : pieces <= 1024 ? 256 : 1024;
}
// Work-groups of the backward pass, each of which leaves a row of partial sums: two to a CU (16383 x 4096 with a residual, 256 : 512 : 1024 of them, 141 : 113 : 112 us and 5 : 5 : 8
// for their sum), but where a row is a work-group's not below eight rows each, down to one to a CU (2048 x 8192 33 + 4 : 39 + 7 : 51 + 12, 500 x 2048 6.5 + 3.0 : 8.0 + 5.0).
inline int layer_norm_groups(int64_t rows, int width) {
  const int lanes = layer_norm_lanes(width), together = lanes < 256 ? 256 / lanes : 1;
  if (lanes > 256) return ColumnRuns(rows, width).runs;   // (a launch of its own)
  const int64_t groups = (rows + together - 1) / together;
  int64_t most = 2 * NUM_CUS;
  if (together == 1 && rows / 8 < most) most = rows / 8 < NUM_CUS ? NUM_CUS : rows / 8;
  return (int)(groups < most ? groups : most);
}
constexpr int LAYER_NORM_MAX_WIDTH = 1 << 15;   // a row on one work-group's registers
hipError_t launch_layer_norm_fwd(const LayerNormArgs& a, bool f32, hipStream_t s);
hipError_t launch_layer_norm_bwd(const LayerNormArgs& a, bool f32, hipStream_t s);

constexpr int DISTILL_STATS = 8;
struct DistillArgs {
  const void *logits, *teacher;               // rows logits_stride elements apart, [rows][top] dense
  const void *ids, *labels;                   // labels or null
  float* loss;                                // forward
  // [rows][DISTILL_STATS], forward written unless null, backward read: the largest logit, 1 / sum exp((z - it) / temperature), 1 / sum exp(z - it); the teacher's
  // largest, 1 / sum exp((t - it) / temperature) or 0 where there is no entry
  float* stats;
  const float* dloss;                         // backward
  void* dlogits;                              // backward: dense
  int64_t rows, logits_stride;
  int vocabulary, top, ids64, labels64;
  float temperature, label_weight;
};
hipError_t launch_distill_fwd(const DistillArgs& a, bool f32, hipStream_t s);
hipError_t launch_distill_bwd(const DistillArgs& a, bool f32, hipStream_t s);

struct DenseArgs {
  const void *x, *weight, *bias, *residual;   // bias and residual or null
  void *y, *z;                                // z: what goes into the activation, dense; forward written unless null, backward read
  const void* dy;                             // backward
  void *dz, *dx, *dweight, *dbias;            // backward; dz: room for it where there is an activation; the others or null
  const float* slabs;                         // forward: the product in fp32 slabs [splits][tokens, out]
  int splits;
  float* partial;                             // backward: [runs][out] sums of dz, null where dbias is not wanted
  int64_t x_stride, residual_stride;
  int tokens, in, out, activation;
};
hipError_t launch_dense_finish(const DenseArgs& a, bool f32, hipStream_t s);
hipError_t launch_dense_dz(const DenseArgs& a, bool f32, hipStream_t s);
hipError_t launch_dense_dbias(const DenseArgs& a, bool f32, hipStream_t s);

}  // namespace sk
