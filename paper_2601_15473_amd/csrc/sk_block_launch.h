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

}  // namespace sk
