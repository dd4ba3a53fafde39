/*
 * libsk -- the operators of a transformer block that stand between its sketched layers
 * (include/sk.h), on AMD MI355X (gfx950): attention, the norms and the position rotation of
 * queries and keys, the token embedding, dropout, layer norm, layers that stay dense, and the loss
 * against a teacher's largest logits; each with its gradients.
 *
 * Common rules (those of include/sk.h unless said otherwise)
 *   - Every pointer is a DEVICE pointer, 16-byte aligned.  Arrays are dense and row-major
 *     unless strides are given; strides count elements, are not negative and are whole
 *     multiples of 16 bytes.
 *   - `dtype` is the storage type of all floating arrays that are not declared float.  Sums,
 *     softmax statistics and norms are fp32; results are rounded to `dtype` once.
 *   - The caller owns every buffer, the workspace included.  The library allocates nothing,
 *     keeps no state between calls and never synchronises: all work is enqueued on `stream`.
 *     Outputs are overwritten in full, not accumulated into, and must not overlap inputs unless
 *     a function says that they may.
 *   - Sums are formed in a fixed order: results are bit-reproducible from run to run.
 *   - Arguments are checked before any HIP call; numbers in device memory (lengths, positions,
 *     token ids) cannot be, and out-of-range ones are given a meaning instead.
 */
#ifndef SK_BLOCK_H
#define SK_BLOCK_H

#include "sk.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Softmax attention of packed heads.
 *   q [batch, q_len, heads, head_dim], k and v [batch, k_len, kv_heads, head_dim], o as q.
 * Query head h reads key and value head h / (heads / kv_heads).  With n = q_lengths[b] queries
 * and m = k_lengths[b] keys of sequence b (all of them where the pointer is NULL; clamped to
 * 0 .. q_len and 0 .. k_len), query i < n sees key j < m, and with `causal` only
 * j - m <= i - n: the last query of a sequence stands at its last key.
 *     o_i = sum_j p_ij v_j,   p_ij = exp(s_ij - lse_i),   s_ij = scale * q_i . k_j,
 *     lse_i = log sum_j exp(s_ij)   over the keys that i sees.
 * A query that sees no key, and a row i >= n, has o = 0 and lse = -infinity.  What lies in keys
 * and values past m and in queries past n is not used, whatever it is.  (Of what counts for some
 * query, a value that is not finite may reach queries that see other keys but not its own, as zero times it.)
 * (Tokens of k or v that overlap in memory, a token stride below head_dim: what is not finite in the
 * last that counts may come out as NaN where it would be infinity.)
 *
 * Scores are fp32: from some 2^24 on they do not tell neighbours apart, and from 2^31 on weights may
 * overflow, and what is formed of them be NaN.
 *
 * Limits (else SK_ERR_UNSUPPORTED): head_dim a multiple of 8 up to 128, heads a multiple of
 * kv_heads, token strides and heads * head_dim up to 2^22, q_len * heads / kv_heads and k_len up to 2^27, and batch * kv_heads times the tiles of 128 rows of
 * either below 2^24.
 */
typedef struct {
  int64_t batch, q_len, k_len;
  int32_t heads, kv_heads, head_dim;
  int32_t causal;            /* 0 or 1 */
  float scale;               /* finite */
  sk_dtype dtype;
  /* Elements between two sequences, two tokens and two heads; the values of a head are consecutive.  (Strides of
     dimensions of size 1 are not looked at.) */
  int64_t q_strides[3], k_strides[3], v_strides[3];
  const int32_t* q_lengths;  /* [batch] device memory, or NULL */
  const int32_t* k_lengths;
} sk_attention_shape;

/* Bytes of workspace of the forward pass, and of the backward pass ((size_t)-1 for a shape that would be refused). */
size_t sk_attention_workspace_bytes(const sk_attention_shape* shape, int32_t backward);

/*
 * o [batch, q_len, heads, head_dim] dense.  For a backward pass: lse [batch, heads, q_len] dense or NULL, and in bf16 o_rest, as o, or
 * NULL: what rounding leaves off o, in bf16 (looked at in bf16 only).
 */
sk_status sk_attention_fwd(const sk_attention_shape* shape, const void* q, const void* k, const void* v, void* o, float* lse,
                           void* o_rest, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The exact derivative of the above, probabilities recomputed from q, k and lse:
 *     dv_j = sum_i p_ij do_i,  ds_ij = scale * p_ij (do_i . v_j - do_i . o_i),  dq_i = sum_j ds_ij k_j,  dk_j = sum_i ds_ij q_i
 * (dk and dv summed over the query heads that share them, too).  o, lse and o_rest are the forward pass's
 * (without o_rest, NULL, do_i . o_i is taken of the rounded o alone: in bf16 dq and dk are then off by a tenth more), d_o as o; dq, dk and dv dense, [batch, tokens, heads, head_dim] of their own.  Zeros for queries and
 * keys past their lengths.
 */
sk_status sk_attention_bwd(const sk_attention_shape* shape, const void* q, const void* k, const void* v, const void* o,
                           const float* lse, const void* o_rest, const void* d_o, void* dq, void* dk, void* dv,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * RMS norm of every query and key head, then the rotation of its first `rotary_dim` features by the
 * token's position:
 *     n = x * w / sqrt(mean(x^2) + eps),   (a, b) -> (a cos - b sin, b cos + a sin)
 * for the pairs (a, b) = n[i], n[i + rotary_dim / 2], or with `interleaved` n[2 i], n[2 i + 1], i < rotary_dim / 2,
 * with cos and sin of table row `position`, column i.
 *   q [tokens, heads, head_dim], k [tokens, kv_heads, head_dim] with strides (token, head);
 *   q_weight, k_weight [head_dim]; positions int32 [tokens] or int64 (position_bytes 4 or 8), clamped to
 *   0 .. table_rows - 1; cos, sin fp32 [table_rows, rotary_dim / 2].
 *   head_dim a multiple of 8 up to 256, rotary_dim a multiple of 8 from 0 (no table needed) to head_dim, strides up to 2^31,
 *   up to 2^25 tokens.
 * kv_heads may be 0 (no keys: k, k_weight and theirs are not looked at).
 */
typedef struct {
  int64_t tokens;
  int32_t heads, kv_heads, head_dim, rotary_dim;
  int32_t interleaved;       /* 0 or 1 */
  int32_t position_bytes;    /* 4 or 8 */
  int64_t table_rows;
  float eps;                 /* >= 0 */
  sk_dtype dtype;
  int64_t q_strides[2], k_strides[2];           /* of the inputs: token, head */
  int64_t q_out_strides[2], k_out_strides[2];   /* of the results (a cache's slots, say); the gradients are dense */
} sk_norm_rope_shape;

/* The results may be the inputs (same pointer and strides).  A result's rows must not lie on one another (SK_ERR_INVALID_ARG: a stride of 0, say). */
sk_status sk_norm_rope_fwd(const sk_norm_rope_shape* shape, const void* q, const void* k, const void* q_weight, const void* k_weight,
                           const float* cos, const float* sin, const void* positions, void* q_out, void* k_out, void* stream);

/*
 * Its gradients, from the inputs and the gradients of the results (dq_out [tokens, heads, head_dim] and dk_out dense):
 * dq, dk dense, dq_weight and dk_weight [head_dim] in `dtype`.  Workspace: sk_norm_rope_workspace_bytes.
 */
sk_status sk_norm_rope_bwd(const sk_norm_rope_shape* shape, const void* q, const void* k, const void* q_weight, const void* k_weight,
                           const float* cos, const float* sin, const void* positions, const void* dq_out, const void* dk_out,
                           void* dq, void* dk, void* dq_weight, void* dk_weight, void* workspace, size_t workspace_bytes, void* stream);
size_t sk_norm_rope_workspace_bytes(const sk_norm_rope_shape* shape);

/*
 * y[t] = scale * table[ids[t]]: ids int32 or int64 (id_bytes 4 or 8) [tokens], table [rows, width], y [tokens, width].
 * An id outside 0 .. rows - 1 gives a row of zeros, and no gradient.  width a multiple of 8 up to 2^20, rows < 2^31, tokens up
 * to 2^27 and tokens * width below 2^36.
 */
sk_status sk_embedding_fwd(const void* ids, int32_t id_bytes, const void* table, void* y, int64_t tokens, int64_t rows,
                           int64_t width, float scale, sk_dtype dtype, void* stream);

/*
 * dtable[v] = scale * sum over t with ids[t] = v of dy[t], in fp32, added up by sorted tokens (token order within a row,
 * in runs of a fixed length); rows without a token are zeros.  Workspace: sk_embedding_workspace_bytes.
 * (Made for a step's tokens: they are sorted in runs of up to 16384, each token's place among the other runs found by search, whose number grows with
 * the square of the tokens.)
 */
sk_status sk_embedding_bwd(const void* ids, int32_t id_bytes, const void* dy, void* dtable, int64_t tokens, int64_t rows,
                           int64_t width, float scale, sk_dtype dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t sk_embedding_workspace_bytes(int64_t tokens, int64_t rows, int64_t width, sk_dtype dtype);

/*
 * y[i] = (w_i >= d ? x[i] * 65536 / (65536 - d) : 0) (+ residual[i]), i < n, with d = p * 65536 to the nearest whole number (p in
 * 0 .. 1; the drop rate is a multiple of 2^-16, and the scale is that rate's) and w_i the i-th 16-bit word of a
 * counter-based generator: Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw 2011), key `seed`, counter
 * (i / 8, offset), both low word first, whose four results are eight words, low halves first.  No mask is stored: the gradient is
 * the same call on dy without a residual.  d = 65536: zeros (+ residual).  residual may be NULL; y may be x or
 * residual.  The calls of one training step take different offsets (or seeds).
 */
sk_status sk_dropout(const void* x, const void* residual, void* y, int64_t n, float p, uint64_t seed, uint64_t offset,
                     sk_dtype dtype, void* stream);

/*
 * Layer norm of rows, with a residual added first:
 *     s = x + residual,   y = (s - mean s) / sqrt(mean (s - mean s)^2 + eps) * weight + bias
 *   x and residual [rows, width] with row strides, weight and bias [width], y and sum (s) [rows, width] dense.  residual, weight, bias and
 * sum may be NULL.  For a backward pass, or NULL: stats [rows, 2] fp32, the mean and what the deviation is divided by, inverted; with a sum in bf16 also
 * sum_rest [rows, width / 8] 32-bit words, what its rounding left off: four bits a value, a word's from the lowest on, signed, in 16ths of a step of the type.
 * The gradients are those at the sum with it, or at the rounded sum without (dweight 0.0024 to 0.0027 off, where one rounding is 0.0017).
 * y is formed of s before its rounding.
 *   width a multiple of 8 up to 2^15, rows below 2^24 (2^22 from a width of 8200 on).
 */
typedef struct {
  int64_t rows, width;
  float eps;                 /* >= 0 */
  sk_dtype dtype;
  int64_t x_stride, residual_stride;   /* elements between rows */
} sk_layer_norm_shape;

sk_status sk_layer_norm_fwd(const sk_layer_norm_shape* shape, const void* x, const void* residual, const void* weight, const void* bias,
                            void* y, void* sum, void* sum_rest, float* stats, void* stream);

/*
 * Its gradients: x [rows, width] is what was normed (the sum, where there was a residual, and sum_rest or NULL), with row stride x_stride; dy and d_sum dense, d_sum the
 * gradient of the sum or NULL; dx (of x, and of the residual) dense, dweight and dbias in `dtype`, or NULL.  Workspace: sk_layer_norm_workspace_bytes,
 * needed for dweight and dbias.
 */
sk_status sk_layer_norm_bwd(const sk_layer_norm_shape* shape, const void* x, const void* sum_rest, const void* weight, const float* stats, const void* dy, const void* d_sum,
                            void* dx, void* dweight, void* dbias, void* workspace, size_t workspace_bytes, void* stream);
size_t sk_layer_norm_workspace_bytes(const sk_layer_norm_shape* shape);

/*
 * A dense layer:  y = act(z) + residual,  z = x weight^T + bias.
 *   x [tokens, in] and residual [tokens, out] with row strides, weight [out, in], bias [out], y [tokens, out] dense.  bias and residual may be NULL.
 * z [tokens, out] dense, for a backward pass of a layer with an activation, or NULL (not looked at without one).
 *   in and out multiples of 8 up to 2^20, up to 2^24 tokens, strides up to 2^20 and not below a row, each matrix below 2^34 values.
 */
typedef enum {
  SK_ACT_NONE = 0,
  SK_ACT_RELU = 1,       /* max(z, 0) */
  SK_ACT_GELU = 2,       /* z Phi(z), Phi the normal distribution's */
  SK_ACT_GELU_TANH = 3,  /* z / 2 (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) */
  SK_ACT_SILU = 4        /* z / (1 + exp(-z)) */
} sk_activation;

typedef struct {
  int64_t tokens, in, out;
  int32_t activation;        /* sk_activation */
  sk_dtype dtype;
  int64_t x_stride, residual_stride;   /* elements between rows */
} sk_dense_shape;

size_t sk_dense_workspace_bytes(const sk_dense_shape* shape, int32_t backward);
sk_status sk_dense_fwd(const sk_dense_shape* shape, const void* x, const void* weight, const void* bias, const void* residual, void* y, void* z,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * Its gradients:  dz = dy act'(z),  dx = dz weight,  dweight = dz^T x,  dbias = sum of dz over tokens  (the residual's is dy).
 *   z: the forward pass's (NULL without an activation), dy [tokens, out], dx [tokens, in], dweight [out, in], dbias [out] dense, in `dtype`; each gradient may be
 * NULL.  In bf16 dz is rounded once, as an operand of both products.
 */
sk_status sk_dense_bwd(const sk_dense_shape* shape, const void* x, const void* weight, const void* z, const void* dy, void* dx, void* dweight,
                       void* dbias, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The loss of logits z [rows, vocabulary] against a teacher's `top` largest logits t at the places c, and against labels:
 *     loss = (1 - label_weight) temperature^2 sum_k p_k (log p_k - log q_c(k)) + label_weight (log sum_j exp z_j - z_label),
 *     p = softmax(t / temperature) over the row's entries,  q = softmax(z / temperature).
 * An entry whose id is outside the vocabulary or whose logit is -infinity is not there (lists may be of different lengths); a place that is named twice has
 * both entries.  A row without an entry has no first term, one whose label is outside the vocabulary (or all, with labels NULL) no second.
 *   logits on any boundary of a value, with a row stride of any number of elements, teacher_logits [rows, top] in `dtype`, teacher_ids [rows, top], labels [rows], loss [rows] fp32.
 * stats [rows, 8] fp32 for a backward pass, or NULL.  (A row whose logits are all -infinity has no softmax: NaN.)
 *   rows below 2^23, vocabulary up to 2^24, top up to 2^16 (0: no teacher; its pointers may be NULL), temperature from 10^-3 to 10^3.
 * Made for lists of some hundred entries: past about a thousand the gradient's time grows with the square of their length.
 */
typedef struct {
  int64_t rows, vocabulary, logits_stride;
  int32_t top;
  int32_t id_bytes, label_bytes;   /* 4 or 8 */
  float temperature, label_weight; /* label_weight in 0 .. 1 */
  sk_dtype dtype;
} sk_distill_shape;

sk_status sk_distill_fwd(const sk_distill_shape* shape, const void* logits, const void* teacher_logits, const void* teacher_ids, const void* labels,
                         float* loss, float* stats, void* stream);
/*
 * Its gradient, from the inputs, the forward pass's stats and the gradient dloss [rows] of every row's loss:
 *     dz_j = dloss [ (1 - label_weight) temperature (q_j - sum_{k: c(k) = j} p_k) + label_weight (softmax(z)_j - [j = label]) ],
 * dlogits [rows, vocabulary] dense in `dtype`; zeros in a row without an entry and a label, whatever its logits are.
 */
sk_status sk_distill_bwd(const sk_distill_shape* shape, const void* logits, const void* teacher_logits, const void* teacher_ids, const void* labels,
                         const float* stats, const float* dloss, void* dlogits, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SK_BLOCK_H */
