// The block operators' C ABI (include/sk_block.h): argument validation and launches.  Validation runs before any HIP call.
#include <cmath>

#include "../../include/sk_block.h"
#include "sk_block_launch.h"
#include "sk_dense_launch.h"

namespace {

using namespace sk;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
template <typename... P>
bool aligned16(const void* p, P... more) { return aligned16(p) && aligned16(more...); }
size_t align_up(size_t v) { return (v + 255) / 256 * 256; }

sk_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return SK_OK;
  note_hip_error(e, what);
  return SK_ERR_HIP;
}
bool known(sk_dtype t) { return t == SK_F32 || t == SK_BF16; }
int esize(sk_dtype t) { return t == SK_BF16 ? 2 : 4; }

// A stride of a dimension of `size`: what it is where it counts, 0 elsewhere; false if it is not one.
bool stride_ok(int64_t size, int64_t stride, sk_dtype t, int64_t most, int64_t& out, sk_status& st) {
  out = 0;
  if (size <= 1) return true;
  if (stride < 0) { st = SK_ERR_INVALID_ARG; return false; }
  if (stride * esize(t) % 16 != 0 || stride > most) { st = SK_ERR_UNSUPPORTED; return false; }
  out = stride;
  return true;
}

constexpr int64_t MOST_ROWS = 1 << 27;          // queries times group, keys: positions are 32-bit in the kernels
constexpr int64_t MOST_TOKEN_STRIDE = 1 << 22;  // a tile's offsets are 32-bit bytes
constexpr int64_t MOST_GROUPS = (1 << 24) - 1;  // work-groups of 256 threads in a launch
constexpr int64_t MOST_THREADS = (int64_t)1 << 32;  // of a launch
constexpr int64_t MOST_STRIDE = (int64_t)1 << 40;

sk_status attention_args(const sk_attention_shape* s, AttentionArgs& a) {
  if (s == nullptr) return SK_ERR_INVALID_ARG;
  if (s->batch < 1 || s->q_len < 1 || s->k_len < 1 || s->heads < 1 || s->kv_heads < 1 || s->head_dim < 1 || !std::isfinite(s->scale) || s->causal < 0 ||
      s->causal > 1)
    return SK_ERR_INVALID_ARG;
  if (!known(s->dtype) || s->head_dim % 8 != 0 || s->head_dim > 128 || s->heads % s->kv_heads != 0) return SK_ERR_UNSUPPORTED;
  const int group = s->heads / s->kv_heads;
  if (s->q_len > MOST_ROWS / group || s->k_len > MOST_ROWS || s->batch > MOST_ROWS || (int64_t)s->heads * s->head_dim > MOST_TOKEN_STRIDE) return SK_ERR_UNSUPPORTED;
  const int64_t tiles = (s->q_len * group + 127) / 128 + (s->k_len + 127) / 128;
  if ((double)s->batch * s->kv_heads * tiles > MOST_GROUPS) return SK_ERR_UNSUPPORTED;
  sk_status st = SK_OK;
  const int64_t most[3] = {MOST_STRIDE, MOST_TOKEN_STRIDE, MOST_STRIDE};
  const int64_t q_sizes[3] = {s->batch, s->q_len, s->heads}, k_sizes[3] = {s->batch, s->k_len, s->kv_heads};
  for (int i = 0; i < 3; ++i)
    if (!stride_ok(q_sizes[i], s->q_strides[i], s->dtype, most[i], a.qs[i], st) || !stride_ok(k_sizes[i], s->k_strides[i], s->dtype, most[i], a.ks[i], st) ||
        !stride_ok(k_sizes[i], s->v_strides[i], s->dtype, most[i], a.vs[i], st))
      return st;
  // (a lone token's tile has nothing behind it: the window of a tile's rows ends with the last only where rows do not overlap)
  if (s->q_len == 1) a.qs[1] = s->head_dim;
  if (s->k_len == 1) a.ks[1] = a.vs[1] = s->head_dim;
  a.batch = (int)s->batch; a.q_len = (int)s->q_len; a.k_len = (int)s->k_len;
  a.heads = s->heads; a.kv_heads = s->kv_heads; a.group = group; a.D = s->head_dim;
  a.causal = s->causal; a.scale = s->scale;
  a.q_lengths = s->q_lengths; a.k_lengths = s->k_lengths;
  return SK_OK;
}
bool lengths_aligned(const AttentionArgs& a) { return ((reinterpret_cast<uintptr_t>(a.q_lengths) | reinterpret_cast<uintptr_t>(a.k_lengths)) & 3u) == 0; }
size_t stat_bytes(const AttentionArgs& a) { return align_up((size_t)a.batch * a.heads * a.q_len * 4); }
size_t parts_bytes(const AttentionArgs& a, int parts) { return parts > 1 ? align_up((size_t)parts * 2 * a.batch * a.k_len * a.kv_heads * a.D * 4) : 0; }
size_t query_shares_bytes(const AttentionArgs& a, int shares) { return shares > 1 ? align_up((size_t)shares * a.batch * a.q_len * a.heads * a.D * 4) : 0; }
size_t attention_bytes(const AttentionArgs& a, bool f32, bool backward) {
  if (!backward) return f32 ? 0 : align_up(attention_fwd_bytes_bf16(a));
  return 2 * stat_bytes(a) + parts_bytes(a, attention_parts(a, f32)) + query_shares_bytes(a, f32 ? 1 : attention_query_shares(a));
}

// Whether two of `tokens` x `heads` rows of D values lie on the same place.
bool rows_overlap(int64_t tokens, int64_t heads, int64_t D, int64_t token_stride, int64_t head_stride) {
  if (tokens > 1 && token_stride < D) return true;
  if (heads > 1 && head_stride < D) return true;
  // (one inside the other's step, as any slice of a tensor is)
  if (tokens == 1 || heads == 1 || token_stride >= (heads - 1) * head_stride + D || head_stride >= (tokens - 1) * token_stride + D) return false;
  for (int64_t h = 1; h < heads; ++h) {   // the tokens whose rows begin next to head h's, on either side
    const int64_t t = h * head_stride / token_stride, past = h * head_stride - t * token_stride;
    if ((t < tokens && past < D) || (t + 1 < tokens && token_stride - past < D)) return true;
  }
  return false;
}

sk_status norm_rope_args(const sk_norm_rope_shape* s, NormRopeArgs& a, bool back) {
  if (s == nullptr) return SK_ERR_INVALID_ARG;
  if (s->tokens < 1 || s->heads < 1 || s->kv_heads < 0 || s->head_dim < 1 || s->rotary_dim < 0 || s->rotary_dim > s->head_dim || s->interleaved < 0 ||
      s->interleaved > 1 || !(s->eps >= 0.f) || !std::isfinite(s->eps) || (s->rotary_dim > 0 && s->table_rows < 1))
    return SK_ERR_INVALID_ARG;
  if (!known(s->dtype) || s->head_dim % 8 != 0 || s->head_dim > 256 || s->rotary_dim % 8 != 0) return SK_ERR_UNSUPPORTED;
  if (s->rotary_dim > 0 && s->position_bytes != 4 && s->position_bytes != 8) return SK_ERR_UNSUPPORTED;
  if (s->tokens > (1 << 25) || s->heads > (1 << 16) || s->kv_heads > (1 << 16)) return SK_ERR_UNSUPPORTED;
  sk_status st = SK_OK;
  const int64_t most = (int64_t)1 << 31;
  const int64_t q_sizes[2] = {s->tokens, s->heads}, k_sizes[2] = {s->tokens, s->kv_heads};
  for (int i = 0; i < 2; ++i) {
    const bool keys = s->kv_heads > 0;
    if (!stride_ok(q_sizes[i], s->q_strides[i], s->dtype, most, a.qs[i], st) ||
        !stride_ok(keys ? k_sizes[i] : 1, s->k_strides[i], s->dtype, most, a.ks[i], st))
      return st;
    a.qos[i] = a.kos[i] = 0;
    if (!back && (!stride_ok(q_sizes[i], s->q_out_strides[i], s->dtype, most, a.qos[i], st) ||
                  !stride_ok(keys ? k_sizes[i] : 1, s->k_out_strides[i], s->dtype, most, a.kos[i], st)))
      return st;
  }
  if (!back && (rows_overlap(s->tokens, s->heads, s->head_dim, a.qos[0], a.qos[1]) ||
                (s->kv_heads > 0 && rows_overlap(s->tokens, s->kv_heads, s->head_dim, a.kos[0], a.kos[1]))))
    return SK_ERR_INVALID_ARG;
  a.tokens = s->tokens; a.table_rows = s->table_rows;
  a.heads = s->heads; a.kv_heads = s->kv_heads; a.D = s->head_dim; a.rotary = s->rotary_dim;
  a.interleaved = s->interleaved; a.pos64 = s->position_bytes == 8;
  a.eps = s->eps;
  return SK_OK;
}
size_t norm_rope_bytes(const NormRopeArgs& a) {
  const int64_t groups = (a.tokens + 3) / 4 < NORM_ROPE_MAX_GROUPS ? (a.tokens + 3) / 4 : NORM_ROPE_MAX_GROUPS;
  return align_up((size_t)groups * 2 * a.D * 4);
}

sk_status embedding_args(const void* ids, int32_t id_bytes, int64_t tokens, int64_t rows, int64_t width, float scale, sk_dtype dtype, EmbeddingArgs& a) {
  if (tokens < 1 || rows < 1 || width < 1 || !std::isfinite(scale)) return SK_ERR_INVALID_ARG;
  if (!known(dtype) || (id_bytes != 4 && id_bytes != 8) || width % 8 != 0 || width > (1 << 20) || rows > INT32_MAX || tokens > MOST_ROWS) return SK_ERR_UNSUPPORTED;
  if ((double)((tokens + 15) / 16) * ((width + 255) / 256) > MOST_GROUPS) return SK_ERR_UNSUPPORTED;
  a = EmbeddingArgs{};
  a.ids = ids; a.ids64 = id_bytes == 8;
  a.tokens = tokens; a.rows = rows; a.width = (int)width; a.scale = scale;
  return SK_OK;
}
struct EmbeddingRoom {
  size_t keys, order, keys_runs, order_runs, partial, total;
  EmbeddingRoom(int64_t tokens, int64_t rows, int64_t width, sk_dtype dtype) {
    const int chunk = embedding_chunk(tokens, width, esize(dtype));
    const size_t list = align_up((size_t)tokens * 4), runs = tokens > embedding_run(tokens, rows, width, esize(dtype)) ? list : 0;
    keys = 0; order = keys + list; keys_runs = order + list; order_runs = keys_runs + runs;
    partial = order_runs + runs;
    total = partial + align_up((size_t)((tokens + chunk - 1) / chunk) * 2 * width * 4);
  }
};

// Of rows `width` long: dense ones, or further apart; false as stride_ok.
bool row_stride_ok(int64_t rows, int64_t width, int64_t stride, sk_dtype t, int64_t most, int64_t& out, sk_status& st) {
  if (!stride_ok(rows, stride, t, most, out, st)) return false;
  if (rows <= 1) out = width;
  return true;
}

sk_status layer_norm_args(const sk_layer_norm_shape* s, LayerNormArgs& a) {
  if (s == nullptr) return SK_ERR_INVALID_ARG;
  if (s->rows < 1 || s->width < 1 || !(s->eps >= 0.f) || !std::isfinite(s->eps)) return SK_ERR_INVALID_ARG;
  if (!known(s->dtype) || s->width % 8 != 0 || s->width > LAYER_NORM_MAX_WIDTH || s->rows >= (1 << 24)) return SK_ERR_UNSUPPORTED;
  if (s->rows * layer_norm_lanes((int)s->width) >= MOST_THREADS) return SK_ERR_UNSUPPORTED;
  sk_status st = SK_OK;
  if (!row_stride_ok(s->rows, s->width, s->x_stride, s->dtype, MOST_STRIDE, a.x_stride, st) ||
      !row_stride_ok(s->rows, s->width, s->residual_stride, s->dtype, MOST_STRIDE, a.residual_stride, st))
    return st;
  a.rows = s->rows; a.width = (int)s->width; a.eps = s->eps;
  return SK_OK;
}
size_t layer_norm_bytes(const LayerNormArgs& a) { return align_up((size_t)layer_norm_groups(a.rows, a.width) * 2 * a.width * 4); }

sk_status dense_layer_args(const sk_dense_shape* s, DenseArgs& a) {
  if (s == nullptr) return SK_ERR_INVALID_ARG;
  if (s->tokens < 1 || s->in < 1 || s->out < 1 || s->activation < 0) return SK_ERR_INVALID_ARG;
  if (!known(s->dtype) || s->activation > SK_ACT_SILU || s->in % 8 != 0 || s->out % 8 != 0 || s->tokens > (1 << 24) || s->in > (1 << 20) || s->out > (1 << 20)) return SK_ERR_UNSUPPORTED;
  const int64_t most = (int64_t)1 << 34;   // values of any of the matrices: work-groups of 256 threads in a launch
  if (s->tokens * s->in >= most || s->tokens * s->out >= most || s->in * s->out >= most) return SK_ERR_UNSUPPORTED;
  sk_status st = SK_OK;
  if (!row_stride_ok(s->tokens, s->in, s->x_stride, s->dtype, 1 << 20, a.x_stride, st) ||
      !row_stride_ok(s->tokens, s->out, s->residual_stride, s->dtype, 1 << 20, a.residual_stride, st))
    return st;
  // (the windows that rows are read through take them for apart)
  if (a.x_stride < s->in || a.residual_stride < s->out) return SK_ERR_UNSUPPORTED;
  a.tokens = (int)s->tokens; a.in = (int)s->in; a.out = (int)s->out; a.activation = s->activation;
  return SK_OK;
}
struct DenseRoom {   // backward: dz | column sums | the products' slabs, one product after the other
  size_t dz, partial, slabs, total;
  DenseRoom(const DenseArgs& a, bool f32) {
    partial = a.activation != SK_ACT_NONE ? align_up((size_t)a.tokens * a.out * (f32 ? 4 : 2)) : 0;
    dz = 0;
    slabs = partial + align_up((size_t)ColumnRuns(a.tokens, a.out).runs * a.out * 4);
    const size_t dx = product_bytes(GEMM_NN, a.tokens, a.in, a.out, f32), dw = product_bytes(GEMM_TN, a.out, a.in, a.tokens, f32);
    total = slabs + (dx > dw ? dx : dw);
  }
};
size_t dense_forward_bytes(const DenseArgs& a, bool f32) {
  const DensePlan d = plan_dense(a.tokens, a.out, a.in, f32);
  return d.fused ? 0 : align_up((size_t)d.splits * a.tokens * a.out * 4);
}
GemmArgs product(const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t M, int64_t N, int64_t K, const void* bias) {
  GemmArgs g{};
  g.A = A; g.B = B; g.C = C; g.bias = bias;
  g.lda = lda; g.ldb = ldb; g.ldc = N;
  g.M = (int)M; g.N = (int)N; g.K = (int)K;
  return g;
}

sk_status distill_args(const sk_distill_shape* s, const void* logits, DistillArgs& a) {
  if (s == nullptr) return SK_ERR_INVALID_ARG;
  if (s->rows < 1 || s->vocabulary < 1 || s->top < 0 || s->logits_stride < 0 || !(s->temperature > 0.f) || !std::isfinite(s->temperature) ||
      !(s->label_weight >= 0.f && s->label_weight <= 1.f))
    return SK_ERR_INVALID_ARG;
  if (!known(s->dtype) || (s->id_bytes != 4 && s->id_bytes != 8) || (s->label_bytes != 4 && s->label_bytes != 8) || s->rows >= (1 << 23) || s->vocabulary > (1 << 24) ||
      s->top > (1 << 16) || s->logits_stride > MOST_STRIDE || !(s->temperature >= 1e-3f && s->temperature <= 1e3f))
    return SK_ERR_UNSUPPORTED;
  // (rows begin anywhere; values where values do)
  if (reinterpret_cast<uintptr_t>(logits) % esize(s->dtype) != 0) return SK_ERR_INVALID_ARG;
  a.logits = logits;
  a.rows = s->rows; a.logits_stride = s->logits_stride;
  a.vocabulary = (int)s->vocabulary; a.top = s->top;
  a.ids64 = s->id_bytes == 8; a.labels64 = s->label_bytes == 8;
  a.temperature = s->temperature; a.label_weight = s->label_weight;
  return SK_OK;
}

}  // namespace

extern "C" {

size_t sk_attention_workspace_bytes(const sk_attention_shape* shape, int32_t backward) {
  AttentionArgs a{};
  if (attention_args(shape, a) != SK_OK) return (size_t)-1;
  return attention_bytes(a, shape->dtype == SK_F32, backward != 0);
}

sk_status sk_attention_fwd(const sk_attention_shape* shape, const void* q, const void* k, const void* v, void* o, float* lse,
                           void* o_rest, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !o || !aligned16(q, k, v, o, lse, o_rest, workspace)) return SK_ERR_INVALID_ARG;
  AttentionArgs a{};
  const sk_status st = attention_args(shape, a);
  if (st != SK_OK) return st;
  if (!lengths_aligned(a)) return SK_ERR_INVALID_ARG;
  const size_t need = attention_bytes(a, shape->dtype == SK_F32, false);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SK_ERR_WORKSPACE;
  a.q = q; a.k = k; a.v = v; a.o = o; a.lse = lse; a.workspace = workspace;
  a.o_rest = shape->dtype == SK_F32 ? nullptr : o_rest;
  return launched(launch_attention_fwd(a, shape->dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_attention_fwd");
}

sk_status sk_attention_bwd(const sk_attention_shape* shape, const void* q, const void* k, const void* v, const void* o,
                           const float* lse, const void* o_rest, const void* d_o, void* dq, void* dk, void* dv, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv || !aligned16(q, k, v, o, lse, o_rest, d_o, dq, dk, dv, workspace)) return SK_ERR_INVALID_ARG;
  AttentionArgs a{};
  const sk_status st = attention_args(shape, a);
  if (st != SK_OK) return st;
  if (!lengths_aligned(a)) return SK_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < attention_bytes(a, shape->dtype == SK_F32, true)) return SK_ERR_WORKSPACE;
  a.q = q; a.k = k; a.v = v; a.o_in = o; a.lse = const_cast<float*>(lse); a.d_o = d_o;
  a.o_rest = shape->dtype == SK_F32 ? nullptr : const_cast<void*>(o_rest);
  a.dq = dq; a.dk = dk; a.dv = dv;
  char* const w = static_cast<char*>(workspace);
  a.lse2 = reinterpret_cast<float*>(w);
  a.delta = reinterpret_cast<float*>(w + stat_bytes(a));
  a.parts = attention_parts(a, shape->dtype == SK_F32);
  a.partial = reinterpret_cast<float*>(w + 2 * stat_bytes(a));
  a.q_shares = shape->dtype == SK_F32 ? 1 : attention_query_shares(a);
  a.q_partial = reinterpret_cast<float*>(w + 2 * stat_bytes(a) + parts_bytes(a, a.parts));
  return launched(launch_attention_bwd(a, shape->dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_attention_bwd");
}

sk_status sk_norm_rope_fwd(const sk_norm_rope_shape* shape, const void* q, const void* k, const void* q_weight, const void* k_weight,
                           const float* cos, const float* sin, const void* positions, void* q_out, void* k_out, void* stream) {
  NormRopeArgs a{};
  if (shape == nullptr) return SK_ERR_INVALID_ARG;
  if (!q || !q_weight || !q_out || !aligned16(q, q_weight, q_out)) return SK_ERR_INVALID_ARG;
  if (shape->kv_heads > 0 && (!k || !k_weight || !k_out || !aligned16(k, k_weight, k_out))) return SK_ERR_INVALID_ARG;
  if (shape->rotary_dim > 0 && (!cos || !sin || !positions || !aligned16(cos, sin, positions))) return SK_ERR_INVALID_ARG;
  const sk_status st = norm_rope_args(shape, a, false);
  if (st != SK_OK) return st;
  a.q = q; a.k = k; a.wq = q_weight; a.wk = k_weight; a.cos = cos; a.sin = sin; a.positions = positions;
  a.q_out = q_out; a.k_out = k_out;
  return launched(launch_norm_rope_fwd(a, shape->dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_norm_rope_fwd");
}

size_t sk_norm_rope_workspace_bytes(const sk_norm_rope_shape* shape) {
  NormRopeArgs a{};
  if (norm_rope_args(shape, a, true) != SK_OK) return (size_t)-1;
  return norm_rope_bytes(a);
}

sk_status sk_norm_rope_bwd(const sk_norm_rope_shape* shape, const void* q, const void* k, const void* q_weight, const void* k_weight,
                           const float* cos, const float* sin, const void* positions, const void* dq_out, const void* dk_out,
                           void* dq, void* dk, void* dq_weight, void* dk_weight, void* workspace, size_t workspace_bytes, void* stream) {
  NormRopeArgs a{};
  if (shape == nullptr) return SK_ERR_INVALID_ARG;
  if (!q || !q_weight || !dq_out || !dq || !dq_weight || !aligned16(q, q_weight, dq_out, dq, dq_weight, workspace)) return SK_ERR_INVALID_ARG;
  if (shape->kv_heads > 0 && (!k || !k_weight || !dk_out || !dk || !dk_weight || !aligned16(k, k_weight, dk_out, dk, dk_weight))) return SK_ERR_INVALID_ARG;
  if (shape->rotary_dim > 0 && (!cos || !sin || !positions || !aligned16(cos, sin, positions))) return SK_ERR_INVALID_ARG;
  const sk_status st = norm_rope_args(shape, a, true);
  if (st != SK_OK) return st;
  if (!workspace || workspace_bytes < norm_rope_bytes(a)) return SK_ERR_WORKSPACE;
  a.q = q; a.k = k; a.wq = q_weight; a.wk = k_weight; a.cos = cos; a.sin = sin; a.positions = positions;
  a.dq_out = dq_out; a.dk_out = dk_out; a.q_out = dq; a.k_out = dk; a.dwq = dq_weight; a.dwk = dk_weight;
  a.partial = static_cast<float*>(workspace);
  return launched(launch_norm_rope_bwd(a, shape->dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_norm_rope_bwd");
}

sk_status sk_embedding_fwd(const void* ids, int32_t id_bytes, const void* table, void* y, int64_t tokens, int64_t rows,
                           int64_t width, float scale, sk_dtype dtype, void* stream) {
  if (!ids || !table || !y || !aligned16(ids, table, y)) return SK_ERR_INVALID_ARG;
  EmbeddingArgs a;
  const sk_status st = embedding_args(ids, id_bytes, tokens, rows, width, scale, dtype, a);
  if (st != SK_OK) return st;
  a.table = table; a.out = y;
  return launched(launch_embedding_fwd(a, dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_embedding_fwd");
}

size_t sk_embedding_workspace_bytes(int64_t tokens, int64_t rows, int64_t width, sk_dtype dtype) {
  EmbeddingArgs a;
  if (embedding_args(nullptr, 8, tokens, rows, width, 1.f, dtype, a) != SK_OK) return (size_t)-1;
  return EmbeddingRoom(tokens, rows, width, dtype).total;
}

sk_status sk_embedding_bwd(const void* ids, int32_t id_bytes, const void* dy, void* dtable, int64_t tokens, int64_t rows,
                           int64_t width, float scale, sk_dtype dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!ids || !dy || !dtable || !aligned16(ids, dy, dtable, workspace)) return SK_ERR_INVALID_ARG;
  EmbeddingArgs a;
  const sk_status st = embedding_args(ids, id_bytes, tokens, rows, width, scale, dtype, a);
  if (st != SK_OK) return st;
  const EmbeddingRoom room(tokens, rows, width, dtype);
  a.run = embedding_run(tokens, rows, width, esize(dtype));
  if (!workspace || workspace_bytes < room.total) return SK_ERR_WORKSPACE;
  char* const w = static_cast<char*>(workspace);
  a.dy = dy; a.out = dtable;
  a.keys = reinterpret_cast<unsigned*>(w + room.keys); a.order = reinterpret_cast<unsigned*>(w + room.order);
  a.keys_runs = reinterpret_cast<unsigned*>(w + room.keys_runs); a.order_runs = reinterpret_cast<unsigned*>(w + room.order_runs);
  a.partial = reinterpret_cast<float*>(w + room.partial);
  return launched(launch_embedding_bwd(a, dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_embedding_bwd");
}

sk_status sk_dropout(const void* x, const void* residual, void* y, int64_t n, float p, uint64_t seed, uint64_t offset,
                     sk_dtype dtype, void* stream) {
  if (!x || !y || !aligned16(x, residual, y) || n < 1 || !(p >= 0.f && p <= 1.f)) return SK_ERR_INVALID_ARG;
  if (!known(dtype)) return SK_ERR_UNSUPPORTED;
  DropoutArgs a;
  a.x = x; a.residual = residual; a.y = y; a.n = n;
  a.drop = (unsigned)std::nearbyint((double)p * 65536.0);
  a.scale = a.drop < 65536 ? (float)(65536.0 / (65536 - a.drop)) : 0.f;
  a.key[0] = (unsigned)seed; a.key[1] = (unsigned)(seed >> 32);
  a.offset[0] = (unsigned)offset; a.offset[1] = (unsigned)(offset >> 32);
  return launched(launch_dropout(a, dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_dropout");
}

sk_status sk_layer_norm_fwd(const sk_layer_norm_shape* shape, const void* x, const void* residual, const void* weight, const void* bias,
                            void* y, void* sum, void* sum_rest, float* stats, void* stream) {
  if (!x || !y || !aligned16(x, residual, weight, bias, y, sum, sum_rest, stats)) return SK_ERR_INVALID_ARG;
  LayerNormArgs a{};
  const sk_status st = layer_norm_args(shape, a);
  if (st != SK_OK) return st;
  if (sum_rest && (!sum || shape->dtype == SK_F32)) return SK_ERR_INVALID_ARG;
  a.x = x; a.residual = residual; a.weight = weight; a.bias = bias; a.y = y; a.s = sum; a.rest = static_cast<unsigned*>(sum_rest); a.stats = stats;
  return launched(launch_layer_norm_fwd(a, shape->dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_layer_norm_fwd");
}

size_t sk_layer_norm_workspace_bytes(const sk_layer_norm_shape* shape) {
  LayerNormArgs a{};
  if (layer_norm_args(shape, a) != SK_OK) return (size_t)-1;
  return layer_norm_bytes(a);
}

sk_status sk_layer_norm_bwd(const sk_layer_norm_shape* shape, const void* x, const void* sum_rest, const void* weight, const float* stats, const void* dy, const void* d_sum,
                            void* dx, void* dweight, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !stats || !dy || !dx || !aligned16(x, sum_rest, weight, stats, dy, d_sum, dx, dweight, dbias, workspace)) return SK_ERR_INVALID_ARG;
  LayerNormArgs a{};
  const sk_status st = layer_norm_args(shape, a);
  if (st != SK_OK) return st;
  if (sum_rest && shape->dtype == SK_F32) return SK_ERR_INVALID_ARG;
  if ((dweight || dbias) && (!workspace || workspace_bytes < layer_norm_bytes(a))) return SK_ERR_WORKSPACE;
  a.x = x; a.rest = static_cast<unsigned*>(const_cast<void*>(sum_rest)); a.weight = weight; a.stats = const_cast<float*>(stats); a.dy = dy; a.ds = d_sum; a.dx = dx; a.dweight = dweight; a.dbias = dbias;
  a.partial = dweight || dbias ? static_cast<float*>(workspace) : nullptr;
  return launched(launch_layer_norm_bwd(a, shape->dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_layer_norm_bwd");
}

size_t sk_dense_workspace_bytes(const sk_dense_shape* shape, int32_t backward) {
  DenseArgs a{};
  if (dense_layer_args(shape, a) != SK_OK) return (size_t)-1;
  return backward ? DenseRoom(a, shape->dtype == SK_F32).total : dense_forward_bytes(a, shape->dtype == SK_F32);
}

sk_status sk_dense_fwd(const sk_dense_shape* shape, const void* x, const void* weight, const void* bias, const void* residual, void* y, void* z,
                       void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !weight || !y || !aligned16(x, weight, bias, residual, y, z, workspace)) return SK_ERR_INVALID_ARG;
  DenseArgs a{};
  const sk_status st = dense_layer_args(shape, a);
  if (st != SK_OK) return st;
  const bool f32 = shape->dtype == SK_F32;
  const size_t need = dense_forward_bytes(a, f32);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SK_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const DensePlan d = plan_dense(a.tokens, a.out, a.in, f32);
  GemmArgs g = product(x, a.x_stride, weight, a.in, y, a.tokens, a.out, a.in, bias);
  hipError_t e;
  if (d.fused) {
    g.splits = 1;
    g.k_per_split = (g.K + 63) / 64 * 64;
    const FinishArgs f = {residual, a.activation != SK_ACT_NONE ? z : nullptr, a.residual_stride};
    e = f32 ? launch_dense_f32(d.tile, a.activation, g, f, s) : d.few ? launch_dense_few_rows(a.activation, g, f, s) : launch_dense_bf16(d.tile, a.activation, g, f, s);
  } else {
    a.x = x; a.weight = weight; a.bias = bias; a.residual = residual; a.y = y; a.z = z;
    a.slabs = static_cast<const float*>(workspace);
    a.splits = d.splits;
    e = launch_product_slabs(g, f32, workspace, s);
    if (e == hipSuccess) e = launch_dense_finish(a, f32, s);
  }
  return launched(e, "sk_dense_fwd");
}

sk_status sk_dense_bwd(const sk_dense_shape* shape, const void* x, const void* weight, const void* z, const void* dy, void* dx, void* dweight,
                       void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !weight || !dy || !aligned16(x, weight, z, dy, dx, dweight, dbias, workspace)) return SK_ERR_INVALID_ARG;
  DenseArgs a{};
  const sk_status st = dense_layer_args(shape, a);
  if (st != SK_OK) return st;
  const bool f32 = shape->dtype == SK_F32, act = a.activation != SK_ACT_NONE;
  if (act && !z) return SK_ERR_INVALID_ARG;
  const DenseRoom room(a, f32);
  if (room.total > 0 && (!workspace || workspace_bytes < room.total)) return SK_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  char* const w = static_cast<char*>(workspace);
  a.x = x; a.weight = weight; a.z = const_cast<void*>(z); a.dy = dy; a.dx = dx; a.dweight = dweight; a.dbias = dbias;
  a.dz = act ? w + room.dz : const_cast<void*>(dy);
  a.partial = dbias ? reinterpret_cast<float*>(w + room.partial) : nullptr;
  hipError_t e = launch_dense_dz(a, f32, s);
  if (e == hipSuccess) e = launch_dense_dbias(a, f32, s);
  if (e == hipSuccess && dx) e = launch_product(GEMM_NN, product(a.dz, a.out, weight, a.in, dx, a.tokens, a.in, a.out, nullptr), f32, w + room.slabs, s);
  if (e == hipSuccess && dweight) e = launch_product(GEMM_TN, product(a.dz, a.out, x, a.x_stride, dweight, a.out, a.in, a.tokens, nullptr), f32, w + room.slabs, s);
  return launched(e, "sk_dense_bwd");
}

sk_status sk_distill_fwd(const sk_distill_shape* shape, const void* logits, const void* teacher_logits, const void* teacher_ids, const void* labels,
                         float* loss, float* stats, void* stream) {
  if (!logits || !loss || !aligned16(teacher_logits, teacher_ids, labels, loss, stats)) return SK_ERR_INVALID_ARG;
  DistillArgs a{};
  const sk_status st = distill_args(shape, logits, a);
  if (st != SK_OK) return st;
  if (a.top > 0 && (!teacher_logits || !teacher_ids)) return SK_ERR_INVALID_ARG;
  a.teacher = teacher_logits; a.ids = teacher_ids; a.labels = labels; a.loss = loss; a.stats = stats;
  return launched(launch_distill_fwd(a, shape->dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_distill_fwd");
}

sk_status sk_distill_bwd(const sk_distill_shape* shape, const void* logits, const void* teacher_logits, const void* teacher_ids, const void* labels,
                         const float* stats, const float* dloss, void* dlogits, void* stream) {
  if (!logits || !stats || !dloss || !dlogits || !aligned16(teacher_logits, teacher_ids, labels, stats, dloss, dlogits)) return SK_ERR_INVALID_ARG;
  DistillArgs a{};
  const sk_status st = distill_args(shape, logits, a);
  if (st != SK_OK) return st;
  if (a.top > 0 && (!teacher_logits || !teacher_ids)) return SK_ERR_INVALID_ARG;
  a.teacher = teacher_logits; a.ids = teacher_ids; a.labels = labels; a.stats = const_cast<float*>(stats); a.dloss = dloss; a.dlogits = dlogits;
  return launched(launch_distill_bwd(a, shape->dtype == SK_F32, static_cast<hipStream_t>(stream)), "sk_distill_bwd");
}

}  // extern "C"
