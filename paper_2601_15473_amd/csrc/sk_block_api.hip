// The block operators' C ABI (include/sk_block.h): argument validation and launches.  Validation runs before any HIP call.
#include <cmath>

#include "../../include/sk_block.h"
#include "sk_block_launch.h"

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

}  // extern "C"
