// C entry points of the operators that complete a decoder: causal attention over packed sequences, norm over the last dimension,
// embedding lookup.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

#include "internal.h"

using namespace muloco;

namespace {

#define BLOCK_CK(call)                                                                                \
  do {                                                                                                \
    cudaError_t e_ = (call);                                                                          \
    if (e_ != cudaSuccess) return ctx_fail(c, MULOCO_ECUDA, "%s failed: %s", #call, cudaGetErrorString(e_)); \
  } while (0)

bool misaligned(const void* p, size_t a) { return (((uintptr_t)p) & (a - 1)) != 0; }

}  // namespace

struct muloco_sequences {
  muloco_ctx* ctx = nullptr;
  int device = 0;
  int64_t tokens = 0, used = 0;         // of the batch, of the sequences
  int64_t n_pairs = 0, n_tiles = 0;
  const AttnTile* table = nullptr;      // pair tiles, query tiles, key tiles
};

namespace {

// Checks the lengths; counts tiles of 256 and of 128 tokens.
muloco_status count_tiles(muloco_ctx* c, const int64_t* lengths, int64_t n, int64_t tokens, muloco_sequences* s) {
  if (n < 0 || (n > 0 && !lengths)) return ctx_fail(c, MULOCO_EINVAL, "lengths is NULL");
  if (tokens < 0 || tokens > INT32_MAX - 2 * ATTN_TILE) return ctx_fail(c, MULOCO_ESHAPE, "tokens must be in 0..2^31-257");
  int64_t used = 0;
  for (int64_t i = 0; i < n; ++i) {
    if (lengths[i] < 0 || lengths[i] > tokens - used)
      return ctx_fail(c, MULOCO_ESHAPE, "sequence %lld of %lld tokens does not fit into a batch of %lld", (long long)i, (long long)lengths[i],
                      (long long)tokens);
    used += lengths[i];
    s->n_pairs += (lengths[i] + 2 * ATTN_TILE - 1) / (2 * ATTN_TILE);
    s->n_tiles += (lengths[i] + ATTN_TILE - 1) / ATTN_TILE;
  }
  s->tokens = tokens;
  s->used = used;
  return MULOCO_OK;
}

size_t table_bytes(const muloco_sequences& s) { return (size_t)(s.n_pairs + 2 * s.n_tiles) * sizeof(AttnTile); }

muloco_status check_attention(muloco_ctx* c, const muloco_attention* a, const muloco_sequences* s) {
  if (!a || !s) return ctx_fail(c, MULOCO_EINVAL, "arguments are NULL");
  if (s->ctx != c) return ctx_fail(c, MULOCO_EINVAL, "the sequences were made with another context");
  if (a->head_dim < 8 || a->head_dim > ATTN_MAX_DIM || (a->head_dim & 7))
    return ctx_fail(c, MULOCO_ESHAPE, "head_dim must be a multiple of 8 in 8..%d (got %d)", ATTN_MAX_DIM, a->head_dim);
  if (a->heads_k < 1 || a->heads_q < 1 || a->heads_q > 65536 || a->heads_q % a->heads_k)
    return ctx_fail(c, MULOCO_ESHAPE, "the count of query heads must be a multiple of that of key heads, at most 65536 (got %d, %d)", a->heads_q, a->heads_k);
  if (!(a->scale > 0.f) || !isfinite(a->scale)) return ctx_fail(c, MULOCO_EINVAL, "scale must be positive and finite");
  if (s->n_tiles * a->heads_q > INT32_MAX) return ctx_fail(c, MULOCO_ESHAPE, "too many tokens and heads for one call");
  if (s->tokens == 0) return MULOCO_OK;
  if (!a->q || !a->k || !a->v) return ctx_fail(c, MULOCO_EINVAL, "q, k or v is NULL");
  if (misaligned(a->q, 16) || misaligned(a->k, 16) || misaligned(a->v, 16))
    return ctx_fail(c, MULOCO_EINVAL, "q, k and v must be 16-byte aligned");
  return MULOCO_OK;
}

// Strides that a copy by tiles can follow; those of a single head or token do not matter.
bool strides_ok(int64_t tokens, int64_t heads, int64_t dim, int64_t ts, int64_t hs) {
  const int64_t most = (int64_t)1 << 38;
  if (heads > 1 && (hs < dim || (hs & 7) || hs > most)) return false;
  if (tokens > 1 && (ts < dim || (ts & 7) || ts > most)) return false;
  return true;
}

muloco_status check_strides(muloco_ctx* c, const muloco_attention* a, int64_t tokens) {
  if (!strides_ok(tokens, a->heads_q, a->head_dim, a->q_token_stride, a->q_head_stride) ||
      !strides_ok(tokens, a->heads_k, a->head_dim, a->k_token_stride, a->k_head_stride) ||
      !strides_ok(tokens, a->heads_k, a->head_dim, a->v_token_stride, a->v_head_stride))
    return ctx_fail(c, MULOCO_ESHAPE, "token and head strides must be multiples of 8 and at least a head long");
  return MULOCO_OK;
}

AttnArgs attention_args(const muloco_attention* a, const muloco_sequences* s, const CtxView& v) {
  AttnArgs k;
  memset(&k, 0, sizeof k);
  k.pair_tiles = s->table;
  k.query_tiles = s->table + s->n_pairs;
  k.key_tiles = k.query_tiles + s->n_tiles;
  k.n_pairs = s->n_pairs; k.n_tiles = s->n_tiles;
  k.tokens = s->tokens;
  k.heads = a->heads_q; k.kv_heads = a->heads_k; k.dim = a->head_dim; k.scale = a->scale;
  k.q = a->q; k.q_ts = a->q_token_stride; k.q_hs = a->q_head_stride;
  k.k = a->k; k.k_ts = a->k_token_stride; k.k_hs = a->k_head_stride;
  k.v = a->v; k.v_ts = a->v_token_stride; k.v_hs = a->v_head_stride;
  k.status = v.status; k.wait_limit_ns = v.wait_limit_ns;
  return k;
}

// Rows behind the last sequence of a dense bf16 [tokens][heads][dim] become zero.
cudaError_t zero_tail(cudaStream_t st, void* x, const muloco_sequences* s, int64_t heads, int64_t dim) {
  const size_t row = (size_t)(heads * dim) * 2;
  return cudaMemsetAsync(static_cast<char*>(x) + (size_t)s->used * row, 0, (size_t)(s->tokens - s->used) * row, st);
}

}  // namespace

extern "C" {

MULOCO_API muloco_status muloco_sequences_bytes(muloco_ctx* c, const int64_t* lengths, int64_t n, int64_t tokens, size_t* bytes) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  if (!bytes) return ctx_fail(c, MULOCO_EINVAL, "bytes is NULL");
  muloco_sequences s;
  const muloco_status r = count_tiles(c, lengths, n, tokens, &s);
  if (r == MULOCO_OK) *bytes = table_bytes(s);
  return r;
}

MULOCO_API muloco_status muloco_sequences_create(muloco_ctx* c, const int64_t* lengths, int64_t n, int64_t tokens, void* table,
                                                 size_t bytes, muloco_sequences** out) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  if (!out) return ctx_fail(c, MULOCO_EINVAL, "out is NULL");
  *out = nullptr;
  muloco_sequences made;
  const muloco_status r = count_tiles(c, lengths, n, tokens, &made);
  if (r != MULOCO_OK) return r;
  const size_t need = table_bytes(made);
  if (need > 0 && (!table || misaligned(table, 16) || bytes < need))
    return ctx_fail(c, MULOCO_EINVAL, "the table takes %zu bytes, 16-byte aligned", need);
  const CtxView v = ctx_view(c);
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  BLOCK_CK(cudaStreamIsCapturing(v.st, &capture));
  if (capture != cudaStreamCaptureStatusNone) return ctx_fail(c, MULOCO_ESTATE, "sequences cannot be made while the stream is captured");
  try {
    // Heaviest first, so that the last thread blocks to start are short: work grows with the tile's offset for queries
    // and with what follows it for keys.  (Among equals the order of the batch, so that a table follows from the lengths alone.)
    std::vector<AttnTile> t;
    t.reserve((size_t)(made.n_pairs + 2 * made.n_tiles));
    auto append = [&](int step) {
      int64_t start = 0;
      for (int64_t i = 0; i < n; start += lengths[i++])
        for (int64_t o = 0; o < lengths[i]; o += step) t.push_back(AttnTile{(int32_t)start, (int32_t)o, (int32_t)lengths[i], 0});
    };
    append(2 * ATTN_TILE);
    append(ATTN_TILE);
    append(ATTN_TILE);
    const auto queries = t.begin() + made.n_pairs, keys = queries + made.n_tiles;
    // (a pair at the end of a sequence may have one tile only)
    auto reach = [](const AttnTile& x, int rows) { return std::min(x.offset + rows, x.length); };
    std::stable_sort(t.begin(), queries, [&](const AttnTile& x, const AttnTile& y) { return reach(x, 256) > reach(y, 256); });
    std::stable_sort(queries, keys, [](const AttnTile& x, const AttnTile& y) { return x.offset > y.offset; });
    std::stable_sort(keys, t.end(), [](const AttnTile& x, const AttnTile& y) { return x.length - x.offset > y.length - y.offset; });
    muloco_sequences* s = new muloco_sequences(made);
    s->ctx = c;
    s->device = ctx_device(c);
    s->table = static_cast<const AttnTile*>(table);
    // (pageable memory: it is read before the call returns)
    const cudaError_t e = need ? cudaMemcpyAsync(table, t.data(), need, cudaMemcpyHostToDevice, v.st) : cudaSuccess;
    if (e != cudaSuccess) {
      delete s;
      return ctx_fail(c, MULOCO_ECUDA, "copy of the tiles failed: %s", cudaGetErrorString(e));
    }
    *out = s;
  } catch (const std::bad_alloc&) {
    return ctx_fail(c, MULOCO_ENOMEM, "no host memory for %lld sequences", (long long)n);
  }
  return MULOCO_OK;
}

MULOCO_API void muloco_sequences_destroy(muloco_sequences* s) {
  if (!s) return;
  const DeviceScope scope(s->device);
  delete s;
}

MULOCO_API muloco_status muloco_causal_attention(muloco_ctx* c, const muloco_attention* a, const muloco_sequences* s, void* o, float* lse) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  muloco_status r = check_attention(c, a, s);
  if (r != MULOCO_OK || s->tokens == 0) return r;
  r = check_strides(c, a, s->tokens);
  if (r != MULOCO_OK) return r;
  if (!o || !lse || misaligned(o, 16) || misaligned(lse, 4)) return ctx_fail(c, MULOCO_EINVAL, "o or lse is NULL or misaligned");
  const CtxView v = ctx_view(c);
  if (s->used < s->tokens) {
    BLOCK_CK(zero_tail(v.st, o, s, a->heads_q, a->head_dim));
    BLOCK_CK(cudaMemset2DAsync(lse + s->used, (size_t)s->tokens * 4, 0, (size_t)(s->tokens - s->used) * 4, (size_t)a->heads_q, v.st));
  }
  if (s->n_tiles == 0) return MULOCO_OK;
  AttnArgs k = attention_args(a, s, v);
  k.o_out = o;
  k.lse = lse;
  k.withhold = ctx_take_withhold(c);
  const char* what = "";
  const cudaError_t e = launch_attention(v.st, k, &what);
  if (e != cudaSuccess) return ctx_fail(c, MULOCO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
  ctx_count_launches(c, 1);
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_causal_attention_backward(muloco_ctx* c, const muloco_attention* a, const muloco_sequences* s,
                                                          const void* d_o, int64_t do_ts, int64_t do_hs, const void* o,
                                                          const float* lse, float* delta, void* dq, void* dk, void* dv) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  muloco_status r = check_attention(c, a, s);
  if (r != MULOCO_OK || s->tokens == 0) return r;
  r = check_strides(c, a, s->tokens);
  if (r != MULOCO_OK) return r;
  if (!strides_ok(s->tokens, a->heads_q, a->head_dim, do_ts, do_hs))
    return ctx_fail(c, MULOCO_ESHAPE, "token and head strides must be multiples of 8 and at least a head long");
  if (!d_o || !o || !lse || !delta || !dq || !dk || !dv) return ctx_fail(c, MULOCO_EINVAL, "an argument is NULL");
  if (misaligned(d_o, 16) || misaligned(o, 16) || misaligned(dq, 16) || misaligned(dk, 16) || misaligned(dv, 16) || misaligned(lse, 4) ||
      misaligned(delta, 4))
    return ctx_fail(c, MULOCO_EINVAL, "tensors must be 16-byte aligned");
  const CtxView v = ctx_view(c);
  if (s->used < s->tokens) {
    BLOCK_CK(zero_tail(v.st, dq, s, a->heads_q, a->head_dim));
    BLOCK_CK(zero_tail(v.st, dk, s, a->heads_k, a->head_dim));
    BLOCK_CK(zero_tail(v.st, dv, s, a->heads_k, a->head_dim));
  }
  if (s->n_tiles == 0) return MULOCO_OK;
  AttnArgs k = attention_args(a, s, v);
  k.o = o;
  k.lse = const_cast<float*>(lse);
  k.g = d_o; k.g_ts = do_ts; k.g_hs = do_hs;
  k.delta = delta;
  k.dq = dq; k.dk = dk; k.dv = dv;
  k.withhold = ctx_take_withhold(c);
  const char* what = "";
  const cudaError_t e = launch_attention_backward(v.st, k, &what);
  if (e != cudaSuccess) return ctx_fail(c, MULOCO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
  ctx_count_launches(c, 2);
  return MULOCO_OK;
}

}  // extern "C"

namespace {

muloco_status check_norm(muloco_ctx* c, const muloco_norm* a) {
  if (!a) return ctx_fail(c, MULOCO_EINVAL, "arguments are NULL");
  if (a->tokens < 0 || a->tokens > INT32_MAX) return ctx_fail(c, MULOCO_ESHAPE, "tokens must be in 0..2^31-1");
  if (a->d < 1 || a->d > NORM_MAX_DIM) return ctx_fail(c, MULOCO_ESHAPE, "d must be in 1..%d (got %lld)", NORM_MAX_DIM, (long long)a->d);
  if (a->dtype != MULOCO_F32 && a->dtype != MULOCO_BF16) return ctx_fail(c, MULOCO_EINVAL, "unknown dtype %d", a->dtype);
  if (!(a->eps >= 0.f)) return ctx_fail(c, MULOCO_EINVAL, "eps must be >= 0");
  if (a->tokens == 0) return MULOCO_OK;
  if (a->tokens > 1 && (a->ldx < a->d || (a->residual && a->ldr < a->d))) return ctx_fail(c, MULOCO_ESHAPE, "row strides must be at least a row long");
  const size_t al = a->dtype == MULOCO_BF16 ? 2 : 4;
  if (!a->x || misaligned(a->x, al) || misaligned(a->residual, al) || misaligned(a->weight, 4) || misaligned(a->bias, 4))
    return ctx_fail(c, MULOCO_EINVAL, "x is NULL, or a pointer is not aligned to its type");
  return MULOCO_OK;
}

// (a single row's stride does not matter)
int64_t stride_of(const muloco_norm* a, const void* p, int64_t ld) { return !p ? 0 : a->tokens > 1 ? ld : a->d; }

NormArgs norm_args(const muloco_norm* a) {
  NormArgs n;
  memset(&n, 0, sizeof n);
  n.tokens = a->tokens; n.d = (int32_t)a->d; n.center = a->center != 0;
  n.ldx = stride_of(a, a->x, a->ldx); n.ldr = stride_of(a, a->residual, a->ldr);
  n.x = a->x; n.weight = a->weight;
  n.eps = a->eps;
  n.inv_d = (float)(1.0 / (double)a->d);
  return n;
}

muloco_status check_embedding(muloco_ctx* c, const muloco_embedding* a) {
  if (!a) return ctx_fail(c, MULOCO_EINVAL, "arguments are NULL");
  if (a->tokens < 0 || a->tokens > INT32_MAX || a->rows < 0 || a->rows > INT32_MAX)
    return ctx_fail(c, MULOCO_ESHAPE, "tokens and rows must be in 0..2^31-1");
  if (a->d < 1 || a->d > (1 << 20)) return ctx_fail(c, MULOCO_ESHAPE, "d must be in 1..2^20 (got %lld)", (long long)a->d);
  if ((a->tokens + a->rows / 32 + 64) * ((a->d + 255) / 256) > ((int64_t)1 << 33)) return ctx_fail(c, MULOCO_ESHAPE, "too many rows for one call");
  if (a->dtype != MULOCO_F32 && a->dtype != MULOCO_BF16) return ctx_fail(c, MULOCO_EINVAL, "unknown dtype %d", a->dtype);
  if (!isfinite(a->scale)) return ctx_fail(c, MULOCO_EINVAL, "scale must be finite");
  if (a->tokens > 0 && (!a->ids || misaligned(a->ids, 8))) return ctx_fail(c, MULOCO_EINVAL, "ids is NULL or not aligned to its type");
  return MULOCO_OK;
}

EmbeddingArgs embedding_args(const muloco_embedding* a, const CtxView& v) {
  EmbeddingArgs e;
  memset(&e, 0, sizeof e);
  e.tokens = a->tokens; e.rows = a->rows; e.ld = a->ld; e.d = (int32_t)a->d;
  e.ids = a->ids; e.scale = a->scale;
  e.status = v.status;
  return e;
}

}  // namespace

extern "C" {

MULOCO_API muloco_status muloco_layer_norm(muloco_ctx* c, const muloco_norm* a, void* h, void* y, float* mean, float* rstd) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  const muloco_status r = check_norm(c, a);
  if (r != MULOCO_OK || a->tokens == 0) return r;
  const size_t al = a->dtype == MULOCO_BF16 ? 2 : 4;
  if (!y || !rstd || (a->center && !mean) || (a->residual && !h) || misaligned(y, al) || misaligned(h, al) || misaligned(mean, 4) ||
      misaligned(rstd, 4))
    return ctx_fail(c, MULOCO_EINVAL, "a result is NULL or not aligned to its type");
  for (const void* in : {a->x, a->residual})
    if (in && (in == y || in == h) && (in == a->x ? a->ldx : a->ldr) != a->d && a->tokens > 1)
      return ctx_fail(c, MULOCO_EINVAL, "a result in place of an input needs that one dense");
  if (a->residual && y == h) return ctx_fail(c, MULOCO_EINVAL, "y and h are the same");
  const CtxView v = ctx_view(c);
  NormArgs n = norm_args(a);
  n.residual = a->residual; n.bias = a->bias;
  n.h = h; n.y = y; n.mean = mean; n.rstd = rstd;
  int launches = 0;
  BLOCK_CK(launch_norm(v.st, n, false, a->dtype == MULOCO_BF16, v.n_sms, &launches));
  ctx_count_launches(c, launches);
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_layer_norm_backward(muloco_ctx* c, const muloco_norm* a, const void* dy, int64_t lddy, const float* mean,
                                                    const float* rstd, void* dx, float* dweight, float* dbias, float* scratch) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  const muloco_status r = check_norm(c, a);
  if (r != MULOCO_OK) return r;
  if (misaligned(dweight, 4) || misaligned(dbias, 4)) return ctx_fail(c, MULOCO_EINVAL, "a pointer is not aligned to its type");
  const CtxView v = ctx_view(c);
  if (a->tokens == 0) {                        // the sums over tokens are empty
    if (dweight) BLOCK_CK(cudaMemsetAsync(dweight, 0, (size_t)a->d * 4, v.st));
    if (dbias) BLOCK_CK(cudaMemsetAsync(dbias, 0, (size_t)a->d * 4, v.st));
    return MULOCO_OK;
  }
  const size_t al = a->dtype == MULOCO_BF16 ? 2 : 4;
  if (!dy || !dx || !rstd || (a->center && !mean) || misaligned(dy, al) || misaligned(dx, al) || misaligned(mean, 4) || misaligned(rstd, 4))
    return ctx_fail(c, MULOCO_EINVAL, "a tensor is NULL or not aligned to its type");
  if (a->tokens > 1 && lddy < a->d) return ctx_fail(c, MULOCO_ESHAPE, "row strides must be at least a row long");
  if ((dweight || dbias) && (!scratch || misaligned(scratch, 16))) return ctx_fail(c, MULOCO_EINVAL, "scratch is NULL or not 16-byte aligned");
  NormArgs n = norm_args(a);
  n.dh = a->residual;
  n.dy = dy; n.ldy = stride_of(a, dy, lddy);
  n.mean = const_cast<float*>(mean); n.rstd = const_cast<float*>(rstd);
  n.dx = dx; n.dweight = dweight; n.dbias = dbias;
  n.partials = dweight || dbias ? scratch : nullptr;
  int launches = 0;
  BLOCK_CK(launch_norm(v.st, n, true, a->dtype == MULOCO_BF16, v.n_sms, &launches));
  ctx_count_launches(c, launches);
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_embedding_lookup(muloco_ctx* c, const muloco_embedding* a, const void* table, void* out) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  const muloco_status r = check_embedding(c, a);
  if (r != MULOCO_OK || a->tokens == 0) return r;
  if (a->rows > 1 && a->ld < a->d) return ctx_fail(c, MULOCO_ESHAPE, "row strides must be at least a row long");
  const size_t al = a->dtype == MULOCO_BF16 ? 2 : 4;
  if ((a->rows > 0 && !table) || !out || misaligned(table, al) || misaligned(out, al))
    return ctx_fail(c, MULOCO_EINVAL, "table or out is NULL or not aligned to its type");
  const CtxView v = ctx_view(c);
  EmbeddingArgs e = embedding_args(a, v);
  e.table = table; e.out = out;
  BLOCK_CK(launch_embedding(v.st, e, a->dtype == MULOCO_BF16));
  ctx_count_launches(c, 1);
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_embedding_scratch(muloco_ctx* c, int64_t tokens, int64_t d, size_t* bytes) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  if (!bytes || tokens < 0 || tokens > INT32_MAX || d < 1 || d > (1 << 20)) return ctx_fail(c, MULOCO_EINVAL, "tokens or d out of range, or bytes NULL");
  *bytes = tokens > 0 ? embedding_scratch(tokens, d) : 0;
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_embedding_backward(muloco_ctx* c, const muloco_embedding* a, const void* dout, int32_t dtable_dtype,
                                                   void* dtable, void* scratch) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  const muloco_status r = check_embedding(c, a);
  if (r != MULOCO_OK) return r;
  if (dtable_dtype != MULOCO_F32 && dtable_dtype != MULOCO_BF16) return ctx_fail(c, MULOCO_EINVAL, "unknown dtype %d", dtable_dtype);
  const size_t al = a->dtype == MULOCO_BF16 ? 2 : 4, out_al = dtable_dtype == MULOCO_BF16 ? 2 : 4;
  if (a->rows > 0 && (!dtable || misaligned(dtable, out_al))) return ctx_fail(c, MULOCO_EINVAL, "dtable is NULL or not aligned to its type");
  const CtxView v = ctx_view(c);
  if (a->tokens == 0) {
    if (a->rows > 0) BLOCK_CK(cudaMemsetAsync(dtable, 0, (size_t)a->rows * (size_t)a->d * out_al, v.st));
    return MULOCO_OK;
  }
  if (a->tokens > 1 && a->ld < a->d) return ctx_fail(c, MULOCO_ESHAPE, "row strides must be at least a row long");
  if (!dout || misaligned(dout, al)) return ctx_fail(c, MULOCO_EINVAL, "dout is NULL or not aligned to its type");
  if (!scratch || misaligned(scratch, 16)) return ctx_fail(c, MULOCO_EINVAL, "scratch is NULL or not 16-byte aligned");
  EmbeddingArgs e = embedding_args(a, v);
  e.dout = dout; e.dtable = dtable; e.scratch = scratch;
  int launches = 0;
  BLOCK_CK(launch_embedding_backward(v.st, e, a->dtype == MULOCO_BF16, dtable_dtype == MULOCO_BF16, &launches));
  ctx_count_launches(c, launches);
  return MULOCO_OK;
}

}  // extern "C"
