// C entry points of the operators that complete a decoder block: causal attention over packed sequences.
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
    return ctx_fail(c, MULOCO_ESHAPE, "the count of query heads must be a multiple of that of key heads (got %d, %d)", a->heads_q, a->heads_k);
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

MULOCO_API void muloco_sequences_destroy(muloco_sequences* s) { delete s; }

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
