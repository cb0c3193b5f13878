// C entry points of the operators around the optimizer: argument checks, tables, launches.
#include <math.h>
#include <string.h>

#include <new>
#include <vector>

#include "internal.h"

using namespace muloco;

namespace {

constexpr int GRAD_RING = 3;

#define OPS_CK(call)                                                                                  \
  do {                                                                                                \
    cudaError_t e_ = (call);                                                                          \
    if (e_ != cudaSuccess) return ctx_fail(c, MULOCO_ECUDA, "%s failed: %s", #call, cudaGetErrorString(e_)); \
  } while (0)

bool misaligned(const void* p, size_t a) { return (((uintptr_t)p) & (a - 1)) != 0; }

}  // namespace

struct muloco_adamw {
  muloco_ctx* ctx = nullptr;
  muloco_adamw_config cfg;
  int n = 0;
  int64_t n_units = 0;
  bool has_default = true;               // every tensor named a gradient at create time
  std::vector<int64_t> numel;
  AdamwUnit* d_units = nullptr;
  const void** d_grads = nullptr;        // gradients of the current step
  const void** h_grads[GRAD_RING] = {nullptr, nullptr, nullptr};
  cudaEvent_t ev[GRAD_RING] = {nullptr, nullptr, nullptr};
  bool used[GRAD_RING] = {false, false, false};
  int next = 0;
};

extern "C" {

MULOCO_API void muloco_adamw_destroy(muloco_adamw* o) {
  if (!o) return;
  const DeviceScope scope(ctx_device(o->ctx));
  cudaStreamSynchronize(ctx_view(o->ctx).st);
  if (o->d_units) cudaFree(o->d_units);
  if (o->d_grads) cudaFree(o->d_grads);
  for (int i = 0; i < GRAD_RING; ++i) {
    if (o->h_grads[i]) cudaFreeHost(o->h_grads[i]);
    if (o->ev[i]) cudaEventDestroy(o->ev[i]);
  }
  delete o;
}

MULOCO_API muloco_status muloco_adamw_create(muloco_ctx* c, const muloco_adamw_config* cfg,
                                             const muloco_adamw_tensor* t, int32_t n, muloco_adamw** out) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  if (!out) return ctx_fail(c, MULOCO_EINVAL, "out is NULL");
  *out = nullptr;
  if (!cfg) return ctx_fail(c, MULOCO_EINVAL, "config is NULL");
  if (n < 0 || (n > 0 && !t)) return ctx_fail(c, MULOCO_EINVAL, "bad tensor table");
  if (cfg->state_bits != 32 && cfg->state_bits != 8) return ctx_fail(c, MULOCO_EINVAL, "state_bits must be 32 or 8");
  if (cfg->grad_dtype != MULOCO_F32 && cfg->grad_dtype != MULOCO_BF16)
    return ctx_fail(c, MULOCO_EINVAL, "unknown grad_dtype %d", cfg->grad_dtype);
  if (!(cfg->beta1 >= 0.f && cfg->beta1 < 1.f) || !(cfg->beta2 >= 0.f && cfg->beta2 < 1.f))
    return ctx_fail(c, MULOCO_EINVAL, "beta1 and beta2 must be in [0, 1)");
  if (!(cfg->eps >= 0.f)) return ctx_fail(c, MULOCO_EINVAL, "eps must be >= 0");
  const bool q8 = cfg->state_bits == 8;
  const size_t g_align = cfg->grad_dtype == MULOCO_BF16 ? 2 : 4;
  int64_t units = 0, base = 0;
  for (int i = 0; i < n; ++i) {
    const muloco_adamw_tensor& d = t[i];
    if (d.n < 0 || d.n > ((int64_t)1 << 40)) return ctx_fail(c, MULOCO_ESHAPE, "tensor %d: bad element count", i);
    if (d.n == 0) continue;
    if (!d.theta || !d.state1 || !d.state2) return ctx_fail(c, MULOCO_EINVAL, "tensor %d: NULL parameters or state", i);
    if (q8 && (!d.scale1 || !d.scale2)) return ctx_fail(c, MULOCO_EINVAL, "tensor %d: 8-bit states need scales", i);
    if (misaligned(d.state1, 16) || misaligned(d.state2, 16))
      return ctx_fail(c, MULOCO_EINVAL, "tensor %d: states must be 16-byte aligned", i);
    if (misaligned(d.theta, 4) || misaligned(d.copy, 2) || misaligned(d.grad, g_align) || misaligned(d.scale1, 4) ||
        misaligned(d.scale2, 4))
      return ctx_fail(c, MULOCO_EINVAL, "tensor %d: a pointer is not aligned to its type", i);
    units += (d.n + ADAMW_UNIT - 1) / ADAMW_UNIT;
  }
  if (units >= ((int64_t)1 << 31)) return ctx_fail(c, MULOCO_ESHAPE, "too many elements for one list");

  muloco_adamw* o = nullptr;
  std::vector<AdamwUnit> table;
  try {
    o = new muloco_adamw();
    o->ctx = c;
    o->cfg = *cfg;
    o->n = n;
    o->numel.resize(n);
    table.resize((size_t)units);
    size_t at = 0;
    const size_t g_elt = cfg->grad_dtype == MULOCO_BF16 ? 2 : 4, s_elt = q8 ? 1 : 4;
    for (int i = 0; i < n; ++i) {
      const muloco_adamw_tensor& d = t[i];
      auto off = [](const void* p, size_t bytes) {
        return p ? const_cast<char*>(reinterpret_cast<const char*>(p)) + bytes : nullptr;
      };
      for (int64_t e = 0; e < d.n; e += ADAMW_UNIT) {
        AdamwUnit& u = table[at++];
        memset(&u, 0, sizeof u);
        u.theta = d.theta + e;
        u.copy = off(d.copy, (size_t)e * 2);
        u.grad = off(d.grad, (size_t)e * g_elt);
        u.s1 = off(d.state1, (size_t)e * s_elt);
        u.s2 = off(d.state2, (size_t)e * s_elt);
        u.scale1 = q8 ? d.scale1 + e / MULOCO_ADAMW_BLOCK : nullptr;
        u.scale2 = q8 ? d.scale2 + e / MULOCO_ADAMW_BLOCK : nullptr;
        u.first = e;
        u.dither_base = base + e;
        u.n = (int32_t)(d.n - e < ADAMW_UNIT ? d.n - e : ADAMW_UNIT);
        u.tensor = i;
        u.wd_mult = d.wd_mult;
        u.lr_mult = isnan(d.lr_mult) ? 1.f : d.lr_mult;
      }
      base += (d.n + MULOCO_ADAMW_BLOCK - 1) / MULOCO_ADAMW_BLOCK * MULOCO_ADAMW_BLOCK;
      if (d.n > 0 && !d.grad) o->has_default = false;
      o->numel[i] = d.n;
    }
  } catch (const std::bad_alloc&) {
    delete o;
    return ctx_fail(c, MULOCO_ENOMEM, "host tables of %d tensors", n);
  }
  o->n_units = units;
  auto bail = [&](cudaError_t e, const char* what) {
    const muloco_status s = ctx_fail(c, e == cudaErrorMemoryAllocation ? MULOCO_ENOMEM : MULOCO_ECUDA, "%s: %s", what,
                                     cudaGetErrorString(e));
    cudaGetLastError();
    muloco_adamw_destroy(o);
    return s;
  };
  if (units > 0) {
    cudaError_t e;
    if ((e = cudaMalloc(&o->d_units, table.size() * sizeof(AdamwUnit))) != cudaSuccess) return bail(e, "unit table");
    if ((e = cudaMalloc(&o->d_grads, n * sizeof(void*))) != cudaSuccess) return bail(e, "gradient table");
    if ((e = cudaMemcpy(o->d_units, table.data(), table.size() * sizeof(AdamwUnit), cudaMemcpyHostToDevice)) != cudaSuccess) return bail(e, "unit table");
    // the copy above may still be on its way from a staging buffer: the kernels read the table without waiting for anything
    if ((e = cudaStreamSynchronize(nullptr)) != cudaSuccess) return bail(e, "unit table");
    for (int i = 0; i < GRAD_RING; ++i) {
      if ((e = cudaMallocHost((void**)&o->h_grads[i], n * sizeof(void*))) != cudaSuccess) return bail(e, "pinned gradient table");
      if ((e = cudaEventCreateWithFlags(&o->ev[i], cudaEventDisableTiming)) != cudaSuccess) return bail(e, "event");
    }
  }
  *out = o;
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_adamw_step(muloco_adamw* o, const void* const* grads, int64_t step, float lr_scale) {
  if (!o) return MULOCO_EINVAL;
  muloco_ctx* c = o->ctx;
  ON_DEVICE(c);
  const CtxView v = ctx_view(c);
  if (step < 1) return ctx_fail(c, MULOCO_EINVAL, "step counts from 1 (got %lld)", (long long)step);
  if (!grads && !o->has_default) return ctx_fail(c, MULOCO_EINVAL, "no gradients given, and none named at create time");
  const size_t g_align = o->cfg.grad_dtype == MULOCO_BF16 ? 2 : 4;
  if (grads)
    for (int i = 0; i < o->n; ++i) {
      if (o->numel[i] > 0 && !grads[i]) return ctx_fail(c, MULOCO_EINVAL, "gradient of tensor %d is NULL", i);
      if (misaligned(grads[i], g_align)) return ctx_fail(c, MULOCO_EINVAL, "gradient of tensor %d is not aligned to its type", i);
    }
  if (o->n_units == 0) return MULOCO_OK;
  const void* const* table = nullptr;    // the gradients that the units name
  if (grads) {
    // the pinned slot is free again once the copy that used it has run
    const int r = o->next;
    if (o->used[r]) OPS_CK(cudaEventSynchronize(o->ev[r]));
    memcpy(o->h_grads[r], grads, o->n * sizeof(void*));
    OPS_CK(cudaMemcpyAsync(o->d_grads, o->h_grads[r], o->n * sizeof(void*), cudaMemcpyHostToDevice, v.st));
    OPS_CK(cudaEventRecord(o->ev[r], v.st));
    o->used[r] = true;
    o->next = (r + 1) % GRAD_RING;
    table = o->d_grads;
  }
  const muloco_adamw_config& f = o->cfg;
  const double bc1 = f.bias_correction ? 1.0 - pow((double)f.beta1, (double)step) : 1.0;
  const double bc2 = f.bias_correction ? 1.0 - pow((double)f.beta2, (double)step) : 1.0;
  AdamwStep a;
  a.lr = (float)((double)f.lr * (double)lr_scale);
  a.lr_wd = (float)((double)f.lr * (double)lr_scale * (double)f.weight_decay);
  a.beta1 = f.beta1; a.beta2 = f.beta2; a.eps = f.eps;
  a.inv_bc1 = (float)(1.0 / bc1);
  a.inv_sqrt_bc2 = (float)(1.0 / sqrt(bc2));
  a.dither = adamw_dither(f.seed, step);
  OPS_CK(launch_adamw_multi(v.st, o->d_units, table, o->n_units, f.state_bits, f.grad_dtype == MULOCO_BF16, a, v.status));
  ctx_count_launches(c, 1);
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_adamw_moments(muloco_adamw* o, float* m, float* v) {
  if (!o) return MULOCO_EINVAL;
  muloco_ctx* c = o->ctx;
  ON_DEVICE(c);
  if (o->cfg.state_bits != 8) return ctx_fail(c, MULOCO_EINVAL, "32-bit states are their own values");
  if (o->n_units == 0) return MULOCO_OK;
  if (!m || !v) return ctx_fail(c, MULOCO_EINVAL, "m or v is NULL");
  if (misaligned(m, 16) || misaligned(v, 16)) return ctx_fail(c, MULOCO_EINVAL, "m and v must be 16-byte aligned");
  const CtxView w = ctx_view(c);
  OPS_CK(launch_adamw_moments(w.st, o->d_units, o->n_units, m, v));
  ctx_count_launches(c, 1);
  return MULOCO_OK;
}

}  // extern "C"

namespace {

muloco_status check_qk(muloco_ctx* c, const muloco_qk_norm* a) {
  if (!a) return ctx_fail(c, MULOCO_EINVAL, "arguments are NULL");
  if (a->tokens < 0 || a->tokens >= ((int64_t)1 << 31)) return ctx_fail(c, MULOCO_ESHAPE, "tokens must be in 0..2^31-1");
  if (a->heads_q < 0 || a->heads_k < 0 || a->heads_q > 65536 || a->heads_k > 65536)
    return ctx_fail(c, MULOCO_ESHAPE, "head counts must be in 0..65536");
  if (a->head_dim < 2 || a->head_dim > QK_MAX_DIM || (a->head_dim & 1))
    return ctx_fail(c, MULOCO_ESHAPE, "head_dim must be even and in 2..%d (got %d)", QK_MAX_DIM, a->head_dim);
  if (a->rotary_dim < 0 || a->rotary_dim > a->head_dim || (a->rotary_dim & 1))
    return ctx_fail(c, MULOCO_ESHAPE, "rotary_dim must be even and in 0..head_dim (got %d)", a->rotary_dim);
  if (a->dtype != MULOCO_F32 && a->dtype != MULOCO_BF16) return ctx_fail(c, MULOCO_EINVAL, "unknown dtype %d", a->dtype);
  if (!(a->eps >= 0.f)) return ctx_fail(c, MULOCO_EINVAL, "eps must be >= 0");
  if (a->tokens > 0 && a->rotary_dim > 0) {
    if (!a->cos || !a->sin) return ctx_fail(c, MULOCO_EINVAL, "cos or sin is NULL");
    if (a->table_len < 1) return ctx_fail(c, MULOCO_ESHAPE, "the rotation's table is empty");
    if (!a->positions && a->table_len < a->tokens)
      return ctx_fail(c, MULOCO_ESHAPE, "the rotation's table has %lld rows for %lld tokens", (long long)a->table_len,
                      (long long)a->tokens);
  }
  const size_t al = a->dtype == MULOCO_BF16 ? 2 : 4;
  if (a->tokens > 0 && ((a->heads_q && (!a->q || misaligned(a->q, al))) || (a->heads_k && (!a->k || misaligned(a->k, al)))))
    return ctx_fail(c, MULOCO_EINVAL, "q or k is NULL or not aligned to its type");
  if (misaligned(a->gain_q, 4) || misaligned(a->gain_k, 4) || misaligned(a->cos, 4) || misaligned(a->sin, 4) ||
      misaligned(a->positions, 8))
    return ctx_fail(c, MULOCO_EINVAL, "a pointer is not aligned to its type");
  return MULOCO_OK;
}

QkArgs qk_args(const muloco_qk_norm* a, const CtxView& v) {
  QkArgs k;
  memset(&k, 0, sizeof k);
  k.t[0].x = a->q; k.t[0].gain = a->gain_q; k.t[0].heads = a->heads_q;
  k.t[0].x_ts = a->q_token_stride; k.t[0].x_hs = a->q_head_stride;
  k.t[1].x = a->k; k.t[1].gain = a->gain_k; k.t[1].heads = a->heads_k;
  k.t[1].x_ts = a->k_token_stride; k.t[1].x_hs = a->k_head_stride;
  k.tokens = a->tokens; k.table_len = a->table_len;
  k.cos = a->cos; k.sin = a->sin; k.positions = a->positions;
  k.dim = a->head_dim; k.rot = a->rotary_dim; k.interleaved = a->interleaved; k.eps = a->eps;
  k.status = v.status;
  return k;
}

muloco_status check_ffn(muloco_ctx* c, const muloco_ffn* a) {
  if (!a) return ctx_fail(c, MULOCO_EINVAL, "arguments are NULL");
  if (a->activation != MULOCO_ACT_SILU && a->activation != MULOCO_ACT_GELU)
    return ctx_fail(c, MULOCO_EINVAL, "unknown activation %d", a->activation);
  if (a->tokens < 0 || a->tokens > ((int64_t)1 << 30)) return ctx_fail(c, MULOCO_ESHAPE, "tokens must be in 0..2^30");
  if (a->d < 8 || a->F < 8 || (a->d & 7) || (a->F & 7) || a->d > (1 << 20) || a->F > (1 << 20))
    return ctx_fail(c, MULOCO_ESHAPE, "d and F must be multiples of 8 in 8..2^20 (got %lld, %lld)", (long long)a->d, (long long)a->F);
  if (a->ldx < a->d || a->ldw1 < a->F || a->ldw3 < a->F || a->ldw2 < a->d || ((a->ldx | a->ldw1 | a->ldw3 | a->ldw2) & 7))
    return ctx_fail(c, MULOCO_ESHAPE, "row strides must be multiples of 8 and at least a row long");
  if (a->tokens * ((a->d + a->F) / 128 + 2) > ((int64_t)1 << 36))
    return ctx_fail(c, MULOCO_ESHAPE, "too many tokens for one call");
  if (!a->w1 || !a->w3 || !a->w2 || (a->tokens > 0 && !a->x)) return ctx_fail(c, MULOCO_EINVAL, "a matrix is NULL");
  if (misaligned(a->x, 16) || misaligned(a->w1, 16) || misaligned(a->w3, 16) || misaligned(a->w2, 16))
    return ctx_fail(c, MULOCO_EINVAL, "matrices must be 16-byte aligned");
  return MULOCO_OK;
}

FfnArgs ffn_args(const muloco_ffn* a, const CtxView& v) {
  FfnArgs f;
  memset(&f, 0, sizeof f);
  f.T = a->tokens; f.d = a->d; f.F = a->F;
  f.x = a->x; f.ldx = a->ldx;
  f.w1 = a->w1; f.ldw1 = a->ldw1; f.w3 = a->w3; f.ldw3 = a->ldw3; f.w2 = a->w2; f.ldw2 = a->ldw2;
  f.act = a->activation;
  f.status = v.status; f.wait_limit_ns = v.wait_limit_ns; f.n_sms = v.n_sms;
  return f;
}

}  // namespace

extern "C" {

MULOCO_API muloco_status muloco_qk_norm_rope(muloco_ctx* c, const muloco_qk_norm* a, void* q_out, int64_t qo_ts,
                                             int64_t qo_hs, void* k_out, int64_t ko_ts, int64_t ko_hs) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  const muloco_status s = check_qk(c, a);
  if (s != MULOCO_OK) return s;
  if (a->tokens == 0 || a->heads_q + a->heads_k == 0) return MULOCO_OK;
  const size_t al = a->dtype == MULOCO_BF16 ? 2 : 4;
  if ((a->heads_q && (!q_out || misaligned(q_out, al))) || (a->heads_k && (!k_out || misaligned(k_out, al))))
    return ctx_fail(c, MULOCO_EINVAL, "q_out or k_out is NULL or not aligned to its type");
  if ((a->heads_q && q_out == a->q && (qo_ts != a->q_token_stride || qo_hs != a->q_head_stride)) ||
      (a->heads_k && k_out == a->k && (ko_ts != a->k_token_stride || ko_hs != a->k_head_stride)))
    return ctx_fail(c, MULOCO_EINVAL, "a result in place of its input needs the input's strides");
  const CtxView v = ctx_view(c);
  QkArgs k = qk_args(a, v);
  k.t[0].out = q_out; k.t[0].o_ts = qo_ts; k.t[0].o_hs = qo_hs;
  k.t[1].out = k_out; k.t[1].o_ts = ko_ts; k.t[1].o_hs = ko_hs;
  OPS_CK(launch_qk_norm(v.st, k, false, a->dtype == MULOCO_BF16, v.n_sms));
  ctx_count_launches(c, 1);
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_qk_norm_rope_backward(muloco_ctx* c, const muloco_qk_norm* a, const void* dq_out,
                                                      int64_t dqo_ts, int64_t dqo_hs, const void* dk_out,
                                                      int64_t dko_ts, int64_t dko_hs, void* dq, void* dk,
                                                      float* dgain_q, float* dgain_k) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  const muloco_status s = check_qk(c, a);
  if (s != MULOCO_OK) return s;
  const CtxView v = ctx_view(c);
  const bool some = a->tokens > 0;
  const size_t al = a->dtype == MULOCO_BF16 ? 2 : 4;
  if (some && ((a->heads_q && (!dq_out || !dq || misaligned(dq_out, al) || misaligned(dq, al))) ||
               (a->heads_k && (!dk_out || !dk || misaligned(dk_out, al) || misaligned(dk, al)))))
    return ctx_fail(c, MULOCO_EINVAL, "a gradient is NULL or not aligned to its type");
  if (misaligned(dgain_q, 4) || misaligned(dgain_k, 4)) return ctx_fail(c, MULOCO_EINVAL, "a pointer is not aligned to its type");
  // a gain that no head uses has a zero gradient
  if (dgain_q && !(some && a->heads_q)) OPS_CK(cudaMemsetAsync(dgain_q, 0, a->head_dim * sizeof(float), v.st));
  if (dgain_k && !(some && a->heads_k)) OPS_CK(cudaMemsetAsync(dgain_k, 0, a->head_dim * sizeof(float), v.st));
  if (!some || a->heads_q + a->heads_k == 0) return MULOCO_OK;
  QkArgs k = qk_args(a, v);
  k.t[0].dy = dq_out; k.t[0].y_ts = dqo_ts; k.t[0].y_hs = dqo_hs; k.t[0].out = dq; k.t[0].dgain = dgain_q;
  k.t[1].dy = dk_out; k.t[1].y_ts = dko_ts; k.t[1].y_hs = dko_hs; k.t[1].out = dk; k.t[1].dgain = dgain_k;
  for (QkTensor& t : k.t) { t.o_hs = a->head_dim; t.o_ts = (int64_t)t.heads * a->head_dim; }
  k.partials = ctx_qk_scratch(c, &k.tickets);
  OPS_CK(launch_qk_norm(v.st, k, true, a->dtype == MULOCO_BF16, v.n_sms));
  ctx_count_launches(c, 1);
  return MULOCO_OK;
}

MULOCO_API muloco_status muloco_gated_ffn(muloco_ctx* c, const muloco_ffn* a, void* g, void* u, void* h, void* y) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  const muloco_status s = check_ffn(c, a);
  if (s != MULOCO_OK) return s;
  if (a->tokens == 0) return MULOCO_OK;
  if (!h || !y) return ctx_fail(c, MULOCO_EINVAL, "h or y is NULL");
  if (misaligned(g, 16) || misaligned(u, 16) || misaligned(h, 16) || misaligned(y, 16))
    return ctx_fail(c, MULOCO_EINVAL, "matrices must be 16-byte aligned");
  const CtxView v = ctx_view(c);
  FfnArgs f = ffn_args(a, v);
  f.g = g; f.u = u; f.h = h; f.y = y;
  f.withhold = ctx_take_withhold(c);
  int n = 0;
  const char* what = "";
  const cudaError_t e = launch_ffn(v.st, f, &n, &what);
  ctx_count_launches(c, n);
  if (e != cudaSuccess) return ctx_fail(c, MULOCO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
  return MULOCO_OK;
}

MULOCO_API int32_t muloco_debug_ffn_forms(int64_t tokens, int64_t d, int64_t F, int32_t n_sms, int64_t* tiles) {
  return ffn_forms(tokens, d, F, n_sms, tiles);
}

MULOCO_API muloco_status muloco_gated_ffn_backward(muloco_ctx* c, const muloco_ffn* a, const void* dy, int64_t lddy,
                                                   const void* g, const void* u, const void* h, void* dg, void* du,
                                                   void* dx, void* dw1, void* dw3, void* dw2) {
  if (!c) return MULOCO_EINVAL;
  ON_DEVICE(c);
  const muloco_status s = check_ffn(c, a);
  if (s != MULOCO_OK) return s;
  if (misaligned(dx, 16) || misaligned(dw1, 16) || misaligned(dw3, 16) || misaligned(dw2, 16))
    return ctx_fail(c, MULOCO_EINVAL, "matrices must be 16-byte aligned");
  const CtxView v = ctx_view(c);
  if (a->tokens == 0) {                       // no token: the sums over tokens are empty
    const size_t bytes = (size_t)a->d * (size_t)a->F * 2;
    if (dw1) OPS_CK(cudaMemsetAsync(dw1, 0, bytes, v.st));
    if (dw3) OPS_CK(cudaMemsetAsync(dw3, 0, bytes, v.st));
    if (dw2) OPS_CK(cudaMemsetAsync(dw2, 0, bytes, v.st));
    return MULOCO_OK;
  }
  if (!dy || !g || !u || !h) return ctx_fail(c, MULOCO_EINVAL, "dy or a tensor of the forward pass is NULL");
  if ((dx || dw1 || dw3) && (!dg || !du)) return ctx_fail(c, MULOCO_EINVAL, "dg or du is NULL");
  if (lddy < a->d || (lddy & 7)) return ctx_fail(c, MULOCO_ESHAPE, "row strides must be multiples of 8 and at least a row long");
  if (misaligned(dy, 16) || misaligned(g, 16) || misaligned(u, 16) || misaligned(h, 16) || misaligned(dg, 16) || misaligned(du, 16))
    return ctx_fail(c, MULOCO_EINVAL, "matrices must be 16-byte aligned");
  FfnArgs f = ffn_args(a, v);
  f.dy = dy; f.lddy = lddy;
  f.g = const_cast<void*>(g); f.u = const_cast<void*>(u); f.h = const_cast<void*>(h);
  f.dg = dg; f.du = du; f.dx = dx; f.dw1 = dw1; f.dw3 = dw3; f.dw2 = dw2;
  f.withhold = ctx_take_withhold(c);
  int n = 0;
  const char* what = "";
  const cudaError_t e = launch_ffn_backward(v.st, f, &n, &what);
  ctx_count_launches(c, n);
  if (e != cudaSuccess) return ctx_fail(c, MULOCO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
  return MULOCO_OK;
}

}  // extern "C"
