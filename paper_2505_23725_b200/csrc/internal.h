// Internal declarations shared by the CUDA translation units of libmuloco.
#pragma once
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <stdint.h>

#include "../../include/muloco.h"
#include "device_scope.h"

namespace muloco {

// Device status word bits (OR-ed by kernels, read by muloco_sync_status).
enum : int { ST_NONFINITE = 1, ST_TIMEOUT = 2, ST_BOUNDS = 4, ST_POSITION = 8, ST_TOKEN = 16 };

// Debug build (-DMULOCO_DEBUG): kernels check the indices they derive (work-list cursors, matrix
// slots, tile coordinates, segment and unit indices) before using them; a failed check raises
// ST_BOUNDS in the status word and the thread skips the access (nothing traps).  In the regular
// build the checks compile to nothing.
#ifdef MULOCO_DEBUG
#define MULOCO_IN_BOUNDS(cond, status) ((cond) ? true : (atomicOr((status), ::muloco::ST_BOUNDS), false))
#else
#define MULOCO_IN_BOUNDS(cond, status) (true)
#endif

// ---------------------------------------------------------------------------
// Muon path: one entry per (worker, hidden matrix) of a chunk.
// The Newton-Schulz workspace always holds X as s x l with s <= l; a matrix
// stored with rows > cols enters and leaves through its transpose.
// ---------------------------------------------------------------------------
struct MatDesc {
  const void* g;   // gradient (fp32 or bf16), tensor layout rows x cols; or raw X for the standalone call
  float* m;        // Muon momentum (fp32), tensor layout; NULL for the standalone call
  void* w;         // parameters W (fp32, updated in place) or output O of the standalone call
  float lr_eff;    // eta' = lr * lr_scale * lr_mult
  float wd_term;   // eta_wd * lambda * wd_mult (multiplies W)
  int32_t transposed;  // 1: tensor is l x s (rows > cols)
  int32_t pad;
  const void* wmap;    // device address of a 128-byte TMA descriptor over W (32 x 32 fp32 boxes) for the
                       // fused parameter update of the tensor-core engine, or NULL (plain accesses)
};

enum SrcMode : int { SRC_MUON = 0, SRC_RAW_F32 = 1, SRC_RAW_BF16 = 2 };
enum SinkMode : int { SINK_UPDATE_W = 0, SINK_STORE_F32 = 1, SINK_STORE_BF16 = 2 };

// prologue: m <- beta m + g; U -> workspace X (bf16 or fp32, s x ldx per slot); partial sums of U^2.
// partial layout: partials[slot * n_part + tile], n_part = ceil(s/32) * ceil(l/128).
void launch_prologue(cudaStream_t st, const MatDesc* mats, int n_mats, int64_t s, int64_t l,
                     int src_mode, int g_is_bf16, float beta, int nesterov, void* X, int x_is_f32,
                     int64_t ldx, float* partials);
int prologue_partials_per_matrix(int64_t s, int64_t l);
// scales[slot] = { r*r, r } with r = 1 / (sqrt(sum partials) + eps)
void launch_finalize_scales(cudaStream_t st, const float* partials, int n_part, int n_mats,
                            float eps, float2* scales, int* status = nullptr);

// fp32 Newton-Schulz engine (CUDA cores).  One call = one of the three products
// of an iteration for all matrices of a chunk.
enum GemmKind : int { GEMM_GRAM = 0, GEMM_POLY = 1, GEMM_APPLY = 2, GEMM_FINAL = 3 };
struct NsIterArgs {
  float a, b, c;            // quintic coefficients
  const float2* scales;     // per-slot {r^2, r}; NULL: no scaling in this call
  const MatDesc* mats;      // for GEMM_FINAL (sink)
  int sink_mode;
  int* status;
  unsigned long long wait_limit_ns = 0;   // tensor-core engine: limit of every device-side wait (0: 2 s)
  int debug_withhold = 0;                 // tensor-core engine, test hook: one operand copy is never issued
};
void launch_ns_fp32(cudaStream_t st, int kind, int n_mats, int64_t s, int64_t l, const float* X,
                    int64_t ldx, const float* A, const float* B, int64_t lds, float* Aout,
                    float* Bout, float* Xout, const NsIterArgs& args);

// bf16 tensor-core engine (tcgen05 / TMEM / TMA); see ns_tc.cu.  One launch runs all products of
// all iterations for the matrices of a chunk; the staged input X0 is chunk-sized, the
// intermediates live in a ring of tc_ring_slots(group) slots.
struct TcGroupPlan;   // opaque per-shape-group plan (tensor maps, tile lists, work lists)
// matrices per group of the work list for min-dimension s (never more than `chunk`)
int tc_group_size(int64_t s, int chunk);
// ring slots for groups of `group` matrices; bytes of the ring (X', X'', A, B for n_slots matrices, bf16)
int tc_ring_slots(int group);
size_t tc_ring_bytes(int64_t s, int64_t ldx, int64_t lds, int n_slots);
// counters: chunk * 3 * ns_steps + 1 ints (tile counters and the ticket counter; zeroed by every launch)
TcGroupPlan* tc_plan_create(int64_t s, int64_t l, int chunk, void* X0, int64_t ldx, void* ring, int64_t lds,
                            int group, int* counters, int ns_steps, char* err, size_t errlen);
void tc_plan_destroy(TcGroupPlan*);
// the whole iteration for the first n_mats matrices of the chunk (args.scales: per-matrix {r^2, r})
cudaError_t tc_launch(cudaStream_t st, TcGroupPlan* plan, int n_mats, const NsIterArgs& args);
int tc_num_sms();
// Encodes (into 128 bytes at `out_host`) the TMA descriptor of a rows x cols fp32 tensor for 32 x 32
// boxes; swizzled for tensors stored s x l, plain for tensors stored l x s.  False when the tensor
// cannot be addressed by TMA (base not 16-byte aligned or cols not a multiple of 4).
bool tc_encode_w_map(void* out_host, void* base, int64_t rows, int64_t cols, int transposed);
constexpr size_t TC_MAP_BYTES = 128;

// AdamW: one entry per (worker, tensor).
struct AdamSeg {
  const void* g;
  float* m;
  float* v;
  float* theta;
  int64_t n;
  int64_t unit_begin;   // first work unit (of ADAM_UNIT elements) of this segment
  float lr;             // alpha
  float lr_wd;          // alpha * lambda * wd_mult
  float inv_bc1;        // 1 / (1 - beta1^t) (1 if no bias correction)
  float inv_sqrt_bc2;   // 1 / sqrt(1 - beta2^t)
};
constexpr int ADAM_UNIT = 2048;
// status: device status word; a non-finite gradient raises ST_NONFINITE (NULL: not checked)
void launch_adamw(cudaStream_t st, const AdamSeg* segs, int n_segs, int64_t n_units, int g_is_bf16,
                  float beta1, float beta2, float eps, int* status);

// Outer sync: one entry per tensor of the fragment.
struct SyncSeg {
  float* theta_g;
  float* u;
  int64_t rows, cols;
  int64_t nblk;         // blocks per row
  int64_t unit_begin;   // first block-unit of this segment
  int64_t rep_index;    // index of this tensor's first replica pointer in the replica table
};
// ef: table of error-feedback accumulators laid out like `replicas` (NULL: no error feedback);
// stages 2 selects the per-worker quantisation of Algorithm 2.
void launch_outer_sync(cudaStream_t st, const SyncSeg* segs, int n_segs, float* const* replicas,
                       int K, int64_t n_units, int block, int quant_bits, float outer_lr,
                       float mu, int* status, int n_sms, int stages = 1, float* const* ef = nullptr,
                       float ef_beta = 1.0f);
// Row-wise quantisation (quant_block == 0): units are rows (SyncSeg.nblk == 1); max_cols is the
// longest row of the fragment.  cudaErrorInvalidValue when a row does not fit shared memory.
cudaError_t launch_outer_sync_rows(cudaStream_t st, const SyncSeg* segs, int n_segs, float* const* replicas,
                                   int K, int64_t n_rows, int64_t max_cols, int quant_bits, float outer_lr,
                                   float mu, int* status, int stages, float* const* ef, float ef_beta);
// K = 1, eta_out = 1, mu = 0, no compression: theta <- theta_1 (exactly), u <- theta - theta_1.
void launch_dp_sync(cudaStream_t st, const SyncSeg* segs, int n_segs, float* const* replicas, int64_t n_units,
                    int* status);
// Worker-sharded outer synchronisation (outer_sync.cu): the three passes around the caller's
// reduce-scatter and all-gather.  Staging buffers are unit-major, 128 floats per unit.
void launch_shard_delta(cudaStream_t st, const SyncSeg* segs, int n_segs, float* const* replicas, int K,
                        int64_t n_units, int block, int quant_bits, int stages, float* const* ef, float ef_beta,
                        float* stage, int* status);
void launch_shard_step(cudaStream_t st, const SyncSeg* segs, int n_segs, int64_t n_units, int64_t unit_begin,
                       int64_t unit_count, int block, int quant_bits, float outer_lr, float mu, float inv_k_total,
                       const float* reduced, float* theta_out, int* status);
void launch_shard_broadcast(cudaStream_t st, const SyncSeg* segs, int n_segs, float* const* replicas, int K,
                            int64_t n_units, int block, const float* theta_all, int* status);
// Top-k sparsification of the workers' deltas (topk.cu).  Scratch: one histogram of
// topk_hist_words_per_problem() words (zero between calls), one prefix word (the threshold key
// after a call) and one counter per (tensor, worker), indexed like the replica table.
// kk_seg[i] = how many entries segment i keeps.  Segments are flat (rows == 1, 128-element units).
// Returns the number of kernels launched.
struct TopkScratch {
  uint32_t* hist = nullptr;
  uint32_t* prefix = nullptr;
  uint32_t* remaining = nullptr;
};
size_t topk_hist_words_per_problem();
int launch_outer_sync_topk(cudaStream_t st, const SyncSeg* segs, int n_segs, float* const* replicas, int K,
                           int64_t n_units, float outer_lr, float mu, int* status, float* const* ef,
                           float ef_beta, const uint32_t* kk_seg, TopkScratch sc);
// Standalone: out = top-k(x) for one device array of n elements; seg_dev describes x as one flat
// segment (theta_g = x, rep_index = 0), kk_dev holds the count to keep.
int launch_topk_raw(cudaStream_t st, const SyncSeg* seg_dev, int64_t n, const float* x, float* out,
                    const uint32_t* kk_dev, TopkScratch sc, int* status);
void launch_pseudogradient(cudaStream_t st, const float* theta_g, float* const* replicas, int K,
                           int64_t n, float* psi_out);
void launch_quantize(cudaStream_t st, const float* psi, int64_t rows, int64_t cols, int block,
                     int bits, int8_t* codes, float* scales, float* dequant, int* status);
void launch_broadcast_init(cudaStream_t st, const float* src, float* const* dst_table, int K,
                           int64_t n);

// ---------------------------------------------------------------------------
// Operators of the training step around the optimizer (adamw.cu, qk_norm.cu, ffn.cu), entered through
// ops_capi.cu.
// ---------------------------------------------------------------------------

// What an entry point needs of its context.
struct CtxView {
  cudaStream_t st;
  int* status;
  int n_sms;
  unsigned long long wait_limit_ns;   // 0: the default
};
CtxView ctx_view(muloco_ctx* c);
muloco_status ctx_fail(muloco_ctx* c, muloco_status s, const char* fmt, ...);
void ctx_count_launches(muloco_ctx* c, int n);
int ctx_device(const muloco_ctx* c);
int ctx_take_withhold(muloco_ctx* c);               // MULOCO_DEBUG_WITHHOLD_COPY, which it clears
// First thing of every entry point that touches the device: the context's device is current until it returns.
#define ON_DEVICE(c)                                                                                          \
  const muloco::DeviceScope device_scope_(muloco::ctx_device(c));                                             \
  if (device_scope_.error() != cudaSuccess)                                                                   \
  return muloco::ctx_fail(c, MULOCO_ECUDA, "device %d: %s", muloco::ctx_device(c), cudaGetErrorString(device_scope_.error()))
// Scratch of the context that the reductions of qk_norm.cu use: QK_SCRATCH_FLOATS floats, then tickets
// (zero between launches).
float* ctx_qk_scratch(muloco_ctx* c, int** tickets);

// Programmatic dependent launch: a kernel launched so may start while the one before it in the stream still
// runs.  grid_wait: until that one is complete and its results can be seen.  grid_release: lets the next kernel start
// (if it was launched so; its own grid_wait holds it back).  Every kernel releases only after its wait, so
// whatever starts early knows everything before its predecessor complete.
#ifdef __CUDACC__
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... P, typename... A>
cudaError_t launch_dependent(void (*kernel)(P...), unsigned grid, unsigned threads, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
#endif

// AdamW over many tensors (include/muloco.h has the layout of the states): one entry per work unit of ADAMW_UNIT
// consecutive elements of a tensor, with everything a block needs, so that its first load names all the others.
constexpr int ADAMW_UNIT = 4 * MULOCO_ADAMW_BLOCK;
struct alignas(16) AdamwUnit {
  float* theta;          // of the unit's first element, like all pointers here
  void* copy;            // bf16 copy of the parameters, or NULL
  void* s1;
  void* s2;
  float* scale1;
  float* scale2;
  const void* grad;      // gradient named at create time, or NULL
  int64_t first;         // the unit's first element inside its tensor
  int64_t dither_base;   // ... and in the padded layout
  int32_t n;             // elements of the unit
  int32_t tensor;
  float wd_mult, lr_mult;
};
struct AdamwStep {
  float lr, lr_wd;       // alpha, alpha * lambda
  float beta1, beta2, eps;
  float inv_bc1, inv_sqrt_bc2;
  uint32_t dither;
};
uint32_t adamw_dither(uint32_t seed, int64_t step);   // what step `step` adds to the element index before hashing
// grads[tensor]: the gradients of this step, or NULL for those in the units
cudaError_t launch_adamw_multi(cudaStream_t st, const AdamwUnit* units, const void* const* grads, int64_t n_units,
                        int state_bits, int g_is_bf16, const AdamwStep& a, int* status);
cudaError_t launch_adamw_moments(cudaStream_t st, const AdamwUnit* units, int64_t n_units, float* m, float* v);

// Query / key norm with rotation.  One of the two tensors of a call:
struct QkTensor {
  const void* x;         // forward input (both passes)
  const void* dy;        // backward: gradient of the result
  void* out;             // forward: result; backward: gradient of x
  const float* gain;     // NULL: ones
  float* dgain;          // backward, or NULL
  int64_t x_ts, x_hs, y_ts, y_hs, o_ts, o_hs;   // token and head strides (elements) of x, dy, out
  int32_t heads, pad;
};
struct QkArgs {
  QkTensor t[2];
  int64_t tokens, table_len;
  const float* cos;
  const float* sin;
  const int64_t* positions;
  int32_t dim, rot, interleaved;
  float eps;
  int32_t pad;
  int* status;
  float* partials;       // backward: gain gradients of the thread blocks
  int* tickets;          // backward: QK_TICKETS of them, zero between launches
};
constexpr int QK_MAX_DIM = 512;
constexpr int QK_MAX_CTAS = 148 * 16;
constexpr int QK_JOIN = 16;                      // thread blocks whose gain sums are joined at a time
constexpr size_t QK_SCRATCH_FLOATS = (size_t)(QK_MAX_CTAS + 2 * (QK_MAX_CTAS / QK_JOIN)) * QK_MAX_DIM;
constexpr size_t QK_TICKETS = 2 * (QK_MAX_CTAS / QK_JOIN + 1);
static_assert(QK_MAX_CTAS % QK_JOIN == 0, "whole groups of blocks");
// one launch, or none when there is no token or head
cudaError_t launch_qk_norm(cudaStream_t st, const QkArgs& a, bool back, int is_bf16, int n_sms);

// Gated feed-forward block.
struct FfnArgs {
  int64_t T, d, F;
  const void* x; int64_t ldx;
  const void* w1; int64_t ldw1;
  const void* w3; int64_t ldw3;
  const void* w2; int64_t ldw2;
  int act;
  void* g; void* u; void* h; void* y;          // forward results; backward inputs (g, u, h)
  const void* dy; int64_t lddy;
  void* dg; void* du; void* dx; void* dw1; void* dw3; void* dw2;
  int* status;
  unsigned long long wait_limit_ns;
  int n_sms;
  int withhold;                                // test hook, of the call's first launch
};
cudaError_t launch_ffn(cudaStream_t st, const FfnArgs& a, int* launches, const char** what);
cudaError_t launch_ffn_backward(cudaStream_t st, const FfnArgs& a, int* launches, const char** what);
int ffn_forms(int64_t T, int64_t d, int64_t F, int n_sms, int64_t* tiles);   // muloco_debug_ffn_forms

// Causal attention over packed sequences: the tiles of a batch, 128 tokens each (pair_tiles: up to 256), heaviest first.
constexpr int ATTN_TILE = 128, ATTN_MAX_DIM = 128;
struct alignas(16) AttnTile {
  int32_t start;         // first token of the sequence
  int32_t offset;        // first token of the tile in the sequence
  int32_t length;        // of the sequence
  int32_t pad;
};
struct AttnArgs {
  const AttnTile* pair_tiles;                  // forward: query tiles of 256
  const AttnTile* query_tiles;                 // backward: query tiles of 128, key tiles of 128
  const AttnTile* key_tiles;
  int64_t n_pairs, n_tiles;
  int64_t tokens;
  int32_t heads, kv_heads, dim;
  float scale;
  const void* q; int64_t q_ts, q_hs;           // token and head strides (elements)
  const void* k; int64_t k_ts, k_hs;
  const void* v; int64_t v_ts, v_hs;
  void* o_out;                                 // forward: o, dense
  float* lse;                                  // [heads][tokens]: written forward, read backward
  const void* o;                               // backward
  const void* g; int64_t g_ts, g_hs;           // do
  float* delta;                                // scratch [heads][tokens]
  void* dq; void* dk; void* dv;                // dense
  int* status;
  unsigned long long wait_limit_ns;
  int withhold;
};
cudaError_t launch_attention(cudaStream_t st, const AttnArgs& a, const char** what);            // one launch
cudaError_t launch_attention_backward(cudaStream_t st, const AttnArgs& a, const char** what);   // two

// Norm over the last dimension.
struct NormArgs {
  int64_t tokens, ldx, ldr, ldy;               // row strides of x, of residual | dh, of dy (the other tensors are dense)
  const void* x;                               // backward: h
  const void* residual;                        // or NULL
  void* h;                                     // forward, with a residual
  void* y;
  const float* weight;                         // NULL: ones
  const float* bias;                           // NULL: zeros
  float* mean;                                 // written forward, read backward (centred)
  float* rstd;
  const void* dy; const void* dh;              // backward; dh or NULL
  void* dx;
  float* dweight; float* dbias;                // or NULL
  float* partials;                             // [NORM_PARTS][2][d], when dweight or dbias is wanted
  int32_t d, center;
  float eps, inv_d;
};
constexpr int NORM_PARTS = MULOCO_NORM_PARTS, NORM_MAX_DIM = 32768;
cudaError_t launch_norm(cudaStream_t st, const NormArgs& a, bool back, int is_bf16, int n_sms, int* launches);

// Embedding lookup.
constexpr int EMB_SORT_BLOCK = 512, EMB_MERGE = 8, EMB_CHUNK = 16;
struct EmbeddingArgs {
  int64_t tokens, rows, ld;                    // ld: row stride of the table (forward), of dout (backward)
  const int64_t* ids;
  const void* table; void* out;                // forward
  const void* dout; void* dtable;              // backward
  void* scratch;                               // embedding_scratch() bytes
  float* partials;                             // in scratch: two partial sums per chunk, d_pad columns each
  int32_t d, d_pad;
  float scale;
  int* status;
};
size_t embedding_scratch(int64_t tokens, int64_t d);
cudaError_t launch_embedding(cudaStream_t st, const EmbeddingArgs& a, int is_bf16);             // one launch
cudaError_t launch_embedding_backward(cudaStream_t st, const EmbeddingArgs& a, int in_bf16, int out_bf16, int* launches);

}  // namespace muloco
