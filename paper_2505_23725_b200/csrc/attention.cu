// Causal attention over packed sequences with shared key heads, forward and backward, on the 5th-generation tensor cores.
//
//   s_ij = scale q_i . k_j  for j <= i of the same sequence,   p = softmax_j s,   o_i = sum_j p_ij v_j,   lse_i = ln sum_j e^s_ij
//   backward, from do:  dv_j = sum_i p_ij do_i,   dp_ij = do_i . v_j,   delta_i = do_i . o_i,   ds = p (dp - delta),
//                       dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i     (dk, dv summed over the group's query heads)
//
// Tiles are 128 tokens of one sequence and one head; the host lays the tiles of a batch out once, heaviest first
// (AttnTile).  Scores never reach memory: a tile of 128 x 128 lies in tensor memory, the threads of a row read it, and what they
// make of it (p or ds) goes back over the scores' columns, rounded to bf16 as the left operand of the next product, which takes it
// from there: that rounding costs as much as the result's own (error of dq against 64 bits 2.4e-3, of a single rounding 1.7e-3).  Rows that several products contract over (v, and in the
// backward pass k, q, do) are zeroed past the end of their sequence in shared memory: there the tile holds
// the next sequence's tokens, whose weight is zero but which may be anything, infinities and NaN too.
//
// Forward: two tiles of 128 queries per thread block take turns, so that the exponentials of one run beside the
// products of the other.  Weights are taken relative to a score that starts as the row's largest of the first key tile and is
// moved (and the sums rescaled) only when the weights of 64 keys add up to more than MOST: the quotient does not depend on it, sums stay far
// inside float32, and the largest score need not be looked for at every tile, a fifth of what a row warp did (11 % of the time).
//
// Backward: two kernels, without atomics, so results do not depend on the order of thread blocks.  The first goes over the keys of a
// query tile (delta, dq), the second over the queries of a key tile with the scores transposed (dk, dv):
// seven products instead of the five that one kernel with sums in global memory would take, and no float32 copy of dq.
//
// Measured (us, among other calls; in brackets in bursts of one call; credited TFLOP/s: 4 and 10 operations per pair, head and entry):
//   8 x 2048 tokens, 16 heads of 128    forward 184 (157 to 175) 749    backward 625 (540 to 580) 550
//   1 x 16384, 16 + 4 heads of 128      forward 1002 (860 to 980) 1098  backward (3290 to 3450)
//   8 x 2048, 16 heads of 64            forward (122 to 143)            backward (435 to 460)
// The moved reference costs the scores read twice more and the sums rewritten: where scores rise along the keys so that it moves at every
// tile, in bursts 268 instead of 157, 1654 instead of 972, 222 instead of 143 (forward, the three lines above); one move in a row 3 %.
// Long sequences with heads of 128 run near the power limit.  Elsewhere a step's chain binds: scores to tensor memory, row warps, weights
// back, products: about 3200 cycles for two forward tiles whose products take 2048 and exponentials 2048, and a unit's end (8000 cycles: last
// product, results to memory, first scores of the next).  Counters, tensor pipe / exponentials: 57 / 57 % with one sequence of 8192 tokens, 44 / 45 %
// with 8 x 2048 (products take 120 thousand of 295 thousand cycles), where units' ends weigh more.
// 96 registers a thread, the most that 576 threads may have: attn_fwd_kernel<128> spills 108 bytes (348 of loads), <64> 28, the others up to 8.
// Tried and dropped: half to all of the exponentials' load on the floating-point pipes (polynomial of degree 5: 5 to 20 % slower, the
// pipe is not what is waited for); one thread per row with registers moved between warpgroups (904 against 857); in the backward
// pass two groups of row warps on alternate steps (682 against 545: a step of a single warp takes twice as long), and dp of the
// next key tile before dq of this one (590 against 556).
#include <string.h>

#include "internal.h"
#include "rows.cuh"
#include "tc_ptx.cuh"

namespace muloco {

namespace {

constexpr int TILE = 128;                     // tokens per tile
constexpr int ATTN_THREADS = 576;             // sixteen warps for the rows, one for copies, one for products
constexpr int ROW_WARPS = 16, COPY_WARP = 16, MMA_WARP = 17;
constexpr uint32_t SLAB = TILE * 128;         // 128 rows of 64 bf16, swizzled
// The columns of a tile are divided among row warps (forward in halves, backward in quarters); each writes its bf16 operand at the
// start of its own columns, so none overwrites scores that another has yet to read.
constexpr uint32_t HALF = 64, QUARTER = 32;
// Of L2's 126 MB: what a section's units read again and again (16, 32, 64 MB: 168, 168, 174 us for 8 x 2048 tokens, 16 heads of 128).
constexpr int64_t SECTION_BYTES = 32 << 20;
constexpr float LN2 = 0.6931471805599453f, LOG2_E = 1.4426950408889634f;
// Steps from its end at which a unit asks for the next: the answer and the first copies are there in time, and the last units are still shared
// out late (1, 2, 3, a whole unit ahead: 181, 180, 178, 184 us forward, 581, 579, 579, 589 backward).
constexpr int ASK_AHEAD = 3;
constexpr float MOST = 65536.0f;              // sum of 64 weights that makes a row's reference move

struct Maps4 { CUtensorMap q, k, v, g; };     // g: do

struct AttnParams {
  const AttnTile* tiles;
  int n_tiles, section;                       // section: heads whose units come together (query heads, or key heads for dk and dv)
  int64_t tokens;
  int heads, group;                           // query heads; of them per key head
  int dim;
  float scale;
  void* out; void* out2;                      // o | dq | dk, dv
  float* lse;                                 // [heads][tokens]
  float* delta;                               // [heads][tokens]
  const void* o; const void* g;               // backward: o (dense), do
  int64_t g_ts, g_hs;                         // strides of do
  int* status;
  unsigned long long wait_limit_ns;
  int withhold;                               // test hook: the first thread block issues no copies
};

// ----------------------------- tensor memory --------------------------------
__device__ __forceinline__ void tm_store32(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
      "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]),
      "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]),
      "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]),
      "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tm_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Behind tc_ld32, which waits for its load: nothing that uses v is moved in front of this.
__device__ __forceinline__ void after_load(uint32_t* v) {
  asm volatile(""
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                 "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]),
                 "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]),
                 "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]),
                 "+r"(v[30]), "+r"(v[31]));
}

// The products' warp runs as one: every lane goes through the same code and the instructions themselves are carried out by the lane that
// `leader` is 1 in.  In code that only one lane enters, the descriptors are moved to the warp's registers one by one:
// 86 cycles a product where the tensor cores need 32 to 64.
__device__ __forceinline__ uint32_t elect_leader() {
  uint32_t leader;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "elect.sync _|p, 0xffffffff;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(leader));
  return leader;
}
// D (tensor memory) = or += A B^T, A and B in shared memory
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "setp.ne.b32 q, %5, 0;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
// ... with A (bf16, two to a column) in tensor memory
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "setp.ne.b32 q, %5, 0;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t leader, uint32_t bar) {
  asm volatile(
      "{\n"
      ".reg .pred q;\n"
      "setp.ne.b32 q, %1, 0;\n"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n"
      "}\n" ::"r"(bar), "r"(leader)
      : "memory");
}

// Operands in shared memory: DP / 64 slabs of 128 rows of 64 entries.  As K-major operand its rows are the 128 rows or columns of the
// result and the contraction runs over the entries; as MN-major operand (right side only) the contraction runs over the
// 128 rows and the entries are the result's columns.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
constexpr uint32_t LBO_K = (16u >> 4) << 16, LBO_MN = (SLAB >> 4) << 16;
__device__ __forceinline__ uint64_t desc(uint32_t lo) { return ((uint64_t)DESC_HI << 32) | lo; }
constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TILE >> 4) << 24);
__host__ __device__ constexpr uint32_t idesc_k(int n) { return IDESC | ((uint32_t)(n >> 3) << 17); }
__host__ __device__ constexpr uint32_t idesc_mn(int n) { return idesc_k(n) | (1u << 16); }

// d[128][128] = a b^T over DP entries
template <int DP>
__device__ __forceinline__ void scores(uint32_t leader, uint32_t d, uint32_t a, uint32_t b) {
#pragma unroll
  for (int k = 0; k < DP / 16; ++k) {
    const uint32_t off = (uint32_t)(k >> 2) * (SLAB >> 4) + (uint32_t)(k & 3) * 2u;
    mma_ss(leader, d, desc(((a >> 4) | LBO_K) + off), desc(((b >> 4) | LBO_K) + off), idesc_k(TILE), k > 0);
  }
}
// d[128][DP] += p b over rows 64 h .. 64 h + 63 of b; p: those 64 columns of the left operand
template <int DP>
__device__ __forceinline__ void weigh_half(uint32_t leader, uint32_t d, uint32_t p, uint32_t b, int h, bool accumulate) {
#pragma unroll
  for (int k = 0; k < 4; ++k)
    mma_ts(leader, d, p + (uint32_t)k * 8u, desc(((b >> 4) | LBO_MN) + (uint32_t)(4 * h + k) * 128u), idesc_mn(DP), accumulate || k > 0);
}
// ... over its 128 rows, p in quarters
template <int DP>
__device__ __forceinline__ void weigh(uint32_t leader, uint32_t d, uint32_t p, uint32_t b, bool accumulate) {
#pragma unroll
  for (int k = 0; k < TILE / 16; ++k)
    mma_ts(leader, d, p + (uint32_t)(k >> 1) * QUARTER + (uint32_t)(k & 1) * 8u, desc(((b >> 4) | LBO_MN) + (uint32_t)k * 128u), idesc_mn(DP),
           accumulate || k > 0);
}

// Rows `first` .. 127 of an operand become zero (one warp); the products that follow see it.
template <int DP>
__device__ __forceinline__ void zero_rows(uint32_t b, int first, int lane) {
  const int n = (TILE - first) * 8;
#pragma unroll 1
  for (int s = 0; s < DP / 64; ++s)
#pragma unroll 1
    for (int i = lane; i < n; i += 32) sts128(b + (uint32_t)s * SLAB + (uint32_t)(first * 128 + i * 16), make_uint4(0u, 0u, 0u, 0u));
  fence_async_smem();
  __syncwarp();
}

template <int DP>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int row) {
#pragma unroll
  for (int s = 0; s < DP / 64; ++s) tma_load_3d(dst + (uint32_t)s * SLAB, map, bar, s * 64, head, row);
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The largest of three; NaN if one is.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Accumulator columns [c0, c0 + n) of this thread's row, times `by`, as bf16 to columns c0 .. of `row` (first `dim` columns exist).
__device__ __forceinline__ void store_columns(uint32_t t_row, __nv_bfloat16* row, int c0, int n, int dim, float by, bool row_ok,
                                              bool wide) {
#pragma unroll 1
  for (int c = c0; c < c0 + n; c += 32) {
    uint32_t v[32];
    float f[32];
    __syncwarp();
    tc_ld32(t_row + (uint32_t)c, v);
    after_load(v);
#pragma unroll
    for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(v[e]) * by;
    const int left = row_ok ? dim - c : 0;
    if (left > 0) store_row32(row + c, f, left, wide);
  }
}

// Units of work: a tile (forward: a pair of tiles) and a head.  The grid has a block per unit; a block that is done with its own
// takes over one that has not started yet (cluster launch control), so units start in the order of the grid as multiprocessors become free, and
// copies and scores of the next unit run beside the end of this one.  The order: heads in sections whose keys and
// values fit into L2 together, the tiles of a section heaviest first.
struct Unit { AttnTile tile; int head; };
__device__ __forceinline__ Unit unit_of(const AttnParams& p, int heads, int u) {
  const int per = p.n_tiles * p.section, s = u / per, r = u - s * per;
  const int left = heads - s * p.section, width = left < p.section ? left : p.section;
  Unit x;
  x.tile = p.tiles[r / width];
  x.head = s * p.section + r % width;
  return x;
}

// Whether any thread of the warps that share a tile's rows says so (barrier `id`, THREADS in all; they take the same turns).
template <int THREADS>
__device__ __forceinline__ bool any_of(int id, bool x) {
  uint32_t r;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.b32 p, %1, 0;\n"
      "barrier.cta.red.or.pred q, %2, %3, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(r)
      : "r"((uint32_t)x), "r"(id), "n"(THREADS)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ bool either(int id, bool x) { return any_of<64>(id, x); }

// The next unit, asked for by the copying thread and read by every warp, through two places in turn.
struct Next {
  uint32_t full, empty, answer;               // barriers (8 bytes a place), answers (16)
  uint32_t turn = 0;
  __device__ __forceinline__ uint32_t place() const { return turn & 1u; }
  __device__ __forceinline__ uint32_t parity() const { return (turn >> 1) & 1u; }
};
__device__ __forceinline__ bool ask(const Next& n, volatile int* abort_flag, uint64_t limit) {
  if (!mbar_wait_cta(n.empty + n.place() * 8u, n.parity() ^ 1u, abort_flag, limit)) return false;
  const uint32_t bar = n.full + n.place() * 8u;
  mbar_expect_tx(bar, 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(n.answer + n.place() * 16u),
               "r"(bar)
               : "memory");
  return true;
}
// A warp's (or the copying thread's) next unit: -1 when there is none, -2 when the block is giving up.
template <bool WARP>
__device__ __forceinline__ int take(Next& n, volatile int* abort_flag, uint64_t limit) {
  bool ok = mbar_wait_cta(n.full + n.place() * 8u, n.parity(), abort_flag, limit);
  if (WARP) ok = __all_sync(0xffffffffu, ok);
  if (!ok) return -2;
  int u;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      ".reg .b128 a;\n"
      "ld.shared.b128 a, [%1];\n"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n"
      "mov.b32 %0, -1;\n"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, a;\n"
      "}\n"
      : "=r"(u)
      : "r"(n.answer + n.place() * 16u)
      : "memory");
  fence_async_smem();                         // the next answer to this place comes behind these reads
  if (WARP) __syncwarp();
  if (!WARP || (threadIdx.x & 31) == 0) mbar_arrive_cta(n.empty + n.place() * 8u);
  ++n.turn;
  return u;
}

// The next unit of warps that meet at barrier `id`: all go on or none does.
template <int THREADS>
__device__ __forceinline__ int take_together(Next& n, int id, volatile int* abort_flag, uint64_t limit) {
  const int u = take<true>(n, abort_flag, limit);
  return any_of<THREADS>(id, u == -2) ? -2 : u;
}

struct Pipe {                                 // position in a ring of N stages
  uint32_t stage = 0, phase = 0;
  template <int N> __device__ __forceinline__ void next() { if (++stage == (uint32_t)N) { stage = 0; phase ^= 1u; } }
};

// Start and end of every kernel: barriers, tensor memory, and the dependent launch.
#define ATTN_BEGIN(cols)                                                                     \
  if (threadIdx.x == 0) {                                                                    \
    abort_flag = 0;                                                                          \
    init_barriers();                                                                         \
    for (int i = 0; i < 2; ++i) {                                                            \
      mbar_init(smem_u32(&bar_next[i]), 1);                                                  \
      mbar_init(smem_u32(&bar_taken[i]), 2 + ROW_WARPS);                                     \
    }                                                                                        \
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");                       \
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");                             \
  }                                                                                          \
  if (warp == MMA_WARP) tmem_alloc<1>(smem_u32(&tmem_base_slot), cols);                      \
  tc_fence_before();                                                                         \
  __syncthreads();                                                                           \
  tc_fence_after();                                                                          \
  const uint32_t tm = tmem_base_slot;                                                        \
  grid_wait();                                                                               \
  grid_release();                                                                            \
  Next next{smem_u32(&bar_next[0]), smem_u32(&bar_taken[0]), smem_u32(&next_answer[0])};

#define ATTN_END(cols)                                                                       \
  __syncwarp();                                                                              \
  if (abort_flag) { /* copies and products still in flight land before memory is released */ \
    const uint64_t t0 = global_timer_ns();                                                   \
    while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);                            \
  }                                                                                          \
  __syncwarp();                                                                              \
  tc_fence_before();                                                                         \
  __syncthreads();                                                                           \
  if (threadIdx.x == 0 && abort_flag) atomicOr(p.status, ST_TIMEOUT);                        \
  if (warp == MMA_WARP) {                                                                    \
    tc_fence_after();                                                                        \
    tmem_dealloc<1>(tm, cols);                                                               \
  }

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
template <int DP>
struct FwdShape {
  static constexpr uint32_t OPERAND = DP * TILE * 2;
  static constexpr int STAGES = DP == 64 ? 8 : 4;              // k and v tiles in turn
  static constexpr uint32_t SMEM = (2 + STAGES) * OPERAND + 1024u;
};

template <int DP>
__global__ void __launch_bounds__(ATTN_THREADS, 1)
attn_fwd_kernel(const __grid_constant__ Maps4 maps, const __grid_constant__ AttnParams p) {
  using Sh = FwdShape<DP>;
  constexpr int STAGES = Sh::STAGES;
  constexpr uint32_t OPERAND = Sh::OPERAND;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_q[2], bar_qempty[2], bar_full[STAGES], bar_empty[STAGES], bar_s[2], bar_p[2][2], bar_o[2];
  __shared__ __align__(16) uint4 next_answer[2];
  __shared__ __align__(8) uint64_t bar_next[2], bar_taken[2];
  __shared__ uint32_t tmem_base_slot;
  __shared__ volatile int abort_flag;
  // what the two threads of a row tell one another (places of their own: the barriers between two uses of a place are those of a step)
  __shared__ float row_largest[2][2][TILE], row_total[2][2][TILE];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring = smem_base + 2 * OPERAND;
  const uint64_t limit = p.wait_limit_ns;
  auto init_barriers = [&] {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&bar_q[t]), 1);
      mbar_init(smem_u32(&bar_qempty[t]), 1);
      mbar_init(smem_u32(&bar_s[t]), 1);
      mbar_init(smem_u32(&bar_p[t][0]), 4);
      mbar_init(smem_u32(&bar_p[t][1]), 4);
      mbar_init(smem_u32(&bar_o[t]), 1);
    }
  };
  ATTN_BEGIN(512)
  constexpr uint32_t TM_O = 256;              // columns: scores of the two tiles, their sums

  // Of a pair of query tiles: their key tiles (the second may be past the end of the sequence, and has none then), rows of the last key
  // tile that exist, when below 128.
  struct Extent { int n_a, n_b, n, tail; };
  auto extent_of = [](const AttnTile& x) {
    Extent e;
    e.n_a = x.offset / TILE + 1;
    e.n_b = x.offset + TILE < x.length ? e.n_a + 1 : 0;
    e.n = e.n_b ? e.n_b : e.n_a;
    e.tail = x.length - (e.n - 1) * TILE;
    return e;
  };

  if (warp == COPY_WARP) {
    if (lane == 0 && !(p.withhold && blockIdx.x == 0)) {
      Pipe at;
      uint32_t turn[2] = {0, 0};
      bool alive = true;
      for (int u = blockIdx.x; u >= 0; u = alive ? take<false>(next, &abort_flag, limit) : -1) {
        const Unit x = unit_of(p, p.heads, u);
        const Extent e = extent_of(x.tile);
        const int kv_head = x.head / p.group;
        for (int k = 0; k < 2 * e.n; ++k) {
          alive = mbar_wait_cta(smem_u32(&bar_empty[at.stage]), at.phase ^ 1u, &abort_flag, limit);
          if (!alive) break;
          const uint32_t bar = smem_u32(&bar_full[at.stage]);
          mbar_expect_tx(bar, OPERAND);
          load_tile<DP>(ring + at.stage * OPERAND, (k & 1) ? &maps.v : &maps.k, bar, kv_head, x.tile.start + (k >> 1) * TILE);
          at.next<STAGES>();
#pragma unroll
          for (int t = 0; t < 2; ++t) {       // the queries' places are free once the last scores of the unit before are complete
            if (k > 0 || !alive || (t && !e.n_b)) continue;
            alive = mbar_wait_cta(smem_u32(&bar_qempty[t]), turn[t] ^ 1u, &abort_flag, limit);
            if (!alive) continue;
            turn[t] ^= 1u;
            mbar_expect_tx(smem_u32(&bar_q[t]), OPERAND);
            load_tile<DP>(smem_base + t * OPERAND, &maps.q, smem_u32(&bar_q[t]), x.head, x.tile.start + x.tile.offset + t * TILE);
          }
          if (alive && k == (e.n > ASK_AHEAD ? 2 * (e.n - ASK_AHEAD) : 0)) alive = ask(next, &abort_flag, limit);
          if (!alive) break;
        }
      }
    }
  } else if (warp == MMA_WARP) {
    const uint32_t leader = elect_leader();
    // Order: scores of key tile 0 for both query tiles; then per key tile j and query tile: p v of j, scores of j + 1.  Products
    // of one thread complete in order, so scores of j + 1 may overwrite the p of j that the product before them reads.  The first
    // query tile has a key tile less than the second: while the last one's weights are made, it starts on the next unit.
    Pipe at;                                  // of the tile that is waited for next
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(bar), parity, &abort_flag, limit));
    };
    auto arrived = [&](uint32_t* stage) {
      if (!wait(&bar_full[at.stage], at.phase)) return false;
      *stage = at.stage;
      at.next<STAGES>();
      return true;
    };
    uint32_t turn_q[2] = {0, 0}, turn_p[2] = {0, 0}, k_stage = 0, v_stage = 0;
    // scores of a unit's key tile (the last one: the queries' place is free then)
    auto score = [&](int t, bool last) {
      scores<DP>(leader, tm + t * 128, smem_base + t * OPERAND, ring + k_stage * OPERAND);
      mma_commit(leader, smem_u32(&bar_s[t]));
      if (last) mma_commit(leader, smem_u32(&bar_qempty[t]));
    };
    auto start = [&](int t, int n_t) {
      if (!wait(&bar_q[t], turn_q[t])) return false;
      turn_q[t] ^= 1u;
      tc_fence_after();
      score(t, n_t == 1);
      return true;
    };
    bool alive = true, ahead = false;         // ahead: the unit's first scores are under way
    int u = blockIdx.x;
    Extent x = extent_of(unit_of(p, p.heads, u).tile);
    while (u >= 0) {
      if (!ahead) alive = arrived(&k_stage) && start(0, x.n_a);
      ahead = false;
      if (alive && x.n_b) alive = start(1, x.n_b);
      if (!alive) break;
      mma_commit(leader, smem_u32(&bar_empty[k_stage]));
      int u_next = -1;
      Extent y = x;
      bool known = false;
      for (int j = 0; j < x.n; ++j) {
        alive = arrived(&v_stage);
        if (!alive) break;
        if (j == x.n - 1 && x.tail < TILE) zero_rows<DP>(ring + v_stage * OPERAND, x.tail, lane);
        if (j + 1 < x.n) alive = arrived(&k_stage);
        if (!alive) break;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int n_t = t ? x.n_b : x.n_a;
          if (j >= n_t || !alive) continue;
          if (t == 1 && j + 1 == x.n) {
            u_next = take<true>(next, &abort_flag, limit);
            known = true;
            if (u_next >= 0) {
              y = extent_of(unit_of(p, p.heads, u_next).tile);
              alive = arrived(&k_stage) && start(0, y.n_a);
              ahead = alive;
            }
            if (!alive) continue;
          }
          const uint32_t sums = tm + TM_O + t * DP, weights = tm + t * 128, values = ring + v_stage * OPERAND;
          // (at the unit's start both halves of the row warps: they have read the sums of the unit before)
          alive = wait(&bar_p[t][0], turn_p[t]) && (j > 0 || wait(&bar_p[t][1], turn_p[t]));
          if (!alive) continue;
          tc_fence_after();
          weigh_half<DP>(leader, sums, weights, values, 0, j > 0);
          alive = wait(&bar_p[t][1], turn_p[t]);
          if (!alive) continue;
          tc_fence_after();
          weigh_half<DP>(leader, sums, weights + HALF, values, 1, true);
          turn_p[t] ^= 1u;
          if (j + 1 < n_t) score(t, j + 2 == n_t);
          else mma_commit(leader, smem_u32(&bar_o[t]));
        }
        if (!alive) break;
        mma_commit(leader, smem_u32(&bar_empty[v_stage]));
        if (j + 1 < x.n) mma_commit(leader, smem_u32(&bar_empty[k_stage]));
      }
      if (!alive) break;
      if (!known) {
        u_next = take<true>(next, &abort_flag, limit);
        if (u_next >= 0) y = extent_of(unit_of(p, p.heads, u_next).tile);
      }
      u = u_next;
      x = y;
    }
  } else {
    // A row belongs to two threads, each with half of its columns: warps 0-3 and 4-7 (first tile), 8-11 and 12-15 (second).
    const int t = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3;
    const int row = quarter * 32 + lane;                       // of the tile; key columns up to `row` of the last key tile count
    const int col0 = half * 64, pair_id = 1 + t * 4 + quarter;
    const uint32_t t_lane = tm + ((uint32_t)(quarter * 32) << 16);
    const uint32_t t_s = t_lane + t * 128 + half * HALF, t_o = t_lane + TM_O + t * DP + half * (DP / 2);
    const float c = p.scale * LOG2_E;
    const Pair c2 = both(c);
    float top = 0.f, total = 0.f;                              // score that the weights refer to (the row's, unscaled); sum of the weights
    Pair shift = both(0.f);
    // 32 of this thread's 64 scores
    auto load_scores = [&](uint32_t (&s)[32], int h, bool last) {
      tc_ld32(t_s + h * 32, s);
      after_load(s);
      if (last) {
#pragma unroll
        for (int e = 0; e < 32; ++e) s[e] = col0 + h * 32 + e > row ? 0xff800000u : s[e];
      }
    };
    // The reference becomes the row's largest score so far; sums and weighted values so far (`some`: there are some) follow.  Only in rows whose
    // own weights ask for it: what a row comes out as does not depend on the others.
    auto move_reference = [&](bool some, bool last, float part) {
      float m = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t s[32];
        load_scores(s, h, last);
#pragma unroll
        for (int e = 0; e < 32; e += 2) m = max3(m, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
      }
      row_largest[t][half][row] = m;
      if (some) row_total[t][half][row] = part;   // (at a unit's start the other thread may not have read the last one's total)
      either(pair_id, false);
      m = max3(m, row_largest[t][half ^ 1][row], some ? top : m);
      if (some && part <= MOST && row_total[t][half ^ 1][row] <= MOST) m = top;
      if (some) {                             // (the product before these scores is complete, as they are)
        const float by = exp2_approx((top - m) * c);
        total *= by;
#pragma unroll 1
        for (int i = 0; i < DP / 2; i += 32) {
          uint32_t v[32];
          tc_ld32(t_o + i, v);
          after_load(v);
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * by);
          tm_store32(t_o + i, v);
        }
        // The next product adds to all columns of the sums once the first half's weights are there: both threads of the row have
        // rescaled theirs before either hands weights over.
        tm_store_wait();
        tc_fence_before();
        either(pair_id, false);
        tc_fence_after();
      }
      top = m;
      // (an infinite maximum makes every weight NaN, as the quotient of infinities is)
      shift = both((top - top) - top * c);
    };
    auto weights = [&](uint32_t (&w)[32], bool last) {
      Pair sum[2] = {both(0.f), both(0.f)};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t s[32];
        load_scores(s, h, last);
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const Pair x = fma2(pair(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2, shift);
          float2 y = parts(x);
          y.x = exp2_approx(y.x);
          y.y = exp2_approx(y.y);
          sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pair(y.x, y.y));
          w[h * 16 + (e >> 1)] = pack_bf16x2(y.x, y.y);
        }
      }
      const float2 sums = parts(add2(sum[0], sum[1]));
      return sums.x + sums.y;
    };
    uint32_t turn_s = 0, turn_o = 0;
    bool alive = true;
    for (int u = blockIdx.x; u >= 0; u = alive ? take_together<64>(next, pair_id, &abort_flag, limit) : -1) {
      const Unit x = unit_of(p, p.heads, u);
      const Extent e = extent_of(x.tile);
      const int n_t = t ? e.n_b : e.n_a;
      if (!n_t) continue;
      const int pos = x.tile.offset + t * TILE + row;
      const bool ok = pos < x.tile.length;    // rows past the end hold another sequence's tokens: nothing goes by them
      top = 0.f;
      total = 0.f;
      for (int j = 0; j < n_t; ++j) {
        alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_s[t]), turn_s, &abort_flag, limit));
        tc_fence_after();
        const bool last = j == n_t - 1;
        uint32_t w[32];
        if (j == 0) move_reference(false, last, 0.f);
        float part = weights(w, last);
        // Where the weights are too large by the reference as it was, or not numbers: once more by a new one.
        if (either(pair_id, !alive || (j > 0 && ok && !(part <= MOST)))) {
          if (either(pair_id, !alive)) { alive = false; break; }
          move_reference(true, last, part);
          part = weights(w, last);
        }
        total += part;
        tm_store32(t_s, w);
        tm_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(smem_u32(&bar_p[t][half]));
        turn_s ^= 1u;
      }
      if (alive) alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_o[t]), turn_o, &abort_flag, limit));
      row_total[t][half][row] = total;
      alive = !either(pair_id, !alive);
      if (!alive) break;
      turn_o ^= 1u;
      tc_fence_after();
      total += row_total[t][half ^ 1][row];
      const int64_t token = (int64_t)x.tile.start + pos;
      __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out) + ((ok ? token : 0) * p.heads + x.head) * p.dim + half * (DP / 2);
      const bool wide = (p.dim & 15) == 0 && ((uintptr_t)p.out & 31) == 0;
      store_columns(t_o, out, 0, DP / 2, p.dim - half * (DP / 2), 1.0f / total, ok, wide);
      if (ok && half == 0) p.lse[(int64_t)x.head * p.tokens + token] = (top * c + log2_approx(total)) * LN2;
    }
  }
  ATTN_END(512)
}

// ---------------------------------------------------------------------------
// backward over the keys of a query tile: delta and dq
// ---------------------------------------------------------------------------
template <int DP>
struct BackShape {
  static constexpr uint32_t OPERAND = DP * TILE * 2;
  static constexpr int STAGES = 2;
  static constexpr uint32_t SMEM = (2 + 2 * STAGES) * OPERAND + 1024u;
};

template <int DP>
__global__ void __launch_bounds__(ATTN_THREADS, 1)
attn_dq_kernel(const __grid_constant__ Maps4 maps, const __grid_constant__ AttnParams p) {
  using Sh = BackShape<DP>;
  constexpr int STAGES = Sh::STAGES;
  constexpr uint32_t OPERAND = Sh::OPERAND;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_q, bar_qempty, bar_kfull[STAGES], bar_kempty[STAGES], bar_vfull[STAGES], bar_vempty[STAGES], bar_s[2], bar_dp,
      bar_ds, bar_done;
  __shared__ __align__(16) uint4 next_answer[2];
  __shared__ __align__(8) uint64_t bar_next[2], bar_taken[2];
  __shared__ uint32_t tmem_base_slot;
  __shared__ volatile int abort_flag;
  __shared__ float row_part[2][4][TILE];      // quarters of a row's delta, two units in turn

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t s_q = smem_base, s_g = smem_base + OPERAND, s_k = smem_base + 2 * OPERAND, s_v = s_k + STAGES * OPERAND;
  const uint64_t limit = p.wait_limit_ns;
  auto init_barriers = [&] {
    mbar_init(smem_u32(&bar_q), 1);
    mbar_init(smem_u32(&bar_qempty), 1);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&bar_kfull[s]), 1);
      mbar_init(smem_u32(&bar_kempty[s]), 1);
      mbar_init(smem_u32(&bar_vfull[s]), 1);
      mbar_init(smem_u32(&bar_vempty[s]), 1);
    }
    mbar_init(smem_u32(&bar_s[0]), 1);
    mbar_init(smem_u32(&bar_s[1]), 1);
    mbar_init(smem_u32(&bar_dp), 1);
    mbar_init(smem_u32(&bar_ds), ROW_WARPS);
    mbar_init(smem_u32(&bar_done), 1);
  };
  ATTN_BEGIN(512)
  constexpr uint32_t TM_DP = 256, TM_DQ = 384;                 // columns: two tiles of scores, dp, dq

  if (warp == COPY_WARP) {
    if (lane == 0 && !(p.withhold && blockIdx.x == 0)) {
      Pipe at;
      uint32_t turn = 0;
      bool alive = true;
      for (int u = blockIdx.x; u >= 0; u = alive ? take<false>(next, &abort_flag, limit) : -1, turn ^= 1u) {
        const Unit x = unit_of(p, p.heads, u);
        const int n = x.tile.offset / TILE + 1, kv_head = x.head / p.group, first_row = x.tile.start + x.tile.offset;
        for (int j = 0; j < n; ++j) {
          alive = mbar_wait_cta(smem_u32(&bar_kempty[at.stage]), at.phase ^ 1u, &abort_flag, limit);
          if (!alive) break;
          mbar_expect_tx(smem_u32(&bar_kfull[at.stage]), OPERAND);
          load_tile<DP>(s_k + at.stage * OPERAND, &maps.k, smem_u32(&bar_kfull[at.stage]), kv_head, x.tile.start + j * TILE);
          if (j == 0) {                       // free once the last scores and dp of the unit before are complete
            alive = mbar_wait_cta(smem_u32(&bar_qempty), turn ^ 1u, &abort_flag, limit);
            if (!alive) break;
            mbar_expect_tx(smem_u32(&bar_q), 2 * OPERAND);
            load_tile<DP>(s_q, &maps.q, smem_u32(&bar_q), x.head, first_row);
            load_tile<DP>(s_g, &maps.g, smem_u32(&bar_q), x.head, first_row);
          }
          alive = mbar_wait_cta(smem_u32(&bar_vempty[at.stage]), at.phase ^ 1u, &abort_flag, limit);
          if (!alive) break;
          mbar_expect_tx(smem_u32(&bar_vfull[at.stage]), OPERAND);
          load_tile<DP>(s_v + at.stage * OPERAND, &maps.v, smem_u32(&bar_vfull[at.stage]), kv_head, x.tile.start + j * TILE);
          at.next<STAGES>();
          if (j == (n > ASK_AHEAD ? n - ASK_AHEAD : 0)) alive = ask(next, &abort_flag, limit);
          if (!alive) break;
        }
      }
    }
  } else if (warp == MMA_WARP) {
    const uint32_t leader = elect_leader();
    // Order: scores and dp of 0; then per key tile j: scores of j + 1 (into the other columns), dp of j + 1 (when the row warps have read
    // that of j), dq += ds k of j.  (The scores of j + 1 may be complete before the row warps have looked for those of j: a barrier for
    // each of the two places.)
    Pipe at, at_v;                            // key tile j; value tile that is waited for next
    uint32_t turn = 0, step = 0;              // step: key tiles so far, over all units
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(bar), parity, &abort_flag, limit));
    };
    bool alive = true;
    for (int u = blockIdx.x; u >= 0; u = alive ? take<true>(next, &abort_flag, limit) : -1, turn ^= 1u) {
      const AttnTile x = unit_of(p, p.heads, u).tile;
      const int n = x.offset / TILE + 1;      // key tiles
      const int tail = x.length - (n - 1) * TILE;              // rows of the last one that exist, when below 128
      // scores of key tile j, which is step `k`, and dp
      auto start = [&](const Pipe& q, int j, uint32_t k) {
        if (!wait(&bar_kfull[q.stage], q.phase)) return false;
        if (j == n - 1 && tail < TILE) zero_rows<DP>(s_k + q.stage * OPERAND, tail, lane);
        tc_fence_after();
        scores<DP>(leader, tm + (k & 1u) * 128, s_q, s_k + q.stage * OPERAND);
        mma_commit(leader, smem_u32(&bar_s[k & 1u]));
        return true;
      };
      auto start_dp = [&](int j) {
        if (!wait(&bar_vfull[at_v.stage], at_v.phase)) return false;
        tc_fence_after();
        scores<DP>(leader, tm + TM_DP, s_g, s_v + at_v.stage * OPERAND);
        mma_commit(leader, smem_u32(&bar_dp));
        mma_commit(leader, smem_u32(&bar_vempty[at_v.stage]));
        at_v.next<STAGES>();
        if (j == n - 1) mma_commit(leader, smem_u32(&bar_qempty));
        return true;
      };
      alive = wait(&bar_q, turn) && start(at, 0, step) && start_dp(0);
      for (int j = 0; alive && j < n; ++j, ++step) {
        Pipe ahead = at;
        ahead.next<STAGES>();
        if (j + 1 < n) alive = start(ahead, j + 1, step + 1);
        alive = alive && wait(&bar_ds, step & 1u);
        if (!alive) break;
        tc_fence_after();
        weigh<DP>(leader, tm + TM_DQ, tm + (step & 1u) * 128, s_k + at.stage * OPERAND, j > 0);
        mma_commit(leader, smem_u32(&bar_kempty[at.stage]));
        if (j + 1 == n) mma_commit(leader, smem_u32(&bar_done));
        if (j + 1 < n) alive = start_dp(j + 1);
        at = ahead;
      }
    }
  } else if (warp < COPY_WARP) {
    const int part = warp >> 2, quarter = warp & 3;            // columns 32 part .. of rows 32 quarter ..
    const int row = quarter * 32 + lane;
    const uint32_t t_lane = tm + ((uint32_t)(quarter * 32) << 16);
    const float c = p.scale * LOG2_E;
    const int id = 1 + quarter;                                // barrier of the four warps that share these rows
    uint32_t turn = 0, step = 0;
    const Pair c2 = both(c);
    bool alive = true;
    for (int u = blockIdx.x; u >= 0; u = alive ? take_together<128>(next, id, &abort_flag, limit) : -1, turn ^= 1u) {
      const Unit x = unit_of(p, p.heads, u);
      const int n = x.tile.offset / TILE + 1;
      const int pos = x.tile.offset + row;
      const bool ok = pos < x.tile.length;
      const int64_t token = (int64_t)x.tile.start + (ok ? pos : 0), stat = (int64_t)x.head * p.tokens + token;
      // the row's sum of what its four threads have, in the same order in all of them
      auto row_sum = [&](float x, bool failed, float* sum) {
        row_part[turn][part][row] = x;
        if (any_of<128>(id, failed)) return false;
        const float* q = &row_part[turn][0][row];
        *sum = (q[0] + q[TILE]) + (q[2 * TILE] + q[3 * TILE]);
        return true;
      };
      const Pair shift = both(-p.lse[stat] * LOG2_E);
      // delta = do . o, with o as it was rounded; each of the row's four threads has a quarter of it.  A row with a single key tile takes the
      // sum of p dp below instead: there o is nearly as large as v, and its rounding would show in dq.
      float delta = 0.f;
      if (n > 1) {
        const int c0 = part * (DP / 4);
        const __nv_bfloat16* o = reinterpret_cast<const __nv_bfloat16*>(p.o) + (token * p.heads + x.head) * p.dim + c0;
        const __nv_bfloat16* g = reinterpret_cast<const __nv_bfloat16*>(p.g) + token * p.g_ts + x.head * p.g_hs + c0;
        Pair acc = both(0.f);
#pragma unroll
        for (int e = 0; e < DP / 4; e += 8) {
          if (c0 + e >= p.dim) break;
          const uint4 a = *reinterpret_cast<const uint4*>(o + e), b = *reinterpret_cast<const uint4*>(g + e);
          acc = fma2(pair_bf16(a.x), pair_bf16(b.x), acc);
          acc = fma2(pair_bf16(a.y), pair_bf16(b.y), acc);
          acc = fma2(pair_bf16(a.z), pair_bf16(b.z), acc);
          acc = fma2(pair_bf16(a.w), pair_bf16(b.w), acc);
        }
        const float2 sums = parts(acc);
        row_sum(sums.x + sums.y, false, &delta);
        if (part == 0 && ok) p.delta[stat] = delta;
      }
      for (int j = 0; j < n; ++j, ++step) {
        const uint32_t t_s = t_lane + (step & 1u) * 128 + part * QUARTER;
        alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_s[step & 1u]), (step >> 1) & 1u, &abort_flag, limit));
        if (!alive && n > 1) break;
        tc_fence_after();
        uint32_t s[32], d[32];
        tc_ld32(t_s, s);
        after_load(s);
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float2 y = parts(fma2(pair(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2, shift));
          s[e] = __float_as_uint(exp2_approx(y.x));
          s[e + 1] = __float_as_uint(exp2_approx(y.y));
        }
        if (alive) alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_dp), step & 1u, &abort_flag, limit));
        if (!alive && n > 1) break;
        tc_fence_after();
        tc_ld32(t_lane + TM_DP + part * QUARTER, d);
        after_load(d);
        uint32_t w[16];
        if (j == n - 1) {                     // where the key comes after the query: no weight, whatever the products hold
          if (n == 1) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 32; ++e) sum += part * 32 + e > row ? 0.f : __uint_as_float(s[e]) * __uint_as_float(d[e]);
            // (a sequence's first query has one key, whose weight is 1, not the 1 +- 2^-18 that its rounded log-sum-exp gives: ds is zero)
            if (part == 0 && row == 0) sum = __uint_as_float(d[0]);
            if (!row_sum(sum, !alive, &delta)) { alive = false; break; }
            if (part == 0 && ok) p.delta[stat] = delta;
          }
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float a = __uint_as_float(s[e]) * (__uint_as_float(d[e]) - delta);
            const float b = __uint_as_float(s[e + 1]) * (__uint_as_float(d[e + 1]) - delta);
            w[e >> 1] = pack_bf16x2(part * 32 + e > row ? 0.f : a, part * 32 + e + 1 > row ? 0.f : b);
          }
        } else {
          const Pair minus = both(-delta);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 y = parts(mul2(pair(__uint_as_float(s[e]), __uint_as_float(s[e + 1])),
                                        add2(pair(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), minus)));
            w[e >> 1] = pack_bf16x2(y.x, y.y);
          }
        }
        tm_store16(t_s, w);
        tm_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(smem_u32(&bar_ds));
      }
      if (alive) alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_done), turn, &abort_flag, limit));
      alive = !any_of<128>(id, !alive);
      if (alive && part < DP / 32) {
        tc_fence_after();
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out) + (token * p.heads + x.head) * p.dim;
        const bool wide = (p.dim & 15) == 0 && ((uintptr_t)p.out & 31) == 0;
        store_columns(t_lane + TM_DQ, out, part * 32, 32, p.dim, p.scale, ok, wide);
      }
    }
  }
  ATTN_END(512)
}

// ---------------------------------------------------------------------------
// backward over the queries of a key tile, for all query heads of its group: dk and dv
// ---------------------------------------------------------------------------
template <int DP>
__global__ void __launch_bounds__(ATTN_THREADS, 1)
attn_dkv_kernel(const __grid_constant__ Maps4 maps, const __grid_constant__ AttnParams p) {
  using Sh = BackShape<DP>;
  constexpr int STAGES = Sh::STAGES;
  constexpr uint32_t OPERAND = Sh::OPERAND;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_kv, bar_kvempty, bar_qfull[STAGES], bar_qempty[STAGES], bar_gfull[STAGES], bar_gempty[STAGES], bar_s, bar_dp,
      bar_p, bar_ds, bar_done;
  __shared__ __align__(16) uint4 next_answer[2];
  __shared__ __align__(8) uint64_t bar_next[2], bar_taken[2];
  __shared__ uint32_t tmem_base_slot;
  __shared__ volatile int abort_flag;
  __shared__ __align__(16) float row_values[ROW_WARPS][2][32]; // of each row warp: log-sum-exp and delta of its 32 queries, negated

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t s_k = smem_base, s_v = smem_base + OPERAND, s_q = smem_base + 2 * OPERAND, s_g = s_q + STAGES * OPERAND;
  const uint64_t limit = p.wait_limit_ns;
  auto init_barriers = [&] {
    mbar_init(smem_u32(&bar_kv), 1);
    mbar_init(smem_u32(&bar_kvempty), 1);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&bar_qfull[s]), 1);
      mbar_init(smem_u32(&bar_qempty[s]), 1);
      mbar_init(smem_u32(&bar_gfull[s]), 1);
      mbar_init(smem_u32(&bar_gempty[s]), 1);
    }
    mbar_init(smem_u32(&bar_s), 1);
    mbar_init(smem_u32(&bar_dp), 1);
    mbar_init(smem_u32(&bar_p), ROW_WARPS);
    mbar_init(smem_u32(&bar_ds), ROW_WARPS);
    mbar_init(smem_u32(&bar_done), 1);
  };
  ATTN_BEGIN(512)
  constexpr uint32_t TM_DP = 128, TM_DV = 256, TM_DK = 256 + DP;           // columns: scores, dp, dv, dk (rows are keys)

  const int kv_heads = p.heads / p.group;
  // Of a key tile: its query tiles, first to end, of `group` heads; rows of the last one that exist, when below 128.
  struct Extent { int first, end, n, tail; };
  auto extent_of = [&](const AttnTile& x) {
    Extent e;
    e.first = x.offset / TILE;
    e.end = (x.length + TILE - 1) / TILE;
    e.n = (e.end - e.first) * p.group;
    e.tail = x.length - (e.end - 1) * TILE;
    return e;
  };

  if (warp == COPY_WARP) {
    if (lane == 0 && !(p.withhold && blockIdx.x == 0)) {
      Pipe at;
      uint32_t turn = 0;
      bool alive = true;
      for (int u = blockIdx.x; u >= 0; u = alive ? take<false>(next, &abort_flag, limit) : -1, turn ^= 1u) {
        const Unit x = unit_of(p, kv_heads, u);
        const Extent e = extent_of(x.tile);
        int head = x.head * p.group, i = e.first;
        for (int it = 0; it < e.n; ++it) {
          alive = mbar_wait_cta(smem_u32(&bar_qempty[at.stage]), at.phase ^ 1u, &abort_flag, limit);
          if (!alive) break;
          mbar_expect_tx(smem_u32(&bar_qfull[at.stage]), OPERAND);
          load_tile<DP>(s_q + at.stage * OPERAND, &maps.q, smem_u32(&bar_qfull[at.stage]), head, x.tile.start + i * TILE);
          if (it == 0) {                      // free once the last scores and dp of the unit before are complete
            alive = mbar_wait_cta(smem_u32(&bar_kvempty), turn ^ 1u, &abort_flag, limit);
            if (!alive) break;
            mbar_expect_tx(smem_u32(&bar_kv), 2 * OPERAND);
            load_tile<DP>(s_k, &maps.k, smem_u32(&bar_kv), x.head, x.tile.start + x.tile.offset);
            load_tile<DP>(s_v, &maps.v, smem_u32(&bar_kv), x.head, x.tile.start + x.tile.offset);
          }
          alive = mbar_wait_cta(smem_u32(&bar_gempty[at.stage]), at.phase ^ 1u, &abort_flag, limit);
          if (!alive) break;
          mbar_expect_tx(smem_u32(&bar_gfull[at.stage]), OPERAND);
          load_tile<DP>(s_g + at.stage * OPERAND, &maps.g, smem_u32(&bar_gfull[at.stage]), head, x.tile.start + i * TILE);
          at.next<STAGES>();
          if (++i == e.end) { i = e.first; ++head; }
          if (it == (e.n > ASK_AHEAD ? e.n - ASK_AHEAD : 0)) alive = ask(next, &abort_flag, limit);
          if (!alive) break;
        }
      }
    }
  } else if (warp == MMA_WARP) {
    const uint32_t leader = elect_leader();
    // Order: scores of 0; then per step: dp, dv += p do, scores of the next, dk += ds q.
    Pipe at;
    uint32_t turn = 0, step = 0;              // step: query tiles so far, over all units
    bool alive = true;
    for (int u = blockIdx.x; u >= 0; u = alive ? take<true>(next, &abort_flag, limit) : -1, turn ^= 1u) {
      const Extent x = extent_of(unit_of(p, kv_heads, u).tile);
      int i = x.first;                        // query tile of the step
      auto queries = [&](const Pipe& q, int i) {
        if (!__all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_qfull[q.stage]), q.phase, &abort_flag, limit))) return false;
        if (i == x.end - 1 && x.tail < TILE) zero_rows<DP>(s_q + q.stage * OPERAND, x.tail, lane);
        return true;
      };
      alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_kv), turn, &abort_flag, limit)) && queries(at, i);
      if (!alive) break;
      tc_fence_after();
      scores<DP>(leader, tm, s_k, s_q + at.stage * OPERAND);
      mma_commit(leader, smem_u32(&bar_s));
      for (int it = 0; it < x.n; ++it, ++step) {
        alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_gfull[at.stage]), at.phase, &abort_flag, limit));
        if (!alive) break;
        if (i == x.end - 1 && x.tail < TILE) zero_rows<DP>(s_g + at.stage * OPERAND, x.tail, lane);
        tc_fence_after();
        scores<DP>(leader, tm + TM_DP, s_v, s_g + at.stage * OPERAND);
        mma_commit(leader, smem_u32(&bar_dp));
        if (it + 1 == x.n) mma_commit(leader, smem_u32(&bar_kvempty));
        alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_p), step & 1u, &abort_flag, limit));
        if (!alive) break;
        tc_fence_after();
        weigh<DP>(leader, tm + TM_DV, tm, s_g + at.stage * OPERAND, it > 0);
        mma_commit(leader, smem_u32(&bar_gempty[at.stage]));
        Pipe ahead = at;
        ahead.next<STAGES>();
        const int i_next = i + 1 == x.end ? x.first : i + 1;
        if (it + 1 < x.n) {
          alive = queries(ahead, i_next);
          if (!alive) break;
          tc_fence_after();
          scores<DP>(leader, tm, s_k, s_q + ahead.stage * OPERAND);
          mma_commit(leader, smem_u32(&bar_s));
        }
        alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_ds), step & 1u, &abort_flag, limit));
        if (!alive) break;
        tc_fence_after();
        weigh<DP>(leader, tm + TM_DK, tm + TM_DP, s_q + at.stage * OPERAND, it > 0);
        mma_commit(leader, smem_u32(&bar_qempty[at.stage]));
        if (it + 1 == x.n) mma_commit(leader, smem_u32(&bar_done));
        at = ahead;
        i = i_next;
      }
    }
  } else if (warp < COPY_WARP) {
    const int part = warp >> 2, quarter = warp & 3;            // columns 32 part .. (queries) of rows 32 quarter ..
    const int row = quarter * 32 + lane;                       // key of the tile
    const uint32_t t_lane = tm + ((uint32_t)(quarter * 32) << 16);
    const uint32_t t_s = t_lane + part * QUARTER, t_dp = t_lane + TM_DP + part * QUARTER;
    const float c = p.scale * LOG2_E;
    const Pair c2 = both(c);
    // each warp brings the log-sum-exp and the delta of its 32 queries into shared memory, fetched a step ahead
    const int col0 = part * 32;
    float* const lse = row_values[warp][0];
    float* const delta = row_values[warp][1];
    uint32_t turn = 0, step = 0;
    bool alive = true;
    for (int u = blockIdx.x; u >= 0; u = alive ? take<true>(next, &abort_flag, limit) : -1, turn ^= 1u) {
      const Unit x = unit_of(p, kv_heads, u);
      const Extent ext = extent_of(x.tile);
      int head = x.head * p.group, i = ext.first;
      float ahead[2];
      auto fetch = [&] {
        const int pos = i * TILE + col0 + lane;
        const int64_t at = (int64_t)head * p.tokens + x.tile.start + pos;
        ahead[0] = pos < x.tile.length ? -LOG2_E * p.lse[at] : 0.f;
        ahead[1] = pos < x.tile.length ? -p.delta[at] : 0.f;
      };
      fetch();
      for (int it = 0; it < ext.n; ++it, ++step) {
        const bool edge = i == ext.first || (i == ext.end - 1 && ext.tail < TILE);       // some of the tile's pairs do not count
        const int last = x.tile.length - i * TILE - 1;                         // columns from .. last count
        const int from = i == ext.first ? row : 0;
        const bool single = x.tile.offset == 0 && i == ext.first && row == 0 && col0 == 0;     // the sequence's first query and key
        __syncwarp();
        lse[lane] = ahead[0];
        delta[lane] = ahead[1];
        __syncwarp();
        if (++i == ext.end) { i = ext.first; ++head; }
        if (it + 1 < ext.n) fetch();
        alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_s), step & 1u, &abort_flag, limit));
        if (!alive) break;
        uint32_t s[32], w[16];
        tc_fence_after();
        tc_ld32(t_s, s);
        after_load(s);
  #pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const float4 l = *reinterpret_cast<const float4*>(lse + e);
          const float2 x = parts(fma2(pair(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2, pair(l.x, l.y)));
          const float2 y = parts(fma2(pair(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])), c2, pair(l.z, l.w)));
          s[e] = __float_as_uint(exp2_approx(x.x));
          s[e + 1] = __float_as_uint(exp2_approx(x.y));
          s[e + 2] = __float_as_uint(exp2_approx(y.x));
          s[e + 3] = __float_as_uint(exp2_approx(y.y));
        }
        if (edge) {
  #pragma unroll
          for (int e = 0; e < 32; ++e) s[e] = col0 + e < from || col0 + e > last ? 0u : s[e];
        }
  #pragma unroll
        for (int e = 0; e < 32; e += 2) w[e >> 1] = pack_bf16x2(__uint_as_float(s[e]), __uint_as_float(s[e + 1]));
        tm_store16(t_s, w);
        tm_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(smem_u32(&bar_p));
        alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_dp), step & 1u, &abort_flag, limit));
        if (!alive) break;
        tc_fence_after();
        uint32_t d[32];
        tc_ld32(t_dp, d);
        after_load(d);
  #pragma unroll
        for (int e = 0; e < 32; e += 4) {
          float4 l = *reinterpret_cast<const float4*>(delta + e);
          if (e == 0 && single) l.x = -__uint_as_float(d[0]);  // (delta is its dp, from another kernel's product: here the same bits)
          const float2 x = parts(mul2(pair(__uint_as_float(s[e]), __uint_as_float(s[e + 1])),
                                      add2(pair(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), pair(l.x, l.y))));
          const float2 y = parts(mul2(pair(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])),
                                      add2(pair(__uint_as_float(d[e + 2]), __uint_as_float(d[e + 3])), pair(l.z, l.w))));
          d[e] = __float_as_uint(x.x); d[e + 1] = __float_as_uint(x.y);
          d[e + 2] = __float_as_uint(y.x); d[e + 3] = __float_as_uint(y.y);
        }
        if (edge) {                           // (zero times what the products hold there need not be zero)
  #pragma unroll
          for (int e = 0; e < 32; ++e) d[e] = col0 + e < from || col0 + e > last ? 0u : d[e];
        }
  #pragma unroll
        for (int e = 0; e < 32; e += 2) w[e >> 1] = pack_bf16x2(__uint_as_float(d[e]), __uint_as_float(d[e + 1]));
        tm_store16(t_dp, w);
        tm_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(smem_u32(&bar_ds));
      }
      if (alive) {
        alive = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bar_done), turn, &abort_flag, limit));
        if (alive) {
          tc_fence_after();
          const int pos = x.tile.offset + row;
          const bool ok = pos < x.tile.length;
          const int64_t at = (((int64_t)x.tile.start + (ok ? pos : 0)) * kv_heads + x.head) * p.dim;
          const bool keys = part >= 2;          // two warps have dv, two dk
          __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(keys ? p.out : p.out2) + at;
          const bool wide = (p.dim & 15) == 0 && (((uintptr_t)p.out | (uintptr_t)p.out2) & 31) == 0;
          store_columns(t_lane + (keys ? TM_DK : TM_DV), out, (part & 1) * (DP / 2), DP / 2, p.dim, keys ? p.scale : 1.0f, ok, wide);
        }
      }
    }
  }
  ATTN_END(512)
}

// ----------------------------- host ------------------------------------------

// A tensor [tokens][heads][dim] in boxes of 64 entries of one head by 128 tokens; entries past dim and rows past the end read as zero.
bool encode(CUtensorMap* map, const void* x, int64_t tokens, int64_t heads, int64_t dim, int64_t ts, int64_t hs) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) return false;
  if (heads == 1) hs = dim;                   // the stride of a single head or token does not matter
  if (tokens == 1) ts = heads * hs;
  const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)hs * 2, (cuuint64_t)ts * 2};
  const cuuint32_t box[3] = {64, 1, TILE}, step[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(x), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DP>
cudaError_t run_forward(cudaStream_t st, const Maps4& m, const AttnParams& p) {
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_smem(attn_fwd_kernel<DP>, (int)FwdShape<DP>::SMEM, &allowed);
  if (e != cudaSuccess) return e;
  return launch_dependent(attn_fwd_kernel<DP>, (unsigned)(p.n_tiles * p.heads), ATTN_THREADS, FwdShape<DP>::SMEM, st, m, p);
}

template <int DP>
cudaError_t run_backward(cudaStream_t st, const Maps4& m, AttnParams p, const AttnArgs& a) {
  static std::atomic<uint64_t> allowed{0}, allowed2{0};
  cudaError_t e = allow_smem(attn_dq_kernel<DP>, (int)BackShape<DP>::SMEM, &allowed);
  if (e == cudaSuccess) e = allow_smem(attn_dkv_kernel<DP>, (int)BackShape<DP>::SMEM, &allowed2);
  if (e != cudaSuccess) return e;
  p.n_tiles = (int)a.n_tiles;
  p.tiles = a.query_tiles;
  p.out = a.dq;
  e = launch_dependent(attn_dq_kernel<DP>, (unsigned)(a.n_tiles * a.heads), ATTN_THREADS, BackShape<DP>::SMEM, st, m, p);
  if (e != cudaSuccess) return e;
  p.withhold = 0;
  p.tiles = a.key_tiles;
  p.section /= p.group;
  p.out = a.dk;
  p.out2 = a.dv;
  return launch_dependent(attn_dkv_kernel<DP>, (unsigned)(a.n_tiles * a.kv_heads), ATTN_THREADS, BackShape<DP>::SMEM, st, m, p);
}

bool prepare(const AttnArgs& a, Maps4* m, AttnParams* p) {
  memset(p, 0, sizeof *p);
  p->tokens = a.tokens;
  p->heads = a.heads; p->group = a.heads / a.kv_heads; p->dim = a.dim;
  p->scale = a.scale;
  p->lse = a.lse; p->delta = a.delta;
  p->o = a.o; p->g = a.g; p->g_ts = a.g_ts; p->g_hs = a.g_hs;
  p->status = a.status;
  p->wait_limit_ns = a.wait_limit_ns ? a.wait_limit_ns : 2000000000ull;
  p->withhold = a.withhold;
  // key heads whose keys and values (backward: and queries and gradients, about as much again for each head of the group) stay in L2 together
  const int64_t bytes = a.tokens * a.dim * 4 * (a.g ? 1 + p->group : 1);
  const int64_t some = SECTION_BYTES / (bytes > 0 ? bytes : 1);
  p->section = (int)(some < 1 ? 1 : some < a.kv_heads ? some : a.kv_heads) * p->group;
  return encode(&m->q, a.q, a.tokens, a.heads, a.dim, a.q_ts, a.q_hs) && encode(&m->k, a.k, a.tokens, a.kv_heads, a.dim, a.k_ts, a.k_hs) &&
         encode(&m->v, a.v, a.tokens, a.kv_heads, a.dim, a.v_ts, a.v_hs) &&
         (!a.g || encode(&m->g, a.g, a.tokens, a.heads, a.dim, a.g_ts, a.g_hs));
}

}  // namespace

cudaError_t launch_attention(cudaStream_t st, const AttnArgs& a, const char** what) {
  const cudaError_t bound = bind_context(what);
  if (bound != cudaSuccess) return bound;
  Maps4 m;
  AttnParams p;
  memset(&m, 0, sizeof m);
  *what = "cuTensorMapEncodeTiled";
  if (!prepare(a, &m, &p)) return cudaErrorInvalidValue;
  *what = "launch of the attention kernel";
  p.tiles = a.pair_tiles;
  p.out = a.o_out;
  p.n_tiles = (int)a.n_pairs;
  return a.dim <= 64 ? run_forward<64>(st, m, p) : run_forward<128>(st, m, p);
}

cudaError_t launch_attention_backward(cudaStream_t st, const AttnArgs& a, const char** what) {
  const cudaError_t bound = bind_context(what);
  if (bound != cudaSuccess) return bound;
  Maps4 m;
  AttnParams p;
  memset(&m, 0, sizeof m);
  *what = "cuTensorMapEncodeTiled";
  if (!prepare(a, &m, &p)) return cudaErrorInvalidValue;
  *what = "launch of the attention kernels of the backward pass";
  return a.dim <= 64 ? run_backward<64>(st, m, p, a) : run_backward<128>(st, m, p, a);
}

}  // namespace muloco
