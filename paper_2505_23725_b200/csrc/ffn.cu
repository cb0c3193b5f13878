// Gated feed-forward block on the 5th-generation tensor cores: tcgen05.mma with fp32 accumulators in
// tensor memory, operands staged by TMA (128-byte swizzle), warp-specialised persistent thread blocks.
//
// One kernel body serves every product of the block; a launch works through the tiles of up to four
// products whose tiles do not depend on one another:
//   forward   G | U = X W1 | X W3, gated in the epilogue            then   Y = H W2
//   backward  dH = dY W2^T, turned into dG and dU in the epilogue   then   dX, dW1, dW3, dW2 in one launch
// An operand whose contraction index is its contiguous axis is staged K-major (64 x 128 boxes), one whose
// other index is contiguous MN-major (two atoms of 64 columns by 64 contraction rows); so no matrix is ever transposed
// in memory: X serves G = X W1 K-major and dW1 = X^T dG MN-major, and W1 likewise.
//
// Tile: a pair of CTAs on neighbouring SMs computes 256 x 256 with tcgen05.mma.cta_group::2 (each CTA stages
// its 128 rows of the left operand and half of the right one and drains its own 128 accumulator rows).  For the
// gated product the two halves of the right operand are 128 columns of W1 and the same 128 columns of W3: an accumulator
// row then holds G in columns 0..127 and U in columns 128..255, and the activation and the product are
// register arithmetic of the epilogue.
//
// Roles: warp 0 issues the copies, warp 1 the MMAs, warps 2..9 run the epilogue (two warps per 32 accumulator
// lanes, half of the columns each).  Two accumulators alternate, so the epilogue of a tile runs beside the
// products of the next.  Thread blocks never wait for one another across a pair, and every wait is bounded: when one
// runs out the block raises ST_TIMEOUT, frees its tensor memory and returns.
//
// Bound by the tensor cores' feed and, after some milliseconds, by the power limit: 16384 tokens at 1024 x 2816 forward 231 us (1.22
// PFLOP/s), 8192 tokens at 2048 x 5632 backward 900 us (1.26 PFLOP/s); under the limit 266 and 1014 us, where the library's products
// alone take 239 and 886.  Unlimited, a slab takes 334 ns, about 635 cycles, where its MMAs need 512.
#include <string.h>

#include <atomic>

#include "internal.h"
#include "tc_ptx.cuh"

namespace muloco {

namespace {

constexpr int BK = 64;                       // contraction slab: 64 bf16 = one 128-byte swizzle row
constexpr int UMMA_K = 16;
constexpr int CG = 2;                        // CTAs per tile
constexpr int BM = 128;                      // rows per CTA
constexpr int TM = 128 * CG, BN = 128 * CG;  // tile
constexpr int EPI_WARPS = 8;
constexpr int FFN_THREADS = 64 + 32 * EPI_WARPS;
// Slabs per pipeline stage.  One per stage (7 stages) was measured slower (8192 x 2048 x 5632 backward 950 us against 886,
// 16384 x 1024 x 2816 forward 244 against 234): the threads that issue copies and MMAs pay a wait
// per stage; three per stage leave two stages, too few to cover a copy's latency (940, 256).
constexpr int SPS = 2;
constexpr int STAGES = 3;
constexpr uint32_t A_BYTES = BM * BK * 2, B_BYTES = 128 * BK * 2, SLAB_BYTES = A_BYTES + B_BYTES;
constexpr uint32_t STAGE_BYTES = SPS * SLAB_BYTES;
constexpr uint32_t SMEM_BYTES = STAGES * STAGE_BYTES + 1024u;
constexpr uint32_t TMEM_COLS = 2 * BN;
constexpr int MAX_PROBS = 4, MAX_MAPS = 12;
constexpr int GROUP_M = 8;                   // tile rows that are worked through together (L2 reuse)

enum Epi : int { EPI_STORE = 0, EPI_GATE = 1, EPI_GATE_BACK = 2 };

struct Maps { CUtensorMap m[MAX_MAPS]; };

// One product: out [M][N] = sum over its (one or two) operand pairs.
struct Prob {
  int tile_begin, m_tiles, n_tiles;
  int M, N;                 // result extents; EPI_GATE: N = F, a tile is 128 columns of it
  int slabs0, slabs;        // contraction slabs of the first operand pair, of both
  int a_mn, b_mn;           // operand is staged MN-major
  int a_wide, b_wide;       // MN-major map delivers both atoms in one copy
  int map_a[2], map_b[2];   // per operand pair (EPI_GATE: map_b = W1, W3)
  void* out;                // EPI_GATE: H; EPI_GATE_BACK: dG
  void* out2;               // EPI_GATE: G or NULL; EPI_GATE_BACK: dU
  void* out3;               // EPI_GATE: U or NULL
  const void* in1;          // EPI_GATE_BACK: G, U
  const void* in2;
};

struct Params {
  Prob prob[MAX_PROBS];
  int n_probs, total_tiles, n_maps, act;
  int withhold;             // test hook: the first thread block issues no copies
  int* status;
  unsigned long long wait_limit_ns;
};

struct Tile { int q, m, n; };

__device__ __forceinline__ Tile decode(const Params& p, int tile) {
  Tile t;
  t.q = 0;
#pragma unroll
  for (int i = 1; i < MAX_PROBS; ++i)
    if (i < p.n_probs && tile >= p.prob[i].tile_begin) t.q = i;
  const Prob& b = p.prob[t.q];
  const int local = tile - b.tile_begin;
  const int per = GROUP_M * b.n_tiles;
  const int g = local / per, rem = local - g * per;
  const int left = b.m_tiles - g * GROUP_M;
  const int size = left < GROUP_M ? left : GROUP_M;
  t.n = rem / size;
  t.m = g * GROUP_M + (rem - t.n * size);
  return t;
}

// 16 bf16 values (32 bytes) per access where the row allows it, else 8.
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void ld_global_32(const void* p, uint32_t* v) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "l"(p));
}
// 32 consecutive values of a row of which the first `n` (a multiple of 8) exist.
__device__ __forceinline__ void store_row32(__nv_bfloat16* row, const float (&f)[32], int n, bool wide) {
  if (wide && n >= 32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = pack_bf16x2(f[h * 16 + 2 * i], f[h * 16 + 2 * i + 1]);
      st_global_32(row + h * 16, v);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 4; ++h)
      if (h * 8 < n)
        *reinterpret_cast<uint4*>(row + h * 8) =
            make_uint4(pack_bf16x2(f[h * 8], f[h * 8 + 1]), pack_bf16x2(f[h * 8 + 2], f[h * 8 + 3]),
                       pack_bf16x2(f[h * 8 + 4], f[h * 8 + 5]), pack_bf16x2(f[h * 8 + 6], f[h * 8 + 7]));
  }
}
__device__ __forceinline__ void load_row32(const __nv_bfloat16* row, uint32_t (&v)[16], int n, bool wide) {
  if (wide && n >= 32) {
    ld_global_32(row, v);
    ld_global_32(row + 16, v + 8);
  } else {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      uint4 u = make_uint4(0u, 0u, 0u, 0u);
      if (h * 8 < n) u = *reinterpret_cast<const uint4*>(row + h * 8);
      v[h * 4] = u.x; v[h * 4 + 1] = u.y; v[h * 4 + 2] = u.z; v[h * 4 + 3] = u.w;
    }
  }
}

// Two float32 operations per instruction.
struct Pair { uint64_t v; };
__device__ __forceinline__ Pair pair(float a, float b) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ Pair both(float a) { return pair(a, a); }
__device__ __forceinline__ Pair pair_bf16(uint32_t w) { return pair(bf16_lo(w), bf16_hi(w)); }
__device__ __forceinline__ float2 parts(Pair p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p.v));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// act(g) = g sigma and, for the backward pass, its slope.  sigma is the logistic function of g (silu) or of
// 2 sqrt(2 / pi) (g + 0.044715 g^3), which makes g sigma the tanh form of gelu.  The exponential and the quotient are the
// hardware's approximations (a few units in the last place of float32): the results are rounded to 8 bits of mantissa.
// Pairs save issue slots (dG and dU of 4001 tokens at 768 x 2048: 30 -> 19 %), though hardly time there (32 -> 31.5 us).
constexpr float GELU_K = 1.5957691216057308f, GELU_C = 0.044715f, LOG2E = 1.4426950408889634f;
__device__ __forceinline__ Pair sigma2(Pair minus_p_log2e) {
  const float2 q = parts(minus_p_log2e);
  float ex, ey, rx, ry;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ex) : "f"(q.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ey) : "f"(q.y));
  const float2 d = parts(add2(pair(ex, ey), both(1.0f)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rx) : "f"(d.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(ry) : "f"(d.y));
  return pair(rx, ry);
}
// sigma, and in `cube` 0.044715 g^3 (gelu)
template <int ACT>
__device__ __forceinline__ Pair act_sigma(Pair g, Pair& cube) {
  if (ACT == MULOCO_ACT_SILU) return sigma2(mul2(g, both(-LOG2E)));
  cube = mul2(mul2(mul2(g, g), both(GELU_C)), g);
  return sigma2(mul2(add2(cube, g), both(-GELU_K * LOG2E)));
}
template <int ACT>
__device__ __forceinline__ Pair act_value(Pair g) {
  Pair cube;
  return mul2(g, act_sigma<ACT>(g, cube));
}
template <int ACT>
__device__ __forceinline__ void act_both(Pair g, Pair& value, Pair& slope) {
  Pair cube;
  const Pair s = act_sigma<ACT>(g, cube);
  value = mul2(g, s);
  const Pair t = mul2(s, fma2(s, both(-1.0f), both(1.0f)));          // sigma (1 - sigma)
  if (ACT == MULOCO_ACT_SILU) slope = fma2(t, g, s);
  else {
    // the exponent's slope times g is beyond float32 from |g| = 2e13 on, where sigma (1 - sigma) has long been 0: kept finite, so
    // that their product is 0 and not NaN
    const float2 q = parts(fma2(cube, both(3.0f * GELU_K), mul2(g, both(GELU_K))));
    slope = fma2(t, pair(fminf(fmaxf(q.x, -1e38f), 1e38f), fminf(fmaxf(q.y, -1e38f), 1e38f)), s);
  }
}

template <int EPI, int ACT>
__global__ void __launch_bounds__(FFN_THREADS, 1)
ffn_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_full[STAGES];     // used in the CTA of rank 0
  __shared__ __align__(8) uint64_t bar_empty[STAGES];
  __shared__ __align__(8) uint64_t bar_tfull[2];
  __shared__ __align__(8) uint64_t bar_tempty[2];        // used in the CTA of rank 0
  __shared__ uint32_t tmem_base_slot;
  __shared__ volatile int abort_flag;

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint64_t limit = p.wait_limit_ns;
  const int worker = blockIdx.x / CG, workers = gridDim.x / CG;

  if (threadIdx.x == 32 * 2) {
#pragma unroll 1
    for (int i = 0; i < p.n_maps; ++i) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.m[i]) : "memory");
  }
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(smem_u32(&bar_tfull[a]), 1);
      mbar_init(smem_u32(&bar_tempty[a]), EPI_WARPS * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<CG>(smem_u32(&tmem_base_slot), TMEM_COLS);
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_slot;
  // Everything above may run beside the end of the kernel before this one; nothing below does.
  grid_wait();
  grid_release();

  if (warp == 0) {
    // ------------------------------ TMA producer ------------------------------
    if (lane == 0 && !(p.withhold && blockIdx.x == 0)) {
      const uint32_t empty0 = smem_u32(&bar_empty[0]);
      const uint32_t full0 = smem_u32(&bar_full[0]);
      const uint32_t full0_bar = map_to_rank(full0, 0);   // both CTAs' copies are counted on the barrier of rank 0
      uint32_t stage = 0, phase = 0;
      bool alive = true;
      for (int tile = worker; alive && tile < p.total_tiles; tile += workers) {
        const Tile t = decode(p, tile);
        const Prob& b = p.prob[t.q];
        const int row_a = t.m * TM + (int)rank * BM;
        // gated product: this CTA's half of the right operand is W1 (rank 0) or W3 (rank 1), same columns
        const int col_b = (EPI == EPI_GATE) ? t.n * 128 : t.n * BN + (int)rank * 128;
        const int slabs = b.slabs, slabs0 = b.slabs0;
        const bool a_mn = b.a_mn, b_mn = b.b_mn, a_wide = b.a_wide, b_wide = b.b_wide;
        const CUtensorMap* ma = &maps.m[b.map_a[0]];
        const CUtensorMap* mb = &maps.m[b.map_b[(EPI == EPI_GATE) ? (int)rank : 0]];
        const CUtensorMap* ma1 = &maps.m[b.map_a[1]];
        const CUtensorMap* mb1 = &maps.m[b.map_b[1]];
        int k0 = 0;
        for (int kb0 = 0; kb0 < slabs; kb0 += SPS) {
          if (!mbar_wait(empty0 + stage * 8u, phase ^ 1u, &abort_flag, limit)) { alive = false; break; }
          const uint32_t bar = full0_bar + stage * 8u;
          const int here = slabs - kb0 < SPS ? slabs - kb0 : SPS;
          if (rank == 0) mbar_expect_tx(full0 + stage * 8u, CG * SLAB_BYTES * (uint32_t)here);
#pragma unroll
          for (int j = 0; j < SPS; ++j) {
            if (j >= here) break;
            const uint32_t sa = smem_base + stage * STAGE_BYTES + (uint32_t)j * SLAB_BYTES;
            const uint32_t sb = sa + A_BYTES;
            if (kb0 + j == slabs0) { ma = ma1; mb = mb1; k0 = 0; }      // the second operand pair
            if (!a_mn) {
              tma_load_2d_pair(sa, ma, bar, k0, row_a);
            } else if (a_wide) {
              tma_load_3d_pair(sa, ma, bar, 0, k0, row_a >> 6);
            } else {
              tma_load_2d_pair(sa, ma, bar, row_a, k0);
              tma_load_2d_pair(sa + BK * 128, ma, bar, row_a + 64, k0);
            }
            if (!b_mn) {
              tma_load_2d_pair(sb, mb, bar, k0, col_b);
            } else if (b_wide) {
              tma_load_3d_pair(sb, mb, bar, 0, k0, col_b >> 6);
            } else {
              tma_load_2d_pair(sb, mb, bar, col_b, k0);
              tma_load_2d_pair(sb + BK * 128, mb, bar, col_b + 64, k0);
            }
            k0 += BK;
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------- MMA issuer -------------------------------
    if (rank == 0 && lane == 0) {
      // fp32 accumulate, bf16 x bf16; bit 15 / bit 16: left / right operand is MN-major
      constexpr uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) |
                                  ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(TM >> 4) << 24);
      // descriptor halves: high = SBO 1024 B | version 1 | 128-byte swizzle; low = address/16 | LBO/16 << 16
      constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
      constexpr uint32_t LBO_K = (16u >> 4) << 16, LBO_MN = ((uint32_t)(BK * 128) >> 4) << 16;
      constexpr uint32_t STEP_K = (UMMA_K * 2) >> 4, STEP_MN = (UMMA_K * 128) >> 4;
      const uint32_t full0 = smem_u32(&bar_full[0]);
      const uint32_t empty0 = smem_u32(&bar_empty[0]);
      const uint32_t empty0_peer = map_to_rank(empty0, 1);
      const uint32_t tfull0 = smem_u32(&bar_tfull[0]);
      const uint32_t tfull0_peer = map_to_rank(tfull0, 1);
      uint32_t stage = 0, phase = 0;
      int local_tile = 0;
      bool alive = true;
      auto release = [&](uint32_t bar, uint32_t bar_peer) {
        tc_commit<CG>(bar);
        tc_commit<CG>(bar_peer);
      };
      for (int tile = worker; alive && tile < p.total_tiles; tile += workers, ++local_tile) {
        const Tile t = decode(p, tile);
        const Prob& b = p.prob[t.q];
        const uint32_t acc = (uint32_t)local_tile & 1u;
        const uint32_t acc_phase = (uint32_t)(local_tile >> 1) & 1u;
        const uint32_t d_tmem = tmem_base + acc * (uint32_t)BN;
        const bool a_mn = b.a_mn, b_mn = b.b_mn;
        const uint32_t idesc = idesc0 | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16);
        const uint32_t lbo_a = a_mn ? LBO_MN : LBO_K, astep = a_mn ? STEP_MN : STEP_K;
        const uint32_t lbo_b = b_mn ? LBO_MN : LBO_K, bstep = b_mn ? STEP_MN : STEP_K;
        const int slabs = b.slabs;
        if (!mbar_wait(smem_u32(&bar_tempty[acc]), acc_phase ^ 1u, &abort_flag, limit)) break;
        tc_fence_after();
        for (int kb0 = 0; kb0 < slabs; kb0 += SPS) {
          if (!mbar_wait(full0 + stage * 8u, phase, &abort_flag, limit)) { alive = false; break; }
          tc_fence_after();
          const int here = slabs - kb0 < SPS ? slabs - kb0 : SPS;
#pragma unroll
          for (int j = 0; j < SPS; ++j) {
            if (j >= here) break;
            const uint32_t sa = smem_base + stage * STAGE_BYTES + (uint32_t)j * SLAB_BYTES;
            const uint32_t alo = (sa >> 4) | lbo_a, blo = ((sa + A_BYTES) >> 4) | lbo_b;
#pragma unroll
            for (int k = 0; k < BK / UMMA_K; ++k) {
              const uint64_t adesc = ((uint64_t)DESC_HI << 32) | (uint64_t)(alo + (uint32_t)k * astep);
              const uint64_t bdesc = ((uint64_t)DESC_HI << 32) | (uint64_t)(blo + (uint32_t)k * bstep);
              tc_mma_bf16<CG>(d_tmem, adesc, bdesc, idesc, (kb0 > 0 || j > 0 || k > 0) ? 1u : 0u);
            }
          }
          release(empty0 + stage * 8u, empty0_peer + stage * 8u);
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if (alive) release(tfull0 + acc * 8u, tfull0_peer + acc * 8u);
      }
    }
    __syncwarp();
  } else {
    // -------------------------------- epilogue --------------------------------
    const int quarter = warp & 3;                    // tensor-memory lanes [32 * quarter, + 32)
    const int side = (warp - 2) >> 2;                // half of the columns
    int local_tile = 0;
    bool alive = true;
    for (int tile = worker; tile < p.total_tiles; tile += workers, ++local_tile) {
      const Tile t = decode(p, tile);
      const Prob& b = p.prob[t.q];
      const int acc = local_tile & 1;
      const uint32_t acc_phase = (uint32_t)(local_tile >> 1) & 1u;
      const int row = t.m * TM + (int)rank * BM + quarter * 32 + lane;
      const bool row_ok = row < b.M;
      const int64_t row_off = (int64_t)(row_ok ? row : 0) * b.N;
      const bool wide = (b.N & 15) == 0 && ((((uintptr_t)b.out | (uintptr_t)b.out2 | (uintptr_t)b.out3 |
                                              (uintptr_t)b.in1 | (uintptr_t)b.in2) & 31) == 0);
      const uint32_t t_row = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * BN);
      constexpr int CHUNKS = (EPI == EPI_GATE) ? 2 : 4;          // of 32 columns, per warp
      const int c_first = (EPI == EPI_GATE) ? side * 64 : side * (BN / 2);
      const int n_first = (EPI == EPI_GATE) ? t.n * 128 + c_first : t.n * BN + c_first;
      uint32_t gv[16], uv[16];
      if (EPI == EPI_GATE_BACK) {                    // the first chunk's G and U are under way before the accumulator is done
        const int left = row_ok ? b.N - n_first : 0;
        load_row32(reinterpret_cast<const __nv_bfloat16*>(b.in1) + row_off + n_first, gv, left, wide);
        load_row32(reinterpret_cast<const __nv_bfloat16*>(b.in2) + row_off + n_first, uv, left, wide);
      }
      if (!mbar_wait(smem_u32(&bar_tfull[acc]), acc_phase, &abort_flag, limit)) alive = false;
      alive = __all_sync(0xffffffffu, alive);
      if (!alive) break;
      tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < CHUNKS; ++c) {
        const int n0 = n_first + c * 32;
        const int left = row_ok ? b.N - n0 : 0;      // columns of this chunk that exist (may be <= 0)
        uint32_t v[32];
        float f[32];
        __syncwarp();                                // rows past the end leave the stores early
        if (EPI == EPI_STORE) {
          tc_ld32(t_row + (uint32_t)(c_first + c * 32), v);
#pragma unroll
          for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(v[e]);
          if (left > 0) store_row32(reinterpret_cast<__nv_bfloat16*>(b.out) + row_off + n0, f, left, wide);
        } else if (EPI == EPI_GATE) {
          uint32_t w[32];
          tc_ld32(t_row + (uint32_t)(c_first + c * 32), v);
          tc_ld32(t_row + (uint32_t)(128 + c_first + c * 32), w);
          if (left > 0 && b.out2) {
#pragma unroll
            for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(v[e]);
            store_row32(reinterpret_cast<__nv_bfloat16*>(b.out2) + row_off + n0, f, left, wide);
          }
          if (left > 0 && b.out3) {
#pragma unroll
            for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(w[e]);
            store_row32(reinterpret_cast<__nv_bfloat16*>(b.out3) + row_off + n0, f, left, wide);
          }
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 h = parts(mul2(act_value<ACT>(pair(__uint_as_float(v[e]), __uint_as_float(v[e + 1]))),
                                        pair(__uint_as_float(w[e]), __uint_as_float(w[e + 1]))));
            f[e] = h.x; f[e + 1] = h.y;
          }
          if (left > 0) store_row32(reinterpret_cast<__nv_bfloat16*>(b.out) + row_off + n0, f, left, wide);
        } else {
          tc_ld32(t_row + (uint32_t)(c_first + c * 32), v);
          float f2[32];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            Pair value, slope;
            act_both<ACT>(pair_bf16(gv[e >> 1]), value, slope);
            const Pair dh = pair(__uint_as_float(v[e]), __uint_as_float(v[e + 1]));
            const float2 x = parts(mul2(mul2(dh, pair_bf16(uv[e >> 1])), slope)), y = parts(mul2(dh, value));
            f[e] = x.x; f[e + 1] = x.y;
            f2[e] = y.x; f2[e + 1] = y.y;
          }
          if (c + 1 < CHUNKS) {
            load_row32(reinterpret_cast<const __nv_bfloat16*>(b.in1) + row_off + n0 + 32, gv, left - 32, wide);
            load_row32(reinterpret_cast<const __nv_bfloat16*>(b.in2) + row_off + n0 + 32, uv, left - 32, wide);
          }
          if (left > 0) {
            store_row32(reinterpret_cast<__nv_bfloat16*>(b.out) + row_off + n0, f, left, wide);
            store_row32(reinterpret_cast<__nv_bfloat16*>(b.out2) + row_off + n0, f2, left, wide);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_rank(smem_u32(&bar_tempty[acc]), 0));
    }
  }

  // ------------------------------- teardown ----------------------------------
  if (abort_flag) {
    // give copies and MMAs still in flight time to land before memory is released
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  __syncwarp();
  tc_fence_before();
  cluster_sync_all();
  // (only here does every thread know of a wait that ran out: the one that copies may have been done before)
  if (threadIdx.x == 0 && abort_flag) atomicOr(p.status, ST_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc<CG>(tmem_base, TMEM_COLS);
  }
}

// ---------------------------------------------------------------------------
// Few tokens.  The 256 x 256 tiles above leave most of the machine idle when there are few of them, and what counts then
// is to pull the weights out of memory with every SM.  Here the product is turned round: 128 columns of
// a weight matrix are the rows of a tile (the left operand), NT tokens its columns, and the contraction is split over the
// S CTAs of a cluster.  Each CTA sums its share in tensor memory (gated product: two accumulators), the partial
// sums cross the cluster through distributed shared memory, every CTA adds up those of NT / S tokens in the order of
// the ranks and applies the epilogue to them.  The second kernel of a pass starts while the first still runs
// (programmatic dependent launch) and has its weights under way by the time its activations are complete.
// ---------------------------------------------------------------------------
constexpr int FEW_EPI_THREADS = 256;
constexpr int FEW_THREADS = 64 + FEW_EPI_THREADS;   // producer, MMA issuer, eight epilogue warps

template <int EPI, int NT>
struct FewShape {
  static constexpr int ACCS = EPI == EPI_GATE ? 2 : 1;             // weight matrices per tile
  static constexpr uint32_t B_BYTES = NT * BK * 2;
  static constexpr uint32_t STAGE = ACCS * A_BYTES + B_BYTES;
  static constexpr uint32_t REDUCE = ACCS * 128u * NT * 4u;        // partial sums, over the pipeline's space
  static constexpr int STAGES = (int)(200u * 1024u / STAGE) < 8 ? (int)(200u * 1024u / STAGE) : 8;
  static constexpr uint32_t SMEM = (STAGES * STAGE > REDUCE ? STAGES * STAGE : REDUCE) + 1024u;
  static constexpr int COLS = ACCS * NT;                           // accumulator columns in use
  static constexpr uint32_t TMEM = COLS < 32 ? 32u : (uint32_t)COLS;
};

struct FewParams {
  int M, T;                  // rows of the transposed result (columns of the output), tokens
  int slabs0, slabs;
  int a_mn, a_wide;
  int n_weights, n_pairs;    // descriptors in use
  void* out; void* out2; void* out3;
  const void* in1; const void* in2;
  int weights_early;         // the kernel before this one does not write the weights
  int withhold;              // test hook: the first thread block issues no copies
  int* status;
  unsigned long long wait_limit_ns;
};
struct FewMaps { CUtensorMap a[2], b[2]; };  // EPI_GATE: a = W1, W3; else one per operand pair

__device__ __forceinline__ float2 ld_cluster_f32x2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
  return v;
}

template <int EPI, int ACT, int NT>
__global__ void __launch_bounds__(FEW_THREADS, 1)
ffn_few_kernel(const __grid_constant__ FewMaps maps, const __grid_constant__ FewParams p) {
  using Sh = FewShape<EPI, NT>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_full[Sh::STAGES];
  __shared__ __align__(8) uint64_t bar_empty[Sh::STAGES];
  __shared__ __align__(8) uint64_t bar_done;
  __shared__ uint32_t tmem_base_slot;
  __shared__ volatile int abort_flag;

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int S = gridDim.x;                   // CTAs of the cluster
  const int share = blockIdx.x;              // rank in it
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint64_t limit = p.wait_limit_ns;
  const int m0 = blockIdx.y * 128, t0 = blockIdx.z * NT;
  const int kb_first = (int)((int64_t)p.slabs * share / S), kb_end = (int)((int64_t)p.slabs * (share + 1) / S);

  if (threadIdx.x == 64) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a[0]) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b[0]) : "memory");
    if (p.n_weights > 1) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a[1]) : "memory");
    if (p.n_pairs > 1) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b[1]) : "memory");
  }
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < Sh::STAGES; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    mbar_init(smem_u32(&bar_done), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<1>(smem_u32(&tmem_base_slot), Sh::TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_slot;

  if (warp == 0) {
    if (lane == 0 && !(p.withhold && (blockIdx.x | blockIdx.y | blockIdx.z) == 0)) {
      const bool a_mn = p.a_mn, a_wide = p.a_wide;
      const int slabs0 = p.slabs0;
      auto load_weights = [&](int kb, uint32_t stage) {
        const uint32_t sa = smem_base + stage * Sh::STAGE;
        const uint32_t bar = smem_u32(&bar_full[stage]);
        mbar_expect_tx(bar, Sh::STAGE);
        const bool second = kb >= slabs0;
        const int k0 = (second ? kb - slabs0 : kb) * BK;
#pragma unroll
        for (int w = 0; w < Sh::ACCS; ++w) {
          const CUtensorMap* ma = &maps.a[EPI == EPI_GATE ? w : (second ? 1 : 0)];
          const uint32_t dst = sa + (uint32_t)w * A_BYTES;
          if (!a_mn) {
            tma_load_2d(dst, ma, bar, k0, m0);
          } else if (a_wide) {
            tma_load_3d(dst, ma, bar, 0, k0, m0 >> 6);
          } else {
            tma_load_2d(dst, ma, bar, m0, k0);
            tma_load_2d(dst + BK * 128, ma, bar, m0 + 64, k0);
          }
        }
      };
      auto load_tokens = [&](int kb, uint32_t stage) {
        const bool second = kb >= slabs0;
        const int k0 = (second ? kb - slabs0 : kb) * BK;
        tma_load_2d(smem_base + stage * Sh::STAGE + Sh::ACCS * A_BYTES, &maps.b[second ? 1 : 0],
                    smem_u32(&bar_full[stage]), k0, t0);
      };
      // Second kernel of a pass: the weights of its first stages do not depend on the first kernel (which only lets this
      // one start once everything before itself is complete), the activations do.
      const int ahead = kb_end - kb_first < Sh::STAGES ? kb_end - kb_first : Sh::STAGES;
      if (!p.weights_early) grid_wait();
      for (int i = 0; i < ahead; ++i) load_weights(kb_first + i, (uint32_t)i);
      if (p.weights_early) grid_wait();
      grid_release();
      for (int i = 0; i < ahead; ++i) load_tokens(kb_first + i, (uint32_t)i);
      uint32_t stage = 0, phase = 0;
      for (int kb = kb_first + ahead; kb < kb_end; ++kb) {
        if (!mbar_wait(smem_u32(&bar_empty[stage]), phase, &abort_flag, limit)) break;
        load_weights(kb, stage);
        load_tokens(kb, stage);
        if (++stage == (uint32_t)Sh::STAGES) { stage = 0; phase ^= 1u; }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
      constexpr uint32_t LBO_K = (16u >> 4) << 16, LBO_MN = ((uint32_t)(BK * 128) >> 4) << 16;
      constexpr uint32_t STEP_K = (UMMA_K * 2) >> 4, STEP_MN = (UMMA_K * 128) >> 4;
      const bool a_mn = p.a_mn;
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) |
                             ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      const uint32_t lbo_a = a_mn ? LBO_MN : LBO_K, astep = a_mn ? STEP_MN : STEP_K;
      uint32_t stage = 0, phase = 0;
      bool alive = true;
      for (int kb = kb_first; kb < kb_end; ++kb) {
        if (!mbar_wait(smem_u32(&bar_full[stage]), phase, &abort_flag, limit)) { alive = false; break; }
        tc_fence_after();
        const uint32_t sa = smem_base + stage * Sh::STAGE;
        // (the address field has 18 bits; above them a shared address carries the rank in the cluster)
        const uint32_t blo = (((sa + Sh::ACCS * A_BYTES) & 0x3FFFFu) >> 4) | LBO_K;
#pragma unroll
        for (int w = 0; w < Sh::ACCS; ++w) {
          const uint32_t alo = (((sa + (uint32_t)w * A_BYTES) & 0x3FFFFu) >> 4) | lbo_a;
#pragma unroll
          for (int k = 0; k < BK / UMMA_K; ++k) {
            const uint64_t adesc = ((uint64_t)DESC_HI << 32) | (uint64_t)(alo + (uint32_t)k * astep);
            const uint64_t bdesc = ((uint64_t)DESC_HI << 32) | (uint64_t)(blo + (uint32_t)k * STEP_K);
            tc_mma_bf16<1>(tmem_base + (uint32_t)(w * NT), adesc, bdesc, idesc, (kb > kb_first || k > 0) ? 1u : 0u);
          }
        }
        tc_commit<1>(smem_u32(&bar_empty[stage]));
        if (++stage == (uint32_t)Sh::STAGES) { stage = 0; phase ^= 1u; }
      }
      if (alive) tc_commit<1>(smem_u32(&bar_done));
    }
    __syncwarp();
  } else {
    grid_wait();
    grid_release();
    mbar_wait(smem_u32(&bar_done), 0, &abort_flag, limit);   // on a timeout the flag is set and the results do not count
    __syncwarp();
  }
  // Every copy of this CTA has landed and been used: the pipeline's space takes its partial sums,
  // [accumulator][token][128 rows].  CTA r of the cluster finishes tokens r NT / S and on, and fetches the others' sums of
  // them through distributed shared memory (8 bytes a lane; with a 4-byte store per element to the CTA that wants it, the
  // whole forward pass of 90 tokens at 360 x 848 took 19 us against 12).
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const int per = NT / S;                            // tokens that each CTA finishes
  if (warp >= 2) {
    const int quarter = warp & 3, side = (warp - 2) >> 2;
    const int r128 = quarter * 32 + lane;
#pragma unroll 1
    for (int c = side * 32; c < Sh::COLS; c += 64) {
      uint32_t v[32];
      tc_ld32(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)c, v);
#pragma unroll
      for (int e = 0; e < 32; ++e)
        if (c + e < Sh::COLS) sts32(smem_base + (uint32_t)(((c + e) * 128 + r128) * 4), v[e]);
    }
  }
  tc_fence_before();
  if (S > 1) cluster_sync_all(); else __syncthreads();
  tc_fence_after();
  if (warp >= 2) {
    // two neighbouring columns per thread, the tokens over the thread groups, four tokens at a time
    constexpr int GROUPS = FEW_EPI_THREADS / 64, BATCH = 4;
    const int id = threadIdx.x - 64;
    const int r = (id & 63) * 2, m = m0 + r;
    const int left = p.T - (t0 + share * per);       // tokens of this CTA that exist
    const int n_tok = left < per ? left : per;
    auto total = [&](int w, int tl) {                // the CTAs' sums in the order of their ranks
      const uint32_t at = smem_base + (uint32_t)(((w * NT + share * per + tl) * 128 + r) * 4);
      if (S == 1) return ld_cluster_f32x2(at);
      float2 y[8];
#pragma unroll
      for (int src = 0; src < 8; ++src)
        if (src < S) y[src] = ld_cluster_f32x2(map_to_rank(at, (uint32_t)src));
      float2 x = y[0];
#pragma unroll
      for (int src = 1; src < 8; ++src)
        if (src < S) { x.x += y[src].x; x.y += y[src].y; }
      return x;
    };
    auto put = [&](void* base, int64_t o, float a0, float a1) {
      if (base) *reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(base) + o) = pack_bf16x2(a0, a1);
    };
    if (m < p.M) {
      for (int tl0 = id >> 6; tl0 < n_tok; tl0 += GROUPS * BATCH) {
        uint32_t gv[BATCH], uv[BATCH];
        if (EPI == EPI_GATE_BACK) {
#pragma unroll
          for (int j = 0; j < BATCH; ++j) {
            const int tl = tl0 + j * GROUPS;
            if (tl >= n_tok) break;
            const int64_t o = (int64_t)(t0 + share * per + tl) * p.M + m;
            gv[j] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(p.in1) + o);
            uv[j] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(p.in2) + o);
          }
        }
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          const int tl = tl0 + j * GROUPS;
          if (tl >= n_tok) break;
          const int64_t o = (int64_t)(t0 + share * per + tl) * p.M + m;
          const float2 x = total(0, tl);
          if (EPI == EPI_STORE) {
            put(p.out, o, x.x, x.y);
          } else if (EPI == EPI_GATE) {
            const float2 y = total(1, tl);
            put(p.out2, o, x.x, x.y);
            put(p.out3, o, y.x, y.y);
            const float2 h = parts(mul2(act_value<ACT>(pair(x.x, x.y)), pair(y.x, y.y)));
            put(p.out, o, h.x, h.y);
          } else {
            Pair value, slope;
            act_both<ACT>(pair_bf16(gv[j]), value, slope);
            const Pair dh = pair(x.x, x.y);
            const float2 dg = parts(mul2(mul2(dh, pair_bf16(uv[j])), slope)), du = parts(mul2(dh, value));
            put(p.out, o, dg.x, dg.y);
            put(p.out2, o, du.x, du.y);
          }
        }
      }
    }
  }
  if (abort_flag) {
    const uint64_t t1 = global_timer_ns();           // let copies and MMAs still in flight land
    while (global_timer_ns() - t1 < 200000ull) __nanosleep(1000);
    if (threadIdx.x == 0) atomicOr(p.status, ST_TIMEOUT);
  }
  // (a CTA's sums stay until the others have fetched them)
  __syncwarp();
  if (S > 1) cluster_sync_all(); else __syncthreads();
  if (warp == 1) tmem_dealloc<1>(tmem_base, Sh::TMEM);
}

// ------------------------------ host side ----------------------------------
// Makes the current device's context this thread's: the descriptor encoder is a driver call, which fails in a
// thread that has made no runtime call yet (a backward pass runs in a thread of its own).
cudaError_t bind_context(const char** what) {
  *what = "cudaSetDevice";
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  return e == cudaSuccess ? cudaSetDevice(dev) : e;
}

// A row-major bf16 matrix as an operand: rows x cols with row pitch ld.
struct Mat { const void* p; int64_t rows, cols, ld; };

bool encode(CUtensorMap* out, const Mat& a, int box_cols, int box_rows) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)a.cols, (cuuint64_t)a.rows};
  cuuint64_t strides[1] = {(cuuint64_t)a.ld * 2};
  cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.p), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same matrix as [cols / 64][rows][64]: both atoms of an MN-major slab in one copy.
bool encode_wide(CUtensorMap* out, const Mat& a) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn || (a.cols & 63) != 0) return false;
  cuuint64_t dims[3] = {64, (cuuint64_t)a.rows, (cuuint64_t)(a.cols / 64)};
  cuuint64_t strides[2] = {(cuuint64_t)a.ld * 2, 128};
  cuuint32_t box[3] = {64, (cuuint32_t)BK, 2};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.p), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Builder {
  Maps maps;
  Params p;
  int n_maps = 0;
  bool ok = true;
  Builder() { memset(&p, 0, sizeof p); }
  int kmajor(const Mat& a) {
    ok = ok && n_maps < MAX_MAPS && encode(&maps.m[n_maps], a, BK, 128);
    return n_maps++;
  }
  int mnmajor(const Mat& a, int* wide) {
    if (n_maps >= MAX_MAPS) { ok = false; return 0; }
    *wide = encode_wide(&maps.m[n_maps], a);
    if (!*wide) ok = ok && encode(&maps.m[n_maps], a, 64, BK);
    return n_maps++;
  }
  // A product of M x N results; its tiles follow those of the products before it.
  Prob& add(int64_t M, int64_t N, int tile_n, int64_t k0, int64_t k1) {
    Prob& b = p.prob[p.n_probs++];
    b.tile_begin = p.total_tiles;
    b.m_tiles = (int)((M + TM - 1) / TM);
    b.n_tiles = (int)((N + tile_n - 1) / tile_n);
    b.M = (int)M; b.N = (int)N;
    b.slabs0 = (int)((k0 + BK - 1) / BK);
    b.slabs = b.slabs0 + (int)((k1 + BK - 1) / BK);
    p.total_tiles += b.m_tiles * b.n_tiles;
    return b;
  }
};

// Raises a kernel's shared-memory limit, once per device (`allowed`: a bit for each of the first 64 that it was raised on; calls
// may come from several threads).
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>* allowed) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (e != cudaSuccess || (allowed->load(std::memory_order_relaxed) & bit)) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) allowed->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <int EPI, int ACT>
cudaError_t launch_kernel(cudaStream_t st, const Builder& b, int n_sms) {
  auto kernel = ffn_kernel<EPI, ACT>;
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(kernel, (int)SMEM_BYTES, &allowed);
  if (e != cudaSuccess) return e;
  const int units = n_sms / CG;
  const int workers = b.p.total_tiles < units ? b.p.total_tiles : units;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)(workers * CG));
  cfg.blockDim = dim3(FFN_THREADS);
  cfg.dynamicSmemBytes = SMEM_BYTES;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = CG; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, b.maps, b.p);
}

cudaError_t launch_built(cudaStream_t st, Builder& b, const FfnArgs& a, int epi, const int* launches, const char** what) {
  *what = "cuTensorMapEncodeTiled";
  if (!b.ok) return cudaErrorInvalidValue;
  *what = "launch of the feed-forward kernel";
  b.p.n_maps = b.n_maps;
  b.p.act = a.act;
  b.p.withhold = a.withhold && *launches == 0;
  b.p.status = a.status;
  b.p.wait_limit_ns = a.wait_limit_ns ? a.wait_limit_ns : 2000000000ull;
  const bool gelu = a.act == MULOCO_ACT_GELU;
  if (epi == EPI_GATE)
    return gelu ? launch_kernel<EPI_GATE, MULOCO_ACT_GELU>(st, b, a.n_sms) : launch_kernel<EPI_GATE, MULOCO_ACT_SILU>(st, b, a.n_sms);
  if (epi == EPI_GATE_BACK)
    return gelu ? launch_kernel<EPI_GATE_BACK, MULOCO_ACT_GELU>(st, b, a.n_sms)
                : launch_kernel<EPI_GATE_BACK, MULOCO_ACT_SILU>(st, b, a.n_sms);
  return launch_kernel<EPI_STORE, MULOCO_ACT_SILU>(st, b, a.n_sms);
}

// ---- few tokens ----
template <int EPI, int ACT, int NT>
cudaError_t launch_few_kernel(cudaStream_t st, const FewMaps& m, const FewParams& p, int split) {
  auto kernel = ffn_few_kernel<EPI, ACT, NT>;
  using Sh = FewShape<EPI, NT>;
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(kernel, (int)Sh::SMEM, &allowed);
  if (e != cudaSuccess) return e;
  // only the stages that the CTA's slabs use, so that the next kernel's blocks may find room beside this one's
  const int slabs = (p.slabs + split - 1) / split;
  const uint32_t used = (uint32_t)(slabs < Sh::STAGES ? slabs : Sh::STAGES) * Sh::STAGE;
  const size_t smem = (used > Sh::REDUCE ? used : Sh::REDUCE) + 1024u;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)split, (unsigned)((p.M + 127) / 128), (unsigned)((p.T + NT - 1) / NT));
  cfg.blockDim = dim3(FEW_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = split; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, m, p);
}

template <int EPI, int ACT>
cudaError_t launch_few_nt(cudaStream_t st, int nt, const FewMaps& m, const FewParams& p, int split) {
  if (nt == 16) return launch_few_kernel<EPI, ACT, 16>(st, m, p, split);
  if (nt == 32) return launch_few_kernel<EPI, ACT, 32>(st, m, p, split);
  if (nt == 64) return launch_few_kernel<EPI, ACT, 64>(st, m, p, split);
  return launch_few_kernel<EPI, ACT, 128>(st, m, p, split);
}

// Tokens per tile.  Wider tiles read the weights fewer times and give fewer CTAs more to do; above 64 tokens, tiles of
// 64 only where they are few.  Whole forward pass, us, tiles of 64 / 128: 256 tokens at 2048 x 5632 (176 tiles of 64)
// 44 / 38, 512 at 1024 x 2816 29 / 27; 64 tokens at 2048 x 5632 30 / 34.
int few_tile(int64_t T, int64_t M, int n_sms) {
  if (T <= 64) return T <= 16 ? 16 : T <= 32 ? 32 : 64;
  return (M + 127) / 128 * ((T + 63) / 64) <= n_sms / 4 ? 64 : 128;
}

struct FewOperand { Mat weight[2]; Mat tokens[2]; };   // per operand pair (gated product: weight = W1, W3)

// One product of the few-token form.  `mn`: the weights are stored contraction index first (MN-major operand).
cudaError_t launch_few(cudaStream_t st, const FfnArgs& a, int epi, const FewOperand& q, bool mn, int n_pairs,
                       FewParams p, const int* launches, const char** what) {
  const int nt = few_tile(a.T, p.M, a.n_sms);
  FewMaps m;
  bool ok = true;
  const int n_weights = epi == EPI_GATE ? 2 : n_pairs;
  p.a_mn = mn;
  p.n_weights = n_weights;
  p.n_pairs = n_pairs;
  for (int w = 0; w < n_weights; ++w) {
    if (mn) {
      const bool wide = encode_wide(&m.a[w], q.weight[w]);
      if (w && wide != (p.a_wide != 0)) ok = false;
      p.a_wide = wide;
      if (!wide) ok = ok && encode(&m.a[w], q.weight[w], 64, BK);
    } else {
      ok = ok && encode(&m.a[w], q.weight[w], BK, 128);
    }
  }
  for (int w = 0; w < n_pairs; ++w) ok = ok && encode(&m.b[w], q.tokens[w], BK, nt);
  *what = "cuTensorMapEncodeTiled";
  if (!ok) return cudaErrorInvalidValue;
  *what = "launch of the feed-forward kernel for few tokens";
  p.T = (int)a.T;
  p.withhold = a.withhold && *launches == 0;
  p.status = a.status;
  p.wait_limit_ns = a.wait_limit_ns ? a.wait_limit_ns : 2000000000ull;
  // Split the contraction until every SM has a CTA.  Clusters of four and eight only while all of them find room at once,
  // which takes whole groups of neighbouring SMs: a second wave of clusters costs more than the split gains (36 tiles in clusters
  // of four: 30 us for the pass, 24 tiles: 24).
  const int64_t tiles = (int64_t)((p.M + 127) / 128) * ((a.T + nt - 1) / nt);
  int split = 1;
  if (p.slabs >= 2 && tiles * 2 <= a.n_sms) split = 2;
  if (p.slabs >= 4 && tiles * 4 <= a.n_sms * 7 / 8) split = 4;
  if (p.slabs >= 8 && tiles * 8 <= a.n_sms * 2 / 3) split = 8;
  const bool gelu = a.act == MULOCO_ACT_GELU;
  if (epi == EPI_GATE)
    return gelu ? launch_few_nt<EPI_GATE, MULOCO_ACT_GELU>(st, nt, m, p, split) : launch_few_nt<EPI_GATE, MULOCO_ACT_SILU>(st, nt, m, p, split);
  if (epi == EPI_GATE_BACK)
    return gelu ? launch_few_nt<EPI_GATE_BACK, MULOCO_ACT_GELU>(st, nt, m, p, split)
                : launch_few_nt<EPI_GATE_BACK, MULOCO_ACT_SILU>(st, nt, m, p, split);
  return launch_few_nt<EPI_STORE, MULOCO_ACT_SILU>(st, nt, m, p, split);
}

int slabs_of(int64_t k) { return (int)((k + BK - 1) / BK); }

// Whether a product of T x N results takes the few-token form: while it has at most a tile of 128 x 128 per SM, up to
// `tokens` tokens, or any number of them while it has at most `tiles` tiles.  Whole pass in us, one side / the other:
//   gated product, few-token form / 256 x 256 tiles: 100 tokens 14 / 25 (768 x 2048), 34 / 54 (2048 x 5632); 256 tokens
//     19 / 17, 38 / 33; 512 tokens 24 / 19, 17 / 14 (360 x 848)
//   Y = H W2: 600 tokens 19 / 26 (768 x 2048, 30 tiles), 1500 tokens 29 / 31 (72 tiles), 38 / 39 (1024 x 2816, 96 tiles)
//   dG and dU: 2048 tokens at 744 x 424 (64 tiles) 33 / 48; 1500 at 360 x 848 (84 tiles) 40 / 41
//   dX: 3000 tokens at 360 x 848 (72 tiles) 53 / 40; 1024 at 768 x 2048 (48 tiles) 47 / 47
struct FewLimit { int64_t tokens, tiles; };
constexpr FewLimit FEW_GATE = {128, 0}, FEW_DOWN = {512, 100}, FEW_GATE_BACK = {512, 64}, FEW_DX = {512, 64};
bool few_tokens(int64_t T, int64_t N, int n_sms, FewLimit limit) {
  const int64_t tiles = (N + 127) / 128 * ((T + 127) / 128);
  return tiles <= n_sms && (T <= limit.tokens || tiles <= limit.tiles);
}
bool few_tokens(const FfnArgs& a, int64_t N, FewLimit limit) { return few_tokens(a.T, N, a.n_sms, limit); }

}  // namespace

int ffn_forms(int64_t T, int64_t d, int64_t F, int n_sms, int64_t* tiles) {
  const int forms = (few_tokens(T, F, n_sms, FEW_GATE) ? 0 : MULOCO_FFN_GATE) | (few_tokens(T, d, n_sms, FEW_DOWN) ? 0 : MULOCO_FFN_Y) |
                    (few_tokens(T, F, n_sms, FEW_GATE_BACK) ? 0 : MULOCO_FFN_GATE_BACK) |
                    (few_tokens(T, d, n_sms, FEW_DX) ? 0 : MULOCO_FFN_DX);
  if (tiles) {
    auto of = [](int64_t m, int64_t n, int64_t width) { return (m + TM - 1) / TM * ((n + width - 1) / width); };
    tiles[0] = forms & MULOCO_FFN_GATE ? of(T, F, 128) : 0;
    tiles[1] = forms & MULOCO_FFN_Y ? of(T, d, BN) : 0;
    tiles[2] = forms & MULOCO_FFN_GATE_BACK ? of(T, F, BN) : 0;
    tiles[3] = 2 * of(d, F, BN) + of(F, d, BN) + (forms & MULOCO_FFN_DX ? of(T, d, BN) : 0);
  }
  return forms;
}

cudaError_t launch_ffn(cudaStream_t st, const FfnArgs& a, int* launches, const char** what) {
  cudaError_t bound = bind_context(what);
  if (bound != cudaSuccess) return bound;
  if (few_tokens(a, a.F, FEW_GATE)) {
    FewParams p;
    memset(&p, 0, sizeof p);
    p.M = (int)a.F; p.slabs0 = p.slabs = slabs_of(a.d);
    p.out = a.h; p.out2 = a.g; p.out3 = a.u;
    FewOperand q{{Mat{a.w1, a.d, a.F, a.ldw1}, Mat{a.w3, a.d, a.F, a.ldw3}}, {Mat{a.x, a.T, a.d, a.ldx}, Mat{}}};
    const cudaError_t e = launch_few(st, a, EPI_GATE, q, true, 1, p, launches, what);
    if (e != cudaSuccess) return e;
  } else {
    Builder b;
    Prob& q = b.add(a.T, a.F, 128, a.d, 0);
    q.map_a[0] = b.kmajor(Mat{a.x, a.T, a.d, a.ldx});
    q.b_mn = 1;
    q.map_b[0] = b.mnmajor(Mat{a.w1, a.d, a.F, a.ldw1}, &q.b_wide);
    int wide3 = 0;
    q.map_b[1] = b.mnmajor(Mat{a.w3, a.d, a.F, a.ldw3}, &wide3);
    b.ok = b.ok && wide3 == q.b_wide;
    q.out = a.h; q.out2 = a.g; q.out3 = a.u;
    const cudaError_t e = launch_built(st, b, a, EPI_GATE, launches, what);
    if (e != cudaSuccess) return e;
  }
  ++*launches;
  cudaError_t e;
  if (few_tokens(a, a.d, FEW_DOWN)) {
    FewParams p;
    memset(&p, 0, sizeof p);
    p.M = (int)a.d; p.slabs0 = p.slabs = slabs_of(a.F);
    p.out = a.y;
    p.weights_early = 1;
    FewOperand r{{Mat{a.w2, a.F, a.d, a.ldw2}, Mat{}}, {Mat{a.h, a.T, a.F, a.F}, Mat{}}};
    e = launch_few(st, a, EPI_STORE, r, true, 1, p, launches, what);
  } else {
    Builder b;
    Prob& q = b.add(a.T, a.d, BN, a.F, 0);
    q.map_a[0] = b.kmajor(Mat{a.h, a.T, a.F, a.F});
    q.b_mn = 1;
    q.map_b[0] = b.mnmajor(Mat{a.w2, a.F, a.d, a.ldw2}, &q.b_wide);
    q.out = a.y;
    e = launch_built(st, b, a, EPI_STORE, launches, what);
  }
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_ffn_backward(cudaStream_t st, const FfnArgs& a, int* launches, const char** what) {
  cudaError_t bound = bind_context(what);
  if (bound != cudaSuccess) return bound;
  const bool few = few_tokens(a, a.d, FEW_DX);
  if ((a.dx || a.dw1 || a.dw3) && few_tokens(a, a.F, FEW_GATE_BACK)) {
    FewParams p;
    memset(&p, 0, sizeof p);
    p.M = (int)a.F; p.slabs0 = p.slabs = slabs_of(a.d);
    p.in1 = a.g; p.in2 = a.u;
    p.out = a.dg; p.out2 = a.du;
    FewOperand q{{Mat{a.w2, a.F, a.d, a.ldw2}, Mat{}}, {Mat{a.dy, a.T, a.d, a.lddy}, Mat{}}};
    cudaError_t e = launch_few(st, a, EPI_GATE_BACK, q, false, 1, p, launches, what);
    if (e != cudaSuccess) return e;
    ++*launches;
  } else if (a.dx || a.dw1 || a.dw3) {
    Builder b;
    Prob& q = b.add(a.T, a.F, BN, a.d, 0);
    q.map_a[0] = b.kmajor(Mat{a.dy, a.T, a.d, a.lddy});
    q.map_b[0] = b.kmajor(Mat{a.w2, a.F, a.d, a.ldw2});
    q.in1 = a.g; q.in2 = a.u;
    q.out = a.dg; q.out2 = a.du;
    cudaError_t e = launch_built(st, b, a, EPI_GATE_BACK, launches, what);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  if (a.dx && few) {
    FewParams p;
    memset(&p, 0, sizeof p);
    p.M = (int)a.d; p.slabs0 = slabs_of(a.F); p.slabs = 2 * p.slabs0;
    p.out = a.dx;
    p.weights_early = 1;
    FewOperand q{{Mat{a.w1, a.d, a.F, a.ldw1}, Mat{a.w3, a.d, a.F, a.ldw3}},
                 {Mat{a.dg, a.T, a.F, a.F}, Mat{a.du, a.T, a.F, a.F}}};
    cudaError_t e = launch_few(st, a, EPI_STORE, q, false, 2, p, launches, what);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  Builder b;
  const Mat dg{a.dg, a.T, a.F, a.F}, du{a.du, a.T, a.F, a.F};
  if (a.dx && !few) {
    Prob& q = b.add(a.T, a.d, BN, a.F, a.F);
    q.map_a[0] = b.kmajor(dg);
    q.map_a[1] = b.kmajor(du);
    q.map_b[0] = b.kmajor(Mat{a.w1, a.d, a.F, a.ldw1});
    q.map_b[1] = b.kmajor(Mat{a.w3, a.d, a.F, a.ldw3});
    q.out = a.dx;
  }
  const Mat x{a.x, a.T, a.d, a.ldx};
  for (int w = 0; w < 2; ++w) {
    void* out = w ? a.dw3 : a.dw1;
    if (!out) continue;
    Prob& q = b.add(a.d, a.F, BN, a.T, 0);
    q.a_mn = q.b_mn = 1;
    q.map_a[0] = b.mnmajor(x, &q.a_wide);
    q.map_b[0] = b.mnmajor(w ? du : dg, &q.b_wide);
    q.out = out;
  }
  if (a.dw2) {
    Prob& q = b.add(a.F, a.d, BN, a.T, 0);
    q.a_mn = q.b_mn = 1;
    q.map_a[0] = b.mnmajor(Mat{a.h, a.T, a.F, a.F}, &q.a_wide);
    q.map_b[0] = b.mnmajor(Mat{a.dy, a.T, a.d, a.lddy}, &q.b_wide);
    q.out = a.dw2;
  }
  if (!b.p.n_probs) return cudaSuccess;
  cudaError_t e = launch_built(st, b, a, EPI_STORE, launches, what);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace muloco
