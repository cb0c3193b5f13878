// Norm over the last dimension, centred (layer norm) or not (root mean square), with the residual sum in front of it, and its
// backward pass.
//
//   h = x + residual,  m = mean h (0 if not centred),  r = 1 / sqrt(mean (h - m)^2 + eps),  n = (h - m) r,  y = n weight + bias
//   backward:  e = dy weight,  dx = r (e - n mean(e n) - mean e) + dh   (mean e only if centred),
//              dweight = sum over tokens of dy n,  dbias = sum over tokens of dy
//
// Bound by memory: every tensor crosses it once, so a row stays in registers between the statistics and the result.  A row is
// held by WPR warps, E entries per lane; the variance is taken around the mean in a second pass over the registers.  The
// sums over tokens: each block adds up its own rows in registers and leaves a partial sum, and a second kernel adds those in the
// order of the blocks.
//
// Measured: 16384 x 2048, bf16, with the residual, forward 46 us (5.8 TB/s, 0.89 of the copy rate); 16384 x 1024, bf16, centred, with dh, backward
// 33 us (4.0 TB/s; 26 in the first kernel, the rest joins the sums), from 66 with loads when a row begins, 58 with 16 entries
// per lane and the next row's loads early in registers, which the compiler moved back.
// float32, 16384 x 2048: forward 80 us, backward 86 (6.7, 6.3 TB/s).  Wider than 8192 entries a thread spills, and a block is one row: bf16 with the
// residual (dh), forward / backward: 4096 x 8192 50 / 106 us, 2048 x 16384 96 / 150, 1024 x 32768 70 / 417 (each moves what takes 41 at the copy rate).
#include <string.h>

#include "convert.cuh"
#include "internal.h"
#include "tc_ptx.cuh"

namespace muloco {

namespace {

// E entries of a row in a lane: chunks of V neighbouring entries, chunk c of lane l starts at (c lanes + l) V.
template <typename T, int V> struct alignas(sizeof(T) * V) Chunk { T v[V]; };

template <typename T, int V, int E>
struct Row {
  Chunk<T, V> c[E / V];
  __device__ __forceinline__ float at(int i) const { return to_f32(c[i / V].v[i % V]); }
};

template <int V>
__device__ __forceinline__ int column(int chunk, int lane, int lanes) { return (chunk * lanes + lane) * V; }

template <typename T, int V, int E>
__device__ __forceinline__ void load_row(Row<T, V, E>& r, const T* p, int d, int lane, int lanes) {
#pragma unroll
  for (int c = 0; c < E / V; ++c) {
    const int col = column<V>(c, lane, lanes);
    if (col < d) {
      r.c[c] = *reinterpret_cast<const Chunk<T, V>*>(p + col);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) r.c[c].v[i] = from_f32<T>(0.f);
    }
  }
}
template <typename T, int V, int E>
__device__ __forceinline__ void store_row(const float (&f)[E], T* p, int d, int lane, int lanes) {
#pragma unroll
  for (int c = 0; c < E / V; ++c) {
    const int col = column<V>(c, lane, lanes);
    Chunk<T, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.v[i] = from_f32<T>(f[c * V + i]);
    if (col < d) *reinterpret_cast<Chunk<T, V>*>(p + col) = o;
  }
}
// float32 vectors of the row's columns (weight, bias)
template <int V>
__device__ __forceinline__ void load_vector(float (&w)[V], const float* p, int col, int d, float otherwise) {
  if (p && col < d) {
    constexpr int W = V % 4 == 0 ? 4 : 1;      // (columns of a chunk of 8 are two accesses of 16 bytes)
#pragma unroll
    for (int i = 0; i < V; i += W) {
      const Chunk<float, W> q = *reinterpret_cast<const Chunk<float, W>*>(p + col + i);
#pragma unroll
      for (int k = 0; k < W; ++k) w[i + k] = q.v[k];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = otherwise;
  }
}

// Sum over the lanes of a row's WPR warps, the same in all of them.  `slots`: WPR floats of this row group; a group's calls alternate
// between two sets of them, so that one barrier is enough.
template <int WPR, int N>
__device__ __forceinline__ void row_sum(float (&x)[N], float* slots, int group, int warp_in_row) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int o = 16; o; o >>= 1) x[n] += __shfl_xor_sync(0xffffffffu, x[n], o);
  if (WPR > 1) {
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) slots[n * WPR + warp_in_row] = x[n];
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(WPR * 32) : "memory");
#pragma unroll
    for (int n = 0; n < N; ++n) {
      x[n] = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) x[n] += slots[n * WPR + w];
    }
  }
}

constexpr int BLOCK_WARPS = 8;
template <int WPR> __host__ __device__ constexpr int block_warps() { return WPR > BLOCK_WARPS ? WPR : BLOCK_WARPS; }

template <typename T, int V, int E, int WPR>
__global__ void __launch_bounds__(block_warps<WPR>() * 32)
norm_kernel(const NormArgs a) {
  constexpr int GROUPS = block_warps<WPR>() / WPR;
  __shared__ float slots[GROUPS][2][WPR];
  const int warp = threadIdx.x >> 5, group = warp / WPR, in_row = warp % WPR;
  const int lane = in_row * 32 + (threadIdx.x & 31), lanes = WPR * 32;
  const int64_t row = (int64_t)blockIdx.x * GROUPS + group;
  grid_wait();
  grid_release();
  if (row >= a.tokens) return;                 // (a whole row group)
  const int d = a.d;
  Row<T, V, E> x, r;
  load_row(x, reinterpret_cast<const T*>(a.x) + row * a.ldx, d, lane, lanes);
  if (a.residual) load_row(r, reinterpret_cast<const T*>(a.residual) + row * a.ldr, d, lane, lanes);
  float f[E];
#pragma unroll
  for (int i = 0; i < E; ++i) f[i] = x.at(i);
  if (a.residual) {
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] += r.at(i);
    store_row<T, V, E>(f, reinterpret_cast<T*>(a.h) + row * d, d, lane, lanes);
  }
  float mean = 0.f;
  if (a.center) {
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < E; ++i) s[0] += f[i];  // (entries past the end are zero)
    row_sum<WPR, 1>(s, slots[group][0], group, in_row);
    mean = s[0] * a.inv_d;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int c = 0; c < E / V; ++c) {
    const bool in = column<V>(c, lane, lanes) < d;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      f[c * V + i] = in ? f[c * V + i] - mean : 0.f;
      q[0] += f[c * V + i] * f[c * V + i];
    }
  }
  row_sum<WPR, 1>(q, slots[group][1], group, in_row);
  const float rstd = 1.0f / sqrtf(q[0] * a.inv_d + a.eps);
#pragma unroll
  for (int c = 0; c < E / V; ++c) {
    const int col = column<V>(c, lane, lanes);
    float w[V], b[V];
    load_vector<V>(w, a.weight, col, d, 1.f);
    load_vector<V>(b, a.bias, col, d, 0.f);
#pragma unroll
    for (int i = 0; i < V; ++i) f[c * V + i] = f[c * V + i] * rstd * w[i] + b[i];
  }
  store_row<T, V, E>(f, reinterpret_cast<T*>(a.y) + row * d, d, lane, lanes);
  if (lane == 0) {
    a.rstd[row] = rstd;
    if (a.center) a.mean[row] = mean;
  }
}

// Rows under way in the backward pass: every lane copies the chunks that it will read itself into shared memory (cp.async), STAGES rows
// ahead, which takes neither registers nor barriers.  Where 16 bytes are not one access, or a row is so long that two of them do not fit, rows
// are loaded when they are needed.
template <typename T, int V, int E, int WPR>
struct BackShape {
  static constexpr int THREADS = block_warps<WPR>() * 32, GROUPS = block_warps<WPR>() / WPR;
  static constexpr int STAGES = sizeof(T) * V == 16 && WPR <= 8 ? (sizeof(T) == 2 ? 4 : 2) : 0;
  static constexpr int STAGE = 3 * E * (int)sizeof(T) * THREADS;        // bytes: dy, h, dh
  static size_t smem(int d, bool sums) {
    const size_t a = (size_t)STAGES * STAGE, b = sums && GROUPS > 1 ? (size_t)GROUPS * d * 4 : 0;
    return a > b ? a : b;
  }
};

__device__ __forceinline__ void copy_async16(void* dst, const void* src, bool some) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(some ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T, int V, int E, int WPR>
__global__ void __launch_bounds__(block_warps<WPR>() * 32, block_warps<WPR>() == 8 ? 2 : 1)
norm_back_kernel(const NormArgs a) {
  using Sh = BackShape<T, V, E, WPR>;
  constexpr int GROUPS = Sh::GROUPS, STAGES = Sh::STAGES, CHUNKS = E / V;
  __shared__ float slots[GROUPS][2][2 * WPR];
  extern __shared__ __align__(16) uint8_t staging[];           // rows under way, then the sums of the block's row groups
  float* const sums = reinterpret_cast<float*>(staging);
  const int warp = threadIdx.x >> 5, group = warp / WPR, in_row = warp % WPR;
  const int lane = in_row * 32 + (threadIdx.x & 31), lanes = WPR * 32;
  const int d = a.d;
  grid_wait();
  grid_release();
  float dw[E], db[E];
#pragma unroll
  for (int i = 0; i < E; ++i) { dw[i] = 0.f; db[i] = 0.f; }
  int turn = 0;
  const int64_t stride = (int64_t)gridDim.x * GROUPS;
  const int64_t first = (int64_t)blockIdx.x * GROUPS + group;
  const T* const gp = reinterpret_cast<const T*>(a.dy);
  const T* const hp = reinterpret_cast<const T*>(a.x);
  const T* const sp = reinterpret_cast<const T*>(a.dh);
  using Ch = Chunk<T, V>;
  // this thread's chunk c of tensor `which` in a stage
  auto place = [&](int stage, int which, int c) {
    return reinterpret_cast<Ch*>(staging + (size_t)stage * Sh::STAGE + ((size_t)(which * CHUNKS + c) * Sh::THREADS + threadIdx.x) * sizeof(Ch));
  };
  auto send = [&](int stage, int64_t row) {
    if (row < a.tokens) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        const int col = column<V>(c, lane, lanes);
        const bool in = col < d;
        const int at = in ? col : 0;
        copy_async16(place(stage, 0, c), gp + row * a.ldy + at, in);
        copy_async16(place(stage, 1, c), hp + row * a.ldx + at, in);
        if (sp) copy_async16(place(stage, 2, c), sp + row * a.ldr + at, in);
      }
    }
    copy_commit();
  };
  int stage = 0;
  if (STAGES) {
#pragma unroll
    for (int k = 0; k < STAGES; ++k) send(k, first + k * stride);
  }
  for (int64_t row = first; row < a.tokens; row += stride, turn ^= 1) {
    const float rstd = a.rstd[row], mean = a.center ? a.mean[row] : 0.f;
    Row<T, V, E> g, h, s;
    if (STAGES) {
      copy_wait<STAGES ? STAGES - 1 : 0>();
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        g.c[c] = *place(stage, 0, c);
        h.c[c] = *place(stage, 1, c);
      }
    } else {
      load_row(g, gp + row * a.ldy, d, lane, lanes);
      load_row(h, hp + row * a.ldx, d, lane, lanes);
      if (sp) load_row(s, sp + row * a.ldr, d, lane, lanes);
    }
    float n[E], e[E], t[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < E / V; ++c) {
      const int col = column<V>(c, lane, lanes);
      float w[V];
      load_vector<V>(w, a.weight, col, d, 1.f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int k = c * V + i;
        const float dy = g.at(k);              // zero past the end, which keeps such entries out of every sum
        n[k] = (h.at(k) - mean) * rstd;
        dw[k] += dy * n[k];
        db[k] += dy;
        e[k] = dy * w[i];
        t[0] += e[k] * n[k];
        t[1] += e[k];
      }
    }
    row_sum<WPR, 2>(t, slots[group][turn], group, in_row);
    const float along = t[0] * a.inv_d, common = a.center ? t[1] * a.inv_d : 0.f;
#pragma unroll
    for (int k = 0; k < E; ++k) e[k] = rstd * (e[k] - n[k] * along - common);
    if (sp) {
      if (STAGES) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) s.c[c] = *place(stage, 2, c);
      }
#pragma unroll
      for (int k = 0; k < E; ++k) e[k] += s.at(k);
    }
    if (STAGES) {                              // (this thread has read all that it copied there)
      send(stage, row + STAGES * stride);
      if (++stage == STAGES) stage = 0;
    }
    store_row<T, V, E>(e, reinterpret_cast<T*>(a.dx) + row * d, d, lane, lanes);
  }
  if (STAGES) copy_wait<0>();
  if (!a.partials) return;
  // partial sums of the block: its row groups one after the other
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which ? !a.dbias : !a.dweight) continue;
    const float* mine = which ? db : dw;
    float* out = a.partials + ((int64_t)blockIdx.x * 2 + which) * d;
    if (GROUPS > 1) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < E / V; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int col = column<V>(c, lane, lanes) + i;
          if (col < d) sums[group * d + col] = mine[c * V + i];
        }
      __syncthreads();
      for (int col = threadIdx.x; col < d; col += blockDim.x) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) s += sums[k * d + col];
        out[col] = s;
      }
    } else {
#pragma unroll
      for (int c = 0; c < E / V; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int col = column<V>(c, lane, lanes) + i;
          if (col < d) out[col] = mine[c * V + i];
        }
    }
  }
}

// dweight and dbias from the blocks' partial sums: 32 columns per block, 16 threads per column take every 16th block's.
constexpr int JOIN = 16;
__global__ void __launch_bounds__(32 * JOIN)
norm_join_kernel(const float* partials, int parts, int d, float* dweight, float* dbias) {
  __shared__ float sums[JOIN][32];
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int which = blockIdx.y, col = blockIdx.x * 32 + lane;
  float* out = which ? dbias : dweight;
  grid_wait();
  grid_release();
  if (!out) return;
  float s = 0.f;
  if (col < d)
#pragma unroll 4
    for (int p = k; p < parts; p += JOIN) s += partials[((int64_t)p * 2 + which) * d + col];
  sums[k][lane] = s;
  __syncthreads();
  if (k == 0 && col < d) {
#pragma unroll
    for (int i = 1; i < JOIN; ++i) s += sums[i][lane];
    out[col] = s;
  }
}

// ----------------------------- host ------------------------------------------
template <typename T, int V, int E, int WPR>
cudaError_t forward(cudaStream_t st, const NormArgs& a, int* launches) {
  constexpr int GROUPS = block_warps<WPR>() / WPR;
  ++*launches;
  return launch_dependent(norm_kernel<T, V, E, WPR>, (unsigned)((a.tokens + GROUPS - 1) / GROUPS), block_warps<WPR>() * 32, 0, st, a);
}

template <typename T, int V, int E, int WPR>
cudaError_t backward(cudaStream_t st, const NormArgs& a, int n_sms, int* launches) {
  using Sh = BackShape<T, V, E, WPR>;
  constexpr int GROUPS = Sh::GROUPS;
  const int64_t needed = (a.tokens + GROUPS - 1) / GROUPS;
  const int most = n_sms * 2 < NORM_PARTS ? n_sms * 2 : NORM_PARTS;
  const int blocks = (int)(needed < most ? needed : most);
  const size_t smem = Sh::smem(a.d, a.partials != nullptr);
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(norm_back_kernel<T, V, E, WPR>, 100 * 1024, &allowed);
  if (e != cudaSuccess) return e;
  e = launch_dependent(norm_back_kernel<T, V, E, WPR>, (unsigned)blocks, Sh::THREADS, smem, st, a);
  ++*launches;
  if (e != cudaSuccess || !a.partials) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((a.d + 31) / 32), 2);
  cfg.blockDim = dim3(32 * JOIN);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  ++*launches;
  return cudaLaunchKernelEx(&cfg, norm_join_kernel, (const float*)a.partials, blocks, (int)a.d, a.dweight, a.dbias);
}

// Entries per lane and warps per row.  Forward, up to 32 entries: a row's two tensors are all that a thread holds.  Backward, 16 while that
// takes: with 32 the rows under way and the sums over tokens leave room for 8 warps on a multiprocessor.
template <typename T, int V>
cudaError_t choose(cudaStream_t st, const NormArgs& a, bool back, int n_sms, int* launches) {
  if (a.d <= 256) return back ? backward<T, V, 8, 1>(st, a, n_sms, launches) : forward<T, V, 8, 1>(st, a, launches);
  if (back) {
    if (a.d <= 512) return backward<T, V, 16, 1>(st, a, n_sms, launches);
    if (a.d <= 1024) return backward<T, V, 16, 2>(st, a, n_sms, launches);
    if (a.d <= 2048) return backward<T, V, 16, 4>(st, a, n_sms, launches);
    if (a.d <= 4096) return backward<T, V, 16, 8>(st, a, n_sms, launches);
    if (a.d <= 8192) return backward<T, V, 16, 16>(st, a, n_sms, launches);
    if (a.d <= 16384) return backward<T, V, 32, 16>(st, a, n_sms, launches);
    return backward<T, V, 32, 32>(st, a, n_sms, launches);
  }
  if (a.d <= 1024) return forward<T, V, 32, 1>(st, a, launches);
  if (a.d <= 2048) return forward<T, V, 32, 2>(st, a, launches);
  if (a.d <= 4096) return forward<T, V, 32, 4>(st, a, launches);
  if (a.d <= 8192) return forward<T, V, 32, 8>(st, a, launches);
  return forward<T, V, 32, 32>(st, a, launches);
}

}  // namespace

cudaError_t launch_norm(cudaStream_t st, const NormArgs& a, bool back, int is_bf16, int n_sms, int* launches) {
  const int v = is_bf16 ? 8 : 4;               // entries in 16 bytes
  const bool wide = a.d % v == 0 && a.ldx % v == 0 && a.ldr % v == 0 && a.ldy % v == 0 && aligned16(a.x) && aligned16(a.residual) &&
                    aligned16(a.h) && aligned16(a.y) && aligned16(a.weight) && aligned16(a.bias) && aligned16(a.dy) && aligned16(a.dh) &&
                    aligned16(a.dx);
  if (is_bf16) return wide ? choose<__nv_bfloat16, 8>(st, a, back, n_sms, launches) : choose<__nv_bfloat16, 1>(st, a, back, n_sms, launches);
  return wide ? choose<float, 4>(st, a, back, n_sms, launches) : choose<float, 1>(st, a, back, n_sms, launches);
}

}  // namespace muloco
