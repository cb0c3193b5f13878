// Norm of queries and keys per head with the position rotation in the same pass, and its backward pass.
//
// Forward, for a head x of `dim` entries:  r = 1 / sqrt(mean x^2 + eps),  n = gain x r,  out = R n, with R the
// rotation of the pairs.  Backward, from dy:  dn = R^T dy,  dgain = sum over tokens and heads of dn x r,
// e = gain dn,  dx = r (e - x r mean(e x r)).  Both are bound by memory: x is read once and the result written once
// (backward: x and dy read, dx written), so everything of a head stays in registers.
//
// A head is held by G neighbouring lanes (a power of two), each with NC chunks of V pairs.  Pair p of the head is
//   p < rot / 2, halves        : (p, p + rot / 2)
//   otherwise                  : (2 p, 2 p + 1)      (interleaved pairs, and the entries that are not rotated)
// so both members of a pair are in one lane and the rotation needs no exchange; a chunk is two vectors of V
// elements.  32 / G heads of one token fit a warp at a time; the warp keeps the token's cosines and sines in
// registers while it walks over the token's heads, and the gains while it walks over tokens.
#include "internal.h"

namespace muloco {

namespace {

constexpr int QK_THREADS = 256;
constexpr int QK_WARPS = QK_THREADS / 32;

template <typename T, int V>
__device__ __forceinline__ void load_vec(const T* p, float (&f)[V]);
template <> __device__ __forceinline__ void load_vec<float, 4>(const float* p, float (&f)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
}
template <> __device__ __forceinline__ void load_vec<float, 1>(const float* p, float (&f)[1]) { f[0] = *p; }
template <> __device__ __forceinline__ void load_vec<__nv_bfloat16, 8>(const __nv_bfloat16* p, float (&f)[8]) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
template <> __device__ __forceinline__ void load_vec<__nv_bfloat16, 4>(const __nv_bfloat16* p, float (&f)[4]) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
  f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
}
template <> __device__ __forceinline__ void load_vec<__nv_bfloat16, 1>(const __nv_bfloat16* p, float (&f)[1]) {
  f[0] = __bfloat162float(*p);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&h);
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[V]);
template <> __device__ __forceinline__ void store_vec<float, 4>(float* p, const float (&f)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
template <> __device__ __forceinline__ void store_vec<float, 1>(float* p, const float (&f)[1]) { *p = f[0]; }
template <> __device__ __forceinline__ void store_vec<__nv_bfloat16, 8>(__nv_bfloat16* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}
template <> __device__ __forceinline__ void store_vec<__nv_bfloat16, 4>(__nv_bfloat16* p, const float (&f)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3]));
}
template <> __device__ __forceinline__ void store_vec<__nv_bfloat16, 1>(__nv_bfloat16* p, const float (&f)[1]) {
  *p = __float2bfloat16_rn(f[0]);
}

// Elements of the two vectors of the chunk that starts at pair p.
struct ChunkAt { int a, b; bool rot; };
__device__ __forceinline__ ChunkAt chunk_at(int p, int half, bool interleaved, int V) {
  ChunkAt c;
  c.rot = p < half;
  if (c.rot && !interleaved) { c.a = p; c.b = p + half; }
  else { c.a = 2 * p; c.b = 2 * p + V; }
  return c;
}

// Turns the V pairs of a chunk by (cos, sign * sin).
template <int V, bool IL>
__device__ __forceinline__ void turn(float (&a)[V], float (&b)[V], const float (&c)[V], const float (&s)[V], float sign) {
  if (!IL) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float y = a[i] * c[i] - sign * b[i] * s[i], z = b[i] * c[i] + sign * a[i] * s[i];
      a[i] = y; b[i] = z;
    }
  } else if (V == 1) {
    const float y = a[0] * c[0] - sign * b[0] * s[0], z = b[0] * c[0] + sign * a[0] * s[0];
    a[0] = y; b[0] = z;
  } else {
    // the 2 V elements lie in order: pair i is elements 2 i and 2 i + 1 of (a, b)
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const float y = a[2 * i] * c[i] - sign * a[2 * i + 1] * s[i], z = a[2 * i + 1] * c[i] + sign * a[2 * i] * s[i];
      a[2 * i] = y; a[2 * i + 1] = z;
    }
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const float y = b[2 * i] * c[V / 2 + i] - sign * b[2 * i + 1] * s[V / 2 + i];
      const float z = b[2 * i + 1] * c[V / 2 + i] + sign * b[2 * i] * s[V / 2 + i];
      b[2 * i] = y; b[2 * i + 1] = z;
    }
  }
}

// Blocks [0, ctas0) serve the first tensor, the others the second.  A warp takes items in steps of the tensor's warps;
// an item is one token and, of its heads, every `split`-th group of 32 / G (split > 1 when there are too few
// tokens to fill the machine).
template <typename T, int V, int NC, bool IL, bool BACK>
__global__ void __launch_bounds__(QK_THREADS)
qk_norm_kernel(const QkArgs p, int ctas0, int G, int split0, int split1) {
  const int which = blockIdx.x < (unsigned)ctas0 ? 0 : 1;
  const QkTensor& t = p.t[which];
  const int cta = which ? blockIdx.x - ctas0 : blockIdx.x;
  const int ctas = which ? gridDim.x - ctas0 : ctas0;
  const int split = which ? split1 : split0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = lane / G, gl = lane & (G - 1);
  const int rows = 32 / G;
  const int half = p.rot >> 1, pairs = p.dim >> 1;
  const float inv_dim = 1.0f / (float)p.dim;

  bool on[NC];
  ChunkAt at[NC];
  float ga[NC][V], gb[NC][V];                // gains of this lane's elements
  float da[NC][V], db[NC][V];                // backward: sums of their gradients
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int pr = (gl + c * G) * V;
    on[c] = pr < pairs;
    at[c] = chunk_at(on[c] ? pr : 0, half, IL, V);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      ga[c][i] = t.gain && on[c] ? t.gain[at[c].a + i] : 1.f;
      gb[c][i] = t.gain && on[c] ? t.gain[at[c].b + i] : 1.f;
      da[c][i] = db[c][i] = 0.f;
    }
  }

  const int64_t items = p.tokens * split;
  const int64_t step = (int64_t)ctas * QK_WARPS;
  for (int64_t it = (int64_t)cta * QK_WARPS + warp; it < items; it += step) {
    const int64_t tok = it / split;
    const int first = (int)(it - tok * split);
    const int64_t pos = p.positions ? p.positions[tok] : tok;
    const bool pos_ok = half == 0 || (pos >= 0 && pos < p.table_len);
    float cs[NC][V], sn[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int i = 0; i < V; ++i) { cs[c][i] = 1.f; sn[c][i] = 0.f; }
      if (on[c] && at[c].rot) {
        if (pos_ok) {
          const int64_t o = pos * half + (gl + c * G) * V;
#pragma unroll
          for (int i = 0; i < V; ++i) { cs[c][i] = __ldg(p.cos + o + i); sn[c][i] = __ldg(p.sin + o + i); }
        }
      }
    }
    if (!pos_ok && lane == 0) atomicOr(p.status, ST_POSITION);
    for (int h0 = first * rows; h0 < t.heads; h0 += split * rows) {
      const int h = h0 + sub;
      const bool row_ok = h < t.heads;
      const T* x = reinterpret_cast<const T*>(t.x) + tok * t.x_ts + (int64_t)(row_ok ? h : 0) * t.x_hs;
      float xa[NC][V], xb[NC][V], ya[NC][V], yb[NC][V];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int i = 0; i < V; ++i) xa[c][i] = xb[c][i] = ya[c][i] = yb[c][i] = 0.f;
        if (row_ok && on[c]) {
          load_vec<T, V>(x + at[c].a, xa[c]);
          load_vec<T, V>(x + at[c].b, xb[c]);
          if (BACK) {
            const T* y = reinterpret_cast<const T*>(t.dy) + tok * t.y_ts + (int64_t)h * t.y_hs;
            load_vec<T, V>(y + at[c].a, ya[c]);
            load_vec<T, V>(y + at[c].b, yb[c]);
          }
        }
      }
      float ss = 0.f, es = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (BACK && at[c].rot) turn<V, IL>(ya[c], yb[c], cs[c], sn[c], -1.f);      // dn = R^T dy
#pragma unroll
        for (int i = 0; i < V; ++i) {
          ss = fmaf(xa[c][i], xa[c][i], ss);
          ss = fmaf(xb[c][i], xb[c][i], ss);
          if (BACK) {
            es = fmaf(ga[c][i] * ya[c][i], xa[c][i], es);
            es = fmaf(gb[c][i] * yb[c][i], xb[c][i], es);
          }
        }
      }
      for (int o = G >> 1; o > 0; o >>= 1) {
        ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (BACK) es += __shfl_xor_sync(0xffffffffu, es, o);
      }
      float r = rsqrtf(fmaf(ss, inv_dim, p.eps));
      if (!pos_ok) r = __int_as_float(0x7fffffff);
      const float k = BACK ? r * r * es * inv_dim : 0.f;      // mean(e x r) r
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (!(row_ok && on[c])) continue;
        T* out = reinterpret_cast<T*>(t.out) + tok * t.o_ts + (int64_t)h * t.o_hs;
        if (!BACK) {
#pragma unroll
          for (int i = 0; i < V; ++i) { xa[c][i] = xa[c][i] * r * ga[c][i]; xb[c][i] = xb[c][i] * r * gb[c][i]; }
          if (at[c].rot) turn<V, IL>(xa[c], xb[c], cs[c], sn[c], 1.f);
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            da[c][i] = fmaf(ya[c][i], xa[c][i] * r, da[c][i]);
            db[c][i] = fmaf(yb[c][i], xb[c][i] * r, db[c][i]);
            xa[c][i] = r * (ga[c][i] * ya[c][i] - xa[c][i] * k);
            xb[c][i] = r * (gb[c][i] * yb[c][i] - xb[c][i] * k);
          }
        }
        store_vec<T, V>(out + at[c].a, xa[c]);
        store_vec<T, V>(out + at[c].b, xb[c]);
      }
    }
  }

  if (BACK && t.dgain) {
    // Sums in a fixed order: the heads side by side in the warp, the warps of the block, then the blocks.
    __shared__ float acc[QK_MAX_DIM];
    __shared__ int last;
    for (int o = G; o < 32; o <<= 1)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          da[c][i] += __shfl_xor_sync(0xffffffffu, da[c][i], o);
          db[c][i] += __shfl_xor_sync(0xffffffffu, db[c][i], o);
        }
    for (int w = 0; w < QK_WARPS; ++w) {
      if (warp == w && sub == 0)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          if (on[c])
#pragma unroll
            for (int i = 0; i < V; ++i) {
              acc[at[c].a + i] = (w ? acc[at[c].a + i] : 0.f) + da[c][i];
              acc[at[c].b + i] = (w ? acc[at[c].b + i] : 0.f) + db[c][i];
            }
      __syncthreads();
    }
    float* mine = p.partials + (size_t)blockIdx.x * p.dim;
    for (int i = threadIdx.x; i < p.dim; i += QK_THREADS) mine[i] = acc[i];
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(p.tickets + which, 1) == ctas - 1;
    __syncthreads();
    if (last) {
      __threadfence();
      const float* all = p.partials + (size_t)(which ? ctas0 : 0) * p.dim;
      for (int i = threadIdx.x; i < p.dim; i += QK_THREADS) {
        float s = 0.f;
        for (int b = 0; b < ctas; ++b) s += __ldcg(all + (size_t)b * p.dim + i);
        t.dgain[i] = s;
      }
      if (threadIdx.x == 0) p.tickets[which] = 0;      // for the next launch
    }
  }
}

template <typename T, int V, int NC>
void launch_v(cudaStream_t st, const QkArgs& a, bool back, int grid, int ctas0, int G, int s0, int s1) {
  if (a.interleaved) {
    if (back) qk_norm_kernel<T, V, NC, true, true><<<grid, QK_THREADS, 0, st>>>(a, ctas0, G, s0, s1);
    else qk_norm_kernel<T, V, NC, true, false><<<grid, QK_THREADS, 0, st>>>(a, ctas0, G, s0, s1);
  } else {
    if (back) qk_norm_kernel<T, V, NC, false, true><<<grid, QK_THREADS, 0, st>>>(a, ctas0, G, s0, s1);
    else qk_norm_kernel<T, V, NC, false, false><<<grid, QK_THREADS, 0, st>>>(a, ctas0, G, s0, s1);
  }
}

// Whether every vector of V elements of `elt` bytes that the kernel touches is aligned.
bool aligned(const QkArgs& a, bool back, int V, int elt) {
  if (a.dim % (2 * V) != 0 || a.rot % (2 * V) != 0) return false;
  for (const QkTensor& t : a.t) {
    if (!t.heads) continue;
    uintptr_t p = (uintptr_t)t.x | (uintptr_t)t.out;
    int64_t s = t.x_ts | t.x_hs | t.o_ts | t.o_hs;
    if (back) { p |= (uintptr_t)t.dy; s |= t.y_ts | t.y_hs; }
    if (p % (V * elt) != 0 || s % V != 0) return false;
  }
  return true;
}

}  // namespace

int launch_qk_norm(cudaStream_t st, const QkArgs& a, bool back, int is_bf16, int n_sms) {
  const int64_t heads = (int64_t)a.t[0].heads + a.t[1].heads;
  if (a.tokens <= 0 || heads <= 0) return 0;
  int V = 1;
  if (is_bf16) V = aligned(a, back, 8, 2) ? 8 : aligned(a, back, 4, 2) ? 4 : 1;
  else V = aligned(a, back, 4, 4) ? 4 : 1;
  const int chunks = (a.dim / 2 + V - 1) / V;
  int G = 1;
  while (G < 32 && G < chunks) G <<= 1;
  const int NC = (chunks + G - 1) / G;
  const int rows = 32 / G;
  // Backward keeps one block's worth of gain sums per resident block: few blocks, many tokens each.
  const int most = n_sms * (back ? 2 : 8) < QK_MAX_CTAS ? n_sms * (back ? 2 : 8) : QK_MAX_CTAS;
  int ctas[2] = {0, 0}, split[2] = {1, 1};
  for (int w = 0; w < 2; ++w) {
    if (!a.t[w].heads) continue;
    const int groups = (a.t[w].heads + rows - 1) / rows;
    const int64_t share = most * (int64_t)a.t[w].heads / heads > 0 ? most * (int64_t)a.t[w].heads / heads : 1;
    const int64_t warps = share * QK_WARPS;
    // a token's heads go to several warps when there are fewer tokens than warps
    while (split[w] < groups && a.tokens * split[w] < warps) split[w] *= 2;
    if (split[w] > groups) split[w] = groups;
    const int64_t need = (a.tokens * split[w] + QK_WARPS - 1) / QK_WARPS;
    ctas[w] = (int)(need < share ? need : share);
  }
  const int grid = ctas[0] + ctas[1];
#define QK_CASE(T, VV, N) launch_v<T, VV, N>(st, a, back, grid, ctas[0], G, split[0], split[1])
  if (is_bf16) {
    if (V == 8) QK_CASE(__nv_bfloat16, 8, 1);
    else if (V == 4) { if (NC == 1) QK_CASE(__nv_bfloat16, 4, 1); else QK_CASE(__nv_bfloat16, 4, 2); }
    else if (NC <= 2) QK_CASE(__nv_bfloat16, 1, 2);
    else QK_CASE(__nv_bfloat16, 1, 8);
  } else {
    if (V == 4) { if (NC == 1) QK_CASE(float, 4, 1); else QK_CASE(float, 4, 2); }
    else if (NC <= 2) QK_CASE(float, 1, 2);
    else QK_CASE(float, 1, 8);
  }
#undef QK_CASE
  return 1;
}

}  // namespace muloco
