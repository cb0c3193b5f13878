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
// elements.  32 / G heads of one token fit a warp at a time; the warp keeps what the token's cosines and sines (and, forward, the
// gains) make of a pair in registers while it walks over the token's heads.
//
// Measured at 16384 tokens, 16 + 16 heads of 128, bf16, in a short burst: forward 45 us (6.2 TB/s, issue slots 62 % taken), backward 76 us
// (5.4 TB/s; 158 registers leave 12 warps per SM); among other work 48 and 85 us.
#include <string.h>

#include <atomic>
#include <type_traits>

#include "internal.h"

namespace muloco {

namespace {

constexpr int QK_THREADS = 128;
constexpr int QK_WARPS = QK_THREADS / 32;

// V float32 values of a lane (V = 1, 2, 4 or 8); products and sums of them two at a time where V allows it.
template <int V> struct Vec { uint64_t p[V / 2]; };
template <> struct Vec<1> { float f; };

__device__ __forceinline__ uint64_t join(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 split2(uint64_t p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
template <int V> __device__ __forceinline__ Vec<V> mul(const Vec<V>& a, const Vec<V>& b) {
  Vec<V> r;
  if constexpr (V == 1) r.f = a.f * b.f;
  else
#pragma unroll
    for (int i = 0; i < V / 2; ++i) r.p[i] = mul2(a.p[i], b.p[i]);
  return r;
}
template <int V> __device__ __forceinline__ Vec<V> mul(const Vec<V>& a, float b) {
  Vec<V> r;
  if constexpr (V == 1) r.f = a.f * b;
  else {
    const uint64_t bb = join(b, b);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) r.p[i] = mul2(a.p[i], bb);
  }
  return r;
}
template <int V> __device__ __forceinline__ Vec<V> fma(const Vec<V>& a, const Vec<V>& b, const Vec<V>& c) {
  Vec<V> r;
  if constexpr (V == 1) r.f = fmaf(a.f, b.f, c.f);
  else
#pragma unroll
    for (int i = 0; i < V / 2; ++i) r.p[i] = fma2(a.p[i], b.p[i], c.p[i]);
  return r;
}
template <int V> __device__ __forceinline__ Vec<V> fma(const Vec<V>& a, float b, const Vec<V>& c) {
  Vec<V> r;
  if constexpr (V == 1) r.f = fmaf(a.f, b, c.f);
  else {
    const uint64_t bb = join(b, b);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) r.p[i] = fma2(a.p[i], bb, c.p[i]);
  }
  return r;
}
template <int V> __device__ __forceinline__ Vec<V> of(const float (&f)[V]) {
  Vec<V> r;
  if constexpr (V == 1) r.f = f[0];
  else
#pragma unroll
    for (int i = 0; i < V / 2; ++i) r.p[i] = join(f[2 * i], f[2 * i + 1]);
  return r;
}
template <int V> __device__ __forceinline__ void to(const Vec<V>& a, float (&f)[V]) {
  if constexpr (V == 1) f[0] = a.f;
  else
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const float2 x = split2(a.p[i]);
      f[2 * i] = x.x;
      f[2 * i + 1] = x.y;
    }
}
template <int V> __device__ __forceinline__ Vec<V> filled(float x) {
  float f[V];
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = x;
  return of<V>(f);
}
template <int V> __device__ __forceinline__ Vec<V> from_shared(const float* p) {
  float f[V];
  if constexpr (V == 1) f[0] = *p;
  else if constexpr (V == 2) {
    const float2 x = *reinterpret_cast<const float2*>(p);
    f[0] = x.x; f[1] = x.y;
  } else
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 x = *reinterpret_cast<const float4*>(p + i);
      f[i] = x.x; f[i + 1] = x.y; f[i + 2] = x.z; f[i + 3] = x.w;
    }
  return of<V>(f);
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
template <int V> __device__ __forceinline__ float sum(const Vec<V>& a) {
  if constexpr (V == 1) return a.f;
  else {
    uint64_t s = a.p[0];
#pragma unroll
    for (int i = 1; i < V / 2; ++i) s = add2(s, a.p[i]);
    const float2 x = split2(s);
    return x.x + x.y;
  }
}
template <int V> __device__ __forceinline__ Vec<V> negated(const Vec<V>& a) {
  float f[V];
  to<V>(a, f);
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = -f[i];
  return of<V>(f);
}
// Even and odd entries of the sequence (a, b): what neighbouring pairs are, and back.
template <int V> __device__ __forceinline__ void pairs_apart(Vec<V>& a, Vec<V>& b) {
  if constexpr (V > 1) {
    float f[V], g[V], x[V], y[V];
    to<V>(a, f); to<V>(b, g);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[i] = 2 * i < V ? f[2 * i] : g[2 * i - V];
      y[i] = 2 * i < V ? f[2 * i + 1] : g[2 * i + 1 - V];
    }
    a = of<V>(x); b = of<V>(y);
  }
}
template <int V> __device__ __forceinline__ void pairs_together(Vec<V>& a, Vec<V>& b) {
  if constexpr (V > 1) {
    float f[V], g[V], x[V], y[V];
    to<V>(a, f); to<V>(b, g);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      x[2 * i] = f[i]; x[2 * i + 1] = g[i];
      y[2 * i] = f[V / 2 + i]; y[2 * i + 1] = g[V / 2 + i];
    }
    a = of<V>(x); b = of<V>(y);
  }
}

// V values as they lie in memory: one access.
template <typename T, int V> struct Raw;
template <> struct Raw<float, 4> { float4 v; };
template <> struct Raw<float, 2> { float2 v; };
template <> struct Raw<float, 1> { float v; };
template <> struct Raw<__nv_bfloat16, 8> { uint4 v; };
template <> struct Raw<__nv_bfloat16, 4> { uint2 v; };
template <> struct Raw<__nv_bfloat16, 2> { uint32_t v; };
template <> struct Raw<__nv_bfloat16, 1> { __nv_bfloat16 v; };
template <typename T, int V> __device__ __forceinline__ Raw<T, V> raw_zero() {
  Raw<T, V> r;
  memset(&r, 0, sizeof r);
  return r;
}
__device__ __forceinline__ uint64_t from_bf16x2(uint32_t w) {
  return join(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ Vec<4> unpack(const Raw<float, 4>& r) { return Vec<4>{{join(r.v.x, r.v.y), join(r.v.z, r.v.w)}}; }
__device__ __forceinline__ Vec<2> unpack(const Raw<float, 2>& r) { return Vec<2>{{join(r.v.x, r.v.y)}}; }
__device__ __forceinline__ Vec<2> unpack(const Raw<__nv_bfloat16, 2>& r) { return Vec<2>{{from_bf16x2(r.v)}}; }
__device__ __forceinline__ Vec<1> unpack(const Raw<float, 1>& r) { return Vec<1>{r.v}; }
__device__ __forceinline__ Vec<8> unpack(const Raw<__nv_bfloat16, 8>& r) {
  return Vec<8>{{from_bf16x2(r.v.x), from_bf16x2(r.v.y), from_bf16x2(r.v.z), from_bf16x2(r.v.w)}};
}
__device__ __forceinline__ Vec<4> unpack(const Raw<__nv_bfloat16, 4>& r) { return Vec<4>{{from_bf16x2(r.v.x), from_bf16x2(r.v.y)}}; }
__device__ __forceinline__ Vec<1> unpack(const Raw<__nv_bfloat16, 1>& r) { return Vec<1>{__bfloat162float(r.v)}; }
__device__ __forceinline__ uint32_t to_bf16x2(uint64_t p) {
  const float2 x = split2(p);
  __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ void store(float* p, const Vec<4>& a) {
  const float2 x = split2(a.p[0]), y = split2(a.p[1]);
  *reinterpret_cast<float4*>(p) = make_float4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ void store(float* p, const Vec<2>& a) { *reinterpret_cast<float2*>(p) = split2(a.p[0]); }
__device__ __forceinline__ void store(float* p, const Vec<1>& a) { *p = a.f; }
__device__ __forceinline__ void store(__nv_bfloat16* p, const Vec<8>& a) {
  *reinterpret_cast<uint4*>(p) = make_uint4(to_bf16x2(a.p[0]), to_bf16x2(a.p[1]), to_bf16x2(a.p[2]), to_bf16x2(a.p[3]));
}
__device__ __forceinline__ void store(__nv_bfloat16* p, const Vec<4>& a) {
  *reinterpret_cast<uint2*>(p) = make_uint2(to_bf16x2(a.p[0]), to_bf16x2(a.p[1]));
}
__device__ __forceinline__ void store(__nv_bfloat16* p, const Vec<2>& a) { *reinterpret_cast<uint32_t*>(p) = to_bf16x2(a.p[0]); }
__device__ __forceinline__ void store(__nv_bfloat16* p, const Vec<1>& a) { *p = __float2bfloat16_rn(a.f); }

// Elements of the two vectors of the chunk that starts at pair p.
struct ChunkAt { int a, b; bool rot; };
__device__ __forceinline__ ChunkAt chunk_at(int p, int half, bool interleaved, int V) {
  ChunkAt c;
  c.rot = p < half;
  if (c.rot && !interleaved) { c.a = p; c.b = p + half; }
  else { c.a = 2 * p; c.b = 2 * p + V; }
  return c;
}

// Asynchronous copies from global to shared memory (4, 8 or 16 bytes), in groups.
template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Steps of a warp that are staged in shared memory: the bytes in flight do not take registers.  Two groups of heads a step, three
// steps (backward two): 16384 tokens, 32 heads of 128, bf16: 47 us forward and 78 backward; with one group and 6 / 5 steps 51 and
// 81, two groups and 5 / 4 steps 49 and 90 (fewer blocks fit an SM).
template <typename T, int V, int NC, bool BACK> struct Stage {
  static constexpr int TABLE = V == 2 ? 2 : 4;                       // table entries per copy
  static constexpr int U = 2;                                     // groups of heads in a step
  static constexpr int DEPTH = BACK ? 2 : 3;
  static constexpr int VEC = V * (int)sizeof(T);
  static constexpr int GROUP = NC * (BACK ? 4 : 2) * 32 * VEC;       // bytes of a group of heads
  static constexpr int DATA = U * GROUP;
  static __host__ __device__ constexpr int bytes(int dim) { return DATA + dim * 4; }     // ... and of its token's cosines and sines
};

// Blocks [0, ctas0) serve the first tensor, the others the second.  A warp takes items in steps of the tensor's warps;
// an item is one token and, of its heads, every `split`-th group of 32 / G (split > 1 when there are too few
// tokens to fill the machine).  A step is U groups of heads.  V > 1: the warp's next steps are on their way into shared memory
// (and, with a token's first step, its cosines and sines) while it works on the current one.
template <typename T, int V, int NC, bool IL, bool BACK>
__global__ void __launch_bounds__(QK_THREADS, V == 1 ? 1 : BACK ? 3 : 4)
qk_norm_kernel(const __grid_constant__ QkArgs p, int ctas0, int G, int split0, int split1) {
  const int which = blockIdx.x < (unsigned)ctas0 ? 0 : 1;
  const QkTensor& t = p.t[which];
  const int cta = which ? blockIdx.x - ctas0 : blockIdx.x;
  const int ctas = which ? gridDim.x - ctas0 : ctas0;
  const int split = which ? split1 : split0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = lane / G, gl = lane & (G - 1);
  const int rows = 32 / G;
  const int half = p.rot >> 1, pairs = p.dim >> 1;
  const int heads = t.heads;
  const float inv_dim = 1.0f / (float)p.dim;

  grid_wait();
  grid_release();
  // the gains, in the order of the pairs' first and second entries per chunk (neighbouring pairs: apart)
  __shared__ __align__(16) float gains[2][QK_MAX_DIM / 2];
  for (int i = threadIdx.x; i < pairs; i += QK_THREADS) {
    const int p0 = i / V * V;
    const ChunkAt c = chunk_at(p0, half, IL, V);
    const int e0 = IL ? 2 * i : c.a + (i - p0), e1 = IL ? 2 * i + 1 : c.b + (i - p0);
    gains[0][i] = t.gain ? t.gain[e0] : 1.f;
    gains[1][i] = t.gain ? t.gain[e1] : 1.f;
  }
  __syncthreads();

  bool on[NC];
  ChunkAt at[NC];
  Vec<V> da[NC], db[NC];                     // backward: sums of the gains' gradients
  const float* g0[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int pr = (gl + c * G) * V;
    on[c] = pr < pairs;
    at[c] = chunk_at(on[c] ? pr : 0, half, IL, V);
    g0[c] = &gains[0][on[c] ? pr : 0];
    da[c] = db[c] = filled<V>(0.f);
  }

  const int64_t items = p.tokens * split;
  const int64_t stride = (int64_t)ctas * QK_WARPS;
  const int64_t it0 = (int64_t)cta * QK_WARPS + warp;
  auto token_of = [&](int64_t it) { return split == 1 ? it : it / split; };
  auto first_of = [&](int64_t it) { return split == 1 ? 0 : (int)(it % split) * rows; };
  const T* const xs = reinterpret_cast<const T*>(t.x);
  const T* const ys = reinterpret_cast<const T*>(t.dy);
  T* const os = reinterpret_cast<T*>(t.out);

  // What a token's cosines and sines become for this lane's pairs (first, second entry), with g the gains:
  //   forward   first' = r (k0 first + k1 second),  second' = r (k2 first + k3 second);  k = g0 c, -g1 s, g0 s, g1 c
  //   backward  dn = R^T dy:  k0 = c, k1 = s, k2 = -s, k3 = c
  Vec<V> k0[NC], k1[NC], k2[NC], k3[BACK ? 1 : NC];
  auto coefficients = [&](int c, const Vec<V>& cs, const Vec<V>& sn) {
    if (BACK) {
      k0[c] = cs; k1[c] = sn; k2[c] = negated<V>(sn);
    } else {
      const Vec<V> ga = from_shared<V>(g0[c]), gb = from_shared<V>(g0[c] + QK_MAX_DIM / 2);
      k0[c] = mul<V>(ga, cs); k1[c] = negated<V>(mul<V>(gb, sn));
      k2[c] = mul<V>(ga, sn); k3[BACK ? 0 : c] = mul<V>(gb, cs);
    }
  };
#pragma unroll
  for (int c = 0; c < NC; ++c) coefficients(c, filled<V>(1.f), filled<V>(0.f));

  // One group: norm and rotation (or their gradient) of the heads whose elements xa, xb (ya, yb) the lanes hold.
  auto work = [&](Vec<V> (&xa)[NC], Vec<V> (&xb)[NC], Vec<V> (&ya)[NC], Vec<V> (&yb)[NC], T* out, bool there, bool pos_ok) {
    Vec<V> sq, ex;
    Vec<V> ea[NC], eb[NC];                   // gain dn
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (IL) pairs_apart<V>(xa[c], xb[c]);
      sq = c ? fma<V>(xa[c], xa[c], sq) : mul<V>(xa[c], xa[c]);
      sq = fma<V>(xb[c], xb[c], sq);
      if (BACK) {
        if (IL) pairs_apart<V>(ya[c], yb[c]);
        const Vec<V> a = ya[c], b = yb[c];
        ya[c] = fma<V>(b, k1[c], mul<V>(a, k0[c]));
        yb[c] = fma<V>(a, k2[c], mul<V>(b, k0[c]));
        ea[c] = mul<V>(from_shared<V>(g0[c]), ya[c]);
        eb[c] = mul<V>(from_shared<V>(g0[c] + QK_MAX_DIM / 2), yb[c]);
        ex = c ? fma<V>(ea[c], xa[c], ex) : mul<V>(ea[c], xa[c]);
        ex = fma<V>(eb[c], xb[c], ex);
      }
    }
    float ss = sum<V>(sq), es = BACK ? sum<V>(ex) : 0.f;
    for (int o = G >> 1; o > 0; o >>= 1) {
      ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (BACK) es += __shfl_xor_sync(0xffffffffu, es, o);
    }
    float r = rsqrtf(fmaf(ss, inv_dim, p.eps));
    if (!pos_ok) r = __int_as_float(0x7fffffff);
    const float k = BACK ? -(r * r * es * inv_dim) : 0.f;         // -mean(e x r) r
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (!(there && on[c])) continue;
      const Vec<V> ra = mul<V>(xa[c], r), rb = mul<V>(xb[c], r);
      Vec<V> oa, ob;
      if (!BACK) {
        oa = fma<V>(rb, k1[c], mul<V>(ra, k0[c]));
        ob = fma<V>(rb, k3[BACK ? 0 : c], mul<V>(ra, k2[c]));
      } else {
        da[c] = fma<V>(ya[c], ra, da[c]);
        db[c] = fma<V>(yb[c], rb, db[c]);
        oa = fma<V>(ra, k, mul<V>(ea[c], r));
        ob = fma<V>(rb, k, mul<V>(eb[c], r));
      }
      if (IL) pairs_together<V>(oa, ob);
      store(out + at[c].a, oa);
      store(out + at[c].b, ob);
    }
  };

  if constexpr (V > 1) {
    using St = Stage<T, V, NC, BACK>;
    constexpr int U = St::U;
    extern __shared__ __align__(16) uint8_t staged[];
    const int per = St::bytes(p.dim);
    uint8_t* const mine = staged + (size_t)warp * St::DEPTH * per;
    const uint32_t mine_s = (uint32_t)__cvta_generic_to_shared(mine);
    const int group_step = split * rows, head_step = U * group_step;
    auto position = [&](int64_t it) -> int64_t {
      if (it >= items) return 0;
      const int64_t tok = token_of(it);
      return p.positions ? p.positions[tok] : tok;
    };
    // the step that is fetched next: item, head of this lane, its row of x (and dy), and the position of its
    // token (read an item ahead)
    int64_t f_it = it0;
    int f_h = 0, f_first = 0;
    const T* f_x = xs;
    const T* f_y = ys;
    auto start_item = [&]() {
      if (f_it >= items) return;
      const int64_t tok = token_of(f_it);
      f_first = first_of(f_it) + sub;
      f_h = f_first;
      f_x = xs + tok * t.x_ts + (int64_t)f_h * t.x_hs;
      if (BACK) f_y = ys + tok * t.y_ts + (int64_t)f_h * t.y_hs;
    };
    start_item();
    int64_t f_pos = position(f_it), f_pos_next = position(f_it + stride);
    int f_slot = 0;
    auto fetch = [&]() {
      if (f_it < items) {
        const uint32_t dst = mine_s + f_slot * per;
        if (f_h == f_first && half > 0 && f_pos >= 0 && f_pos < p.table_len)
          for (int i = lane; i < 2 * half / St::TABLE; i += 32) {       // half cosines, then half sines
            const bool s = i >= half / St::TABLE;
            const int e = (s ? i - half / St::TABLE : i) * St::TABLE;
            copy_async<4 * St::TABLE>(dst + St::DATA + ((s ? half : 0) + e) * 4, (s ? p.sin : p.cos) + f_pos * half + e);
          }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (f_h < heads)
#pragma unroll
            for (int c = 0; c < NC; ++c)
              if (on[c]) {
                const uint32_t d = dst + u * St::GROUP + ((c * (BACK ? 4 : 2)) * 32 + lane) * St::VEC;
                copy_async<St::VEC>(d, f_x + at[c].a);
                copy_async<St::VEC>(d + 32 * St::VEC, f_x + at[c].b);
                if (BACK) {
                  copy_async<St::VEC>(d + 64 * St::VEC, f_y + at[c].a);
                  copy_async<St::VEC>(d + 96 * St::VEC, f_y + at[c].b);
                }
              }
          f_h += group_step;
          f_x += group_step * t.x_hs;
          if (BACK) f_y += group_step * t.y_hs;
        }
        if (f_h - sub >= heads) {
          f_it += stride;
          start_item();
          f_pos = f_pos_next;
          f_pos_next = position(f_it + stride);
        }
      }
      copy_commit();
      f_slot = f_slot + 1 == St::DEPTH ? 0 : f_slot + 1;
    };
    for (int i = 0; i < St::DEPTH - 1; ++i) fetch();
    int slot = 0;
    int64_t pos = position(it0), pos_next = position(it0 + stride);
    for (int64_t it = it0; it < items; it += stride) {
      const bool pos_ok = half == 0 || (pos >= 0 && pos < p.table_len);
      if (!pos_ok && lane == 0) atomicOr(p.status, ST_POSITION);
      const int first = first_of(it);
      T* out = os + token_of(it) * t.o_ts + (int64_t)(first + sub) * t.o_hs;
      for (int h0 = first; h0 < heads; h0 += head_step) {
        copy_wait<St::DEPTH - 2>();
        __syncwarp();                          // every lane's copies of this step have landed; the slot before it is free
        fetch();
        const uint8_t* src = mine + slot * per;
        if (h0 == first && pos_ok)
#pragma unroll
          for (int c = 0; c < NC; ++c)
            if (on[c] && at[c].rot) {
              const float* tab = reinterpret_cast<const float*>(src + St::DATA) + (gl + c * G) * V;
              coefficients(c, from_shared<V>(tab), from_shared<V>(tab + half));
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (u > 0 && h0 + u * group_step >= heads) break;      // the whole warp
          const bool there = h0 + u * group_step + sub < heads;
          Vec<V> xa[NC], xb[NC], ya[NC], yb[NC];
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            Raw<T, V> a = raw_zero<T, V>(), b = a, d = a, e = a;
            if (there && on[c]) {
              const uint8_t* q = src + u * St::GROUP + ((c * (BACK ? 4 : 2)) * 32 + lane) * St::VEC;
              a = *reinterpret_cast<const Raw<T, V>*>(q);
              b = *reinterpret_cast<const Raw<T, V>*>(q + 32 * St::VEC);
              if (BACK) {
                d = *reinterpret_cast<const Raw<T, V>*>(q + 64 * St::VEC);
                e = *reinterpret_cast<const Raw<T, V>*>(q + 96 * St::VEC);
              }
            }
            xa[c] = unpack(a);
            xb[c] = unpack(b);
            if (BACK) { ya[c] = unpack(d); yb[c] = unpack(e); }
          }
          work(xa, xb, ya, yb, out, there, pos_ok);
          out += group_step * t.o_hs;
        }
        slot = slot + 1 == St::DEPTH ? 0 : slot + 1;
      }
      pos = pos_next;
      pos_next = position(it + 2 * stride);
    }
  } else {
    // elements one by one: odd head sizes, strides and addresses
    for (int64_t it = it0; it < items; it += stride) {
      const int64_t tok = token_of(it);
      const int64_t pos = p.positions ? p.positions[tok] : tok;
      const bool pos_ok = half == 0 || (pos >= 0 && pos < p.table_len);
      if (!pos_ok && lane == 0) atomicOr(p.status, ST_POSITION);
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (on[c] && at[c].rot && pos_ok)
          coefficients(c, Vec<V>{__ldg(p.cos + pos * half + gl + c * G)}, Vec<V>{__ldg(p.sin + pos * half + gl + c * G)});
      for (int h0 = first_of(it); h0 < heads; h0 += split * rows) {
        const int h = h0 + sub;
        const T* x = xs + tok * t.x_ts + (int64_t)h * t.x_hs;
        const T* y = ys + (BACK ? tok * t.y_ts + (int64_t)h * t.y_hs : 0);
        Vec<V> xa[NC], xb[NC], ya[NC], yb[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const bool there = h < heads && on[c];
          xa[c].f = there ? (float)x[at[c].a] : 0.f;
          xb[c].f = there ? (float)x[at[c].b] : 0.f;
          if (BACK) {
            ya[c].f = there ? (float)y[at[c].a] : 0.f;
            yb[c].f = there ? (float)y[at[c].b] : 0.f;
          }
        }
        work(xa, xb, ya, yb, os + tok * t.o_ts + (int64_t)h * t.o_hs, h < heads, pos_ok);
      }
    }
  }

  if (BACK && t.dgain) {
    // Sums in a fixed order: the heads side by side in the warp, the warps of the block, then the blocks.
    __shared__ float acc[QK_MAX_DIM];
    __shared__ int last;
    float fa[NC][V], fb[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (IL) pairs_together<V>(da[c], db[c]);
      to<V>(da[c], fa[c]);
      to<V>(db[c], fb[c]);
    }
    for (int o = G; o < 32; o <<= 1)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          fa[c][i] += __shfl_xor_sync(0xffffffffu, fa[c][i], o);
          fb[c][i] += __shfl_xor_sync(0xffffffffu, fb[c][i], o);
        }
    for (int w = 0; w < QK_WARPS; ++w) {
      if (warp == w && sub == 0)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          if (on[c])
#pragma unroll
            for (int i = 0; i < V; ++i) {
              acc[at[c].a + i] = (w ? acc[at[c].a + i] : 0.f) + fa[c][i];
              acc[at[c].b + i] = (w ? acc[at[c].b + i] : 0.f) + fb[c][i];
            }
      __syncthreads();
    }
    // Blocks are joined sixteen at a time, by whichever of the sixteen comes last, and the sixteens by whichever of them comes last:
    // one round of loads each, where a single block that added up all of them took 8 us.
    const int n_groups = (ctas + QK_JOIN - 1) / QK_JOIN, group = cta / QK_JOIN;
    const int in_group = group + 1 < n_groups ? QK_JOIN : ctas - group * QK_JOIN;
    float* const rows1 = p.partials + (size_t)(which ? ctas0 : 0) * p.dim;                        // one row per block
    float* const rows2 = p.partials + (size_t)(QK_MAX_CTAS + (which ? QK_MAX_CTAS / QK_JOIN : 0)) * p.dim;   // ... per group
    int* const tickets = p.tickets + which * (QK_MAX_CTAS / QK_JOIN + 1);
    // Writes acc to `row` and returns whether this block is the last of `of` to do so.
    auto hand_in = [&](float* row, int* ticket, int of) {
      for (int i = threadIdx.x; i < p.dim; i += QK_THREADS) row[i] = acc[i];
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        last = atomicAdd(ticket, 1) == of - 1;
        if (last) *ticket = 0;                             // for the next launch
      }
      __syncthreads();
      if (last) __threadfence();
      return last != 0;
    };
    // acc <- the sum of n rows, in the order of the rows for every thread group and then of the groups
    auto add_up = [&](const float* all, int n, auto width) {
      constexpr int W = decltype(width)::value;
      const int cols = p.dim / W;
      const int groups = cols < QK_THREADS ? QK_THREADS / cols : 1;
      for (int c0 = 0; c0 < cols; c0 += QK_THREADS) {
        const int col = c0 + threadIdx.x % (cols < QK_THREADS ? cols : QK_THREADS);
        const int g = groups > 1 ? threadIdx.x / cols : 0;
        float s[W];
#pragma unroll
        for (int i = 0; i < W; ++i) s[i] = 0.f;
        if (col < cols && g < groups) {
          for (int b0 = g; b0 < n; b0 += 8 * groups) {     // eight loads under way
            float f[8][W];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int b = b0 + j * groups;
              const float* q = all + (size_t)b * p.dim + col * W;
              if constexpr (W == 4) {
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                if (b < n) x = __ldcg(reinterpret_cast<const float4*>(q));
                f[j][0] = x.x; f[j][1] = x.y; f[j][2] = x.z; f[j][3] = x.w;
              } else {
                f[j][0] = b < n ? __ldcg(q) : 0.f;
              }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int i = 0; i < W; ++i) s[i] += f[j][i];
          }
        }
        for (int k = 0; k < groups; ++k) {
          __syncthreads();
          if (col < cols && g == k)
#pragma unroll
            for (int i = 0; i < W; ++i) acc[col * W + i] = (k ? acc[col * W + i] : 0.f) + s[i];
        }
      }
      __syncthreads();
    };
    auto join = [&](const float* all, int n) {
      if (p.dim % 4 == 0) add_up(all, n, std::integral_constant<int, 4>());
      else add_up(all, n, std::integral_constant<int, 1>());
    };
    if (ctas > 1) {
      if (!hand_in(rows1 + (size_t)cta * p.dim, tickets + group, in_group)) return;
      join(rows1 + (size_t)group * QK_JOIN * p.dim, in_group);
      if (n_groups > 1) {
        if (!hand_in(rows2 + (size_t)group * p.dim, tickets + QK_MAX_CTAS / QK_JOIN, n_groups)) return;
        join(rows2, n_groups);
      }
    }
    for (int i = threadIdx.x; i < p.dim; i += QK_THREADS) t.dgain[i] = acc[i];
  }
}

template <typename T, int V, int NC, bool IL, bool BACK>
cudaError_t launch_one(cudaStream_t st, const QkArgs& a, int n_sms, int G) {
  auto kernel = qk_norm_kernel<T, V, NC, IL, BACK>;
  size_t smem = 0;
  int resident = BACK ? 8 : 16;              // blocks per SM: V == 1 has nothing staged and wants many
  if constexpr (V > 1) {
    using St = Stage<T, V, NC, BACK>;
    smem = (size_t)QK_WARPS * St::DEPTH * St::bytes(a.dim);
    // the resident blocks (a second wave of blocks costs a third of the rate), asked for once per device and head size: one byte
    // each, 0 while not known, so that calls from several threads find the answer for their own size or ask themselves
    static std::atomic<uint8_t> known[8][QK_MAX_DIM / 2 + 1];
    int dev = 0, blocks = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev < 8) blocks = known[dev][a.dim / 2].load(std::memory_order_relaxed);
    if (e == cudaSuccess && blocks == 0) {
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               (int)(QK_WARPS * St::DEPTH * St::bytes(QK_MAX_DIM)));
      if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kernel, QK_THREADS, smem);
      if (e == cudaSuccess && blocks < 1) e = cudaErrorLaunchOutOfResources;
      if (e == cudaSuccess && dev < 8) known[dev][a.dim / 2].store((uint8_t)blocks, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) return e;
    resident = blocks;
  }
  // The blocks are shared out by what a token costs in either tensor: its groups of heads, and about one more for what is done
  // once per token (12 + 3 heads of 64, f32, 4099 tokens, backward: 27 us when shared out by heads).  A token's
  // heads go to several warps when there are fewer tokens than warps.
  const int rows = 32 / G;
  const int64_t most = (int64_t)n_sms * resident < QK_MAX_CTAS - 1 ? (int64_t)n_sms * resident : QK_MAX_CTAS - 1;
  int groups[2], ctas[2] = {0, 0}, split[2] = {1, 1};
  int64_t cost[2];
  for (int w = 0; w < 2; ++w) {
    groups[w] = (a.t[w].heads + rows - 1) / rows;
    cost[w] = groups[w] ? groups[w] + 1 : 0;
  }
  for (int w = 0; w < 2; ++w) {
    if (!groups[w]) continue;
    int64_t share = w ? most - most * cost[0] / (cost[0] + cost[1]) : most * cost[0] / (cost[0] + cost[1]);
    if (share < 1) share = 1;
    while (split[w] < groups[w] && a.tokens * split[w] < share * QK_WARPS) split[w] *= 2;
    if (split[w] > groups[w]) split[w] = groups[w];
    const int64_t need = (a.tokens * split[w] + QK_WARPS - 1) / QK_WARPS;
    ctas[w] = (int)(need < share ? need : share);
  }
  return launch_dependent(kernel, (unsigned)(ctas[0] + ctas[1]), QK_THREADS, smem, st, a, ctas[0], G, split[0], split[1]);
}

template <typename T, int V, int NC>
cudaError_t launch_v(cudaStream_t st, const QkArgs& a, bool back, int n_sms, int G) {
  if (a.interleaved)
    return back ? launch_one<T, V, NC, true, true>(st, a, n_sms, G) : launch_one<T, V, NC, true, false>(st, a, n_sms, G);
  return back ? launch_one<T, V, NC, false, true>(st, a, n_sms, G) : launch_one<T, V, NC, false, false>(st, a, n_sms, G);
}

// Whether every vector of V elements of `elt` bytes that the kernel touches is aligned.
bool aligned(const QkArgs& a, bool back, int V, int elt) {
  if (a.dim % (2 * V) != 0 || a.rot % (2 * V) != 0) return false;
  const int table = V == 2 ? 2 : 4;                                  // entries of a table row per copy
  if (a.rot % (2 * table) != 0 || (((uintptr_t)a.cos | (uintptr_t)a.sin) & (4 * table - 1)) != 0) return false;
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

cudaError_t launch_qk_norm(cudaStream_t st, const QkArgs& a, bool back, int is_bf16, int n_sms) {
  const int64_t heads = (int64_t)a.t[0].heads + a.t[1].heads;
  if (a.tokens <= 0 || heads <= 0) return cudaSuccess;
  int V = 1;
  if (is_bf16) V = aligned(a, back, 8, 2) ? 8 : aligned(a, back, 4, 2) ? 4 : aligned(a, back, 2, 2) ? 2 : 1;
  else V = aligned(a, back, 4, 4) ? 4 : aligned(a, back, 2, 4) ? 2 : 1;
  const int chunks = (a.dim / 2 + V - 1) / V;
  int G = 1;
  while (G < 32 && G < chunks) G <<= 1;
  const int NC = (chunks + G - 1) / G;
#define QK_CASE(T, VV, N) return launch_v<T, VV, N>(st, a, back, n_sms, G)
  if (is_bf16) {
    if (V == 8) QK_CASE(__nv_bfloat16, 8, 1);
    else if (V == 4) { if (NC == 1) QK_CASE(__nv_bfloat16, 4, 1); else QK_CASE(__nv_bfloat16, 4, 2); }
    else if (V == 2) { if (NC == 1) QK_CASE(__nv_bfloat16, 2, 1); else if (NC == 2) QK_CASE(__nv_bfloat16, 2, 2); else QK_CASE(__nv_bfloat16, 2, 4); }
    else if (NC <= 2) QK_CASE(__nv_bfloat16, 1, 2);
    else QK_CASE(__nv_bfloat16, 1, 8);
  } else {
    if (V == 4) { if (NC == 1) QK_CASE(float, 4, 1); else QK_CASE(float, 4, 2); }
    else if (V == 2) { if (NC == 1) QK_CASE(float, 2, 1); else if (NC == 2) QK_CASE(float, 2, 2); else QK_CASE(float, 2, 4); }
    else if (NC <= 2) QK_CASE(float, 1, 2);
    else QK_CASE(float, 1, 8);
  }
#undef QK_CASE
}

}  // namespace muloco
