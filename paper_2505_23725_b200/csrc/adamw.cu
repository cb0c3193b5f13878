// AdamW over many tensors in one launch, with moments in 32 or in 8 bits (Section 4.3).
//
// A warp owns a block of 256 elements: lane i holds elements 4 i .. 4 i + 3 of each half of the block, so
// that every access of the warp is one run of full lines.  With 8-bit states the block is also
// what shares a scale: the warp decodes its 256 codes, updates in float32, takes the block's largest
// magnitudes with one warp-wide integer maximum each (the bits of non-negative floats order like
// integers) and encodes again, all in registers: one read and one write of everything.
#include "internal.h"

namespace muloco {

namespace {

constexpr int AW_THREADS = 256;
constexpr int AW_WARPS = AW_THREADS / 32;
constexpr float AW_TINY = 1e-36f;       // blocks at or below this magnitude are encoded as zeros
constexpr float AW_MAGIC = 12582912.0f; // 1.5 * 2^23: adding it leaves the integer part in the low bits

// Mueller's 32-bit integer hash.
__host__ __device__ __forceinline__ uint32_t hash32(uint32_t x) {
  x = ((x >> 16) ^ x) * 0x45d9f3bu;
  x = ((x >> 16) ^ x) * 0x45d9f3bu;
  return (x >> 16) ^ x;
}

struct Four { float x[4]; };

// Four consecutive elements of which the first `cnt` exist.
__device__ __forceinline__ Four load_f32(const float* p, bool vec, int cnt) {
  Four r;
  if (vec && cnt == 4) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    r.x[0] = v.x; r.x[1] = v.y; r.x[2] = v.z; r.x[3] = v.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.x[e] = e < cnt ? p[e] : 0.f;
  }
  return r;
}
__device__ __forceinline__ void store_f32(float* p, const Four& v, bool vec, int cnt) {
  if (vec && cnt == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v.x[0], v.x[1], v.x[2], v.x[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) p[e] = v.x[e];
  }
}
template <bool GBF16>
__device__ __forceinline__ Four load_grad(const void* g, int64_t i, bool vec, int cnt) {
  if (!GBF16) {
    const float* p = reinterpret_cast<const float*>(g) + i;
    if (vec && cnt == 4) {
      const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
      return Four{{v.x, v.y, v.z, v.w}};
    }
    return load_f32(p, false, cnt);
  }
  const __nv_bfloat16* p = reinterpret_cast<const __nv_bfloat16*>(g) + i;
  Four r;
  if (vec && cnt == 4) {
    const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p));
    r.x[0] = __uint_as_float(v.x << 16); r.x[1] = __uint_as_float(v.x & 0xFFFF0000u);
    r.x[2] = __uint_as_float(v.y << 16); r.x[3] = __uint_as_float(v.y & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.x[e] = e < cnt ? __bfloat162float(p[e]) : 0.f;
  }
  return r;
}
__device__ __forceinline__ void store_copy(void* c, int64_t i, const Four& v, bool vec, int cnt) {
  __nv_bfloat16* p = reinterpret_cast<__nv_bfloat16*>(c) + i;
  if (vec && cnt == 4) {
    __nv_bfloat162 lo = __floats2bfloat162_rn(v.x[0], v.x[1]), hi = __floats2bfloat162_rn(v.x[2], v.x[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) p[e] = __float2bfloat16_rn(v.x[e]);
  }
}

// One block of 256 elements of tensor `s`, by one warp.  Returns whether a gradient was not finite.
template <int BITS, bool GBF16>
__device__ __forceinline__ bool adamw_block(const AdamwSeg& s, const void* g, int64_t blk, const AdamwStep& a) {
  const int lane = threadIdx.x & 31;
  const bool vec_g = (((uintptr_t)g) & (GBF16 ? 7 : 15)) == 0;
  const bool vec_t = (((uintptr_t)s.theta) & 15) == 0;
  const bool vec_c = (((uintptr_t)s.copy) & 7) == 0;
  const int64_t i0 = blk * MULOCO_ADAMW_BLOCK + lane * 4;
  const float om1 = 1.0f - a.beta1, om2 = 1.0f - a.beta2;
  const float lr = a.lr * s.lr_mult, lr_wd = a.lr_wd * (s.lr_mult * s.wd_mult);

  Four gr[2], th[2];
  uint32_t c1[2], c2[2];
  Four m[2], v[2];
  int cnt[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t i = i0 + h * 128;
    const int64_t left = s.n - i;
    cnt[h] = left >= 4 ? 4 : (left > 0 ? (int)left : 0);
    gr[h] = load_grad<GBF16>(g, i, vec_g, cnt[h]);
    th[h] = load_f32(s.theta + i, vec_t, cnt[h]);
    if (BITS == 8) {
      // the padding of the last block belongs to the state and is read and written with it
      c1[h] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(s.s1) + i);
      c2[h] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(s.s2) + i);
    } else {
      m[h] = load_f32(reinterpret_cast<const float*>(s.s1) + i, true, cnt[h]);
      v[h] = load_f32(reinterpret_cast<const float*>(s.s2) + i, true, cnt[h]);
    }
  }
  float sc1 = 0.f, sc2 = 0.f;
  if (BITS == 8) { sc1 = s.scale1[blk]; sc2 = s.scale2[blk]; }

  bool bad = false;
  float max1 = 0.f, max2 = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float ge = gr[h].x[e];
      bad |= !(fabsf(ge) <= 3.402823466e38f);
      float root;
      if (BITS == 8) {
        const bool there = e < cnt[h];
        const float k1 = (float)(int)(int8_t)(c1[h] >> (8 * e)), k2 = (float)((c2[h] >> (8 * e)) & 0xffu);
        const float mo = __fmul_rn(there ? k1 : 0.f, sc1);
        const float ro = __fmul_rn(there ? k2 : 0.f, sc2);
        const float mn = __fadd_rn(__fmul_rn(mo, a.beta1), __fmul_rn(ge, om1));
        const float vn = __fadd_rn(__fmul_rn(__fmul_rn(ro, ro), a.beta2), __fmul_rn(__fmul_rn(ge, ge), om2));
        root = __fsqrt_rn(vn);
        m[h].x[e] = mn;
        v[h].x[e] = root;                       // the root is what is encoded
        // integer maxima: bits of non-negative floats order like integers, a NaN above all
        max1 = __uint_as_float(max(__float_as_uint(max1), __float_as_uint(fabsf(mn))));
        max2 = __uint_as_float(max(__float_as_uint(max2), __float_as_uint(root)));
      } else {
        m[h].x[e] = fmaf(a.beta1, m[h].x[e], om1 * ge);
        v[h].x[e] = fmaf(a.beta2, v[h].x[e], om2 * ge * ge);
        root = sqrtf(v[h].x[e]);
      }
      const float den = fmaf(root, a.inv_sqrt_bc2, a.eps);
      // two ulp of the quotient, an update of about lr: far below theta's own rounding
      const float upd = __fdividef(m[h].x[e] * a.inv_bc1, den);
      // (that quotient flushes to zero for denominators above 2^126, where the true one is below 2^-100)
      th[h].x[e] = th[h].x[e] - fmaf(lr, upd, lr_wd * th[h].x[e]);
    }

  float inv1 = 0.f, inv2 = 0.f;
  if (BITS == 8) {
    max1 = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(max1)));
    max2 = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(max2)));
    inv1 = max1 > AW_TINY ? __fdiv_rn(127.f, max1) : 0.f;
    inv2 = max2 > AW_TINY ? __fdiv_rn(255.f, max2) : 0.f;
    if (lane == 0) {
      s.scale1[blk] = __fmul_rn(max1, 1.0f / 127.0f);
      s.scale2[blk] = __fmul_rn(max2, 1.0f / 255.0f);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t i = i0 + h * 128;
    if (BITS == 8) {
      uint32_t o1 = 0, o2 = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t r = hash32((uint32_t)(s.dither_base + i + e) + a.dither);
        const float u1 = (float)(r & 0xffffu) * 1.52587890625e-5f, u2 = (float)(r >> 16) * 1.52587890625e-5f;
        float t1 = __fadd_rn(__fmul_rn(m[h].x[e], inv1), u1);
        float t2 = __fadd_rn(__fmul_rn(v[h].x[e], inv2), u2);
        t1 = fminf(fmaxf(t1, -127.f), 127.f);
        t2 = fminf(fmaxf(t2, v[h].x[e] > 0.f ? 1.f : 0.f), 255.f);
        o1 |= (__float_as_uint(__fadd_rd(t1, AW_MAGIC)) & 0xffu) << (8 * e);
        o2 |= (__float_as_uint(__fadd_rd(t2, AW_MAGIC)) & 0xffu) << (8 * e);
      }
      *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(s.s1) + i) = o1;
      *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(s.s2) + i) = o2;
    } else {
      store_f32(reinterpret_cast<float*>(s.s1) + i, m[h], true, cnt[h]);
      store_f32(reinterpret_cast<float*>(s.s2) + i, v[h], true, cnt[h]);
    }
    store_f32(s.theta + i, th[h], vec_t, cnt[h]);
    if (s.copy) store_copy(s.copy, i, th[h], vec_c, cnt[h]);
  }
  return bad;
}

template <int BITS, bool GBF16>
__global__ void __launch_bounds__(AW_THREADS)
adamw_multi_kernel(const AdamwSeg* __restrict__ segs, const int* __restrict__ unit_seg,
                   const void* const* __restrict__ grads, int n_segs, AdamwStep a, int* __restrict__ status) {
  const int64_t unit = blockIdx.x;
  const int si = unit_seg[unit];
  if (!MULOCO_IN_BOUNDS(si >= 0 && si < n_segs, status)) return;
  const AdamwSeg s = segs[si];
  const int64_t blk = (unit - s.unit_begin) * AW_WARPS + (threadIdx.x >> 5);
  if (blk * MULOCO_ADAMW_BLOCK >= s.n) return;
  const bool bad = adamw_block<BITS, GBF16>(s, grads[si], blk, a);
  if (__any_sync(0xffffffffu, bad) && (threadIdx.x & 31) == 0) atomicOr(status, ST_NONFINITE);
}

__global__ void __launch_bounds__(AW_THREADS)
adamw_moments_kernel(const AdamwSeg* __restrict__ segs, const int* __restrict__ unit_seg, int n_segs,
                     float* __restrict__ m, float* __restrict__ v, int* __restrict__ status) {
  const int64_t unit = blockIdx.x;
  const int si = unit_seg[unit];
  if (!MULOCO_IN_BOUNDS(si >= 0 && si < n_segs, status)) return;
  const AdamwSeg s = segs[si];
  const int64_t blk = (unit - s.unit_begin) * AW_WARPS + (threadIdx.x >> 5);
  if (blk * MULOCO_ADAMW_BLOCK >= s.n) return;
  const float sc1 = s.scale1[blk], sc2 = s.scale2[blk];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t i = blk * MULOCO_ADAMW_BLOCK + h * 128 + (threadIdx.x & 31) * 4;
    const uint32_t c1 = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(s.s1) + i);
    const uint32_t c2 = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(s.s2) + i);
    float4 om, ov;
    float* pm = &om.x;
    float* pv = &ov.x;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      pm[e] = __fmul_rn((float)(int)(int8_t)(c1 >> (8 * e)), sc1);
      const float r = __fmul_rn((float)((c2 >> (8 * e)) & 0xffu), sc2);
      pv[e] = __fmul_rn(r, r);
    }
    __stcs(reinterpret_cast<float4*>(m + s.dither_base + i), om);
    __stcs(reinterpret_cast<float4*>(v + s.dither_base + i), ov);
  }
}

}  // namespace

int64_t adamw_units(int64_t n) {
  const int64_t per = (int64_t)AW_WARPS * MULOCO_ADAMW_BLOCK;
  return (n + per - 1) / per;
}

uint32_t adamw_dither(uint32_t seed, int64_t step) { return hash32(hash32(seed) + (uint32_t)step); }

void launch_adamw_multi(cudaStream_t st, const AdamwSeg* segs, const int* unit_seg, const void* const* grads,
                        int n_segs, int64_t n_units, int state_bits, int g_is_bf16, const AdamwStep& a, int* status) {
  if (n_units <= 0) return;
  const unsigned grid = (unsigned)n_units;   // one unit per block, in address order
  if (state_bits == 8) {
    if (g_is_bf16) adamw_multi_kernel<8, true><<<grid, AW_THREADS, 0, st>>>(segs, unit_seg, grads, n_segs, a, status);
    else adamw_multi_kernel<8, false><<<grid, AW_THREADS, 0, st>>>(segs, unit_seg, grads, n_segs, a, status);
  } else {
    if (g_is_bf16) adamw_multi_kernel<32, true><<<grid, AW_THREADS, 0, st>>>(segs, unit_seg, grads, n_segs, a, status);
    else adamw_multi_kernel<32, false><<<grid, AW_THREADS, 0, st>>>(segs, unit_seg, grads, n_segs, a, status);
  }
}

void launch_adamw_moments(cudaStream_t st, const AdamwSeg* segs, const int* unit_seg, int n_segs, int64_t n_units,
                          float* m, float* v, int* status) {
  if (n_units <= 0) return;
  adamw_moments_kernel<<<(unsigned)n_units, AW_THREADS, 0, st>>>(segs, unit_seg, n_segs, m, v, status);
}

}  // namespace muloco
