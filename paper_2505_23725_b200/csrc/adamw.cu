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
static_assert(ADAMW_UNIT == AW_THREADS / 32 * MULOCO_ADAMW_BLOCK, "one block of elements per warp");
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

// Byte e of w as a float, exactly: the byte becomes the low mantissa bits of 2^23.
__device__ __forceinline__ float byte_f32(uint32_t w, int e) {
  return __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440u | (uint32_t)e)) - 8388608.0f;
}
// The low (h = 0) or high half of w as a float, exactly.
__device__ __forceinline__ float half_f32(uint32_t w, int h) {
  return __uint_as_float(__byte_perm(w, 0x4B000000u, h ? 0x7432u : 0x7410u)) - 8388608.0f;
}
// Byte 0 of a, b, c, d as the bytes of a word.
__device__ __forceinline__ uint32_t pack_bytes(float a, float b, float c, float d) {
  const uint32_t lo = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040u);
  const uint32_t hi = __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040u);
  return __byte_perm(lo, hi, 0x5410u);
}

// One block of 256 elements by one warp.  FULL: all of them exist and every access is aligned.  Returns whether a
// gradient was not finite.
template <int BITS, bool GBF16, bool FULL>
__device__ __forceinline__ bool adamw_block(const AdamwUnit& s, const void* g, int blk, const AdamwStep& a) {
  const int lane = threadIdx.x & 31;
  const bool vec_g = FULL || (((uintptr_t)g) & (GBF16 ? 7 : 15)) == 0;
  const bool vec_t = FULL || (((uintptr_t)s.theta) & 15) == 0;
  const bool vec_c = FULL || (((uintptr_t)s.copy) & 7) == 0;
  const int i0 = blk * MULOCO_ADAMW_BLOCK + lane * 4;
  const float om1 = 1.0f - a.beta1, om2 = 1.0f - a.beta2;
  const float lr = a.lr * s.lr_mult, lr_wd = a.lr_wd * (s.lr_mult * s.wd_mult);

  Four gr[2], th[2];
  uint32_t c1[2], c2[2];
  Four m[2], v[2];
  int cnt[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = i0 + h * 128;
    const int left = s.n - i;
    cnt[h] = FULL || left >= 4 ? 4 : (left > 0 ? left : 0);
    gr[h] = load_grad<GBF16>(g, i, vec_g, cnt[h]);
    th[h] = load_f32(s.theta + i, vec_t, cnt[h]);
    if (BITS == 8) {
      // the padding of the last block belongs to the state: it is read, counts as zero and is written
      c1[h] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(s.s1) + i);
      c2[h] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(s.s2) + i);
    } else {
      m[h] = load_f32(reinterpret_cast<const float*>(s.s1) + i, true, cnt[h]);
      v[h] = load_f32(reinterpret_cast<const float*>(s.s2) + i, true, cnt[h]);
    }
  }
  float sc1 = 0.f, sc2 = 0.f;
  if (BITS == 8) { sc1 = s.scale1[blk]; sc2 = s.scale2[blk]; }

  float finite = 0.f;                           // 0 * g summed: NaN as soon as one gradient is not finite
  float max1 = 0.f, max2 = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (BITS == 8) {
      c1[h] ^= 0x80808080u;                     // two's complement codes plus 128
      if (!FULL) {
        const uint32_t keep = cnt[h] >= 4 ? 0xffffffffu : (1u << (8 * cnt[h])) - 1u;
        c1[h] = (c1[h] & keep) | (0x80808080u & ~keep);
        c2[h] &= keep;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float ge = gr[h].x[e];
      finite = fmaf(ge, 0.f, finite);
      float root;
      if (BITS == 8) {
        const float mo = __fmul_rn(byte_f32(c1[h], e) - 128.0f, sc1);
        const float ro = __fmul_rn(byte_f32(c2[h], e), sc2);
        const float mn = __fadd_rn(__fmul_rn(mo, a.beta1), __fmul_rn(ge, om1));
        const float vn = __fadd_rn(__fmul_rn(__fmul_rn(ro, ro), a.beta2), __fmul_rn(__fmul_rn(ge, ge), om2));
        root = __fsqrt_rn(vn);
        m[h].x[e] = mn;
        v[h].x[e] = root;                       // the root is what is encoded
        max1 = fmaxf(max1, fabsf(mn));
        max2 = fmaxf(max2, root);
      } else {
        m[h].x[e] = fmaf(a.beta1, m[h].x[e], om1 * ge);
        v[h].x[e] = fmaf(a.beta2, v[h].x[e], om2 * ge * ge);
        root = sqrtf(v[h].x[e]);
      }
      // The quotient to two ulp: an update of about lr, far below theta's own rounding.  (It is zero for denominators
      // above 2^126, where the true one is too small to change theta.)
      const float den = fmaf(root, a.inv_sqrt_bc2, a.eps);
      const float upd = __fdividef(m[h].x[e] * a.inv_bc1, den);
      th[h].x[e] = th[h].x[e] - fmaf(lr, upd, lr_wd * th[h].x[e]);
    }
  }
  const bool bad = __any_sync(0xffffffffu, !(finite == 0.f));

  float inv1 = 0.f, inv2 = 0.f;
  if (BITS == 8) {
    // bits of non-negative floats order like integers: one integer maximum per moment
    max1 = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(max1)));
    max2 = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(max2)));
    if (bad) max1 = max2 = __int_as_float(0x7fffffff);      // such a block's moments are NaN from here on
    inv1 = max1 > AW_TINY ? __fdiv_rn(127.f, max1) : 0.f;
    inv2 = max2 > AW_TINY ? __fdiv_rn(255.f, max2) : 0.f;
    if (lane == 0) {
      s.scale1[blk] = __fmul_rn(max1, 1.0f / 127.0f);
      s.scale2[blk] = __fmul_rn(max2, 1.0f / 255.0f);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = i0 + h * 128;
    if (BITS == 8) {
      float t1[4], t2[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t r = hash32((uint32_t)s.dither_base + a.dither + (uint32_t)(i + e));
        // x * inv rounded, plus u rounded: u = k 2^-16 is exact, so the second step is one fused operation
        t1[e] = fmaf(half_f32(r, 0), 1.52587890625e-5f, __fmul_rn(m[h].x[e], inv1));
        t2[e] = fmaf(half_f32(r, 1), 1.52587890625e-5f, __fmul_rn(v[h].x[e], inv2));
        t1[e] = __fadd_rd(fminf(fmaxf(t1[e], -127.f), 127.f), AW_MAGIC);
        // at least 1 wherever v > 0: a root of a float32 is at least 2^-75, times 2^126 saturates to 1
        t2[e] = __fadd_rd(fminf(fmaxf(t2[e], __saturatef(v[h].x[e] * 8.507059173023462e37f)), 255.f), AW_MAGIC);
      }
      *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(s.s1) + i) = pack_bytes(t1[0], t1[1], t1[2], t1[3]);
      *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(s.s2) + i) = pack_bytes(t2[0], t2[1], t2[2], t2[3]);
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
__global__ void __launch_bounds__(AW_THREADS, 4)
adamw_multi_kernel(const AdamwUnit* __restrict__ units, const void* const* __restrict__ grads, AdamwStep a,
                   int* __restrict__ status) {
  const AdamwUnit s = units[blockIdx.x];
  const int blk = threadIdx.x >> 5;
  if (blk * MULOCO_ADAMW_BLOCK >= s.n) return;
  const void* g = s.grad;
  if (grads)
    g = reinterpret_cast<const uint8_t*>(grads[s.tensor]) + s.first * (GBF16 ? 2 : 4);
  const bool full = (blk + 1) * MULOCO_ADAMW_BLOCK <= s.n &&
                    ((((uintptr_t)s.theta) & 15) | (((uintptr_t)s.copy) & 7) | (((uintptr_t)g) & (GBF16 ? 7 : 15))) == 0;
  const bool bad = full ? adamw_block<BITS, GBF16, true>(s, g, blk, a) : adamw_block<BITS, GBF16, false>(s, g, blk, a);
  if (bad && (threadIdx.x & 31) == 0) atomicOr(status, ST_NONFINITE);
}

__global__ void __launch_bounds__(AW_THREADS)
adamw_moments_kernel(const AdamwUnit* __restrict__ units, float* __restrict__ m, float* __restrict__ v) {
  const AdamwUnit& s = units[blockIdx.x];
  const int blk = threadIdx.x >> 5;
  if (blk * MULOCO_ADAMW_BLOCK >= s.n) return;
  const float sc1 = s.scale1[blk], sc2 = s.scale2[blk];
  uint32_t c1[2], c2[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = blk * MULOCO_ADAMW_BLOCK + h * 128 + (threadIdx.x & 31) * 4;
    c1[h] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(s.s1) + i) ^ 0x80808080u;
    c2[h] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(s.s2) + i);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = blk * MULOCO_ADAMW_BLOCK + h * 128 + (threadIdx.x & 31) * 4;
    Four om, ov;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      om.x[e] = __fmul_rn(byte_f32(c1[h], e) - 128.0f, sc1);
      const float r = __fmul_rn(byte_f32(c2[h], e), sc2);
      ov.x[e] = __fmul_rn(r, r);
    }
    __stcs(reinterpret_cast<float4*>(m + s.dither_base + i), make_float4(om.x[0], om.x[1], om.x[2], om.x[3]));
    __stcs(reinterpret_cast<float4*>(v + s.dither_base + i), make_float4(ov.x[0], ov.x[1], ov.x[2], ov.x[3]));
  }
}

}  // namespace

uint32_t adamw_dither(uint32_t seed, int64_t step) { return hash32(hash32(seed) + (uint32_t)step); }

void launch_adamw_multi(cudaStream_t st, const AdamwUnit* units, const void* const* grads, int64_t n_units,
                        int state_bits, int g_is_bf16, const AdamwStep& a, int* status) {
  if (n_units <= 0) return;
  const unsigned grid = (unsigned)n_units;   // one unit per block, in address order
  if (state_bits == 8) {
    if (g_is_bf16) adamw_multi_kernel<8, true><<<grid, AW_THREADS, 0, st>>>(units, grads, a, status);
    else adamw_multi_kernel<8, false><<<grid, AW_THREADS, 0, st>>>(units, grads, a, status);
  } else {
    if (g_is_bf16) adamw_multi_kernel<32, true><<<grid, AW_THREADS, 0, st>>>(units, grads, a, status);
    else adamw_multi_kernel<32, false><<<grid, AW_THREADS, 0, st>>>(units, grads, a, status);
  }
}

void launch_adamw_moments(cudaStream_t st, const AdamwUnit* units, int64_t n_units, float* m, float* v) {
  if (n_units <= 0) return;
  adamw_moments_kernel<<<(unsigned)n_units, AW_THREADS, 0, st>>>(units, m, v);
}

}  // namespace muloco
