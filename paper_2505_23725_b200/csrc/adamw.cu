// AdamW over many tensors in one launch, with moments in 32 or in 8 bits (Section 4.3).
//
// A warp owns a block of 256 elements: lane i holds elements 4 i .. 4 i + 3 of each half of the block, so
// that every access of the warp is one run of full lines.  With 8-bit states the block is also
// what shares a scale: the warp decodes its 256 codes, updates in float32, takes the block's largest
// magnitudes with one warp-wide integer maximum each (the bits of non-negative floats order like
// integers) and encodes again, all in registers: one read and one write of everything.
//
// 32-bit states are bound by memory (134M elements, bf16 gradients: 505 us, 6.9 TB/s).  8-bit states move 14 to 16
// bytes an element, and at the memory's rate there are about 77 issue slots for the 14: the 68 that it takes (two conversions, the
// moments, a correctly rounded root, a hash of two dithers, two encodings) are what the paired operations and byte moves below
// save for.  49M elements with bf16 gradients and a bf16 copy: 140 us, 5.6 TB/s; 374M with f32 gradients 971-1013 us, 5.9-6.2 TB/s.
#include "internal.h"

namespace muloco {

namespace {

constexpr int AW_THREADS = 128;
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

// Two float32 operations per instruction, each rounded as its scalar form.
struct Pair { uint64_t v; };
__device__ __forceinline__ Pair pair(float a, float b) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ Pair both(float a) { return pair(a, a); }
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
__device__ __forceinline__ Pair add2_down(Pair a, Pair b) {
  Pair r;
  asm("add.rm.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
// A product that stays one: mul2 followed by add2 was measured to come out fused (other last bits than mul and add), a
// fused operation with a zero addend is not fused again.  (-0 becomes +0.)
__device__ __forceinline__ Pair mul2_alone(Pair a, Pair b) { return fma2(a, b, both(0.f)); }
// Integers of a few bits as floats, exactly: they become the low mantissa bits of 2^23, which is taken off again.
__device__ __forceinline__ float byte_bits(uint32_t w, int e) {      // byte e
  return __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440u | (uint32_t)e));
}
__device__ __forceinline__ float half_bits(uint32_t w, int h) {      // low (h = 0) or high half
  return __uint_as_float(__byte_perm(w, 0x4B000000u, h ? 0x7432u : 0x7410u));
}
constexpr float AW_2P23 = 8388608.0f;
// The larger of two, NaN when one of them is NaN (its bits, 0x7fffffff, are above those of every number).
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Byte 0 of a, b, c, d as the bytes of a word.
__device__ __forceinline__ uint32_t pack_bytes(float a, float b, float c, float d) {
  const uint32_t lo = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040u);
  const uint32_t hi = __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040u);
  return __byte_perm(lo, hi, 0x5410u);
}

// One block of 256 elements by one warp.  FULL: all of them exist and every access is aligned.  Returns whether a
// gradient was not finite, or (8-bit states) the block's new moments are not.
template <int BITS, bool GBF16, bool FULL>
__device__ __forceinline__ bool adamw_block(const AdamwUnit& s, const void* g, int blk, const AdamwStep& a) {
  const int lane = threadIdx.x & 31;
  const bool vec_g = FULL || (((uintptr_t)g) & (GBF16 ? 7 : 15)) == 0;
  const bool vec_t = FULL || (((uintptr_t)s.theta) & 15) == 0;
  const bool vec_c = FULL || (((uintptr_t)s.copy) & 7) == 0;
  const int i0 = blk * MULOCO_ADAMW_BLOCK + lane * 4;
  const float om1 = 1.0f - a.beta1, om2 = 1.0f - a.beta2;
  const float lr = a.lr * a.inv_bc1 * s.lr_mult, lr_wd = a.lr_wd * (s.lr_mult * s.wd_mult);

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

  Pair finite = both(0.f);                      // 32-bit states: 0 * g summed, NaN as soon as one gradient is not finite
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
    for (int e = 0; e < 4; e += 2) {
      const Pair g2 = pair(gr[h].x[e], gr[h].x[e + 1]);
      if (BITS == 32) finite = fma2(g2, both(0.f), finite);
      Pair mn;
      float2 root;
      if (BITS == 8) {
        // products and sums rounded one by one
        const Pair mo = mul2(add2(pair(byte_bits(c1[h], e), byte_bits(c1[h], e + 1)), both(-(AW_2P23 + 128.0f))), both(sc1));
        const Pair ro = mul2(add2(pair(byte_bits(c2[h], e), byte_bits(c2[h], e + 1)), both(-AW_2P23)), both(sc2));
        mn = add2(mul2_alone(mo, both(a.beta1)), mul2_alone(g2, both(om1)));
        const float2 vn = parts(add2(mul2_alone(mul2(ro, ro), both(a.beta2)), mul2_alone(mul2(g2, g2), both(om2))));
        root = make_float2(__fsqrt_rn(vn.x), __fsqrt_rn(vn.y));
        const float2 mp = parts(mn);
        m[h].x[e] = mp.x; m[h].x[e + 1] = mp.y;
        v[h].x[e] = root.x; v[h].x[e + 1] = root.y;       // the root is what is encoded
        max1 = max_nan(max1, max_nan(fabsf(mp.x), fabsf(mp.y)));
        max2 = max_nan(max2, max_nan(root.x, root.y));
      } else {
        mn = fma2(pair(m[h].x[e], m[h].x[e + 1]), both(a.beta1), mul2(g2, both(om1)));
        const float2 vn = parts(fma2(pair(v[h].x[e], v[h].x[e + 1]), both(a.beta2), mul2(mul2(g2, g2), both(om2))));
        root = make_float2(sqrtf(vn.x), sqrtf(vn.y));
        const float2 mp = parts(mn);
        m[h].x[e] = mp.x; m[h].x[e + 1] = mp.y;
        v[h].x[e] = vn.x; v[h].x[e + 1] = vn.y;
      }
      // The fast reciprocal (one ulp): the update is about lr, far below theta's own rounding.  Its flush to zero does
      // not matter: a root of a float32 is zero or at least 2^-75.
      const float2 den = parts(fma2(pair(root.x, root.y), both(a.inv_sqrt_bc2), both(a.eps)));
      const Pair upd = mul2(mn, pair(rcp_fast(den.x), rcp_fast(den.y)));
      const Pair t2 = pair(th[h].x[e], th[h].x[e + 1]);
      const float2 tn = parts(fma2(upd, both(-lr), fma2(t2, both(-lr_wd), t2)));
      th[h].x[e] = tn.x; th[h].x[e + 1] = tn.y;
    }
  }
  bool bad = false;
  if (BITS == 32) {
    const float2 fin = parts(finite);
    bad = __any_sync(0xffffffffu, !(fin.x + fin.y == 0.f));
  }

  float inv1 = 0.f, inv2 = 0.f;
  if (BITS == 8) {
    // bits of non-negative floats order like integers, those of infinity and NaN above the rest: one integer maximum per moment
    max1 = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(max1)));
    max2 = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(max2)));
    // A gradient that is not finite, a scale that was not, a square beyond float32: the block's scales are NaN, and so are its
    // moments, this step's and those of every step to come, each of which reports it again.
    bad = !(max1 < __int_as_float(0x7f800000) && max2 < __int_as_float(0x7f800000));
    if (bad) max1 = max2 = __int_as_float(0x7fffffff);
    // even lanes deal with the first moment's scale, odd lanes with the second's: one division for both
    const bool odd = lane & 1;
    const float mx = odd ? max2 : max1;
    const float inv = mx > AW_TINY ? __fdiv_rn(odd ? 255.f : 127.f, mx) : 0.f;
    if (lane < 2) (odd ? s.scale2 : s.scale1)[blk] = __fmul_rn(mx, odd ? 1.0f / 255.0f : 1.0f / 127.0f);
    inv1 = __shfl_sync(0xffffffffu, inv, 0);
    inv2 = __shfl_sync(0xffffffffu, inv, 1);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = i0 + h * 128;
    if (BITS == 8) {
      float t1[4], t2[4];
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const uint32_t r0 = hash32((uint32_t)s.dither_base + a.dither + (uint32_t)(i + e));
        const uint32_t r1 = hash32((uint32_t)s.dither_base + a.dither + (uint32_t)(i + e + 1));
        const Pair unit = both(1.52587890625e-5f), off = both(-AW_2P23);
        const Pair k1 = add2(pair(half_bits(r0, 0), half_bits(r1, 0)), off), k2 = add2(pair(half_bits(r0, 1), half_bits(r1, 1)), off);
        // x * inv rounded, plus u rounded: u = k 2^-16 is exact, so the second step is one fused operation
        const float2 a1 = parts(fma2(k1, unit, mul2(pair(m[h].x[e], m[h].x[e + 1]), both(inv1))));
        const float2 a2 = parts(fma2(k2, unit, mul2(pair(v[h].x[e], v[h].x[e + 1]), both(inv2))));
        // at least 1 wherever v > 0: a root of a float32 is at least 2^-75, times 2^126 saturates to 1
        const float lo0 = __saturatef(v[h].x[e] * 8.507059173023462e37f), lo1 = __saturatef(v[h].x[e + 1] * 8.507059173023462e37f);
        const Pair magic = both(AW_MAGIC);
        const float2 b1 = parts(add2_down(pair(fminf(fmaxf(a1.x, -127.f), 127.f), fminf(fmaxf(a1.y, -127.f), 127.f)), magic));
        const float2 b2 = parts(add2_down(pair(fminf(fmaxf(a2.x, lo0), 255.f), fminf(fmaxf(a2.y, lo1), 255.f)), magic));
        t1[e] = b1.x; t1[e + 1] = b1.y;
        t2[e] = b2.x; t2[e + 1] = b2.y;
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

// Blocks of four warps: a block's warps start and end together, and small blocks stagger those that wait for memory against
// those that compute.  8-bit states at ten blocks per SM (48 registers): 374M elements 992 us, with 256 threads and four per SM
// 1070; 32-bit states want the registers (505 us for 134M elements, 531 at ten per SM).
template <int BITS, bool GBF16>
__global__ void __launch_bounds__(AW_THREADS, BITS == 8 ? 10 : 8)
adamw_multi_kernel(const AdamwUnit* __restrict__ units, const void* const* __restrict__ grads, AdamwStep a,
                   int* __restrict__ status) {
  const AdamwUnit s = units[blockIdx.x];      // written before the first launch: needs no wait
  grid_wait();
  grid_release();
  const void* g = s.grad;
  if (grads) g = reinterpret_cast<const uint8_t*>(grads[s.tensor]) + s.first * (GBF16 ? 2 : 4);
  const bool aligned =
      ((((uintptr_t)s.theta) & 15) | (((uintptr_t)s.copy) & 7) | (((uintptr_t)g) & (GBF16 ? 7 : 15))) == 0;
  const int blk = threadIdx.x >> 5;
  if (blk * MULOCO_ADAMW_BLOCK >= s.n) return;
  const bool bad = aligned && (blk + 1) * MULOCO_ADAMW_BLOCK <= s.n ? adamw_block<BITS, GBF16, true>(s, g, blk, a)
                                                                    : adamw_block<BITS, GBF16, false>(s, g, blk, a);
  if (bad && (threadIdx.x & 31) == 0) atomicOr(status, ST_NONFINITE);
}

__global__ void __launch_bounds__(AW_THREADS)
adamw_moments_kernel(const AdamwUnit* __restrict__ units, float* __restrict__ m, float* __restrict__ v) {
  const AdamwUnit& s = units[blockIdx.x];
  grid_wait();
  grid_release();
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
      om.x[e] = __fmul_rn(byte_bits(c1[h], e) - (AW_2P23 + 128.0f), sc1);
      const float r = __fmul_rn(byte_bits(c2[h], e) - AW_2P23, sc2);
      ov.x[e] = __fmul_rn(r, r);
    }
    __stcs(reinterpret_cast<float4*>(m + s.dither_base + i), make_float4(om.x[0], om.x[1], om.x[2], om.x[3]));
    __stcs(reinterpret_cast<float4*>(v + s.dither_base + i), make_float4(ov.x[0], ov.x[1], ov.x[2], ov.x[3]));
  }
}

}  // namespace

uint32_t adamw_dither(uint32_t seed, int64_t step) { return hash32(hash32(seed) + (uint32_t)step); }

cudaError_t launch_adamw_multi(cudaStream_t st, const AdamwUnit* units, const void* const* grads, int64_t n_units,
                               int state_bits, int g_is_bf16, const AdamwStep& a, int* status) {
  if (n_units <= 0) return cudaSuccess;
  const auto kernel = state_bits == 8 ? (g_is_bf16 ? adamw_multi_kernel<8, true> : adamw_multi_kernel<8, false>)
                                      : (g_is_bf16 ? adamw_multi_kernel<32, true> : adamw_multi_kernel<32, false>);
  // one unit per block, in address order
  return launch_dependent(kernel, (unsigned)n_units, AW_THREADS, 0, st, units, grads, a, status);
}

cudaError_t launch_adamw_moments(cudaStream_t st, const AdamwUnit* units, int64_t n_units, float* m, float* v) {
  if (n_units <= 0) return cudaSuccess;
  return launch_dependent(adamw_moments_kernel, (unsigned)n_units, AW_THREADS, 0, st, units, m, v);
}

}  // namespace muloco
