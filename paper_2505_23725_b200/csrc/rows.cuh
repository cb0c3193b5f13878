// Rows of bf16 in 32-byte accesses, and float32 arithmetic on two values per instruction: shared by the kernels
// that work on accumulator rows.
#pragma once
#include "tc_ptx.cuh"

namespace muloco {

namespace {

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

}  // namespace

}  // namespace muloco
