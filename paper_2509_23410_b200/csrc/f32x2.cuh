// Pairs of fp32 in a 64-bit register: one instruction for two of them (sm_100).
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace patch {

typedef unsigned long long f2;
__device__ __forceinline__ f2 mk2(float a, float b) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void un2(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f2 swap2(f2 v) { float a, b; un2(v, a, b); return mk2(b, a); }
__device__ __forceinline__ float sum2(f2 v) { float a, b; un2(v, a, b); return a + b; }
// two bf16 -> two fp32 and back
__device__ __forceinline__ f2 widen2(uint32_t u) { return mk2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u)); }
__device__ __forceinline__ uint32_t narrow2(f2 v) {
    float a, b;
    un2(v, a, b);
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace patch
