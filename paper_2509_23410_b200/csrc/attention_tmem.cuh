// What the attention kernels on tcgen05 share: operand descriptors, products with an operand in TMEM, a thread's row of scores between TMEM
// and registers, and the softmax of 64 of them.
#pragma once
#include "attention.cuh"
#include "f32x2.cuh"

namespace patch {
namespace attn {
namespace blk {

// MN-major operand in 128-byte-swizzled atoms of 64 elements x 8 rows (the rows are the product's K): start address, stride between
// the 64-element atoms, stride between groups of eight rows.
__device__ __forceinline__ uint64_t desc_mnmajor_sw128(uint32_t saddr, uint32_t atom_stride) {
    return uint64_t((saddr & 0x3FFFFu) >> 4) | (uint64_t(atom_stride >> 4) << 16) | (uint64_t(1024 >> 4) << 32) |
           (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
// D[tmem] (+)= A[tmem] * B[smem]: lane = row of A, a 32-bit column holds two consecutive K elements
__device__ __forceinline__ void mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
#define PATCH_R32(v) "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), \
    "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), \
    "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
#define PATCH_S32(v) "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), \
    "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), \
    "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
// 32 lanes x 32 consecutive 32-bit columns <-> 32 registers per thread (thread = lane)
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];" : PATCH_R32(v) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31};" ::PATCH_S32(v), "r"(taddr) : "memory");
}
#undef PATCH_R32
#undef PATCH_S32
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// n consecutive columns, n = 16 or 32
__device__ __forceinline__ void load_quarter(uint32_t taddr, uint32_t (&v)[32]) { tmem_ld32(taddr, v); }
__device__ __forceinline__ void load_quarter(uint32_t taddr, uint32_t (&v)[16]) { tmem_ld16(taddr, v); }
// true in one lane of the (converged) warp, always the same one
__device__ __forceinline__ bool elect_one() {
    uint32_t pred;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(pred));
    return pred != 0;
}
// scores past the row's last column: -inf
__device__ __forceinline__ void hide(uint32_t (&v)[32], int left) {
#pragma unroll
    for (int c = 0; c < 32; ++c)
        if (c >= left) v[c] = 0xFF800000u;
}
__device__ __forceinline__ float top_of(const uint32_t (&v)[32], float top) {
    float t[4] = {top, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int c = 0; c < 32; ++c) t[c & 3] = fmaxf(t[c & 3], __uint_as_float(v[c]));
    return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
}
// Maximum of 32 n scores of the row and `top`.
__device__ __forceinline__ float row_top(uint32_t t_s, int n, int left, float top = -INFINITY) {
#pragma unroll 1
    for (int q = 0; q < n; ++q) {
        uint32_t v[32];
        tmem_ld32(t_s + 32u * q, v);
        tmem_ld_wait();
        hide(v, left - 32 * q);
        top = top_of(v, top);
    }
    return top;
}
// 2^exponent(s, base, scale) of 64 scores of the row (softmax_rule.cuh, two at a time) as bf16 and the sum of the unrounded values.
__device__ __forceinline__ float probabilities(uint32_t t_s, int left, bool partly, float scale, float base, uint32_t (&pr)[32]) {
    const f2 scale2 = mk2(scale, scale), base2 = mk2(-base, -base);
    f2 sum[2] = {0ull, 0ull};
    uint32_t v[2][32];
    tmem_ld32(t_s, v[0]);
    tmem_ld32(t_s + 32u, v[1]);
    tmem_ld_wait();
    if (partly) {
        hide(v[0], left);
        hide(v[1], left - 32);
    }
#pragma unroll
    for (int c = 0; c < 64; c += 2) {
        float e0, e1;
        un2(mul2(add2(mk2(__uint_as_float(v[c >> 5][c & 31]), __uint_as_float(v[c >> 5][(c & 31) + 1])), base2), scale2), e0, e1);
        e0 = ex2(e0);
        e1 = ex2(e1);
        sum[(c >> 1) & 1] = add2(sum[(c >> 1) & 1], mk2(e0, e1));
        pr[c >> 1] = pack2(e0, e1);
    }
    float a, b;
    un2(add2(sum[0], sum[1]), a, b);
    return a + b;
}

}  // namespace blk
}  // namespace attn
}  // namespace patch
