// Causal attention within packed sequences and its gradient (public header: patch_sequence_attention, ..._backward).
//
// Mathematics.  For sequence rows i >= j of one head: s_ij = q_i . k_j, p_ij = 2^((s_ij - m_i) scale log2 e) / l_i with a running maximum
// m and sum l.  The gradient recomputes p_ij = 2^(s_ij scale log2 e - lse_i log2 e) and, with delta_i = go_i . o_i,
//     gs_ij = p_ij (go_i . v_j - delta_i) scale,  gq_i = sum_j gs_ij k_j,  gk_j = sum_i gs_ij q_i,  gv_j = sum_i p_ij go_i,
// the sums of gk and gv also over the query heads that share the key head.  Products take bf16 operands and fp32 accumulators; p and gs are
// rounded to bf16 for theirs (the sum l takes p unrounded).
//
// A CTA owns 64 rows of a sequence: queries of one head (result, gq) or keys of one key head (gk, gv; it walks over the group's query
// heads, so that shared heads need no atomics and equal calls give equal bits).
#include <math.h>
#include "attention_sequence.cuh"

namespace patch {
namespace seq {

using attn::ex2;
using attn::pack2;

constexpr int kRows = 64;                    // of a tile of queries or keys
constexpr int kThreads = 128;

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <int D> constexpr int kPitch = D + 8;                     // elements of a row in shared memory
template <int D> constexpr int kTileElements = kRows * kPitch<D>;

// rows [row, row + 64) of a head, zeros from `end` on
template <int D>
__device__ __forceinline__ void load_tile(__nv_bfloat16* to, const __nv_bfloat16* from, int64_t ld, int row, int end) {
    for (int i = threadIdx.x; i < kRows * (D / 8); i += kThreads) {
        const int r = i / (D / 8), c = i - r * (D / 8);
        const uint4 v = row + r < end ? *reinterpret_cast<const uint4*>(from + int64_t(row + r) * ld + 8 * c) : make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(to + r * kPitch<D> + 8 * c) = v;
    }
}
// s[16 rows of this warp x 64] = A B^T of two tiles of shared memory
template <int D>
__device__ __forceinline__ void product(float (&s)[8][4], const __nv_bfloat16* A, const __nv_bfloat16* Bt) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t a[4];
        ldmatrix(a, smem_u32(A + (16 * warp + (lane & 15)) * kPitch<D> + 16 * kk + 8 * (lane >> 4)));
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            uint32_t b[4];
            ldmatrix(b, smem_u32(Bt + (8 * j + (lane & 7) + 8 * (lane >> 4)) * kPitch<D> + 16 * kk + 8 * ((lane >> 3) & 1)));
            mma(s[j], a, b[0], b[1]);
            mma(s[j + 1], a, b[2], b[3]);
        }
    }
}
// acc[16 rows x D] += P[16 x 64] T, P in registers as `product` leaves it, T a tile of 64 rows
template <int D>
__device__ __forceinline__ void accumulate(float (&acc)[D / 8][4], const float (&p)[8][4], const __nv_bfloat16* T) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
        const uint32_t a[4] = {pack2(p[2 * kk][0], p[2 * kk][1]), pack2(p[2 * kk][2], p[2 * kk][3]), pack2(p[2 * kk + 1][0], p[2 * kk + 1][1]),
                               pack2(p[2 * kk + 1][2], p[2 * kk + 1][3])};
#pragma unroll
        for (int j = 0; j < D / 8; j += 2) {
            uint32_t b[4];
            ldmatrix_t(b, smem_u32(T + (16 * kk + (lane & 7) + 8 * ((lane >> 3) & 1)) * kPitch<D> + 8 * j + 8 * (lane >> 4)));
            mma(acc[j], a, b[0], b[1]);
            mma(acc[j + 1], a, b[2], b[3]);
        }
    }
}
// 16 rows of this warp of a result, in bf16
template <int D>
__device__ __forceinline__ void store_rows(__nv_bfloat16* to, int64_t ld, int row, int end, const float (&acc)[D / 8][4], float f0, float f1) {
    const int lane = threadIdx.x & 31, r = row + 16 * (threadIdx.x >> 5) + (lane >> 2);
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
        if (r < end) *reinterpret_cast<uint32_t*>(to + int64_t(r) * ld + 8 * j + 2 * (lane & 3)) = pack2(acc[j][0] * f0, acc[j][1] * f0);
        if (r + 8 < end) *reinterpret_cast<uint32_t*>(to + int64_t(r + 8) * ld + 8 * j + 2 * (lane & 3)) = pack2(acc[j][2] * f1, acc[j][3] * f1);
    }
}

// (lse log2 e, delta) of every row and head, [Hq][M]
template <int D>
__global__ void __launch_bounds__(256) delta_kernel(const Problem p, const float* lse, float2* stats) {
    const int64_t group = (int64_t(blockIdx.x) * 256 + threadIdx.x) / (D / 8);
    const int c = threadIdx.x & (D / 8 - 1);
    if (group >= int64_t(p.M) * p.Hq) return;
    const int64_t row = group / p.Hq;
    const int h = int(group - row * p.Hq);
    const uint4 a = *reinterpret_cast<const uint4*>(p.o + row * p.ldo + h * D + 8 * c), b = *reinterpret_cast<const uint4*>(p.go + row * p.ldgo + h * D + 8 * c);
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sum = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), sum);
        sum = fmaf(__uint_as_float(x[i] & 0xFFFF0000u), __uint_as_float(y[i] & 0xFFFF0000u), sum);
    }
#pragma unroll
    for (int d = D / 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (c == 0) stats[int64_t(h) * p.M + row] = make_float2(lse[group] * 1.44269504f, sum);
}

template <int D>
__global__ void __launch_bounds__(kThreads) query_grad_kernel(const Problem p, const float2* stats, __nv_bfloat16* gq, int64_t ldgq) {
    extern __shared__ __align__(16) __nv_bfloat16 sm[];
    __nv_bfloat16 *sq = sm, *sgo = sq + kTileElements<D>, *sk = sgo + kTileElements<D>, *sv = sk + kTileElements<D>;
    if (blockIdx.x == 0 && blockIdx.y == 0) check_starts(p, threadIdx.x, kThreads);
    const Tile t = tile_of<kRows>(p, gridDim.x - 1 - blockIdx.x);
    if (t.first < 0) return;
    const int h = blockIdx.y, kvh = h / p.G, lane = threadIdx.x & 31, row = t.begin + t.first;
    load_tile<D>(sq, p.q + int64_t(h) * D, p.ldq, row, t.end);
    load_tile<D>(sgo, p.go + int64_t(h) * D, p.ldgo, row, t.end);
    float acc[D / 8][4] = {};
    const int mine = row + 16 * (threadIdx.x >> 5) + (lane >> 2);
    float2 st[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) st[x] = mine + 8 * x < t.end ? stats[int64_t(h) * p.M + mine + 8 * x] : make_float2(0.0f, 0.0f);
    for (int key = t.begin; key <= row; key += kRows) {
        __syncthreads();
        load_tile<D>(sk, p.k + int64_t(kvh) * D, p.ldk, key, t.end);
        load_tile<D>(sv, p.v + int64_t(kvh) * D, p.ldv, key, t.end);
        __syncthreads();
        float s[8][4], gp[8][4];
        product<D>(s, sq, sk);
        product<D>(gp, sgo, sv);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool sees = key + 8 * j + 2 * (lane & 3) + (i & 1) <= mine + 8 * (i >> 1);
                s[j][i] = sees ? ex2(fmaf(s[j][i], p.scale_log2, -st[i >> 1].x)) * (gp[j][i] - st[i >> 1].y) : 0.0f;
            }
        accumulate<D>(acc, s, sk);
    }
    store_rows<D>(gq + int64_t(h) * D, ldgq, row, t.end, acc, p.scale, p.scale);
}

template <int D>
__global__ void __launch_bounds__(kThreads) key_grad_kernel(const Problem p, const float2* stats, __nv_bfloat16* gk, int64_t ldgk, __nv_bfloat16* gv, int64_t ldgv) {
    extern __shared__ __align__(16) __nv_bfloat16 sm[];
    __nv_bfloat16 *sk = sm, *sv = sk + kTileElements<D>, *sq = sv + kTileElements<D>, *sgo = sq + kTileElements<D>;
    __shared__ float2 st[kRows];
    const Tile t = tile_of<kRows>(p, blockIdx.x);                         // a sequence's first keys, which most rows see, first
    if (t.first < 0) return;
    const int kvh = blockIdx.y, lane = threadIdx.x & 31, row = t.begin + t.first;
    load_tile<D>(sk, p.k + int64_t(kvh) * D, p.ldk, row, t.end);
    load_tile<D>(sv, p.v + int64_t(kvh) * D, p.ldv, row, t.end);
    float acc_k[D / 8][4] = {}, acc_v[D / 8][4] = {};
    const int mine = row + 16 * (threadIdx.x >> 5) + (lane >> 2);
    for (int h = kvh * p.G; h < (kvh + 1) * p.G; ++h) {
        for (int from = row; from < t.end; from += kRows) {
            __syncthreads();
            load_tile<D>(sq, p.q + int64_t(h) * D, p.ldq, from, t.end);
            load_tile<D>(sgo, p.go + int64_t(h) * D, p.ldgo, from, t.end);
            if (threadIdx.x < kRows) st[threadIdx.x] = from + int(threadIdx.x) < t.end ? stats[int64_t(h) * p.M + from + threadIdx.x] : make_float2(0.0f, 0.0f);
            __syncthreads();
            float s[8][4], gp[8][4];
            product<D>(s, sk, sq);
            product<D>(gp, sv, sgo);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 8 * j + 2 * (lane & 3) + (i & 1);
                    const bool sees = from + at >= mine + 8 * (i >> 1) && from + at < t.end;
                    const float e = sees ? ex2(fmaf(s[j][i], p.scale_log2, -st[at].x)) : 0.0f;
                    s[j][i] = e;
                    gp[j][i] = sees ? e * (gp[j][i] - st[at].y) : 0.0f;
                }
            accumulate<D>(acc_v, s, sgo);
            accumulate<D>(acc_k, gp, sq);
        }
    }
    store_rows<D>(gk + int64_t(kvh) * D, ldgk, row, t.end, acc_k, p.scale, p.scale);
    store_rows<D>(gv + int64_t(kvh) * D, ldgv, row, t.end, acc_v, 1.0f, 1.0f);
}

template <int D>
static int backward(const Problem& p, const float* lse, float2* stats, __nv_bfloat16* gq, int64_t ldgq, __nv_bfloat16* gk, int64_t ldgk, __nv_bfloat16* gv,
                    int64_t ldgv, cudaStream_t s) {
    static std::atomic<uint64_t> configured_q{0}, configured_k{0};
    const uint32_t smem = 4 * kTileElements<D> * 2;
    int rc = allow_dynamic_smem(query_grad_kernel<D>, smem, configured_q);
    if (!rc) rc = allow_dynamic_smem(key_grad_kernel<D>, smem, configured_k);
    if (rc) return rc;
    const int64_t groups = int64_t(p.M) * p.Hq;
    delta_kernel<D><<<unsigned((groups * (D / 8) + 255) / 256), 256, 0, s>>>(p, lse, stats);
    if (cudaGetLastError() != cudaSuccess) return PATCH_ERR_CUDA;
    const unsigned tiles = unsigned(most_tiles(p.M, p.B, kRows));
    query_grad_kernel<D><<<dim3(tiles, unsigned(p.Hq)), kThreads, smem, s>>>(p, stats, gq, ldgq);
    if (cudaGetLastError() != cudaSuccess) return PATCH_ERR_CUDA;
    key_grad_kernel<D><<<dim3(tiles, unsigned(p.Hkv)), kThreads, smem, s>>>(p, stats, gk, ldgk, gv, ldgv);
    return cudaGetLastError() == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}

// ---- checks of arguments ----
static int check_shape(int64_t M, int Hq, int Hkv, int D, int64_t B) {
    if (M < 0 || M > 0x7FFFFFFF - 256 || B < 0 || B > (1 << 20) || (D != 64 && D != 128) || Hkv < 1 || Hq < Hkv || Hq % Hkv || Hq > 4096) return PATCH_ERR_SHAPE;
    // CTAs of a launch are counted in 31 bits
    return M * Hq * (D / 8) > (int64_t(1) << 38) || most_tiles(M, B, kRows) * Hq > 0x7FFFFFFF ? PATCH_ERR_SHAPE : PATCH_OK;
}
static int check_rows(const void* x, int64_t ld, int64_t H, int64_t D) {
    if (!x) return PATCH_ERR_NULL;
    if (ld < H * D || ld % 8 || ld > (int64_t(1) << 28)) return PATCH_ERR_SHAPE;
    return aligned16(x) ? PATCH_OK : PATCH_ERR_ALIGN;
}
static int check_scale(float scale) { return scale > 0.0f && scale <= 2e38f ? PATCH_OK : PATCH_ERR_SHAPE; }

}  // namespace seq
}  // namespace patch

using namespace patch;
using B16 = __nv_bfloat16;

extern "C" int patch_sequence_attention(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t M, int Hq, int Hkv, int D,
                                        const int32_t* starts, int64_t B, float scale, void* O, int64_t ldo, float* lse, int* status_dev, void* stream) {
    int rc = seq::check_shape(M, Hq, Hkv, D, B);
    if (rc || (rc = seq::check_scale(scale))) return rc;
    if (M == 0 || B == 0) return PATCH_OK;
    if ((rc = seq::check_rows(Q, ldq, Hq, D)) || (rc = seq::check_rows(K, ldk, Hkv, D)) || (rc = seq::check_rows(V, ldv, Hkv, D)) ||
        (rc = seq::check_rows(O, ldo, Hq, D)))
        return rc;
    if (!starts) return PATCH_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(starts) & 3u) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return PATCH_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    const seq::Problem p = {static_cast<const B16*>(Q), static_cast<const B16*>(K), static_cast<const B16*>(V), nullptr, nullptr, ldq, ldk, ldv, 0, 0, starts,
                            int(B), int(M), Hq, Hkv, Hq / Hkv, scale, scale * 1.44269504f, status_dev};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return seq::launch_forward(p, D, static_cast<B16*>(O), ldo, lse, s);
}

extern "C" int patch_sequence_attention_backward_workspace_size(int64_t M, int64_t B, int Hq, int Hkv, int D, size_t* bytes_out) {
    if (!bytes_out) return PATCH_ERR_NULL;
    const int rc = seq::check_shape(M, Hq, Hkv, D, B);
    if (rc) return rc;
    *bytes_out = size_t(M) * Hq * sizeof(float2);
    return PATCH_OK;
}

extern "C" int patch_sequence_attention_backward(const void* gO, int64_t ldgo, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                                 const void* O, int64_t ldo, const float* lse, int64_t M, int Hq, int Hkv, int D, const int32_t* starts, int64_t B,
                                                 float scale, void* gQ, int64_t ldgq, void* gK, int64_t ldgk, void* gV, int64_t ldgv, void* workspace,
                                                 size_t workspace_bytes, int* status_dev, void* stream) {
    size_t need = 0;
    int rc = patch_sequence_attention_backward_workspace_size(M, B, Hq, Hkv, D, &need);
    if (rc || (rc = seq::check_scale(scale))) return rc;
    if (M == 0 || B == 0) return PATCH_OK;
    if ((rc = seq::check_rows(gO, ldgo, Hq, D)) || (rc = seq::check_rows(Q, ldq, Hq, D)) || (rc = seq::check_rows(K, ldk, Hkv, D)) ||
        (rc = seq::check_rows(V, ldv, Hkv, D)) || (rc = seq::check_rows(O, ldo, Hq, D)) || (rc = seq::check_rows(gQ, ldgq, Hq, D)) ||
        (rc = seq::check_rows(gK, ldgk, Hkv, D)) || (rc = seq::check_rows(gV, ldgv, Hkv, D)))
        return rc;
    if (!lse || !starts || !workspace) return PATCH_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(starts) & 3u) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PATCH_ERR_ALIGN;
    if (workspace_bytes < need) return PATCH_ERR_SIZE;
    if ((rc = check_device())) return rc;
    const seq::Problem p = {static_cast<const B16*>(Q), static_cast<const B16*>(K), static_cast<const B16*>(V), static_cast<const B16*>(O), static_cast<const B16*>(gO),
                            ldq, ldk, ldv, ldo, ldgo, starts, int(B), int(M), Hq, Hkv, Hq / Hkv, scale, scale * 1.44269504f, status_dev};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    B16 *gq = static_cast<B16*>(gQ), *gk = static_cast<B16*>(gK), *gv = static_cast<B16*>(gV);
    float2* stats = static_cast<float2*>(workspace);
    return D == 128 ? seq::backward<128>(p, lse, stats, gq, ldgq, gk, ldgk, gv, ldgv, s) : seq::backward<64>(p, lse, stats, gq, ldgq, gk, ldgk, gv, ldgv, s);
}
