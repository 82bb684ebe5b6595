// Norms of queries and keys for each head with the position rotation in the same pass, its gradient, and the form that
// writes keys and values to their slots of a paged cache (public header: patch_qk_norm_rope, ..._backward, patch_kv_append).
//
// Mathematics.  A head x of D elements becomes y = R(p) (r x * w), r = 1 / sqrt(mean(x^2) + eps).  Both the weight and
// the rotation are fixed for a (token, kind of head), so they are folded into two coefficients per element once per token:
//     y_j = r (x_j A_j + x_{j'} B_j),   A_j = w_j c,  B_j = -+ w_{j'} s       (j' = the other element of j's pair),
// and a head then costs one sum of squares and two multiply-adds per element.  The gradient turns gy back (g = R^T gy:
// the same form with the sine's sign changed) and needs two sums over the head, of x^2 and of g w x, taken together:
//     gx = r g w - x r^3 mean(g w x),   gw_j = sum g_j x_j r.
//
// Layout.  A group of LANES lanes owns a head, 16 bytes (8 elements) per lane: 8 lanes for D <= 64, 16 for D <= 128, 32
// for D <= 256, so a warp works on 4, 2 or 1 heads and every load and store is 16 bytes per lane, 128 consecutive bytes or more
// per head.  Pairs (i, i + R/2) sit R/16 lanes apart (one 4-register exchange of the raw bf16 values), pairs (2i, 2i + 1) in one
// lane.  A group keeps its token's coefficients in registers and walks over several heads of the token.
//
// What bounds it: HBM.  Four bytes move per element (six in the gradient), plus 4 R bytes of table per token.
#include "patch_internal.cuh"
#include "sm100_ptx.cuh"

namespace patch {
namespace rope {

constexpr int kThreads = 256;
constexpr int kAhead = 4;                 // heads whose loads are in flight together

struct Heads {                            // one kind of head (queries or keys) of the forward kernels
    const __nv_bfloat16* x;
    int64_t ldx;
    __nv_bfloat16* y;                     // result rows, or null where a cache takes them
    int64_t ldy;
    const __nv_bfloat16* w;               // null: no norm
    int H;                                // heads
    int groups;                           // groups of lanes per token
    int per;                              // heads per group
};
struct Cache {
    __nv_bfloat16 *k, *v;
    const __nv_bfloat16* src_v;
    int64_t ldv, page_stride, n_slots;
    const int64_t* slots;
    int shift, D;                         // log2(page_size)
    __device__ __forceinline__ int64_t at(int64_t slot, int h) const {
        return (slot >> shift) * page_stride + ((int64_t(h) << shift) + (slot & ((int64_t(1) << shift) - 1))) * D;
    }
};
struct Turn {
    const float* cos_sin;
    const int32_t* positions;
    int64_t max_positions;
    int R;
};

__device__ __forceinline__ uint4 ld16(const void* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void st16(void* p, uint4 v) { *reinterpret_cast<uint4*>(p) = v; }
__device__ __forceinline__ void unpack(uint4 v, float (&f)[8]) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// One group of lanes: its lane's place in the head, who holds the other halves of its pairs, and the mask its exchanges use
// (groups of a warp may walk over different numbers of heads).
template <int LANES, bool INTER>
struct Group {
    int c;                  // chunk of the head this lane holds: elements 8c .. 8c + 7
    int partner;            // lane (in the warp) with the other elements of the pairs
    uint32_t mask;
    bool on, turned;        // inside the head; inside the rotated part
    float side;             // sign of the sine: -1 where this lane holds the pairs' first elements
    __device__ __forceinline__ Group(int D, int R) {
        const int lane = threadIdx.x & 31;
        c = lane & (LANES - 1);
        mask = LANES == 32 ? 0xFFFFFFFFu : ((1u << (LANES & 31)) - 1u) << (lane & ~(LANES - 1));
        on = c * 8 < D;
        turned = c * 8 < R;
        const bool first = c * 16 < R;
        side = first ? -1.0f : 1.0f;
        partner = INTER || !turned ? lane : first ? lane + R / 16 : lane - R / 16;
    }
    // the pairs' other elements; zeros where nothing is rotated
    __device__ __forceinline__ uint4 other(uint4 v) const {
        if constexpr (INTER) {
            v.x = __byte_perm(v.x, 0, 0x1032); v.y = __byte_perm(v.y, 0, 0x1032);
            v.z = __byte_perm(v.z, 0, 0x1032); v.w = __byte_perm(v.w, 0, 0x1032);
        } else {
            v.x = __shfl_sync(mask, v.x, partner); v.y = __shfl_sync(mask, v.y, partner);
            v.z = __shfl_sync(mask, v.z, partner); v.w = __shfl_sync(mask, v.w, partner);
        }
        return turned ? v : make_uint4(0u, 0u, 0u, 0u);
    }
    // c and (signed) s of this lane's eight elements at position p: y_j = x_j c_j + x_{j'} s_j
    __device__ __forceinline__ void angles(const Turn& t, int64_t p, float (&co)[8], float (&si)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) { co[i] = 1.0f; si[i] = 0.0f; }
        if (!turned) return;
        const float* row = t.cos_sin + p * t.R;
        if constexpr (INTER) {
            const float4 a = *reinterpret_cast<const float4*>(row + 4 * c), b = *reinterpret_cast<const float4*>(row + t.R / 2 + 4 * c);
            const float ca[4] = {a.x, a.y, a.z, a.w}, sa[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                co[2 * i] = co[2 * i + 1] = ca[i];
                si[2 * i] = -sa[i];
                si[2 * i + 1] = sa[i];
            }
        } else {
            const float* r = row + 8 * c - (side > 0.0f ? t.R / 2 : 0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 a = *reinterpret_cast<const float4*>(r + 4 * h), b = *reinterpret_cast<const float4*>(r + t.R / 2 + 4 * h);
                co[4 * h] = a.x; co[4 * h + 1] = a.y; co[4 * h + 2] = a.z; co[4 * h + 3] = a.w;
                si[4 * h] = side * b.x; si[4 * h + 1] = side * b.y; si[4 * h + 2] = side * b.z; si[4 * h + 3] = side * b.w;
            }
        }
    }
    __device__ __forceinline__ float sum(float v) const {
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor_sync(mask, v, d);
        return v;
    }
};

__device__ __forceinline__ int64_t position(const Turn& t, int64_t m, int* status_dev) {
    if (t.R == 0) return 0;
    const int64_t p = t.positions[m];
    if (p >= 0 && p < t.max_positions) return p;
    if (status_dev) atomicCAS(status_dev, PATCH_OK, PATCH_ERR_SIZE);
    return 0;
}

// Forward.  Groups are numbered token by token, the token's query groups first.
template <int LANES, bool INTER, bool APPEND>
__global__ void __launch_bounds__(kThreads)
rope_kernel(const Heads q, const Heads k, const Cache cache, const Turn turn, int64_t M, int D, float eps, int* status_dev) {
    const int per_token = q.groups + k.groups;
    const int64_t idx = (int64_t(blockIdx.x) * kThreads + threadIdx.x) / LANES;
    const int64_t m = idx / per_token;
    if (m >= M) return;
    const int gi = int(idx - m * per_token);
    const bool is_q = gi < q.groups;
    const Heads& hd = is_q ? q : k;
    const int h0 = (is_q ? gi : gi - q.groups) * hd.per, h1 = min(hd.H, h0 + hd.per);
    const Group<LANES, INTER> g(D, turn.R);
    const int e = g.c * 8;
    const bool norm = hd.w != nullptr;

    int64_t slot = -1;
    if (APPEND && !is_q) {
        slot = cache.slots[m];
        if (slot >= cache.n_slots) {
            if (status_dev) atomicCAS(status_dev, PATCH_OK, PATCH_ERR_SIZE);
            slot = -1;
        }
    }
    const __nv_bfloat16* x = hd.x + m * hd.ldx + e;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    uint4 raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) raw[i] = g.on && h0 + i < h1 ? ld16(x + int64_t(h0 + i) * D) : zero;

    float A[8], B[8];
    g.angles(turn, position(turn, m, status_dev), A, B);
    if (norm) {
        const uint4 wr = g.on ? ld16(hd.w + e) : zero;
        float w[8], wo[8];
        unpack(wr, w);
        unpack(g.other(wr), wo);
#pragma unroll
        for (int i = 0; i < 8; ++i) { A[i] *= w[i]; B[i] *= wo[i]; }
    }
    const float inv_d = 1.0f / float(D);
    for (int h = h0; h < h1; h += kAhead) {
        uint4 next[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) next[i] = g.on && h + kAhead + i < h1 ? ld16(x + int64_t(h + kAhead + i) * D) : zero;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (h + i >= h1) break;
            float v[8], o[8];
            unpack(raw[i], v);
            unpack(g.other(raw[i]), o);
            float r = 1.0f;
            if (norm) {
                float ss = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = fmaf(v[j], v[j], ss);
                r = rsqrtf(fmaf(g.sum(ss), inv_d, eps));
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = r * fmaf(v[j], A[j], o[j] * B[j]);
            if (!g.on) continue;
            if (APPEND && !is_q) {
                if (slot >= 0) {
                    const int64_t at = cache.at(slot, h + i) + e;
                    st16(cache.k + at, pack(v));
                    st16(cache.v + at, ld16(cache.src_v + m * cache.ldv + int64_t(h + i) * D + e));
                }
            } else {
                st16(hd.y + m * hd.ldy + int64_t(h + i) * D + e, pack(v));
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) raw[i] = next[i];
    }
}

struct GradHeads {                        // one kind of head of the gradient kernel
    const __nv_bfloat16 *gy, *x;
    int64_t ldgy, ldx;
    __nv_bfloat16* gx;
    int64_t ldgx;
    const __nv_bfloat16* w;               // null: no norm
    int H, groups, per;
};

// Gradient.  A group keeps its place in the token (which kind, which heads) and walks over tokens, so that the weight's
// gradient stays in registers; a block then adds its groups' sums in group order and writes one row of partial sums per kind.
template <int LANES, bool INTER>
__global__ void __launch_bounds__(kThreads)
rope_backward_kernel(const GradHeads q, const GradHeads k, const Turn turn, int64_t M, int D, float eps, int64_t token_stride,
                     float* __restrict__ partial, int* status_dev) {
    constexpr int kGroups = kThreads / LANES;
    __shared__ float sums[kGroups][LANES * 8];
    __shared__ int kinds[kGroups];
    const int per_token = q.groups + k.groups;
    const int group = threadIdx.x / LANES;
    const int64_t idx = int64_t(blockIdx.x) * kGroups + group;
    const int64_t first = idx / per_token;
    const int gi = int(idx - first * per_token);
    const bool is_q = gi < q.groups;
    const GradHeads& hd = is_q ? q : k;
    const int h0 = (is_q ? gi : gi - q.groups) * hd.per, h1 = min(hd.H, h0 + hd.per);
    const Group<LANES, INTER> g(D, turn.R);
    const int e = g.c * 8;
    const bool norm = hd.w != nullptr;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    const float inv_d = 1.0f / float(D);
    float w[8], gw[8];
    unpack(norm && g.on ? ld16(hd.w + e) : zero, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) gw[j] = 0.0f;
    if (first < token_stride) {           // the last groups of the grid may be over
        for (int64_t m = first; m < M; m += token_stride) {
            float co[8], si[8];
            g.angles(turn, position(turn, m, status_dev), co, si);
            const __nv_bfloat16* gy = hd.gy + m * hd.ldgy + e;
            const __nv_bfloat16* x = hd.x + m * hd.ldx + e;
            __nv_bfloat16* gx = hd.gx + m * hd.ldgx + e;
            for (int h = h0; h < h1; h += kAhead) {
                uint4 ry[kAhead], rx[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const bool in = g.on && h + i < h1;
                    ry[i] = in ? ld16(gy + int64_t(h + i) * D) : zero;
                    rx[i] = in && norm ? ld16(x + int64_t(h + i) * D) : zero;
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (h + i >= h1) break;
                    float v[8], t[8];
                    unpack(ry[i], v);
                    unpack(g.other(ry[i]), t);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = fmaf(v[j], co[j], -t[j] * si[j]);     // R^T gy
                    if (norm) {
                        unpack(rx[i], t);
                        float ss = 0.0f, gx_sum = 0.0f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            ss = fmaf(t[j], t[j], ss);
                            gx_sum = fmaf(v[j] * w[j], t[j], gx_sum);
                        }
                        ss = g.sum(ss);
                        gx_sum = g.sum(gx_sum);
                        const float r = rsqrtf(fmaf(ss, inv_d, eps));
                        const float back = r * r * (gx_sum * inv_d);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            gw[j] = fmaf(v[j], t[j] * r, gw[j]);
                            v[j] = r * fmaf(v[j], w[j], -t[j] * back);
                        }
                    }
                    if (g.on) st16(gx + int64_t(h + i) * D, pack(v));
                }
            }
        }
    }
    if (!partial) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[group][e + j] = gw[j];
    if (g.c == 0) kinds[group] = is_q ? 0 : 1;
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * D; j += kThreads) {
        const int kind = j / D, d = j - kind * D;
        float s = 0.0f;
        for (int i = 0; i < kGroups; ++i) s += kinds[i] == kind ? sums[i][d] : 0.0f;
        partial[int64_t(blockIdx.x) * 2 * D + j] = s;
    }
}

// Column sums of the partial rows: a block takes 32 columns, its 32 warps take rows, in a fixed order.
__global__ void __launch_bounds__(1024)
rope_weight_sum_kernel(const float* __restrict__ partial, int rows, int D, float* __restrict__ gwq, float* __restrict__ gwk) {
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (j < 2 * D)
        for (int r = warp; r < rows; r += 32) s += partial[int64_t(r) * 2 * D + j];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && j < 2 * D) {
        s = 0.0f;
        for (int i = 0; i < 32; ++i) s += sums[i][lane];
        float* out = j < D ? gwq : gwk;
        if (out) out[j < D ? j : j - D] = s;
    }
}

// ---------------------------------------------------------------------------------------------
// host side

static int lanes_of(int D) { return D <= 64 ? 8 : D <= 128 ? 16 : 32; }

static int check_rope(const patch_rope_t* rope, int D, const int32_t* positions, Turn* t) {
    *t = Turn{nullptr, nullptr, 0, 0};
    if (!rope || rope->rotary_dim == 0) return PATCH_OK;
    const int R = rope->rotary_dim;
    if (R < 0 || R > D || R % (rope->interleaved ? 8 : 16) || rope->max_positions < 1) return PATCH_ERR_SHAPE;
    if (!rope->cos_sin_dev || !positions) return PATCH_ERR_NULL;
    if (!aligned16(rope->cos_sin_dev)) return PATCH_ERR_ALIGN;
    *t = Turn{rope->cos_sin_dev, positions, rope->max_positions, R};
    return PATCH_OK;
}
static int check_rows(const void* p, int64_t ld, int H, int D) {
    if (H == 0) return PATCH_OK;
    if (!p) return PATCH_ERR_NULL;
    if (ld < int64_t(H) * D || ld % 8) return PATCH_ERR_SHAPE;
    return aligned16(p) ? PATCH_OK : PATCH_ERR_ALIGN;
}
static int check_heads(int64_t M, int Hq, int Hkv, int D) {
    if (M < 0 || Hq < 0 || Hkv < 0 || Hq > (1 << 16) || Hkv > (1 << 16) || D < 8 || D > 256 || D % 8) return PATCH_ERR_SHAPE;
    return PATCH_OK;
}

// Heads per group of lanes: a group that walks over several heads reads its token's table row and weights once for all
// of them, but while the launch has fewer groups than the GPU's SMs can hold (128 warps' worth of 16-lane groups
// each), splitting the token further fills more of the GPU.
static int heads_per_group(int64_t M, int heads, int lanes) {
    const int64_t room = int64_t(sm_count()) * (2048 / lanes);
    int per = 1;
    while (per < 8 && M * heads / (2 * per) >= room) per *= 2;
    return per;
}
static unsigned blocks_for(int64_t groups, int lanes) { return unsigned((groups * lanes + kThreads - 1) / kThreads); }

template <int LANES, bool INTER>
static int launch_forward(const Heads& q, const Heads& k, const Cache* cache, const Turn& t, int64_t M, int D, float eps,
                          int* status_dev, cudaStream_t s) {
    const int64_t groups = M * (q.groups + k.groups);
    if ((groups * LANES + kThreads - 1) / kThreads > 0x7FFFFFFF) return PATCH_ERR_SHAPE;
    if (cache) rope_kernel<LANES, INTER, true><<<blocks_for(groups, LANES), kThreads, 0, s>>>(q, k, *cache, t, M, D, eps, status_dev);
    else rope_kernel<LANES, INTER, false><<<blocks_for(groups, LANES), kThreads, 0, s>>>(q, k, Cache{}, t, M, D, eps, status_dev);
    return cudaGetLastError() == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}
static int forward(Heads q, Heads k, const Cache* cache, const Turn& t, bool inter, int64_t M, int D, float eps, int* status_dev,
                   cudaStream_t s) {
    const int lanes = lanes_of(D), per = heads_per_group(M, q.H + k.H, lanes);
    q.per = k.per = per;
    q.groups = (q.H + per - 1) / per;
    k.groups = (k.H + per - 1) / per;
    if (lanes == 8) return inter ? launch_forward<8, true>(q, k, cache, t, M, D, eps, status_dev, s) : launch_forward<8, false>(q, k, cache, t, M, D, eps, status_dev, s);
    if (lanes == 16) return inter ? launch_forward<16, true>(q, k, cache, t, M, D, eps, status_dev, s) : launch_forward<16, false>(q, k, cache, t, M, D, eps, status_dev, s);
    return inter ? launch_forward<32, true>(q, k, cache, t, M, D, eps, status_dev, s) : launch_forward<32, false>(q, k, cache, t, M, D, eps, status_dev, s);
}

// Blocks of the gradient kernel: enough to fill the GPU, at most one group of lanes per (token, group of heads).
constexpr int kMaxBackwardBlocks = 160 * 6;
static int backward_blocks(int64_t M, int per_token, int lanes) {
    const int64_t want = blocks_for(M * per_token, lanes) ? (M * per_token * lanes + kThreads - 1) / kThreads : 1;
    const int64_t cap = int64_t(sm_count()) * 6 < kMaxBackwardBlocks ? int64_t(sm_count()) * 6 : kMaxBackwardBlocks;
    return int(want < cap ? want : cap);
}
template <int LANES, bool INTER>
static int launch_backward(const GradHeads& q, const GradHeads& k, const Turn& t, int64_t M, int D, float eps, float* partial,
                           float* gwq, float* gwk, int* status_dev, cudaStream_t s) {
    const int per_token = q.groups + k.groups;
    int blocks = backward_blocks(M, per_token, LANES);
    const int64_t least = (per_token * LANES + kThreads - 1) / kThreads;       // every group of a token has to be somewhere
    if (blocks < least) blocks = int(least);
    const int64_t stride = int64_t(blocks) * (kThreads / LANES) / per_token;
    rope_backward_kernel<LANES, INTER><<<blocks, kThreads, 0, s>>>(q, k, t, M, D, eps, stride, partial, status_dev);
    if (partial) rope_weight_sum_kernel<<<(2 * D + 31) / 32, 1024, 0, s>>>(partial, blocks, D, gwq, gwk);
    return cudaGetLastError() == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}

}  // namespace rope

int validate_kv_cache(const patch_kv_cache_t* c) {
    if (!c) return PATCH_ERR_NULL;
    if (c->num_pages < 1 || c->num_pages > 0x7FFFFFFF || c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)) ||
        c->Hkv < 1 || c->Hkv > (1 << 16) || c->D < 8 || c->D > 256 || c->D % 8 || c->reserved)
        return PATCH_ERR_SHAPE;
    if (c->page_stride % 8 || c->page_stride < int64_t(c->Hkv) * c->page_size * c->D ||
        c->page_stride > (int64_t(1) << 62) / c->num_pages)
        return PATCH_ERR_SHAPE;
    if (!c->k_dev || !c->v_dev) return PATCH_ERR_NULL;
    return aligned16(c->k_dev) && aligned16(c->v_dev) ? PATCH_OK : PATCH_ERR_ALIGN;
}

}  // namespace patch

using namespace patch;

extern "C" int patch_qk_norm_rope(const void* Q, int64_t ldq, int Hq, const void* K, int64_t ldk, int Hkv, int64_t M, int D,
                                  const void* wq, const void* wk, float eps, const patch_rope_t* rope, const int32_t* positions,
                                  void* Qo, int64_t ldqo, void* Ko, int64_t ldko, int* status_dev, void* stream) {
    int rc = rope::check_heads(M, Hq, Hkv, D);
    if (rc) return rc;
    if (M == 0 || Hq + Hkv == 0) return PATCH_OK;
    rope::Turn t;
    if ((rc = rope::check_rope(rope, D, positions, &t))) return rc;
    if ((rc = rope::check_rows(Q, ldq, Hq, D)) || (rc = rope::check_rows(K, ldk, Hkv, D)) ||
        (rc = rope::check_rows(Qo, ldqo, Hq, D)) || (rc = rope::check_rows(Ko, ldko, Hkv, D)))
        return rc;
    if (!aligned16(wq) || !aligned16(wk)) return PATCH_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    using T = const __nv_bfloat16*;
    const rope::Heads q = {static_cast<T>(Q), ldq, static_cast<__nv_bfloat16*>(Qo), ldqo, static_cast<T>(wq), Hq, 0, 0};
    const rope::Heads k = {static_cast<T>(K), ldk, static_cast<__nv_bfloat16*>(Ko), ldko, static_cast<T>(wk), Hkv, 0, 0};
    return rope::forward(q, k, nullptr, t, rope && rope->interleaved, M, D, eps, status_dev, static_cast<cudaStream_t>(stream));
}

extern "C" int patch_kv_append(const patch_kv_cache_t* cache, const void* K, int64_t ldk, const void* V, int64_t ldv,
                               const int64_t* slots, int64_t M, const void* wk, float eps, const patch_rope_t* rope,
                               const int32_t* positions, const void* Q, int64_t ldq, int Hq, const void* wq, void* Qo,
                               int64_t ldqo, int* status_dev, void* stream) {
    int rc = validate_kv_cache(cache);
    if (rc) return rc;
    const int D = cache->D, Hkv = cache->Hkv;
    if ((rc = rope::check_heads(M, Hq, Hkv, D))) return rc;
    if (M == 0) return PATCH_OK;
    rope::Turn t;
    if ((rc = rope::check_rope(rope, D, positions, &t))) return rc;
    if (!slots) return PATCH_ERR_NULL;
    if ((rc = rope::check_rows(K, ldk, Hkv, D)) || (rc = rope::check_rows(V, ldv, Hkv, D)) ||
        (rc = rope::check_rows(Q, ldq, Hq, D)) || (rc = rope::check_rows(Qo, ldqo, Hq, D)))
        return rc;
    if (!aligned16(wq) || !aligned16(wk)) return PATCH_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    using T = const __nv_bfloat16*;
    const rope::Heads q = {static_cast<T>(Q), ldq, static_cast<__nv_bfloat16*>(Qo), ldqo, static_cast<T>(wq), Hq, 0, 0};
    const rope::Heads k = {static_cast<T>(K), ldk, nullptr, 0, static_cast<T>(wk), Hkv, 0, 0};
    rope::Cache c = {static_cast<__nv_bfloat16*>(cache->k_dev), static_cast<__nv_bfloat16*>(cache->v_dev), static_cast<T>(V), ldv,
                     cache->page_stride, cache->num_pages * cache->page_size, slots, 0, D};
    while ((1 << c.shift) < cache->page_size) ++c.shift;
    return rope::forward(q, k, &c, t, rope && rope->interleaved, M, D, eps, status_dev, static_cast<cudaStream_t>(stream));
}

extern "C" int patch_qk_norm_rope_backward_workspace_size(int64_t M, int Hq, int Hkv, int D, size_t* bytes_out) {
    if (!bytes_out) return PATCH_ERR_NULL;
    int rc = rope::check_heads(M, Hq, Hkv, D);
    if (rc) return rc;
    // one row of 2 D partial sums per block; a token's groups of lanes never need more blocks than its heads
    const int64_t least = (int64_t(Hq + Hkv) * rope::lanes_of(D) + rope::kThreads - 1) / rope::kThreads;
    const int64_t blocks = least > rope::kMaxBackwardBlocks ? least : rope::kMaxBackwardBlocks;
    *bytes_out = size_t(blocks) * 2 * D * sizeof(float);
    return PATCH_OK;
}

extern "C" int patch_qk_norm_rope_backward(const void* gQo, int64_t ldgqo, const void* gKo, int64_t ldgko, const void* Q, int64_t ldq,
                                           int Hq, const void* K, int64_t ldk, int Hkv, int64_t M, int D, const void* wq,
                                           const void* wk, float eps, const patch_rope_t* rope, const int32_t* positions, void* gQ,
                                           int64_t ldgq, void* gK, int64_t ldgk, float* gwq, float* gwk, void* workspace,
                                           size_t workspace_bytes, int* status_dev, void* stream) {
    int rc = rope::check_heads(M, Hq, Hkv, D);
    if (rc) return rc;
    rope::Turn t = {nullptr, nullptr, 0, 0};
    if (M > 0 && (rc = rope::check_rope(rope, D, positions, &t))) return rc;
    if (Hq == 0) wq = nullptr;
    if (Hkv == 0) wk = nullptr;
    if ((wq && !gwq) || (wk && !gwk)) return PATCH_ERR_NULL;
    if (!aligned16(wq) || !aligned16(wk)) return PATCH_ERR_ALIGN;
    if (M > 0) {
        if ((rc = rope::check_rows(gQo, ldgqo, Hq, D)) || (rc = rope::check_rows(gKo, ldgko, Hkv, D)) ||
            (rc = rope::check_rows(gQ, ldgq, Hq, D)) || (rc = rope::check_rows(gK, ldgk, Hkv, D)) ||
            (wq && (rc = rope::check_rows(Q, ldq, Hq, D))) || (wk && (rc = rope::check_rows(K, ldk, Hkv, D))))
            return rc;
        if (wq || wk) {
            size_t need = 0;
            if ((rc = patch_qk_norm_rope_backward_workspace_size(M, Hq, Hkv, D, &need))) return rc;
            if (!workspace) return PATCH_ERR_NULL;
            if (workspace_bytes < need) return PATCH_ERR_SIZE;
            if (reinterpret_cast<uintptr_t>(workspace) & 255u) return PATCH_ERR_ALIGN;
        }
    }
    if ((rc = check_device())) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (M == 0 || Hq + Hkv == 0) {          // no tokens: the weights' gradients are zero
        if ((wq && cudaMemsetAsync(gwq, 0, size_t(D) * 4, s) != cudaSuccess) ||
            (wk && cudaMemsetAsync(gwk, 0, size_t(D) * 4, s) != cudaSuccess))
            return PATCH_ERR_CUDA;
        return PATCH_OK;
    }
    using T = const __nv_bfloat16*;
    rope::GradHeads q = {static_cast<T>(gQo), static_cast<T>(Q), ldgqo, ldq, static_cast<__nv_bfloat16*>(gQ), ldgq, static_cast<T>(wq), Hq, 0, 0};
    rope::GradHeads k = {static_cast<T>(gKo), static_cast<T>(K), ldgko, ldk, static_cast<__nv_bfloat16*>(gK), ldgk, static_cast<T>(wk), Hkv, 0, 0};
    const int lanes = rope::lanes_of(D), per = rope::heads_per_group(M, Hq + Hkv, lanes);
    q.per = k.per = per;
    q.groups = (Hq + per - 1) / per;
    k.groups = (Hkv + per - 1) / per;
    float* partial = wq || wk ? static_cast<float*>(workspace) : nullptr;
    gwq = wq ? gwq : nullptr;
    gwk = wk ? gwk : nullptr;
    const bool inter = rope && rope->interleaved;
    if (lanes == 8) return inter ? rope::launch_backward<8, true>(q, k, t, M, D, eps, partial, gwq, gwk, status_dev, s)
                                 : rope::launch_backward<8, false>(q, k, t, M, D, eps, partial, gwq, gwk, status_dev, s);
    if (lanes == 16) return inter ? rope::launch_backward<16, true>(q, k, t, M, D, eps, partial, gwq, gwk, status_dev, s)
                                  : rope::launch_backward<16, false>(q, k, t, M, D, eps, partial, gwq, gwk, status_dev, s);
    return inter ? rope::launch_backward<32, true>(q, k, t, M, D, eps, partial, gwq, gwk, status_dev, s)
                 : rope::launch_backward<32, false>(q, k, t, M, D, eps, partial, gwq, gwk, status_dev, s);
}
