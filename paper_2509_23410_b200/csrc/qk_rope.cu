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
// Layout.  A group of LANES lanes owns a head, 8 elements per lane: 8 lanes for D <= 64, 16 for D <= 128, 32 for D <= 256, so a
// warp works on 4, 2 or 1 heads.  A lane of the rotated part takes four elements of the first half and their four partners
// of the second (pairs (i, i + R/2); two 8-byte loads, each 64 consecutive bytes or more per group), or eight consecutive elements
// (pairs (2i, 2i + 1), and the unrotated rest): either way a pair meets in one lane, needs no exchange between lanes, and shares one
// cosine and sine.  (Sixteen consecutive bytes per lane with an exchange of the raw values: 162 warp instructions per head
// against about 60; that version issued 0.71 instructions per cycle and stayed at 4.1 TB/s.)  Arithmetic is in pairs of fp32
// (one instruction each).  A group keeps its token's coefficients in registers and walks over several heads of the token.
//
// What bounds it: HBM.  Four bytes move per element (six in the gradient), plus 4 R bytes of table per token.  Measured: 16384 tokens
// of 32 + 8 heads of 128 in 58.5 us (5.9 TB/s, a copy's 6.5); 8191 tokens of 40 heads with their values into the cache in 84.3 us
// (6.0 TB/s); gradient of 2047 tokens of 40 + 40 heads in 29.5 us (4.3 TB/s), of 16384 tokens of 32 + 8 heads of 64 in 52.7 us (4.8
// TB/s).  One token appended takes 3.0 us, which is a launch and three dependent reads.
#include "patch_internal.cuh"
#include "sm100_ptx.cuh"
#include "f32x2.cuh"

namespace patch {
namespace rope {

constexpr int kThreads = 256;
constexpr int kAhead = 4;                 // heads whose loads are in flight together
constexpr int kGradAhead = 2;             // the same in the gradient, which loads two operands per head

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

struct Raw { uint2 a, b; };               // a lane's eight bf16 of a head
__device__ __forceinline__ void widen(const Raw& r, f2 (&v)[4]) {
    v[0] = widen2(r.a.x); v[1] = widen2(r.a.y); v[2] = widen2(r.b.x); v[3] = widen2(r.b.y);
}

// One group of lanes.  DT: head size known at compile time (then every lane is inside the head), 0: given at run time.
// INTER: pairs (2i, 2i + 1).  FULL: the whole head is rotated.
template <int LANES, int DT, bool INTER, bool FULL>
struct Group {
    int c;                  // lane's number in the group
    int o0, o1;             // its elements of a head: o0 .. o0 + 3 and o1 .. o1 + 3
    uint32_t mask;          // lanes of the group (groups of a warp may walk over different numbers of heads)
    bool on, turned;        // inside the head; inside the rotated part
    __device__ __forceinline__ Group(int D, int R) {
        const int lane = threadIdx.x & 31;
        c = lane & (LANES - 1);
        mask = LANES == 32 ? 0xFFFFFFFFu : ((1u << (LANES & 31)) - 1u) << (lane & ~(LANES - 1));
        on = DT == LANES * 8 || c * 8 < D;
        turned = FULL || c * 8 < R;
        o0 = !INTER && turned ? 4 * c : 8 * c;
        o1 = !INTER && turned ? 4 * c + R / 2 : 8 * c + 4;
    }
    __device__ __forceinline__ Raw load(const __nv_bfloat16* head, bool in = true) const {
        Raw r = {make_uint2(0u, 0u), make_uint2(0u, 0u)};
        if (on && in) {
            r.a = *reinterpret_cast<const uint2*>(head + o0);
            r.b = *reinterpret_cast<const uint2*>(head + o1);
        }
        return r;
    }
    __device__ __forceinline__ void store(__nv_bfloat16* head, const f2 (&v)[4]) const {
        if (!on) return;
        *reinterpret_cast<uint2*>(head + o0) = make_uint2(narrow2(v[0]), narrow2(v[1]));
        *reinterpret_cast<uint2*>(head + o1) = make_uint2(narrow2(v[2]), narrow2(v[3]));
    }
    // the pairs' other elements; zeros where nothing is rotated (an infinity there must not meet a zero sine)
    __device__ __forceinline__ void other(const f2 (&v)[4], f2 (&o)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[i] = INTER ? swap2(v[i]) : v[i ^ 2];
            if (!FULL) o[i] = turned ? o[i] : 0ull;
        }
    }
    // cosines and signed sines of this lane's elements at position p: y = x co + other(x) si
    __device__ __forceinline__ void angles(const Turn& t, int64_t p, f2 (&co)[4], f2 (&si)[4]) const {
        float4 cs = make_float4(1.f, 1.f, 1.f, 1.f), sn = make_float4(0.f, 0.f, 0.f, 0.f);
        if (turned && on) {
            const float* row = t.cos_sin + p * t.R + 4 * c;
            cs = *reinterpret_cast<const float4*>(row);
            sn = *reinterpret_cast<const float4*>(row + t.R / 2);
        }
        if constexpr (INTER) {
            co[0] = mk2(cs.x, cs.x); co[1] = mk2(cs.y, cs.y); co[2] = mk2(cs.z, cs.z); co[3] = mk2(cs.w, cs.w);
            si[0] = mk2(-sn.x, sn.x); si[1] = mk2(-sn.y, sn.y); si[2] = mk2(-sn.z, sn.z); si[3] = mk2(-sn.w, sn.w);
        } else {
            co[0] = co[2] = mk2(cs.x, cs.y); co[1] = co[3] = mk2(cs.z, cs.w);
            si[0] = mk2(-sn.x, -sn.y); si[1] = mk2(-sn.z, -sn.w); si[2] = mk2(sn.x, sn.y); si[3] = mk2(sn.z, sn.w);
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
template <int LANES, int DT, bool INTER, bool FULL, bool APPEND>
__global__ void __launch_bounds__(kThreads, 4)
rope_kernel(const Heads q, const Heads k, const Cache cache, const Turn turn, int64_t M, int d, float eps, int* status_dev) {
    const int D = DT ? DT : d;
    const int per_token = q.groups + k.groups;
    const int64_t idx = (int64_t(blockIdx.x) * kThreads + threadIdx.x) / LANES;
    const int64_t m = idx / per_token;
    if (m >= M) return;
    const int gi = int(idx - m * per_token);
    const bool is_q = gi < q.groups;
    const Heads& hd = is_q ? q : k;
    const int h0 = (is_q ? gi : gi - q.groups) * hd.per, h1 = min(hd.H, h0 + hd.per);
    const Group<LANES, DT, INTER, FULL> g(D, FULL ? D : turn.R);
    const bool norm = hd.w != nullptr, store_kv = APPEND && !is_q;

    const __nv_bfloat16* x = hd.x + m * hd.ldx + int64_t(h0) * D;
    Raw raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) raw[i] = g.load(x + i * D, h0 + i < h1);
    int64_t slot = -1;
    if (store_kv) {
        slot = cache.slots[m];
        if (slot >= cache.n_slots) {
            if (status_dev) atomicCAS(status_dev, PATCH_OK, PATCH_ERR_SIZE);
            slot = -1;
        }
    }
    f2 A[4], B[4];
    g.angles(turn, position(turn, m, status_dev), A, B);
    if (norm) {
        f2 w[4], wo[4];
        widen(g.load(hd.w), w);
        g.other(w, wo);
#pragma unroll
        for (int i = 0; i < 4; ++i) { A[i] = mul2(A[i], w[i]); B[i] = mul2(B[i], wo[i]); }
    }
    // results: rows of heads, or the token's slot of the cache
    __nv_bfloat16* y = store_kv ? cache.k + cache.at(slot < 0 ? 0 : slot, h0) : hd.y + m * hd.ldy + int64_t(h0) * D;
    const int64_t step = store_kv ? int64_t(D) << cache.shift : D;
    const bool keep = !store_kv || slot >= 0;
    const float inv_d = 1.0f / float(D);
    for (int h = h0; h < h1; h += kAhead) {
        if (h > h0) {
            x += kAhead * D;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) raw[i] = g.load(x + i * D, h + i < h1);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (h + i >= h1) break;
            f2 v[4], o[4];
            widen(raw[i], v);
            g.other(v, o);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = mul2(o[j], B[j]);
            if (norm) {
                f2 ss = mul2(v[0], v[0]);
#pragma unroll
                for (int j = 1; j < 4; ++j) ss = fma2(v[j], v[j], ss);
                const float r = rsqrtf(fmaf(g.sum(sum2(ss)), inv_d, eps));
                const f2 rr = mk2(r, r);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = mul2(rr, fma2(v[j], A[j], o[j]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fma2(v[j], A[j], o[j]);
            }
            if (keep) g.store(y, v);
            y += step;
        }
    }
    if (store_kv && keep && g.on) {                  // the same heads of V, copied
        const __nv_bfloat16* src = cache.src_v + m * cache.ldv + int64_t(h0) * D + 8 * g.c;
        __nv_bfloat16* dst = cache.v + cache.at(slot, h0) + 8 * g.c;
        for (int h = h0; h < h1; h += kAhead) {
            uint4 t[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (h + i < h1) t[i] = *reinterpret_cast<const uint4*>(src + i * D);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (h + i < h1) *reinterpret_cast<uint4*>(dst + i * step) = t[i];
            src += kAhead * D;
            dst += kAhead * step;
        }
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
template <int LANES, int DT, bool INTER, bool FULL>
__global__ void __launch_bounds__(kThreads, 3)
rope_backward_kernel(const GradHeads q, const GradHeads k, const Turn turn, int64_t M, int d, float eps, int64_t token_stride,
                     float* __restrict__ partial, int* status_dev) {
    constexpr int kGroups = kThreads / LANES;
    __shared__ float sums[kGroups][LANES * 8];
    __shared__ int kinds[kGroups];
    const int D = DT ? DT : d;
    // The kernel that adds up the partial sums waits for this one's end by itself.  Without weights there is none: what follows then is the
    // caller's, and a GEMM whose input is promised to be there would not wait.
    if (partial) grid_launch_dependents();
    const int per_token = q.groups + k.groups;
    const int group = threadIdx.x / LANES;
    const int64_t idx = int64_t(blockIdx.x) * kGroups + group;
    const int64_t first = idx / per_token;
    const int gi = int(idx - first * per_token);
    const bool is_q = gi < q.groups;
    const GradHeads& hd = is_q ? q : k;
    const int h0 = (is_q ? gi : gi - q.groups) * hd.per, h1 = min(hd.H, h0 + hd.per);
    const Group<LANES, DT, INTER, FULL> g(D, FULL ? D : turn.R);
    const bool norm = hd.w != nullptr;
    const float inv_d = 1.0f / float(D);
    const f2 minus = mk2(-1.0f, -1.0f);
    f2 w[4] = {0ull, 0ull, 0ull, 0ull}, gw[4] = {0ull, 0ull, 0ull, 0ull};
    if (norm) widen(g.load(hd.w), w);
    if (first < token_stride) {           // the last groups of the grid may be over
        for (int64_t m = first; m < M; m += token_stride) {
            const __nv_bfloat16* gy = hd.gy + m * hd.ldgy + int64_t(h0) * D;
            const __nv_bfloat16* x = hd.x + m * hd.ldx + int64_t(h0) * D;
            __nv_bfloat16* gx = hd.gx + m * hd.ldgx + int64_t(h0) * D;
            f2 co[4], si[4];
            g.angles(turn, position(turn, m, status_dev), co, si);
#pragma unroll
            for (int j = 0; j < 4; ++j) si[j] = mul2(si[j], minus);          // R^T
            for (int h = h0; h < h1; h += kGradAhead) {
                Raw ry[kGradAhead], rx[kGradAhead];
#pragma unroll
                for (int i = 0; i < kGradAhead; ++i) {
                    ry[i] = g.load(gy + i * D, h + i < h1);
                    rx[i] = g.load(x + i * D, norm && h + i < h1);
                }
#pragma unroll
                for (int i = 0; i < kGradAhead; ++i) {
                    if (h + i >= h1) break;
                    f2 v[4], t[4];
                    widen(ry[i], v);
                    g.other(v, t);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = fma2(v[j], co[j], mul2(t[j], si[j]));
                    if (norm) {
                        widen(rx[i], t);
                        f2 wg[4], ss = 0ull, gs = 0ull;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            wg[j] = mul2(v[j], w[j]);
                            ss = fma2(t[j], t[j], ss);
                            gs = fma2(wg[j], t[j], gs);
                        }
                        const float sx = g.sum(sum2(ss)), sg = g.sum(sum2(gs));
                        const float r = rsqrtf(fmaf(sx, inv_d, eps)), back = -r * r * (sg * inv_d);
                        const f2 rr = mk2(r, r), bb = mk2(back, back);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            t[j] = mul2(t[j], rr);
                            gw[j] = fma2(v[j], t[j], gw[j]);
                            v[j] = fma2(wg[j], rr, mul2(t[j], bb));
                        }
                    }
                    g.store(gx + i * D, v);
                }
                gy += kGradAhead * D;
                x += kGradAhead * D;
                gx += kGradAhead * D;
            }
        }
    }
    if (!partial) return;
    if (g.on) {
#pragma unroll
        for (int j = 0; j < 4; ++j) un2(gw[j], sums[group][(j < 2 ? g.o0 : g.o1 - 4) + 2 * j], sums[group][(j < 2 ? g.o0 : g.o1 - 4) + 2 * j + 1]);
    }
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
    grid_dependency_wait();
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
    if (R < 0 || R > D || R % 8 || rope->max_positions < 1) return PATCH_ERR_SHAPE;
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
    const int64_t room = int64_t(sm_count()) * (1024 / lanes);
    int per = 1;
    while (per < 8 && M * heads / per > room) per *= 2;
    return per;
}
static unsigned blocks_for(int64_t groups, int lanes) { return unsigned((groups * lanes + kThreads - 1) / kThreads); }

// Runs `f` with the kernel variant for heads of D elements of which R are rotated as its template arguments: heads of 64 and
// 128 have kernels of their own with D known at compile time (offsets become immediates, no lane is outside the head), and
// so has the head that is rotated as a whole; any other D or R takes the general ones.
template <class F>
static int dispatch(int D, int R, bool inter, F&& f) {
#define PATCH_ROPE_CASE(LANES, DT) \
    return R == D ? (inter ? f.template operator()<LANES, DT, true, true>() : f.template operator()<LANES, DT, false, true>()) \
                  : (inter ? f.template operator()<LANES, DT, true, false>() : f.template operator()<LANES, DT, false, false>())
    if (D == 64) PATCH_ROPE_CASE(8, 64);
    if (D == 128) PATCH_ROPE_CASE(16, 128);
#undef PATCH_ROPE_CASE
    if (D <= 64) return inter ? f.template operator()<8, 0, true, false>() : f.template operator()<8, 0, false, false>();
    if (D <= 128) return inter ? f.template operator()<16, 0, true, false>() : f.template operator()<16, 0, false, false>();
    return inter ? f.template operator()<32, 0, true, false>() : f.template operator()<32, 0, false, false>();
}

struct Forward {
    const Heads &q, &k;
    const Cache* cache;
    const Turn& t;
    int64_t M;
    int D;
    float eps;
    int* status_dev;
    cudaStream_t s;
    template <int LANES, int DT, bool INTER, bool FULL> int operator()() const {
        const int64_t groups = M * (q.groups + k.groups);
        if ((groups * LANES + kThreads - 1) / kThreads > 0x7FFFFFFF) return PATCH_ERR_SHAPE;
        const unsigned blocks = blocks_for(groups, LANES);
        if (cache) rope_kernel<LANES, DT, INTER, FULL, true><<<blocks, kThreads, 0, s>>>(q, k, *cache, t, M, D, eps, status_dev);
        else rope_kernel<LANES, DT, INTER, FULL, false><<<blocks, kThreads, 0, s>>>(q, k, Cache{}, t, M, D, eps, status_dev);
        return cudaGetLastError() == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
    }
};
static int forward(Heads q, Heads k, const Cache* cache, const Turn& t, bool inter, int64_t M, int D, float eps, int* status_dev,
                   cudaStream_t s) {
    const int lanes = lanes_of(D), per = heads_per_group(M, q.H + k.H, lanes);
    q.per = k.per = per;
    q.groups = (q.H + per - 1) / per;
    k.groups = (k.H + per - 1) / per;
    return dispatch(D, t.R, inter, Forward{q, k, cache, t, M, D, eps, status_dev, s});
}

// Blocks of the gradient kernel: enough to fill the GPU, at most one group of lanes per (token, group of heads).
constexpr int kMaxBackwardBlocks = 160 * 3;
static int backward_blocks(int64_t M, int per_token, int lanes) {
    const int64_t want = (M * per_token * lanes + kThreads - 1) / kThreads;
    const int64_t cap = int64_t(sm_count()) * 3 < kMaxBackwardBlocks ? int64_t(sm_count()) * 3 : kMaxBackwardBlocks;
    return int(want < cap ? want : cap);
}
struct Backward {
    const GradHeads &q, &k;
    const Turn& t;
    int64_t M;
    int D;
    float eps;
    float *partial, *gwq, *gwk;
    int* status_dev;
    cudaStream_t s;
    template <int LANES, int DT, bool INTER, bool FULL> int operator()() const {
        const int per_token = q.groups + k.groups;
        int blocks = backward_blocks(M, per_token, LANES);
        const int least = (per_token * LANES + kThreads - 1) / kThreads;       // every group of a token has to be somewhere
        if (blocks < least) blocks = least;
        const int64_t stride = int64_t(blocks) * (kThreads / LANES) / per_token;
        rope_backward_kernel<LANES, DT, INTER, FULL><<<blocks, kThreads, 0, s>>>(q, k, t, M, D, eps, stride, partial, status_dev);
        if (cudaGetLastError() != cudaSuccess) return PATCH_ERR_CUDA;
        if (!partial) return PATCH_OK;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        cfg.gridDim = dim3(unsigned(2 * D + 31) / 32, 1, 1);
        cfg.blockDim = dim3(1024, 1, 1);
        cfg.stream = s;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, rope_weight_sum_kernel, static_cast<const float*>(partial), blocks, D, gwq, gwk) == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
    }
};

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
    return rope::dispatch(D, t.R, rope && rope->interleaved, rope::Backward{q, k, t, M, D, eps, partial, gwq, gwk, status_dev, s});
}
