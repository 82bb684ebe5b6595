// What is learned and scored from a row of logits: log probabilities of given tokens with entropy and top alternatives, their gradient, and
// distillation from a teacher's top logits with its gradient (public header: patch_token_logprobs, ..._backward, patch_distill_loss,
// ..._backward).
//
// Mathematics.  With m the row's maximum and c = log2(e) / T, one pass gives S = sum 2^((x - m) c) and, for the entropy, sum 2^((x - m) c)
// (x - m): every thread keeps a running maximum and rescales its sums when it grows (difference first, scale second, so that the largest
// element's exponent is exactly 0), threads are joined by the same rule.  Sums are fp32 over some hundred elements of a thread, then over
// a tree in a fixed order: equal calls give equal bits.
//
// Top k.  A thread's running maximum is also the best of the thread's elements, so the pass over the row pays nothing for them:
// the k-th largest of the threads' bests is a lower bound of the k-th largest element, found by a bisection over the sort key with one vote
// of the block per bit; only threads whose best reaches it can hold one of the k, and a warp reads each such thread's elements again (from
// L2) and keeps those that reach it, k to 2 k of them in most rows.  A candidate's rank is the number of candidates before it.  Rows with thousands of
// elements at the border (all equal, all masked) take the exact way round: the k-th key by bisection over the row, what lies above it, and
// the first elements that equal it.
#include <math.h>
#include "patch_internal.cuh"
#include "sm100_ptx.cuh"
#include "f32x2.cuh"

namespace patch {
namespace logits {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPerSm = 3;                    // CTAs that fit an SM: 80 registers a thread
constexpr int kAhead = 4;                    // vectors of 16 bytes that a thread has on their way together
constexpr int kMost = 256;                   // alternatives or teacher's entries of a row, at most; kMost <= kThreads
constexpr int kCandidates = 2048;
constexpr int kCells = 32;                   // see Cells, per thread
constexpr int kFound = 2048;                 // cells that reach the border, most often k to 1.5 k
constexpr size_t kListBytes = kCandidates * sizeof(uint64_t) + kFound * sizeof(uint32_t);
constexpr int kMaxParts = 8;                 // CTAs of a cluster that share a row
constexpr int64_t kMaxV = int64_t(1) << 20;  // a bit per element fits shared memory
static_assert(kMost <= kThreads && kMaxParts * kMost <= kCandidates, "lists of all parts of a row fit the candidates");

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void store16(void* p, uint4 v) {
    asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(float x) { return x; }

// Sixteen bytes of a row.
template <class T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    uint32_t w[4];
    __device__ __forceinline__ void set(uint4 v) { w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0xFF80FF80u; }          // -inf
    __device__ __forceinline__ void hide(uint32_t mask) {          // elements whose bit is set: -inf
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((mask >> i) & 1u) w[i >> 1] = (i & 1) ? (w[i >> 1] & 0xFFFFu) | 0xFF800000u : (w[i >> 1] & 0xFFFF0000u) | 0xFF80u;
    }
    __device__ __forceinline__ f2 pair(int i) const { return widen2(w[i]); }
    __device__ __forceinline__ float top() const {                 // largest element that is a number
        __nv_bfloat162 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
        const __nv_bfloat162 t = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(t), __high2float(t));
    }
};
template <> struct Vec<float> {
    static constexpr int N = 4;
    uint32_t w[4];
    __device__ __forceinline__ void set(uint4 v) { w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0xFF800000u; }
    __device__ __forceinline__ void hide(uint32_t mask) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((mask >> i) & 1u) w[i] = 0xFF800000u;
    }
    __device__ __forceinline__ f2 pair(int i) const { return mk2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])); }
    __device__ __forceinline__ float top() const {
        return fmaxf(fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])), fmaxf(__uint_as_float(w[2]), __uint_as_float(w[3])));
    }
};
template <class T> __device__ __forceinline__ float element(const Vec<T>& v, int i) {
    float a, b;
    un2(v.pair(i >> 1), a, b);
    return (i & 1) ? b : a;
}
template <class T> __device__ __forceinline__ uint4 to_raw(const float (&x)[Vec<T>::N]);
template <> __device__ __forceinline__ uint4 to_raw<__nv_bfloat16>(const float (&x)[8]) {
    return make_uint4(narrow2(mk2(x[0], x[1])), narrow2(mk2(x[2], x[3])), narrow2(mk2(x[4], x[5])), narrow2(mk2(x[6], x[7])));
}
template <> __device__ __forceinline__ uint4 to_raw<float>(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <class T> __device__ __forceinline__ T rounded(float x);
template <> __device__ __forceinline__ float rounded<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <class T> struct Batch { Vec<T> v[kAhead]; };

// A CTA's part of a row: vector numbers part * kThreads + thread, then every parts * kThreads-th.  The row's last vector may be short.
template <class T> struct Row {
    static constexpr int N = Vec<T>::N;
    const T* z;
    int V, whole, count;                     // elements; whole vectors; vectors
    int first, step;
    __device__ __forceinline__ Row(const T* z_, int V_, int part, int parts)
        : z(z_), V(V_), whole(V_ / N), count((V_ + N - 1) / N), first(part * kThreads + threadIdx.x), step(parts * kThreads) {}
    // vector v, -inf past the row's end
    __device__ __forceinline__ Vec<T> load(int v) const {
        Vec<T> x;
        if (v < whole) {
            x.set(load16(z + int64_t(v) * N));
            return x;
        }
        x.clear();
        if (v < count) {
            for (int i = v * N; i < V; ++i) {
                if constexpr (sizeof(T) == 2) {
                    const uint32_t h = *reinterpret_cast<const uint16_t*>(z + i);
                    uint32_t& w = x.w[(i - v * N) >> 1];
                    w = (i & 1) ? (w & 0xFFFFu) | (h << 16) : (w & 0xFFFF0000u) | h;
                } else {
                    x.w[i - v * N] = *reinterpret_cast<const uint32_t*>(z + i);
                }
            }
        }
        return x;
    }
    __device__ __forceinline__ void store(T* g, int v, const float (&y)[N]) const {
        if (v < whole) {
            store16(g + int64_t(v) * N, to_raw<T>(y));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (v * N + i < V) g[v * N + i] = rounded<T>(y[i]);
        }
    }
    // A thread's vectors come in batches that are loaded together, one batch ahead of the arithmetic.  Batch b holds vectors
    // at(b, 0) .. at(b, kAhead - 1); those that are not whole are -inf (the row's short last vector is the caller's: `rest`).
    __device__ __forceinline__ int at(int b, int u) const { return first + (b * kAhead + u) * step; }
    __device__ __forceinline__ int batches() const { return whole > first ? (whole - first + kAhead * step - 1) / (kAhead * step) : 0; }
    __device__ __forceinline__ void fetch(Batch<T>& x, int b) const {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int v = at(b, u);
            if (v < whole) x.v[u].set(load16(z + int64_t(v) * N));
            else x.v[u].clear();
        }
    }
    __device__ __forceinline__ bool rest() const { return count > whole && whole >= first && (whole - first) % step == 0; }
    // f(batch number, batch) for all of them; `ahead` holds the first one, and whatever next(ahead) fetches afterwards
    template <class F, class Next> __device__ __forceinline__ void each(Batch<T>& ahead, F&& f, Next&& next) const {
        const int n = batches();
        if (n == 0) next(ahead);
#pragma unroll 2
        for (int b = 0; b < n; ++b) {
            Batch<T> x = ahead;
            if (b + 1 < n) fetch(ahead, b + 1);
            else next(ahead);
            f(b, x);
        }
    }
};

// maximum, sum of 2^((x - m) c), sum of that times (x - m)
struct Sums { float m, s, t; };
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float c) {
    if (b.m == -INFINITY) return Sums{a.m, a.s + b.s, a.t + b.t};        // nothing in b, or NaN
    if (a.m == -INFINITY) return Sums{b.m, a.s + b.s, a.t + b.t};
    const float m = fmaxf(a.m, b.m), da = fmaxf(a.m - m, -1e30f), db = fmaxf(b.m - m, -1e30f), fa = ex2(da * c), fb = ex2(db * c);
    return Sums{m, a.s * fa + b.s * fb, fa * (a.t + da * a.s) + fb * (b.t + db * b.s)};
}

struct Shared {
    Sums warp[kWarps];
    Sums part;                               // of this CTA, read by the cluster
    float value[kMost];                      // see the kernels
    int id[kMost];
    int n, n2;
    int scan[kWarps];
};

// Sums of 32 lanes, of the first N of them: the largest maximum, then every lane's sums times one factor, added up in a fixed order.
template <int N> __device__ __forceinline__ Sums sum_of_lanes(Sums x, float c) {
    float m = x.m;
#pragma unroll
    for (int d = N / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    if (x.m > -INFINITY) {                   // else nothing, or NaN
        const float d = fmaxf(x.m - m, -1e30f), f = ex2(d * c);
        x.t = f * (x.t + d * x.s);
        x.s *= f;
    }
#pragma unroll
    for (int d = N / 2; d > 0; d >>= 1) {
        x.s += __shfl_xor_sync(0xFFFFFFFFu, x.s, d);
        x.t += __shfl_xor_sync(0xFFFFFFFFu, x.t, d);
    }
    return Sums{m, x.s, x.t};
}
// Sums of a row from those of every thread; all threads get them.  `c`: log2(e) / T.
__device__ __forceinline__ Sums sum_up(Sums x, float c, Shared& sh, int parts) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    x = sum_of_lanes<32>(x, c);
    if (lane == 0) sh.warp[warp] = x;
    __syncthreads();
    x = sum_of_lanes<kWarps>(sh.warp[lane & (kWarps - 1)], c);
    if (parts == 1) {
        __syncthreads();                     // sh.warp may be written again
        return x;
    }
    if (threadIdx.x == 0) sh.part = x;
    cluster_sync_all();
    for (int r = 0; r < parts; ++r) {
        const uint32_t at = map_to_rank(smem_u32(&sh.part), r);
        Sums o;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.m) : "r"(at));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.s) : "r"(at + 4));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.t) : "r"(at + 8));
        x = r ? join(x, o, c) : o;
    }
    return x;
}

// One pass over a thread's elements, COUNT vectors at a time.  HIDE: elements whose bit is set in `bits` do not count.
template <class T, bool ENTROPY>
struct Scan {
    static constexpr int N = Vec<T>::N;
    float m = -INFINITY, c;
    f2 s2 = 0ull, t2 = 0ull;
    __device__ __forceinline__ explicit Scan(float c_) : c(c_) {}
    template <int COUNT> __device__ __forceinline__ float take(const Vec<T> (&e)[COUNT]) {       // returns the largest element
        float top = e[0].top();
#pragma unroll
        for (int u = 1; u < COUNT; ++u) top = fmaxf(top, e[u].top());
        if (top > m) {
            if (m > -INFINITY) {
                const float d = fmaxf(m - top, -1e30f), f = ex2(d * c);
                if (ENTROPY) t2 = mul2(mk2(f, f), fma2(mk2(d, d), s2, t2));
                s2 = mul2(mk2(f, f), s2);
            }
            m = top;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        const f2 b2 = mk2(-base, -base), c2 = mk2(c, c);
#pragma unroll
        for (int u = 0; u < COUNT; ++u)
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const f2 d = add2(e[u].pair(i), b2);
                float a, b;
                un2(mul2(d, c2), a, b);
                const f2 p = mk2(ex2(a), ex2(b));
                s2 = add2(s2, p);
                if (ENTROPY) {
                    un2(d, a, b);            // a masked element: 0 times a number, not times -inf
                    t2 = fma2(p, mk2(fmaxf(a, -1e30f), fmaxf(b, -1e30f)), t2);
                }
            }
        return top;
    }
    __device__ __forceinline__ Sums sums() const { return Sums{m, sum2(s2), sum2(t2)}; }
};
template <class T> __device__ __forceinline__ void hide_listed(Vec<T>& x, int v, const uint32_t* bits) {
    constexpr int N = Vec<T>::N;
    const uint32_t mask = (bits[v / (32 / N)] >> (v % (32 / N) * N)) & ((1u << N) - 1u);
    if (mask) x.hide(mask);
}
// The largest element of every 2^shift batches of a thread, for the alternatives: cell [batch >> shift][thread].
struct Cells {
    float* at;
    int shift;
    static __host__ __device__ int shift_of(int batches) {
        int s = 0;
        while ((batches >> s) >= kCells) ++s;
        return s;
    }
};
template <class T, bool ENTROPY, bool HIDE, bool TOP, class Next>
__device__ __forceinline__ Sums scan_row(const Row<T>& row, Batch<T>& ahead, float c, const uint32_t* bits, const Cells& cells, Next&& next) {
    Scan<T, ENTROPY> scan(c);
    float cell = -INFINITY;
    row.each(ahead, [&](int b, Batch<T>& x) {
        if (HIDE) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (row.at(b, u) < row.whole) hide_listed(x.v[u], row.at(b, u), bits);
        }
        const float top = scan.take(x.v);
        if (TOP) {
            cell = fmaxf(cell, top);
            if (((b + 1) & ((1 << cells.shift) - 1)) == 0 || b + 1 == row.batches()) {
                cells.at[(b >> cells.shift) * kThreads + threadIdx.x] = cell;
                cell = -INFINITY;
            }
        }
    }, next);
    if (row.rest()) {
        Vec<T> x[1] = {row.load(row.whole)};
        if (HIDE) hide_listed(x[0], row.whole, bits);
        scan.take(x);
    }
    return scan.sums();
}

// Order of the alternatives: larger value first, then lower index.  A value's sort key; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (!(x > -INFINITY)) x = -INFINITY;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key); }
__device__ __forceinline__ uint64_t candidate(uint32_t key, int index) { return (uint64_t(key) << 32) | uint32_t(~index); }
__device__ __forceinline__ int block_sum(int n, Shared& sh) {
    n = __reduce_add_sync(0xFFFFFFFFu, n);
    if ((threadIdx.x & 31) == 0) sh.scan[threadIdx.x >> 5] = n;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += sh.scan[w];
    __syncthreads();
    return sum;
}

// The k first candidates of `list` [n], in order, to `out`.  Keys are distinct.  Eight lanes count for one candidate.
__device__ __forceinline__ void rank(const uint64_t* list, int n, int k, uint64_t* out) {
    const int sub = threadIdx.x & 7;
    for (int i0 = 0; i0 < n; i0 += kThreads / 8) {
        const int i = i0 + (threadIdx.x >> 3);
        const uint64_t mine = i < n ? list[i] : 0ull;
        int before = 0;
#pragma unroll 4
        for (int j = sub; j < n; j += 8) before += list[j] > mine;
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) before += __shfl_xor_sync(0xFFFFFFFFu, before, d);
        if (sub == 0 && i < n && before < k) out[before] = mine;
    }
}

// The first k elements, in order, of this CTA's part of a row (which has k) -> top[k].  `best`: the largest of the thread's elements; `cells`:
// of its batches.  All threads of the CTA; ends with a barrier.
template <class T>
__device__ __forceinline__ void top_of_part(const Row<T>& row, float best, const Cells& cells, int k, uint64_t* list, uint64_t* top, Shared& sh) {
    constexpr int N = Vec<T>::N;
    constexpr int kLowest = sizeof(T) == 2 ? 16 : 0;                      // bf16 keys differ in their high halves
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t mine = row.first < row.count ? key_of(best) >> kLowest : 0u;        // an element's key is above 0
    uint32_t border = 0;
    for (int bit = 31 - kLowest; bit >= 0; --bit) {
        const uint32_t next = border | (1u << bit);
        const int n = __syncthreads_count(mine >= next);
        if (n >= k) border = next;
        if (n == k) break;
    }
    // candidates of vector v whose keys are `least` or more
    auto look = [&](int v, uint32_t least) {
        const Vec<T> x = row.load(v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t key = key_of(element(x, i));
            if ((key >> kLowest) >= least && v * N + i < row.V) {
                const int at = atomicAdd(&sh.n, 1);
                if (at < kCandidates) list[at] = candidate(key, v * N + i);
            }
        }
    };
    // cells that reach the border, and the short last vector
    uint32_t* const found = reinterpret_cast<uint32_t*>(list + kCandidates);
    if (threadIdx.x == 0) sh.n = sh.n2 = 0;
    __syncthreads();
    if (mine >= border && mine) {
        const int n = (row.batches() + (1 << cells.shift) - 1) >> cells.shift;
        for (int g = 0; g < n; ++g)
            if ((key_of(cells.at[g * kThreads + threadIdx.x]) >> kLowest) >= border) {
                const int at = atomicAdd(&sh.n2, 1);
                if (at < kFound) found[at] = uint32_t(g) << 16 | threadIdx.x;
            }
        if (row.rest()) look(row.whole, border);
    }
    __syncthreads();
    int n = sh.n2;
    auto key_of_cell = [&](uint32_t f) { return key_of(cells.at[(f >> 16) * kThreads + (f & 0xFFFFu)]) >> kLowest; };
    if (n > 2 * k && n <= kFound) {          // the threads' bests were few for a k of this size: the k-th cell is a better border
        uint32_t better = 0;
        for (int bit = 31 - kLowest; bit >= 0; --bit) {
            int sum = 0;
            for (int i = threadIdx.x; i < n; i += kThreads) sum += key_of_cell(found[i]) >= (better | (1u << bit));
            if (block_sum(sum, sh) >= k) better |= 1u << bit;
        }
        border = max(border, better);
    }
    if (n <= kFound) {
        const int each = kAhead << cells.shift;                    // vectors of a cell
        for (int i = threadIdx.x; i < n * each; i += kThreads) {
            const uint32_t f = found[i / each];
            const int v = row.first - int(threadIdx.x) + int(f & 0xFFFFu) + (int(f >> 16) * each + i % each) * row.step;
            if (v < row.whole && key_of_cell(f) >= border) look(v, border);
        }
    }
    __syncthreads();
    const bool few = n <= kFound && sh.n <= kCandidates;
    n = sh.n;
    __syncthreads();
    if (few) {
        rank(list, n, k, top);
        __syncthreads();
        return;
    }
    // Many elements at the border.  The k-th key itself: the border where fewer than k lie above it, else by bisection over the row.
    auto count = [&](uint32_t least) {
        int sum = 0;
        for (int v = row.first; v < row.count; v += row.step) {
            const Vec<T> x = row.load(v);
#pragma unroll
            for (int i = 0; i < N; ++i) sum += (key_of(element(x, i)) >> kLowest) >= least && v * N + i < row.V;
        }
        return block_sum(sum, sh);
    };
    if (count(border + 1) >= k) {
        border = 0;
        for (int bit = 31 - kLowest; bit >= 0; --bit)
            if (count(border | (1u << bit)) >= k) border |= 1u << bit;
    }
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    for (int v = row.first; v < row.count; v += row.step) look(v, border + 1);                   // fewer than k
    __syncthreads();
    int have = sh.n;
    for (int v0 = row.first - threadIdx.x; v0 < row.count && have < k; v0 += row.step) {         // and the first ones that equal it
        const int v = v0 + threadIdx.x;
        uint32_t equal = 0;
        Vec<T> x;
        if (v < row.count) {
            x = row.load(v);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if ((key_of(element(x, i)) >> kLowest) == border && v * N + i < row.V) equal |= 1u << i;
        }
        const int own = __popc(equal);
        int before = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xFFFFFFFFu, before, d);
            if (lane >= d) before += o;
        }
        if (lane == 31) sh.scan[warp] = before;
        __syncthreads();
        int sum = 0;
        before -= own;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += sh.scan[w];
            sum += sh.scan[w];
        }
        __syncthreads();
        int at = have + before;
        for (uint32_t todo = equal; todo && at < k; todo &= todo - 1, ++at) {
            const int i = __ffs(todo) - 1;
            list[at] = candidate(key_of(element(x, i)), v * N + i);
        }
        have += sum;
    }
    __syncthreads();
    rank(list, min(have, k), k, top);
    __syncthreads();
}

struct LogProbs {
    int64_t ldz, M;
    int V, k, parts, cell_shift;
    float c, temperature;
    const int64_t* tokens;
    float *logp, *entropy, *lse, *top_logp;
    int32_t* top_ids;
    int* status;
};

template <class T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(kThreads, kPerSm) logprobs_kernel(const T* z, const LogProbs p) {
    __shared__ Shared sh;
    __shared__ uint64_t top[TOP ? kMost : 1];
    extern __shared__ uint64_t list[];       // TOP: kCandidates, then numbers of kFound cells, then the cells
    const Cells cells = {reinterpret_cast<float*>(list + kCandidates) + kFound, p.cell_shift};
    const int part = p.parts > 1 ? int(cluster_ctarank()) : 0;
    const int64_t rows = gridDim.x / p.parts;
    Batch<T> ahead;
    if (int64_t m = blockIdx.x / p.parts; m < p.M) Row<T>(z + m * p.ldz, p.V, part, p.parts).fetch(ahead, 0);
    for (int64_t m = blockIdx.x / p.parts; m < p.M; m += rows) {
        const Row<T> row(z + m * p.ldz, p.V, part, p.parts);
        const Sums own = scan_row<T, ENTROPY, false, TOP>(row, ahead, p.c, nullptr, cells, [&](Batch<T>& x) {
            if (m + rows < p.M) Row<T>(z + (m + rows) * p.ldz, p.V, part, p.parts).fetch(x, 0);
        });
        const Sums x = sum_up(own, p.c, sh, p.parts);
        const float base = x.m == -INFINITY ? 0.0f : x.m;
        const bool none = x.m == -INFINITY && !(x.s != x.s);      // every element is -inf: no distribution
        const float ln = TOP || (part == 0 && threadIdx.x == 0) ? logf(x.s) : 0.0f;
        if (part == 0 && threadIdx.x == 0) {
            if (p.tokens) {
                const int64_t t = p.tokens[m];
                float y = 0.0f;
                if (t >= p.V) {
                    if (p.status) atomicCAS(p.status, PATCH_OK, PATCH_ERR_SIZE);
                } else if (t >= 0) {
                    y = none ? -INFINITY : (as_float(row.z[t]) - base) / p.temperature - ln;
                }
                p.logp[m] = y;
            }
            if (p.lse) p.lse[m] = none ? -INFINITY : base / p.temperature + ln;
            if (ENTROPY) p.entropy[m] = none ? 0.0f : ln - x.t / (x.s * p.temperature);
        }
        if (TOP) {
            top_of_part(row, own.m, cells, p.k, list, top, sh);
            if (p.parts > 1) {
                cluster_sync_all();
                if (part == 0) {
                    for (int i = threadIdx.x; i < p.parts * p.k; i += kThreads) {
                        const int r = i / p.k;
                        uint64_t v;
                        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(map_to_rank(smem_u32(top + (i - r * p.k)), r)) : "memory");
                        list[i] = v;
                    }
                }
                cluster_sync_all();          // the others' lists have been read
                if (part == 0) rank(list, p.parts * p.k, p.k, top);
                __syncthreads();
            }
            if (part == 0) {
                for (int i = threadIdx.x; i < p.k; i += kThreads) {
                    const uint64_t v = top[i];
                    const int id = int(~uint32_t(v));
                    p.top_ids[m * p.k + i] = id;
                    p.top_logp[m * p.k + i] = none ? -INFINITY : (value_of(uint32_t(v >> 32)) - base) / p.temperature - ln;
                }
            }
            __syncthreads();
        } else if (p.parts > 1) {
            cluster_sync_all();              // the sums have been read
        }
    }
}

struct LogProbsGrad {
    int64_t ldz, ldg, M;
    int V, parts;
    float c, temperature;
    const int64_t* tokens;
    const float *lse, *glogp, *entropy, *gentropy;
    int* status;
};
// gz = p (a + b (ln p + H)) + (v is the token) glogp / T,  a = -glogp / T,  b = -gentropy / T
template <class T, bool ENTROPY>
__global__ void __launch_bounds__(kThreads) logprobs_grad_kernel(const T* z, T* gz, const LogProbsGrad p) {
    constexpr int N = Vec<T>::N;
    const int64_t m = blockIdx.x / p.parts;
    const Row<T> row(z + m * p.ldz, p.V, int(blockIdx.x - m * p.parts), p.parts);
    T* const g = gz + m * p.ldg;
    int64_t token = p.tokens && p.glogp ? p.tokens[m] : -1;
    if (token >= p.V) {
        if (p.status && threadIdx.x == 0) atomicCAS(p.status, PATCH_OK, PATCH_ERR_SIZE);
        token = -1;
    }
    const float lse = p.lse[m], up = token >= 0 ? p.glogp[m] / p.temperature : 0.0f, b = ENTROPY ? -p.gentropy[m] / p.temperature : 0.0f;
    if (lse == -INFINITY || (up == 0.0f && b == 0.0f)) {           // nothing is asked of the row, or it has no distribution: zeros whatever it holds
        const float zero[N] = {};
        for (int v = row.first; v < row.count; v += row.step) row.store(g, v, zero);
        return;
    }
    const float base = lse * p.temperature, h = ENTROPY ? p.entropy[m] : 0.0f, a = -up;
    const int tv = token >= 0 ? int(token) / N : -1;
    constexpr float kLn2 = 0.693147180559945f;
    auto one = [&](int v, const Vec<T>& x) {
        float y[N];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            float e[2];
            un2(mul2(add2(x.pair(i), mk2(-base, -base)), mk2(p.c, p.c)), e[0], e[1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float q = ex2(e[j]);
                y[2 * i + j] = ENTROPY ? q * (a + b * fmaf(fmaxf(e[j], -1e30f), kLn2, h)) : q * a;
            }
        }
        if (v == tv) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (tv * N + i == token) y[i] += up;
        }
        row.store(g, v, y);
    };
    Batch<T> ahead;
    row.fetch(ahead, 0);
    row.each(ahead, [&](int b, const Batch<T>& x) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (row.at(b, u) < row.whole) one(row.at(b, u), x.v[u]);
    }, [](Batch<T>&) {});
    if (row.rest()) one(row.whole, row.load(row.whole));
}

struct Distill {
    int64_t ldz, ldg, M;
    int V, K, parts;
    float c, temperature;
    const int32_t* ids;
    const float* t;
    float* loss;
    float* stats;                            // [M][2]: ln sum exp of the row, ln p_rest
    const float* gloss;
    int* status;
};
// What a row's entries say: of thread i < K.
struct Entry {
    int id;                                  // -1: none
    float q, x;                              // teacher's probability; the student's logit
    float q_all;                             // of all entries with this id
    bool first;                              // no earlier entry has it
};
__device__ __forceinline__ float block_total(float x, Shared& sh) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5].m = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) x += sh.warp[w].m;
    __syncthreads();
    return x;
}
__device__ __forceinline__ float block_top(float x, Shared& sh) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, d));
    if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5].m = x;
    __syncthreads();
    x = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) x = fmaxf(x, sh.warp[w].m);
    __syncthreads();
    return x;
}
// The entries of row m.  q_sum: sum of the teacher's listed probabilities (1 or, with no entry, 0 where they are renormalised).
template <class T, bool REST>
__device__ __forceinline__ Entry entry_of(const Distill& p, int64_t m, const T* z, float& q_sum, Shared& sh) {
    Entry e = {-1, 0.0f, 0.0f, 0.0f, false};
    const int i = threadIdx.x;
    float t = -INFINITY;
    if (i < p.K) {
        const int id = p.ids[m * p.K + i];
        if (id >= p.V) {
            if (p.status) atomicCAS(p.status, PATCH_OK, PATCH_ERR_SIZE);
        } else if (id >= 0) {
            e.id = id;
            e.x = as_float(z[id]);
            t = p.t[m * p.K + i];
        }
    }
    if (REST) {
        e.q = e.id >= 0 ? expf(t) : 0.0f;
        q_sum = block_total(e.q, sh);
    } else {
        const float top = block_top(t, sh);
        const float w = e.id < 0 || t == -INFINITY ? 0.0f : expf(t - top);
        const float sum = block_total(w, sh);
        e.q = sum == 0.0f ? 0.0f : w / sum;
        q_sum = sum == 0.0f ? 0.0f : 1.0f;
    }
    if (i < p.K) {
        sh.id[i] = e.id;
        sh.value[i] = e.q;
    }
    __syncthreads();
    if (e.id >= 0) {
        e.first = true;
        for (int j = 0; j < p.K; ++j)
            if (sh.id[j] == e.id) {
                e.q_all += sh.value[j];
                if (j < i) e.first = false;
            }
    }
    __syncthreads();                         // the lists may be written again
    return e;
}
// Gradient of a row's part: w_v (c p_rest - q_rest) g / T for elements that are not listed, w_v = 2^((x - base) c) / rest_s (all
// elements where REST is false: p_v g / T), then the listed ones, which need the barrier.
template <class T, class Next>
__device__ __forceinline__ void write_gradient(const Row<T>& row, Batch<T>& ahead, T* g, float base, float c, float factor, const Entry& e, float listed, int parts,
                                               int part, Next&& next) {
    constexpr int N = Vec<T>::N;
    auto one = [&](int v, const Vec<T>& x) {
        float y[N];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            float a, b;
            un2(mul2(add2(x.pair(i), mk2(-base, -base)), mk2(c, c)), a, b);
            un2(mul2(mk2(ex2(a), ex2(b)), mk2(factor, factor)), y[2 * i], y[2 * i + 1]);
        }
        row.store(g, v, y);
    };
    row.each(ahead, [&](int b, const Batch<T>& x) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (row.at(b, u) < row.whole) one(row.at(b, u), x.v[u]);
    }, next);
    if (row.rest()) one(row.whole, row.load(row.whole));
    __syncthreads();
    if (e.first && (e.id / N / kThreads) % parts == part) g[e.id] = rounded<T>(listed);
}
template <class T>
__device__ __forceinline__ void write_zeros(const Row<T>& row, T* g) {
    const float zero[Vec<T>::N] = {};
    for (int v = row.first; v < row.count; v += row.step) row.store(g, v, zero);
}

template <class T, bool REST, bool GRAD>
__global__ void __launch_bounds__(kThreads, kPerSm) distill_kernel(const T* z, T* gz, const Distill p) {
    __shared__ Shared sh;
    extern __shared__ uint32_t bits[];       // REST: a bit per element, set where it is listed
    const int part = p.parts > 1 ? int(cluster_ctarank()) : 0;
    if (REST) {
        for (int i = threadIdx.x; i < (p.V + 31) / 32; i += kThreads) bits[i] = 0u;
        __syncthreads();
    }
    const int64_t rows = gridDim.x / p.parts;
    Batch<T> ahead;
    if (int64_t m = blockIdx.x / p.parts; m < p.M) Row<T>(z + m * p.ldz, p.V, part, p.parts).fetch(ahead, 0);
    for (int64_t m = blockIdx.x / p.parts; m < p.M; m += rows) {
        const Row<T> row(z + m * p.ldz, p.V, part, p.parts);
        auto next_row = [&](Batch<T>& x) {
            if (m + rows < p.M) Row<T>(z + (m + rows) * p.ldz, p.V, part, p.parts).fetch(x, 0);
        };
        float q_sum;
        const Entry e = entry_of<T, REST>(p, m, row.z, q_sum, sh);
        if (REST) {
            if (e.first) atomicOr(&bits[e.id >> 5], 1u << (e.id & 31));
            __syncthreads();
        }
        const Sums x = sum_up(scan_row<T, false, REST, false>(row, ahead, p.c, bits, Cells{}, [&](Batch<T>& y) {
                                  if (GRAD) row.fetch(y, 0); else next_row(y);
                              }), p.c, sh, p.parts);
        if (REST && e.first) atomicAnd(&bits[e.id >> 5], ~(1u << (e.id & 31)));       // read again only behind the next row's barriers
        // the sums over all elements, and which part of them is not listed
        Sums all = x;
        float p_rest = 1.0f, ln_rest = 0.0f;
        if (REST) {
            const float mine = e.first ? e.x : -INFINITY, top = block_top(mine, sh);
            const float nan = e.first && !(e.x == e.x) ? e.x : 0.0f;
            const Sums listed = {top, block_total(top > -INFINITY && e.first ? ex2((e.x - top) * p.c) : nan, sh), 0.0f};
            all = join(x, listed, p.c);
            const float p_listed = listed.m == -INFINITY ? listed.s : ex2((listed.m - all.m) * p.c) * listed.s / all.s;
            p_rest = x.m == -INFINITY ? x.s : ex2((x.m - all.m) * p.c) * x.s / all.s;
            // ln p_rest without what a difference of two logarithms loses where it is near 0, and where p_rest is below the numbers of fp32
            ln_rest = p_listed < 0.5f ? log1pf(-p_listed) : p_rest > 1e-30f ? logf(p_rest) : (x.m - all.m) / p.temperature + logf(x.s) - logf(all.s);
        }
        const bool none = all.m == -INFINITY && !(all.s != all.s);          // every element is -inf: no distribution
        const float ln = logf(all.s), base = all.m == -INFINITY ? 0.0f : all.m;
        const float q_rest = REST ? fmaxf(1.0f - q_sum, 0.0f) : 0.0f;
        const float lnp = none ? -INFINITY : (e.x - base) / p.temperature - ln;
        const float ce = block_total(e.q != 0.0f ? -e.q * lnp : 0.0f, sh);
        if (part == 0 && threadIdx.x == 0) {
            p.loss[m] = ce + (q_rest > 0.0f ? -q_rest * (none ? -INFINITY : ln_rest) : 0.0f);
            if (p.stats) { p.stats[2 * m] = none ? -INFINITY : base / p.temperature + ln; p.stats[2 * m + 1] = ln_rest; }
        }
        if (GRAD) {
            const float g = p.gloss ? p.gloss[m] / p.temperature : 1.0f / p.temperature;
            T* const to = gz + m * p.ldg;
            if (g == 0.0f || none) {
                write_zeros(row, to);
                next_row(ahead);
            } else {
                const float q_all = q_sum + q_rest, factor = x.s == 0.0f ? 0.0f : g * (q_all * p_rest - q_rest) / x.s;
                write_gradient(row, ahead, to, x.m == -INFINITY ? 0.0f : x.m, p.c, factor, e, g * (q_all * expf(lnp) - e.q_all), p.parts, part, next_row);
            }
        }
        if (p.parts > 1) cluster_sync_all(); else __syncthreads();
    }
}

template <class T, bool REST>
__global__ void __launch_bounds__(kThreads) distill_grad_kernel(const T* z, T* gz, const Distill p) {
    __shared__ Shared sh;
    const int64_t m = blockIdx.x / p.parts;
    const int part = int(blockIdx.x - m * p.parts);
    const Row<T> row(z + m * p.ldz, p.V, part, p.parts);
    T* const to = gz + m * p.ldg;
    float q_sum;
    const Entry e = entry_of<T, REST>(p, m, row.z, q_sum, sh);
    const float g = p.gloss ? p.gloss[m] / p.temperature : 1.0f / p.temperature, lse = p.stats[2 * m], ln_rest = REST ? p.stats[2 * m + 1] : 0.0f;
    if (g == 0.0f || lse == -INFINITY) {
        write_zeros(row, to);
        return;
    }
    const float q_rest = REST ? fmaxf(1.0f - q_sum, 0.0f) : 0.0f, q_all = q_sum + q_rest;
    const bool none = ln_rest == -INFINITY;                        // everything is listed, or masked
    Batch<T> ahead;
    row.fetch(ahead, 0);
    write_gradient(row, ahead, to, none ? 0.0f : (lse + ln_rest) * p.temperature, p.c, none ? 0.0f : g * (q_all * expf(ln_rest) - q_rest), e,
                   g * (q_all * expf(e.x / p.temperature - lse) - e.q_all), p.parts, part, [](Batch<T>&) {});
}

// CTAs that share a row.  Four CTAs fit an SM; a row is shared (and read by a cluster, which joins its sums in distributed shared memory) where
// rows alone would leave SMs empty, as long as every thread keeps a few vectors.
static int parts_of(int64_t M, int64_t vectors) {
    const int64_t room = kPerSm * int64_t(sm_count());
    int parts = 1;
    while (parts < kMaxParts && M * parts * 2 <= room && vectors >= int64_t(parts) * 2 * kThreads) parts *= 2;
    return parts;
}
// Parts of a row where nothing has to be joined.
static int64_t segments_of(int64_t vectors) {
    const int64_t n = (vectors + kThreads * kAhead * 2 - 1) / (kThreads * kAhead * 2);
    return n < 1 ? 1 : n;
}
template <class... A>
static int launch_rows(void (*kern)(A...), int64_t M, int parts, size_t smem, cudaStream_t s, A... args) {
    const int64_t most = (int64_t(sm_count()) * kPerSm) / parts, clusters = M < most ? M : most;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3(unsigned(clusters * parts), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {unsigned(parts), 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kern, args...) == cudaSuccess) return PATCH_OK;
    cudaGetLastError();                      // reported here, not by the next call
    return PATCH_ERR_CUDA;
}

template <class T, bool ENTROPY, bool TOP>
static int launch_logprobs(const T* z, LogProbs p, cudaStream_t s) {
    auto kern = logprobs_kernel<T, ENTROPY, TOP>;
    size_t smem = 0;
    if (TOP) {
        const int vectors = p.V / Vec<T>::N, batches = (vectors + p.parts * kThreads * kAhead - 1) / (p.parts * kThreads * kAhead);
        p.cell_shift = Cells::shift_of(batches);
        smem = kListBytes + size_t((batches + (1 << p.cell_shift) - 1) >> p.cell_shift) * kThreads * sizeof(float);
        static std::atomic<uint64_t> configured{0};
        if (int rc = allow_dynamic_smem(kern, uint32_t(kListBytes + kCells * kThreads * sizeof(float)), configured)) return rc;
    }
    return launch_rows(kern, p.M, p.parts, smem, s, z, p);
}
template <class T>
static int launch_logprobs(const void* Z, const LogProbs& p, cudaStream_t s) {
    const T* z = static_cast<const T*>(Z);
    if (p.k) return p.entropy ? launch_logprobs<T, true, true>(z, p, s) : launch_logprobs<T, false, true>(z, p, s);
    return p.entropy ? launch_logprobs<T, true, false>(z, p, s) : launch_logprobs<T, false, false>(z, p, s);
}

// ---- checks of arguments ----
static bool bad_type(int dtype) { return dtype != PATCH_LOGITS_BF16 && dtype != PATCH_LOGITS_F32; }
static int check_shape(int dtype, int64_t M, int64_t V, float temperature) {
    if (bad_type(dtype) || M < 0 || M > (int64_t(1) << 31) - 1 || V < 1 || V > kMaxV) return PATCH_ERR_SHAPE;
    const float c = 1.44269504f / temperature;
    if (!(temperature > 0.0f) || !isfinite(temperature) || !isfinite(c) || !(c > 0.0f)) return PATCH_ERR_SHAPE;
    return PATCH_OK;
}
static int check_rows(const void* p, int64_t ld, int64_t M, int64_t V) {
    if (!p) return PATCH_ERR_NULL;
    if (ld < V || ld % 8 || ld > (int64_t(1) << 61) / (M ? M : 1)) return PATCH_ERR_SHAPE;
    return aligned16(p) ? PATCH_OK : PATCH_ERR_ALIGN;
}
static bool misaligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

}  // namespace logits
}  // namespace patch

using namespace patch;
using namespace patch::logits;

extern "C" int patch_token_logprobs(const void* Z, int64_t ldz, int dtype, int64_t M, int64_t V, const int64_t* tokens, int k, float temperature,
                                    float* logp, float* entropy, float* lse, int32_t* top_ids, float* top_logp, int* status_dev, void* stream) {
    int rc = check_shape(dtype, M, V, temperature);
    if (rc) return rc;
    if (k < 0 || k > kMost || k > V) return PATCH_ERR_SHAPE;
    if (M == 0) return PATCH_OK;
    if ((rc = check_rows(Z, ldz, M, V))) return rc;
    if ((tokens != nullptr) != (logp != nullptr) || (k > 0 && (!top_ids || !top_logp))) return PATCH_ERR_NULL;
    if (!logp && !entropy && !lse && !k) return PATCH_ERR_NULL;    // nothing is asked for
    if (misaligned(tokens, 8) || misaligned(logp, 4) || misaligned(entropy, 4) || misaligned(lse, 4) || misaligned(top_ids, 4) || misaligned(top_logp, 4))
        return PATCH_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (sm_count() <= 0) return PATCH_ERR_CUDA;
    const int parts = parts_of(M, V / (dtype == PATCH_LOGITS_BF16 ? 8 : 4));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    LogProbs p = {ldz, M, int(V), k, parts, 0, 1.44269504f / temperature, temperature, tokens, logp, entropy, lse, top_logp, top_ids, status_dev};
    return dtype == PATCH_LOGITS_BF16 ? launch_logprobs<__nv_bfloat16>(Z, p, s) : launch_logprobs<float>(Z, p, s);
}

extern "C" int patch_token_logprobs_backward(const void* Z, int64_t ldz, int dtype, int64_t M, int64_t V, const int64_t* tokens, float temperature,
                                             const float* lse, const float* glogp, const float* entropy, const float* gentropy, void* gZ, int64_t ldg,
                                             int* status_dev, void* stream) {
    int rc = check_shape(dtype, M, V, temperature);
    if (rc) return rc;
    if (M == 0) return PATCH_OK;
    if ((rc = check_rows(Z, ldz, M, V)) || (rc = check_rows(gZ, ldg, M, V))) return rc;
    if (gZ == Z && ldg != ldz) return PATCH_ERR_SHAPE;
    if (!lse || (!glogp && !gentropy) || (glogp != nullptr && !tokens) || (gentropy != nullptr && !entropy)) return PATCH_ERR_NULL;
    if (misaligned(tokens, 8) || misaligned(lse, 4) || misaligned(glogp, 4) || misaligned(entropy, 4) || misaligned(gentropy, 4)) return PATCH_ERR_ALIGN;
    const int64_t parts = segments_of(V / (dtype == PATCH_LOGITS_BF16 ? 8 : 4));
    if (M * parts > 0x7FFFFFFF) return PATCH_ERR_SHAPE;
    if ((rc = check_device())) return rc;
    const LogProbsGrad p = {ldz, ldg, M, int(V), int(parts), 1.44269504f / temperature, temperature, tokens, lse, glogp, entropy, gentropy, status_dev};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const unsigned grid = unsigned(M * parts);
    if (dtype == PATCH_LOGITS_BF16) {
        const auto* z = static_cast<const __nv_bfloat16*>(Z);
        auto* g = static_cast<__nv_bfloat16*>(gZ);
        if (gentropy) logprobs_grad_kernel<__nv_bfloat16, true><<<grid, kThreads, 0, s>>>(z, g, p);
        else logprobs_grad_kernel<__nv_bfloat16, false><<<grid, kThreads, 0, s>>>(z, g, p);
    } else {
        const auto* z = static_cast<const float*>(Z);
        auto* g = static_cast<float*>(gZ);
        if (gentropy) logprobs_grad_kernel<float, true><<<grid, kThreads, 0, s>>>(z, g, p);
        else logprobs_grad_kernel<float, false><<<grid, kThreads, 0, s>>>(z, g, p);
    }
    return cudaGetLastError() == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}

namespace {
int check_distill(const void* Z, int64_t ldz, int dtype, int64_t M, int64_t V, const int32_t* ids, const float* t, int K, float temperature, int flags) {
    int rc = check_shape(dtype, M, V, temperature);
    if (rc) return rc;
    if (K < 1 || K > kMost || (flags & ~PATCH_DISTILL_REST)) return PATCH_ERR_SHAPE;
    if (M == 0) return PATCH_OK;
    if ((rc = check_rows(Z, ldz, M, V))) return rc;
    if (!ids || !t) return PATCH_ERR_NULL;
    return misaligned(ids, 4) || misaligned(t, 4) ? PATCH_ERR_ALIGN : PATCH_OK;
}
template <class T, bool REST, bool GRAD>
int launch_distill(const T* z, T* g, const Distill& p, cudaStream_t s) {
    const size_t smem = REST ? size_t(p.V + 31) / 32 * 4 : 0;
    auto kern = distill_kernel<T, REST, GRAD>;
    static std::atomic<uint64_t> configured{0};
    if (REST) {
        if (int rc = allow_dynamic_smem(kern, uint32_t(kMaxV / 8), configured)) return rc;
    }
    return launch_rows(kern, p.M, p.parts, smem, s, z, g, p);
}
template <class T>
int launch_distill(const void* Z, void* gZ, const Distill& p, bool rest, cudaStream_t s) {
    const T* z = static_cast<const T*>(Z);
    T* g = static_cast<T*>(gZ);
    if (rest) return g ? launch_distill<T, true, true>(z, g, p, s) : launch_distill<T, true, false>(z, g, p, s);
    return g ? launch_distill<T, false, true>(z, g, p, s) : launch_distill<T, false, false>(z, g, p, s);
}
template <class T>
int launch_distill_grad(const void* Z, void* gZ, const Distill& p, bool rest, cudaStream_t s) {
    const T* z = static_cast<const T*>(Z);
    T* g = static_cast<T*>(gZ);
    const unsigned grid = unsigned(p.M * p.parts);
    if (rest) distill_grad_kernel<T, true><<<grid, kThreads, 0, s>>>(z, g, p);
    else distill_grad_kernel<T, false><<<grid, kThreads, 0, s>>>(z, g, p);
    return cudaGetLastError() == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}
}  // namespace

extern "C" int patch_distill_loss(const void* Z, int64_t ldz, int dtype, int64_t M, int64_t V, const int32_t* ids, const float* t, int K,
                                  float temperature, int flags, float* loss, float* stats, const float* gloss, void* gZ, int64_t ldg,
                                  int* status_dev, void* stream) {
    int rc = check_distill(Z, ldz, dtype, M, V, ids, t, K, temperature, flags);
    if (rc || M == 0) return rc;
    if (!loss) return PATCH_ERR_NULL;
    if (gZ && (rc = check_rows(gZ, ldg, M, V))) return rc;
    if (gZ == Z && ldg != ldz) return PATCH_ERR_SHAPE;
    if (misaligned(loss, 4) || misaligned(stats, 4) || misaligned(gloss, 4)) return PATCH_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (sm_count() <= 0) return PATCH_ERR_CUDA;
    const int parts = parts_of(M, V / (dtype == PATCH_LOGITS_BF16 ? 8 : 4));
    const Distill p = {ldz, ldg, M, int(V), K, parts, 1.44269504f / temperature, temperature, ids, t, loss, stats, gloss, status_dev};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool rest = flags & PATCH_DISTILL_REST;
    return dtype == PATCH_LOGITS_BF16 ? launch_distill<__nv_bfloat16>(Z, gZ, p, rest, s) : launch_distill<float>(Z, gZ, p, rest, s);
}

extern "C" int patch_distill_loss_backward(const void* Z, int64_t ldz, int dtype, int64_t M, int64_t V, const int32_t* ids, const float* t, int K,
                                           float temperature, int flags, const float* stats, const float* gloss, void* gZ, int64_t ldg,
                                           int* status_dev, void* stream) {
    int rc = check_distill(Z, ldz, dtype, M, V, ids, t, K, temperature, flags);
    if (rc || M == 0) return rc;
    if (!stats) return PATCH_ERR_NULL;
    if ((rc = check_rows(gZ, ldg, M, V))) return rc;
    if (gZ == Z) return PATCH_ERR_SHAPE;                           // parts of a row read listed logits that others would have overwritten
    if (misaligned(stats, 4) || misaligned(gloss, 4)) return PATCH_ERR_ALIGN;
    const int64_t parts = segments_of(V / (dtype == PATCH_LOGITS_BF16 ? 8 : 4));
    if (M * parts > 0x7FFFFFFF) return PATCH_ERR_SHAPE;
    if ((rc = check_device())) return rc;
    const Distill p = {ldz, ldg, M, int(V), K, int(parts), 1.44269504f / temperature, temperature, ids, t, nullptr, const_cast<float*>(stats), gloss, status_dev};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool rest = flags & PATCH_DISTILL_REST;
    return dtype == PATCH_LOGITS_BF16 ? launch_distill_grad<__nv_bfloat16>(Z, gZ, p, rest, s) : launch_distill_grad<float>(Z, gZ, p, rest, s);
}
