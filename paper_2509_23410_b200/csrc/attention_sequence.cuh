// Shared by the kernels of the attention within packed sequences: the problem, and which rows a CTA owns.
#pragma once
#include <algorithm>
#include "attention_tmem.cuh"

namespace patch {
namespace seq {

struct Problem {
    const __nv_bfloat16 *q, *k, *v, *o, *go;
    int64_t ldq, ldk, ldv, ldo, ldgo;
    const int32_t* starts;
    int B, M, Hq, Hkv, G;
    float scale, scale_log2;
    int* status;
};

// SMs of the GPU that this is built for, a CTA each.  A constant, as the order of the gradient's sums goes by it (key_splits), which depends on the arguments alone, and as
// the workspace's size is asked for without a device.
constexpr int kSms = 148;

// Key heads whose items (`items` of a head) are taken together, the largest over all sequences first: what their items read again and again (`bytes` of a head)
// stays in L2, whose halves hold copies of what both read, and the last group has items enough, four an SM, to end together.  (gq of four
// sequences of 2048, all 32 heads at once, 134 MB of keys and values: 226 us, three groups 200.  Groups too small for the latter: gk and
// gv of nine sequences, 4001 tokens, 32/8 heads, 122 us, all at once 98.)
inline int heads_at_once(int heads, int64_t bytes, int64_t items) {
    const int64_t most = std::max((int64_t(48) << 20) / bytes, (4 * kSms + items - 1) / items), groups = most >= heads ? 1 : (heads + most - 1) / most;
    return int((heads + groups - 1) / groups);
}
// Tiles of all sequences in one line: sequence b's first tile is number starts[b] / rows + b, and it has at most as many as lie before
// the next one's first.
struct Tile { int begin, end, first; };      // rows of the sequence; the tile's first row, counted from `begin` (-1: no tile)
__host__ __device__ __forceinline__ int64_t most_tiles(int64_t M, int64_t B, int rows) { return M / rows + B; }
__device__ __forceinline__ int clamped(const Problem& p, int b) { return min(max(p.starts[b], 0), p.M); }
// By one warp, all lanes: a search in 32 parts, so that up to 31 sequences take one look and thousands three.
template <int ROWS>
__device__ __forceinline__ Tile tile_of(const Problem& p, int slot) {
    const int lane = threadIdx.x & 31;
    int lo = -1, hi = p.B;                   // the last sequence whose first tile is at or before `slot` is lo or lies between the two
    while (hi - lo > 1) {
        const int each = (hi - lo + 31) / 32, b = lo + 1 + lane * each;
        const bool before = b < hi && clamped(p, b) / ROWS + b <= slot;
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, before));  // lanes 0 .. n - 1, where the starts ascend
        const int last = n ? lo + 1 + (n - 1) * each : lo, next = lo + 1 + n * each;
        hi = n < 32 && next < hi ? next : hi;
        lo = last;
    }
    Tile t = {0, 0, -1};
    if (lo < 0) return t;
    t.begin = clamped(p, lo);
    t.end = max(clamped(p, lo + 1), t.begin);
    const int first = (slot - (t.begin / ROWS + lo)) * ROWS;
    if (first >= 0 && first < t.end - t.begin) t.first = first;
    return t;
}
// The items in the order in which CTAs take them, those with most work first, so that no CTA begins a long one when the others are about to end.  An item's
// work grows with the tiles up to its own (OF_KEYS: from its own to the sequence's end): with up to 128 sequences (lengths in registers, four to
// a lane) a head's items come by their size over all sequences.  With more of them each sequence is a small part of the whole, and they come one behind
// the other, the largest items of each first.  `heads` of them come in groups of `group` (heads_at_once).  By one warp, all lanes.
template <int ROWS, bool OF_KEYS>
struct Order {
    static constexpr int kMost = 128;
    const Problem& p;
    const int heads, group;
    int n[kMost / 32], most = 0;             // tiles of sequence lane + 32 i; the longest sequence's
    __device__ __forceinline__ Order(const Problem& p_, int heads_, int group_) : p(p_), heads(heads_), group(group_) {
#pragma unroll
        for (int i = 0; i < kMost / 32; ++i) {
            const int b = (threadIdx.x & 31) + 32 * i;
            n[i] = p.B <= kMost && b < p.B ? (max(clamped(p, b + 1) - clamped(p, b), 0) + ROWS - 1) / ROWS : 0;
            most = max(most, n[i]);
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
    }
    // items of x or more tiles
    __device__ __forceinline__ int items(int x) const {
        int c = 0;
#pragma unroll
        for (int i = 0; i < kMost / 32; ++i) c += max(n[i] - x + 1, 0);
        return __reduce_add_sync(0xFFFFFFFFu, c);
    }
    __device__ __forceinline__ Tile take(unsigned at, int& head) const {
        const unsigned tiles = unsigned(most_tiles(p.M, p.B, ROWS)), first = at / (tiles * group) * group, here = min(unsigned(group), unsigned(heads) - first);
        const int number = int((at - tiles * first) / here);
        head = int(first + (at - tiles * first) % here);
        if (p.B > kMost) return tile_of<ROWS>(p, OF_KEYS ? number : int(tiles) - 1 - number);
        Tile t = {0, 0, -1};
        if (number >= items(1)) return t;
        int lo = 1, hi = most + 1, before = 0;       // items(lo) > number >= items(hi) = before
        while (hi - lo > 1) {
            const int x = (lo + hi) / 2, c = items(x);
            if (c > number) lo = x;
            else hi = x, before = c;
        }
        int k = number - before;                     // the k-th sequence of `lo` tiles or more
#pragma unroll
        for (int i = 0; i < kMost / 32; ++i) {
            const unsigned has = __ballot_sync(0xFFFFFFFFu, n[i] >= lo);
            if (k >= 0 && k < __popc(has)) {
                const unsigned lane = threadIdx.x & 31, own = __ballot_sync(0xFFFFFFFFu, ((has >> lane) & 1u) && __popc(has & ((1u << lane) - 1u)) == k);
                const int b = 32 * i + __ffs(own) - 1;
                t.begin = clamped(p, b);
                t.end = max(clamped(p, b + 1), t.begin);
                t.first = (OF_KEYS ? (t.end - t.begin + ROWS - 1) / ROWS - lo : lo - 1) * ROWS;
            }
            k -= __popc(has);
        }
        return t;
    }
};
// starts out of order or out of range are reported (every tile stays within the rows all the same)
__device__ __forceinline__ void check_starts(const Problem& p, int thread, int threads) {
    if (!p.status) return;
    bool bad = false;
#pragma unroll 4
    for (int b = thread; b <= p.B; b += threads) bad |= p.starts[b] < 0 || p.starts[b] > p.M || (b && p.starts[b] < p.starts[b - 1]);
    if (bad) atomicCAS(p.status, PATCH_OK, PATCH_ERR_SIZE);
}

// A CTA that has started takes the place of one that has not: asked for ahead, answered in shared memory.  Launch order is kept, and what is left
// over is balanced by itself, whatever the lengths in device memory are.  One question at a time; its answer is waited for before the CTA ends.
__device__ __forceinline__ void ask_for_next(uint4* answer, uint64_t* bar) {
    mbar_expect_tx(smem_u32(bar), 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)), "r"(smem_u32(bar)) : "memory");
}
// the CTA number taken over; false: none is left (do not ask again)
__device__ __forceinline__ bool answered(const uint4* answer, unsigned& next) {
    uint32_t there;
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b128 r;\n\tld.shared.b128 r, [%2];\n\tclusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
                 "selp.u32 %1, 1, 0, p;\n\tmov.u32 %0, 0;\n\t@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%0, _, _, _}, r;\n\t}"
                 : "=r"(next), "=r"(there) : "r"(smem_u32(answer)) : "memory");
    attn::blk::fence_async_shared();                    // read before the next answer is written
    return there != 0;
}

// Behind the CTA's last barrier, before its tensor memory goes: where a wait was given up, by whichever role, copies, answers and products may still be on their way.
__device__ __forceinline__ void let_land(volatile int* abort_flag) {
    if (!*abort_flag) return;
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < kDrainLimitNs) {}
}

constexpr int kTileRows = 128;               // of a tile in shared memory: [64-element half][row][128 bytes, swizzled]
template <int D> constexpr uint32_t kTileBytes = kTileRows * D * 2;

// The producer warp's side of a ring of tiles.  All lanes call together.
template <int D, int RING>
struct Loader {
    uint8_t* smem;                           // the ring
    uint64_t *full, *empty, *tail;           // tail: of tiles that need work behind the copy, by stage
    volatile int* abort_flag;
    int* status;
    int stage = 0, issued = 0;
    uint32_t phase = 0;
    bool ok = true;

    __device__ __forceinline__ Loader(uint8_t* smem_, uint64_t* full_, uint64_t* empty_, uint64_t* tail_, volatile int* abort_, int* status_)
        : smem(smem_), full(full_), empty(empty_), tail(tail_), abort_flag(abort_), status(status_) {}
#ifdef PATCH_FAULT_INJECTION
    uint32_t inject = 0u;                    // test build: a status word holding kInjectMagic + kernel makes CTA 0 announce sixteen bytes more than its first
    __device__ __forceinline__ void heed(int kernel) {             // stage will ever receive
        if (blockIdx.x != 0 || !status || *status != kInjectMagic + kernel) return;
        inject = 16u;
        __syncwarp();
        if ((threadIdx.x & 31) == 0) *status = PATCH_OK;
    }
#else
    static constexpr uint32_t inject = 0u;
    __device__ __forceinline__ void heed(int) {}
#endif
    __device__ __forceinline__ void wait(uint64_t& bar, uint32_t parity) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bar), parity, abort_flag, status)) && ok;
    }
    // 128 rows from `row` on of one head into the next stage; `left` < 128: rows from there on become zeros (by Mender, which hands the tile on)
    __device__ __forceinline__ void load(const CUtensorMap* map, int row, int chunk, int left, uint64_t policy) {
        if (issued >= RING) wait(empty[stage], phase ^ 1u);
        if (!ok) return;
        if ((threadIdx.x & 31) == 0) {
            const uint32_t bar = smem_u32(left < kTileRows ? &tail[stage] : &full[stage]);
            mbar_expect_tx(bar, kTileBytes<D> + (issued == 0 ? inject : 0u));
            tma_tile_load_3d(smem_u32(smem) + stage * kTileBytes<D>, map, 0, row, chunk, bar, policy);
        }
        __syncwarp();
        ++issued;
        if (++stage == RING) { stage = 0; phase ^= 1u; }
    }
};
// A warp that follows the loads and puts zeros behind a sequence's end: a probability of 0 times whatever lies there is not always 0.  (The producer itself,
// waiting for each such copy, held up short sequences by 3 us.)  It mends the even or the odd numbers, of the two operands of a tile: the forward kernel has one
// for its values, the kernel of gq one for its keys, and that of gk and gv one each for queries and gradients.
template <int D, int RING>
struct Mender {
    uint8_t* smem;
    uint64_t *full, *tail;
    volatile int* abort_flag;
    int* status;
    const int which;                         // 0 or 1
    int number = 0;                          // of loads so far
    uint32_t phases = 0;                     // of the tail barriers, by stage
    bool ok = true;
    // the next load of the producer, with its `left`
    __device__ __forceinline__ void next(int left) {
        const int i = number++, stage = i % RING;
        if (left >= kTileRows || !ok) return;
        phases ^= 1u << stage;               // (those of the other numbers count too: an odd ring gives a stage both)
        if ((i & 1) != which) return;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspended(smem_u32(&tail[stage]), ~(phases >> stage) & 1u, abort_flag, status));
        if (!ok) return;
        uint8_t* const tile = smem + stage * kTileBytes<D>;
        const int lane = threadIdx.x & 31;
        for (int j = left * (D / 8) + lane; j < kTileRows * (D / 8); j += 32) {
            const int r = j / (D / 8), c = j - r * (D / 8);
            *reinterpret_cast<uint4*>(tile + (c >> 3) * (kTileRows * 128) + r * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        attn::blk::fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&full[stage]));
    }
};

// 32 rows (a warp's, lane = row) of COLS fp32 columns of TMEM, times `f` of the lane's row, as bf16 (or as they are, F32) into rows [row, end).  Four
// neighbouring lanes exchange their 64 bytes, so that a store writes 64 consecutive bytes of eight rows (a lane that writes its own row alone touches 32 lines
// with every 16 bytes: 4 000 cycles of the load-store unit for an item of 256 x 128, against 1 000).
template <int COLS, bool F32 = false>
__device__ __forceinline__ void store_rows(uint32_t t, void* to, int64_t ld, int row, int end, float f) {
    constexpr int kStep = F32 ? 16 : 32, kBytes = F32 ? 4 : 2;     // columns of 64 bytes
    const int lane = threadIdx.x & 31, sub = lane & 3;
    if (row >= end) return;                  // none of them
#pragma unroll 2
    for (int q = 0; q < COLS / kStep; ++q) {
        uint32_t v[kStep], w[4][4];                                // w: 16-byte chunks of the lane's row, then chunk `sub` of four rows
        attn::blk::load_quarter(t + uint32_t(kStep) * q, v);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            if constexpr (F32) w[c >> 2][c & 3] = __float_as_uint(__uint_as_float(v[c]) * f);
            else w[c >> 2][c & 3] = attn::pack2(__uint_as_float(v[2 * c]) * f, __uint_as_float(v[2 * c + 1]) * f);
        }
#pragma unroll
        for (int bit = 1; bit <= 2; bit <<= 1) {
            const bool high = sub & bit;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (c & bit) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, high ? w[c][i] : w[c | bit][i], bit);
                    if (high) w[c][i] = got; else w[c | bit][i] = got;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = row + (lane & ~3) + j;
            if (r < end) *reinterpret_cast<uint4*>(static_cast<char*>(to) + int64_t(r) * ld * kBytes + 64 * q + 16 * sub) = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
        }
    }
}

int launch_forward(const Problem& p, int D, __nv_bfloat16* o, int64_t ldo, float* lse, cudaStream_t s);
// Into how many parts the query heads of a key head are cut for gk and gv: 1, or a divisor of the group where the items were few.  By the sizes
// alone (sequences may leave fewer tiles than M and B allow for).
int key_splits(int64_t M, int64_t B, int Hkv, int G);
// stats: [Hq][M] of scratch; parts: [split][2][M][Hkv][D] where there are several
int launch_backward(const Problem& p, int D, const float* lse, float2* stats, float* parts, int splits, __nv_bfloat16* gq, int64_t ldgq, __nv_bfloat16* gk, int64_t ldgk, __nv_bfloat16* gv,
                    int64_t ldgv, cudaStream_t s);

}  // namespace seq
}  // namespace patch
