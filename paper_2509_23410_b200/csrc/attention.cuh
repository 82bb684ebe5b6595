// Shared by the attention kernels: the problem as the kernels see it, the work list (which CTA owns which tiles of which
// item) and the partial results that the joining kernel adds up.
//
// Work list.  An item is a set of query rows of one key head that read the same keys: rows of the batch against the shared
// prefix, or one sequence's rows against its own keys.  An item's keys are cut into tiles; all tiles of all items,
// item after item, form one line of U units, and every CTA owns a stretch of it (of equal length, where all run at once): the same amount of
// work whatever the lengths are, at the price of items that several CTAs share.  An item also has a few units without a tile, which
// stand for what it costs by itself.  Each CTA writes one partial result (running maximum, sum and unnormalised output, fp32)
// per item it has a share of.  Along the line the pair (item, CTA) changes one step at a time, so item + c numbers the partial
// results; the CTAs with an item's first and last tile note their numbers for the joining kernel.
#pragma once
#include "sm100_ptx.cuh"
#include "softmax_rule.cuh"

namespace patch {
namespace attn {

constexpr int kMaxBatch = 2048;
constexpr int kMaxSms = 160;                  // sizes the workspace

struct Problem {
    const __nv_bfloat16* Q;
    int64_t ldq;
    int B, T, Hkv, G;                         // G query heads per key head
    const int32_t* prefix_pages;
    int prefix_len;
    const int32_t* table;
    int64_t ld_table;
    const int32_t* lens;
    int shift, num_pages;                     // log2(page_size)
    float scale_log2;                         // scale * log2(e): 2^(s scale_log2) = e^(s scale)
    int* status;
    uint32_t g_mul;                           // ceil(2^32 / G) where the product below is exact for every row, else 0
    // token of row r of a key head's rows; one multiplication instead of a division's thirty instructions
    __device__ __forceinline__ int token(int r) const { return g_mul ? int(__umulhi(uint32_t(r), g_mul)) : G == 1 ? r : r / G; }
};

// The decode kernel (attention_decode_sm100.cu) takes rows in blocks of kDecodeRows, the block kernel (attention_block_sm100.cu) in
// blocks of kBlockRows.
constexpr int kDecodeRows = 16, kBlockRows = 128;

// The line of units of one kernel.  Blocks of query rows are items of their own.
struct Line {
    int blocks_p, blocks_s;                   // row blocks per key head: prefix items, suffix items (0: none in this kernel)
    int tiles_p;                              // key tiles of a prefix item
    int cost;                                 // units of an item beside its tiles
    int tile_log2;                            // keys of a tile
};
// Tiles of one row block against a sequence's `keys` keys.  STEPS: up to the last key that its last row sees.  In a long prompt, whose
// blocks see ever more of it, half of all tiles would be masked out: 2048 tokens of the 7B shape 152 us -> 119, 8192 tokens with
// 8 key heads of 4 rows 1562 -> 953.  Up to kMostLevelTokens all blocks count as seeing all keys: 512 tokens 30.0 us against 30.3,
// 300 tokens 31.6 against 32.6.  A block that sees nothing keeps one tile, so that every item has a part.  (Decided at compile time:
// asked of a variable it cost decode steps, which never need it, 1 to 5 us.)
constexpr int kMostLevelTokens = 512;
template <bool STEPS> __device__ __forceinline__ int tiles_of(const Problem& p, const Line& w, int keys, int block) {
    if (STEPS && keys) {
        const int last = min((block + 1) * kBlockRows, p.T * p.G) - 1;
        keys = max(1, keys - (p.T - 1 - p.token(last)));
    }
    return (keys >> w.tile_log2) + ((keys & ((1 << w.tile_log2) - 1)) != 0);
}
// units of one key head and sequence
template <bool STEPS> __device__ __forceinline__ int head_units(const Problem& p, const Line& w, int keys) {
    if (!keys) return 0;
    if (!STEPS) return (tiles_of<STEPS>(p, w, keys, 0) + w.cost) * w.blocks_s;
    int sum = 0;
    for (int i = 0; i < w.blocks_s; ++i) sum += tiles_of<STEPS>(p, w, keys, i) + w.cost;
    return sum;
}
// Where partial results go, of prefix items and of suffix items.
struct Parts {
    float* o;                                 // [slot][rows][D], see `quarters`
    float2* ml;                               // [slot][rows]: maximum of the scores (unscaled), sum
    int2* span;                               // [item]: first and last CTA with a share of it
    int rows;                                 // rows of a slot
    int quarters;                             // 0: rows of D; 1: by quarters of the columns, [slot][4][rows][D / 4], 16-byte chunk c of
                                              // row r at chunk c ^ (r & (D / 16 - 1)) (how the block kernel's shared memory holds them)
    template <int D> __device__ __forceinline__ int64_t chunk(int64_t slot, int r, int c) const {       // in elements, chunk c of row r
        if (!quarters) return (slot * rows + r) * D + 4 * c;
        const int q = c / (D / 16), cc = (c & (D / 16 - 1)) ^ (r & (D / 16 - 1));
        return ((slot * 4 + q) * rows + r) * (D / 4) + 4 * cc;
    }
};
struct Results { Parts p, s; };

// len -> clamped length of sequence b's own keys
__device__ __forceinline__ int suffix_len(const Problem& p, int b) {
    const int64_t n = p.lens[b], most = p.ld_table << p.shift;
    if (n < 0 || n > most) {
        if (p.status) atomicCAS(p.status, PATCH_OK, PATCH_ERR_SIZE);
        return n < 0 ? 0 : int(most < 0x7FFFFFFF ? most : 0x7FFFFFFF);
    }
    return int(n);
}

// Executed by one warp: where the kernel has suffix items, units before each sequence (of one key head) and the clamped
// lengths (unless `lens` is null).  Returns the batch's own keys.  (Every CTA waits for this: four groups of lengths are on their way at
// once.)
template <bool STEPS> __device__ __forceinline__ int64_t lay_out(const Problem& p, const Line& w, int* cum, int* lens) {
    constexpr int kAtOnce = 4;
    const int lane = threadIdx.x & 31;
    int before = 0;
    int64_t keys = 0;
    for (int g0 = 0; g0 < p.B; g0 += 32 * kAtOnce) {
        int n[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) n[i] = g0 + 32 * i + lane < p.B ? suffix_len(p, g0 + 32 * i + lane) : 0;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int b = g0 + 32 * i + lane;
            keys += n[i];
            if (!w.blocks_s || g0 + 32 * i >= p.B) continue;
            int t = head_units<STEPS>(p, w, n[i]);
            if (lens && b < p.B) lens[b] = n[i];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xFFFFFFFFu, t, d);
                if (lane >= d) t += o;
            }
            if (b < p.B) cum[b + 1] = before + t;
            before += __shfl_sync(0xFFFFFFFFu, t, 31);
        }
    }
    if (lane == 0 && w.blocks_s) cum[0] = 0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) keys += __shfl_xor_sync(0xFFFFFFFFu, keys, d);
    return keys;
}

// Units are counted in 32 bits (the host refuses what would not fit): a 64-bit division costs every CTA hundreds of cycles.
__device__ __forceinline__ int prefix_units(const Line& w, int Hkv) { return Hkv * w.blocks_p * (w.tiles_p + w.cost); }
__device__ __forceinline__ int total_units(const Line& w, const Problem& p, const int* cum) {
    return prefix_units(w, p.Hkv) + (w.blocks_s ? cum[p.B] * p.Hkv : 0);
}
// First unit of CTA c's share of U units among n <= U CTAs: equal shares where all CTAs run at once; where they take turns on whatever
// SMs another kernel leaves free (`turns` = 1 / (4 n^2) then, else 0), shares that shrink from 7/4 to 1/4 of the average, so that
// the last ones to run are short.  No share is empty: a CTA between an item's first and last one has a tile of it.
__device__ __forceinline__ int share_start(int U, int c, int n, double turns) {
    if (turns == 0.0 || U < 8 * n) {              // (also where the launch has more CTAs than there is work for)
        const int each = U / n, more = U - each * n;
        return c * each + min(c, more);
    }
    return c == n ? U : int(double(U) * (double(c) * double(7 * n - 3 * c)) * turns);
}

// One CTA's share of the line, item by item.
template <bool STEPS> struct Share {
    const Problem& p;
    const Line& w;
    const int* cum;
    const int* len;                           // null: looked up where they came from
    int b, kvh, block, item;                  // b < 0: the prefix; item: number among the prefix's or the suffixes' items
    int tiles, keys;
    int t0, t1;                               // the share's tiles of the item
    int u, u1;                                // the item's first unit, the share's end

    __device__ __forceinline__ Share(const Problem& p_, const Line& w_, const int* cum_, const int* len_)
        : p(p_), w(w_), cum(cum_), len(len_), b(-1), kvh(0), block(0), item(0), tiles(0), keys(0), t0(0), t1(0), u(0), u1(0) {}
    __device__ __forceinline__ void operator=(const Share& o) {
        b = o.b; kvh = o.kvh; block = o.block; item = o.item; tiles = o.tiles; keys = o.keys; t0 = o.t0; t1 = o.t1; u = o.u; u1 = o.u1;
    }
    __device__ __forceinline__ void at_sequence(int b_) {
        b = b_;
        keys = len ? len[b] : suffix_len(p, b);
        tiles = tiles_of<STEPS>(p, w, keys, 0);
    }
    __device__ __forceinline__ void clip() { t1 = min(tiles, u1 - u - w.cost); }
    // to the first item of units [u0, end) that has a tile among them; false: none
    __device__ __forceinline__ bool start(int u0, int end) {
        if (u0 >= end) return false;
        const int before = prefix_units(w, p.Hkv);
        int place;                            // of u0 among its item's units
        if (u0 < before) {
            const int each = w.tiles_p + w.cost;
            item = u0 / each;
            b = -1;
            kvh = item / w.blocks_p;
            block = item - kvh * w.blocks_p;
            tiles = w.tiles_p;
            keys = p.prefix_len;
            place = u0 - item * each;
        } else {
            const int v = u0 - before, q = v / p.Hkv;
            int lo = 0, hi = p.B;             // the sequence with cum[lo] <= q < cum[lo + 1]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (cum[mid] <= q) lo = mid; else hi = mid;
            }
            at_sequence(lo);
            const int r = v - cum[lo] * p.Hkv, head = cum[lo + 1] - cum[lo];
            kvh = r / head;
            place = r - kvh * head;
            if (!STEPS) {
                block = place / (tiles + w.cost);
                place -= block * (tiles + w.cost);
            } else {
                for (block = 0; place >= tiles + w.cost; tiles = tiles_of<STEPS>(p, w, keys, ++block)) place -= tiles + w.cost;
            }
            item = (lo * p.Hkv + kvh) * w.blocks_s + block;
        }
        u = u0 - place;
        u1 = end;
        t0 = place < w.cost ? 0 : place - w.cost;
        clip();
        return t0 < t1 || next();
    }
    // to the next item with a tile in the share; false: none
    __device__ __forceinline__ bool next() {
        u += tiles + w.cost;
        if (u + w.cost >= u1) return false;
        ++item;
        if (++block == (b < 0 ? w.blocks_p : w.blocks_s)) {
            block = 0;
            if (++kvh == p.Hkv) {
                kvh = 0;
                int n = b + 1;                // u < u1: there is a sequence with tiles
                while (n + 1 < p.B && cum[n + 1] == cum[n]) ++n;
                item = n * p.Hkv * w.blocks_s;
                at_sequence(n);
            }
        }
        if (b >= 0 && STEPS) tiles = tiles_of<STEPS>(p, w, keys, block);
        t0 = 0;
        clip();
        return true;
    }
    __device__ __forceinline__ void note(const Results& to, int cta) const {
        int2* span = (b < 0 ? to.p.span : to.s.span) + item;
        if (t0 == 0) span->x = cta;
        if (t1 == tiles) span->y = cta;
    }
    __device__ __forceinline__ int rows() const { return b < 0 ? p.B * p.T * p.G : p.T * p.G; }
    __device__ __forceinline__ const int32_t* list() const { return b < 0 ? p.prefix_pages : p.table + b * p.ld_table; }
    __device__ __forceinline__ int pages() const { return int((int64_t(keys) + (1 << p.shift) - 1) >> p.shift); }
};

// The page lists on their way into L2 while the lengths are looked up (they are needed next; both come from HBM in a step of a
// model whose weights have passed through L2 since).  Executed by `n` threads of every CTA.
__device__ __forceinline__ void prefetch_lists(const Problem& p, const Line& w, int n, int t) {
    const int64_t lines_p = w.blocks_p ? ((int64_t(p.prefix_len) >> p.shift) * 4 + 127) / 128 : 0;
    const int64_t lines = lines_p + (w.blocks_s ? (p.B * p.ld_table * 4 + 127) / 128 : 0);
    for (int64_t i = int64_t(blockIdx.x) * n + t; i < lines; i += int64_t(gridDim.x) * n) {
        const char* at = i < lines_p ? reinterpret_cast<const char*>(p.prefix_pages) + i * 128 : reinterpret_cast<const char*>(p.table) + (i - lines_p) * 128;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
    }
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// rows of one page (and of one half or all halves, by the map's box) of one head -> shared memory
__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap* map, int row, int half, int head, int page, uint32_t bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %3, %4, %5, %6}], [%7], %8;"
        ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(half), "r"(head), "r"(page), "r"(bar), "l"(policy) : "memory");
}

constexpr int kDecodeKeys = 64, kBlockKeys = 128;     // keys of a tile
constexpr int kDecodeCost = 1, kBlockCost = 3;        // Line::cost
constexpr int kMaxShares = 4 * kMaxSms;               // CTAs of one launch, at most
int launch_attn_decode(const patch_kv_cache_t* c, const Problem& p, const Line& w, const Results& to, bool after_block, cudaStream_t s);
// one launch for everything: clusters of `split` CTAs (1, 2, 4, 8 or 16; 16 is more than the portable size and allowed explicitly)
int launch_attn_direct(const patch_kv_cache_t* c, const Problem& p, int split, __nv_bfloat16* O, int64_t ldo, float* lse, cudaStream_t s);
int launch_attn_block(const patch_kv_cache_t* c, const Problem& p, const Line& w, const Results& to, bool decode_follows, cudaStream_t s);

}  // namespace attn

int validate_kv_cache(const patch_kv_cache_t* c);
// Tensor map over the keys or values of a cache as (element in a 64-element half, slot, half, head, page); the box is `rows`
// slots of `halves` halves of one head of one page, 128-byte swizzle.
int make_kv_tensor_map(CUtensorMap* map, const patch_kv_cache_t* c, const void* base, int rows, int halves);

}  // namespace patch
