// Shared by the attention kernels: the problem as the kernels see it, the work list (which CTA owns which tiles of which
// item) and the partial results that the joining kernel adds up.
//
// Work list.  An item is a set of query rows of one key head that read the same keys: the batch's rows against the shared
// prefix, or one sequence's rows against its own keys.  An item's keys are cut into tiles; all tiles of all items,
// item after item, form one line of U units, and CTA c of n owns units [c U / n, (c + 1) U / n): every CTA gets the same number of
// tiles whatever the lengths are, at the price of items that several CTAs share.  Each CTA writes one partial result
// (running maximum, sum and unnormalised output, fp32) per item it has a share of.  Along the line the pair (item,
// CTA) changes one step at a time, so item + c numbers the partial results without gaps worth caring about, and the joining
// kernel finds an item's partial results from its first and last unit.
#pragma once
#include "sm100_ptx.cuh"

namespace patch {
namespace attn {

constexpr int kMaxBatch = 2048;
constexpr int kMaxCtas = 160;                 // CTAs of an attention launch: one per SM, at most these (sizes the workspace)

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
    float scale_log2;                         // scale * log2(e): scores are kept in powers of two
    int* status;
};

// Line of units of one kernel.  rows_p / rows_s: query rows of a prefix / suffix item; blocks of kRows rows are items of their own.
struct Line {
    int blocks_p, blocks_s;                   // row blocks per key head: prefix items (0: none in this kernel), suffix items (0: none)
    int tiles_p;                              // key tiles of a prefix item
};

// len -> clamped length of sequence b's own keys
__device__ __forceinline__ int suffix_len(const Problem& p, int b) {
    const int64_t n = p.lens[b], most = p.ld_table << p.shift;
    if (n < 0 || n > most) {
        if (p.status) atomicCAS(p.status, PATCH_OK, PATCH_ERR_SIZE);
        return n < 0 ? 0 : int(most < 0x7FFFFFFF ? most : 0x7FFFFFFF);
    }
    return int(n);
}

// First unit after which ... the CTA that owns unit u of U spread over n <= U CTAs.
__device__ __forceinline__ int owner(int64_t u, int64_t U, int n) { return int(((u + 1) * n - 1) / U); }

// The walk of one CTA along the line: the item that holds a unit, and the items after it.  `cum` is the number of key tiles before each
// sequence (one key head, one row block), `len` the clamped lengths, both in shared memory.
struct Walk {
    const Problem& p;
    const Line& w;
    const int* cum;
    const int* len;
    int b, kvh, block, tiles, keys;           // b < 0: the prefix
    int item;

    __device__ __forceinline__ Walk(const Problem& p_, const Line& w_, const int* cum_, const int* len_) : p(p_), w(w_), cum(cum_), len(len_) {}
    __device__ __forceinline__ int64_t prefix_units() const { return int64_t(p.Hkv) * w.blocks_p * w.tiles_p; }
    __device__ __forceinline__ int per() const { return p.Hkv * w.blocks_s; }          // items of a sequence
    __device__ __forceinline__ int64_t total() const { return prefix_units() + int64_t(cum[p.B]) * per(); }
    __device__ __forceinline__ void at_sequence(int b_) {
        b = b_;
        tiles = cum[b + 1] - cum[b];
        keys = len[b];
    }
    // to the item of unit u; returns the tile
    __device__ __forceinline__ int seek(int64_t u) {
        const int64_t before = prefix_units();
        if (u < before) {
            item = int(u / w.tiles_p);
            b = -1;
            kvh = item / w.blocks_p;
            block = item - kvh * w.blocks_p;
            tiles = w.tiles_p;
            keys = p.prefix_len;
            return int(u - int64_t(item) * w.tiles_p);
        }
        const int64_t v = u - before, q = v / per();
        int lo = 0, hi = p.B;                 // the sequence with cum[lo] <= q < cum[lo + 1]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cum[mid] <= q) lo = mid; else hi = mid;
        }
        at_sequence(lo);
        const int64_t r = v - int64_t(cum[lo]) * per();
        const int sub = int(r / tiles);
        kvh = sub / w.blocks_s;
        block = sub - kvh * w.blocks_s;
        item = p.Hkv * w.blocks_p + lo * per() + sub;
        return int(r - int64_t(sub) * tiles);
    }
    // to the next item that has tiles (there is one)
    __device__ __forceinline__ void next() {
        ++item;
        if (++block < (b < 0 ? w.blocks_p : w.blocks_s)) return;
        block = 0;
        if (++kvh < p.Hkv) return;
        kvh = 0;
        int n = b + 1;
        while (n + 1 < p.B && cum[n + 1] == cum[n]) ++n;
        item = p.Hkv * w.blocks_p + n * per();
        at_sequence(n);
    }
};

}  // namespace attn

int validate_kv_cache(const patch_kv_cache_t* c);
// Tensor map over the keys or values of a cache as (element in a 64-element half, slot, half, head, page); the box is `rows`
// slots of `halves` halves of one head of one page, 128-byte swizzle.
int make_kv_tensor_map(CUtensorMap* map, const patch_kv_cache_t* c, const void* base, int rows, int halves);

}  // namespace patch
