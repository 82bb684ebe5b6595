// Shared by the kernels of the attention within packed sequences: the problem, and which rows a CTA owns.
#pragma once
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

// Tiles of all sequences in one line: sequence b's first tile is number starts[b] / rows + b, and it has at most as many as lie before
// the next one's first.
struct Tile { int begin, end, first; };      // rows of the sequence; the tile's first row, counted from `begin` (-1: no tile)
__host__ __device__ __forceinline__ int64_t most_tiles(int64_t M, int64_t B, int rows) { return M / rows + B; }
__device__ __forceinline__ int clamped(const Problem& p, int b) { return min(max(p.starts[b], 0), p.M); }
template <int ROWS>
__device__ __forceinline__ Tile tile_of(const Problem& p, int slot) {
    int lo = -1, hi = p.B;                   // the last sequence whose first tile is at or before `slot`
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (clamped(p, mid) / ROWS + mid <= slot) lo = mid; else hi = mid;
    }
    Tile t = {0, 0, -1};
    if (lo < 0) return t;
    t.begin = clamped(p, lo);
    t.end = max(clamped(p, lo + 1), t.begin);
    const int first = (slot - (t.begin / ROWS + lo)) * ROWS;
    if (first >= 0 && first < t.end - t.begin) t.first = first;
    return t;
}
// starts out of order or out of range are reported (every tile stays within the rows all the same)
__device__ __forceinline__ void check_starts(const Problem& p, int thread, int threads) {
    if (!p.status) return;
    bool bad = false;
#pragma unroll 4
    for (int b = thread; b <= p.B; b += threads) bad |= p.starts[b] < 0 || p.starts[b] > p.M || (b && p.starts[b] < p.starts[b - 1]);
    if (bad) atomicCAS(p.status, PATCH_OK, PATCH_ERR_SIZE);
}

int launch_forward(const Problem& p, int D, __nv_bfloat16* o, int64_t ldo, float* lse, cudaStream_t s);

}  // namespace seq
}  // namespace patch
