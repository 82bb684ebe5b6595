// Attention of a batch that shares a prefix, over the paged cache: entry points, choice of kernels and the joining kernel (public
// header: patch_prefix_attention; kernels: attention_decode_sm100.cu, attention_block_sm100.cu; work list: attention.cuh).
//
// The batch's query rows of one key head are one operand against the shared prefix (B T G rows), a sequence's rows (T G) one
// against its own keys.  Softmax parts over disjoint keys join exactly: with m = max m_i and w_i = 2^((m_i - m) scale),
// o = sum w_i o_i and l = sum w_i l_i, the result is o / l.
#include "attention.cuh"

namespace patch {
namespace attn {

// Number of an item's parts.  A launch that gave up (PATCH_ERR_TIMEOUT) may have left items without a note: whatever lies there then
// must not lead out of the workspace.
__device__ __forceinline__ int parts_of(int2 span) {
    return unsigned(span.x) < unsigned(kMaxShares) && unsigned(span.y) < unsigned(kMaxShares) && span.x <= span.y ? span.y - span.x + 1 : 0;
}

// Joins the partial results: one warp per query row and head.  Bound by the latency of two dependent reads (which CTAs, their
// results); the (m, l) of up to 32 parts are read at once, one per lane, and with them the outputs of the first eight (asked for
// after the factors are known they cost 1.0 to 1.7 us more).
template <int D>
__global__ void __launch_bounds__(256)
attn_join_kernel(const Problem p, const Results from, const int blocks_p, const int blocks_s, __nv_bfloat16* __restrict__ O, int64_t ldo,
                 float* __restrict__ lse) {
    constexpr int V = D / 32, kAhead = 8;             // elements per lane; parts asked for together with their (m, l)
    const int lane = threadIdx.x & 31;
    const int row = blockIdx.x * 8 + (threadIdx.x >> 5), Hq = p.Hkv * p.G;
    const bool on = row < p.B * p.T * Hq;
    const int tok = row / Hq, hq = row - tok * Hq, kvh = hq / p.G, gq = hq - kvh * p.G, b = tok / p.T;
    const bool own = on && suffix_len(p, b) > 0;
    grid_dependency_wait();
    if (!on) return;

    // slot of the item's first part, and the row's place in a slot
    int count[2] = {0, 0}, place[2] = {0, 0};
    int64_t at[2] = {0, 0};
    if (blocks_p) {
        const int r = tok * p.G + gq, blk = r / from.p.rows, item = kvh * blocks_p + blk;
        const int2 span = from.p.span[item];
        count[0] = parts_of(span);
        at[0] = int64_t(item) + span.x;
        place[0] = r - blk * from.p.rows;
    }
    if (own) {
        const int r = (tok - b * p.T) * p.G + gq, blk = r / from.s.rows, item = (b * p.Hkv + kvh) * blocks_s + blk;
        const int2 span = from.s.span[item];
        count[1] = parts_of(span);
        at[1] = int64_t(item) + span.x;
        place[1] = r - blk * from.s.rows;
    }
    // this lane's elements of the first part, and from part to part
    const int c = lane * V / 4, in_chunk = lane * V % 4;
    const float* src[2] = {from.p.o + from.p.chunk<D>(at[0], place[0], c) + in_chunk, from.s.o + from.s.chunk<D>(at[1], place[1], c) + in_chunk};
    const int64_t step[2] = {int64_t(from.p.rows) * D, int64_t(from.s.rows) * D};
    float m = -INFINITY, l = 0.0f, acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    const int all = count[0] + count[1];
    for (int k0 = 0; k0 < all; k0 += 32) {
        const int here = all - k0 < 32 ? all - k0 : 32;
        // this lane's part: its (m, l)
        const int k = k0 + lane;
        const bool of_p = k < count[0];
        const Parts& part = of_p ? from.p : from.s;
        const int64_t slot = of_p ? at[0] + k : at[1] + (k - count[0]);
        const int r = of_p ? place[0] : place[1];
        const float2 mine = lane < here ? part.ml[slot * part.rows + r] : make_float2(-INFINITY, 0.0f);
        // elements of part k0 + q
        auto elements = [&](int q, float* v) {
            const int k1 = k0 + q;
            const float* from_o = k1 < count[0] ? src[0] + k1 * step[0] : src[1] + (k1 - count[0]) * step[1];
            if constexpr (V == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(from_o);
            else *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(from_o);
        };
        float v[kAhead][V];
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            if (q < here) elements(q, v[q]);
            else
#pragma unroll
                for (int i = 0; i < V; ++i) v[q][i] = 0.0f;
        float mx = fmaxf(m, mine.x);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, d));
        if (!__any_sync(0xFFFFFFFFu, mine.y != 0.0f)) continue;      // saw nothing (a row of NaN has seen something: its sum is NaN)
        const float f = ex2(exponent(mine.x, mx, p.scale_log2)), a = ex2(exponent(m, mx, p.scale_log2));
        float add = mine.y * f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) add += __shfl_xor_sync(0xFFFFFFFFu, add, d);
        l = l * a + add;
        m = mx;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] *= a;
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {           // past `here` the factor is 0
            const float fq = __shfl_sync(0xFFFFFFFFu, f, q);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = fmaf(v[q][i], fq, acc[i]);
        }
#pragma unroll 8
        for (int q = kAhead; q < here; ++q) {
            const float fq = __shfl_sync(0xFFFFFFFFu, f, q);
            float w[V];
            elements(q, w);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = fmaf(w[i], fq, acc[i]);
        }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // nothing seen: 0
    __nv_bfloat16* dst = O + int64_t(tok) * ldo + int64_t(hq) * D + lane * V;
    if constexpr (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2(acc[0] * inv, acc[1] * inv), pack2(acc[2] * inv, acc[3] * inv));
    else *reinterpret_cast<uint32_t*>(dst) = pack2(acc[0] * inv, acc[1] * inv);
    if (lse && lane == 0) lse[row] = l == 0.0f ? -INFINITY : (m * p.scale_log2 + log2f(l)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------------------------
// host side

// Which kernel serves a phase.  The prefix: the decode kernel where its 16 rows of mma.sync hold all rows (HBM is what it waits
// for).  More rows are more blocks there, all of which read the keys (from L2 but for the first), so that is for work so small that it
// ends before the block kernel, whose chain of queries, tiles and result takes 12 us at least, would: up to 4000 tiles of 64 keys and
// 16 rows.  Measured, decode kernel against block kernel: 16 sequences, 40 heads of 7 rows, 4 + 900 keys 56 us against 62; 7
// sequences, 40 heads of 4 rows, 1454 + 10 keys 16.7 against 22.0 (1 920 tiles); 19 sequences, 8 heads of 16 rows, 929 + 40 keys 17.7
// against 20.6 (2 432); 29 sequences, 8 heads of 4 rows, 4478 + 500 keys 28.9 against 27.6 (4 544).  A sequence's own keys, where its
// T G rows are more than 16: items are short, and an item costs the block kernel about 6 us (queries, first tile, result), so where page
// tables end at 1024 keys up to four blocks of 16 rows stay on the decode kernel, with the keys from L2 from the second block on.
// Measured, 16 sequences, 28 rows, 8 key heads: 200 keys 13.6 us there against 17.3, 800 keys 21.6 against 28.0, 4096 keys 85.4
// against 52.8.  Where suffixes go to the block kernel the prefix does too, so that there is one kernel less.
constexpr int64_t kMostPrefixUnits = 4000;
constexpr int kMostDecodeRows = 64, kMostDecodeKeys = 1024;
static bool block_prefix(int64_t rows, int64_t Hkv, int64_t prefix_len) {
    return rows > kDecodeRows && (rows + kDecodeRows - 1) / kDecodeRows * Hkv * ((prefix_len + kDecodeKeys - 1) / kDecodeKeys + kDecodeCost) > kMostPrefixUnits;
}
static bool block_suffixes(int64_t rows, int64_t keys) { return rows > kMostDecodeRows || (rows > kDecodeRows && keys > kMostDecodeKeys); }

// CTAs of a cluster for each item of the small problems that take one launch of their own (attn_direct_kernel), 0 for the others.
// There every item reads the prefix for itself, so it is a matter of how many tiles there are in all (by the tables' width): up to
// eight for each CTA that can run at once.  Measured on the same inputs call after call (from L2; one sequence of 128 + 64 keys that come
// from HBM takes 5.9 us), one launch against two or three, 7B heads: one sequence, 128 + 100 keys 5.2 us against 8.3, 4096 + 100 keys (7 tiles a slot) 15.4 against 18.0, 4 x (1024 + 100) (8 a slot) 11.9 against 11.9; 8 key heads of 4
// rows, 16 x (64 + 500) 9.0 us against 26.1 (32 rows or more of a prefix are the block kernel's otherwise).  A second wave of items
// is worth it only where a prefix would be a launch of its own: 2 items a slot 14.6 us against 32.8 with one, 3 items a slot without 14.1
// against 12.2.  Clusters of 16 (more than the portable 8) pay from four tiles a CTA: 71 tiles an item 10.4 us against 11.4, 16
// tiles 7.7 against 6.8.
static int direct_split(int64_t rows, int64_t heads, int64_t prefix_len, int64_t table_keys) {
    const int64_t slots = 2 * sm_count(), items = heads * ((rows + kDecodeRows - 1) / kDecodeRows);
    const int64_t tiles = (prefix_len + kDecodeKeys - 1) / kDecodeKeys + (table_keys + kDecodeKeys - 1) / kDecodeKeys;
    if (tiles > 8 * slots || items * tiles > 8 * slots || items > (prefix_len ? 2 : 1) * slots) return 0;
    int split = 1;                                   // all CTAs at once, and each with a tile at least
    while (split < 16 && 2 * split * items <= slots && tiles >= (split < 8 ? 2 * split : 64)) split *= 2;
    return split;
}

struct Plan {
    bool block_p, block_s;                           // prefix / suffixes on the block kernel
    int blocks_p, blocks_s, rows_p, rows_s;          // row blocks per key head, rows of a slot
    size_t span_s, ml_p, ml_s, o_p, o_s, bytes;      // workspace: [spans of prefix items | of suffix items | (m, l) | outputs]
};
static Plan plan_of(const patch_kv_cache_t* c, int64_t B, int64_t T, int64_t G, int64_t prefix_len, int64_t table_keys) {
    Plan q;
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    auto rows = [&](int64_t all, bool block, int& blocks) {
        const int most = block ? kBlockRows : kDecodeRows;
        blocks = int((all + most - 1) / most);
        return int(all < most ? all : most);
    };
    q.block_s = block_suffixes(T * G, table_keys);
    q.block_p = q.block_s ? B * T * G > kDecodeRows : block_prefix(B * T * G, c->Hkv, prefix_len);
    q.rows_p = rows(B * T * G, q.block_p, q.blocks_p);
    q.rows_s = rows(T * G, q.block_s, q.blocks_s);
    // a slot for every item and every CTA that may share one
    const size_t items_p = size_t(c->Hkv) * q.blocks_p, items_s = size_t(c->Hkv) * B * q.blocks_s;
    const size_t slots_p = items_p + kMaxShares, slots_s = items_s + kMaxShares;
    q.span_s = up(items_p * 8);
    q.ml_p = q.span_s + up(items_s * 8);
    q.ml_s = q.ml_p + up(slots_p * q.rows_p * 8);
    q.o_p = q.ml_s + up(slots_s * q.rows_s * 8);
    q.o_s = q.o_p + up(slots_p * q.rows_p * size_t(c->D) * 4);
    q.bytes = q.o_s + up(slots_s * q.rows_s * size_t(c->D) * 4);
    return q;
}

static int check_batch(const patch_kv_cache_t* c, int64_t B, int T, int Hq) {
    int rc = validate_kv_cache(c);
    if (rc) return rc;
    if (c->D != 64 && c->D != 128) return PATCH_ERR_SHAPE;
    if (B < 0 || B > kMaxBatch || T < 1 || Hq < 1 || Hq > (1 << 16) || Hq % c->Hkv) return PATCH_ERR_SHAPE;
    if (B * T > 0x7FFFFFFF / c->D / Hq) return PATCH_ERR_SHAPE;
    return PATCH_OK;
}

}  // namespace attn

int make_kv_tensor_map(CUtensorMap* map, const patch_kv_cache_t* c, const void* base, int rows, int halves) {
    EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return PATCH_ERR_CUDA;
    const cuuint64_t row = cuuint64_t(c->D) * 2;
    const cuuint64_t dims[5] = {64, cuuint64_t(c->page_size), cuuint64_t(c->D / 64), cuuint64_t(c->Hkv), cuuint64_t(c->num_pages)};
    const cuuint64_t strides[4] = {row, 128, row * c->page_size, cuuint64_t(c->page_stride) * 2};
    const cuuint32_t box[5] = {64, cuuint32_t(rows), cuuint32_t(halves), 1, 1};
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? PATCH_OK : PATCH_ERR_CUDA;
}

}  // namespace patch

using namespace patch;

extern "C" int patch_prefix_attention_workspace_size(const patch_kv_cache_t* cache, int64_t B, int T, int Hq, size_t* bytes_out) {
    if (!bytes_out) return PATCH_ERR_NULL;
    int rc = attn::check_batch(cache, B, T, Hq);
    if (rc) return rc;
    // whatever the prefix's length and the tables' width will be
    const int64_t G = Hq / cache->Hkv;
    *bytes_out = 0;
    for (int64_t prefix : {int64_t(0), int64_t(1) << 30})
        for (int64_t keys : {int64_t(0), int64_t(1) << 40}) {
            const size_t n = attn::plan_of(cache, B, T, G, prefix, keys).bytes;
            if (n > *bytes_out) *bytes_out = n;
        }
    return PATCH_OK;
}

extern "C" int patch_prefix_attention(const patch_kv_cache_t* cache, const void* Q, int64_t ldq, int64_t B, int T, int Hq,
                                      const int32_t* prefix_pages, int64_t prefix_len, const int32_t* page_table, int64_t ld_table,
                                      const int32_t* suffix_lens, float scale, void* O, int64_t ldo, float* lse, void* workspace,
                                      size_t workspace_bytes, int* status_dev, void* stream) {
    using namespace attn;
    int rc = check_batch(cache, B, T, Hq);
    if (rc) return rc;
    if (prefix_len < 0 || prefix_len > 0x7FFFFF00 || ld_table < 0 || ld_table > 0x7FFFFFFF || !(scale > 0.0f) || scale > 2.0e38f) return PATCH_ERR_SHAPE;
    if (B == 0) return PATCH_OK;
    if (!Q || !O || !suffix_lens || (prefix_len && !prefix_pages) || (ld_table && !page_table)) return PATCH_ERR_NULL;
    const int D = cache->D;
    if (ldq < int64_t(Hq) * D || ldo < int64_t(Hq) * D || ldq % 8 || ldo % 8) return PATCH_ERR_SHAPE;
    if (!aligned16(Q) || !aligned16(O)) return PATCH_ERR_ALIGN;
    const int G = Hq / cache->Hkv;
    size_t need = 0;
    if ((rc = patch_prefix_attention_workspace_size(cache, B, T, Hq, &need))) return rc;
    if (!workspace) return PATCH_ERR_NULL;
    if (workspace_bytes < need) return PATCH_ERR_SIZE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return PATCH_ERR_ALIGN;
    const Plan q = plan_of(cache, B, T, G, prefix_len, ld_table * cache->page_size);
    auto tiles = [&](int keys) { return int((prefix_len + keys - 1) / keys); };
    // units are counted in 32 bits
    const int64_t own = (ld_table * cache->page_size + kDecodeKeys - 1) / kDecodeKeys + 8;
    if (int64_t(cache->Hkv) * q.blocks_p * (int64_t(tiles(kDecodeKeys)) + 8) + B * own * cache->Hkv * q.blocks_s > 0x7FFFFFFF) return PATCH_ERR_SHAPE;
    if ((rc = check_device())) return rc;
    Problem p = {static_cast<const __nv_bfloat16*>(Q), ldq, int(B), T, cache->Hkv, G, prefix_pages, int(prefix_len), page_table,
                 ld_table, suffix_lens, 0, int(cache->num_pages), scale * 1.4426950408889634f, status_dev, 0u};
    while ((1 << p.shift) < cache->page_size) ++p.shift;
    // r * ceil(2^32 / G) is at most r G above r 2^32 / G: exact while that stays below 2^32
    if (G > 1 && B * T * G * int64_t(G) < (int64_t(1) << 32)) p.g_mul = uint32_t(((uint64_t(1) << 32) + G - 1) / G);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (const int split = direct_split(int64_t(T) * G, B * cache->Hkv, prefix_len, ld_table * cache->page_size))
        return launch_attn_direct(cache, p, split, static_cast<__nv_bfloat16*>(O), ldo, lse, s);
    const Results to = {{reinterpret_cast<float*>(ws + q.o_p), reinterpret_cast<float2*>(ws + q.ml_p), reinterpret_cast<int2*>(ws), q.rows_p, q.block_p},
                        {reinterpret_cast<float*>(ws + q.o_s), reinterpret_cast<float2*>(ws + q.ml_s), reinterpret_cast<int2*>(ws + q.span_s), q.rows_s, q.block_s}};
    const bool prefix = prefix_len > 0;
    const Line dec = {prefix && !q.block_p ? q.blocks_p : 0, q.block_s ? 0 : q.blocks_s, tiles(kDecodeKeys), kDecodeCost, 6};
    const Line blk = {prefix && q.block_p ? q.blocks_p : 0, q.block_s ? q.blocks_s : 0, tiles(kBlockKeys), kBlockCost, 7};
    const bool use_block = blk.blocks_p || blk.blocks_s, use_decode = dec.blocks_p || dec.blocks_s;
    if (use_block && (rc = launch_attn_block(cache, p, blk, to, use_decode, s))) return rc;
    if (use_decode && (rc = launch_attn_decode(cache, p, dec, to, use_block, s))) return rc;
    const int64_t out_rows = B * T * Hq;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3(unsigned((out_rows + 7) / 8), 1, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(O);
    const int blocks_p = prefix ? q.blocks_p : 0;
    const cudaError_t e = D == 128 ? cudaLaunchKernelEx(&cfg, attn_join_kernel<128>, p, to, blocks_p, q.blocks_s, o, ldo, lse)
                                   : cudaLaunchKernelEx(&cfg, attn_join_kernel<64>, p, to, blocks_p, q.blocks_s, o, ldo, lse);
    return e == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}
