// Attention of a batch that shares a prefix, over the paged cache: entry points, choice of kernels and the joining kernel (public
// header: patch_prefix_attention; kernels: attention_decode_sm100.cu, attention_block_sm100.cu; work list: attention.cuh).
//
// The batch's query rows of one key head are one operand against the shared prefix (B T G rows), a sequence's rows (T G) one
// against its own keys.  Softmax parts over disjoint keys join exactly: with m = max m_i, o = sum 2^(m_i - m) o_i and
// l = sum 2^(m_i - m) l_i, the result is o / l.
#include "attention.cuh"

namespace patch {
namespace attn {

// One line of units and the CTAs that shared it.
struct Source { Line w; const int* cum; int ctas; };

// Joins the partial results: one warp per query row and head.  Bound by the latency of a few dependent reads from L2; the
// (m, l) pairs of up to 32 parts are read at once, one per lane, and their outputs four at a time.
template <int D>
__global__ void __launch_bounds__(256)
attn_join_kernel(const Problem p, const Source sp, const Source ss, const Parts parts, __nv_bfloat16* __restrict__ O, int64_t ldo,
                 float* __restrict__ lse) {
    constexpr int V = D / 32;                        // elements per lane
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int64_t row = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const int Hq = p.Hkv * p.G;
    if (row >= int64_t(p.B) * p.T * Hq) return;
    const int tok = int(row / Hq), hq = int(row - int64_t(tok) * Hq), kvh = hq / p.G, gq = hq - kvh * p.G, b = tok / p.T;

    float m = -INFINITY, l = 0.0f, acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    // the parts of one item: tiles are `count` units from `first` on; (m, l) and outputs of the slots item + CTA
    auto add = [&](const Source& src, int64_t first, int64_t count, int64_t item, int r, const float* o, const float2* ml, int rows) {
        if (count <= 0) return;
        const int64_t total = total_units(src.w, p.Hkv, src.cum[p.B]);
        const int n = total < src.ctas ? int(total) : src.ctas;
        const int c0 = owner(first, total, n), parts_n = owner(first + count - 1, total, n) - c0 + 1;
        const int64_t at = (item + c0) * rows + r;
        for (int k0 = 0; k0 < parts_n; k0 += 32) {
            const int here = parts_n - k0 < 32 ? parts_n - k0 : 32;
            const float2 mine = lane < here ? ml[at + int64_t(k0 + lane) * rows] : make_float2(-INFINITY, 0.0f);
            float mx = fmaxf(m, mine.x);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, d));
            if (mx == -INFINITY) continue;
            const float f = ex2(mine.x - mx), a = ex2(m - mx);
            float add_l = mine.y * f;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) add_l += __shfl_xor_sync(0xFFFFFFFFu, add_l, d);
            l = l * a + add_l;
            m = mx;
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] *= a;
#pragma unroll 4
            for (int k = 0; k < here; ++k) {
                const float* src_o = o + (at + int64_t(k0 + k) * rows) * D + lane * V;
                const float fk = __shfl_sync(0xFFFFFFFFu, f, k);
                float v[V];
                if constexpr (V == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(src_o);
                else *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(src_o);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = fmaf(v[i], fk, acc[i]);
            }
        }
    };
    if (sp.w.blocks_p) {
        const int r = tok * p.G + gq, blk = r / parts.rows_p, item = kvh * sp.w.blocks_p + blk;
        add(sp, int64_t(item) * (sp.w.tiles_p + sp.w.cost) + sp.w.cost, sp.w.tiles_p, item, r - blk * parts.rows_p, parts.o_p, parts.ml_p, parts.rows_p);
    }
    {
        const int r = (tok - b * p.T) * p.G + gq, blk = r / parts.rows_s, sub = kvh * ss.w.blocks_s + blk, per = p.Hkv * ss.w.blocks_s;
        const int each = ss.cum[b + 1] - ss.cum[b];
        add(ss, prefix_units(ss.w, p.Hkv) + int64_t(ss.cum[b]) * per + int64_t(sub) * each + ss.w.cost, each - ss.w.cost, int64_t(b) * per + sub,
            r - blk * parts.rows_s, parts.o_s, parts.ml_s, parts.rows_s);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // nothing seen: 0
    __nv_bfloat16* dst = O + int64_t(tok) * ldo + int64_t(hq) * D + lane * V;
    if constexpr (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2(acc[0] * inv, acc[1] * inv), pack2(acc[2] * inv, acc[3] * inv));
    else *reinterpret_cast<uint32_t*>(dst) = pack2(acc[0] * inv, acc[1] * inv);
    if (lse && lane == 0) lse[row] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------------------------
// host side

// Which kernel serves a phase, and its items' rows.  Up to 16 rows the decode kernel's tile (16 rows of mma.sync) holds them
// and HBM is what it waits for; more rows would have it read the keys once per 16.
struct Plan {
    bool block_p, block_s;                           // prefix / suffixes on the block kernel
    int blocks_p, blocks_s, rows_p, rows_s;          // row blocks per key head, rows of a slot
    size_t cum_block, ml_p, ml_s, o_p, o_s, bytes;   // workspace: [units of the decode kernel | of the block kernel | (m, l) | outputs]
};
static Plan plan_of(const patch_kv_cache_t* c, int64_t B, int64_t T, int64_t G) {
    Plan q;
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    auto rows = [&](int64_t all, bool& block, int& blocks) {
        block = all > kFewRows;
        blocks = block ? int((all + kBlockRows - 1) / kBlockRows) : 1;
        return int(all < kBlockRows ? all : kBlockRows);
    };
    q.rows_p = rows(B * T * G, q.block_p, q.blocks_p);
    q.rows_s = rows(T * G, q.block_s, q.blocks_s);
    // a slot for every item and every CTA that may share one (the decode kernel has two CTAs per SM)
    const size_t slots_p = size_t(c->Hkv) * q.blocks_p + 2 * kMaxSms, slots_s = size_t(c->Hkv) * B * q.blocks_s + 2 * kMaxSms;
    q.cum_block = up(size_t(B + 1) * 4);
    q.ml_p = 2 * q.cum_block;
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
}  // namespace patch

using namespace patch;

extern "C" int patch_prefix_attention_workspace_size(const patch_kv_cache_t* cache, int64_t B, int T, int Hq, size_t* bytes_out) {
    if (!bytes_out) return PATCH_ERR_NULL;
    int rc = attn::check_batch(cache, B, T, Hq);
    if (rc) return rc;
    *bytes_out = attn::plan_of(cache, B, T, Hq / cache->Hkv).bytes;
    return PATCH_OK;
}

extern "C" int patch_prefix_attention(const patch_kv_cache_t* cache, const void* Q, int64_t ldq, int64_t B, int T, int Hq,
                                      const int32_t* prefix_pages, int64_t prefix_len, const int32_t* page_table, int64_t ld_table,
                                      const int32_t* suffix_lens, float scale, void* O, int64_t ldo, float* lse, void* workspace,
                                      size_t workspace_bytes, int* status_dev, void* stream) {
    using namespace attn;
    int rc = check_batch(cache, B, T, Hq);
    if (rc) return rc;
    if (prefix_len < 0 || prefix_len > 0x7FFFFF00 || ld_table < 0 || !(scale > 0.0f) || scale > 3.0e38f) return PATCH_ERR_SHAPE;
    if (B == 0) return PATCH_OK;
    // units of a sequence, summed over the batch, are counted in 32 bits (tiles of 64 keys or more, and each item's own cost)
    if (ld_table > 0x7FFFFFFF || B * ((ld_table * cache->page_size + 63) / 64 + 8) > 0x7FFFFFFF) return PATCH_ERR_SHAPE;
    if (!Q || !O || !suffix_lens || (prefix_len && !prefix_pages) || (ld_table && !page_table)) return PATCH_ERR_NULL;
    const int D = cache->D;
    if (ldq < int64_t(Hq) * D || ldo < int64_t(Hq) * D || ldq % 8 || ldo % 8) return PATCH_ERR_SHAPE;
    if (!aligned16(Q) || !aligned16(O)) return PATCH_ERR_ALIGN;
    const int G = Hq / cache->Hkv;
    const Plan q = plan_of(cache, B, T, G);
    if (!workspace) return PATCH_ERR_NULL;
    if (workspace_bytes < q.bytes) return PATCH_ERR_SIZE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return PATCH_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    const int sms = sm_count() < kMaxSms ? sm_count() : kMaxSms;
    if (sms <= 0) return PATCH_ERR_CUDA;
    Problem p = {static_cast<const __nv_bfloat16*>(Q), ldq, int(B), T, cache->Hkv, G, prefix_pages, int(prefix_len), page_table,
                 ld_table, suffix_lens, 0, int(cache->num_pages), scale * 1.4426950408889634f, status_dev};
    while ((1 << p.shift) < cache->page_size) ++p.shift;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const Parts parts = {reinterpret_cast<float*>(ws + q.o_p), reinterpret_cast<float*>(ws + q.o_s), reinterpret_cast<float2*>(ws + q.ml_p),
                         reinterpret_cast<float2*>(ws + q.ml_s), q.rows_p, q.rows_s};
    const bool prefix = prefix_len > 0;
    Source dec = {{prefix && !q.block_p ? 1 : 0, q.block_s ? 0 : 1, 0, kDecodeCost}, reinterpret_cast<const int*>(ws), decode_ctas(sms)};
    Source blk = {{prefix && q.block_p ? q.blocks_p : 0, q.block_s ? q.blocks_s : 0, 0, kBlockCost}, reinterpret_cast<const int*>(ws + q.cum_block), sms};
    dec.w.tiles_p = int((prefix_len + kDecodeKeys - 1) / kDecodeKeys);
    blk.w.tiles_p = int((prefix_len + kBlockKeys - 1) / kBlockKeys);
    const bool use_block = blk.w.blocks_p || blk.w.blocks_s, use_decode = dec.w.blocks_p || dec.w.blocks_s;
    if (use_block && (rc = launch_attn_block(cache, p, blk.w, parts, const_cast<int*>(blk.cum), s))) return rc;
    if (use_decode && (rc = launch_attn_decode(cache, p, dec.w, parts, const_cast<int*>(dec.cum), use_block, s))) return rc;
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
    const cudaError_t e = D == 128 ? cudaLaunchKernelEx(&cfg, attn_join_kernel<128>, p, q.block_p ? blk : dec, q.block_s ? blk : dec, parts, o, ldo, lse)
                                   : cudaLaunchKernelEx(&cfg, attn_join_kernel<64>, p, q.block_p ? blk : dec, q.block_s ? blk : dec, parts, o, ldo, lse);
    return e == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}
