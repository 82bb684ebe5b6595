// Attention over the paged cache for items of few query rows, taken in blocks of at most 16, and for small problems in one launch
// (public header: patch_prefix_attention; the work list and the partial results are described in attention.cuh).
//
// Mathematics.  For every row the running maximum m of the scores s = q.k, the sum l of 2^((s - m) scale) and the unnormalised output
// o = sum 2^((s - m) scale) v; parts of the keys are joined with weights 2^((m_i - m) scale) (softmax_rule.cuh).  All three are fp32; the
// probabilities are rounded to bf16 for the product with V (they are at most 1; the sum takes them unrounded).
//
// Kernel.  Every CTA, two to an SM (one for more than 1231 sequences of heads of 128), walks over its share of the work list (attention.cuh).  Warp 4 alone knows the list: it requests tiles
// of 64 keys and values with TMA, one copy per page and operand, into a ring of stages, and with an item's first tile the
// item's query rows; a note in the stage says what the tile is.  Warps 0..3 each take 16 of the 64 keys: S = Q K^T
// (16 rows x 16 keys), probabilities in registers, O += P V, with a maximum of their own, so that within an item no warp waits
// for another.  At the end of a share the four warps' results are joined in shared memory, while the SM's other CTA
// streams.
// What bounds it: HBM.  A 64-key tile is 32 KB (D = 128), about 1 430 cycles of an SM's share of the bandwidth; its
// 32 + 32 products of 16 x 8 x 16 per warp and the softmax of 16 x 16 scores take half of that.  Batches with many short
// items live off the hand-over between items: with every warp looking its items up and fetching their queries itself, an
// item cost about 1.5 us on top of its tiles (16 sequences of up to 1024 keys behind 2048, 32 heads: 59 us against a floor of
// 27; now 34: 28 in this kernel, 6 from its end to the joining kernel's).
#include "attention.cuh"

namespace patch {
namespace attn {

constexpr int kRows = kDecodeRows;            // query rows of an item
constexpr int kKeys = kDecodeKeys;
constexpr int kStages = 2;
constexpr int kWarps = 4;                     // consuming warps
constexpr int kThreads = 32 * (kWarps + 1);

template <int D> struct Cfg {
    static constexpr uint32_t kOperandBytes = kKeys * D * 2;
    static constexpr uint32_t kStageBytes = 2 * kOperandBytes;
    static constexpr uint32_t kQPitch = D * 2 + 16;                          // bytes; eight rows of a fragment fall into different banks
    static constexpr uint32_t kQBytes = kRows * kQPitch;
    static constexpr int kJoinPitch = D + 8;                                 // floats, likewise
    static constexpr uint32_t kQOffset = kStages * kStageBytes;
    static constexpr uint32_t kJoinOffset = kQOffset + kStages * kQBytes;
    static constexpr uint32_t kJoinBytes = kWarps * kRows * kJoinPitch * 4;
    static constexpr uint32_t kMlOffset = kJoinOffset + kJoinBytes;          // (m, l) of every warp and row
    static constexpr uint32_t kNoteOffset = kMlOffset + kWarps * kRows * 8;
    static constexpr uint32_t kBarOffset = kNoteOffset + kStages * 32;
    static constexpr uint32_t kCumOffset = kBarOffset + 128;
    static constexpr uint32_t kFixedBytes = kCumOffset + 1024;               // + alignment of the ring
    // The sequences' units and lengths are kept behind that.  Where with both of them two CTAs no longer fit an SM, lengths are not kept but
    // looked up again (in L1): at D = 128 two CTAs fit up to 1231 sequences instead of 615.  616 sequences of up to 1024 keys of 2 heads
    // took 115 us with one CTA per SM, 85 with two; for fewer sequences the look-up costs the launches beside the block kernel 0.6 us.
    static constexpr uint32_t kMostForTwo = 228 * 1024 / 2 - 1024;          // the hardware takes 1 KB for each CTA
    __host__ __device__ static constexpr bool keeps_lengths(int B) { return kFixedBytes + uint32_t(2 * B + 1) * 4 <= kMostForTwo; }
    static constexpr uint32_t smem_bytes(int B) { return kFixedBytes + uint32_t(keeps_lengths(B) ? 2 * B + 1 : B + 1) * 4; }
};
// What a stage holds.
struct Note { int slot, key0, keys, rows, block, flags, pad[2]; };
// first / last tile of the CTA's share of an item; the sequence's own keys; no tile: the end; first tile of the prefix's or the own keys
constexpr int kFirst = 1, kLast = 2, kOwn = 4, kEnd = 8, kTurns = 16;
static_assert(sizeof(Note) == 32, "note");

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr) : "memory");
}
// c[16 x 8] += a[16 x 16] b[16 x 8]
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// A warp's part of an item: 16 query rows against its 16 keys of every tile.
template <int D> struct Rows {
    using C = Cfg<D>;
    uint32_t qa[D / 16][4];
    float o[D / 8][4], m0, m1, l0, l1;
    int see0, see1;                                  // keys that the lane's rows g and g + 8 see
    int g, t4, warp;
    uint32_t k_at, k_sw, k_c, v_at, v_sw, v_c, half_bytes;

    // a copy brings 2^rows_log2 rows of one page
    __device__ __forceinline__ Rows(int warp_, int lane, int rows_log2) : m0(-INFINITY), m1(-INFINITY), l0(0.0f), l1(0.0f), see0(0), see1(0) {
        warp = warp_;
        g = lane >> 2;
        t4 = lane & 3;
        // address of this lane's row of a 16 x 16 block of keys (K: lanes 0..7 keys 0..7 at element 0, 8..15 keys 0..7 at element 8,
        // 16..31 keys 8..15; V: lanes 0..15 keys 0..15 at element 0, 16..31 at element 8)
        const int krow = warp * 16 + (lane & 7) + ((lane >> 4) << 3), vrow = warp * 16 + (lane & 15);
        const int in_copy = (1 << rows_log2) - 1;
        const uint32_t copy_bytes = uint32_t(D * 2) << rows_log2;
        half_bytes = 128u << rows_log2;
        k_at = uint32_t(krow >> rows_log2) * copy_bytes + uint32_t(krow & in_copy) * 128u;
        k_sw = krow & 7;
        k_c = (lane >> 3) & 1;
        v_at = C::kOperandBytes + uint32_t(vrow >> rows_log2) * copy_bytes + uint32_t(vrow & in_copy) * 128u;
        v_sw = vrow & 7;
        v_c = lane >> 4;
        clear();
    }
    __device__ __forceinline__ void clear() {
        m0 = m1 = -INFINITY;
        l0 = l1 = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    }
    // rows past the item's are whatever lies there: their results are never stored
    __device__ __forceinline__ void queries(uint32_t slot, int lane) {
        const uint32_t at = slot + (lane & 15) * C::kQPitch + (lane >> 4) * 16u;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) ldmatrix4(at + i * 32, qa[i][0], qa[i][1], qa[i][2], qa[i][3]);
    }
    __device__ __forceinline__ void sees(const Problem& p, int first_row, int keys, bool own) {
        see0 = own ? keys - (p.T - 1 - p.token(first_row + g)) : keys;
        see1 = own ? keys - (p.T - 1 - p.token(first_row + g + 8)) : keys;
    }
    // the tile of keys key0 .. of `keys` in the stage at `sb`
    __device__ __forceinline__ void tile(uint32_t sb, int tile_key0, int keys, float scale_log2) {
        const int key0 = tile_key0 + warp * 16, left = keys - key0;          // this warp's keys
        if (left <= 0) return;
        float sc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            uint32_t b0, b1, b2, b3;
            ldmatrix4(sb + k_at + (i >> 2) * half_bytes + (((uint32_t((i & 3) * 2) + k_c) ^ k_sw) << 4), b0, b1, b2, b3);
            mma16816(sc[0], qa[i], b0, b1);
            mma16816(sc[1], qa[i], b2, b3);
        }
        if (key0 + 16 > (see0 < see1 ? see0 : see1)) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int key = key0 + 8 * j + 2 * t4 + e;
                    if (key >= see0) sc[j][e] = -INFINITY;
                    if (key >= see1) sc[j][2 + e] = -INFINITY;
                }
        }
        float x0 = fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[1][0], sc[1][1]));
        float x1 = fmaxf(fmaxf(sc[0][2], sc[0][3]), fmaxf(sc[1][2], sc[1][3]));
        x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 1));
        x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 1));
        x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 2));
        x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 2));
        if (__any_sync(0xFFFFFFFFu, x0 > m0 || x1 > m1)) {
            const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
            const float a0 = n0 == -INFINITY ? 1.0f : ex2(exponent(m0, n0, scale_log2)), a1 = n1 == -INFINITY ? 1.0f : ex2(exponent(m1, n1, scale_log2));
            m0 = n0;
            m1 = n1;
            l0 *= a0;
            l1 *= a1;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) { o[i][0] *= a0; o[i][1] *= a0; o[i][2] *= a1; o[i][3] *= a1; }
        }
        const float c0 = base_of(m0), c1 = base_of(m1);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sc[j][0] = ex2(exponent(sc[j][0], c0, scale_log2));
            sc[j][1] = ex2(exponent(sc[j][1], c0, scale_log2));
            sc[j][2] = ex2(exponent(sc[j][2], c1, scale_log2));
            sc[j][3] = ex2(exponent(sc[j][3], c1, scale_log2));
            l0 += sc[j][0] + sc[j][1];
            l1 += sc[j][2] + sc[j][3];
        }
        const uint32_t pa[4] = {pack2(sc[0][0], sc[0][1]), pack2(sc[0][2], sc[0][3]), pack2(sc[1][0], sc[1][1]), pack2(sc[1][2], sc[1][3])};
        // values past the length may be anything, and 0 times that is not always 0: they are taken as 0
        uint32_t keep0 = 0xFFFFFFFFu, keep1 = 0xFFFFFFFFu;
        if (left < 16) {
            const int k0 = 2 * t4;
            keep0 = (k0 < left ? 0x0000FFFFu : 0u) | (k0 + 1 < left ? 0xFFFF0000u : 0u);
            keep1 = (k0 + 8 < left ? 0x0000FFFFu : 0u) | (k0 + 9 < left ? 0xFFFF0000u : 0u);
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            uint32_t b0, b1, b2, b3;
            ldmatrix4_trans(sb + v_at + (i >> 2) * half_bytes + (((uint32_t((i & 3) * 2) + v_c) ^ v_sw) << 4), b0, b1, b2, b3);
            mma16816(o[2 * i], pa, b0 & keep0, b1 & keep1);
            mma16816(o[2 * i + 1], pa, b2 & keep0, b3 & keep1);
        }
    }
    // this warp's part of `rows` rows into the join buffer
    __device__ __forceinline__ void hand_over(float* join_o, float2* join_ml, int rows) {
        l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 1);
        l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 1);
        l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 2);
        l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 2);
        float* jo = join_o + (warp * kRows + g) * C::kJoinPitch + 2 * t4;
        if (g < rows) {
#pragma unroll
            for (int i = 0; i < D / 8; ++i) *reinterpret_cast<float2*>(jo + 8 * i) = make_float2(o[i][0], o[i][1]);
            if (t4 == 0) join_ml[warp * kRows + g] = make_float2(m0, l0);
        }
        if (g + 8 < rows) {
#pragma unroll
            for (int i = 0; i < D / 8; ++i) *reinterpret_cast<float2*>(jo + 8 * C::kJoinPitch + 8 * i) = make_float2(o[i][2], o[i][3]);
            if (t4 == 0) join_ml[warp * kRows + g + 8] = make_float2(m1, l1);
        }
    }
};
// Four elements (chunk c) of row r from the four warps' parts in the join buffer, and the row's (m, l).
template <int D> __device__ __forceinline__ float4 joined(const float* join_o, const float2* join_ml, int r, int c, float scale_log2, float2& ml_out) {
    float mx = -INFINITY, ls = 0.0f;
#pragma unroll
    for (int q = 0; q < kWarps; ++q) mx = fmaxf(mx, join_ml[q * kRows + r].x);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < kWarps; ++q) {
        const float2 ml = join_ml[q * kRows + r];
        const float a = ml.x == -INFINITY ? 0.0f : ex2(exponent(ml.x, mx, scale_log2));
        const float4 v = *reinterpret_cast<const float4*>(join_o + (q * kRows + r) * Cfg<D>::kJoinPitch + 4 * c);
        ls = fmaf(ml.y, a, ls);
        sum.x = fmaf(v.x, a, sum.x); sum.y = fmaf(v.y, a, sum.y); sum.z = fmaf(v.z, a, sum.z); sum.w = fmaf(v.w, a, sum.w);
    }
    ml_out = make_float2(mx, ls);
    return sum;
}

// AFTER: launched behind the block kernel, which need not have ended when this one starts; it ends after it.
template <int D, bool AFTER>
__global__ void __launch_bounds__(kThreads, 2)
attn_decode_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Problem p, const Line w,
                   const Results to, const double turns) {
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t bar_full = base + C::kBarOffset, bar_empty = bar_full + 8 * kStages;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kBarOffset + 16 * kStages);
    Note* notes = reinterpret_cast<Note*>(smem + C::kNoteOffset);
    int* cum = reinterpret_cast<int*>(smem + C::kCumOffset);
    int* lens = C::keeps_lengths(p.B) ? cum + p.B + 1 : nullptr;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    grid_launch_dependents();                        // the joining kernel waits for this one's end by itself
    if (threadIdx.x == 32) {
        for (int i = 0; i < kStages; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, kWarps); }
        *abort_flag = 0;
        mbar_init_fence();
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
    }
    if (warp == 0) lay_out<false>(p, w, cum, lens);
    else if (warp < kWarps) prefetch_lists(p, w, 32 * (kWarps - 1), threadIdx.x - 32);
    __syncthreads();
    const int total = total_units(w, p, cum);
    // a CTA costs about as much as half a dozen tiles: the second half of the launch's CTAs is for work that is worth them
    int ctas = gridDim.x;
    if (AFTER) ctas = max(ctas / 2, min(ctas, total / 6));
    ctas = min(ctas, total);
    const bool busy = int(blockIdx.x) < ctas;
    // a copy brings the rows of one page that fall into a tile
    const int rows_log2 = p.shift < 6 ? p.shift : 6;
    const uint32_t copy_bytes = uint32_t(D * 2) << rows_log2;

    if (warp == kWarps) {
        // ---------------- producer ----------------
        if (!busy) {
            if (AFTER && blockIdx.x == 0) grid_dependency_wait();
            return;
        }
        const uint64_t policy = l2_policy_evict_first();
        int stage = 0, issued = 0;
        uint32_t phase = 0;
        bool ok = true;
#ifdef PATCH_FAULT_INJECTION
        // test build: a status word holding kInjectMagic makes CTA 1 (CTA 0 may have no tile) announce sixteen bytes more
        // than its first stage will ever receive
        uint32_t inject = 0u;
        if (blockIdx.x == 1 && p.status && *p.status == kInjectMagic) {
            inject = 16u;
            __syncwarp();
            if (lane == 0) *p.status = PATCH_OK;
        }
#else
        constexpr uint32_t inject = 0u;
#endif
        // this lane's page number of an item: entry page0 + lane of its list
        auto fetch = [&](const Share<false>& s, int page0) { return page0 + lane < s.pages() ? s.list()[page0 + lane] : 0; };
        Share<false> s(p, w, cum, lens), ahead(s);
        bool have = s.start(share_start(total, blockIdx.x, ctas, ctas == gridDim.x ? turns : 0.0),
                            share_start(total, blockIdx.x + 1, ctas, ctas == gridDim.x ? turns : 0.0));
        int page0 = have ? int((int64_t(s.t0) * kKeys) >> p.shift) : 0;
        int mine = have ? fetch(s, page0) : 0;
        while (have && ok) {
            if (lane == 0) s.note(to, blockIdx.x);
            // the next item's pages are on their way while this one's tiles are requested
            ahead = s;
            const bool more = ahead.next();
            int mine_ahead = 0;
            if (more) mine_ahead = ahead.b == s.b && page0 == 0 ? mine : fetch(ahead, 0);      // another head: the same list
            for (int i = s.t0; i < s.t1 && ok; ++i) {
                const int64_t key0 = int64_t(i) * kKeys;
                const int first = int(key0 >> p.shift);
                if (first >= page0 + 32) {
                    page0 = first;                   // a tile's pages divide 32, so a tile never straddles a reload
                    mine = fetch(s, page0);
                }
                int page = __shfl_sync(0xFFFFFFFFu, mine, (first - page0) + (p.shift < 6 ? (lane >> 1) & ((kKeys >> rows_log2) - 1) : 0));
                const int keys = s.keys - key0 < kKeys ? int(s.keys - key0) : kKeys;
                const int copies = (keys + (1 << rows_log2) - 1) >> rows_log2;
                if (lane < 2 * copies && (page < 0 || page >= p.num_pages)) {
                    if (p.status) atomicCAS(p.status, PATCH_OK, PATCH_ERR_FORMAT);
                    page = 0;
                }
                // everything is at hand before the slot is: between its release and the copies there are a wait and two instructions
                const uint32_t full = bar_full + 8 * stage, dst = base + stage * C::kStageBytes + (lane & 1) * C::kOperandBytes + (lane >> 1) * copy_bytes;
                const CUtensorMap* map = lane & 1 ? &map_v : &map_k;
                const int row_in_page = p.shift < 6 ? 0 : int(key0 & ((1 << p.shift) - 1));
                const bool opens = i == s.t0, on = lane < 2 * copies;
                const int rows = opens ? min(kRows, s.rows() - s.block * kRows) : 0;
                const uint32_t bytes = uint32_t(copies) * 2u * copy_bytes + uint32_t(rows) * D * 2u;
                ok = __all_sync(0xFFFFFFFFu, issued < kStages || mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status));
                if (!ok) break;
                if (lane == 0) mbar_expect_tx_only(full, bytes + (issued == 0 ? inject : 0u));
                __syncwarp();
                if (on) tma_load_page(dst, map, row_in_page, 0, s.kvh, page, full, policy);
                if (opens && lane >= 16 && lane - 16 < rows) {
                    const int r = s.block * kRows + lane - 16;
                    const int t = p.token(r);
                    const int64_t tok = (s.b < 0 ? 0 : int64_t(s.b) * p.T) + t;
                    tma_bulk_load(base + C::kQOffset + stage * C::kQBytes + (lane - 16) * C::kQPitch,
                                  p.Q + tok * p.ldq + int64_t(s.kvh * p.G + r - t * p.G) * D, D * 2, full, policy);
                }
                if (lane == 0) {                     // the phase ends with this arrival and the bytes: the note is there by then
                    notes[stage] = Note{s.item + int(blockIdx.x), int(key0), s.keys, min(kRows, s.rows() - s.block * kRows), s.block,
                                        (opens ? kFirst : 0) | (i + 1 == s.t1 ? kLast : 0) | (s.b < 0 ? 0 : kOwn), {0, 0}};
                    mbar_arrive(full);
                }
                ++issued;
                if (++stage == kStages) { stage = 0; phase ^= 1u; }
            }
            s = ahead;
            have = more;
            page0 = 0;
            mine = mine_ahead;
        }
        if (lane == 0 && ok && (issued < kStages || mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status))) {
            notes[stage].flags = kEnd;
            mbar_arrive(bar_full + 8 * stage);
        }
        if (AFTER && blockIdx.x == 0) grid_dependency_wait();
        if (*abort_flag) {                           // wait (bounded) for the copies in flight before the CTA may leave
            const uint64_t t0 = global_timer_ns();
            for (int j = issued > kStages ? issued - kStages : 0; j < issued; ++j)
                while (!mbar_try_wait(bar_full + 8 * (j % kStages), uint32_t(j / kStages) & 1u) && global_timer_ns() - t0 < kDrainLimitNs) {}
        }
        return;
    }

    // ---------------- consumers ----------------
    if (!busy) return;
    float* join_o = reinterpret_cast<float*>(smem + C::kJoinOffset);
    float2* join_ml = reinterpret_cast<float2*>(smem + C::kMlOffset);
    int stage = 0;
    uint32_t phase = 0;
    Rows<D> rows(warp, lane, rows_log2);
    bool failed = false;
    for (;;) {
        failed = __any_sync(0xFFFFFFFFu, !mbar_wait(bar_full + 8 * stage, phase, abort_flag, p.status));
        if (failed) break;
        const Note n = notes[stage];
        if (n.flags & kEnd) break;
        if (n.flags & kFirst) {
            rows.queries(base + C::kQOffset + stage * C::kQBytes, lane);
            rows.sees(p, n.block * kRows, n.keys, n.flags & kOwn);
            rows.clear();
        }
        rows.tile(base + stage * C::kStageBytes, n.key0, n.keys, p.scale_log2);
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_empty + 8 * stage);
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
        if (!(n.flags & kLast)) continue;

        // the four warps' parts of this share -> one partial result
        if (barrier_any(false, 1, 32 * kWarps)) return;          // the join buffer is free; true: a warp gave up, all leave
        rows.hand_over(join_o, join_ml, n.rows);
        if (barrier_any(false, 1, 32 * kWarps)) return;
        const Parts& part = n.flags & kOwn ? to.s : to.p;
        const int64_t row0 = int64_t(n.slot) * part.rows;
        for (int i = threadIdx.x; i < n.rows * (D / 4); i += 32 * kWarps) {
            const int r = i / (D / 4), c = i - r * (D / 4);
            float2 ml;
            *reinterpret_cast<float4*>(part.o + (row0 + r) * D + 4 * c) = joined<D>(join_o, join_ml, r, c, p.scale_log2, ml);
            if (c == 0) part.ml[row0 + r] = ml;
        }
    }
    if (failed) barrier_any(true, 1, 32 * kWarps);
}

// Small problems, in one launch and without partial results in memory: a cluster of CTAs owns a block of one sequence's rows of a key
// head, its CTAs take equal parts of the tiles of the prefix and of the sequence's own keys, and join in distributed shared memory.  The
// prefix is read by every sequence (from L2 after the first), which is cheap as long as all there is to read is a few tiles per CTA:
// one sequence behind 128 keys of the 7B shape 8.3 us -> 5.2 with its inputs in L2.  What is left is one chain: barriers, page numbers, a tile from HBM, its products, two joins.
template <int D>
__global__ void __launch_bounds__(kThreads, 2)
attn_direct_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Problem p, const int split,
                   __nv_bfloat16* __restrict__ O, const int64_t ldo, float* __restrict__ lse) {
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t bar_full = base + C::kBarOffset, bar_empty = bar_full + 8 * kStages;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kBarOffset + 16 * kStages);
    Note* notes = reinterpret_cast<Note*>(smem + C::kNoteOffset);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int item = blockIdx.x / split, rank = int(cluster_ctarank()), blocks = (p.T * p.G + kRows - 1) / kRows;
    const int b = item / (p.Hkv * blocks), head_block = item - b * p.Hkv * blocks, kvh = head_block / blocks, row0 = (head_block - kvh * blocks) * kRows;
    const int rows_n = min(kRows, p.T * p.G - row0);
    const int rows_log2 = p.shift < 6 ? p.shift : 6;
    const uint32_t copy_bytes = uint32_t(D * 2) << rows_log2;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, kWarps); }
        *abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == kWarps && lane == 0) { tma_prefetch_map(&map_k); tma_prefetch_map(&map_v); }
    const int own_keys = warp == kWarps ? suffix_len(p, b) : 0;
    __syncthreads();

    if (warp == kWarps) {
        const uint64_t policy = l2_policy_evict_first();
        const int tiles_p = p.prefix_len / kKeys + (p.prefix_len % kKeys != 0), tiles = tiles_p + own_keys / kKeys + (own_keys % kKeys != 0);
        const int t0 = tiles * rank / split, t1 = tiles * (rank + 1) / split;
        int stage = 0, issued = 0, page0 = -64, mine = 0;
        uint32_t phase = 0;
        bool ok = true;
#ifdef PATCH_FAULT_INJECTION
        uint32_t inject = 0u;                        // as above, in CTA 0
        if (blockIdx.x == 0 && p.status && *p.status == kInjectMagic) {
            inject = 16u;
            __syncwarp();
            if (lane == 0) *p.status = PATCH_OK;
        }
#else
        constexpr uint32_t inject = 0u;
#endif
        for (int i = t0; i < t1 && ok; ++i) {
            const bool own = i >= tiles_p, opens = i == t0, turns = opens || i == tiles_p;
            const int64_t key0 = int64_t(own ? i - tiles_p : i) * kKeys;
            const int keys = own ? own_keys : p.prefix_len, first = int(key0 >> p.shift);
            if (turns || first >= page0 + 32) {
                const int32_t* list = own ? p.table + b * p.ld_table : p.prefix_pages;
                page0 = first;
                mine = page0 + lane < int((int64_t(keys) + (1 << p.shift) - 1) >> p.shift) ? list[page0 + lane] : 0;
            }
            int page = __shfl_sync(0xFFFFFFFFu, mine, (first - page0) + (p.shift < 6 ? (lane >> 1) & ((kKeys >> rows_log2) - 1) : 0));
            const int copies = int(min(int64_t(kKeys), keys - key0) + (1 << rows_log2) - 1) >> rows_log2;
            const bool on = lane < 2 * copies;
            if (on && (page < 0 || page >= p.num_pages)) {
                if (p.status) atomicCAS(p.status, PATCH_OK, PATCH_ERR_FORMAT);
                page = 0;
            }
            const uint32_t full = bar_full + 8 * stage, dst = base + stage * C::kStageBytes + (lane & 1) * C::kOperandBytes + (lane >> 1) * copy_bytes;
            ok = __all_sync(0xFFFFFFFFu, issued < kStages || mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status));
            if (!ok) break;
            if (lane == 0) mbar_expect_tx_only(full, uint32_t(copies) * 2u * copy_bytes + (opens ? uint32_t(rows_n) * D * 2u : 0u) + (issued == 0 ? inject : 0u));
            __syncwarp();
            if (on) tma_load_page(dst, lane & 1 ? &map_v : &map_k, p.shift < 6 ? 0 : int(key0 & ((1 << p.shift) - 1)), 0, kvh, page, full, policy);
            if (opens && lane >= 16 && lane - 16 < rows_n) {
                const int r = row0 + lane - 16, t = p.token(r);
                tma_bulk_load(base + C::kQOffset + stage * C::kQBytes + (lane - 16) * C::kQPitch,
                              p.Q + (int64_t(b) * p.T + t) * p.ldq + int64_t(kvh * p.G + r - t * p.G) * D, D * 2, full, policy);
            }
            if (lane == 0) {
                notes[stage] = Note{0, int(key0), keys, rows_n, 0, (opens ? kFirst : 0) | (turns ? kTurns : 0) | (own ? kOwn : 0), {0, 0}};
                mbar_arrive(full);
            }
            ++issued;
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        if (lane == 0 && ok && (issued < kStages || mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status))) {
            notes[stage].flags = kEnd;
            mbar_arrive(bar_full + 8 * stage);
        }
        if (*abort_flag) {
            const uint64_t start = global_timer_ns();
            for (int j = issued > kStages ? issued - kStages : 0; j < issued; ++j)
                while (!mbar_try_wait(bar_full + 8 * (j % kStages), uint32_t(j / kStages) & 1u) && global_timer_ns() - start < kDrainLimitNs) {}
        }
        __syncwarp();
    } else {
        float* join_o = reinterpret_cast<float*>(smem + C::kJoinOffset);
        float2* join_ml = reinterpret_cast<float2*>(smem + C::kMlOffset);
        int stage = 0;
        uint32_t phase = 0;
        Rows<D> rows(warp, lane, rows_log2);
        bool failed = false;
        for (;;) {
            failed = __any_sync(0xFFFFFFFFu, !mbar_wait(bar_full + 8 * stage, phase, abort_flag, p.status));
            if (failed) break;
            const Note n = notes[stage];
            if (n.flags & kEnd) break;
            if (n.flags & kFirst) rows.queries(base + C::kQOffset + stage * C::kQBytes, lane);
            if (n.flags & kTurns) rows.sees(p, row0, n.keys, n.flags & kOwn);
            rows.tile(base + stage * C::kStageBytes, n.key0, n.keys, p.scale_log2);
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_empty + 8 * stage);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        rows.hand_over(join_o, join_ml, rows_n);
        if (!barrier_any(failed, 1, 32 * kWarps)) {
            // this CTA's part, where the first stage was
            float* part_o = reinterpret_cast<float*>(smem);
            float2* part_ml = reinterpret_cast<float2*>(smem + kRows * D * 4);
            for (int i = threadIdx.x; i < rows_n * (D / 4); i += 32 * kWarps) {
                const int r = i / (D / 4), c = i - r * (D / 4);
                float2 ml;
                *reinterpret_cast<float4*>(part_o + r * D + 4 * c) = joined<D>(join_o, join_ml, r, c, p.scale_log2, ml);
                if (c == 0) part_ml[r] = ml;
            }
        }
    }
    __syncwarp();
    cluster_sync_all();                              // also where a wait ran out: every thread of the cluster comes here
    if (warp < kWarps) {
        for (int i = rank * 32 * kWarps + threadIdx.x; i < rows_n * (D / 4); i += split * 32 * kWarps) {
            const int r = i / (D / 4), c = i - r * (D / 4);
            float m = -INFINITY, l = 0.0f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int q = 0; q < split; ++q) {
                float2 ml;
                float4 v;
                asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(ml.x), "=f"(ml.y) : "r"(map_to_rank(base + kRows * D * 4 + r * 8, q)) : "memory");
                asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(map_to_rank(base + r * D * 4 + c * 16, q)) : "memory");
                if (ml.y == 0.0f) continue;          // saw nothing (a row of NaN has seen something: its sum is NaN)
                const float mx = fmaxf(m, ml.x), a = m == -INFINITY ? 0.0f : ex2(exponent(m, mx, p.scale_log2)), f = ex2(exponent(ml.x, mx, p.scale_log2));
                acc.x = acc.x * a + v.x * f; acc.y = acc.y * a + v.y * f; acc.z = acc.z * a + v.z * f; acc.w = acc.w * a + v.w * f;
                l = l * a + ml.y * f;
                m = mx;
            }
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;       // nothing seen: 0
            const int t = p.token(row0 + r), head = kvh * p.G + row0 + r - t * p.G;
            const int64_t tok = int64_t(b) * p.T + t;
            *reinterpret_cast<uint2*>(O + tok * ldo + int64_t(head) * D + 4 * c) = make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
            if (lse && c == 0) lse[tok * (p.Hkv * p.G) + head] = l == 0.0f ? -INFINITY : (m * p.scale_log2 + log2f(l)) * 0.6931471805599453f;
        }
    }
    __syncwarp();
    cluster_sync_all();                              // nobody leaves while a peer may still read its shared memory
}

template <int D>
static int launch_direct(const patch_kv_cache_t* c, const Problem& p, int split, __nv_bfloat16* O, int64_t ldo, float* lse, cudaStream_t stream) {
    CUtensorMap mk, mv;
    const int rows = c->page_size < kKeys ? c->page_size : kKeys;
    int rc = make_kv_tensor_map(&mk, c, c->k_dev, rows, D / 64);
    if (!rc) rc = make_kv_tensor_map(&mv, c, c->v_dev, rows, D / 64);
    if (rc) return rc;
    auto kern = attn_direct_kernel<D>;
    static std::atomic<uint64_t> configured{0};
    const int device = current_device();
    if (device >= 0 && !((configured.load(std::memory_order_acquire) >> device) & 1u) &&
        cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return PATCH_ERR_CUDA;
    if ((rc = allow_dynamic_smem(kern, Cfg<D>::kFixedBytes, configured))) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3(unsigned(p.B * p.Hkv * ((p.T * p.G + kRows - 1) / kRows) * split), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = Cfg<D>::kFixedBytes;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(split);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, mk, mv, p, split, O, ldo, lse) == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}
int launch_attn_direct(const patch_kv_cache_t* c, const Problem& p, int split, __nv_bfloat16* O, int64_t ldo, float* lse, cudaStream_t s) {
    return c->D == 128 ? launch_direct<128>(c, p, split, O, ldo, lse, s) : launch_direct<64>(c, p, split, O, ldo, lse, s);
}

template <int D, bool AFTER>
static int launch(const patch_kv_cache_t* c, const Problem& p, const Line& w, const Results& to, cudaStream_t stream) {
    CUtensorMap mk, mv;
    const int rows = c->page_size < kKeys ? c->page_size : kKeys;
    int rc = make_kv_tensor_map(&mk, c, c->k_dev, rows, D / 64);
    if (!rc) rc = make_kv_tensor_map(&mv, c, c->v_dev, rows, D / 64);
    if (rc) return rc;
    auto kern = attn_decode_kernel<D, AFTER>;
    static std::atomic<uint64_t> configured{0};
    if ((rc = allow_dynamic_smem(kern, Cfg<D>::smem_bytes(kMaxBatch), configured))) return rc;
    const int sms = sm_count() < kMaxSms ? sm_count() : kMaxSms;
    if (sms <= 0) return PATCH_ERR_CUDA;
    // Alone, one wave: two CTAs per SM where they fit, else one (two waves of equal shares would follow one another: 2048 sequences of up to
    // 1024 keys of 2 heads 356 us, 336 in one wave).  Beside the block kernel, more and ever smaller shares that run on whatever SMs
    // it leaves free.
    const int ctas = (AFTER ? 4 : Cfg<D>::smem_bytes(p.B) > Cfg<D>::kMostForTwo ? 1 : 2) * sms;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3(unsigned(ctas), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = Cfg<D>::smem_bytes(p.B);
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = AFTER ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, mk, mv, p, w, to, AFTER ? 0.25 / ctas / ctas : 0.0) == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}

int launch_attn_decode(const patch_kv_cache_t* c, const Problem& p, const Line& w, const Results& to, bool after_block, cudaStream_t s) {
    if (c->D == 128) return after_block ? launch<128, true>(c, p, w, to, s) : launch<128, false>(c, p, w, to, s);
    return after_block ? launch<64, true>(c, p, w, to, s) : launch<64, false>(c, p, w, to, s);
}

}  // namespace attn
}  // namespace patch
