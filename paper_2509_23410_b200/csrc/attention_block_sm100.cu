// Attention over the paged cache for items of more than 16 query rows: the batch's rows of one key head against the shared prefix,
// or a sequence's many tokens (a prompt, drafted tokens) against its own keys (the rule is in attention.cu; public header:
// patch_prefix_attention; the work list and the partial results are described in attention.cuh).
//
// Mathematics.  As in the decode kernel: running maximum m, sum l and unnormalised output o of every row, fp32, probabilities
// 2^((s - m) scale).  Any m serves as long as nothing overflows, so it is the maximum of the row's first tile and is raised only when half
// a tile's sum of probabilities passes 256: the sum is needed anyway, no maximum is taken of the other tiles, and the accumulator is rarely
// rescaled.  (The relative rounding of the bf16 probabilities does not depend on their size.)
//
// Kernel.  One CTA per SM, an item is at most 128 query rows, a tile 128 keys; two streams x = 0, 1 take every second tile with the same
// rows:
//     S_x = Q K^T (shared x shared -> TMEM),  P_x = 2^((S_x - m_x) scale) (TMEM -> registers -> TMEM, over S_x),  O_x += P_x V (TMEM x shared)
// so that one stream multiplies while the other is in its softmax; the two results are joined in TMEM at the end.  (256 rows to an
// item, a stream for each half, reads the keys once instead of twice, the second time from L2, but was the slower one
// throughout: 52 us against 44 for 256 rows and 32768 keys of 8 heads, 76 against 74 for 512 rows.)
//   warp 0       producer: tiles of keys and values, one TMA box per page and 64-element half, into a ring of 32 KB stages (D = 128),
//                as many as fit beside the query tiles
//   warp 1       issues the MMAs; zeroes the rows of V past the item's last key (a probability of 0 times whatever the
//                cache holds there is not always 0)
//   warps 4..7   softmax of stream 0, one thread per row; warps 8..11 stream 1.  They also bring an item's query rows into the
//                swizzled layout (any head count per key head, any row pitch) and write its partial result, half of the columns each.
// What bounds it: a tile's 64 KB of keys and values take an SM 2 850 cycles of HBM, its two products 1 024 and its exponentials 1 024,
// but a stream's tile is a chain -- scores, softmax, products -- of 4 000 to 5 000 cycles, so two streams need 2 000 to 2 500 a tile: HBM
// bounds one block of 128 rows, the chain more of them.  An item costs 7 000 cycles before its first scores and 4 200 for its result
// (24 items of 320 rows and 4093 keys: 17 us).
// Tried: tiles of 64 keys with two score buffers per stream, so that no stream waits for its own products: 5 600 cycles per 128
// keys and two streams -- twice the MMAs of the scores and twice the waits, and the warp that issues them became the bottleneck.
#include "attention.cuh"
#include "attention_tmem.cuh"

namespace patch {
namespace attn {
namespace blk {

constexpr int kKeys = kBlockKeys;
constexpr int kMaxRing = 8;
constexpr int kThreads = 384;
constexpr uint32_t kTmemCols = 512;                   // S_x at 128 x, O_x at 256 + 128 x

template <int D> struct Cfg {
    static constexpr uint32_t kAtom = kKeys * 128;    // 64 elements of every key
    static constexpr uint32_t kQAtom = 128 * 128;     // 64 elements of every query row
    static constexpr uint32_t kTile = kKeys * D * 2;  // one operand of a key tile = one ring stage
    static constexpr uint32_t kQTile = 128 * D * 2;
    static constexpr uint32_t kBarBytes = 256;
};
// Shared memory: [ring | query tile | barriers | units and lengths of the sequences, where the kernel has suffix items].
struct Room { int ring; uint32_t q, bars, cum, bytes; };
template <int D>
static Room room_of(const Line& w, int B) {
    using C = Cfg<D>;
    Room r;
    const uint32_t cum = w.blocks_s ? uint32_t(2 * B + 1) * 4 : 0, rest = C::kQTile + C::kBarBytes + cum + 1024;
    r.ring = int((227u * 1024 - rest) / C::kTile);
    if (r.ring > kMaxRing) r.ring = kMaxRing;
    r.q = r.ring * C::kTile;
    r.bars = r.q + C::kQTile;
    r.cum = r.bars + C::kBarBytes;
    r.bytes = rest + r.ring * C::kTile;
    return r;
}

// How many SMs the block kernel takes where the decode kernel has the suffixes.  Together they are done no sooner than HBM has
// delivered the keys and values and the SMs have done their cycles; with as many SMs as its own cycles need in that time, the block
// kernel ends with the decode kernel, which streams from the other SMs meanwhile -- one is short of arithmetic, the other of
// bandwidth.  Cycles measured: 2 000 for a tile, 3 300 where HBM is waited for (one block of rows), 11 000 for an
// item's queries and result (left out, 16 sequences of 40 heads behind 4 keys took 167 us instead of 62: forty items on four SMs),
// 700 for a tile of the decode kernel (two CTAs share its latencies; each sequence's keys are counted once, though for 17 to 64 rows of
// a sequence the decode kernel walks them once per 16 rows, from L2: its work is then taken for less than it is); bandwidth in bytes per cycle of 6.5 TB/s at 1.9 GHz.  64
// sequences behind 32768 keys (8 key heads): 80 us against 101 with the block kernel on all SMs first.
template <int D>
__device__ __forceinline__ int sms_beside_decode(const Problem& p, const Line& w, float keys, int sms) {
    const float heads = float(p.Hkv);
    const float mine = heads * (w.tiles_p * (w.blocks_p == 1 ? 3300.0f : 2000.0f * w.blocks_p) + 11000.0f * w.blocks_p);
    const float theirs = heads * keys / kDecodeKeys * 700.0f;
    const float bytes = heads * (keys + float(p.prefix_len)) * D * 4.0f;
    const float time = fmaxf(bytes / 3420.0f, (mine + theirs) / sms);
    return max(1, min(sms, int(ceilf(mine / time))));
}
}  // namespace blk

template <int D, bool STEPS>
__global__ void __launch_bounds__(blk::kThreads, 1)
attn_block_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Problem p, const Line w,
                  const Results to, const blk::Room room, const bool share_gpu) {
    using namespace blk;
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - smem_u32(smem_raw));
    const int ring = room.ring;
    // per stream x, at 8 x: bar_s scores, bar_p probabilities (the second half's at 16 + 8 x), bar_h product of the first half
    const uint32_t bar_full = base + room.bars, bar_empty = bar_full + 8 * kMaxRing, bar_q = bar_empty + 8 * kMaxRing, bar_s = bar_q + 8,
                   bar_p = bar_s + 16, bar_h = bar_p + 32, bar_o = bar_h + 16;
    uint32_t* misc = reinterpret_cast<uint32_t*>(smem + room.bars + 224);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 1);
    float* own_keys = reinterpret_cast<float*>(misc + 2);
    int* cum = reinterpret_cast<int*>(smem + room.cum);
    int* lens = cum + p.B + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    grid_launch_dependents();
    if (threadIdx.x == 32) {
        for (int i = 0; i < ring; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
        mbar_init(bar_q, 8);                                   // one arrival per softmax warp
        for (int x = 0; x < 2; ++x) { mbar_init(bar_s + 8 * x, 1); mbar_init(bar_p + 8 * x, 4); mbar_init(bar_p + 16 + 8 * x, 4); mbar_init(bar_h + 8 * x, 1); }
        mbar_init(bar_o, 1);
        *abort_flag = 0;
        mbar_init_fence();
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
    }
    if (warp == 0) {
        const float keys = float(lay_out<STEPS>(p, w, cum, lens));
        if (lane == 0) *own_keys = keys;
    }
    if (warp == 2) tmem_alloc(smem_u32(misc), kTmemCols);
    if (warp >= 4) prefetch_lists(p, w, 256, threadIdx.x - 128);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *misc;

    // Shares: where every prefix item can have two CTAs or more to itself, as many for each and equal parts of its tiles (an item
    // that a CTA has to share with another one costs it queries and a result twice); else equal stretches of the line.
    Line line = w;
    const int sms = share_gpu ? sms_beside_decode<D>(p, w, *own_keys, gridDim.x) : int(gridDim.x), items = p.Hkv * w.blocks_p;
    const bool aligned = !w.blocks_s && 2 * items <= sms;
    if (aligned) line.cost = 0;
    const int total = total_units(line, p, cum), each = aligned ? min(sms / items, w.tiles_p) : 0;
    const int ctas = aligned ? each * items : min(total, sms);
    auto start_of = [&](int c) {
        if (!aligned) return share_start(total, c, ctas, 0.0);
        const int item = c / each;
        return item * w.tiles_p + share_start(w.tiles_p, c - item * each, each, 0.0);
    };
    const bool busy = int(blockIdx.x) < ctas;
    const int u0 = busy ? start_of(blockIdx.x) : 0, u1 = busy ? start_of(blockIdx.x + 1) : 0;
    Share<STEPS> s(p, line, cum, lens);

    if (warp == 0) {
        // ---------------- producer: K0 K1, then V0 K2 V1 K3 ... as they are consumed ----------------
        const uint64_t policy = l2_policy_evict_first();
        const int rows_log2 = p.shift < 7 ? p.shift : 7;       // rows of a box: what one page gives to a tile
        const uint32_t box_bytes = 128u << rows_log2;
        int stage = 0, issued = 0;
        uint32_t phase = 0;
        bool ok = true;
#ifdef PATCH_FAULT_INJECTION
        uint32_t inject = 0u;                                  // as in the decode kernel
        if (blockIdx.x == 0 && p.status && *p.status == kInjectMagic) {
            inject = 16u;
            __syncwarp();
            if (lane == 0) *p.status = PATCH_OK;
        }
#else
        constexpr uint32_t inject = 0u;
#endif
        for (bool have = s.start(u0, u1); have && ok; have = s.next()) {
            if (lane == 0) s.note(to, blockIdx.x);
            const int n_pages = s.pages();
            const int n = s.t1 - s.t0;
            // page numbers of the item's K tiles and V tiles, one per lane; the two run two tiles apart
            int at[2] = {-64, -64}, mine[2] = {0, 0};
            auto load = [&](int i, int v) {                    // tile i of the share, v = 0: keys, 1: values
                const int64_t key0 = int64_t(s.t0 + i) * kKeys;
                const int first = int(key0 >> p.shift);
                if (first >= at[v] + 32 || at[v] < 0) {
                    at[v] = first;
                    mine[v] = first + lane < n_pages ? s.list()[first + lane] : 0;
                }
                const int box = lane >> 1;                     // lane: box of the tile, half
                int page = __shfl_sync(0xFFFFFFFFu, mine[v], (first - at[v]) + (p.shift < 7 ? box & ((kKeys >> rows_log2) - 1) : 0));
                const int keys = s.keys - key0 < kKeys ? int(s.keys - key0) : kKeys;
                const int boxes = (keys + (1 << rows_log2) - 1) >> rows_log2;
                const bool on = box < boxes && (lane & 1) < D / 64;
                if (on && (page < 0 || page >= p.num_pages)) {
                    if (p.status) atomicCAS(p.status, PATCH_OK, PATCH_ERR_FORMAT);
                    page = 0;
                }
                // everything is at hand before the slot is
                const uint32_t full = bar_full + 8 * stage, dst = base + stage * C::kTile + (lane & 1) * C::kAtom + box * box_bytes;
                const CUtensorMap* map = v ? &map_v : &map_k;
                const int row_in_page = p.shift < 7 ? 0 : int(key0 & ((1 << p.shift) - 1));
                ok = __all_sync(0xFFFFFFFFu, issued < ring || mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status));
                if (!ok) return;
                if (lane == 0) mbar_expect_tx(full, uint32_t(boxes) * uint32_t(D / 64) * box_bytes + (issued == 0 ? inject : 0u));
                __syncwarp();
                if (on) tma_load_page(dst, map, row_in_page, lane & 1, s.kvh, page, full, policy);
                ++issued;
                if (++stage == ring) { stage = 0; phase ^= 1u; }
            };
            for (int i = 0; i < 2 && i < n && ok; ++i) load(i, 0);
            for (int i = 0; i < n && ok; ++i) {
                load(i, 1);
                if (i + 2 < n && ok) load(i + 2, 0);
            }
        }
        if (*abort_flag) {
            const uint64_t t0 = global_timer_ns();
            for (int j = issued > ring ? issued - ring : 0; j < issued; ++j)
                while (!mbar_try_wait(bar_full + 8 * (j % ring), uint32_t(j / ring) & 1u) && global_timer_ns() - t0 < kDrainLimitNs) {}
        }
    } else if (warp == 1) {
        // ---------------- MMAs ----------------
        constexpr uint32_t idesc_s = instr_desc(kKeys, false), idesc_o = instr_desc(D, false) | (1u << 16);      // V is MN-major
        int stage = 0;
        uint32_t phase = 0, phase_q = 0, phase_p = 0;          // phase_p: bit x
        bool ok = true;
        auto wait = [&](uint32_t bar, uint32_t parity) {
            ok = mbar_wait(bar, parity, abort_flag, p.status) && ok;
            tc_fence_after();
        };
        auto advance = [&] { if (++stage == ring) { stage = 0; phase ^= 1u; } };
        auto scores = [&](int x, uint32_t q_tile, uint32_t k_tile) {
            const uint64_t dq = desc_kmajor_sw128(q_tile), dk = desc_kmajor_sw128(k_tile);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                mma_dense(tmem + 128u * x, dq + uint64_t(((ks >> 2) * C::kQAtom + (ks & 3) * 32) >> 4),
                          dk + uint64_t(((ks >> 2) * C::kAtom + (ks & 3) * 32) >> 4), idesc_s, ks != 0);
            mma_commit(bar_s + 8 * x);
        };
        auto outputs = [&](int x, uint32_t v_tile, bool first, int half) {          // of 64 keys
            const uint64_t dv = desc_mnmajor_sw128(v_tile + half * 64 * 128, C::kAtom);
#pragma unroll
            for (int ks = 0; ks < kKeys / 32; ++ks)
                mma_ta(tmem + 256u + 128u * x, tmem + 128u * x + 32u * half + 8u * ks, dv + uint64_t((ks * 2048) >> 4), idesc_o, !(first && ks == 0));
        };
        // One thread runs an item from its first tile to its last (a vote of the warp at every wait cost 200 to 400 cycles each);
        // only a tile with rows past the last key, an item's last, brings the warp together.  Loops stay rolled: this warp's few
        // instructions compete with the softmax warps' for the instruction cache.
        for (bool have = s.start(u0, u1); have && ok; have = s.next()) {
            const int n = s.t1 - s.t0, valid = s.keys - (s.t1 - 1) * kKeys;          // valid: rows of the last tile
            const uint32_t q_tile = base + room.q;
            const bool leader = elect_one();
            int i = -2;                                        // tile whose products are next; below 0: scores only
            uint32_t v_stage = 0;
            if (leader) wait(bar_q, phase_q);
            phase_q ^= 1u;
            for (bool zeroed = valid >= kKeys;; zeroed = true) {
                if (leader) {
#pragma unroll 1
                    for (; i < n && ok; ++i) {
                        const int x = i & 1;
                        if (i >= 0) {
                            if (i + 1 < n || !zeroed || valid >= kKeys) {            // else the tile is here and its rows are zeroed
                                wait(bar_full + 8 * stage, phase);
                                v_stage = stage;
                                advance();
                            }
                            if (i + 1 == n && !zeroed) break;
#pragma unroll 1
                            for (int half = 0; half < 2 && ok; ++half) {
                                wait(bar_p + 16 * half + 8 * x, (phase_p >> x) & 1u);
                                if (ok) outputs(x, base + v_stage * C::kTile, i < 2 && half == 0, half);
                                if (ok && half == 0) mma_commit(bar_h + 8 * x);
                            }
                            phase_p ^= 1u << x;
                            if (ok) mma_commit(bar_empty + 8 * v_stage);     // (a tile that was not waited for is not the producer's to load again)
                        }
                        if (i + 2 < n) {                       // the scores of the tile that takes this one's place
                            wait(bar_full + 8 * stage, phase);
                            if (ok) {
                                scores(x, q_tile, base + stage * C::kTile);
                                mma_commit(bar_empty + 8 * stage);
                            }
                            advance();
                        }
                    }
                    if (ok && zeroed) mma_commit(bar_o);
                }
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (zeroed || !ok) break;
                // rows past the last key: zeros
                v_stage = __reduce_max_sync(0xFFFFFFFFu, v_stage);
                for (int j = valid * (D / 8) + lane; j < kKeys * (D / 8); j += 32) {
                    const int r = j / (D / 8), c = j - r * (D / 8);
                    *reinterpret_cast<uint4*>(smem + v_stage * C::kTile + (c >> 3) * C::kAtom + r * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                fence_async_shared();
                __syncwarp();
            }
        }
    } else if (warp >= 4) {
        // ---------------- softmax: thread = row of the stream ----------------
        const int x = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lanes = uint32_t(quad * 32) << 16;
        const uint32_t t_s = tmem + lanes + 128u * x, t_o = tmem + lanes + 256u + 128u * x;
        float2* ml = reinterpret_cast<float2*>(smem + room.q);       // (m, l) of both streams' rows, where the queries were
        uint32_t phase_s = 0, phase_h = 0, phase_o = 0;
        bool failed = false;
        for (bool have = s.start(u0, u1); have && !failed; have = s.next()) {
            const int n = s.t1 - s.t0, first = s.block * kBlockRows, here = min(kBlockRows, s.rows() - first);
            const bool valid = row < here;
            // query rows into the swizzled layout, 16 of them by every warp, a row (256 bytes at D = 128) by D / 8 neighbouring lanes --
            // a lane per row would touch 32 lines with every load; rows past the item's are zeros
            {
                constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
                const int c = lane & (kLanes - 1), warp_row = 16 * (warp - 4) + lane / kLanes;
                uint8_t* dst = smem + room.q + (c >> 3) * C::kQAtom;
                const __nv_bfloat16* from = p.Q + (s.b < 0 ? 0 : int64_t(s.b) * p.T) * p.ldq + int64_t(s.kvh) * p.G * D + 8 * c;
                uint4 v[16 / kAtOnce];
#pragma unroll
                for (int i = 0; i < 16 / kAtOnce; ++i) {
                    const int rr = first + warp_row + i * kAtOnce, tok = p.token(rr);
                    v[i] = rr < s.rows() ? *reinterpret_cast<const uint4*>(from + tok * p.ldq + int64_t(rr - tok * p.G) * D) : make_uint4(0u, 0u, 0u, 0u);
                }
#pragma unroll
                for (int i = 0; i < 16 / kAtOnce; ++i) *reinterpret_cast<uint4*>(dst + atom_chunk_offset(warp_row + i * kAtOnce, c & 7)) = v[i];
                fence_async_shared();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_q);
            const int see = s.b < 0 ? s.keys : s.keys - (p.T - 1 - p.token(first + row));      // keys the row sees
            float m = -INFINITY, l = 0.0f;
            for (int j = 0; 2 * j + x < n; ++j) {
                failed = __any_sync(0xFFFFFFFFu, !mbar_wait(bar_s + 8 * x, phase_s, abort_flag, p.status));
                if (failed) break;
                phase_s ^= 1u;
                tc_fence_after();
                const int left = see - (s.t0 + 2 * j + x) * kKeys;      // columns the row sees
                const bool partly = __any_sync(0xFFFFFFFFu, left < kKeys);
                if (j == 0) m = row_top(t_s, kKeys / 32, left);
                // The products of the first half of the keys start while the second half is worked on.
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    const uint32_t t_h = t_s + 64u * half;
                    uint32_t pr[32];
                    for (bool raised = false;; raised = true) {
                        const float sum = probabilities(t_h, left - 64 * half, partly, p.scale_log2, base_of(m), pr);
                        if (!__any_sync(0xFFFFFFFFu, raise_maximum(sum, m, raised))) {
                            l += sum;
                            break;
                        }
                        // a higher maximum, and the scores (still in TMEM) once more: then the sum is at most the number of keys
                        const float up = row_top(t_h, 2, left - 64 * half, m), a = up == -INFINITY ? 1.0f : ex2(exponent(m, up, p.scale_log2));
                        m = up;
                        l *= a;
                        if (j == 0 && half == 0) continue;
                        // the scores were issued behind the stream's last product, which is therefore done; the first half's is waited for
                        if (half == 1) {
                            failed = __any_sync(0xFFFFFFFFu, !mbar_wait(bar_h + 8 * x, phase_h, abort_flag, p.status));
                            if (failed) break;
                            tc_fence_after();
                        }
#pragma unroll 1
                        for (int q = 0; q < D / 32; ++q) {
                            uint32_t o[32];
                            tmem_ld32(t_o + 32u * q, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * a);
                            tmem_st32(t_o + 32u * q, o);
                        }
                        tmem_st_wait();
                    }
                    if (failed) break;
                    tmem_st32(t_s + 32u * half, pr);
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_p + 16 * half + 8 * x);
                }
                phase_h ^= 1u;
                if (failed) break;
            }
            if (!failed) failed = !mbar_wait(bar_o, phase_o, abort_flag, p.status);
            phase_o ^= 1u;
            tc_fence_after();
            ml[128 * x + row] = make_float2(m, l);
            if (barrier_any(failed, 1, 256)) { failed = true; break; }
            // ---- the partial result: both streams hold a part of the same rows, each joins half of the columns, a quarter at a time
            // through shared memory (where the queries were) and from there in one copy ----
            const Parts& part = s.b < 0 ? to.p : to.s;
            const int64_t slot = s.item + int64_t(blockIdx.x);
            const float2 a = ml[row], b = ml[128 + row];
            const float mx = fmaxf(a.x, b.x);
            const float fa = a.x == -INFINITY ? 0.0f : ex2(exponent(a.x, mx, p.scale_log2)), fb = b.x == -INFINITY ? 0.0f : ex2(exponent(b.x, mx, p.scale_log2));
            if (valid && x == 0) part.ml[slot * part.rows + row] = make_float2(mx, a.y * fa + b.y * fb);
            barrier_any(false, 1, 256);                        // (m, l) have been read
            constexpr uint32_t kQuarter = 128 * D;             // bytes of 128 rows
            constexpr int kChunks = D / 16;                    // of a row
            uint8_t* const stage = smem + room.q + x * kQuarter;
#pragma unroll 1
            for (int q = 2 * x; q < 2 * x + 2; ++q) {
                uint32_t o[D / 4], o1[D / 4];
                load_quarter(tmem + lanes + 256u + (D / 4) * q, o);
                if (n > 1) load_quarter(tmem + lanes + 384u + (D / 4) * q, o1);
                tmem_ld_wait();
                if (q & 1) {                                   // the first copy has read the buffer
                    if (row == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    barrier_any(false, 2 + x, 128);
                }
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    uint32_t v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[i] = __float_as_uint(__uint_as_float(o[4 * c + i]) * fa + (n > 1 ? __uint_as_float(o1[4 * c + i]) * fb : 0.0f));
                    *reinterpret_cast<uint4*>(stage + row * D + ((c ^ (row & (kChunks - 1))) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
                }
                fence_async_shared();
                barrier_any(false, 2 + x, 128);
                if (row == 0) {
                    float* dst = part.o + (slot * 4 + q) * part.rows * (D / 4);
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(stage)), "r"(uint32_t(here) * D) : "memory");
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
            }
            if (row == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            tc_fence_before();
            if (barrier_any(false, 1, 256)) { failed = true; break; }             // nobody's accumulators are read any more
        }
    }
    if (warp >= 4 && (threadIdx.x & 127) == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");     // results have been written
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 2) tmem_dealloc(tmem, blk::kTmemCols);
}

template <int D, bool STEPS>
static int launch_block(const patch_kv_cache_t* c, const Problem& p, const Line& w, const Results& to, bool share_gpu, cudaStream_t stream) {
    CUtensorMap mk, mv;
    const int rows = c->page_size < blk::kKeys ? c->page_size : blk::kKeys;
    int rc = make_kv_tensor_map(&mk, c, c->k_dev, rows, 1);
    if (!rc) rc = make_kv_tensor_map(&mv, c, c->v_dev, rows, 1);
    if (rc) return rc;
    auto kern = attn_block_kernel<D, STEPS>;
    static std::atomic<uint64_t> configured{0};
    if ((rc = allow_dynamic_smem(kern, 227 * 1024, configured))) return rc;
    const blk::Room room = blk::room_of<D>(w, p.B);
    const int sms = sm_count();
    if (sms <= 0) return PATCH_ERR_CUDA;
    kern<<<sms < kMaxSms ? sms : kMaxSms, blk::kThreads, room.bytes, stream>>>(mk, mv, p, w, to, room, share_gpu);
    return cudaGetLastError() == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}

int launch_attn_block(const patch_kv_cache_t* c, const Problem& p, const Line& w, const Results& to, bool decode_follows, cudaStream_t s) {
    if (w.blocks_s && p.T > kMostLevelTokens)
        return c->D == 128 ? launch_block<128, true>(c, p, w, to, decode_follows, s) : launch_block<64, true>(c, p, w, to, decode_follows, s);
    return c->D == 128 ? launch_block<128, false>(c, p, w, to, decode_follows, s) : launch_block<64, false>(c, p, w, to, decode_follows, s);
}

}  // namespace attn
}  // namespace patch
