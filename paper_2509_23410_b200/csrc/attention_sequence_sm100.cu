// Causal attention within packed sequences on tcgen05 (public header: patch_sequence_attention; mathematics in attention_sequence.cu).
//
// A CTA owns an SM and takes items of 256 query rows of one head and sequence, as two streams of 128 rows that share the tiles of 128 keys:
//     S_x = Q_x K^T (shared x shared -> TMEM),  P_x = 2^((S_x - m_x) scale) (TMEM -> registers -> TMEM, over S_x),  O_x += P_x V (TMEM x shared)
// with the softmax rule of the other attention kernels (softmax_rule.cuh): the maximum is the first tile's and is raised only when half a tile's sum
// passes a limit.
//   warp 0       producer: takes items, their queries and tiles of keys and values by TMA into a ring
//   warp 1       issues the MMAs
//   warp 2       zeros over the values behind a sequence's end
//   warps 4..7   softmax and results of stream 0, one thread per row; warps 8..11 stream 1
// Items are the CTAs of the launch: one that has started takes the place of others that have not (clusterlaunchcontrol), so that the lengths, which
// lie in device memory, balance by themselves and the next item's queries and keys are on their way while the last one's results are written.
//
// What bounds it: the two streams alternate on the tensor cores, and a stream's way from its scores to its probabilities (128 columns a thread: exponential,
// sum, two roundings) is as long as the other one's products, so that neither waits much; what is lost is the end of an item, where stream 1 has the
// tile on the diagonal more (some 5000 cycles in which stream 0 has nothing), and the halves of diagonal tiles that the mask hides.  8191 tokens,
// 32/8 heads, D = 128: 476 us, 1.16 PFLOP/s of visible scores, 0.67 of what a large library product reaches; in a long run the power limit makes 540 of it.
// 16384 tokens of 23 sequences, 40 heads: 237 us, of which tiles that are partly visible make a third more work than the scores that count; 300
// tokens, 32 heads: 12 us, which are a launch and one item.  One stream of 128 rows at a time left the tensor cores idle during the exponentials;
// results through warps of their own, a share of the exponentials as polynomials, and streams that run free of each other's order gave nothing or lost
// (the last: 474 -> 550 us, they fall into step).
#include "attention_sequence.cuh"

namespace patch {
namespace seq {

using namespace attn;
using namespace attn::blk;

namespace fwd {

constexpr int kRows = 256;                   // of an item
constexpr int kKeys = 128;
constexpr int kThreads = 384;
constexpr int kRing = 4;                     // stages of a tile of keys or values
constexpr uint32_t kTmemCols = 512;          // S_x at 128 x, O_x at 256 + 128 x

struct Item { int head, begin, end, first; };         // head < 0: no more

template <int D> struct Cfg {
    static constexpr uint32_t kAtom = 128 * 128;       // 64 elements of 128 rows
    static constexpr uint32_t kTile = 128 * D * 2;
    static constexpr uint32_t kQ = kRing * kTile;      // queries of the two streams
    static constexpr uint32_t kMisc = kQ + 2 * kTile;
    static constexpr uint32_t kBytes = kMisc + 512 + 1024;
};

// shared memory behind the tiles
struct Misc {
    uint64_t full[kRing], empty[kRing];
    uint64_t q_full[2], q_empty[2], s[2], p[4], half[2], o_full[2], o_empty[2];         // p: [half of the keys][stream]
    uint64_t item_full[2], item_empty[2], taken, tail[kRing];
    alignas(16) uint4 answer;                // of the launch control
    Item item[2];
    uint32_t tmem;
    int abort;
};
static_assert(sizeof(Misc) <= 512, "fits behind the tiles");

}  // namespace fwd

template <int D>
__global__ void __launch_bounds__(fwd::kThreads, 1)
sequence_forward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Problem p,
                        const int group, __nv_bfloat16* const o, const int64_t ldo, float* const lse) {
    using namespace fwd;
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - smem_u32(smem_raw));
    Misc& sh = *reinterpret_cast<Misc*>(smem + C::kMisc);
    volatile int* abort_flag = &sh.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 32) {
        for (int i = 0; i < kRing; ++i) { mbar_init(smem_u32(&sh.full[i]), 1); mbar_init(smem_u32(&sh.empty[i]), 1); mbar_init(smem_u32(&sh.tail[i]), 1); }
        for (int x = 0; x < 2; ++x) {
            mbar_init(smem_u32(&sh.q_full[x]), 1);
            mbar_init(smem_u32(&sh.q_empty[x]), 1);
            mbar_init(smem_u32(&sh.s[x]), 1);
            mbar_init(smem_u32(&sh.p[x]), 4);
            mbar_init(smem_u32(&sh.p[2 + x]), 4);
            mbar_init(smem_u32(&sh.half[x]), 1);
            mbar_init(smem_u32(&sh.o_full[x]), 1);
            mbar_init(smem_u32(&sh.o_empty[x]), 4);
            mbar_init(smem_u32(&sh.item_full[x]), 1);
            mbar_init(smem_u32(&sh.item_empty[x]), 10);            // the MMA thread, the mender and eight softmax warps
        }
        mbar_init(smem_u32(&sh.taken), 1);
        sh.abort = 0;
        mbar_init_fence();
        tma_prefetch_map(&map_q);
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
    }
    if (warp == 2) tmem_alloc(smem_u32(&sh.tmem), kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;

    // tiles of keys that stream x of an item needs
    auto tiles_of_stream = [](const Item& it, int x) {
        const int n = it.end - it.begin, first = it.first + 128 * x;
        return first < n ? first / kKeys + 1 : 0;
    };

    if (warp == 0) {
        // ---------------- producer ----------------
        const uint64_t keep = l2_policy_evict_last(), once = l2_policy_evict_first();
        const Order<kRows, false> order(p, p.Hq, group);
        Loader<D, kRing> ring(smem, sh.full, sh.empty, sh.tail, abort_flag, p.status);
        ring.heed(0);
        int items = 0;
        uint32_t used_q = 0, phase_q = 0, phase_taken = 0;                   // used_q, phase_q: bit x
        unsigned at = blockIdx.x;
        for (;;) {
            if (lane == 0) ask_for_next(&sh.answer, &sh.taken);
            __syncwarp();
            if (at == 0) check_starts(p, lane, 32);
            int head;
            const Tile t = order.take(at, head);
            if (t.first >= 0) {
                const Item it = {head, t.begin, t.end, t.first};
                if (items >= 2) ring.wait(sh.item_empty[items & 1], uint32_t((items >> 1) - 1) & 1u);
                if (ring.ok && lane == 0) {
                    sh.item[items & 1] = it;
                    mbar_arrive(smem_u32(&sh.item_full[items & 1]));
                }
                ++items;
                for (int x = 0; x < 2 && ring.ok; ++x) {
                    if (!tiles_of_stream(it, x)) continue;
                    if ((used_q >> x) & 1u) {
                        ring.wait(sh.q_empty[x], (phase_q >> x) & 1u);
                        phase_q ^= 1u << x;
                    }
                    used_q |= 1u << x;
                    if (ring.ok && lane == 0) {
                        mbar_expect_tx(smem_u32(&sh.q_full[x]), C::kTile);
                        tma_tile_load_3d(base + C::kQ + x * C::kTile, &map_q, 0, it.begin + it.first + 128 * x, head * (D / 64), smem_u32(&sh.q_full[x]), once);
                    }
                }
                const int n = max(tiles_of_stream(it, 0), tiles_of_stream(it, 1)), chunk = head / p.G * (D / 64);
                for (int j = 0; j < n && ring.ok; ++j) {
                    const int row = it.begin + j * kKeys;
                    ring.load(&map_k, row, chunk, kKeys, keep);
                    if (ring.ok) ring.load(&map_v, row, chunk, it.end - row, keep);
                }
            }
            // the answer is waited for whatever happened
            const bool before = ring.ok;
            ring.ok = true;
            ring.wait(sh.taken, phase_taken);
            phase_taken ^= 1u;
            const bool more = ring.ok && answered(&sh.answer, at);
            ring.ok = ring.ok && before;
            __syncwarp();
            if (!ring.ok || !more) break;
        }
        if (ring.ok && items >= 2) ring.wait(sh.item_empty[items & 1], uint32_t((items >> 1) - 1) & 1u);
        if (ring.ok && lane == 0) {
            sh.item[items & 1].head = -1;
            mbar_arrive(smem_u32(&sh.item_full[items & 1]));
        }
    } else if (warp == 1) {
        // ---------------- MMAs: one thread ----------------
        constexpr uint32_t idesc_s = instr_desc(kKeys, false), idesc_o = instr_desc(D, false) | (1u << 16);      // V is MN-major
        if (elect_one()) {
            int stage = 0;
            uint32_t phase = 0, phase_q = 0, phase_p = 0, phase_o = 0;      // the latter three: bit x
            bool ok = true, began[2] = {false, false};
            auto wait = [&](uint64_t& bar, uint32_t parity) {
                ok = ok && mbar_wait(smem_u32(&bar), parity, abort_flag, p.status);
                tc_fence_after();
            };
            // (nothing after a wait given up: the producer would announce a copy to a barrier whose last one has not landed)
            auto commit = [&](uint64_t& bar) { if (ok) mma_commit(smem_u32(&bar)); };
            auto advance = [&](int& s, uint32_t& ph) { if (++s == kRing) { s = 0; ph ^= 1u; } };
            auto scores = [&](int x, int k_stage) {
                const uint64_t dq = desc_kmajor_sw128(base + C::kQ + x * C::kTile), dk = desc_kmajor_sw128(base + k_stage * C::kTile);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint64_t off = uint64_t(((ks >> 2) * C::kAtom + (ks & 3) * 32) >> 4);
                    mma_dense(tmem + 128u * x, dq + off, dk + off, idesc_s, ks != 0);
                }
                commit(sh.s[x]);
            };
            auto outputs = [&](int x, int v_stage, bool first, int half) {         // of 64 keys
                const uint64_t dv = desc_mnmajor_sw128(base + v_stage * C::kTile + half * 64 * 128, C::kAtom);
#pragma unroll
                for (int ks = 0; ks < kKeys / 32; ++ks)
                    mma_ta(tmem + 256u + 128u * x, tmem + 128u * x + 32u * half + 8u * ks, dv + uint64_t((ks * 2048) >> 4), idesc_o, !(first && ks == 0));
            };
            for (int item = 0; ok; ++item) {
                wait(sh.item_full[item & 1], uint32_t(item >> 1) & 1u);
                if (!ok) break;
                const Item it = sh.item[item & 1];
                mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
                if (it.head < 0) break;
                const int n[2] = {tiles_of_stream(it, 0), tiles_of_stream(it, 1)}, most = max(n[0], n[1]);
                wait(sh.full[stage], phase);                       // the first tile's scores
                for (int x = 0; x < 2 && ok; ++x) {
                    if (!n[x]) continue;
                    wait(sh.q_full[x], (phase_q >> x) & 1u);
                    phase_q ^= 1u << x;
                    if (ok) scores(x, stage);
                    if (n[x] == 1) commit(sh.q_empty[x]);
                }
                commit(sh.empty[stage]);
                advance(stage, phase);
#pragma unroll 1
                for (int j = 0; j < most && ok; ++j) {
                    const int v_stage = stage;
                    wait(sh.full[v_stage], phase);
                    advance(stage, phase);
                    const bool more = j + 1 < most;
#pragma unroll 1
                    for (int x = 0; x < 2 && ok; ++x) {
                        if (j >= n[x]) continue;
                        if (j == 0) {
                            if (began[x]) {                        // the last item's results have been read
                                wait(sh.o_empty[x], (phase_o >> x) & 1u);
                                phase_o ^= 1u << x;
                            }
                            began[x] = true;
                        }
#pragma unroll 1
                        for (int half = 0; half < 2 && ok; ++half) {
                            wait(sh.p[2 * half + x], (phase_p >> x) & 1u);
                            if (ok) outputs(x, v_stage, j == 0 && half == 0, half);
                            if (half == 0) commit(sh.half[x]);
                        }
                        phase_p ^= 1u << x;
                        if (j + 1 == n[x]) {
                            commit(sh.o_full[x]);
                        } else {
                            wait(sh.full[stage], phase);           // the same tile for both streams
                            if (ok) scores(x, stage);
                            if (j + 2 == n[x]) commit(sh.q_empty[x]);
                        }
                    }
                    commit(sh.empty[v_stage]);
                    if (more) {
                        commit(sh.empty[stage]);
                        advance(stage, phase);
                    }
                }
            }
        }
    } else if (warp == 2) {
        // ---------------- values behind a sequence's end ----------------
        Mender<D, kRing> mender{smem, sh.full, sh.tail, abort_flag, p.status, 1};
        for (int item = 0; mender.ok; ++item) {
            if (!__all_sync(0xFFFFFFFFu, mbar_wait_suspended(smem_u32(&sh.item_full[item & 1]), uint32_t(item >> 1) & 1u, abort_flag, p.status))) break;
            const Item it = sh.item[item & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
            if (it.head < 0) break;
            const int n = max(tiles_of_stream(it, 0), tiles_of_stream(it, 1));
            for (int j = 0; j < n; ++j) {
                mender.next(kKeys);
                mender.next(it.end - it.begin - j * kKeys);
            }
        }
    } else if (warp >= 4) {
        // ---------------- softmax: thread = row of the stream ----------------
        const int x = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lanes = uint32_t(quad * 32) << 16;
        const uint32_t t_s = tmem + lanes + 128u * x, t_o = tmem + lanes + 256u + 128u * x;
        uint32_t phase_s = 0, phase_h = 0, phase_o = 0;
        bool failed = false;
        auto wait = [&](uint64_t& bar, uint32_t parity) {
            failed = __any_sync(0xFFFFFFFFu, !mbar_wait(smem_u32(&bar), parity, abort_flag, p.status)) || failed;
            tc_fence_after();
        };
        for (int item = 0;; ++item) {
            wait(sh.item_full[item & 1], uint32_t(item >> 1) & 1u);
            if (failed) break;
            const Item it = sh.item[item & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
            if (it.head < 0) break;
            const int n = tiles_of_stream(it, x);
            if (!n) continue;
            float m = -INFINITY, l = 0.0f;
            for (int j = 0; j < n; ++j) {
                wait(sh.s[x], phase_s);
                if (failed) break;
                phase_s ^= 1u;
                const bool partly = j == n - 1;                    // the tile on the diagonal
                const int left = partly ? row + 1 : kKeys;         // columns the row sees
                if (j == 0) m = row_top(t_s, 1, left);             // every row sees the first of them
                // The products of the first half of the keys start while the second half is worked on.
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    const uint32_t t_h = t_s + 64u * half;
                    uint32_t pr[32];
                    for (bool raised = false;; raised = true) {
                        const float sum = probabilities(t_h, left - 64 * half, partly, p.scale_log2, base_of(m), pr);
                        const bool raise = raise_maximum(sum, m, raised);
                        if (!__any_sync(0xFFFFFFFFu, raise)) {
                            l += sum;
                            break;
                        }
                        // a higher maximum, and the scores (still in TMEM) once more: then the sum is at most the number of keys.  Rows that need none keep
                        // theirs, factor 1: a row's bits are its own, whatever the warp's other rows hold, which may lie behind the sequence's end
                        const float top = row_top(t_h, 2, left - 64 * half, m), up = raise ? top : m, a = raise ? ex2(exponent(m, up, p.scale_log2)) : 1.0f;
                        m = up;
                        l *= a;
                        if (j == 0 && half == 0) continue;
                        // the scores were issued behind the stream's last product, which is therefore done; the first half's is waited for
                        if (half == 1) {
                            wait(sh.half[x], phase_h);
                            if (failed) break;
                        }
#pragma unroll 1
                        for (int q = 0; q < D / 32; ++q) {
                            uint32_t v[32];
                            tmem_ld32(t_o + 32u * q, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(__uint_as_float(v[c]) * a);
                            tmem_st32(t_o + 32u * q, v);
                        }
                        tmem_st_wait();
                    }
                    if (failed) break;
                    tmem_st32(t_s + 32u * half, pr);
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh.p[2 * half + x]));
                }
                phase_h ^= 1u;
                if (failed) break;
            }
            if (!failed) wait(sh.o_full[x], phase_o);
            if (failed) break;
            phase_o ^= 1u;
            const int r = it.first + 128 * x + row;
            const bool valid = r < it.end - it.begin;
            const float f = 1.0f / l;
            store_rows<D>(t_o, o + int64_t(it.head) * D, ldo, it.begin + it.first + 128 * x + quad * 32, it.end, f);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.o_empty[x]));
            if (valid && lse) lse[int64_t(it.begin + r) * p.Hq + it.head] = m * p.scale + logf(l);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 2) {
        let_land(abort_flag);
        tmem_dealloc(tmem, kTmemCols);
    }
}

template <int D>
static int launch(const Problem& p, __nv_bfloat16* o, int64_t ldo, float* lse, cudaStream_t s) {
    using C = fwd::Cfg<D>;
    CUtensorMap mq, mk, mv;
    int rc = make_x_chunk_tensor_map(&mq, p.q, p.ldq, p.M, int64_t(p.Hq) * D, 128, D / 64);
    if (!rc) rc = make_x_chunk_tensor_map(&mk, p.k, p.ldk, p.M, int64_t(p.Hkv) * D, 128, D / 64);
    if (!rc) rc = make_x_chunk_tensor_map(&mv, p.v, p.ldv, p.M, int64_t(p.Hkv) * D, 128, D / 64);
    if (rc) return rc;
    auto kern = sequence_forward_kernel<D>;
    static std::atomic<uint64_t> configured{0};
    if ((rc = allow_dynamic_smem(kern, C::kBytes, configured))) return rc;
    kern<<<unsigned(most_tiles(p.M, p.B, fwd::kRows) * p.Hq), fwd::kThreads, C::kBytes, s>>>(mq, mk, mv, p, heads_at_once(p.Hkv, int64_t(p.M) * D * 4, most_tiles(p.M, p.B, fwd::kRows) * p.G) * p.G, o, ldo, lse);
    return cudaGetLastError() == cudaSuccess ? PATCH_OK : PATCH_ERR_CUDA;
}
int launch_forward(const Problem& p, int D, __nv_bfloat16* o, int64_t ldo, float* lse, cudaStream_t s) {
    return D == 128 ? launch<128>(p, o, ldo, lse, s) : launch<64>(p, o, ldo, lse, s);
}

}  // namespace seq
}  // namespace patch
