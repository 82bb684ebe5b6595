// Gradient of the causal attention within packed sequences on tcgen05 (public header: patch_sequence_attention_backward; mathematics in
// attention_sequence.cu).
//
// Two kernels, so that every sum has one owner and an order of its own: gq by blocks of 128 queries over their keys (three products a tile), gk and
// gv by blocks of 128 keys of a key head over the queries that see them, head by head of the group (four products a tile).  The scores are computed in
// both, seven products instead of five; the price of sums in fp32 atomics would be an order that changes from call to call, and their traffic.
// A CTA owns an SM; roles, rings and the taking of items are the forward kernel's.  Warps 4..11 do the elementwise part of a tile of 128 x 128,
// a thread 64 columns of a row; warps 12..15 write an item's results while the next one is worked on.
//
//   gq:      S = Q K^T (two buffers), GP = GO V^T,   GS = P (GP - delta) (over S),   GQ += GS K
//            order of the MMAs: GP(j + 1), GQ(j), S(j + 2): the exponentials of j + 1 run beside the first, its GS needs no more than that
//   gk, gv:  S^T = K Q^T,  GP^T = V GO^T (lane = key, column = query),  P^T (shared memory),  GS^T (over GP^T),  GV += P^T GO,  GK += GS^T Q
//            order of the MMAs: S(t + 1) as soon as S(t) is in registers, GV(t), GK(t), GP(t + 1).  (With P^T over S^T, S(t + 1) behind GV(t): the
//            elementwise warps waited 870 of 3140 cycles a tile for it)
// TMEM: 512 columns in both (two of scores or one, one of GP, the accumulators).
//
// What bounds it: in both the chain of a tile through the elementwise warps, beside the tensor cores' part of it.  D = 128: gq 2130 cycles a tile where the products
// take 1536, gk and gv 2800 where they take 2048; D = 64 has half the products and nearly the same times.  Four sequences of 2048, 32 heads, D = 128:
// statistics 29 us, gq 200, gk and gv 278, 505 to 580 together as the power limit allows; 4001 tokens of nine sequences, 32/8 heads, D = 64: 8, 44, 64, 115
// together, the largest items' length and the tiles' hidden parts.
#include "attention_sequence.cuh"

namespace patch {
namespace seq {

using namespace attn;
using namespace attn::blk;

namespace bwd {

constexpr int kRows = 128;                   // of an item and of a tile
constexpr int kThreads = 512;
constexpr uint32_t kTmemCols = 512;

struct Item { int head, begin, end, first; };         // head < 0: no more

template <int D> struct Cfg {
    static constexpr int kRing = D == 128 ? 5 : 8;
    static constexpr uint32_t kAtom = 128 * 128;       // 64 elements of 128 rows
    static constexpr uint32_t kTile = kTileBytes<D>;
    static constexpr uint32_t kOwn = kRing * kTile;    // the item's own two tiles
    static constexpr uint32_t kMisc = kOwn + 2 * kTile;
    static constexpr int kKeyRing = D == 128 ? 4 : 6;  // gk, gv: a tile's room is P^T's
    static constexpr uint32_t kP = kKeyRing * kTile;   // two atoms of 64 queries
    static_assert(kP + 32768 <= kOwn, "the ring's place");
    static constexpr uint32_t kStats = kMisc + 512;    // of two tiles of queries: [lse log2 e: 128 | delta: 128]
    static constexpr uint32_t kBytes = kStats + 2 * 1024;                      // the array itself is aligned: 227 KB leave nothing to round
    static_assert(kBytes <= 227 * 1024, "shared memory of an SM");
};

struct Misc {
    uint64_t full[8], empty[8];
    uint64_t own_full, own_empty, s[2], s_read, gp, p[2], p_read, gs[2], done, read;  // p, gs: by half of the columns; s: by buffer
    uint64_t item_full[2], item_empty[2], stats_full[2], stats_empty[2], taken, tail[8];
    alignas(16) uint4 answer;
    Item item[2];
    uint32_t tmem;
    int abort;
};
static_assert(sizeof(Misc) <= 512, "fits behind the tiles");

__device__ __forceinline__ void init(Misc& sh, int ring, int readers) {
    for (int i = 0; i < ring; ++i) { mbar_init(smem_u32(&sh.full[i]), 1); mbar_init(smem_u32(&sh.empty[i]), 1); mbar_init(smem_u32(&sh.tail[i]), 1); }
    for (int x = 0; x < 2; ++x) {
        mbar_init(smem_u32(&sh.s[x]), 1);
        mbar_init(smem_u32(&sh.p[x]), 4);
        mbar_init(smem_u32(&sh.gs[x]), 4);
        mbar_init(smem_u32(&sh.item_full[x]), 1);
        mbar_init(smem_u32(&sh.item_empty[x]), readers);
        mbar_init(smem_u32(&sh.stats_full[x]), 1);
        mbar_init(smem_u32(&sh.stats_empty[x]), 8);
    }
    mbar_init(smem_u32(&sh.own_full), 1);
    mbar_init(smem_u32(&sh.own_empty), 1);
    mbar_init(smem_u32(&sh.gp), 1);
    mbar_init(smem_u32(&sh.s_read), 8);
    mbar_init(smem_u32(&sh.p_read), 1);
    mbar_init(smem_u32(&sh.done), 1);
    mbar_init(smem_u32(&sh.read), 4);
    mbar_init(smem_u32(&sh.taken), 1);
    sh.abort = 0;
    mbar_init_fence();
}

// D[128 x 128] = A B^T, both K-major tiles of shared memory
template <int D>
__device__ __forceinline__ void product(uint32_t d_tmem, uint32_t a, uint32_t b) {
    const uint64_t da = desc_kmajor_sw128(a), db = desc_kmajor_sw128(b);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        const uint64_t off = uint64_t(((ks >> 2) * Cfg<D>::kAtom + (ks & 3) * 32) >> 4);
        mma_dense(d_tmem, da + off, db + off, instr_desc(128, false), ks != 0);
    }
}
// D[128 x D] (+)= A[128 x 64, bf16 in TMEM] B[64 rows of a tile]
template <int D>
__device__ __forceinline__ void accumulate(uint32_t d_tmem, uint32_t a_tmem, uint32_t b, int half, bool first) {
    const uint64_t db = desc_mnmajor_sw128(b + half * 64 * 128, Cfg<D>::kAtom);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) mma_ta(d_tmem, a_tmem + 8u * ks, db + uint64_t((ks * 2048) >> 4), instr_desc(D, false) | (1u << 16), !(first && ks == 0));
}
// the same with A in shared memory: one atom of 64 columns, K-major
template <int D>
__device__ __forceinline__ void accumulate_from_shared(uint32_t d_tmem, uint32_t a, uint32_t b, int half, bool first) {
    const uint64_t da = desc_kmajor_sw128(a), db = desc_mnmajor_sw128(b + half * 64 * 128, Cfg<D>::kAtom);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) mma_dense(d_tmem, da + uint64_t((ks * 32) >> 4), db + uint64_t((ks * 2048) >> 4), instr_desc(D, false) | (1u << 16), !(first && ks == 0));
}
// The elementwise warps (4 .. 11) take registers of the others: 256 x 168 + 256 x 88 = 512 x 128, the launch's.  Each by all warps of two (one)
// groups of four.
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 168;"); }
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 88;"); }
// 2^x of a pair
__device__ __forceinline__ f2 powers(f2 x) {
    float a, b;
    un2(x, a, b);
    return mk2(ex2(a), ex2(b));
}

}  // namespace bwd

// (lse log2 e, delta) of every row and head, [Hq][M].  D / 8 lanes to a head of four rows, whose loads are on their way together and whose results fill a
// sector of 32 bytes: bound by the reads of O and GO.
template <int D>
__global__ void __launch_bounds__(256) delta_kernel(const Problem p, const float* lse, float2* stats) {
    constexpr int kLanes = D / 8, kRows = 4, kGroups = 256 / kLanes;
    grid_launch_dependents();                // they wait for what is written here
    const int c = threadIdx.x & (kLanes - 1);
    const int64_t group = int64_t(blockIdx.x) * kGroups + threadIdx.x / kLanes, row = group / p.Hq * kRows;
    const int h = int(group % p.Hq), rows = int(min(int64_t(kRows), p.M - row));      // none or fewer behind the last row
    uint4 a[kRows], b[kRows];
    float l[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (i >= rows) continue;
        a[i] = *reinterpret_cast<const uint4*>(p.o + (row + i) * p.ldo + h * D + 8 * c);
        b[i] = *reinterpret_cast<const uint4*>(p.go + (row + i) * p.ldgo + h * D + 8 * c);
        if (c == 0) l[i] = lse[(row + i) * p.Hq + h];
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t x[4] = {a[i].x, a[i].y, a[i].z, a[i].w}, y[4] = {b[i].x, b[i].y, b[i].z, b[i].w};
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sum = fmaf(__uint_as_float(x[j] << 16), __uint_as_float(y[j] << 16), sum);
            sum = fmaf(__uint_as_float(x[j] & 0xFFFF0000u), __uint_as_float(y[j] & 0xFFFF0000u), sum);
        }
#pragma unroll
        for (int d = kLanes / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (c == 0 && i < rows) stats[int64_t(h) * p.M + row + i] = make_float2(l[i] * 1.44269504f, sum);
    }
}

// ---------------------------------------------------------------------------------------------
// gq
template <int D>
__global__ void __launch_bounds__(bwd::kThreads, 1)
sequence_query_grad_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_go, const __grid_constant__ CUtensorMap map_k,
                           const __grid_constant__ CUtensorMap map_v, const Problem p, const float2* const stats, const int group, __nv_bfloat16* const gq,
                           const int64_t ldgq) {
    using namespace bwd;
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    Misc& sh = *reinterpret_cast<Misc*>(smem + C::kMisc);
    volatile int* abort_flag = &sh.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 32) {
        init(sh, C::kRing, 14);                                    // an item's readers: the MMA thread, the mender, twelve warps
        tma_prefetch_map(&map_q);
        tma_prefetch_map(&map_go);
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
    }
    if (warp == 2) tmem_alloc(smem_u32(&sh.tmem), kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem, t_gp = tmem + 256, t_gq = tmem + 384;      // scores: tmem + 128 (j & 1)

    if (warp >= 4 && warp < 12) {
        take_registers();
        // ---------------- elementwise: thread = row, half of the columns ----------------
        const int half = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lanes = uint32_t(quad * 32) << 16;
        uint32_t phase_s = 0, phase_gp = 0;                        // phase_s: bit of the buffer
        bool failed = false;
        auto wait = [&](uint64_t& bar, uint32_t parity) {
            failed = __any_sync(0xFFFFFFFFu, !mbar_wait(smem_u32(&bar), parity, abort_flag, p.status)) || failed;
            tc_fence_after();
        };
        grid_dependency_wait();              // the statistics
        grid_launch_dependents();            // which the kernel of gk and gv, the next one, then finds as well
        const f2 scale2 = mk2(p.scale_log2, p.scale_log2);
        for (int item = 0;; ++item) {
            wait(sh.item_full[item & 1], uint32_t(item >> 1) & 1u);
            if (failed) break;
            const Item it = sh.item[item & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
            if (it.head < 0) break;
            const int n = it.first / kRows + 1, r = it.first + row;
            const bool valid = r < it.end - it.begin;
            const float2 st = valid ? stats[int64_t(it.head) * p.M + it.begin + r] : make_float2(0.0f, 0.0f);
            const f2 lse2 = mk2(-st.x, -st.x), delta2 = mk2(-st.y, -st.y);
            for (int j = 0; j < n; ++j) {
                const uint32_t t_s = tmem + lanes + 128u * (j & 1) + 64u * half;
                wait(sh.s[j & 1], (phase_s >> (j & 1)) & 1u);
                if (failed) break;
                phase_s ^= 1u << (j & 1);
                const bool partly = j == n - 1;                    // the tile on the diagonal
                const int left = row + 1 - 64 * half;              // columns the row sees there
                uint32_t e[2][32];
                tmem_ld32(t_s, e[0]);
                tmem_ld32(t_s + 32u, e[1]);
                tmem_ld_wait();
                if (partly) {
                    hide(e[0], left);
                    hide(e[1], left - 32);
                }
#pragma unroll
                for (int c = 0; c < 64; c += 2) {
                    float a, b;
                    un2(powers(fma2(mk2(__uint_as_float(e[c >> 5][c & 31]), __uint_as_float(e[c >> 5][(c & 31) + 1])), scale2, lse2)), a, b);
                    e[c >> 5][c & 31] = __float_as_uint(a);
                    e[c >> 5][(c & 31) + 1] = __float_as_uint(b);
                }
                wait(sh.gp, phase_gp);
                if (failed) break;
                phase_gp ^= 1u;
                uint32_t gs[32];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t v[32];
                    tmem_ld32(tmem + lanes + 256u + 64u * half + 32u * i, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        float a, b;
                        un2(mul2(mk2(__uint_as_float(e[i][c]), __uint_as_float(e[i][c + 1])),
                                 add2(mk2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), delta2)), a, b);
                        gs[16 * i + (c >> 1)] = pack2(a, b);
                    }
                }
                if (partly) {                                      // keys after the query, and behind the sequence's end: 0 whatever the values hold there
#pragma unroll
                    for (int c = 0; c < 64; c += 2) {
                        if (c >= left) gs[c >> 1] = 0u;
                        else if (c + 1 >= left) gs[c >> 1] &= 0xFFFFu;
                    }
                }
                tmem_st32(t_s, gs);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.gs[half]));
            }
            if (failed) break;
        }
    } else {
    give_registers();
    if (warp == 0) {
        // ---------------- producer ----------------
        const uint64_t keep = l2_policy_evict_last(), once = l2_policy_evict_first();
        const Order<kRows, false> order(p, p.Hq, group);
        Loader<D, C::kRing> ring(smem, sh.full, sh.empty, sh.tail, abort_flag, p.status);
        ring.heed(0);
        int items = 0;
        uint32_t phase_own = 0, phase_taken = 0;
        unsigned at = blockIdx.x;
        // (The first question waits for the kernel before: a CTA that started beside it would take work from SMs that are about to be free.)
        auto ask = [&] {
            if (lane == 0) ask_for_next(&sh.answer, &sh.taken);
            __syncwarp();
        };
        for (bool first = true;; first = false) {
            if (!first) ask();
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
                if (ring.ok && items >= 1) {
                    ring.wait(sh.own_empty, phase_own);
                    phase_own ^= 1u;
                }
                ++items;
                if (ring.ok && lane == 0) {
                    const uint32_t bar = smem_u32(&sh.own_full);
                    mbar_expect_tx(bar, 2 * C::kTile);
                    tma_tile_load_3d(base + C::kOwn, &map_q, 0, it.begin + it.first, head * (D / 64), bar, once);
                    tma_tile_load_3d(base + C::kOwn + C::kTile, &map_go, 0, it.begin + it.first, head * (D / 64), bar, once);
                }
                __syncwarp();
                const int n = it.first / kRows + 1, chunk = head / p.G * (D / 64);
                for (int j = 0; j < n && ring.ok; ++j) {
                    const int row = it.begin + j * kRows;
                    ring.load(&map_k, row, chunk, it.end - row, keep);
                    if (ring.ok) ring.load(&map_v, row, chunk, kRows, keep);
                }
            }
            if (first) {
                grid_dependency_wait();
                ask();
            }
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
        if (elect_one()) {
            // stages of the ring: keys of tile j in number `k0 + 2 j` of the item, values behind them
            int at = 0;                                            // tiles used before this item
            uint32_t phase_own = 0, phase_gs = 0, phase_read = 0;
            bool ok = true, began = false;
            auto wait = [&](uint64_t& bar, uint32_t parity) {
                ok = ok && mbar_wait(smem_u32(&bar), parity, abort_flag, p.status);
                tc_fence_after();
            };
            // (nothing after a wait given up: the producer would announce a copy to a barrier whose last one has not landed)
            auto commit = [&](uint64_t& bar) { if (ok) mma_commit(smem_u32(&bar)); };
            auto arrived = [&](int i) { wait(sh.full[i % C::kRing], uint32_t(i / C::kRing) & 1u); return base + (i % C::kRing) * C::kTile; };
            auto release = [&](int i) { commit(sh.empty[i % C::kRing]); };
            const uint32_t q_tile = base + C::kOwn, go_tile = q_tile + C::kTile;
            for (int item = 0; ok; ++item) {
                wait(sh.item_full[item & 1], uint32_t(item >> 1) & 1u);
                if (!ok) break;
                const Item it = sh.item[item & 1];
                mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
                if (it.head < 0) break;
                const int n = it.first / kRows + 1;
                wait(sh.own_full, phase_own);
                phase_own ^= 1u;
                auto scores = [&](int j) {
                    const uint32_t k_tile = arrived(at + 2 * j);
                    if (ok) product<D>(tmem + 128u * (j & 1), q_tile, k_tile);
                    commit(sh.s[j & 1]);
                };
                auto gps = [&](int j) {
                    const uint32_t v_tile = arrived(at + 2 * j + 1);
                    if (ok) product<D>(t_gp, go_tile, v_tile);
                    commit(sh.gp);
                    release(at + 2 * j + 1);
                };
                if (ok) scores(0);
                if (ok) gps(0);
                if (ok && n > 1) scores(1);
                if (n == 1) commit(sh.own_empty);
#pragma unroll 1
                for (int j = 0; j < n && ok; ++j) {
                    const uint32_t k_tile = base + ((at + 2 * j) % C::kRing) * C::kTile;
                    if (j == 0) {
                        if (began) {
                            wait(sh.read, phase_read);             // the last item's result has been read
                            phase_read ^= 1u;
                        }
                        began = true;
                    }
                    wait(sh.gs[0], phase_gs);
                    wait(sh.gs[1], phase_gs);
                    phase_gs ^= 1u;
                    if (ok && j + 1 < n) gps(j + 1);               // (GP(j) has been read)
                    if (j + 2 == n) commit(sh.own_empty);      // the last product with the item's own tiles
                    if (ok) {
                        accumulate<D>(t_gq, tmem + 128u * (j & 1), k_tile, 0, j == 0);
                        accumulate<D>(t_gq, tmem + 128u * (j & 1) + 64u, k_tile, 1, false);
                    }
                    release(at + 2 * j);
                    if (j + 1 == n) commit(sh.done);
                    if (ok && j + 2 < n) scores(j + 2);
                }
                at += 2 * n;
            }
        }
    } else if (warp == 2) {
        // ---------------- keys behind a sequence's end ----------------
        Mender<D, C::kRing> mender{smem, sh.full, sh.tail, abort_flag, p.status, 0};
        for (int item = 0; mender.ok; ++item) {
            if (!__all_sync(0xFFFFFFFFu, mbar_wait_suspended(smem_u32(&sh.item_full[item & 1]), uint32_t(item >> 1) & 1u, abort_flag, p.status))) break;
            const Item it = sh.item[item & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
            if (it.head < 0) break;
            for (int j = 0; j <= it.first / kRows; ++j) {
                mender.next(it.end - it.begin - j * kRows);
                mender.next(kRows);
            }
        }
    } else if (warp >= 4) {
        // ---------------- results: thread = row ----------------
        const int quad = warp & 3;
        bool failed = false;
        auto wait = [&](uint64_t& bar, uint32_t parity) {
            failed = __any_sync(0xFFFFFFFFu, !mbar_wait_suspended(smem_u32(&bar), parity, abort_flag, p.status)) || failed;
            tc_fence_after();
        };
        for (int item = 0;; ++item) {
            wait(sh.item_full[item & 1], uint32_t(item >> 1) & 1u);
            if (failed) break;
            const Item it = sh.item[item & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
            if (it.head < 0) break;
            wait(sh.done, uint32_t(item) & 1u);
            if (failed) break;
            store_rows<D>(t_gq + (uint32_t(quad * 32) << 16), gq + int64_t(it.head) * D, ldgq, it.begin + it.first + quad * 32, it.end, p.scale);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.read));
        }
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

// ---------------------------------------------------------------------------------------------
// gk, gv
template <int D>
__global__ void __launch_bounds__(bwd::kThreads, 1)
sequence_key_grad_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_go, const __grid_constant__ CUtensorMap map_k,
                         const __grid_constant__ CUtensorMap map_v, const Problem p, const float2* const stats, float* const parts, const int splits,
                         const int group, __nv_bfloat16* const gk, const int64_t ldgk, __nv_bfloat16* const gv, const int64_t ldgv) {
    using namespace bwd;
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    Misc& sh = *reinterpret_cast<Misc*>(smem + C::kMisc);
    float* const stats_sh = reinterpret_cast<float*>(smem + C::kStats);
    volatile int* abort_flag = &sh.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 32) {
        init(sh, C::kKeyRing, 15);                                 // an item's readers: the MMA thread, two menders, twelve warps
        tma_prefetch_map(&map_q);
        tma_prefetch_map(&map_go);
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
    }
    if (warp == 2) tmem_alloc(smem_u32(&sh.tmem), kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem, t_gp = tmem + 128, t_gv = tmem + 256, t_gk = tmem + 384;
    // an item's head is split * Hkv + key head; its query heads are those of the split
    const int heads = p.G / splits;
    // tiles of queries that see the item's keys, of one head; tile i of the item is tile first / kRows + i % tiles of head i / tiles
    auto tiles_of_item = [](const Item& it) { return (it.end - it.begin + kRows - 1) / kRows - it.first / kRows; };

    if (warp >= 4 && warp < 12) {
        take_registers();
        // ---------------- elementwise: thread = key, half of the queries ----------------
        const int half = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lanes = uint32_t(quad * 32) << 16, t_s = tmem + lanes + 64u * half, t_g = t_gp + lanes + 64u * half;
        uint32_t phase = 0;
        int k = 0;
        bool failed = false;
        auto wait = [&](uint64_t& bar, uint32_t parity) {
            failed = __any_sync(0xFFFFFFFFu, !mbar_wait(smem_u32(&bar), parity, abort_flag, p.status)) || failed;
            tc_fence_after();
        };
        const f2 scale2 = mk2(p.scale_log2, p.scale_log2);
        for (int item = 0;; ++item) {
            wait(sh.item_full[item & 1], uint32_t(item >> 1) & 1u);
            if (failed) break;
            const Item it = sh.item[item & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
            if (it.head < 0) break;
            const int tiles = tiles_of_item(it), n = tiles * heads;
            int of_head = 0;
            for (int t = 0; t < n; ++t, ++k) {
                const bool partly = of_head == 0;                  // the tile on the diagonal
                if (++of_head == tiles) of_head = 0;
                wait(sh.stats_full[k & 1], uint32_t(k >> 1) & 1u);
                const float4* lse4 = reinterpret_cast<const float4*>(stats_sh + 256 * (k & 1) + 64 * half);
                const float4* delta4 = lse4 + 32;
                float4 l4[16];                                     // before the scores: the products leave little of shared memory's time
#pragma unroll
                for (int i = 0; i < 16; ++i) l4[i] = lse4[i];
                if (!failed) wait(sh.s[0], phase);
                if (failed) break;
                uint32_t e[2][32];
                tmem_ld32(t_s, e[0]);
                tmem_ld32(t_s + 32u, e[1]);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.s_read));
                if (k >= 1) wait(sh.p_read, uint32_t(k - 1) & 1u); // the last tile's product with P^T is done
                if (failed) break;
                uint8_t* const p_row = smem + C::kP + half * C::kAtom;
#pragma unroll
                for (int c = 0; c < 64; c += 8) {
                    uint32_t out[4];
#pragma unroll
                    for (int i = 0; i < 8; i += 4) {
                        const float4 l = l4[(c + i) >> 2];
                        uint32_t* const x = &e[c >> 5][(c & 31) + i];
                        float a[4];
                        un2(powers(fma2(mk2(__uint_as_float(x[0]), __uint_as_float(x[1])), scale2, mk2(l.x, l.y))), a[0], a[1]);
                        un2(powers(fma2(mk2(__uint_as_float(x[2]), __uint_as_float(x[3])), scale2, mk2(l.z, l.w))), a[2], a[3]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[j] = __float_as_uint(a[j]);
                        out[i >> 1] = pack2(a[0], a[1]);
                        out[(i >> 1) + 1] = pack2(a[2], a[3]);
                    }
                    *reinterpret_cast<uint4*>(p_row + atom_chunk_offset(row, c >> 3)) = make_uint4(out[0], out[1], out[2], out[3]);
                }
                if (partly) {                                      // queries before the key: zeros, a second time over the row
#pragma unroll
                    for (int c = 0; c < 64; c += 8) {
                        uint32_t out[4];
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            uint32_t* const x = &e[c >> 5][(c & 31) + i];
                            if (64 * half + c + i < row) x[0] = 0u;
                            if (64 * half + c + i + 1 < row) x[1] = 0u;
                            out[i >> 1] = pack2(__uint_as_float(x[0]), __uint_as_float(x[1]));
                        }
                        *reinterpret_cast<uint4*>(p_row + atom_chunk_offset(row, c >> 3)) = make_uint4(out[0], out[1], out[2], out[3]);
                    }
                }
                fence_async_shared();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.p[half]));
                wait(sh.gp, phase);
                if (failed) break;
                uint32_t out[32];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t v[32];
                    tmem_ld32(t_g + 32u * i, v);
                    float4 d4[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) d4[j] = delta4[8 * i + j];
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        const float4 d = d4[c >> 2];
                        float a, b;
                        un2(mul2(mk2(__uint_as_float(e[i][c]), __uint_as_float(e[i][c + 1])), add2(mk2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), mk2(d.x, d.y))), a, b);
                        out[16 * i + (c >> 1)] = pack2(a, b);
                        un2(mul2(mk2(__uint_as_float(e[i][c + 2]), __uint_as_float(e[i][c + 3])),
                                 add2(mk2(__uint_as_float(v[c + 2]), __uint_as_float(v[c + 3])), mk2(d.z, d.w))), a, b);
                        out[16 * i + (c >> 1) + 1] = pack2(a, b);
                    }
                }
                tmem_st32(t_g, out);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&sh.gs[half]));
                    mbar_arrive(smem_u32(&sh.stats_empty[k & 1]));
                }
                phase ^= 1u;
            }
            if (failed) break;
        }
    } else {
    give_registers();
    if (warp == 0) {
        // ---------------- producer ----------------
        const uint64_t keep = l2_policy_evict_last(), once = l2_policy_evict_first();
        Loader<D, C::kKeyRing> ring(smem, sh.full, sh.empty, sh.tail, abort_flag, p.status);
        ring.heed(1);
        const Order<kRows, true> order(p, p.Hkv * splits, group);
        int items = 0, k = 0;                                      // k: tiles of queries so far
        uint32_t phase_own = 0, phase_taken = 0;
        unsigned at = blockIdx.x;
        // (The first question waits for the kernel before: a CTA that started beside it would take work from SMs that are about to be free.)
        auto ask = [&] {
            if (lane == 0) ask_for_next(&sh.answer, &sh.taken);
            __syncwarp();
        };
        for (bool first = true;; first = false) {
            if (!first) ask();
            int part;                                  // parts of a key head side by side
            const Tile t = order.take(at, part);
            const int kvh = part / splits, split = part - kvh * splits, which = split * p.Hkv + kvh;
            if (t.first >= 0) {
                const Item it = {which, t.begin, t.end, t.first};
                if (items >= 2) ring.wait(sh.item_empty[items & 1], uint32_t((items >> 1) - 1) & 1u);
                if (ring.ok && lane == 0) {
                    sh.item[items & 1] = it;
                    mbar_arrive(smem_u32(&sh.item_full[items & 1]));
                }
                if (ring.ok && items >= 1) {
                    ring.wait(sh.own_empty, phase_own);
                    phase_own ^= 1u;
                }
                ++items;
                if (ring.ok && lane == 0) {
                    const uint32_t bar = smem_u32(&sh.own_full);
                    mbar_expect_tx(bar, 2 * C::kTile);
                    tma_tile_load_3d(base + C::kOwn, &map_k, 0, it.begin + it.first, kvh * (D / 64), bar, once);
                    tma_tile_load_3d(base + C::kOwn + C::kTile, &map_v, 0, it.begin + it.first, kvh * (D / 64), bar, once);
                }
                __syncwarp();
                for (int h = kvh * p.G + split * heads, h1 = h + heads; h < h1 && ring.ok; ++h)
                    for (int row = it.begin + it.first; row < it.end && ring.ok; row += kRows, ++k) {
                        float2 v[4];                               // statistics of the tile's queries; behind the end: probability 0
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[i] = row + lane + 32 * i < it.end ? stats[int64_t(h) * p.M + row + lane + 32 * i] : make_float2(INFINITY, 0.0f);
                        ring.load(&map_q, row, h * (D / 64), it.end - row, keep);
                        if (ring.ok) ring.load(&map_go, row, h * (D / 64), it.end - row, keep);
                        if (k >= 2 && ring.ok) ring.wait(sh.stats_empty[k & 1], uint32_t((k >> 1) - 1) & 1u);
                        if (!ring.ok) break;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            stats_sh[256 * (k & 1) + lane + 32 * i] = -v[i].x;
                            stats_sh[256 * (k & 1) + 128 + lane + 32 * i] = -v[i].y;
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&sh.stats_full[k & 1]));
                    }
            }
            if (first) {
                grid_dependency_wait();
                ask();
            }
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
        if (elect_one()) {
            int at = 0;                                            // tiles used before this item; queries of its tile t in number at + 2 t, gradients behind them
            uint32_t phase_own = 0, phase_p = 0, phase_read = 0;
            bool ok = true, began = false;
            auto wait = [&](uint64_t& bar, uint32_t parity) {
                ok = ok && mbar_wait(smem_u32(&bar), parity, abort_flag, p.status);
                tc_fence_after();
            };
            // (nothing after a wait given up: the producer would announce a copy to a barrier whose last one has not landed)
            auto commit = [&](uint64_t& bar) { if (ok) mma_commit(smem_u32(&bar)); };
            auto place = [&](int i) { return base + (i % C::kKeyRing) * C::kTile; };
            auto arrived = [&](int i) { wait(sh.full[i % C::kKeyRing], uint32_t(i / C::kKeyRing) & 1u); return place(i); };
            auto release = [&](int i) { commit(sh.empty[i % C::kKeyRing]); };
            const uint32_t k_tile = base + C::kOwn, v_tile = k_tile + C::kTile;
            for (int item = 0; ok; ++item) {
                wait(sh.item_full[item & 1], uint32_t(item >> 1) & 1u);
                if (!ok) break;
                const Item it = sh.item[item & 1];
                mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
                if (it.head < 0) break;
                const int n = tiles_of_item(it) * heads;
                wait(sh.own_full, phase_own);
                phase_own ^= 1u;
                auto scores = [&](int t) {
                    const uint32_t q_tile = arrived(at + 2 * t);
                    if (ok) product<D>(tmem, k_tile, q_tile);
                    commit(sh.s[0]);
                };
                auto gps = [&](int t) {
                    const uint32_t go_tile = arrived(at + 2 * t + 1);
                    if (ok) product<D>(t_gp, v_tile, go_tile);
                    commit(sh.gp);
                };
                if (ok) scores(0);
                if (ok) gps(0);
#pragma unroll 1
                for (int t = 0; t < n && ok; ++t) {
                    if (t == 0) {
                        if (began) {
                            wait(sh.read, phase_read);             // the last item's results have been read
                            phase_read ^= 1u;
                        }
                        began = true;
                    }
                    if (t + 1 < n) {
                        wait(sh.s_read, phase_p);                  // the scores are in registers
                        if (ok) scores(t + 1);
                    }
#pragma unroll 1
                    for (int half = 0; half < 2 && ok; ++half) {
                        wait(sh.p[half], phase_p);
                        if (ok) accumulate_from_shared<D>(t_gv, base + C::kP + half * C::kAtom, place(at + 2 * t + 1), half, t == 0 && half == 0);
                    }
                    commit(sh.p_read);
                    release(at + 2 * t + 1);
#pragma unroll 1
                    for (int half = 0; half < 2 && ok; ++half) {
                        wait(sh.gs[half], phase_p);
                        if (ok) accumulate<D>(t_gk, t_gp + 64u * half, place(at + 2 * t), half, t == 0 && half == 0);
                    }
                    if (t + 1 == n) wait(sh.s_read, phase_p);      // (every tile's)
                    phase_p ^= 1u;
                    release(at + 2 * t);
                    if (ok && t + 1 < n) gps(t + 1);
                }
                commit(sh.own_empty);
                commit(sh.done);
                at += 2 * n;
            }
        }
        __syncwarp();                                              // the other lanes, in the wait for gq's kernel below, would hold this one up: one token 20 -> 16 us
    } else if (warp < 4) {
        // ---------------- queries and gradients behind a sequence's end ----------------
        Mender<D, C::kKeyRing> mender{smem, sh.full, sh.tail, abort_flag, p.status, warp - 2};
        for (int item = 0; mender.ok; ++item) {
            if (!__all_sync(0xFFFFFFFFu, mbar_wait_suspended(smem_u32(&sh.item_full[item & 1]), uint32_t(item >> 1) & 1u, abort_flag, p.status))) break;
            const Item it = sh.item[item & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
            if (it.head < 0) break;
            for (int h = 0; h < heads; ++h)
                for (int row = it.begin + it.first; row < it.end; row += kRows) {
                    mender.next(it.end - row);
                    mender.next(it.end - row);
                }
        }
    } else {
        // ---------------- results: thread = key ----------------
        const int quad = warp & 3;
        const uint32_t lanes = uint32_t(quad * 32) << 16;
        bool failed = false;
        auto wait = [&](uint64_t& bar, uint32_t parity) {
            failed = __any_sync(0xFFFFFFFFu, !mbar_wait_suspended(smem_u32(&bar), parity, abort_flag, p.status)) || failed;
            tc_fence_after();
        };
        for (int item = 0;; ++item) {
            wait(sh.item_full[item & 1], uint32_t(item >> 1) & 1u);
            if (failed) break;
            const Item it = sh.item[item & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.item_empty[item & 1]));
            if (it.head < 0) break;
            wait(sh.done, uint32_t(item) & 1u);
            if (failed) break;
            const int row0 = it.begin + it.first + quad * 32;
            if (splits == 1) {
                store_rows<D>(t_gv + lanes, gv + int64_t(it.head) * D, ldgv, row0, it.end, 1.0f);
                store_rows<D>(t_gk + lanes, gk + int64_t(it.head) * D, ldgk, row0, it.end, p.scale);
            } else {
                const int split = it.head / p.Hkv, ld = p.Hkv * D;
                float* const to = parts + int64_t(2 * split) * p.M * ld + (it.head - split * p.Hkv) * D;
                store_rows<D, true>(t_gk + lanes, to, ld, row0, it.end, p.scale);
                store_rows<D, true>(t_gv + lanes, to + int64_t(p.M) * ld, ld, row0, it.end, 1.0f);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.read));
        }
    }
    }
    grid_dependency_wait();                  // not done before gq is
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 2) {
        let_land(abort_flag);
        tmem_dealloc(tmem, kTmemCols);
    }
}

// gk and gv from the splits' sums, in their order: eight columns of a row and result per thread
template <int D>
__global__ void __launch_bounds__(256) join_kernel(const Problem p, const float* const parts, const int splits, __nv_bfloat16* gk, int64_t ldgk, __nv_bfloat16* gv, int64_t ldgv) {
    grid_dependency_wait();
    const int width = p.Hkv * D, chunks = width / 8;
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x, row = i / (2 * chunks);
    const int rest = int(i - row * 2 * chunks), what = rest / chunks, c = rest - what * chunks;
    if (row < clamped(p, 0) || row >= clamped(p, p.B)) return;     // sequences lie one behind the other
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f), b = a;
    for (int s = 0; s < splits; ++s) {
        const float4* from = reinterpret_cast<const float4*>(parts + (int64_t(2 * s + what) * p.M + row) * width + 8 * c);
        const float4 x = from[0], y = from[1];
        a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w;
        b.x += y.x; b.y += y.y; b.z += y.z; b.w += y.w;
    }
    *reinterpret_cast<uint4*>((what ? gv + row * ldgv : gk + row * ldgk) + 8 * c) = make_uint4(pack2(a.x, a.y), pack2(a.z, a.w), pack2(b.x, b.y), pack2(b.z, b.w));
}

// Where both kernels find SMs at once, as many parts as leave it so (300 tokens of three sequences, 32/8 heads: two parts 20 us, four 23).  Otherwise enough items for
// every SM (up to half as many again), and enough that the largest, which stand for a whole sequence's queries, are no longer than an SM's share of the
// whole: with sequences of one length that is about two items an SM; items of 8 tiles need no cutting for that.  (One sequence of 8192, 40/4 heads: 2.70 -> 2.28
// ms; four of 16/2 heads, 8000 tokens, D = 64: 393 -> 234 us; 4001 tokens of nine with 32/8 heads, which have two, would lose 2 us to
// their sums' way through memory.)
int key_splits(int64_t M, int64_t B, int Hkv, int G) {
    if (M == 0 || B == 0) return 1;
    const int64_t seqs = B < M ? B : M, tiles = (M / seqs + 127) / 128, items = seqs * tiles * Hkv;
    int n = 1;
    for (int d = 1; d <= G; ++d) {
        if (G % d) continue;
        if (items * (G + 1) <= kSms ? items * (G + d) <= kSms : 2 * items * d <= 3 * kSms || (items * n < 2 * kSms - 16 && tiles * G > 8 * n)) n = d;
    }
    return n;
}

template <int D>
static int launch(const Problem& p, const float* lse, float2* stats, float* parts, int splits, __nv_bfloat16* gq, int64_t ldgq, __nv_bfloat16* gk, int64_t ldgk, __nv_bfloat16* gv,
                  int64_t ldgv, cudaStream_t s) {
    using C = bwd::Cfg<D>;
    CUtensorMap mq, mgo, mk, mv;
    int rc = make_x_chunk_tensor_map(&mq, p.q, p.ldq, p.M, int64_t(p.Hq) * D, 128, D / 64);
    if (!rc) rc = make_x_chunk_tensor_map(&mgo, p.go, p.ldgo, p.M, int64_t(p.Hq) * D, 128, D / 64);
    if (!rc) rc = make_x_chunk_tensor_map(&mk, p.k, p.ldk, p.M, int64_t(p.Hkv) * D, 128, D / 64);
    if (!rc) rc = make_x_chunk_tensor_map(&mv, p.v, p.ldv, p.M, int64_t(p.Hkv) * D, 128, D / 64);
    static std::atomic<uint64_t> configured_q{0}, configured_k{0};
    if (!rc) rc = allow_dynamic_smem(sequence_query_grad_kernel<D>, C::kBytes, configured_q);
    if (!rc) rc = allow_dynamic_smem(sequence_key_grad_kernel<D>, C::kBytes, configured_k);
    if (rc) return rc;
    const int64_t groups = (int64_t(p.M) + 3) / 4 * p.Hq, tiles = most_tiles(p.M, p.B, bwd::kRows);
    const int64_t per_block = 256 / (D / 8);
    delta_kernel<D><<<unsigned((groups + per_block - 1) / per_block), 256, 0, s>>>(p, lse, stats);
    if (cudaGetLastError() != cudaSuccess) return PATCH_ERR_CUDA;
    // The two kernels are launched dependently: the first sets up beside the statistics, the second takes SMs as the first leaves them (a small problem
    // has both at once).  Its CTAs start when all of the first one's have found the statistics, and leave when that one is done.
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.blockDim = dim3(bwd::kThreads, 1, 1);
    cfg.dynamicSmemBytes = C::kBytes;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const float2* const found = stats;
    int at_once = heads_at_once(p.Hkv, int64_t(p.M) * D * 4, tiles * p.G);      // keys and values
    cfg.gridDim = dim3(unsigned(tiles * p.Hq), 1, 1);
    bool ok = cudaLaunchKernelEx(&cfg, sequence_query_grad_kernel<D>, mq, mgo, mk, mv, p, found, at_once * p.G, gq, ldgq) == cudaSuccess;
    at_once = heads_at_once(p.Hkv, int64_t(p.M) * D * 4 * p.G, tiles * splits);    // queries and their gradients
    cfg.gridDim = dim3(unsigned(tiles * p.Hkv * splits), 1, 1);
    ok = ok && cudaLaunchKernelEx(&cfg, sequence_key_grad_kernel<D>, mq, mgo, mk, mv, p, found, parts, splits, at_once * splits, gk, ldgk, gv, ldgv) == cudaSuccess;
    if (splits > 1) {
        cfg.blockDim = dim3(256, 1, 1);
        cfg.dynamicSmemBytes = 0;
        cfg.gridDim = dim3(unsigned((int64_t(p.M) * p.Hkv * (D / 8) * 2 + 255) / 256), 1, 1);
        ok = ok && cudaLaunchKernelEx(&cfg, join_kernel<D>, p, static_cast<const float*>(parts), splits, gk, ldgk, gv, ldgv) == cudaSuccess;
    }
    if (ok) return PATCH_OK;
    cudaGetLastError();                      // reported here, not by the next call
    return PATCH_ERR_CUDA;
}
int launch_backward(const Problem& p, int D, const float* lse, float2* stats, float* parts, int splits, __nv_bfloat16* gq, int64_t ldgq, __nv_bfloat16* gk, int64_t ldgk, __nv_bfloat16* gv,
                    int64_t ldgv, cudaStream_t s) {
    return D == 128 ? launch<128>(p, lse, stats, parts, splits, gq, ldgq, gk, ldgk, gv, ldgv, s) : launch<64>(p, lse, stats, parts, splits, gq, ldgq, gk, ldgk, gv, ldgv, s);
}

}  // namespace seq
}  // namespace patch
