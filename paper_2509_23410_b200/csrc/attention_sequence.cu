// Causal attention within packed sequences and its gradient (public header: patch_sequence_attention, ..._backward).
//
// Mathematics.  For sequence rows i >= j of one head: s_ij = q_i . k_j, p_ij = 2^((s_ij - m_i) scale log2 e) / l_i with a running maximum
// m and sum l.  The gradient recomputes p_ij = 2^(s_ij scale log2 e - lse_i log2 e) and, with delta_i = go_i . o_i,
//     gs_ij = p_ij (go_i . v_j - delta_i) scale,  gq_i = sum_j gs_ij k_j,  gk_j = sum_i gs_ij q_i,  gv_j = sum_i p_ij go_i,
// the sums of gk and gv also over the query heads that share the key head.  Products take bf16 operands and fp32 accumulators; p and gs are
// rounded to bf16 for theirs (the sum l takes p unrounded).
//
// The kernels are in attention_sequence_sm100.cu and attention_sequence_grad_sm100.cu; here are the checks of arguments.
#include <math.h>
#include "attention_sequence.cuh"

namespace patch {
namespace seq {

// ---- checks of arguments ----
static int check_shape(int64_t M, int Hq, int Hkv, int D, int64_t B) {
    if (M < 0 || M > 0x7FFFFFFF - 256 || B < 0 || B > (1 << 20) || (D != 64 && D != 128) || Hkv < 1 || Hq < Hkv || Hq % Hkv || Hq > 4096) return PATCH_ERR_SHAPE;
    // CTAs of a launch are counted in 31 bits
    return M * Hq * (D / 8) > (int64_t(1) << 38) || most_tiles(M, B, kTileRows) * Hq > 0x7FFFFFFF ? PATCH_ERR_SHAPE : PATCH_OK;
}
static int check_rows(const void* x, int64_t ld, int64_t H, int64_t D) {
    if (!x) return PATCH_ERR_NULL;
    if (ld < H * D || ld % 8 || ld > (int64_t(1) << 28)) return PATCH_ERR_SHAPE;
    return aligned16(x) ? PATCH_OK : PATCH_ERR_ALIGN;
}
static size_t stats_bytes(int64_t M, int Hq) { return (size_t(M) * Hq * sizeof(float2) + 255) / 256 * 256; }
static int check_scale(float scale) { return scale > 0.0f && scale <= 2e38f ? PATCH_OK : PATCH_ERR_SHAPE; }

}  // namespace seq
}  // namespace patch

using namespace patch;
using B16 = __nv_bfloat16;

extern "C" int patch_sequence_attention(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t M, int Hq, int Hkv, int D,
                                        const int32_t* starts, int64_t B, float scale, void* O, int64_t ldo, float* lse, int* status_dev, void* stream) {
    int rc = seq::check_shape(M, Hq, Hkv, D, B);
    if (rc || (rc = seq::check_scale(scale))) return rc;
    if (M == 0 || B == 0) return PATCH_OK;
    if ((rc = seq::check_rows(Q, ldq, Hq, D)) || (rc = seq::check_rows(K, ldk, Hkv, D)) || (rc = seq::check_rows(V, ldv, Hkv, D)) ||
        (rc = seq::check_rows(O, ldo, Hq, D)))
        return rc;
    if (!starts) return PATCH_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(starts) & 3u) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return PATCH_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    const seq::Problem p = {static_cast<const B16*>(Q), static_cast<const B16*>(K), static_cast<const B16*>(V), nullptr, nullptr, ldq, ldk, ldv, 0, 0, starts,
                            int(B), int(M), Hq, Hkv, Hq / Hkv, scale, scale * 1.44269504f, status_dev};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return seq::launch_forward(p, D, static_cast<B16*>(O), ldo, lse, s);
}

extern "C" int patch_sequence_attention_backward_workspace_size(int64_t M, int64_t B, int Hq, int Hkv, int D, size_t* bytes_out) {
    if (!bytes_out) return PATCH_ERR_NULL;
    const int rc = seq::check_shape(M, Hq, Hkv, D, B);
    if (rc) return rc;
    const int splits = seq::key_splits(M, B, Hkv, Hq / Hkv);
    *bytes_out = seq::stats_bytes(M, Hq) + (splits > 1 ? size_t(splits) * 2 * M * Hkv * D * sizeof(float) : 0);
    return PATCH_OK;
}

extern "C" int patch_sequence_attention_backward(const void* gO, int64_t ldgo, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                                 const void* O, int64_t ldo, const float* lse, int64_t M, int Hq, int Hkv, int D, const int32_t* starts, int64_t B,
                                                 float scale, void* gQ, int64_t ldgq, void* gK, int64_t ldgk, void* gV, int64_t ldgv, void* workspace,
                                                 size_t workspace_bytes, int* status_dev, void* stream) {
    size_t need = 0;
    int rc = patch_sequence_attention_backward_workspace_size(M, B, Hq, Hkv, D, &need);
    if (rc || (rc = seq::check_scale(scale))) return rc;
    if (M == 0 || B == 0) return PATCH_OK;
    if ((rc = seq::check_rows(gO, ldgo, Hq, D)) || (rc = seq::check_rows(Q, ldq, Hq, D)) || (rc = seq::check_rows(K, ldk, Hkv, D)) ||
        (rc = seq::check_rows(V, ldv, Hkv, D)) || (rc = seq::check_rows(O, ldo, Hq, D)) || (rc = seq::check_rows(gQ, ldgq, Hq, D)) ||
        (rc = seq::check_rows(gK, ldgk, Hkv, D)) || (rc = seq::check_rows(gV, ldgv, Hkv, D)))
        return rc;
    if (!lse || !starts || !workspace) return PATCH_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(starts) & 3u) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PATCH_ERR_ALIGN;
    if (workspace_bytes < need) return PATCH_ERR_SIZE;
    if ((rc = check_device())) return rc;
    const seq::Problem p = {static_cast<const B16*>(Q), static_cast<const B16*>(K), static_cast<const B16*>(V), static_cast<const B16*>(O), static_cast<const B16*>(gO),
                            ldq, ldk, ldv, ldo, ldgo, starts, int(B), int(M), Hq, Hkv, Hq / Hkv, scale, scale * 1.44269504f, status_dev};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    B16 *gq = static_cast<B16*>(gQ), *gk = static_cast<B16*>(gK), *gv = static_cast<B16*>(gV);
    float2* stats = static_cast<float2*>(workspace);
    float* parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + seq::stats_bytes(M, Hq));
    return seq::launch_backward(p, D, lse, stats, parts, seq::key_splits(M, B, Hkv, Hq / Hkv), gq, ldgq, gk, ldgk, gv, ldgv, s);
}
