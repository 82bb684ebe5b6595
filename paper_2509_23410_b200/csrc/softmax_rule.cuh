// The arithmetic of a running softmax as all attention kernels do it, without a CUDA type, so that it also compiles for the CPU
// (tests/test_softmax_rule.py runs it there).
//
// Maxima are maxima of the fp32 sums q.k themselves, and a probability is 2^((s - m) scale): the difference first, then the scale in powers
// of two.  The largest score's exponent is then exactly 0, whatever its size, all others are below, and parts are joined with weights
// 2^((m_i - m) scale) by the same rule.  (2^(s scale - m) with a scaled, hence rounded, maximum saves an instruction of two where the product is
// left unrounded, but then the exponent of the largest score is the rounding error of m: nothing for scores below 2^22 or so, more than 8 from 2^28
// on, more than 128 from 2^31 on: probabilities that overflow or all vanish.  Rounding the product as well does not help: the
// compiler joins it with the subtraction.)
#pragma once
#include <math.h>
#ifdef __CUDACC__
#define PATCH_HD __host__ __device__ __forceinline__
#else
#define PATCH_HD inline
#endif

namespace patch {
namespace attn {

// what is subtracted from the scores of a row whose maximum is m: nothing where nothing has been seen yet
PATCH_HD float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
PATCH_HD float exponent(float s, float base, float scale) { return (s - base) * scale; }

// The block kernel's rule (attention_block_sm100.cu): a row's maximum stays what it is until a part of a tile sums to more than this ...
constexpr float kMostSum = 256.0f;
// ... and is raised at most once for the part: afterwards no exponent of it is above 0.  The count ends the loop whatever the numbers are.
PATCH_HD bool raise_maximum(float sum, float m, bool raised) { return !raised && sum > kMostSum && m != INFINITY; }

}  // namespace attn
}  // namespace patch
