// Dense feed-forward block: what its two paths share (ffn_sm100.cu: tensor cores, ffn_few.cu: few tokens).
#pragma once

#include "operators.h"

namespace moe {

constexpr int kFfnFewTokens = 32;  // most tokens of the second

// Whether a forward call that saves nothing runs the kernels for few tokens: their rows have to fit shared memory.
bool ffn_few_fits(int tokens, int h, int f);
// act [tokens][f] is scratch of the tensors' type
cudaError_t launch_ffn_few(const void* x, const void* W1, const void* W3, const void* W2, const void* residual, int tokens,
                            int h, int f, int dtype, void* act, void* y, cudaStream_t st);

#ifdef __CUDACC__
// 1 / (1 + exp(-g)) by the fast exponential and quotient.  By their documented bounds the error is 2 + 1.16 |g| and 2 units of
// the last place, where exp(-g) counts: a few about 0, 2^-18 of the value at g = -50, 2^-17 at -87; 0 below that.
__device__ __forceinline__ float ffn_sigmoid(float g) { return __fdividef(1.0f, 1.0f + __expf(-g)); }
#endif

}  // namespace moe
