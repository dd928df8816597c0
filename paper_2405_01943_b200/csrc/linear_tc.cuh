// What the tensor-core kernels of dass_linear share.  Internal header.
#pragma once

#include "linear_common.cuh"
#include "tc_common.cuh"

namespace dass {

// The activation before a rounding to bf16 (8 bits): __expf and an approximate quotient are exact enough by 2^10.
template <int ACT>
__device__ __forceinline__ float lt_act(float x)
{
    if constexpr (ACT == DASS_ACT_SILU) return __fdividef(x, 1.0f + __expf(-x));
    else if constexpr (ACT == DASS_ACT_GELU_TANH)           // 0.5 (1 + tanh z) = sigmoid(2 z)
        return __fdividef(x, 1.0f + __expf(-1.5957691216057308f * x * fmaf(0.044715f * x, x, 1.0f)));
    else if constexpr (ACT == DASS_ACT_RELU) return fmaxf(x, 0.0f);
    else return x;
}

}  // namespace dass
