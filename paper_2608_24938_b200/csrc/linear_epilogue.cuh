// What the dense-product kernels do to a sum: activation, rounding to the output type.
#pragma once
#include "common.cuh"

namespace exfold {

__device__ __forceinline__ float linear_act(float v, int act) {
    switch (act) {  // uniform over the launch
        case EXFOLD_ACT_RELU: return v < 0.f ? 0.f : v;  // NaN stays
        case EXFOLD_ACT_GELU: return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
        case EXFOLD_ACT_GELU_TANH: return 0.5f * v * (1.0f + tanhf(0.79788456080286536f * (v + 0.044715f * v * v * v)));
        case EXFOLD_ACT_SILU: return v / (1.0f + expf(-v));
        default: return v;
    }
}

__device__ __forceinline__ void linear_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void linear_store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

}  // namespace exfold
