// What the dense-product kernels do to their sums: bias, activation, residual, one rounding to the output type.
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
__device__ __forceinline__ float linear_f32(float v) { return v; }
__device__ __forceinline__ float linear_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
// Four neighbours at once (aligned to their size)
__device__ __forceinline__ float4 linear_load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 linear_load4(const __nv_bfloat16* p) {
    const uint2 t = *reinterpret_cast<const uint2*>(p);
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&t.x));
    const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&t.y));
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void linear_store4(float* p, const float4& v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void linear_store4(__nv_bfloat16* p, const float4& v) {
    __nv_bfloat162 h[2] = {__floats2bfloat162_rn(v.x, v.y), __floats2bfloat162_rn(v.z, v.w)};
    *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(h);
}

// Four neighbouring outputs (n a multiple of 4) of a row, bf16 operands; O is y's and the residual's type. Rows that are not
// aligned to four elements, and the last N % 4 columns, go element by element.
template <typename O>
struct LinearEpilogue {
    const LinearParams& p;
    const bool vec;       // y and residual
    const bool vec_bias;
    __device__ __forceinline__ explicit LinearEpilogue(const LinearParams& q)
        : p(q),
          vec(((reinterpret_cast<uintptr_t>(q.y) | reinterpret_cast<uintptr_t>(q.residual)) & (4 * sizeof(O) - 1)) == 0 &&
              (q.ldy & 3) == 0 && (q.residual == nullptr || (q.ldr & 3) == 0)),
          vec_bias((reinterpret_cast<uintptr_t>(q.bias) & 7) == 0) {}
    struct Extra {
        float4 bias, residual;
    };
    // What comes from memory, asked for before the sum is there
    __device__ __forceinline__ Extra fetch(int64_t m, int n) const {
        Extra e;
        e.bias = e.residual = make_float4(0.f, 0.f, 0.f, 0.f);
        const bool four = n + 4 <= p.N;
        if (p.bias != nullptr) {
            const __nv_bfloat16* b = reinterpret_cast<const __nv_bfloat16*>(p.bias) + n;
            if (vec_bias && four) e.bias = linear_load4(b);
            else each(n, [&](int j) { at(e.bias, j) = linear_f32(b[j]); });
        }
        if (p.residual != nullptr) {
            const O* r = reinterpret_cast<const O*>(p.residual) + m * p.ldr + n;
            if (vec && four) e.residual = linear_load4(r);
            else each(n, [&](int j) { at(e.residual, j) = linear_f32(r[j]); });
        }
        return e;
    }
    __device__ __forceinline__ void finish(int64_t m, int n, float4 s, const Extra& e) const {
        s.x = linear_act(s.x + e.bias.x, p.act) + e.residual.x;
        s.y = linear_act(s.y + e.bias.y, p.act) + e.residual.y;
        s.z = linear_act(s.z + e.bias.z, p.act) + e.residual.z;
        s.w = linear_act(s.w + e.bias.w, p.act) + e.residual.w;
        O* y = reinterpret_cast<O*>(p.y) + m * p.ldy + n;
        if (vec && n + 4 <= p.N) linear_store4(y, s);
        else each(n, [&](int j) { linear_store(y + j, at(s, j)); });
    }

private:
    static __device__ __forceinline__ float& at(float4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }
    template <typename F>
    __device__ __forceinline__ void each(int n, const F& f) const {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < p.N) f(j);
    }
};

}  // namespace exfold
