// What the dense-product kernels do to their sums: bias, activation, residual, one rounding to the output type.
#pragma once
#include <cooperative_groups.h>

#include "common.cuh"

namespace exfold {

// In forms that keep their relative accuracy where they tend to 0 (1 + erf and 1 + tanh leave a result at -5 two digits).
//
// v Phi(v), Phi(-x) = 1/2 erfc(x / sqrt 2) = exp(-x^2 / 2) t P(t) with t = 1 / (1 + x / sqrt 8): erfc times exp(x^2) as a polynomial in
// such a t is Hastings' form; this one (degree 8) was fitted for this file in equal ripples of the relative error, 4.3e-8 for x up
// to 14, behind which exp underflows. 64 x 14336 x 4096 with erff 25.3 us, with erfcf 26.0, with this 25.2.
__device__ __forceinline__ float linear_gelu(float v) {
    const float t = __fdividef(1.0f, fmaf(fabsf(v), 0.353553391f, 1.0f));
    float h = -0.0295346081f;
    h = fmaf(h, t, 0.142288089f);
    h = fmaf(h, t, -0.243601158f);
    h = fmaf(h, t, 0.139034897f);
    h = fmaf(h, t, -0.013313693f);
    h = fmaf(h, t, 0.101343781f);
    h = fmaf(h, t, 0.121551797f);
    h = fmaf(h, t, 0.141187668f);
    h = fmaf(h, t, 0.141043201f);
    h *= t * exp2f(-0.721347520f * (v * v));
    return v * (v < 0.f ? h : 1.0f - h);
}
__device__ __forceinline__ float linear_act(float v, int act) {
    switch (act) {  // uniform over the launch
        case EXFOLD_ACT_RELU: return v < 0.f ? 0.f : v;  // NaN stays
        case EXFOLD_ACT_GELU: return linear_gelu(v);
        // 1/2 (1 + tanh u) = 1 / (1 + exp(-2 u)); an exponential above 2^126 makes the quotient 0. 777 x 1411 x 2040 with tanhf 14.5 us,
        // with a rounded quotient 17.7, with this 14.5
        case EXFOLD_ACT_GELU_TANH: return __fdividef(v, 1.0f + expf(-1.59576912f * fmaf(0.044715f * v, v * v, v)));
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

template <typename O>
struct LinearFour;  // four neighbours as they lie in memory
template <>
struct LinearFour<float> { using type = float4; };
template <>
struct LinearFour<__nv_bfloat16> { using type = uint2; };

// Four neighbouring outputs of a row, bf16 operands; O is y's and the residual's type. For products whose groups of four are all whole
// and aligned (whole()).
template <typename O>
struct LinearEpilogue {
    using Raw = typename LinearFour<O>::type;
    const LinearParams& p;
    __host__ __device__ __forceinline__ explicit LinearEpilogue(const LinearParams& q) : p(q) {}
    __host__ __device__ __forceinline__ bool whole() const {
        const uintptr_t rows = reinterpret_cast<uintptr_t>(p.y) | reinterpret_cast<uintptr_t>(p.residual);
        return (rows & (4 * sizeof(O) - 1)) == 0 && (reinterpret_cast<uintptr_t>(p.bias) & 7) == 0 &&
               ((p.ldy | p.N | (p.residual != nullptr ? p.ldr : 0)) & 3) == 0;
    }
    // What comes from memory, asked for before the sum is there. Kept as it was loaded: a conversion would wait for the load, and
    // the next loads for the conversion.
    struct Extra {
        uint2 bias;
        Raw residual;
    };
    __device__ __forceinline__ Extra fetch(int64_t m, int n) const {
        Extra e;
        e.bias = make_uint2(0u, 0u);
        e.residual = Raw{};
        if (p.bias != nullptr) e.bias = *reinterpret_cast<const uint2*>(reinterpret_cast<const __nv_bfloat16*>(p.bias) + n);
        if (p.residual != nullptr) e.residual = *reinterpret_cast<const Raw*>(reinterpret_cast<const O*>(p.residual) + m * p.ldr + n);
        return e;
    }
    __device__ __forceinline__ void finish(int64_t m, int n, float4 s, const Extra& e) const {
        if (p.bias != nullptr) {
            const float4 b = linear_load4(reinterpret_cast<const __nv_bfloat16*>(&e.bias));
            s = make_float4(s.x + b.x, s.y + b.y, s.z + b.z, s.w + b.w);
        }
        s = make_float4(linear_act(s.x, p.act), linear_act(s.y, p.act), linear_act(s.z, p.act), linear_act(s.w, p.act));
        if (p.residual != nullptr) {
            const float4 r = linear_load4(reinterpret_cast<const O*>(&e.residual));
            s = make_float4(s.x + r.x, s.y + r.y, s.z + r.z, s.w + r.w);
        }
        linear_store4(reinterpret_cast<O*>(p.y) + m * p.ldy + n, s);
    }
};

// The S partial tiles of a cluster (rows x cols floats, cols 32, 64, 128 or 256, rows `ld` floats apart, at `part` in the shared memory of
// the cluster's CTAs first + k step) added up in the order of k and taken through the epilogue. The CTAs share the work: this one is
// number `me` of S, and its thread `tid` of THREADS takes every so-manieth group of four outputs. Bias and residual of U groups are
// asked for ahead, the first ones by begin(), while the products are still running; all loads of U groups are in flight together
// (those of places past the tile's end go to its last place). In a chain they made this part of a 128 x 256 tile 20 us.
// WHOLE: every group of four outputs is whole and aligned; else a thread takes single outputs, neighbours in neighbouring lanes.
// B: the bias' type (groups of four: bf16).
template <int S, typename O, int THREADS, bool WHOLE, typename B = __nv_bfloat16>
struct LinearReduce {
    static constexpr int U = S >= 8 ? 1 : S == 1 ? 4 : 2, kStride = S * THREADS;
    const LinearEpilogue<O>& ep;
    int rows, shift, total, n0, i0;
    int64_t row0;
    typename LinearEpilogue<O>::Extra extra[U];

    __device__ __forceinline__ LinearReduce(const LinearEpilogue<O>& e, int rows_, int cols, int64_t row0_, int n0_, int me, int tid)
        : ep(e), rows(rows_), shift(cols == 256 ? 6 : cols == 128 ? 5 : cols == 64 ? 4 : 3), total(rows_ << shift), n0(n0_), i0(me * THREADS + tid), row0(row0_) {}
    __device__ __forceinline__ void begin() {
        if (i0 >= total) return;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = min(i0 + u * kStride, total - 1), r = i >> shift, c = (i - (r << shift)) * 4;
            extra[u] = ep.fetch(row0 + r, min(n0 + c, ep.p.N - 4));
        }
    }
    __device__ __forceinline__ void run(const float* part, int ld, int first, int step) {
        cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
        const float* src[S];
#pragma unroll
        for (int k = 0; k < S; ++k) src[k] = S == 1 ? part : cluster.map_shared_rank(const_cast<float*>(part), first + k * step);
        for (; i0 < total; i0 += U * kStride) {
            float4 v[U][S];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = min(i0 + u * kStride, total - 1), r = i >> shift, c = (i - (r << shift)) * 4;
#pragma unroll
                for (int k = 0; k < S; ++k) v[u][k] = *reinterpret_cast<const float4*>(src[k] + (size_t)r * ld + c);
            }
            typename LinearEpilogue<O>::Extra now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) now[u] = extra[u];
            const int at = i0;
            i0 += U * kStride;
            begin();
            i0 = at;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kStride, r = i >> shift, c = (i - (r << shift)) * 4;
                float4 t = v[u][0];
#pragma unroll
                for (int k = 1; k < S; ++k) {
                    t.x += v[u][k].x;
                    t.y += v[u][k].y;
                    t.z += v[u][k].z;
                    t.w += v[u][k].w;
                }
                if (i < total && n0 + c < ep.p.N) ep.finish(row0 + r, n0 + c, t, now[u]);
            }
        }
    }
};
template <int S, typename O, int THREADS, typename B>
struct LinearReduce<S, O, THREADS, false, B> {
    static constexpr int U = S >= 8 ? 2 : S >= 3 ? 4 : 8, kStride = S * THREADS;
    const LinearParams& l;
    int shift, total, n0, i0;
    int64_t row0;
    B bias[U];
    O residual[U];

    __device__ __forceinline__ LinearReduce(const LinearEpilogue<O>& e, int rows, int cols, int64_t row0_, int n0_, int me, int tid)
        : l(e.p), shift(cols == 256 ? 8 : cols == 128 ? 7 : cols == 64 ? 6 : 5), total(rows << shift), n0(n0_), i0(me * THREADS + tid), row0(row0_) {}
    __device__ __forceinline__ void begin() {
        if (i0 >= total) return;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = min(i0 + u * kStride, total - 1), r = i >> shift, n = min(n0 + i - (r << shift), l.N - 1);
            if (l.bias != nullptr) bias[u] = reinterpret_cast<const B*>(l.bias)[n];
            if (l.residual != nullptr) residual[u] = reinterpret_cast<const O*>(l.residual)[(row0 + r) * l.ldr + n];
        }
    }
    __device__ __forceinline__ void run(const float* part, int ld, int first, int step) {
        cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
        const float* src[S];
#pragma unroll
        for (int k = 0; k < S; ++k) src[k] = S == 1 ? part : cluster.map_shared_rank(const_cast<float*>(part), first + k * step);
        for (; i0 < total; i0 += U * kStride) {
            float v[U][S];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = min(i0 + u * kStride, total - 1), r = i >> shift;
#pragma unroll
                for (int k = 0; k < S; ++k) v[u][k] = src[k][(size_t)r * ld + i - (r << shift)];
            }
            float b[U], a[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                b[u] = l.bias != nullptr ? linear_f32(bias[u]) : 0.f;
                a[u] = l.residual != nullptr ? linear_f32(residual[u]) : 0.f;
            }
            const int at = i0;
            i0 += U * kStride;
            begin();
            i0 = at;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kStride, r = i >> shift, n = n0 + i - (r << shift);
                float t = v[u][0];
#pragma unroll
                for (int k = 1; k < S; ++k) t += v[u][k];
                if (l.bias != nullptr) t += b[u];
                t = linear_act(t, l.act);
                if (l.residual != nullptr) t += a[u];
                if (i < total && n < l.N) linear_store(reinterpret_cast<O*>(l.y) + (row0 + r) * l.ldy + n, t);
            }
        }
    }
};

}  // namespace exfold
