// Dense product with bias, activation and residual in its epilogue, y = act(x W^T + b) + r: the CUDA-core kernel, for fp32
// operands and for bf16 ones that the tensor-core kernels cannot load.
#include <algorithm>

#include "common.cuh"
#include "linear_epilogue.cuh"

namespace exfold {

namespace {

constexpr int kLsThreads = 256;
constexpr int kLsBK = 16;

// Two products at once: the packed form issues half as many instructions
__device__ __forceinline__ void fma2(float2& c, const float2& a, const float2& b) {
    asm("fma.rn.f32x2 %0, %1, %2, %0;"
        : "+l"(reinterpret_cast<unsigned long long&>(c))
        : "l"(reinterpret_cast<const unsigned long long&>(a)), "l"(reinterpret_cast<const unsigned long long&>(b)));
}

// BM x BN outputs per block, K in steps of 16 through shared memory (transposed, double buffered); a thread owns TM x TN of
// them. VEC: rows of x and w can be read four elements at a time.
template <typename T, typename O, int BM, int BN, bool VEC>
__global__ void __launch_bounds__(kLsThreads) linear_simt_kernel(LinearParams p) {
    constexpr int TM = BM / 16, TN = BN / 16;
    constexpr int kA = BM * kLsBK / 4 / kLsThreads, kB = BN * kLsBK / 4 / kLsThreads;  // groups of four elements per thread
    __shared__ __align__(16) float sa[2][kLsBK][BM + 4];
    __shared__ __align__(16) float sb[2][kLsBK][BN + 4];
    const T* x = reinterpret_cast<const T*>(p.x);
    const T* w = reinterpret_cast<const T*>(p.w);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int n_tiles = (p.N + BN - 1) / BN;
    const int64_t m0 = (int64_t)(blockIdx.x / n_tiles) * BM;
    const int n0 = (int)(blockIdx.x % n_tiles) * BN;
    grid_dep_launch();
    grid_dep_wait();
    if (blockIdx.x == 0 && tid < 4) reinterpret_cast<int*>(p.status)[tid] = 0;
    float ra[kA][4], rb[kB][4];
    auto fetch = [&](const T* base, int64_t row, int64_t rows, int64_t ld, int k, float (&v)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = 0.f;
        if (row >= rows) return;
        const T* src = base + row * ld + k;
        if (VEC && k + 4 <= p.K) {
            const float4 t = linear_load4(src);
            v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k + j < p.K) v[j] = linear_f32(src[j]);
        }
    };
    auto load = [&](int k0) {
#pragma unroll
        for (int u = 0; u < kA; ++u) {
            const int i = tid + u * kLsThreads;
            fetch(x, m0 + i / 4, p.T, p.ldx, k0 + i % 4 * 4, ra[u]);
        }
#pragma unroll
        for (int u = 0; u < kB; ++u) {
            const int i = tid + u * kLsThreads;
            fetch(w, n0 + i / 4, p.N, p.ldw, k0 + i % 4 * 4, rb[u]);
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int u = 0; u < kA; ++u) {
            const int i = tid + u * kLsThreads;
#pragma unroll
            for (int j = 0; j < 4; ++j) sa[buf][i % 4 * 4 + j][i / 4] = ra[u][j];
        }
#pragma unroll
        for (int u = 0; u < kB; ++u) {
            const int i = tid + u * kLsThreads;
#pragma unroll
            for (int j = 0; j < 4; ++j) sb[buf][i % 4 * 4 + j][i / 4] = rb[u][j];
        }
    };
    float2 acc[TM][TN / 2];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN / 2; ++j) acc[i][j] = make_float2(0.f, 0.f);
    load(0);
    store(0);
    __syncthreads();
    int buf = 0;
    for (int k0 = 0; k0 < p.K; k0 += kLsBK) {
        const bool more = k0 + kLsBK < p.K;
        if (more) load(k0 + kLsBK);
#pragma unroll
        for (int k = 0; k < kLsBK; ++k) {
            // a thread's rows and columns lie four apart from its neighbours': 16-byte reads without bank conflicts
            float a[TM];
            float2 b[TN / 2];
#pragma unroll
            for (int u = 0; u < TM / 4; ++u) {
                const float4 v = *reinterpret_cast<const float4*>(&sa[buf][k][u * 64 + ty * 4]);
                a[4 * u] = v.x; a[4 * u + 1] = v.y; a[4 * u + 2] = v.z; a[4 * u + 3] = v.w;
            }
#pragma unroll
            for (int u = 0; u < TN / 4; ++u) {
                const float4 v = *reinterpret_cast<const float4*>(&sb[buf][k][u * 64 + tx * 4]);
                b[2 * u] = make_float2(v.x, v.y);
                b[2 * u + 1] = make_float2(v.z, v.w);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN / 2; ++j) fma2(acc[i][j], make_float2(a[i], a[i]), b[j]);
        }
        if (more) store(buf ^ 1);
        __syncthreads();
        buf ^= 1;
    }
    const T* bias = reinterpret_cast<const T*>(p.bias);
    O* y = reinterpret_cast<O*>(p.y);
    const O* r = reinterpret_cast<const O*>(p.residual);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int n = n0 + (j >> 2) * 64 + tx * 4 + (j & 3);
        if (n >= p.N) continue;
        const float bv = bias != nullptr ? linear_f32(bias[n]) : 0.f;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t m = m0 + (i >> 2) * 64 + ty * 4 + (i & 3);
            if (m >= p.T) continue;
            float v = linear_act(((j & 1) ? acc[i][j / 2].y : acc[i][j / 2].x) + bv, p.act);
            if (r != nullptr) v += linear_f32(r[m * p.ldr + n]);
            linear_store(y + m * p.ldy + n, v);
        }
    }
}

template <typename T, typename O, bool VEC>
cudaError_t launch_simt_t(const LinearParams& p, int sms, cudaStream_t s) {
    auto blocks = [&](int b) { return ((p.T + b - 1) / b) * ((p.N + b - 1) / b); };
    const bool large = blocks(128) >= sms;
    const int64_t grid = blocks(large ? 128 : 64);
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    if (large) return launch_pdl(linear_simt_kernel<T, O, 128, 128, VEC>, (unsigned)grid, kLsThreads, 0, s, p);
    return launch_pdl(linear_simt_kernel<T, O, 64, 64, VEC>, (unsigned)grid, kLsThreads, 0, s, p);
}

}  // namespace

cudaError_t launch_linear_simt(const LinearParams& p, bool bf16, bool out_bf16, int sms, cudaStream_t s) {
    const uintptr_t bytes = bf16 ? 8 : 16;
    const bool vec = ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.w)) & (bytes - 1)) == 0 && ((p.ldx | p.ldw) & 3) == 0;
    if (!bf16) return vec ? launch_simt_t<float, float, true>(p, sms, s) : launch_simt_t<float, float, false>(p, sms, s);
    if (out_bf16)
        return vec ? launch_simt_t<__nv_bfloat16, __nv_bfloat16, true>(p, sms, s) : launch_simt_t<__nv_bfloat16, __nv_bfloat16, false>(p, sms, s);
    return vec ? launch_simt_t<__nv_bfloat16, float, true>(p, sms, s) : launch_simt_t<__nv_bfloat16, float, false>(p, sms, s);
}

}  // namespace exfold
