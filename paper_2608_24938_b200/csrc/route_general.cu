// Routing by a model's own router: softmax or sigmoid scores, a bias for the choice, expert groups, Top-K, weights; and the
// gradient of those weights with respect to the router scores.
#include <algorithm>

#include "common.cuh"

namespace exfold {

namespace {

constexpr int kGrThreads = 256;
constexpr int kGrWarps = kGrThreads / 32;
constexpr float kMaskedScore = -3.402823466e38f;  // this and -infinity

// Order-preserving image of a double; every NaN is the largest, -0 is +0
__device__ __forceinline__ unsigned long long order64(double c) {
    if (c != c) return ~0ull;
    const unsigned long long b = (unsigned long long)__double_as_longlong(c + 0.0);
    return (b >> 63) ? ~b : b | (1ull << 63);
}

// The same of a float
__device__ __forceinline__ unsigned order32(float f) { return f != f ? 0xffffffffu : float_order_key(f); }

// One warp per token, expert lane + 32 q in register q. Choices are compared in 64 bits: two experts' choices may differ by
// less than an fp32 rounding of them.
template <int NPL>
__global__ void __launch_bounds__(kGrThreads) route_general_kernel(RouteGeneralParams p) {
    extern __shared__ unsigned long long s_key[];  // [warps][N], with groups only
    __shared__ int hist[kMaxExperts];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int N = p.N, K = p.K;
    grid_dep_launch();
    if (p.load != nullptr) {
        for (int e = threadIdx.x; e < N; e += kGrThreads) hist[e] = 0;
        __syncthreads();
    }
    grid_dep_wait();
    for (int64_t i = (int64_t)blockIdx.x * kGrWarps + warp; i < p.T; i += (int64_t)gridDim.x * kGrWarps) {
        const float* z = p.logits + i * N;
        float v[NPL];
        unsigned long long key[NPL];
        unsigned cand = 0, masked = 0;  // bits of this lane's experts
        float zmax = -INFINITY;
#pragma unroll
        for (int q = 0; q < NPL; ++q) {
            const int e = lane + 32 * q;
            v[q] = e < N ? z[e] : -INFINITY;
            if (e < N) cand |= 1u << q;
            if (v[q] <= kMaskedScore) masked |= 1u << q;
            zmax = isnan(v[q]) || v[q] > zmax ? v[q] : zmax;
        }
        double sum = 0.0;
        if (p.softmax) {
            zmax = float_from_order_key(__reduce_max_sync(0xffffffffu, order32(zmax)));
#pragma unroll
            for (int q = 0; q < NPL; ++q)
                if (!((masked >> q) & 1u)) sum += exp((double)v[q] - (double)zmax);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        auto score = [&](float zz) -> double {
            if (zz <= kMaskedScore) return 0.0;
            return p.softmax ? exp((double)zz - (double)zmax) / sum : 1.0 / (1.0 + exp(-(double)zz));
        };
#pragma unroll
        for (int q = 0; q < NPL; ++q) {
            const int e = lane + 32 * q;
            const double c = (masked >> q) & 1u ? -INFINITY : p.by_score ? score(v[q]) + (p.bias != nullptr && e < N ? (double)p.bias[e] : 0.0) : (double)v[q];
            key[q] = order64(c);
        }
        if (p.n_groups > 1) {
            // groups: lane g takes group g's score and its place among the groups
            unsigned long long* sk = s_key + warp * N;
            __syncwarp();
#pragma unroll
            for (int q = 0; q < NPL; ++q)
                if (lane + 32 * q < N) sk[lane + 32 * q] = key[q];
            __syncwarp();
            const int per = N / p.n_groups;
            unsigned long long k1 = 0, k2 = 0;
            if (lane < p.n_groups)
                for (int j = 0; j < per; ++j) {
                    const unsigned long long k = sk[lane * per + j];
                    if (k > k1) { k2 = k1; k1 = k; }
                    else if (k > k2) k2 = k;
                }
            if (p.group_top2) {
                auto value = [](unsigned long long k) {
                    if (k == ~0ull) return (double)NAN;
                    return __longlong_as_double((long long)((k >> 63) ? k & ~(1ull << 63) : ~k));
                };
                const unsigned long long none = order64(-INFINITY);
                if (k2 > none) k1 = order64(value(k1) + value(k2));
            }
            int place = 0;
            for (int g = 0; g < p.n_groups; ++g) {
                const unsigned long long kg = __shfl_sync(0xffffffffu, k1, g);
                if (kg > k1 || (kg == k1 && g < lane)) ++place;
            }
            const unsigned stay = __ballot_sync(0xffffffffu, lane < p.n_groups && place < p.top_groups);
#pragma unroll
            for (int q = 0; q < NPL; ++q)
                if (!((stay >> min(31, (lane + 32 * q) / per)) & 1u)) cand &= ~(1u << q);
        }
        int my_id = 0;
        for (int k = 0; k < K; ++k) {
            unsigned long long bk = 0;
            int be = 0x7fffffff;
#pragma unroll
            for (int q = 0; q < NPL; ++q)
                if (((cand >> q) & 1u) && (be == 0x7fffffff || key[q] > bk)) {
                    bk = key[q];
                    be = lane + 32 * q;
                }
            const bool has = be != 0x7fffffff;
            const unsigned hi = __reduce_max_sync(0xffffffffu, has ? (unsigned)(bk >> 32) : 0u);
            const bool top = has && (unsigned)(bk >> 32) == hi;
            const unsigned lo = __reduce_max_sync(0xffffffffu, top ? (unsigned)bk : 0u);
            be = __reduce_min_sync(0xffffffffu, top && (unsigned)bk == lo ? be : 0x7fffffff);
            if ((be & 31) == lane) cand &= ~(1u << (be >> 5));
            if (lane == k) my_id = be;
        }
        double s = lane < K ? score(z[my_id]) : 0.0;
        if (p.renormalise) {
            double total = 0.0;
            for (int k = 0; k < K; ++k) total += __shfl_sync(0xffffffffu, s, k);
            s = total != 0.0 ? s / total : 0.0;
        }
        if (lane < K) {
            p.ids[i * K + lane] = my_id;
            p.w[i * K + lane] = (float)(s * (double)p.scale);
            if (p.load != nullptr) atomicAdd(&hist[my_id], 1);
        }
    }
    if (p.load != nullptr) {
        __syncthreads();
        for (int e = threadIdx.x; e < N; e += kGrThreads) {
            if (gridDim.x == 1) p.load[e] = hist[e];
            else if (hist[e] != 0) atomicAdd(&p.load[e], hist[e]);
        }
    }
}

// One warp per token: lane k < K holds the chosen expert k, the row is put together in registers
template <int NPL>
__global__ void __launch_bounds__(kGrThreads) route_backward_kernel(RouteBackwardParams p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int N = p.N, K = p.K;
    grid_dep_launch();
    grid_dep_wait();
    for (int64_t i = (int64_t)blockIdx.x * kGrWarps + warp; i < p.T; i += (int64_t)gridDim.x * kGrWarps) {
        const float* z = p.logits + i * N;
        const bool dense = p.softmax && !p.renormalise;
        float out[NPL];
#pragma unroll
        for (int q = 0; q < NPL; ++q) out[q] = 0.f;
        int id = lane < K ? p.ids[i * K + lane] : -1;
        if (id < 0 || id >= N) id = -1;
        const float g = id >= 0 ? p.dw[i * K + lane] : 0.f;
        const float zk = id >= 0 ? z[id] : -INFINITY;
        const bool live = zk > kMaskedScore || isnan(zk);
        float dz;  // of the chosen expert
        if (dense) {
            float v[NPL], zmax = -INFINITY;
#pragma unroll
            for (int q = 0; q < NPL; ++q) {
                v[q] = lane + 32 * q < N ? z[lane + 32 * q] : -INFINITY;
                zmax = isnan(v[q]) || v[q] > zmax ? v[q] : zmax;
            }
            zmax = float_from_order_key(__reduce_max_sync(0xffffffffu, order32(zmax)));
            float sum = 0.f;
#pragma unroll
            for (int q = 0; q < NPL; ++q) {
                out[q] = v[q] <= kMaskedScore ? 0.f : expf(v[q] - zmax);
                sum += out[q];
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float sk = live ? expf(zk - zmax) / sum : 0.f;
            dz = live ? p.scale * g * sk : 0.f;
            float dot = dz;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
#pragma unroll
            for (int q = 0; q < NPL; ++q) out[q] = out[q] == 0.f ? 0.f : -dot * (out[q] / sum);
        } else {
            double s = 0.0, rest = 1.0;  // score (softmax: up to a factor), 1 - score
            if (p.softmax) {
                const float m = float_from_order_key(__reduce_max_sync(0xffffffffu, order32(live ? zk : -INFINITY)));
                if (live) s = exp((double)zk - (double)m);
            } else if (live) {
                const double e = exp(-fabs((double)zk)), r = 1.0 / (1.0 + e);
                s = zk >= 0.f ? r : e * r;
                rest = zk >= 0.f ? e * r : r;
                if (isnan(zk)) s = rest = NAN;
            }
            double ds = (double)g;
            double factor = s;
            if (p.renormalise) {
                double total = s, dot = live ? s * (double)g : 0.0;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    total += __shfl_xor_sync(0xffffffffu, total, o);
                    dot += __shfl_xor_sync(0xffffffffu, dot, o);
                }
                factor = total != 0.0 ? s / total : 0.0;
                ds = total != 0.0 ? (double)g - dot / total : 0.0;
            }
            dz = live ? (float)((double)p.scale * factor * ds * rest) : 0.f;
        }
        for (int k = 0; k < K; ++k) {
            const int e = __shfl_sync(0xffffffffu, id, k);
            const float d = __shfl_sync(0xffffffffu, dz, k);
            if (e < 0 || (e & 31) != lane) continue;
#pragma unroll
            for (int q = 0; q < NPL; ++q)
                if (q == (e >> 5)) out[q] += d;
        }
        float* dst = p.dlogits + i * N;
#pragma unroll
        for (int q = 0; q < NPL; ++q)
            if (lane + 32 * q < N) dst[lane + 32 * q] = out[q];
    }
}

}  // namespace

cudaError_t launch_route_general(const RouteGeneralParams& p, int sms, cudaStream_t s) {
    const unsigned blocks = (unsigned)std::max<int64_t>(1, std::min<int64_t>((p.T + kGrWarps - 1) / kGrWarps, (int64_t)8 * sms));
    if (p.load != nullptr && (blocks > 1 || p.T == 0)) {
        cudaError_t e = cudaMemsetAsync(p.load, 0, (size_t)p.N * sizeof(int32_t), s);
        if (e != cudaSuccess) return e;
    }
    if (p.T == 0) return cudaSuccess;
    const size_t smem = p.n_groups > 1 ? (size_t)kGrWarps * p.N * sizeof(unsigned long long) : 0;
    switch ((p.N + 31) / 32) {
        case 1: return launch_pdl(route_general_kernel<1>, blocks, kGrThreads, smem, s, p);
        case 2: return launch_pdl(route_general_kernel<2>, blocks, kGrThreads, smem, s, p);
        case 3: case 4: return launch_pdl(route_general_kernel<4>, blocks, kGrThreads, smem, s, p);
        default: return launch_pdl(route_general_kernel<8>, blocks, kGrThreads, smem, s, p);
    }
}

cudaError_t launch_route_backward(const RouteBackwardParams& p, int sms, cudaStream_t s) {
    if (p.T == 0) return cudaSuccess;
    const unsigned blocks = (unsigned)std::min<int64_t>((p.T + kGrWarps - 1) / kGrWarps, (int64_t)8 * sms);
    switch ((p.N + 31) / 32) {
        case 1: return launch_pdl(route_backward_kernel<1>, blocks, kGrThreads, 0, s, p);
        case 2: return launch_pdl(route_backward_kernel<2>, blocks, kGrThreads, 0, s, p);
        case 3: case 4: return launch_pdl(route_backward_kernel<4>, blocks, kGrThreads, 0, s, p);
        default: return launch_pdl(route_backward_kernel<8>, blocks, kGrThreads, 0, s, p);
    }
}

}  // namespace exfold
