// Dense product with epilogue, bf16 operands, at most 8 tokens: the weights stream from global memory straight into the fragments of
// mma.sync m16n8k16, as in decode_small.cu.
//
// Next to no arithmetic is done on a weight, so the time is the weights' bytes over HBM and every fixed cost on the way: no tensor
// memory, no tensor maps, no barriers but one per CTA. A work item is 16 features; a lane loads 32 contiguous bytes of a weight
// row (4 lanes a whole 128-byte line), and since the order of K inside a product does not matter, those 16 elements serve as the
// lane's K positions of four MMAs while the tokens, the 8-column operand, use the same order. The warps of a CTA, and where items
// are few the CTAs of a cluster, split K; their sums meet in shared memory in a fixed order.
#include <algorithm>

#include "common.cuh"
#include "linear_epilogue.cuh"
#include "ptx.cuh"

#include <cooperative_groups.h>

namespace exfold {

namespace {

namespace cg = cooperative_groups;

constexpr int kSmMaxWarps = 16;
constexpr int kSmKC = 64;     // K elements per chunk: one 128-byte line of a weight row
constexpr int kSmUnroll = 2;  // chunks per warp in flight while as many are multiplied

// 16 elements at p, of which the first n (a multiple of 8, maybe none) exist; the rest are zeros
template <bool WIDE, bool STREAM>
__device__ __forceinline__ void ld16(uint32_t (&r)[8], const __nv_bfloat16* p, int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = 0u;
    if constexpr (WIDE) {
        if (n <= 0) return;
        if constexpr (STREAM)  // read once: not kept in L1
            asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                         : "l"(p));
        else
            asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                         : "l"(p));
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (n > 8 * h) {
                const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + h);
                r[4 * h] = v.x; r[4 * h + 1] = v.y; r[4 * h + 2] = v.z; r[4 * h + 3] = v.w;
            }
    }
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// WIDE: 32-byte loads
template <typename O, bool WIDE>
__global__ void __launch_bounds__(32 * kSmMaxWarps, 1) linear_small_kernel(LinearParams p, int split) {
    __shared__ float4 s_red[kSmMaxWarps][32];
    __shared__ float s_out[8][16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = (int)blockDim.x >> 5;
    const int part = (int)blockIdx.x % split, n0 = (int)blockIdx.x / split * 16;
    const int T = (int)p.T, K = p.K, nch = (K + kSmKC - 1) / kSmKC;
    const int lr = lane >> 2, lk = (lane & 3) * 16;
    const __nv_bfloat16* w0 = reinterpret_cast<const __nv_bfloat16*>(p.w) + (int64_t)min(n0 + lr, p.N - 1) * p.ldw + lk;
    const __nv_bfloat16* w1 = reinterpret_cast<const __nv_bfloat16*>(p.w) + (int64_t)min(n0 + lr + 8, p.N - 1) * p.ldw + lk;
    const __nv_bfloat16* x = reinterpret_cast<const __nv_bfloat16*>(p.x) + (int64_t)lr * p.ldx + lk;
    const int step = split * n_warps;
    uint32_t an[kSmUnroll][2][8], xn[kSmUnroll][8];
    auto load = [&](int j0) {
#pragma unroll
        for (int u = 0; u < kSmUnroll; ++u) {
            const int j = j0 + u * step, left = j < nch ? min(16, K - j * kSmKC - lk) : 0;
            ld16<WIDE, true>(an[u][0], w0 + (int64_t)j * kSmKC, left);
            ld16<WIDE, true>(an[u][1], w1 + (int64_t)j * kSmKC, left);
            ld16<WIDE, false>(xn[u], x + (int64_t)j * kSmKC, lr < T ? left : 0);
        }
    };
    grid_dep_wait();
    if (blockIdx.x == 0 && tid < 4) reinterpret_cast<int*>(p.status)[tid] = 0;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    const int first = part * n_warps + warp;
    load(first);
    for (int j0 = first; j0 < nch; j0 += kSmUnroll * step) {
        uint32_t a[kSmUnroll][2][8], b[kSmUnroll][8];
#pragma unroll
        for (int u = 0; u < kSmUnroll; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                a[u][0][i] = an[u][0][i];
                a[u][1][i] = an[u][1][i];
                b[u][i] = xn[u][i];
            }
        load(j0 + kSmUnroll * step);
#pragma unroll
        for (int u = 0; u < kSmUnroll; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                mma16816(acc, a[u][0][2 * i], a[u][1][2 * i], a[u][0][2 * i + 1], a[u][1][2 * i + 1], b[u][2 * i], b[u][2 * i + 1]);
    }
    s_red[warp][lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    grid_dep_launch();
    // lane l of the first warp ends up with tokens l / 16 + 2 u, feature l % 16: what that needs besides the sums
    const int col = n0 + (lane & 15), tok0 = lane >> 4;
    const bool ends = part == 0 && warp == 0 && col < p.N;
    __nv_bfloat16 bias = __float2bfloat16_rn(0.f);
    O residual[4];
    if (ends) {
        if (p.bias != nullptr) bias = reinterpret_cast<const __nv_bfloat16*>(p.bias)[col];
        if (p.residual != nullptr)
#pragma unroll
            for (int u = 0; u < 4; ++u) residual[u] = reinterpret_cast<const O*>(p.residual)[(int64_t)min(tok0 + 2 * u, T - 1) * p.ldr + col];
    }
    __syncthreads();
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (warp == 0) {
        sum = s_red[0][lane];
        for (int v = 1; v < n_warps; ++v) {
            const float4 q = s_red[v][lane];
            sum.x += q.x;
            sum.y += q.y;
            sum.z += q.z;
            sum.w += q.w;
        }
    }
    if (split > 1) {  // the cluster's parts in order
        cg::cluster_group cluster = cg::this_cluster();
        if (warp == 0) s_red[0][lane] = sum;
        cluster.sync();
        if (warp == 0 && part == 0)
            for (int q = 1; q < split; ++q) {
                const float4 v = cluster.map_shared_rank(&s_red[0][0], q)[lane];
                sum.x += v.x;
                sum.y += v.y;
                sum.z += v.z;
                sum.w += v.w;
            }
        cluster.sync();  // no CTA leaves while its part may still be read
    }
    if (warp == 0 && part == 0) {
        const int t = (lane & 3) * 2;  // sum.x, .y: feature lr, tokens t and t + 1; .z, .w: feature lr + 8
        s_out[t][lr] = sum.x;
        s_out[t + 1][lr] = sum.y;
        s_out[t][lr + 8] = sum.z;
        s_out[t + 1][lr + 8] = sum.w;
        __syncwarp();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = tok0 + 2 * u;
            if (!ends || k >= T) continue;
            float v = s_out[k][lane & 15];
            if (p.bias != nullptr) v += linear_f32(bias);
            v = linear_act(v, p.act);
            if (p.residual != nullptr) v += linear_f32(residual[u]);
            linear_store(reinterpret_cast<O*>(p.y) + k * p.ldy + col, v);
        }
    }
}

}  // namespace

// Whether this kernel takes a call (both operands start on 16-byte boundaries, with rows multiples of 8 elements apart). Up to two rounds
// of items: every round starts with empty pipes. This kernel / linear_tile.cu, on the GPU with bias and residual (tokens x features x K):
// 1 x 4096 x 4096 8.9 / 9.7 us, 1 x 768 x 2048 3.8 / 4.3, 4 x 6144 x 4096 14.2 / 18.3, 1 x 8192 x 2048 9.5 / 9.8, 1 x 14336 x 4096 24.9 / 21.1,
// 8 x 14336 x 1024 13.2 / 9.0. (A persistent form, the next item's weights asked for while one item's sums meet, spilled registers:
// 1 x 4096 x 4096 9.4 us, 1 x 14336 x 4096 25.3.)
bool linear_small_fits(const LinearParams& p, int sms) { return p.T <= 8 && p.K % 8 == 0 && (p.N + 15) / 16 <= 4 * sms; }

cudaError_t launch_linear_small(const LinearParams& p, bool out_bf16, int sms, cudaStream_t s) {
    const bool wide = ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.w)) & 31) == 0 && ((p.ldx | p.ldw | p.K) & 15) == 0;
    // 16 warps per SM: one CTA of 16 warps where there are no more items than SMs (a cluster per item when there are at most half
    // as many), else CTAs of 8 warps
    const int items = (p.N + 15) / 16, nch = (p.K + kSmKC - 1) / kSmKC;
    const int warps = std::min(items <= sms ? kSmMaxWarps : kSmMaxWarps / 2, std::max(1, nch));
    int split = 1;
    while (split < 8 && items * split * 2 <= sms && nch >= 2 * split * warps) split *= 2;
    auto go = [&](auto kernel) { return launch_pdl_cluster(kernel, (unsigned)(items * split), 32 * warps, 0, split, s, p, split); };
    if (out_bf16) return wide ? go(linear_small_kernel<__nv_bfloat16, true>) : go(linear_small_kernel<__nv_bfloat16, false>);
    return wide ? go(linear_small_kernel<float, true>) : go(linear_small_kernel<float, false>);
}

}  // namespace exfold
