// Prefill routing on given routes: a token's K experts and weights come from the caller (a router that Eq. 2 does not
// describe). Retained set (Eq. 10), minimum-loss assignment (Eq. 12) and folding (Eq. 13) as in route_prefill.cu, and the same
// block histograms for the scatter kernel.
#include <algorithm>

#include "common.cuh"
#include "route_token.cuh"

namespace exfold {

namespace {

// One warp per token, lane k < K owns route k. Eq. 10 ranks by the product w h, one fp32 rounding, so that any implementation
// of it has the same order. A token is one chain of loads (ids, h, table entries): a warp per token of the block up to one block
// per SM, then the blocks fill the SMs.
__global__ void __launch_bounds__(kRouteMaxThreads) prefill_given_kernel(PrefillGivenParams gp) {
    __shared__ int hist[kMaxExperts];
    const PrefillRouteParams& p = gp.r;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int N = p.N, K = p.K, Kp = p.Kp, Ko = K - Kp;
    grid_dep_launch();
    for (int e = threadIdx.x; e < N; e += blockDim.x) hist[e] = 0;
    __syncthreads();
    grid_dep_wait();
    if (p.status != nullptr && blockIdx.x == 0 && threadIdx.x < 4) reinterpret_cast<int*>(p.status)[threadIdx.x] = 0;
    if (p.queue != nullptr && blockIdx.x == 0 && threadIdx.x < 2) p.queue[threadIdx.x] = 0;
    for (int tl = warp; tl < kRouteTokensPerBlock; tl += warps) {
        const int64_t i = (int64_t)blockIdx.x * kRouteTokensPerBlock + tl;
        if (i >= p.T) break;
        int id = lane < K ? gp.in_ids[i * K + lane] : 0;
        float w = lane < K ? gp.in_w[i * K + lane] : 0.f;
        if (id < 0 || id >= N) id = 0, w = 0.f;
        const uint32_t key = lane < K ? float_order_key(Ko > 0 ? __fmul_rn(w, gp.h[id]) : w) : 0u;
        const TokenRoute r = fold_token<true>(p, id, w, key, lane);
        if (r.kept) {
            p.ids[i * Kp + r.rank] = r.id;
            p.w[i * Kp + r.rank] = r.w;
            atomicAdd(&hist[r.id], 1);
        } else if (r.omitted) {
            p.omit_src[i * Ko + (r.rank - Kp)] = r.id;
            p.omit_tgt[i * Ko + (r.rank - Kp)] = r.tgt;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < N; e += blockDim.x) {
        const int c = hist[e];
        p.block_hist[(size_t)blockIdx.x * N + e] = c;
        if (c != 0 && p.sb_hist != nullptr) atomicAdd(&p.sb_hist[(size_t)(blockIdx.x / kRouteSuperBlock) * N + e], c);
    }
}

}  // namespace

cudaError_t launch_prefill_given(PrefillGivenParams p, cudaStream_t s) {
    const int nblk = (int)((p.r.T + kRouteTokensPerBlock - 1) / kRouteTokensPerBlock);
    if (nblk <= kRouteSuperBlock) {
        p.r.sb_hist = nullptr;  // one super-block: the scatter kernel adds up the block rows itself
    } else {  // the super-block histograms are added up with atomics: they start at zero
        const size_t nsb = (size_t)(nblk + kRouteSuperBlock - 1) / kRouteSuperBlock;
        cudaError_t e = cudaMemsetAsync(p.r.sb_hist, 0, nsb * p.r.N * sizeof(int32_t), s);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(prefill_given_kernel, nblk, nblk <= kRouteFewBlocks ? kRouteMaxThreads : kRouteThreads, 0, s, p);
}

}  // namespace exfold
