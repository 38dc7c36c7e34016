// Dense product with epilogue, bf16 operands, few tokens or few tiles: one CTA per 128 tokens x bn features, K split over a
// cluster.
//
// A decode batch reads the whole weight matrix for a few tokens, so its time is the weights' bytes over HBM and what a launch
// costs; a short prompt has fewer 256 x 256 tiles than SM pairs. Either way the work has to be spread over K: a cluster of `split`
// CTAs shares a tile, each multiplies its part of K into its own tensor memory, the fp32 partial tiles meet in shared memory, and
// every CTA sums a share of the rows over the cluster through distributed shared memory in rank order (the same bits every time) and
// takes them through bias, activation and residual.
// The token box has only the rows there are, up to 128; the rest of the MMA's 128 rows is whatever follows in shared memory and
// ends in accumulator rows that nobody reads. Columns past K are the tensor maps' zero fill.
#include <algorithm>

#include "common.cuh"
#include "linear_epilogue.cuh"
#include "ptx.cuh"

#include <cooperative_groups.h>

namespace exfold {

namespace {

namespace cg = cooperative_groups;

constexpr int kLtThreads = 192;  // warp 0: TMA producer, warp 1: MMA issuer, warps 2-5: accumulator rows; all: epilogue
constexpr int kLtMaxStages = 12;
constexpr int kLtBK = kGemmBK;

template <typename O>
__global__ void __launch_bounds__(kLtThreads) linear_tile_kernel(const __grid_constant__ LinearTileParams p) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kLtMaxStages];
    __shared__ __align__(8) uint64_t empty_bar[kLtMaxStages];
    __shared__ __align__(8) uint64_t done_bar;
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s;
    unsigned char* tiles =
        reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int split = p.plan.split, bn = p.plan.bn, stages = p.plan.stages, rank = (int)cluster.block_rank();
    const int nt = (p.l.N + bn - 1) / bn, tile = (int)blockIdx.x / split;
    const int n0 = tile % nt * bn;
    const int64_t row0 = (int64_t)(tile / nt) * kTileM;
    uint32_t tmem_cols = 32;
    while ((int)tmem_cols < bn) tmem_cols *= 2;
    if (threadIdx.x == 0) {
        ptx::prefetch_tmap(&p.tm_x);
        ptx::prefetch_tmap(&p.tm_w);
        for (int s = 0; s < stages; ++s) {
            ptx::mbar_init(&full_bar[s], 1);
            ptx::mbar_init(&empty_bar[s], 1);
        }
        ptx::mbar_init(&done_bar, 1);
        abort_s = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc(&tmem_base_s, tmem_cols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    grid_dep_wait();
    if (blockIdx.x == 0 && threadIdx.x < 4) reinterpret_cast<int*>(p.l.status)[threadIdx.x] = 0;
    const uint32_t tmem_base = tmem_base_s;
    volatile int* abort_flag = &abort_s;
    const int nkb = (p.l.K + kLtBK - 1) / kLtBK;
    const int kb0 = rank * nkb / split, kb1 = (rank + 1) * nkb / split;  // never empty: split <= nkb
    const int a_bytes = p.plan.a_rows * kLtBK * 2, stage_bytes = a_bytes + bn * kLtBK * 2;
    const int rows = (int)min((int64_t)kTileM, p.l.T - row0);
    const int part_ld = bn + 4;  // floats: 16-byte aligned rows, the rows of a quarter warp in distinct banks

    if (warp == 0) {
        if (ptx::elect_one()) {
            int stage = 0, phase = 0;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!ptx::mbar_wait_local(&empty_bar[stage], phase ^ 1, abort_flag, p.l.status, 1)) break;
                unsigned char* dst = tiles + stage * stage_bytes;
                ptx::mbar_expect_tx(&full_bar[stage], stage_bytes);
                ptx::tma_load_2d(dst + a_bytes, &p.tm_w, &full_bar[stage], kb * kLtBK, n0);
                ptx::tma_load_2d(dst, &p.tm_x, &full_bar[stage], kb * kLtBK, (int)row0);
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (ptx::elect_one()) {
            const uint32_t idesc = ptx::make_idesc_bf16(128, 0) | ((uint32_t)(bn >> 3) << 17);
            const uint32_t lo0 = (ptx::smem_u32(tiles) & 0x3FFFFu) >> 4;
            const uint32_t hi = (uint32_t)(ptx::make_kmajor_sw128_desc(0) >> 32);
            int stage = 0, phase = 0;
            bool ok = true, ready = false;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!ready && !ptx::mbar_wait_local(&full_bar[stage], phase, abort_flag, p.l.status, 3)) {
                    ok = false;
                    break;
                }
                const int ns = stage + 1 == stages ? 0 : stage + 1, nphase = ns == 0 ? phase ^ 1 : phase;
                const uint32_t a_lo = lo0 + (uint32_t)(stage * stage_bytes >> 4);
                ready = ptx::umma_kblock_bf16(tmem_base, a_lo, a_lo + (a_bytes >> 4), hi, idesc, kb > kb0 ? 1u : 0u,
                                              &empty_bar[stage], &full_bar[ns], nphase);
                stage = ns;
                phase = nphase;
            }
            if (ok) ptx::umma_commit(&done_bar);
        }
        __syncwarp();
    } else {
        // partial tile -> shared memory (the ring is free once every MMA has completed)
        const int q = warp & 3;
        int ok = 1;
        if (lane == 0) ok = ptx::mbar_wait_local(&done_bar, 0, abort_flag, p.l.status, 4) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (ok && q * 32 < rows) {
            ptx::tc_fence_after();
            float* dst = reinterpret_cast<float*>(tiles) + (size_t)(q * 32 + lane) * part_ld;
            for (int c = 0; c < bn; c += 32) {
                uint32_t v[32];
                ptx::tmem_ld32(tmem_base + c + ((uint32_t)(q * 32) << 16), v);
                ptx::tmem_ld_wait();
                if (q * 32 + lane < rows) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4*>(dst + c + 4 * j) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                }
            }
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (abort_s) __nanosleep(100000);  // let any copy still in flight land before shared memory is released
    cluster.sync();                    // every part of the tile is in place
    {
        const LinearEpilogue<O> ep(p.l);
        const int cols = bn / 4;
        for (int i = rank * kLtThreads + threadIdx.x; i < rows * cols; i += split * kLtThreads) {
            const int r = i / cols, c = i % cols * 4;
            if (n0 + c >= p.l.N) continue;
            const typename LinearEpilogue<O>::Extra extra = ep.fetch(row0 + r, n0 + c);
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < split; ++k) {
                const float4 v = *reinterpret_cast<const float4*>(cluster.map_shared_rank(reinterpret_cast<float*>(tiles), k) + (size_t)r * part_ld + c);
                s.x += v.x;
                s.y += v.y;
                s.z += v.z;
                s.w += v.w;
            }
            ep.finish(row0 + r, n0 + c, s, extra);
        }
    }
    grid_dep_launch();
    cluster.sync();  // no CTA leaves while its part may still be read
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem_base, tmem_cols);
    }
}

}  // namespace

LinearTilePlan linear_tile_plan(int64_t T, int N, int K, int sms) {
    LinearTilePlan q{};
    q.a_rows = (int)std::min<int64_t>(kTileM, (T + 15) / 16 * 16);
    const int nkb = (K + kLtBK - 1) / kLtBK;
    const int64_t mt = (T + kTileM - 1) / kTileM;
    q.bn = N <= 32 ? 32 : N <= 64 ? 64 : 128;
    const int64_t tiles = mt * ((N + q.bn - 1) / q.bn);
    q.split = 1;
    while (q.split < 8 && tiles * q.split * 2 <= 2 * sms && nkb >= 8 * q.split) q.split *= 2;
    const int stage_bytes = (q.a_rows + q.bn) * kLtBK * 2;
    const int per = (nkb + q.split - 1) / q.split;
    const int room = 104 * 1024;  // two CTAs per SM
    q.stages = std::max(2, std::min(std::min(kLtMaxStages, per), room / stage_bytes));
    // the ring, with what the last stage's 128 operand rows reach behind it; then the partial tile
    const size_t ring = (size_t)q.stages * stage_bytes + std::max(0, kTileM * kLtBK * 2 - stage_bytes);
    q.smem = std::max(ring, (size_t)q.a_rows * (q.bn + 4) * sizeof(float)) + 1024;
    // Never more than two CTAs per SM: their tensor memory then fits beside any other kernel's that shares the SM, and no CTA waits
    // for columns that a CTA of another cluster holds while that one waits for its own cluster's barrier
    q.smem = std::max(q.smem, (size_t)77 * 1024);
    return q;
}

cudaError_t launch_linear_tile(const LinearTileParams& p, bool out_bf16, cudaStream_t s) {
    const LinearTilePlan& q = p.plan;
    const int64_t grid = (p.l.T + kTileM - 1) / kTileM * ((p.l.N + q.bn - 1) / q.bn) * q.split;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    auto go = [&](auto kernel) {
        const cudaError_t e = ensure_smem(kernel, q.smem);
        return e != cudaSuccess ? e : launch_pdl_cluster(kernel, (unsigned)grid, kLtThreads, q.smem, q.split, s, p);
    };
    return out_bf16 ? go(linear_tile_kernel<__nv_bfloat16>) : go(linear_tile_kernel<float>);
}

}  // namespace exfold
