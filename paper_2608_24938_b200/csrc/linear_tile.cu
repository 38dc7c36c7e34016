// Dense product with epilogue, bf16 operands, few tokens or few tiles: one CTA per 128 tokens (or fewer, all tiles alike) x bn features,
// K split over a cluster.
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

constexpr int kLtEpiWarps = 8;  // two per quadrant of the accumulator's lanes
constexpr int kLtThreads = 64 + 32 * kLtEpiWarps;  // warp 0: TMA producer, warp 1: MMA issuer, the others: epilogue
constexpr int kLtMaxStages = 12;
constexpr int kLtBK = kGemmBK;

// WHOLE: every group of four outputs is whole and aligned
template <typename O, int SPLIT, bool WHOLE>
__global__ void __launch_bounds__(kLtThreads, 2) linear_tile_kernel(const __grid_constant__ LinearTileParams p) {
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
    constexpr int split = SPLIT;
    const int bn = p.plan.bn, stages = p.plan.stages, rank = (int)cluster.block_rank();
    const int nt = (p.l.N + bn - 1) / bn, tile = (int)blockIdx.x / split;
    const int n0 = tile % nt * bn;
    const int64_t row0 = (int64_t)(tile / nt) * p.plan.a_rows;
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
    const int rows = (int)min((int64_t)p.plan.a_rows, p.l.T - row0);
    const int part_ld = bn + 4;  // floats: 16-byte aligned rows, the rows of a quarter warp in distinct banks
    const LinearEpilogue<O> ep(p.l);
    LinearReduce<SPLIT, O, 32 * kLtEpiWarps, WHOLE> reduce(ep, rows, bn, row0, n0, rank, (int)threadIdx.x - 64);

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
        reduce.begin();  // bias and residual: on their way while the tile is multiplied
        // partial tile -> shared memory (the ring is free once every MMA has completed)
        const int q = warp & 3, half = (warp - 2) >> 2;
        int ok = 1;
        if (lane == 0) ok = ptx::mbar_wait_local(&done_bar, 0, abort_flag, p.l.status, 4) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (ok && q * 32 < rows) {
            ptx::tc_fence_after();
            float* dst = reinterpret_cast<float*>(tiles) + (size_t)(q * 32 + lane) * part_ld;
            for (int c = 32 * half; c < bn; c += 64) {
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
    if (warp >= 2) reduce.run(reinterpret_cast<const float*>(tiles), part_ld, 0, 1);
    grid_dep_launch();
    cluster.sync();  // no CTA leaves while its part may still be read
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem_base, tmem_cols);
    }
}

}  // namespace

// Row tiles alike, as few as 128 rows allow. 64 features per tile; where their tiles leave no room to split, 128 and a split take less
// operand traffic. K is split while two CTAs per SM have room for the parts (one alone takes in 73 KB per us, two 110) and a part has four
// k-blocks; in three where that leaves the SMs better balanced than two or four. On the GPU, with bias and residual, 64 features / 128 in
// two: 64 x 14336 x 4096 (tokens x features x K) 25.9 / 24.6 us, 128 x 14336 x 4096 31.7 / 28.4, 512 x 4096 x 4096 26.9 / 23.3; the other way
// 64 x 4096 x 4096 in 64 x 4 parts / 128 x 2 11.0 / 13.1, 256 x 4096 x 4096 16.9 / 20.1, 1024 x 2048 x 768 10.8 / 12.1.
LinearTilePlan linear_tile_plan(int64_t T, int N, int K, int sms) {
    LinearTilePlan q{};
    const int64_t mt = (T + kTileM - 1) / kTileM;
    q.a_rows = (int)(((T + mt - 1) / mt + 15) / 16 * 16);
    const int nkb = (K + kLtBK - 1) / kLtBK;
    q.bn = N <= 32 ? 32 : 64;
    int64_t tiles = mt * ((N + q.bn - 1) / q.bn);
    const int64_t wide = mt * ((N + 127) / 128);
    if (tiles > sms && wide <= sms && nkb >= 16) {
        q.bn = 128;
        tiles = wide;
    }
    // k-blocks that the SM with the most of them gets
    auto most = [&](int split) { return (tiles * split + sms - 1) / sms * ((nkb + split - 1) / split); };
    q.split = 1;
    while (q.split < 8 && tiles * q.split <= sms && nkb >= 8 * q.split) q.split *= 2;
    if ((q.split == 2 || q.split == 4) && tiles * 3 <= 2 * sms && nkb >= 12 && most(3) < most(q.split)) q.split = 3;
    const int stage_bytes = (q.a_rows + q.bn) * kLtBK * 2;
    const int per = (nkb + q.split - 1) / q.split;
    q.stages = std::max(2, std::min(std::min(kLtMaxStages, per), 104 * 1024 / stage_bytes));
    // the ring, with what the last stage's 128 operand rows reach behind it; then the partial tile
    const size_t ring = (size_t)q.stages * stage_bytes + std::max(0, kTileM * kLtBK * 2 - stage_bytes);
    q.smem = std::max(ring, (size_t)q.a_rows * (q.bn + 4) * sizeof(float)) + 1024;
    // Never more than two CTAs per SM: their tensor memory then fits beside any other kernel's that shares the SM, and no CTA waits
    // for columns that a CTA of another cluster holds while that one waits for its own cluster's barrier
    q.smem = std::max(q.smem, (size_t)77 * 1024);
    return q;
}

// Whether the tiles of 256 x 256 on CTA pairs (linear_pair.cu) are the faster ones. Those take a third less operand traffic, but whole
// rounds of items and a longer way in and out: about 0.31 us per k-block of a round and 9 us; the tiles here what they load at
// 18 TB/s and 6 us. Measured, pairs / tiles: 512 x 4096 x 4096 27.9 / 22.9 us, 1024 x 4096 x 4096 30.1 / 49.1, 300 x 14336 x 4096
// 48.7 / 77.6, 1024 x 2048 x 768 12.7 / 10.6, 2048 x 768 x 2048 18.0 / 16.3.
bool linear_prefers_pairs(int64_t T, int N, int K, int sms) {
    const int64_t nkb = (K + kLtBK - 1) / kLtBK;
    const int64_t items = (T + 255) / 256 * ((N + 255) / 256), pairs = std::max(1, sms / 2), rounds = (items + pairs - 1) / pairs;
    const LinearTilePlan q = linear_tile_plan(T, N, K, sms);
    const double tiles = (double)((T + kTileM - 1) / kTileM) * (double)((N + q.bn - 1) / q.bn);
    const double t_tile = tiles * (double)nkb * (q.a_rows + q.bn) * (kLtBK * 2) / 18e6 + 6.0;
    return 0.31 * (double)(rounds * nkb) + 9.0 < t_tile;
}

cudaError_t launch_linear_tile(const LinearTileParams& p, bool out_bf16, cudaStream_t s) {
    const LinearTilePlan& q = p.plan;
    const int64_t grid = (p.l.T + q.a_rows - 1) / q.a_rows * ((p.l.N + q.bn - 1) / q.bn) * q.split;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    auto go = [&](auto kernel) {
        const cudaError_t e = ensure_smem(kernel, q.smem);
        return e != cudaSuccess ? e : launch_pdl_cluster(kernel, (unsigned)grid, kLtThreads, q.smem, q.split, s, p);
    };
    auto pick = [&](auto one, auto two, auto three, auto four, auto eight) {
        return q.split == 1 ? go(one) : q.split == 2 ? go(two) : q.split == 3 ? go(three) : q.split == 4 ? go(four) : go(eight);
    };
    const bool whole = out_bf16 ? LinearEpilogue<__nv_bfloat16>(p.l).whole() : LinearEpilogue<float>(p.l).whole();
#define EXFOLD_LT(O, W) \
    pick(linear_tile_kernel<O, 1, W>, linear_tile_kernel<O, 2, W>, linear_tile_kernel<O, 3, W>, linear_tile_kernel<O, 4, W>, linear_tile_kernel<O, 8, W>)
    if (out_bf16) return whole ? EXFOLD_LT(__nv_bfloat16, true) : EXFOLD_LT(__nv_bfloat16, false);
    return whole ? EXFOLD_LT(float, true) : EXFOLD_LT(float, false);
#undef EXFOLD_LT
}

}  // namespace exfold
