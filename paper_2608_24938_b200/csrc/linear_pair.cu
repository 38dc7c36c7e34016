// Dense product with epilogue, bf16 operands, many tokens: CTA pairs (tcgen05 cta_group::2), 256 tokens x 256 features per pair.
//
// A pair's k-block (K = 64) needs 32 KB per SM for 512 cycles of the tensor pipe, what an SM takes in from L2; a single CTA's
// 128 x 256 tile needs 48 KB for the same. Six stages of 32 KB are in flight, two 256-column accumulators hand a finished tile to the
// epilogue warps while the next one is multiplied. Roles per CTA: warps 0 and 1 TMA producers (k-blocks dealt in turn; own token
// rows, own half of the weight rows, both CTAs' bytes counted on the leader's barrier), warp 2 MMA issuer (leader), the other eight
// epilogue: two per quadrant of the accumulator's lanes, half of the columns each.
//
// An epilogue warp works on 32 rows x 128 bytes of y at a time: the residual comes into its buffer by TMA, each lane adds its row of
// the accumulator in place, and the buffer leaves by TMA, which also clips what lies past T, and past N in whole 16-byte pieces: where
// rows end inside one, their last columns leave by plain stores. Where y or the residual is not aligned for TMA, rows go through the
// buffer and plain loads and stores.
#include <algorithm>

#include "common.cuh"
#include "linear_epilogue.cuh"
#include "ptx.cuh"

namespace exfold {

namespace {

constexpr int kLpBK = kGemmBK;
constexpr int kLpStages = 6;
constexpr int kLpTileBytes = kTileM * kLpBK * 2;  // 16 KB: this CTA's token rows, or its half of the weight rows
constexpr int kLpStageBytes = 2 * kLpTileBytes;
constexpr int kLpEpiWarps = 8;
constexpr int kLpOutBytes = 32 * 128;             // per epilogue warp: 32 rows x 128 bytes
constexpr int kLpSmem = kLpStages * kLpStageBytes + kLpEpiWarps * kLpOutBytes + 1024;
constexpr int kLpThreads = 32 * (3 + kLpEpiWarps);
constexpr int kLpTmemCols = 512;

// Work order: bands of row tiles; within a band the feature tiles, each against all row tiles of the band
__device__ __forceinline__ void decode_tile(const LinearPairParams& p, int w, int* m, int* n) {
    const int per = p.band * p.nt, b = w / per, left = w - b * per;
    const int rows = min(p.band, p.mt - b * p.band);
    *n = left / rows;
    *m = b * p.band + left - *n * rows;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&v);
}

// 32 accumulator columns from `col` on: bias and activation. FULL: all 32 exist and the bias is aligned to 16 bytes.
template <int ACT, bool FULL>
__device__ __forceinline__ void bias_act(float (&f)[32], const uint32_t (&v)[32], const LinearParams& l, int col) {
    const __nv_bfloat16* bias = reinterpret_cast<const __nv_bfloat16*>(l.bias) + col;
    if (l.bias == nullptr) {
#pragma unroll
        for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]);
    } else if (FULL) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // every lane the same address
            const uint4 b = __ldg(reinterpret_cast<const uint4*>(bias) + j);
            const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&b);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float2 t = __bfloat1622float2(h[u]);
                f[8 * j + 2 * u] = __uint_as_float(v[8 * j + 2 * u]) + t.x;
                f[8 * j + 2 * u + 1] = __uint_as_float(v[8 * j + 2 * u + 1]) + t.y;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]) + (col + j < l.N ? __bfloat162float(bias[j]) : 0.f);
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) f[j] = linear_act(f[j], ACT);
}
template <bool FULL>
__device__ __forceinline__ void bias_act(float (&f)[32], const uint32_t (&v)[32], const LinearParams& l, int col) {
    switch (l.act) {
        case EXFOLD_ACT_RELU: return bias_act<EXFOLD_ACT_RELU, FULL>(f, v, l, col);
        case EXFOLD_ACT_GELU: return bias_act<EXFOLD_ACT_GELU, FULL>(f, v, l, col);
        case EXFOLD_ACT_GELU_TANH: return bias_act<EXFOLD_ACT_GELU_TANH, FULL>(f, v, l, col);
        case EXFOLD_ACT_SILU: return bias_act<EXFOLD_ACT_SILU, FULL>(f, v, l, col);
        default: return bias_act<EXFOLD_ACT_NONE, FULL>(f, v, l, col);
    }
}

// 32 columns (the h-th of the warp's buffer) of this lane's row, onto the residual that lies there or in place of nothing. 16-byte
// chunk c of a row lies at c ^ (row & 7), the tensor maps' swizzle.
template <typename O>
__device__ __forceinline__ void put_cols(unsigned char* buf, int lane, int h, const float (&f)[32], bool has_res) {
    constexpr int kPieces = 32 * (int)sizeof(O) / 16;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        uint4* at = reinterpret_cast<uint4*>(buf + lane * 128 + (((h * kPieces + j) ^ (lane & 7)) << 4));
        uint4 o = has_res ? *at : make_uint4(0u, 0u, 0u, 0u);
        if constexpr (sizeof(O) == 2) {
            const __nv_bfloat162* r = reinterpret_cast<const __nv_bfloat162*>(&o);
            float g[8];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float2 t = __bfloat1622float2(r[u]);
                g[2 * u] = has_res ? f[8 * j + 2 * u] + t.x : f[8 * j + 2 * u];
                g[2 * u + 1] = has_res ? f[8 * j + 2 * u + 1] + t.y : f[8 * j + 2 * u + 1];
            }
            o = make_uint4(pack2(g[0], g[1]), pack2(g[2], g[3]), pack2(g[4], g[5]), pack2(g[6], g[7]));
        } else {
            float* g = reinterpret_cast<float*>(&o);
#pragma unroll
            for (int u = 0; u < 4; ++u) g[u] = has_res ? f[4 * j + u] + g[u] : f[4 * j + u];
        }
        *at = o;
    }
}
// The warp's 32 rows x 32 sums to memory, for y or a residual that no tensor map takes: through the buffer, so that a row's 32
// columns are loaded and stored at once. add: the residual, lane = column, all rows asked for together and ahead (in batches of eight rows,
// each behind the stores of the one before, 777 x 1411 x 2040 took 49 us)
template <typename O>
__device__ __forceinline__ void fetch_rows(const LinearParams& l, O (&add)[32], int64_t row0, int rows, int col) {
    const O* r = reinterpret_cast<const O*>(l.residual) + row0 * l.ldr + col;
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < rows && col < l.N) add[i] = r[i * l.ldr];
}
template <typename O>
__device__ __forceinline__ void store_rows(const LinearParams& l, unsigned char* buf, int lane, const float (&f)[32], const O (&add)[32],
                                           int64_t row0, int rows, int col) {
    put_cols<float>(buf, lane, 0, f, false);
    __syncwarp();
    O* y = reinterpret_cast<O*>(l.y) + row0 * l.ldy + col + lane;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const float v = *reinterpret_cast<const float*>(buf + i * 128 + (((lane >> 2) ^ (i & 7)) << 4) + (lane & 3) * 4);
        if (i < rows && col + lane < l.N) linear_store(y + i * l.ldy, l.residual != nullptr ? v + linear_f32(add[i]) : v);
    }
    __syncwarp();
}

// The columns from `col` to N of the warp's rows, from where put_cols left them. For rows that end inside a 16-byte piece: a tiled store
// writes all of that piece, and so the caller's next elements where rows lie apart (zeros, seen with 4099 fp32 columns in rows of 4112).
template <typename O>
__device__ __forceinline__ void store_last_cols(const LinearParams& l, const unsigned char* buf, int lane, int64_t row0, int rows, int col) {
    O* y = reinterpret_cast<O*>(l.y) + row0 * l.ldy + col;
    for (int c = lane; c < min(128 / (int)sizeof(O), l.N - col); c += 32) {
        const int at = c * (int)sizeof(O);
#pragma unroll 4
        for (int i = 0; i < rows; ++i) y[i * l.ldy + c] = *reinterpret_cast<const O*>(buf + i * 128 + (((at >> 4) ^ (i & 7)) << 4) + (at & 15));
    }
}

// TMA: y and the residual go by tensor maps
template <typename O, bool TMA>
__global__ void __launch_bounds__(kLpThreads, 1) linear_pair_kernel(const __grid_constant__ LinearPairParams p) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kLpStages];   // used in the leader
    __shared__ __align__(8) uint64_t empty_bar[kLpStages];  // one per CTA, released by the leader's commits
    __shared__ __align__(8) uint64_t tfull_bar[2];          // one per CTA
    __shared__ __align__(8) uint64_t tempty_bar[2];         // used in the leader: the epilogue warps of both CTAs
    __shared__ __align__(8) uint64_t res_bar[kLpEpiWarps];  // an epilogue warp's residual
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s;
    unsigned char* tiles =
        reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
    const int rank = (int)ptx::cluster_ctarank();  // 0 = leader
    if (threadIdx.x == 0) {
        ptx::prefetch_tmap(&p.tm_x);
        ptx::prefetch_tmap(&p.tm_w);
        for (int s = 0; s < kLpStages; ++s) {
            ptx::mbar_init(&full_bar[s], 1);
            ptx::mbar_init(&empty_bar[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(&tfull_bar[s], 1);
            ptx::mbar_init(&tempty_bar[s], 2 * kLpEpiWarps);
        }
        for (int s = 0; s < kLpEpiWarps; ++s) ptx::mbar_init(&res_bar[s], 1);
        if (TMA) ptx::prefetch_tmap(&p.tm_y);
        if (TMA && p.l.residual != nullptr) ptx::prefetch_tmap(&p.tm_r);
        abort_s = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 2) {
        ptx::tmem_alloc_pair(&tmem_base_s, kLpTmemCols);
        ptx::tmem_relinquish_pair();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_sync_all();  // both CTAs' barriers are initialised and their tensor memory allocated
    ptx::tc_fence_after();
    grid_dep_wait();
    if (blockIdx.x == 0 && threadIdx.x < 4) reinterpret_cast<int*>(p.l.status)[threadIdx.x] = 0;
    const uint32_t tmem_base = tmem_base_s;
    volatile int* abort_flag = &abort_s;
    const int nkb = (p.l.K + kLpBK - 1) / kLpBK, total = p.mt * p.nt;
    const int w_begin = (int)blockIdx.x >> 1, w_stride = (int)gridDim.x >> 1;

    if (warp < 2) {
        // ------------------------------------------------ TMA producers (both CTAs; k-block c belongs to producer c % 2)
        if (ptx::elect_one()) {
            int stage = 0, phase = 0, turn = 0;
            bool ok = true;
            for (int w = w_begin; w < total && ok; w += w_stride) {
                int m, n;
                decode_tile(p, w, &m, &n);
                const int arow = m * 256 + rank * kTileM, brow = n * 256 + rank * 128;
                for (int kb = 0; kb < nkb; ++kb) {
                    if (turn == warp) {
                        if (!ptx::mbar_wait_local(&empty_bar[stage], phase ^ 1, abort_flag, p.l.status, 1)) {
                            ok = false;
                            break;
                        }
                        unsigned char* dst = tiles + stage * kLpStageBytes;
                        if (rank == 0) ptx::mbar_expect_tx(&full_bar[stage], 2 * kLpStageBytes);  // both CTAs' bytes
                        ptx::tma_load_2d_pair(dst, &p.tm_x, &full_bar[stage], kb * kLpBK, arow);
                        ptx::tma_load_2d_pair(dst + kLpTileBytes, &p.tm_w, &full_bar[stage], kb * kLpBK, brow);
                    }
                    turn ^= 1;
                    if (++stage == kLpStages) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 2) {
        // ------------------------------------------------ MMA issuer (leader CTA only)
        if (rank == 0 && ptx::elect_one()) {
            constexpr uint32_t idesc = ptx::make_idesc_bf16(256, 256);
            const uint32_t lo0 = (ptx::smem_u32(tiles) & 0x3FFFFu) >> 4;
            constexpr uint32_t lo_step = (uint32_t)kLpStageBytes >> 4, lo_b = (uint32_t)kLpTileBytes >> 4;
            const uint32_t desc_hi = (uint32_t)(ptx::make_kmajor_sw128_desc(0) >> 32);
            int stage = 0, phase = 0, iter = 0;
            bool ok = true, ready = false;
            static_assert(kLpStages == 6, "the k-loop below is written out for six ring stages");
            for (int w = w_begin; w < total && ok; w += w_stride, ++iter) {
                const int as = iter & 1, aphase = (iter >> 1) & 1;
                if (!ptx::mbar_wait_local(&tempty_bar[as], aphase ^ 1, abort_flag, p.l.status, 2)) break;
                ptx::tc_fence_after();
                const uint32_t d_tmem = tmem_base + as * 256;
                // written out once per ring stage: with the stage a compile-time constant a k-block costs this thread the MMA
                // sequence, one compare and one branch
                int kb = 0;
#define EXFOLD_LP_KBLOCK(S)                                                                                        \
    {                                                                                                               \
        constexpr int NS = (S) + 1 == kLpStages ? 0 : (S) + 1;                                                      \
        const uint32_t nphase = NS == 0 ? phase ^ 1 : phase;                                                        \
        if (!ready && !ptx::mbar_wait_local(&full_bar[S], phase, abort_flag, p.l.status, 3)) {                      \
            ok = false;                                                                                             \
            break;                                                                                                  \
        }                                                                                                           \
        ready = ptx::umma_kblock_bf16_pair(d_tmem, lo0 + (S) * lo_step, lo0 + (S) * lo_step + lo_b, desc_hi, idesc, \
                                           kb > 0 ? 1u : 0u, &empty_bar[S], &full_bar[NS], nphase);                 \
        if (NS == 0) phase ^= 1;                                                                                    \
        if (++kb == nkb) {                                                                                          \
            stage = NS;                                                                                             \
            break;                                                                                                  \
        }                                                                                                           \
    }
                while (ok && kb < nkb) {
                    switch (stage) {
                        case 0: EXFOLD_LP_KBLOCK(0)
                        case 1: EXFOLD_LP_KBLOCK(1)
                        case 2: EXFOLD_LP_KBLOCK(2)
                        case 3: EXFOLD_LP_KBLOCK(3)
                        case 4: EXFOLD_LP_KBLOCK(4)
                        default: EXFOLD_LP_KBLOCK(5)
                    }
                    if (kb < nkb) stage = 0;  // fell through the last stage: the ring wraps
                }
#undef EXFOLD_LP_KBLOCK
                if (ok) ptx::umma_commit_pair(&tfull_bar[as], 3);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ epilogue warps (own rows; TMEM lane quadrant = warp % 4)
        const int q = warp & 3, half = (warp - 3) >> 2;
        unsigned char* buf = tiles + kLpStages * kLpStageBytes + (warp - 3) * kLpOutBytes;
        uint64_t* rbar = &res_bar[warp - 3];
        const bool has_res = p.l.residual != nullptr, full_bias = (reinterpret_cast<uintptr_t>(p.l.bias) & 15) == 0;
        constexpr int kCols = 128 / (int)sizeof(O);  // of y per trip
        uint32_t rphase = 0;
        int iter = 0;
        for (int w = w_begin; w < total; w += w_stride, ++iter) {
            const int as = iter & 1, aphase = (iter >> 1) & 1;
            int m, n;
            decode_tile(p, w, &m, &n);
            const int64_t row0 = (int64_t)m * 256 + rank * kTileM + q * 32;
            const int rows = (int)max((int64_t)0, min((int64_t)32, p.l.T - row0));
            const int col0 = n * 256 + half * 128;
            int ok = 1;
            const bool some = rows > 0 && col0 < p.l.N;
            if (TMA && some && has_res && lane == 0) {  // on its way while the tile is multiplied
                ptx::tma_store_wait_read();
                ptx::mbar_expect_tx(rbar, kLpOutBytes);
                ptx::tma_load_2d(buf, &p.tm_r, rbar, col0, (int)row0);
            }
            O add[TMA ? 1 : 32];
            if constexpr (!TMA)
                if (some && has_res) fetch_rows<O>(p.l, add, row0, rows, col0 + lane);
            if (lane == 0) ok = ptx::mbar_wait_local(&tfull_bar[as], aphase, abort_flag, p.l.status, 4) ? 1 : 0;
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            ptx::tc_fence_after();
            const uint32_t taddr = tmem_base + as * 256 + half * 128 + ((uint32_t)(q * 32) << 16);
            if (TMA && some) {
#pragma unroll 1
                for (int cc = 0; cc < 128 && col0 + cc < p.l.N; cc += kCols) {
                    if (has_res) {  // every lane sees the copy's end itself, and with it the bytes
                        ok = ptx::mbar_wait_local(rbar, rphase, abort_flag, p.l.status, 5) ? 1 : 0;
                        rphase ^= 1;
                        ok = __all_sync(0xffffffffu, ok);
                    } else {
                        if (lane == 0) ptx::tma_store_wait_read();  // the buffer is free
                        __syncwarp();
                    }
                    if (!ok) break;
#pragma unroll
                    for (int h = 0; h < kCols / 32; ++h) {
                        const int col = col0 + cc + 32 * h;
                        uint32_t v[32];
                        float f[32];
                        ptx::tmem_ld32(taddr + cc + 32 * h, v);
                        ptx::tmem_ld_wait();
                        if (full_bias && col + 32 <= p.l.N) bias_act<true>(f, v, p.l, col);
                        else bias_act<false>(f, v, p.l, col);
                        put_cols<O>(buf, lane, h, f, has_res);
                    }
                    const bool last_cols = col0 + cc + kCols > p.l.N && p.l.N % (16 / (int)sizeof(O)) != 0;
                    if (last_cols) {
                        __syncwarp();
                        store_last_cols<O>(p.l, buf, lane, row0, rows, col0 + cc);
                    }
                    ptx::store_fence();  // what was written to the buffer before the store, what was read before the next residual
                    __syncwarp();
                    if (lane == 0 && !last_cols) {
                        ptx::tma_store_2d(&p.tm_y, buf, col0 + cc, (int)row0);
                        if (has_res && cc + kCols < 128 && col0 + cc + kCols < p.l.N) {  // the next columns' residual
                            ptx::tma_store_wait_read();
                            ptx::mbar_expect_tx(rbar, kLpOutBytes);
                            ptx::tma_load_2d(buf, &p.tm_r, rbar, col0 + cc + kCols, (int)row0);
                        }
                    }
                }
                if (!ok) break;
            }
            if constexpr (!TMA) {
                if (some) {
#pragma unroll 1
                    for (int col = col0; col < min(col0 + 128, p.l.N); col += 32) {
                        uint32_t v[32];
                        float f[32];
                        ptx::tmem_ld32(taddr + col - col0, v);
                        ptx::tmem_ld_wait();
                        if (full_bias && col + 32 <= p.l.N) bias_act<true>(f, v, p.l, col);
                        else bias_act<false>(f, v, p.l, col);
                        store_rows<O>(p.l, buf, lane, f, add, row0, rows, col);
                        if (has_res && col + 32 < col0 + 128) fetch_rows<O>(p.l, add, row0, rows, col + 32 + lane);
                    }
                }
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_leader(&tempty_bar[as]);
        }
        if (TMA && lane == 0) ptx::tma_store_wait();
    }

    // ------------------------------------------------ teardown
    if (threadIdx.x == 96) grid_dep_launch();  // after the epilogue loop
    ptx::tc_fence_before();
    __syncthreads();
    if (abort_s) __nanosleep(100000);  // let any copy still in flight land before shared memory is released
    ptx::cluster_sync_all();           // the peer is done with this CTA's shared and tensor memory
    if (warp == 2) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc_pair(tmem_base, kLpTmemCols);
    }
}

}  // namespace

cudaError_t launch_linear_pair(LinearPairParams p, bool out_bf16, int sms, cudaStream_t s) {
    p.mt = (int)((p.l.T + 255) / 256);
    p.nt = (p.l.N + 255) / 256;
    // Bands of 16 MB of token rows, which stay in L2 while the weights pass by (and the pairs that run together share few of both). In
    // long loops, at the power limit, 8 / 16 / 32 / 48 / 64 MB and one band: 8192 x 4096 x 4096 202 / 215 / 213 / 220 / 231 / 238 us, 16384 x
    // 4096 x 4096 437 / 430 / 434 / 455 / 506 / 554, 8192 x 14336 x 4096 802 / 749 / 760 / 797 / 849 / 846.
    p.band = (int)std::max<int64_t>(1, std::min<int64_t>(p.mt, (16 << 20) / ((int64_t)p.l.K * 512)));
    const int bands = (p.mt + p.band - 1) / p.band;
    p.band = (p.mt + bands - 1) / bands;
    if ((int64_t)p.mt * p.nt > 0x3fffffff) return cudaErrorInvalidValue;
    const int total = p.mt * p.nt, pairs = std::max(1, sms / 2), rounds = (total + pairs - 1) / pairs;
    const int grid = 2 * ((total + rounds - 1) / rounds);  // the pairs that take work finish together
    auto go = [&](auto kernel) {
        const cudaError_t e = ensure_smem(kernel, kLpSmem);
        return e != cudaSuccess ? e : launch_pdl_cluster(kernel, grid, kLpThreads, kLpSmem, 2, s, p);
    };
    if (out_bf16) return p.tma_io ? go(linear_pair_kernel<__nv_bfloat16, true>) : go(linear_pair_kernel<__nv_bfloat16, false>);
    return p.tma_io ? go(linear_pair_kernel<float, true>) : go(linear_pair_kernel<float, false>);
}

}  // namespace exfold
