// Dense product with bias, activation and residual in its epilogue, y = act(x W^T + b) + r, on the CUDA cores: fp32 operands, which
// tensor cores would round, and bf16 ones that no tensor map takes.
//
//   few tokens   A warp takes 8 features x 8 tokens, its lanes along K: 16 loads of 16 bytes per lane feed 256 multiply-adds, straight
//       from global memory (the weights of a token group after the first come from L2). The warps of a CTA split K; the 64 sums of a warp
//       are reduced over the lanes by halving exchanges (62 shuffles) and meet in shared memory, in order.
//   tiles        64 x 64 outputs per CTA of 128 threads, 8 x 4 of them per thread; K in steps of 16 through two shared-memory stages,
//       the next step's loads in registers meanwhile. Rows lie along K with a pitch of 20 floats: what a quarter warp reads in 16-byte
//       pieces hits distinct banks. K is split over a cluster (LinearReduce) until four CTAs share an SM.
//   large tiles  128 x 128 outputs per CTA of 256 threads, 8 x 8 per thread, stages transposed, two multiply-adds per instruction
//       (fma.rn.f32x2; with single ones both kernels stop at 32 TFLOP/s, half of what the packed form can do).
#include <algorithm>

#include "common.cuh"
#include "linear_epilogue.cuh"

namespace exfold {

namespace {

// Four elements at p, of which the first `left` exist; the rest are zeros. VEC: aligned to four
template <bool VEC, typename T>
__device__ __forceinline__ float4 load4(const T* p, int left) {
    if (VEC && left >= 4) return linear_load4(p);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (left > 0) v.x = linear_f32(p[0]);
    if (left > 1) v.y = linear_f32(p[1]);
    if (left > 2) v.z = linear_f32(p[2]);
    if (left > 3) v.w = linear_f32(p[3]);
    return v;
}

// c += a b, both halves: one instruction
__device__ __forceinline__ void fma2(float2& c, const float2& a, const float2& b) {
    asm("fma.rn.f32x2 %0, %1, %2, %0;"
        : "+l"(reinterpret_cast<unsigned long long&>(c))
        : "l"(reinterpret_cast<const unsigned long long&>(a)), "l"(reinterpret_cast<const unsigned long long&>(b)));
}

// ---------------------------------------------------------------- few tokens
constexpr int kLfWarps = 8, kLfTile = 8;  // features, and tokens, of a CTA

// Sum over the lanes of each of 64 values; lane l ends up with those of values l and l + 32 in v[0] and v[32]
__device__ __forceinline__ void halve64(float (&v)[64], int lane) {
#pragma unroll
    for (int half = 0; half < 64; half += 32)
#pragma unroll
        for (int n = 16; n > 0; n >>= 1) {
            const bool up = (lane & n) != 0;
#pragma unroll
            for (int j = 0; j < n; ++j) {
                const float give = up ? v[half + j] : v[half + j + n], keep = up ? v[half + j + n] : v[half + j];
                v[half + j] = keep + __shfl_xor_sync(0xffffffffu, give, n);
            }
        }
}

template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(32 * kLfWarps) linear_few_kernel(LinearParams p) {
    __shared__ float s_sum[kLfWarps][64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
    const int fblocks = (p.N + kLfTile - 1) / kLfTile;
    const int n0 = (int)(blockIdx.x % fblocks) * kLfTile;
    const int64_t m0 = (int64_t)(blockIdx.x / fblocks) * kLfTile;
    const T* x = reinterpret_cast<const T*>(p.x) + lane * 4;
    const T* w = reinterpret_cast<const T*>(p.w) + lane * 4;
    grid_dep_launch();
    grid_dep_wait();
    if (blockIdx.x == 0 && threadIdx.x < 4) reinterpret_cast<int*>(p.status)[threadIdx.x] = 0;
    // thread t < 64 ends up with token t / 8, feature t % 8
    const int col = n0 + (int)(threadIdx.x & 7);
    const int64_t tok = m0 + (threadIdx.x >> 3);
    const bool ends = threadIdx.x < 64 && col < p.N && tok < p.T;
    T bias{};
    O residual{};
    float acc[64];  // [feature][token]: value 8 f + t
#pragma unroll
    for (int i = 0; i < 64; ++i) acc[i] = 0.f;
    for (int k0 = warp * 128; k0 < p.K; k0 += warps * 128) {
        const int left = p.K - k0 - lane * 4;
        float4 a[8], b[8];
#pragma unroll
        for (int f = 0; f < 8; ++f) a[f] = load4<VEC>(w + min(n0 + f, p.N - 1) * p.ldw + k0, left);
#pragma unroll
        for (int t = 0; t < 8; ++t) b[t] = load4<VEC>(x + min(m0 + t, p.T - 1) * p.ldx + k0, left);
#pragma unroll
        for (int f = 0; f < 8; ++f)
#pragma unroll
            for (int t = 0; t < 8; ++t)
                acc[8 * f + t] += fmaf(a[f].w, b[t].w, fmaf(a[f].z, b[t].z, fmaf(a[f].y, b[t].y, a[f].x * b[t].x)));
    }
    if (ends) {
        if (p.bias != nullptr) bias = reinterpret_cast<const T*>(p.bias)[col];
        if (p.residual != nullptr) residual = reinterpret_cast<const O*>(p.residual)[tok * p.ldr + col];
    }
    halve64(acc, lane);
    s_sum[warp][lane] = acc[0];
    s_sum[warp][lane + 32] = acc[32];
    __syncthreads();
    for (int i = threadIdx.x; i < 64; i += blockDim.x) {  // one pass with two warps or more
        const int n = n0 + (i & 7);
        const int64_t m = m0 + (i >> 3);
        if (n >= p.N || m >= p.T) continue;
        const int at = (i & 7) * 8 + (i >> 3);
        float v = s_sum[0][at];
        for (int q = 1; q < warps; ++q) v += s_sum[q][at];
        if (i != (int)threadIdx.x) {
            if (p.bias != nullptr) bias = reinterpret_cast<const T*>(p.bias)[n];
            if (p.residual != nullptr) residual = reinterpret_cast<const O*>(p.residual)[m * p.ldr + n];
        }
        if (p.bias != nullptr) v += linear_f32(bias);
        v = linear_act(v, p.act);
        if (p.residual != nullptr) v += linear_f32(residual);
        linear_store(reinterpret_cast<O*>(p.y) + m * p.ldy + n, v);
    }
}

// ---------------------------------------------------------------- tiles
constexpr int kLsThreads = 128;
constexpr int kLsBM = 64, kLsBN = 64, kLsBK = 16, kLsPitch = kLsBK + 4;

template <typename T, typename O, bool VEC, int SPLIT>
__global__ void __launch_bounds__(kLsThreads) linear_simt_kernel(LinearParams p) {
    constexpr int BM = kLsBM, TX = 16, TY = kLsThreads / TX, TM = BM / TY, TN = kLsBN / TX;
    constexpr int kLoadsA = BM * kLsBK / 4 / kLsThreads, kLoadsB = kLsBN * kLsBK / 4 / kLsThreads;  // of four elements
    constexpr int kStage = (BM + kLsBN) * kLsPitch, kPart = kLsBN + 1;
    // two stages of both operands; then the partial tile
    __shared__ __align__(16) float smem[2 * kStage > BM * kPart ? 2 * kStage : BM * kPart];
    const T* x = reinterpret_cast<const T*>(p.x);
    const T* w = reinterpret_cast<const T*>(p.w);
    const int tid = threadIdx.x, tx = tid % TX, ty = tid / TX;
    const int n_tiles = (p.N + kLsBN - 1) / kLsBN;
    const int rank = (int)blockIdx.x % SPLIT, tile = (int)blockIdx.x / SPLIT;
    const int64_t m0 = (int64_t)(tile / n_tiles) * BM;
    const int n0 = tile % n_tiles * kLsBN;
    const int steps = (p.K + kLsBK - 1) / kLsBK, s0 = (int)((int64_t)rank * steps / SPLIT), s1 = (int)((int64_t)(rank + 1) * steps / SPLIT);
    grid_dep_launch();
    grid_dep_wait();
    if (blockIdx.x == 0 && tid < 4) reinterpret_cast<int*>(p.status)[tid] = 0;
    const LinearEpilogue<O> ep(p);
    LinearReduce<SPLIT, O, kLsThreads, false, T> reduce(ep, (int)min((int64_t)BM, p.T - m0), kLsBN, m0, n0, rank, tid);
    // thread t loads rows t / 4 + 32 u, four elements at 4 (t % 4)
    const int lrow = tid >> 2, lk = (tid & 3) * 4;
    const T* px[kLoadsA];
    const T* pw[kLoadsB];
#pragma unroll
    for (int u = 0; u < kLoadsA; ++u) px[u] = x + min(m0 + lrow + 32 * u, p.T - 1) * p.ldx + lk;
#pragma unroll
    for (int u = 0; u < kLoadsB; ++u) pw[u] = w + (int64_t)min(n0 + lrow + 32 * u, p.N - 1) * p.ldw + lk;
    float4 ra[kLoadsA], rb[kLoadsB];
    auto load = [&](int s) {
        const int left = p.K - s * kLsBK - lk;
#pragma unroll
        for (int u = 0; u < kLoadsA; ++u) ra[u] = load4<VEC>(px[u] + (int64_t)s * kLsBK, left);
#pragma unroll
        for (int u = 0; u < kLoadsB; ++u) rb[u] = load4<VEC>(pw[u] + (int64_t)s * kLsBK, left);
    };
    auto store = [&](int buf) {
        float* dst = smem + buf * kStage + lrow * kLsPitch + lk;
#pragma unroll
        for (int u = 0; u < kLoadsA; ++u) *reinterpret_cast<float4*>(dst + 32 * u * kLsPitch) = ra[u];
#pragma unroll
        for (int u = 0; u < kLoadsB; ++u) *reinterpret_cast<float4*>(dst + (BM + 32 * u) * kLsPitch) = rb[u];
    };
    // outputs of this thread: rows ty + TY i, columns tx + TX j
    float acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = 0.f;
    load(s0);
    store(0);
    __syncthreads();
    int buf = 0;
    for (int s = s0; s < s1; ++s, buf ^= 1) {
        if (s + 1 < s1) load(s + 1);
        const float* sa = smem + buf * kStage + ty * kLsPitch;
        const float* sb = smem + buf * kStage + (BM + tx) * kLsPitch;
#pragma unroll
        for (int k = 0; k < kLsBK; k += 4) {
            float4 b[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) b[j] = *reinterpret_cast<const float4*>(sb + TX * j * kLsPitch + k);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const float4 a = *reinterpret_cast<const float4*>(sa + TY * i * kLsPitch + k);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = fmaf(a.x, b[j].x, acc[i][j]);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = fmaf(a.y, b[j].y, acc[i][j]);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = fmaf(a.z, b[j].z, acc[i][j]);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = fmaf(a.w, b[j].w, acc[i][j]);
            }
        }
        if (s + 1 < s1) store(buf ^ 1);
        __syncthreads();
    }
    reduce.begin();
    float* part = smem;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) part[(ty + TY * i) * kPart + tx + TX * j] = acc[i][j];
    if (SPLIT > 1) cooperative_groups::this_cluster().sync();
    else __syncthreads();
    reduce.run(part, kPart, 0, 1);
    if (SPLIT > 1) cooperative_groups::this_cluster().sync();  // no CTA leaves while its part may still be read
}

// ---------------------------------------------------------------- large tiles
// 128 x 128 outputs per CTA of 256 threads, 8 x 8 of them per thread. Stages lie transposed (a k's rows next to each other), so that a
// thread reads the 16 operands of a k in four 16-byte pieces and holds no more of them than that: 64 bytes for 64 multiply-adds, the rate at
// which shared memory returns them.
constexpr int kLbThreads = 256, kLbTile = 128, kLbPitch = kLbTile + 4;

template <typename T, typename O, bool VEC, int SPLIT>
__global__ void __launch_bounds__(kLbThreads, 1) linear_simt_big_kernel(LinearParams p) {
    constexpr int kPart = kLbTile + 1, kStage = 2 * kLsBK * kLbPitch;
    extern __shared__ __align__(16) float smem[];  // two stages of both operands; then the partial tile
    const T* x = reinterpret_cast<const T*>(p.x);
    const T* w = reinterpret_cast<const T*>(p.w);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int n_tiles = (p.N + kLbTile - 1) / kLbTile;
    const int rank = (int)blockIdx.x % SPLIT, tile = (int)blockIdx.x / SPLIT;
    const int64_t m0 = (int64_t)(tile / n_tiles) * kLbTile;
    const int n0 = tile % n_tiles * kLbTile;
    const int steps = (p.K + kLsBK - 1) / kLsBK, s0 = (int)((int64_t)rank * steps / SPLIT), s1 = (int)((int64_t)(rank + 1) * steps / SPLIT);
    grid_dep_launch();
    grid_dep_wait();
    if (blockIdx.x == 0 && tid < 4) reinterpret_cast<int*>(p.status)[tid] = 0;
    // thread t loads rows t / 4 and t / 4 + 64 of both operands, four elements at 4 (t % 4)
    const int lrow = tid >> 2, lk = (tid & 3) * 4;
    const T* px[2];
    const T* pw[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        px[u] = x + min(m0 + lrow + 64 * u, p.T - 1) * p.ldx + lk;
        pw[u] = w + (int64_t)min(n0 + lrow + 64 * u, p.N - 1) * p.ldw + lk;
    }
    float4 ra[2], rb[2];
    auto load = [&](int s) {
        const int left = p.K - s * kLsBK - lk;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            ra[u] = load4<VEC>(px[u] + (int64_t)s * kLsBK, left);
            rb[u] = load4<VEC>(pw[u] + (int64_t)s * kLsBK, left);
        }
    };
    auto store = [&](int buf) {
        float* a = smem + buf * kStage + lk * kLbPitch + lrow;
        float* b = a + kLsBK * kLbPitch;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            a[64 * u] = ra[u].x; a[kLbPitch + 64 * u] = ra[u].y; a[2 * kLbPitch + 64 * u] = ra[u].z; a[3 * kLbPitch + 64 * u] = ra[u].w;
            b[64 * u] = rb[u].x; b[kLbPitch + 64 * u] = rb[u].y; b[2 * kLbPitch + 64 * u] = rb[u].z; b[3 * kLbPitch + 64 * u] = rb[u].w;
        }
    };
    // outputs of this thread: rows 4 ty + i and 64 + 4 ty + i, columns 4 tx + j and 64 + 4 tx + j
    float2 acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = make_float2(0.f, 0.f);
    load(s0);
    store(0);
    __syncthreads();
    int buf = 0;
    for (int s = s0; s < s1; ++s, buf ^= 1) {
        if (s + 1 < s1) load(s + 1);
        const float* sa = smem + buf * kStage + 4 * ty;
        const float* sb = smem + buf * kStage + kLsBK * kLbPitch + 4 * tx;
#pragma unroll 4
        for (int k = 0; k < kLsBK; ++k) {
            const float4 a0 = *reinterpret_cast<const float4*>(sa + k * kLbPitch), a1 = *reinterpret_cast<const float4*>(sa + k * kLbPitch + 64);
            const float4 b0 = *reinterpret_cast<const float4*>(sb + k * kLbPitch), b1 = *reinterpret_cast<const float4*>(sb + k * kLbPitch + 64);
            const float a[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
            const float2 b[4] = {make_float2(b0.x, b0.y), make_float2(b0.z, b0.w), make_float2(b1.x, b1.y), make_float2(b1.z, b1.w)};
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) fma2(acc[i][j], make_float2(a[i], a[i]), b[j]);
        }
        if (s + 1 < s1) store(buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            smem[((i >> 2) * 64 + 4 * ty + (i & 3)) * kPart + (j >> 2) * 64 + 4 * tx + (j & 3)] = (j & 1) ? acc[i][j >> 1].y : acc[i][j >> 1].x;
    const LinearEpilogue<O> ep(p);
    LinearReduce<SPLIT, O, kLbThreads, false, T> reduce(ep, (int)min((int64_t)kLbTile, p.T - m0), kLbTile, m0, n0, rank, tid);
    reduce.begin();
    if (SPLIT > 1) cooperative_groups::this_cluster().sync();
    else __syncthreads();
    reduce.run(smem, kPart, 0, 1);
    if (SPLIT > 1) cooperative_groups::this_cluster().sync();  // no CTA leaves while its part may still be read
}
constexpr size_t kLbSmem = sizeof(float) * (2 * 2 * kLsBK * kLbPitch > kLbTile * (kLbTile + 1) ? 2 * 2 * kLsBK * kLbPitch : kLbTile * (kLbTile + 1));

template <typename T, typename O, bool VEC>
cudaError_t launch_simt_t(const LinearParams& p, int sms, cudaStream_t s) {
    // few tokens / tiles: 32 x 1024 x 1024 11.1 / 15.2 us, 32 x 2000 x 2000 31.4 / 32.1, 48 x 512 x 512 5.2 / 6.2, 64 x 256 x 128 3.0 / 4.1,
    // 64 x 1024 x 1024 19.3 / 16.0
    if (p.T <= 32 || (p.T <= 64 && p.K <= 512)) {
        const int64_t grid = (int64_t)((p.N + kLfTile - 1) / kLfTile) * ((p.T + kLfTile - 1) / kLfTile);
        return launch_pdl(linear_few_kernel<T, O, VEC>, (unsigned)grid, 32 * std::max(1, std::min(kLfWarps, (p.K + 127) / 128)), 0, s, p);
    }
    const int64_t tiles = ((p.T + kLsBM - 1) / kLsBM) * ((p.N + kLsBN - 1) / kLsBN);
    if (tiles > 0x0fffffff) return cudaErrorInvalidValue;
    // Large tiles: a CTA per SM at 0.31 TFLOP/s, 1.7 us per step of 16 and 5 us for itself, with the split that fills the SMs best; the small
    // ones, 32 TFLOP/s together. Small / large: 1024 x 2000 x 1000 (tokens x features x K) 137 / 109 us, 1024 x 1000 x 2048 131 / 114, 512 x 2048 x 1024 69 / 62, 256 x
    // 2048 x 2048 68 / 60, 1000 x 500 x 500 22 / 23, 300 x 700 x 1000 21.6 / 34.
    const int64_t big = ((p.T + kLbTile - 1) / kLbTile) * ((p.N + kLbTile - 1) / kLbTile), steps = (p.K + kLsBK - 1) / kLsBK;
    int big_split = 1;
    auto us = [&](int q) { return (double)((big * q + sms - 1) / sms) * (1.7 * (double)((steps + q - 1) / q) + 5.0); };
    for (int q = 2; q <= 8 && q * 2 <= steps; q *= 2)
        if (us(q) < us(big_split)) big_split = q;
    if (us(big_split) < 2.0 * (double)p.T * p.N * p.K / 32e6 + 5.0) {
        auto go = [&](auto kernel) {
            const cudaError_t e = ensure_smem(kernel, kLbSmem);
            return e != cudaSuccess ? e : launch_pdl_cluster(kernel, (unsigned)(big * big_split), kLbThreads, kLbSmem, big_split, s, p);
        };
        switch (big_split) {
            case 1: return go(linear_simt_big_kernel<T, O, VEC, 1>);
            case 2: return go(linear_simt_big_kernel<T, O, VEC, 2>);
            case 4: return go(linear_simt_big_kernel<T, O, VEC, 4>);
            default: return go(linear_simt_big_kernel<T, O, VEC, 8>);
        }
    }
    // 64 x 1024 x 1024 (tokens x features x K) in 1 / 2 / 4 / 8 parts 63.0 / 29.5 / 17.3 / 16.0 us, 300 x 700 x 1000 62.9 / 46.4 / 35.1 /
    // 21.6, 1000 x 500 x 500 57.7 / 37.0 / 22.2 / 27.1, 1024 x 1000 x 2048 259 / 131 / 133 / 130
    int split = 1;
    while (split < 8 && tiles * split * 2 <= 4 * sms && p.K >= 4 * kLsBK * split) split *= 2;
    auto go = [&](auto kernel) { return launch_pdl_cluster(kernel, (unsigned)(tiles * split), kLsThreads, 0, split, s, p); };
    switch (split) {
        case 1: return go(linear_simt_kernel<T, O, VEC, 1>);
        case 2: return go(linear_simt_kernel<T, O, VEC, 2>);
        case 4: return go(linear_simt_kernel<T, O, VEC, 4>);
        default: return go(linear_simt_kernel<T, O, VEC, 8>);
    }
}

// Rows of any alignment -> rows of `to` elements (a multiple of 8), zeros behind the K there are. Aligned 16-byte loads inside the
// matrix, shifted to the row's start; the matrix' ends element by element.
struct PackRows {
    const __nv_bfloat16* src;
    __nv_bfloat16* dst;
    int64_t rows, ld;
};
__global__ void __launch_bounds__(256) pack_rows_kernel(PackRows x, PackRows w, int K, int to, DeviceStatus* status) {
    grid_dep_launch();
    grid_dep_wait();
    if (blockIdx.x == 0 && threadIdx.x < 4) reinterpret_cast<int*>(status)[threadIdx.x] = 0;
    const int chunks = to / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (x.rows + w.rows) * chunks; i += (int64_t)gridDim.x * 256) {
        int64_t r = i / chunks;
        const int k = (int)(i - r * chunks) * 8;
        const bool first = r < x.rows;
        const PackRows& m = first ? x : w;
        if (!first) r -= x.rows;
        const __nv_bfloat16* src = m.src + r * m.ld + k;
        const uintptr_t at = reinterpret_cast<uintptr_t>(src), low = at & ~(uintptr_t)15;
        const uintptr_t begin = reinterpret_cast<uintptr_t>(m.src), end = reinterpret_cast<uintptr_t>(m.src + (m.rows - 1) * m.ld + K);
        uint32_t o[4] = {0u, 0u, 0u, 0u};
        if (k + 8 <= K && low >= begin && low + 32 <= end) {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(low)), b = __ldg(reinterpret_cast<const uint4*>(low + 16));
            const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            const int words = (int)(at - low) >> 2, bits = ((int)(at - low) & 2) * 8;
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (words == s)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = __funnelshift_r(v[s + j], v[min(s + j + 1, 7)], bits);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + j < K) reinterpret_cast<__nv_bfloat16*>(o)[j] = src[j];
        }
        *reinterpret_cast<uint4*>(m.dst + r * to + k) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

}  // namespace

cudaError_t launch_linear_pack(const LinearParams& p, void* xp, void* wp, int to, int sms, cudaStream_t s) {
    const PackRows x{reinterpret_cast<const __nv_bfloat16*>(p.x), reinterpret_cast<__nv_bfloat16*>(xp), xp != nullptr ? p.T : 0, p.ldx};
    const PackRows w{reinterpret_cast<const __nv_bfloat16*>(p.w), reinterpret_cast<__nv_bfloat16*>(wp), wp != nullptr ? p.N : 0, p.ldw};
    const int64_t chunks = (x.rows + w.rows) * (to / 8);
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>((chunks + 255) / 256, (int64_t)16 * sms));
    return launch_pdl(pack_rows_kernel, grid, 256, 0, s, x, w, p.K, to, p.status);
}

cudaError_t launch_linear_simt(const LinearParams& p, bool bf16, bool out_bf16, int sms, cudaStream_t s) {
    const uintptr_t bytes = bf16 ? 8 : 16;
    const bool vec = ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.w)) & (bytes - 1)) == 0 && ((p.ldx | p.ldw) & 3) == 0;
    if (!bf16) return vec ? launch_simt_t<float, float, true>(p, sms, s) : launch_simt_t<float, float, false>(p, sms, s);
    if (out_bf16)
        return vec ? launch_simt_t<__nv_bfloat16, __nv_bfloat16, true>(p, sms, s) : launch_simt_t<__nv_bfloat16, __nv_bfloat16, false>(p, sms, s);
    return vec ? launch_simt_t<__nv_bfloat16, float, true>(p, sms, s) : launch_simt_t<__nv_bfloat16, float, false>(p, sms, s);
}

}  // namespace exfold
