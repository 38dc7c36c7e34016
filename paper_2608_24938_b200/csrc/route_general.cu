// Routing by a model's own router: softmax or sigmoid scores, a bias for the choice, expert groups, Top-K, weights; and the
// gradient of those weights with respect to the router scores.
//
// A warp takes a token at a time: expert lane + 32 q in register q of NPL. A call reads 4 N bytes per token and is bound by
// instructions, so what is done per token is kept short:
//
//   choice    Choices are scores + bias, and two of them may differ by less than an fp32 rounding, so they are compared as computed in
//             64 bits. That is done only where it matters: choices are computed and ranked in fp32, K + 1 of them, and only where two
//             neighbours in that ranking lie closer than the fp32 error (below) are these K + 1 ranked again by 64-bit choices: one
//             token in a few hundred. Where that leaves the set open (the next one is as close, or a group is), or a softmax has a bias,
//             all experts are (pick_exact). Scores ranked as they are (no bias) need no second look.
//   Top-K     each lane sorts its NPL keys; a round is a warp-wide maximum over the lanes' heads and the lowest expert that has it,
//             and that one's lane moves its next key up
//   weights   of the K chosen in 64 bits, rounded once: one lane per slot, up to four tokens of a warp at once
//
// Error of an fp32 choice, in half steps of 1 (2^-24; a score s is at most 1). Sigmoid: __expf is off by 2 + 1.2 |z| steps, which count
// s (1 - s) times: below 1.3; the sum 1, the quotient 4. Softmax: the argument's rounding counts d e^-d <= 0.4, expf 4, the sum 13, the
// quotient 4: below 22. And the addition's half step of the choice. Two choices are sure of their order if further apart than twice that.
//
// GPU time, 64-bit choices for every token -> now (sigmoid, bias, Top-8): 16384 tokens x 128 experts 23.2 -> 10.6 us, 777 x 256 in 8 groups
// with the load 13.2 -> 6.3, one token 4.4 -> 2.5; gradient, a token per warp -> now: 16384 x 128 13.0 -> 3.8, softmax over all experts 6.3.
// Ranking by one word (24 bits of the choice, 8 of the expert: one reduction per round instead of two) took 12.1 and 6.9 us (blocks of 256 threads: 12.8 and 5.9).
#include <algorithm>

#include "common.cuh"

namespace exfold {

namespace {

constexpr int kGrThreads = 256;
constexpr float kMaskedScore = -3.402823466e38f;  // this and -infinity
constexpr float kRounding = 1.f / (1 << 24);
constexpr float kErrSigmoid = 2.f * 6.5f * kRounding, kErrSoftmax = 2.f * 22.f * kRounding, kErrChoice = 2.f * kRounding;

// Order-preserving image of a double; every NaN is the largest, -0 is +0
__device__ __forceinline__ unsigned long long order64(double c) {
    if (c != c) return ~0ull;
    const unsigned long long b = (unsigned long long)__double_as_longlong(c + 0.0);
    return (b >> 63) ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ double from_order64(unsigned long long k) {
    return k == ~0ull ? (double)NAN : __longlong_as_double((long long)((k >> 63) ? k & ~(1ull << 63) : ~k));
}
// The same of a float
__device__ __forceinline__ unsigned order32(float f) { return f != f ? 0xffffffffu : float_order_key(f); }
__device__ __forceinline__ float from_order32(unsigned k) { return k == 0xffffffffu ? NAN : float_from_order_key(k); }

// Whether a, ranked before b by fp32 choices whose scores may be off by err / 2, might come after it in 64 bits
__device__ __forceinline__ bool close_call(float a, float b, float err) {
    return !(a - b > err + kErrChoice * fmaxf(fabsf(a), fabsf(b))) && a > -INFINITY && b > -INFINITY;  // a NaN is not close to what follows it
}

// `n` experts, one per lane, in the order of 64-bit choices (sigmoid scores): lane k returns the k-th
__device__ __forceinline__ int rank_exact(const RouteGeneralParams& p, const float* z, int id, int n, int lane) {
    unsigned long long key = 0;
    if (lane < n) {
        const float v = z[id];
        double c = 1.0 / (1.0 + exp(-(double)v));
        if (p.bias != nullptr) c += (double)p.bias[id];
        key = order64(v <= kMaskedScore ? -INFINITY : c);
    }
    int place = lane < n ? 0 : lane, out = id;
    for (int j = 0; j < n; ++j) {
        const unsigned long long kj = __shfl_sync(0xffffffffu, key, j);
        const int ij = __shfl_sync(0xffffffffu, id, j);
        if (lane < n && (kj > key || (kj == key && ij < id))) ++place;
    }
    for (int j = 0; j < n; ++j) {
        const int pj = __shfl_sync(0xffffffffu, place, j), ij = __shfl_sync(0xffffffffu, id, j);
        if (pj == lane) out = ij;
    }
    return out;
}

// One token's experts from 64-bit choices: lane k < K returns the k-th. sk: scratch of N words of the warp.
template <int NPL>
__device__ __forceinline__ int pick_exact(const RouteGeneralParams& p, const float* z, unsigned long long* sk, int lane) {
    const int N = p.N, K = p.K;
    unsigned long long key[NPL];
    unsigned cand = 0;
    float zmax = -INFINITY;
#pragma unroll
    for (int q = 0; q < NPL; ++q) {
        const float v = lane + 32 * q < N ? z[lane + 32 * q] : -INFINITY;
        zmax = isnan(v) || v > zmax ? v : zmax;
    }
    zmax = from_order32(__reduce_max_sync(0xffffffffu, order32(zmax)));
    double sum = 0.0;
    if (p.softmax) {
#pragma unroll
        for (int q = 0; q < NPL; ++q) {
            const float v = lane + 32 * q < N ? z[lane + 32 * q] : -INFINITY;
            if (!(v <= kMaskedScore)) sum += exp((double)v - (double)zmax);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
#pragma unroll
    for (int q = 0; q < NPL; ++q) {
        const int e = lane + 32 * q;
        const float v = e < N ? z[e] : -INFINITY;
        double c = (double)v;
        if (p.by_score) {
            c = p.softmax ? exp((double)v - (double)zmax) / sum : 1.0 / (1.0 + exp(-(double)v));
            if (p.bias != nullptr && e < N) c += (double)p.bias[e];
        }
        if (v <= kMaskedScore) c = -INFINITY;
        if (e < N) cand |= 1u << q;
        key[q] = order64(c);
    }
    if (p.n_groups > 1) {  // lane g takes group g's score and its place among the groups
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
        if (p.group_top2 && k2 > order64(-INFINITY)) k1 = order64(from_order64(k1) + from_order64(k2));
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
    return my_id;
}

// Groups on fp32 choices (key: their images, cleared for the experts of groups that do not stay). Returns whether the choice of groups
// is certain. Each group is read by 32 / 2^ceil(log2 groups) lanes.
template <int NPL>
__device__ __forceinline__ bool pick_groups(const RouteGeneralParams& p, unsigned (&key)[NPL], unsigned* sk, int lane) {
    const int N = p.N, G = p.n_groups, per = N / G;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < NPL; ++q)
        if (lane + 32 * q < N) sk[lane + 32 * q] = key[q];
    __syncwarp();
    int lanes = 32;
    while (lanes * G > 32) lanes >>= 1;
    const int g = lane / lanes;
    unsigned k1 = 0, k2 = 0;
    if (g < G)
        for (int j = lane % lanes; j < per; j += lanes) {
            const unsigned k = sk[g * per + j];
            k2 = max(k2, min(k1, k));
            k1 = max(k1, k);
        }
    for (int o = lanes >> 1; o > 0; o >>= 1) {
        const unsigned a = __shfl_xor_sync(0xffffffffu, k1, o), b = __shfl_xor_sync(0xffffffffu, k2, o);
        k2 = max(min(k1, a), max(k2, b));
        k1 = max(k1, a);
    }
    // The group's value lies between lower and upper in 64 bits: a choice is off by its score's error and a rounding of its own size, the
    // sum of two by both and one of its own. (Choices of opposite signs are far larger than their sum, and so are their roundings.)
    unsigned lower = k1, upper = k1;  // a masked or a NaN group is what it is
    const float c1 = from_order32(k1);
    if (c1 > -INFINITY) {
        const float score_off = (p.softmax ? kErrSoftmax : kErrSigmoid) * 0.5f;
        float value = c1, off = score_off + kRounding * fabsf(c1);
        if (p.group_top2 && k2 > order32(-INFINITY)) {
            const float c2 = from_order32(k2);
            value += c2;
            off += score_off + kRounding * (fabsf(c2) + fabsf(value));
            k1 = order32(value);
        }
        off = 1.01f * off + kRounding * fabsf(value);  // with the roundings of these lines
        lower = isinf(off) ? order32(-INFINITY) : order32(value - off);  // the sum overflowed: anywhere
        upper = isinf(off) ? 0xffffffffu : order32(value + off);
    }
    if (g >= G) k1 = 0;
    int place = 0;
    for (int o = 0; o < G; ++o) {
        const unsigned ko = __shfl_sync(0xffffffffu, k1, o * lanes);
        if (ko > k1 || (ko == k1 && o < g)) ++place;
    }
    const bool in = g < G && place < p.top_groups;
    const unsigned stay = __ballot_sync(0xffffffffu, in);
    const unsigned last = __reduce_min_sync(0xffffffffu, in ? lower : 0xffffffffu), next = __reduce_max_sync(0xffffffffu, in || g >= G ? 0u : upper);
#pragma unroll
    for (int q = 0; q < NPL; ++q)
        if (!((stay >> min(31, (lane + 32 * q) / per * lanes)) & 1u)) key[q] = 0;
    return !p.by_score || last > next || next == order32(-INFINITY);  // (every group left out is masked: those go by their places)
}

// Descending; neighbours change places only if the second is larger, so equal keys stay in the order of their experts
template <int NPL>
__device__ __forceinline__ void sort_keys(unsigned (&key)[NPL], int (&id)[NPL]) {
#pragma unroll
    for (int r = 0; r < NPL; ++r)
#pragma unroll
        for (int a = r & 1; a + 1 < NPL; a += 2) {
            const bool swap = key[a + 1] > key[a];
            const unsigned k = key[a];
            const int i = id[a];
            key[a] = swap ? key[a + 1] : k;
            id[a] = swap ? id[a + 1] : i;
            key[a + 1] = swap ? k : key[a + 1];
            id[a + 1] = swap ? i : id[a + 1];
        }
}

__global__ void __launch_bounds__(kMaxExperts) clear_load_kernel(int32_t* load, int N) {
    grid_dep_launch();
    grid_dep_wait();
    if ((int)threadIdx.x < N) load[threadIdx.x] = 0;
}

// Blocks of 128 threads up to 128 experts: the compiler may use more registers, and an SM gets the next warps sooner (16384 tokens of 128
// experts 12.8 -> 10.6 us; 777 tokens of 256 experts in groups 5.9 -> 7.3)
constexpr int route_threads(int npl) { return npl <= 4 ? 128 : kGrThreads; }

// SLOTS: lanes per token when the weights are computed, K rounded up to 8, 16 or 32; a warp takes `batch` <= 32 / SLOTS tokens at a time
template <int NPL, int SLOTS>
__global__ void __launch_bounds__(route_threads(NPL)) route_general_kernel(const __grid_constant__ RouteGeneralParams p) {
    extern __shared__ unsigned long long s_key[];  // [warps][N]
    __shared__ int hist[kMaxExperts];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
    const int N = p.N, K = p.K, batch = p.batch;
    unsigned long long* sk = s_key + warp * N;
    grid_dep_launch();
    if (p.load != nullptr) {
        for (int e = threadIdx.x; e < N; e += blockDim.x) hist[e] = 0;
        __syncthreads();
    }
    grid_dep_wait();
    float bias[NPL];
#pragma unroll
    for (int q = 0; q < NPL; ++q) bias[q] = p.bias != nullptr && lane + 32 * q < N ? p.bias[lane + 32 * q] : 0.f;
    const int64_t step = (int64_t)gridDim.x * warps * batch;
    for (int64_t i0 = ((int64_t)blockIdx.x * warps + warp) * batch; i0 < p.T; i0 += step) {
        const int here = (int)min((int64_t)batch, p.T - i0);
        int my_id = 0;              // lane SLOTS t + k: of token i0 + t, slot k
        double my_max = 0.0, my_sum = 1.0;  // softmax over all experts: that token's
        float v[NPL];
#pragma unroll
        for (int q = 0; q < NPL; ++q) v[q] = lane + 32 * q < N ? p.logits[i0 * N + lane + 32 * q] : -INFINITY;
        for (int t = 0; t < here; ++t) {
            const float* z = p.logits + (i0 + t) * N;
            float next[NPL];  // the next token's scores on their way
#pragma unroll
            for (int q = 0; q < NPL; ++q) next[q] = t + 1 < here && lane + 32 * q < N ? z[N + lane + 32 * q] : -INFINITY;
            unsigned key[NPL];
            int id[NPL];
            if (p.softmax && (p.by_score || !p.renormalise)) {
                float zmax = -INFINITY;
#pragma unroll
                for (int q = 0; q < NPL; ++q) zmax = isnan(v[q]) || v[q] > zmax ? v[q] : zmax;
                zmax = from_order32(__reduce_max_sync(0xffffffffu, order32(zmax)));
                float ex[NPL], sum = 0.f;
                if (!p.renormalise) {  // the weights are quotients of the whole sum
                    double part = 0.0;
#pragma unroll
                    for (int q = 0; q < NPL; ++q) {
                        const double e = v[q] <= kMaskedScore ? 0.0 : exp((double)v[q] - (double)zmax);
                        part += e;
                        ex[q] = (float)e;
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
                    sum = (float)part;
                    if (lane / SLOTS == t) {
                        my_max = (double)zmax;
                        my_sum = part;
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < NPL; ++q) {
                        ex[q] = v[q] <= kMaskedScore ? 0.f : expf(v[q] - zmax);
                        sum += ex[q];
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                }
#pragma unroll
                for (int q = 0; q < NPL; ++q) key[q] = order32(p.by_score ? __fdividef(ex[q], sum) + bias[q] : v[q]);
            } else {
#pragma unroll
                for (int q = 0; q < NPL; ++q)
                    key[q] = order32(p.by_score ? __fdividef(1.f, 1.f + __expf(v[q] < -80.f ? 80.f : -v[q])) + bias[q] : v[q]);
            }
#pragma unroll
            for (int q = 0; q < NPL; ++q) {
                if (v[q] <= kMaskedScore) key[q] = order32(-INFINITY);
                if (lane + 32 * q >= N) key[q] = 0;
                id[q] = lane + 32 * q;
            }
            bool sure = true;
            if (p.n_groups > 1) sure = pick_groups<NPL>(p, key, reinterpret_cast<unsigned*>(sk), lane);
            sort_keys<NPL>(key, id);
            int pick = 0;            // lane k: the k-th
            unsigned pick_key = 0;
            const int rounds = p.by_score ? min(K + 1, 32) : K;
            for (int k = 0; k < rounds; ++k) {
                const unsigned best = __reduce_max_sync(0xffffffffu, key[0]);
                const int e = (int)__reduce_min_sync(0xffffffffu, key[0] == best ? (unsigned)id[0] : 0xffffffffu);
                if (lane == k) {
                    pick = e;
                    pick_key = best;
                }
                if (e == id[0]) {
#pragma unroll
                    for (int q = 0; q + 1 < NPL; ++q) {
                        key[q] = key[q + 1];
                        id[q] = id[q + 1];
                    }
                    key[NPL - 1] = 0;
                    id[NPL - 1] = -1;
                }
            }
            if (p.by_score) {
                const float err = p.softmax ? kErrSoftmax : kErrSigmoid, c = from_order32(pick_key), before = __shfl_up_sync(0xffffffffu, c, 1);
                // (a key of 0 is no expert: there are no more)
                const unsigned close = __ballot_sync(0xffffffffu, lane > 0 && lane < rounds && pick_key != 0 && close_call(before, c, err));
                if (close != 0 || !sure || rounds == K) {  // warp-uniform
                    const unsigned more = __reduce_max_sync(0xffffffffu, key[0]);
                    // the set is open: its last one is as close to the next as may be
                    const bool open = (rounds == K || ((close >> K) & 1u)) && more != 0 &&
                                      close_call(__shfl_sync(0xffffffffu, c, rounds - 1), from_order32(more), err);
                    if (p.softmax || !sure || open) pick = pick_exact<NPL>(p, z, sk, lane);
                    else if (close != 0) pick = rank_exact(p, z, pick, __popc(__ballot_sync(0xffffffffu, pick_key != 0)), lane);
                }
            }
            const int mine = __shfl_sync(0xffffffffu, pick, lane % SLOTS);
            if (lane / SLOTS == t) my_id = mine;
#pragma unroll
            for (int q = 0; q < NPL; ++q) v[q] = next[q];
        }
        // weights of all tokens of the batch
        const int t = lane / SLOTS, k = lane % SLOTS;
        const bool slot = t < here && k < K;
        const int64_t i = i0 + t;
        const float zk = slot ? p.logits[i * N + my_id] : -INFINITY;
        const bool live = slot && !(zk <= kMaskedScore);
        double s = 0.0;
        if (!p.softmax) {
            if (live) s = 1.0 / (1.0 + exp(-(double)zk));
        } else if (p.renormalise) {
            unsigned m = order32(live ? zk : -INFINITY);
#pragma unroll
            for (int o = SLOTS / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (live) s = exp((double)zk - (double)from_order32(m));
        } else if (live) {
            s = exp((double)zk - my_max) / my_sum;
        }
        if (p.renormalise) {
            double total = s;
#pragma unroll
            for (int o = SLOTS / 2; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
            s = total != 0.0 ? s / total : 0.0;
        }
        if (slot) {
            p.ids[i * K + k] = my_id;
            p.w[i * K + k] = (float)(s * (double)p.scale);
            if (p.load != nullptr) atomicAdd(&hist[my_id], 1);
        }
    }
    if (p.load == nullptr) return;
    __syncthreads();
    for (int e = threadIdx.x; e < N; e += blockDim.x) {
        if (gridDim.x == 1) p.load[e] = hist[e];
        else if (hist[e] != 0) atomicAdd(&p.load[e], hist[e]);
    }
}

// Tokens of a warp at a time. The rows of four tokens of more than 128 experts do not fit the registers of four blocks per SM (16384 x 256,
// softmax over all: 10.6 us, with two 9.7).
__host__ __device__ constexpr int back_batch(int nq, int slots, bool dense) { return dense && nq > 1 && slots < 16 ? 2 : 32 / slots; }

// The gradient, up to `batch` <= back_batch tokens of a warp at a time: lane SLOTS t + k holds token t's chosen expert k. Rows are written
// without the chosen ones (zeros, or the softmax over all experts), and those after them. VEC: rows of whole, aligned groups of four,
// expert 4 lane + j + 128 q in v[q][j]; else expert lane + 32 (4 q + j). A row is 4 N bytes written, and as many read where the softmax is
// over all experts.
//
// Softmax over all experts, R the sum of exp(z - max) over the experts that were not chosen, e_k those of the chosen, E = R + sum e_k:
// a chosen one gets s_k (g_k R + sum_j (g_k - g_j) e_j) / E, any other -s sum_j g_j e_j / E. A confident router's s_k is close to 1, and as
// g_k s_k - s_k sum_j g_j s_j its entry would be what is left of two nearly equal numbers. R is an fp32 sum of its own terms; the e_j and
// their sums are 64-bit ones, one lane per slot.
// DENSE: softmax over all experts.
template <int NQ, int SLOTS, bool VEC, bool DENSE>
__global__ void __launch_bounds__(kGrThreads, 4) route_backward_kernel(const __grid_constant__ RouteBackwardParams p) {
    constexpr int kBatch = back_batch(NQ, SLOTS, DENSE);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
    const int N = p.N, K = p.K, batch = p.batch;
    constexpr int kWords = kMaxExperts / 32;
    __shared__ unsigned s_chosen[DENSE ? kGrThreads / 32 : 1][kBatch * kWords];  // bits of each token's chosen experts
    unsigned* chosen = s_chosen[DENSE ? warp : 0];
    auto expert = [&](int q, int j) { return VEC ? 4 * lane + 128 * q + j : lane + 32 * (4 * q + j); };
    grid_dep_launch();
    grid_dep_wait();
    const int64_t step = (int64_t)gridDim.x * warps * batch;
    for (int64_t i0 = ((int64_t)blockIdx.x * warps + warp) * batch; i0 < p.T; i0 += step) {
        const int here = (int)min((int64_t)batch, p.T - i0);
        const int t = lane / SLOTS, k = lane % SLOTS;
        const int64_t i = i0 + t;
        int id = t < here && k < K ? p.ids[i * K + k] : -1;
        if (id >= N) id = -1;
        const float g = id >= 0 ? p.dw[i * K + k] : 0.f;
        const float zk = id >= 0 ? p.logits[i * N + id] : -INFINITY;
        const bool live = zk > kMaskedScore || isnan(zk);
        float ex[DENSE ? kBatch : 1][NQ][4];  // exp(z - max) of each token's experts
        float my_max = 0.f, my_rest = 0.f;
        if constexpr (DENSE) {
            if (lane < kBatch * kWords) chosen[lane] = 0u;
            __syncwarp();
            if (id >= 0) atomicOr(&chosen[t * kWords + (id >> 5)], 1u << (id & 31));
            __syncwarp();
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (u >= here) break;
                const float* z = p.logits + (i0 + u) * N;
                float zmax = -INFINITY;
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    if (VEC) {
                        float4 w = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                        if (expert(q, 0) < N) w = *reinterpret_cast<const float4*>(z + expert(q, 0));
                        ex[u][q][0] = w.x; ex[u][q][1] = w.y; ex[u][q][2] = w.z; ex[u][q][3] = w.w;
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) ex[u][q][j] = expert(q, j) < N ? z[expert(q, j)] : -INFINITY;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) zmax = isnan(ex[u][q][j]) || ex[u][q][j] > zmax ? ex[u][q][j] : zmax;
                }
                zmax = from_order32(__reduce_max_sync(0xffffffffu, order32(zmax)));
                float rest = 0.f;
#pragma unroll
                for (int q = 0; q < NQ; ++q)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int e = expert(q, j);  // (of no expert: 0, whatever the bit)
                        ex[u][q][j] = ex[u][q][j] <= kMaskedScore ? 0.f : expf(ex[u][q][j] - zmax);
                        rest += (chosen[u * kWords + ((e >> 5) & (kWords - 1))] >> (e & 31)) & 1u ? 0.f : ex[u][q][j];
                    }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
                if (t == u) {
                    my_max = zmax;
                    my_rest = rest;
                }
            }
        }
        float dz, others = 0.f;  // of the chosen expert; the other experts' as a factor of exp(z - max)
        if constexpr (DENSE) {
            const double e = live ? exp((double)zk - (double)my_max) : 0.0;
            double sum = e, dot = e * (double)g;
#pragma unroll
            for (int o = SLOTS / 2; o > 0; o >>= 1) {
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
                dot += __shfl_xor_sync(0xffffffffu, dot, o);
            }
            const double all = sum + (double)my_rest, inv = all != 0.0 ? 1.0 / all : 0.0, factor = (double)p.scale * inv * inv;
            dz = live ? (float)(factor * e * ((double)g * (double)my_rest + ((double)g * sum - dot))) : 0.f;
            others = (float)(-factor * dot);
        } else {
            double s = 0.0, rest = 1.0;  // score (softmax: up to a factor), 1 - score
            if (p.softmax) {
                unsigned m = order32(live ? zk : -INFINITY);
#pragma unroll
                for (int o = SLOTS / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                if (live) s = exp((double)zk - (double)from_order32(m));
            } else if (live) {
                const double e = exp(-fabs((double)zk)), r = 1.0 / (1.0 + e);
                s = zk >= 0.f ? r : e * r;
                rest = zk >= 0.f ? e * r : r;
                if (isnan(zk)) s = rest = NAN;
            }
            double ds = (double)g;
            double factor = s;
            if (p.renormalise) {
                double total = s, part = live ? s * (double)g : 0.0;
#pragma unroll
                for (int o = SLOTS / 2; o > 0; o >>= 1) {
                    total += __shfl_xor_sync(0xffffffffu, total, o);
                    part += __shfl_xor_sync(0xffffffffu, part, o);
                }
                const double inv = total != 0.0 ? 1.0 / total : 0.0;
                factor = s * inv;
                ds = total != 0.0 ? (double)g - part * inv : 0.0;
            }
            dz = live ? (float)((double)p.scale * factor * ds * rest) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (u >= here) break;
            const float f = DENSE ? __shfl_sync(0xffffffffu, others, SLOTS * u) : 0.f;
            float* dst = p.dlogits + (i0 + u) * N;
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                float o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = DENSE ? ex[DENSE ? u : 0][q][j] : 0.f;
                    o[j] = e != 0.f ? f * e : 0.f;  // a masked expert has none
                }
                if (VEC) {
                    if (expert(q, 0) < N) *reinterpret_cast<float4*>(dst + expert(q, 0)) = make_float4(o[0], o[1], o[2], o[3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (expert(q, j) < N) dst[expert(q, j)] = o[j];
                }
            }
        }
        __syncwarp();
        if (id >= 0) p.dlogits[i * N + id] = dz;
    }
}

}  // namespace

cudaError_t launch_route_general(RouteGeneralParams p, int sms, cudaStream_t s) {
    const int threads = route_threads((p.N + 31) / 32), kWarps = threads / 32;
    const int slots = p.K <= 8 ? 8 : p.K <= 16 ? 16 : 32;
    // Long prompts: several tokens of a warp share the 64-bit part; short ones take a warp each, it is one token's chain of latencies then
    p.batch = p.T >= (int64_t)sms * 32 ? 32 / slots : 1;
    const unsigned blocks = (unsigned)std::max<int64_t>(1, std::min<int64_t>((p.T + kWarps * p.batch - 1) / (kWarps * p.batch), (int64_t)8 * sms * (kGrThreads / threads)));
    // load: several CTAs add theirs up in memory, which a kernel clears first (a memset, which the next kernel cannot be launched under,
    // took 3.5 us of a call; CTAs of a cluster that add up between themselves, for 64 tokens, 0.9 us more than this)
    if (p.load != nullptr && (blocks > 1 || p.T == 0)) {
        cudaError_t e = launch_pdl(clear_load_kernel, 1, kMaxExperts, 0, s, p.load, p.N);
        if (e != cudaSuccess) return e;
    }
    if (p.T == 0) return cudaSuccess;
    const size_t smem = p.n_groups > 1 ? (size_t)kWarps * p.N * sizeof(unsigned long long) : 0;
    auto go = [&](auto kernel) { return launch_pdl(kernel, blocks, threads, smem, s, p); };
#define EXFOLD_ROUTE(NPL) \
    return slots == 8 ? go(route_general_kernel<NPL, 8>) : slots == 16 ? go(route_general_kernel<NPL, 16>) : go(route_general_kernel<NPL, 32>)
    switch ((p.N + 31) / 32) {
        case 1: EXFOLD_ROUTE(1);
        case 2: EXFOLD_ROUTE(2);
        case 3: case 4: EXFOLD_ROUTE(4);
        default: EXFOLD_ROUTE(8);
    }
#undef EXFOLD_ROUTE
}

cudaError_t launch_route_backward(RouteBackwardParams p, int sms, cudaStream_t s) {
    if (p.T == 0) return cudaSuccess;
    constexpr int kWarps = kGrThreads / 32;
    const int slots = p.K <= 8 ? 8 : p.K <= 16 ? 16 : 32;
    const bool dense = p.softmax && !p.renormalise;
    p.batch = p.T >= (int64_t)sms * kWarps * 4 ? back_batch(p.N <= 128 ? 1 : 2, slots, dense) : 1;
    const unsigned blocks = (unsigned)std::min<int64_t>((p.T + kWarps * p.batch - 1) / (kWarps * p.batch), (int64_t)8 * sms);
    const bool vec = p.N % 4 == 0 && ((reinterpret_cast<uintptr_t>(p.logits) | reinterpret_cast<uintptr_t>(p.dlogits)) & 15) == 0;
    auto go = [&](auto kernel) { return launch_pdl(kernel, blocks, kGrThreads, 0, s, p); };
#define EXFOLD_BACK_D(NQ, V, D) \
    (slots == 8 ? go(route_backward_kernel<NQ, 8, V, D>) : slots == 16 ? go(route_backward_kernel<NQ, 16, V, D>) : go(route_backward_kernel<NQ, 32, V, D>))
#define EXFOLD_BACK(NQ, V) (dense ? EXFOLD_BACK_D(NQ, V, true) : EXFOLD_BACK_D(NQ, V, false))
    if (p.N <= 128) return vec ? EXFOLD_BACK(1, true) : EXFOLD_BACK(1, false);
    return vec ? EXFOLD_BACK(2, true) : EXFOLD_BACK(2, false);
#undef EXFOLD_BACK_D
#undef EXFOLD_BACK
}

}  // namespace exfold
