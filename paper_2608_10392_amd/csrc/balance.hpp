// Balance loss of the residual experts over a routing record, their counts,
// and the gradient (include/unif_moe_ops.h).
//
// The loads c_sj and the affinities' sums of a group are a pass over the record
// (8 K bytes a token); the gradient is a second one, whose dl_tj = p_tj (a_sj -
// sum_m p_tm a_sm), a_sj = weight K c_sj / (G n_s sum_m c_sm), feeds two
// products, dX += dl W and dW += dl^T X. Reading X and reading and writing dX
// bound it.
#pragma once
#include "common.hpp"

namespace unifmoe {

struct BalanceParams {
    int N, d, K, B;
    int group;             // tokens per group
    int groups;
    int pieces;            // per group, of `piece` tokens
    int piece;
    int blocks;            // loads count blocks
    float weight;
    const uint8_t* valid;
    const int* nsh;
    const int* nres;
    const int* eids;       // [N, K]
    const float* wts;      // [N, K]
    const void* X;
    const float* Wr;       // [K+1, d]
    const float* dX_in;
    float* dX;
    const float* dW_in;
    float* dW;
    float* loss;
    int64_t* counts;       // [groups, K+1]
    float* mass;           // [groups, pieces, K] sums of affinities
    int* load;             // [groups, pieces, K+2]: loads, the shared expert's, valid tokens
    float* slope;          // [groups, K]: a_sj
    double* gloss;         // [groups]: L_s
    float* dl;             // [N, K]
    float* part;           // [slices][K][d]
    int slices;
};

// Loads and affinity sums of one piece of a group per wave: 64 tokens at a
// time, their affinities put in expert order in LDS (selected experts with the
// sign bit set), then one lane per expert adds its column.
constexpr int kBalWaves = 4;
__host__ __device__ __forceinline__ int balance_lds_words(int K) { return 64 * (K | 1) + 64; }

__global__ __launch_bounds__(64 * kBalWaves) void balance_count_kernel(BalanceParams p) {
    extern __shared__ float lds[];
    const int w = (int)threadIdx.x >> 6, lane = lane_id(), K = p.K, ld = K | 1;
    float* const tile = lds + w * balance_lds_words(K);
    int* const unit = reinterpret_cast<int*>(tile + 64 * ld);
    const int64_t u = (int64_t)blockIdx.x * kBalWaves + w;
    if (u >= (int64_t)p.groups * p.pieces) return;
    const int64_t g = u / p.pieces, g0 = g * p.group, g1 = g0 + p.group < p.N ? g0 + p.group : p.N;
    const int64_t t0 = g0 + (u - g * p.pieces) * p.piece, t1 = t0 + p.piece < g1 ? t0 + p.piece : g1;
    float mass = 0.f;
    int load = 0, shared = 0, tokens = 0;
    for (int64_t tb = t0; tb < t1; tb += 64) {
        const int64_t t = tb + lane;
        const bool ok = t < t1 && (p.valid == nullptr || p.valid[t] != 0);
        for (int j = 0; j < K; ++j) tile[lane * ld + j] = 0.f;
        unit[lane] = 0;
        if (ok) {
            const int b = p.blocks ? p.nsh[t] : 0, k = min(p.nres[t], K);
            unit[lane] = p.blocks ? p.B - b : 1;
            shared += p.blocks ? b : 1;
            ++tokens;
            for (int i = 0; i < K; ++i) {
                const int e = p.eids[(size_t)t * K + i];
                if (e < 1 || e > K) continue;
                const uint32_t v = __float_as_uint(p.wts[(size_t)t * K + i]) & 0x7fffffffu;
                tile[lane * ld + e - 1] = __uint_as_float(i < k ? v | 0x80000000u : v);
            }
        }
        wait_lgkmcnt0();
        __builtin_amdgcn_wave_barrier();
        if (lane < K)
            for (int q = 0; q < 64; ++q) {
                const uint32_t v = __float_as_uint(tile[q * ld + lane]);
                mass += __uint_as_float(v & 0x7fffffffu);
                if (v >> 31) load += unit[q];
            }
        wait_lgkmcnt0();
        __builtin_amdgcn_wave_barrier();
    }
    for (int o = 32; o > 0; o >>= 1) {
        shared += __shfl_xor(shared, o);
        tokens += __shfl_xor(tokens, o);
    }
    if (lane < K) {
        p.mass[u * K + lane] = mass;
        p.load[u * (K + 2) + lane] = load;
    }
    if (lane == 0) {
        p.load[u * (K + 2) + K] = shared;
        p.load[u * (K + 2) + K + 1] = tokens;
    }
}

__device__ __forceinline__ double wave_sum(double v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// One wave per group: the pieces' sums in order, the counts, L_s and the slopes.
__global__ __launch_bounds__(64) void balance_group_kernel(BalanceParams p) {
    const int64_t g = blockIdx.x;
    const int lane = lane_id(), K = p.K;
    double mass = 0.0;
    int64_t load = 0, shared = 0, tokens = 0;
    for (int q = 0; q < p.pieces; ++q) {
        const int64_t u = g * p.pieces + q;
        if (lane < K) {
            mass += (double)p.mass[u * K + lane];
            load += p.load[u * (K + 2) + lane];
        }
        shared += p.load[u * (K + 2) + K];
        tokens += p.load[u * (K + 2) + K + 1];
    }
    const double total = wave_sum((double)load), n = (double)tokens;
    const bool some = tokens > 0 && total > 0.0;
    const double share = some ? (double)load / total : 0.0;
    const double l = wave_sum(some ? share * mass / n : 0.0) * K;
    if (p.counts != nullptr) {
        if (lane < K) p.counts[g * (K + 1) + 1 + lane] = load;
        if (lane == 0) p.counts[g * (K + 1)] = shared;
    }
    if (lane < K) p.slope[g * K + lane] = some ? (float)((double)p.weight * K * share / (n * (double)p.groups)) : 0.f;
    if (lane == 0) p.gloss[g] = l;
}

// *loss = the groups' mean, 256 strided partial sums and a fixed tree.
__global__ __launch_bounds__(256) void balance_loss_kernel(BalanceParams p) {
    __shared__ double part[256];
    double s = 0.0;
    for (int64_t g = threadIdx.x; g < p.groups; g += 256) s += p.gloss[g];
    part[threadIdx.x] = s;
    __syncthreads();
    for (int h = 128; h > 0; h >>= 1) {
        if ((int)threadIdx.x < h) part[threadIdx.x] += part[threadIdx.x + h];
        __syncthreads();
    }
    if (threadIdx.x == 0) *p.loss = p.groups > 0 ? (float)(part[0] / p.groups) : 0.f;
}

// dl of every token, one thread each.
__global__ __launch_bounds__(256) void balance_dl_kernel(BalanceParams p) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= p.N) return;
    const int K = p.K;
    float* const dl = p.dl + (size_t)t * K;
    for (int j = 0; j < K; ++j) dl[j] = 0.f;
    if (p.valid != nullptr && p.valid[t] == 0) return;
    const float* const slope = p.slope + t / p.group * K;
    float mean = 0.f;
    for (int i = 0; i < K; ++i) {
        const int e = p.eids[(size_t)t * K + i];
        if (e >= 1 && e <= K) mean = fmaf(p.wts[(size_t)t * K + i], slope[e - 1], mean);
    }
    for (int i = 0; i < K; ++i) {
        const int e = p.eids[(size_t)t * K + i];
        if (e >= 1 && e <= K) dl[e - 1] = p.wts[(size_t)t * K + i] * (slope[e - 1] - mean);
    }
}

template <class T>
__device__ __forceinline__ float to_f32(T v) { return v; }
template <>
__device__ __forceinline__ float to_f32<u16>(u16 v) { return bf2f(v); }

// dX = dX_in + dl W, 16 tokens x 256 columns per workgroup.
__global__ __launch_bounds__(256) void balance_dx_kernel(BalanceParams p) {
    __shared__ float dls[16][64];
    const int64_t t0 = (int64_t)blockIdx.x * 16;
    const int n = (int)blockIdx.y * 256 + (int)threadIdx.x, K = p.K;
    for (int x = threadIdx.x; x < 16 * K; x += 256) dls[x / K][x % K] = t0 + x / K < p.N ? p.dl[(size_t)t0 * K + x] : 0.f;
    __syncthreads();
    if (n >= p.d) return;
    float acc[16];
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    for (int j = 0; j < K; ++j) {
        const float w = p.Wr[(size_t)(j + 1) * p.d + n];
        for (int i = 0; i < 16; ++i) acc[i] = fmaf(dls[i][j], w, acc[i]);
    }
    for (int i = 0; i < 16; ++i)
        if (t0 + i < p.N) {
            const size_t at = (size_t)(t0 + i) * p.d + n;
            p.dX[at] = p.dX_in != nullptr ? p.dX_in[at] + acc[i] : acc[i];
        }
}

// Partial dl^T X of one slice of the tokens: a thread per column, 8 experts at
// a time. Padded tokens' rows are not read.
template <class T>
__global__ __launch_bounds__(256) void balance_dw_kernel(BalanceParams p) {
    const int n = (int)blockIdx.x * 256 + (int)threadIdx.x, K = p.K, j0 = (int)blockIdx.y * 8;
    const int64_t t0 = (int64_t)blockIdx.z * p.N / p.slices, t1 = (int64_t)(blockIdx.z + 1) * p.N / p.slices;
    if (n >= p.d) return;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t t = t0; t < t1; ++t) {
        if (p.valid != nullptr && p.valid[t] == 0) continue;
        const float x = to_f32(static_cast<const T*>(p.X)[(size_t)t * p.d + n]);
        for (int j = 0; j < 8; ++j)
            if (j0 + j < K) acc[j] = fmaf(p.dl[(size_t)t * K + j0 + j], x, acc[j]);
    }
    for (int j = 0; j < 8; ++j)
        if (j0 + j < K) p.part[((size_t)blockIdx.z * K + j0 + j) * p.d + n] = acc[j];
}

// dW = dW_in + the slices' sum in order (row 0: dW_in).
__global__ __launch_bounds__(256) void balance_dw_sum_kernel(BalanceParams p) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, n = (size_t)(p.K + 1) * p.d;
    if (i >= n) return;
    double s = p.dW_in != nullptr ? (double)p.dW_in[i] : 0.0;
    if (i >= (size_t)p.d)
        for (int k = 0; k < p.slices; ++k) s += (double)p.part[(size_t)k * (n - p.d) + i - p.d];
    p.dW[i] = (float)s;
}

}  // namespace unifmoe
