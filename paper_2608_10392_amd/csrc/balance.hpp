// Balance loss of the residual experts over a routing record, their counts,
// and the gradient (include/unif_moe_ops.h).
//
// The loads c_sj and the affinities' sums of a group are a pass over the record
// (8 K bytes a token). The gradient is a second one: dl_tj = p_tj (a_sj -
// sum_m p_tm a_sm), a_sj = weight K c_sj / (G n_s sum_m c_sm), feeds the two
// products dX += dl W and dW += dl^T X. Reading X and reading and writing dX
// bound it: (2 or 4) + 8 bytes an element against 4 K operations, on the fp32
// matrix cores.
#pragma once
#include "common.hpp"

namespace unifmoe {

struct BalanceParams {
    int N, d, K, B;
    int group;             // tokens per group
    int groups;
    int pieces;            // workgroups per group in the count
    int piece;             // tokens of a group per workgroup
    int blocks;            // loads count blocks
    int past;              // dX is larger than the caches: stored past them
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
    uint64_t* sums;        // [groups, pieces, 2 K + 2]: a piece's sums of affinities (fp64), loads, the shared
                           // expert's load and valid tokens (int64)
    float* slope;          // [groups, K]: a_sj
    double* gloss;         // [groups]: L_s
    float* part;           // [parts][K][d]: partial dl^T X
    int parts;             // workgroups along the tokens
    int steps;             // of 16 tokens, per workgroup
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Sum over eight lanes side by side, in all of them.
__device__ __forceinline__ float eight_sum(float v) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, true));    // quad_perm [1,0,3,2]
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, true));    // quad_perm [2,3,0,1]
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true));   // mirrored eight
    return v;
}

// LDS writes of a wave's lanes before, its reads after, in order.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A group's sums, lane j those of expert j: its counts, L_s and slopes.
__device__ __forceinline__ void balance_finish_group(const BalanceParams& p, int64_t g, double mass, int64_t load,
                                                     int64_t shared, int64_t tokens) {
    const int lane = lane_id(), K = p.K;
    const double total = wave_sum((double)load), n = (double)tokens;
    const bool some = tokens > 0 && total > 0.0;
    const double share = some ? (double)load / total : 0.0;
    const double l = wave_sum(some ? share * mass / n : 0.0) * K;
    if (p.counts != nullptr) {
        if (lane < K) p.counts[g * (K + 1) + 1 + lane] = load;
        if (lane == 0) p.counts[g * (K + 1)] = shared;
    }
    if (lane < K) p.slope[g * K + lane] = some ? (float)((double)p.weight * K * share / (n * (double)p.groups)) : 0.f;
    if (lane == 0) {
        p.gloss[g] = l;
        if (p.groups == 1) *p.loss = (float)l;
    }
}

// Loads and affinity sums of one piece of a group per workgroup. A wave takes
// 64 tokens at a time: the record's entries are read side by side and put in
// expert order in LDS (selected experts with the sign bit set), then lane j +
// w h adds expert j's entries of the h-th of 64 / w runs of tokens, w the
// experts rounded up to a power of two. A group of one piece is finished here.
// Latency bound: all of a tile's loads are issued at once (50,432 tokens, K = 16: 8.8
// us, 0.8 TB/s; entry by entry and token by token it took 46).
constexpr int kBalWaves = 8, kBalBatch = 16;
__host__ __device__ __forceinline__ int balance_wave_words(int K) { return 64 * (K | 1) + 2 * 64; }

__global__ __launch_bounds__(kWave* kBalWaves) void balance_count_kernel(BalanceParams p) {
    extern __shared__ float lds[];
    __shared__ double masses[kBalWaves][kWave];
    __shared__ int loads[kBalWaves][kWave + 2];
    const int w = (int)threadIdx.x >> 6, nw = (int)blockDim.x >> 6, lane = lane_id(), K = p.K, ld = K | 1;
    float* const tile = lds + w * balance_wave_words(K);
    int* const unit = reinterpret_cast<int*>(tile + 64 * ld);   // what a selected expert of the token counts
    int* const chosen = unit + 64;                              // experts selected, -1: padded
    const int64_t u = (int64_t)flat_block();
    if (u >= (int64_t)p.groups * p.pieces) return;
    const int64_t g = u / p.pieces, g0 = g * p.group, g1 = g0 + p.group < p.N ? g0 + p.group : p.N;
    const int64_t t0 = g0 + (u - g * p.pieces) * p.piece, t1 = t0 + p.piece < g1 ? t0 + p.piece : g1;
    const int wide = K <= 1 ? 1 : 1 << (32 - __builtin_clz(K - 1));
    const int j = lane & (wide - 1), h = lane / wide, run = wide;   // 64 / (64 / wide) tokens per run
    double mass = 0.0;
    int load = 0, shared = 0, tokens = 0;
    for (int64_t tb = t0 + 64 * w; tb < t1; tb += 64 * nw) {
        // all of the tile's loads first, as far as the registers go: they come
        // from HBM, and a tile is short
        const int entries = (int)(t1 - tb < 64 ? t1 - tb : 64) * K;
        const int* const ids = p.eids + (size_t)tb * K;
        const float* const wts = p.wts + (size_t)tb * K;
        int e[kBalBatch];
        float v[kBalBatch];
        auto fetch = [&](int i0) {
#pragma unroll
            for (int c = 0; c < kBalBatch; ++c) {
                const int i = min(i0 + c * kWave, entries - 1);   // past the last entry: read and not used
                e[c] = ids[i];
                v[c] = wts[i];
            }
        };
        fetch(lane);
        const int64_t t = tb + lane, tc = t < t1 ? t : t1 - 1;
        const int nres = p.nres[tc], b = p.blocks ? p.nsh[tc] : 0;
        const bool ok = (p.valid == nullptr || p.valid[tc] != 0) && t < t1;
        for (int i = lane; i < 64 * ld; i += kWave) tile[i] = 0.f;
        unit[lane] = p.blocks ? p.B - b : 1;
        chosen[lane] = ok ? min(nres, K) : -1;
        if (ok) {
            shared += p.blocks ? b : 1;
            ++tokens;
        }
        wave_sync();
        int q = lane / K, r = lane - q * K;         // token and rank of entry `lane`
        const int dq = kWave / K, dr = kWave - dq * K;
        for (int i0 = lane; i0 < entries; i0 += kBalBatch * kWave) {
            if (i0 != lane) fetch(i0);
#pragma unroll
            for (int c = 0; c < kBalBatch; ++c) {
                const bool on = i0 + c * kWave < entries;
                if (on && e[c] >= 1 && e[c] <= K && chosen[q] >= 0)
                    tile[q * ld + e[c] - 1] =
                        __uint_as_float((__float_as_uint(v[c]) & 0x7fffffffu) | (r < chosen[q] ? 0x80000000u : 0u));
                q += dq;
                r += dr;
                if (r >= K) {
                    r -= K;
                    ++q;
                }
                q = min(q, 63);   // past the last entry
            }
        }
        wave_sync();
        if (j < K) {
            float m = 0.f;
#pragma unroll 8
            for (int i = 0; i < run; ++i) {
                const uint32_t v = __float_as_uint(tile[(h * run + i) * ld + j]);
                m += __uint_as_float(v & 0x7fffffffu);
                load += (v >> 31) ? unit[h * run + i] : 0;
            }
            mass += (double)m;
        }
        wave_sync();
    }
    for (int o = 32; o >= wide; o >>= 1) {
        mass += __shfl_xor(mass, o);
        load += __shfl_xor(load, o);
    }
    for (int o = 32; o > 0; o >>= 1) {
        shared += __shfl_xor(shared, o);
        tokens += __shfl_xor(tokens, o);
    }
    masses[w][lane] = mass;
    loads[w][lane] = load;
    if (lane == 0) {
        loads[w][kWave] = shared;
        loads[w][kWave + 1] = tokens;
    }
    __syncthreads();
    if (w != 0) return;
    double m = 0.0;
    int64_t l = 0, s = 0, n = 0;
    for (int i = 0; i < nw; ++i) {
        if (lane < K) {
            m += masses[i][lane];
            l += loads[i][lane];
        }
        s += loads[i][kWave];
        n += loads[i][kWave + 1];
    }
    if (p.pieces == 1) {
        balance_finish_group(p, g, m, l, s, n);
        return;
    }
    uint64_t* const out = p.sums + u * (2 * K + 2);
    if (lane < K) {
        out[lane] = __builtin_bit_cast(uint64_t, m);
        out[K + lane] = (uint64_t)l;
    }
    if (lane == 0) {
        out[2 * K] = (uint64_t)s;
        out[2 * K + 1] = (uint64_t)n;
    }
}

// One workgroup per group of several pieces: a thread per word of a piece's sums
// and stretch of the pieces, the stretches added in order.
constexpr int kBalGroupThreads = 1024, kBalStretches = 32;
__global__ __launch_bounds__(kBalGroupThreads) void balance_group_kernel(BalanceParams p) {
    __shared__ uint64_t stretch[kBalGroupThreads];
    __shared__ uint64_t total[2 * kWave + 2];
    const int64_t g = (int64_t)flat_block();
    if (g >= p.groups) return;
    const int K = p.K, words = 2 * K + 2, wide = 1 << (32 - __builtin_clz(words - 1));
    const int n = min(kBalGroupThreads / wide, kBalStretches), h = (int)threadIdx.x / wide, c = (int)threadIdx.x % wide;
    if (h < n && c < words) {
        const int q0 = (int)((int64_t)h * p.pieces / n), q1 = (int)((int64_t)(h + 1) * p.pieces / n);
        const uint64_t* const src = p.sums + g * p.pieces * words + c;
        double m = 0.0;
        uint64_t l = 0;
        for (int q = q0; q < q1; q += 16) {
            uint64_t v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = src[(size_t)min(q + i, q1 - 1) * words];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (q + i >= q1) continue;
                m += __builtin_bit_cast(double, v[i]);
                l += v[i];
            }
        }
        stretch[threadIdx.x] = c < K ? __builtin_bit_cast(uint64_t, m) : l;
    }
    __syncthreads();
    if ((int)threadIdx.x < words) {
        double m = 0.0;
        uint64_t l = 0;
        for (int i = 0; i < n; ++i) {
            m += __builtin_bit_cast(double, stretch[i * wide + threadIdx.x]);
            l += stretch[i * wide + threadIdx.x];
        }
        total[threadIdx.x] = (int)threadIdx.x < K ? __builtin_bit_cast(uint64_t, m) : l;
    }
    __syncthreads();
    if (threadIdx.x >= kWave) return;
    const int j = min((int)threadIdx.x, K - 1);
    const bool on = (int)threadIdx.x < K;
    balance_finish_group(p, g, on ? __builtin_bit_cast(double, total[j]) : 0.0, on ? (int64_t)total[K + j] : 0,
                         (int64_t)total[2 * K], (int64_t)total[2 * K + 1]);
}

// *loss = the groups' mean: strided partial sums, a wave's by a butterfly, the
// waves in order.
__device__ __forceinline__ void balance_mean(const BalanceParams& p) {
    __shared__ double part[16];
    const int nw = (int)blockDim.x >> 6, w = (int)threadIdx.x >> 6;
    double s = 0.0;
    for (int64_t g0 = threadIdx.x; g0 < p.groups; g0 += 8 * (int64_t)blockDim.x) {
        double v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t g = g0 + i * (int64_t)blockDim.x;
            v[i] = p.gloss[g < p.groups ? g : g0];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s += g0 + i * (int64_t)blockDim.x < p.groups ? v[i] : 0.0;
    }
    s = wave_sum(s);
    if (lane_id() == 0) part[w] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    s = 0.0;
    for (int i = 0; i < nw; ++i) s += part[i];
    *p.loss = p.groups > 0 ? (float)(s / p.groups) : 0.f;
}
__global__ __launch_bounds__(1024) void balance_mean_kernel(BalanceParams p) { balance_mean(p); }

// The gradients of `steps` 16-token steps per workgroup. Its waves hold 16 NC
// columns each, lane l the NC consecutive ones from 16-lane column l % 16 on, so
// that one load gives a lane its operand of NC products (product i stands for
// every NC-th column): for v_mfma_f32_16x16x4_f32, X[t + l / 16] is the right
// operand of dl^T X and W_j the one of dl W, whose sums dX_in is added to. The
// router's rows and the sums of dl^T X stay in registers. The next 16 tokens'
// rows are loaded while the current ones are multiplied.
//
// dl is formed in LDS a tile of 8 tokens per wave ahead (the waves are even in
// number, so a tile is whole steps), eight lanes per token: a wave loads its
// tokens' entries when the tile before begins, the slopes of their experts after
// its first step, and writes dl behind its last; one barrier per tile. Padded
// tokens have dl = 0, and their rows of X are not used. HBM bound: 50,432 x 768 bf16,
// K = 16 86 us, 4.7 TB/s of 10 bytes an element; 131,072 x 1,024, K = 32 285 us, 4.9
// TB/s, the matrix cores busy 40% of it at 153 TFLOP/s. In 8 columns a lane, fewer
// waves fit: 408 us for 372 there, before the ranges were sized to run at once.
template <class T, int NC>
struct BalRow {
    typedef T mem __attribute__((ext_vector_type(NC), aligned(sizeof(T))));
};
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(u16 v) { return bf2f(v); }

// Waves that a compute unit holds, by their registers (two or three per SIMD), and
// the most of a workgroup.
__host__ __device__ constexpr int balance_waves(int K) { return K <= 16 ? 12 : 8; }

template <int KT>
struct BalEntries {
    static constexpr int M = 2 * KT;   // entries per lane: ranks sub + 8 m
    int e[M];                          // expert, 0: none
    float v[M], a[M];                  // affinity, slope
};

template <class T, int KT, int NC>
__global__ __launch_bounds__(balance_waves(16 * KT) * kWave, balance_waves(16 * KT) / 4) void balance_grad_kernel(BalanceParams p) {
    constexpr int KP = 16 * KT, LD = KP + 4;   // LDS row: the 16 rows' reads of 4 neighbours meet no bank twice
    extern __shared__ float dls[];             // [2][tile][LD]
    if ((int)blockIdx.x == p.parts) {   // one workgroup more than the tokens need: the groups' mean
        if (blockIdx.y == 0) balance_mean(p);
        return;
    }
    typedef typename BalRow<T, NC>::mem x_mem;
    typedef typename BalRow<float, NC>::mem f_mem;
    typedef T x_raw __attribute__((ext_vector_type(NC)));
    typedef float f_raw __attribute__((ext_vector_type(NC)));
    const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), nw = (int)blockDim.x >> 6;
    const int lr = lane & 15, lq = lane >> 4, K = p.K;
    // This lane's columns: from col on, loaded from at (the row's last NC where
    // fewer are left); columns before col belong to other lanes.
    const int col = (((int)blockIdx.y * nw + w) * 16 + lr) * NC;
    const uint32_t at = (uint32_t)min(col, p.d - NC);
    const int own = (int)at >= col ? 0 : min(col - (int)at, NC);   // first own element (NC: none)
    const int64_t first = (int64_t)blockIdx.x * p.steps * 16;
    const int64_t end = first + p.steps * 16 < p.N ? first + p.steps * 16 : p.N;
    const bool add = p.dX_in != nullptr;

    f_raw W[4 * KT];
#pragma unroll
    for (int kk = 0; kk < 4 * KT; ++kk) {
        const int j = 4 * kk + lq;
        W[kk] = f_raw{};
        if (p.dX != nullptr && j < K) W[kk] = *reinterpret_cast<const f_mem*>(p.Wr + (size_t)(j + 1) * p.d + at);
    }
    f32x4 dW[KT][NC];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < NC; ++i) dW[kt][i] = f32x4{0.f, 0.f, 0.f, 0.f};

    x_raw x[4];   // rows t + 4 q + lq of X
    f_raw s[4];   // rows t + 4 lq + r of dX_in
    // A step's rows have a scalar base and a lane's 32-bit offset; rows past the
    // last token are read as the last one and used nowhere.
    const uint32_t xoff = ((uint32_t)lq * p.d + at) * (uint32_t)sizeof(T), soff = ((uint32_t)lq * 4 * p.d + at) * 4u;
    auto load_x = [&](int64_t t) {
        if (p.dW == nullptr) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t row = t + 4 * q < p.N ? t + 4 * q : p.N - 1;
            uint32_t off = xoff;
            if (t + 16 > p.N) off = ((uint32_t)min((int64_t)lq, p.N - 1 - row) * p.d + at) * (uint32_t)sizeof(T);
            x[q] = *reinterpret_cast<const x_mem*>(static_cast<const char*>(p.X) + (size_t)row * p.d * sizeof(T) + off);
        }
    };
    auto load_s = [&](int64_t t) {
        if (!add) return;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t row = t + r < p.N ? t + r : p.N - 1;
            uint32_t off = soff;
            if (t + 16 > p.N) off = ((uint32_t)min((int64_t)lq * 4, p.N - 1 - row) * p.d + at) * 4u;
            s[r] = *reinterpret_cast<const f_mem*>(reinterpret_cast<const char*>(p.dX_in) + (size_t)row * p.d * 4 + off);
        }
    };
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = f_raw{};
    load_x(first);
    load_s(first);

    const int tile = 8 * nw, sub = lane & 7, mine = 8 * w + (lane >> 3);   // this lane's token of a tile
    uint32_t* const used = reinterpret_cast<uint32_t*>(dls + 2 * tile * LD);   // [2][tile]: tokens that are real
    BalEntries<KT> en;
    bool real;
    auto fetch = [&](int64_t tb) {
        const int64_t t = tb + mine;
        real = t < end && (p.valid == nullptr || p.valid[t < end ? t : first] != 0);
#pragma unroll
        for (int m = 0; m < BalEntries<KT>::M; ++m) {
            const int i = sub + 8 * m;
            const bool on = real && i < K;
            const size_t at = on ? (size_t)t * K + i : 0;
            const int e = p.eids[at];
            en.v[m] = p.wts[at];
            en.e[m] = on && e >= 1 && e <= K ? e : 0;
        }
    };
    auto slopes = [&](int64_t tb) {
        const int64_t t = tb + mine;
        const size_t row = p.groups > 1 && t < end ? (size_t)((uint32_t)t / (uint32_t)p.group) * K : 0;
#pragma unroll
        for (int m = 0; m < BalEntries<KT>::M; ++m) en.a[m] = p.slope[row + max(en.e[m], 1) - 1];
    };
    auto write = [&](int b) {
        float s = 0.f;
#pragma unroll
        for (int m = 0; m < BalEntries<KT>::M; ++m) s = en.e[m] ? fmaf(en.v[m], en.a[m], s) : s;
        s = eight_sum(s);
        float* const row = dls + (b * tile + mine) * LD;
        // zeros first (a wave's LDS writes land in order): tokens without the expert, the columns past K
#pragma unroll
        for (int m = 0; m < BalEntries<KT>::M; ++m) row[sub + 8 * m] = 0.f;
#pragma unroll
        for (int m = 0; m < BalEntries<KT>::M; ++m)
            if (en.e[m]) row[en.e[m] - 1] = en.v[m] * (en.a[m] - s);
        if (sub == 0) used[b * tile + mine] = real ? 1u : 0u;
    };
    fetch(first);
    slopes(first);
    write(0);
    lds_barrier();
    const bool check = p.valid != nullptr;
    int buf = 0;
    for (int64_t tb = first; tb < end; tb += tile) {
        const bool ahead = tb + tile < end;
        if (ahead) fetch(tb + tile);
        for (int64_t t16 = tb; t16 < end && t16 < tb + tile; t16 += 16) {
            const int in_tile = buf * tile + (int)(t16 - tb);
            const float* const dl = dls + in_tile * LD;
            const bool more = t16 + 16 < end;
            if (p.dW != nullptr) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float b[NC];
#pragma unroll
                    for (int i = 0; i < NC; ++i) b[i] = to_f32(x[q][i]);
                    if (check || t16 + 16 > end) {
                        const bool on = used[in_tile + 4 * q + lq] != 0;
#pragma unroll
                        for (int i = 0; i < NC; ++i) b[i] = on ? b[i] : 0.f;
                    }
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) {
                        const float a = dl[(4 * q + lq) * LD + 16 * kt + lr];
#pragma unroll
                        for (int i = 0; i < NC; ++i)
                            dW[kt][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, b[i], dW[kt][i], 0, 0, 0);
                    }
                }
                if (more) load_x(t16 + 16);
            }
            if (p.dX != nullptr) {
                f32x4 acc[NC];
#pragma unroll
                for (int i = 0; i < NC; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < 4 * KT; ++kk) {
                    const float a = dl[lr * LD + 4 * kk + lq];
#pragma unroll
                    for (int i = 0; i < NC; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, W[kk][i], acc[i], 0, 0, 0);
                }
                f_raw v[4];   // dX_in is added last: one rounding at its magnitude
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int i = 0; i < NC; ++i) v[r][i] = s[r][i] + acc[i][r];
                if (more) load_s(t16 + 16);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (t16 + 4 * lq + r >= end) continue;
                    char* const out = reinterpret_cast<char*>(p.dX) + (size_t)(t16 + r) * p.d * 4 + soff;
                    if (own == 0 && p.past) __builtin_nontemporal_store(v[r], reinterpret_cast<f_mem*>(out));
                    else if (own == 0) *reinterpret_cast<f_mem*>(out) = v[r];
                    else
#pragma unroll
                        for (int i = 0; i < NC; ++i)
                            if (i >= own) reinterpret_cast<float*>(out)[i] = v[r][i];
                }
            }
            if (ahead && t16 == tb) slopes(tb + tile);
        }
        buf ^= 1;
        if (ahead) write(buf);
        lds_barrier();
    }
    if (p.dW == nullptr) return;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = 16 * kt + 4 * lq + r;
            if (j >= K) continue;
            float* const out = p.part + ((size_t)blockIdx.x * K + j) * p.d + at;
            f_raw v;
#pragma unroll
            for (int i = 0; i < NC; ++i) v[i] = dW[kt][i][r];
            if (own == 0) *reinterpret_cast<f_mem*>(out) = v;
            else
#pragma unroll
                for (int i = 0; i < NC; ++i)
                    if (i >= own) out[i] = v[i];
        }
}

// dW = dW_in + the parts' sum (row 0: dW_in): 64 elements per workgroup, each
// wave a stretch of the parts, all in fp64 and in order.
constexpr int kBalSumWaves = 16;
__global__ __launch_bounds__(kWave* kBalSumWaves) void balance_dw_sum_kernel(BalanceParams p) {
    __shared__ double stretch[kBalSumWaves][kWave];
    const int lane = lane_id(), w = (int)threadIdx.x >> 6;
    const size_t n = (size_t)p.K * p.d, i = (size_t)blockIdx.x * kWave + lane;   // over all K + 1 rows
    const size_t k0 = (size_t)w * p.parts / kBalSumWaves, k1 = (size_t)(w + 1) * p.parts / kBalSumWaves;
    double s = 0.0;
    if (i >= (size_t)p.d && i < n + p.d) {
        const float* const src = p.part + (i - p.d);
        size_t k = k0;
        for (; k + 8 <= k1; k += 8) {
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = src[(k + c) * n];
#pragma unroll
            for (int c = 0; c < 8; ++c) s += (double)v[c];
        }
        for (; k < k1; ++k) s += (double)src[k * n];
    }
    stretch[w][lane] = s;
    __syncthreads();
    if (w != 0 || i >= n + p.d) return;
    s = p.dW_in != nullptr ? (double)p.dW_in[i] : 0.0;
    for (int k = 0; k < kBalSumWaves; ++k) s += stretch[k][lane];
    p.dW[i] = (float)s;
}

}  // namespace unifmoe
