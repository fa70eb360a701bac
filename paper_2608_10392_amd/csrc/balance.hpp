// Balance loss of the residual experts over a routing record, their counts,
// and the gradient (include/unif_moe_ops.h).
//
// The loads c_sj and the affinities' sums of a group are a pass over the record
// (8 K bytes a token), the slopes dl_tj = p_tj (a_sj - sum_m p_tm a_sm), a_sj =
// weight K c_sj / (G n_s sum_m c_sm), a second one, which leaves them in expert
// order. They feed the two products dX += dl W and dW += dl^T X. Reading X and
// reading and writing dX bound it: (2 or 4) + 8 bytes an element against 4 K
// operations, on the fp32 matrix cores.
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
    double* gloss;         // [groups]: L_s
    float* dl;             // [N, KP]: dl in expert order, zeros past K (NULL: no gradients)
    int KP;                // K rounded up to 16
    float* part;           // [parts][K][d]: partial dl^T X
    int parts;             // workgroups along the tokens
    int steps;             // of 16 tokens, per workgroup
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// LDS writes of a wave's lanes before, its reads after, in order.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A group's sums, lane j those of expert j: its counts and L_s (where `write`),
// and its a_sj into `slope`.
__device__ __forceinline__ void balance_finish_group(const BalanceParams& p, int64_t g, double mass, int64_t load,
                                                     int64_t shared, int64_t tokens, bool write, float* slope) {
    const int lane = lane_id(), K = p.K;
    const double total = wave_sum((double)load), n = (double)tokens;
    const bool some = tokens > 0 && total > 0.0;
    const double share = some ? (double)load / total : 0.0;
    const double l = wave_sum(some ? share * mass / n : 0.0) * K;
    if (lane < K) slope[lane] = some ? (float)((double)p.weight * K * share / (n * (double)p.groups)) : 0.f;
    if (!write) return;
    if (p.counts != nullptr) {
        if (lane < K) p.counts[g * (K + 1) + 1 + lane] = load;
        if (lane == 0) p.counts[g * (K + 1)] = shared;
    }
    if (lane == 0) {
        p.gloss[g] = l;
        if (p.groups == 1) *p.loss = (float)l;
    }
}

// A wave's tile of the record: 64 tokens' entries in expert order in LDS, read side
// by side (the affinity, selected experts with the sign bit set; zeros for padded
// tokens and experts that a token lacks).
constexpr int kBalWaves = 8, kBalBatch = 16;
__host__ __device__ __forceinline__ int balance_wave_words(int K) { return 64 * (K | 1) + 2 * 64; }

struct BalTile {
    float* p;      // [64][K | 1]
    int* unit;     // [64] what a selected expert of the token counts; then its mean slope
    int* chosen;   // [64] experts selected, -1: padded
    int shared, tokens;   // this lane's share of the shared expert's load and of the valid tokens
    __device__ __forceinline__ BalTile(float* lds, int w, int K)
        : p(lds + w * balance_wave_words(K)), unit(reinterpret_cast<int*>(p + 64 * (K | 1))), chosen(unit + 64), shared(0),
          tokens(0) {}

    // The tokens from tb on, before t1. All of the tile's loads are issued first,
    // as far as the registers go: they come from HBM, and a tile is short.
    __device__ __forceinline__ void fill(const BalanceParams& bp, int64_t tb, int64_t t1) {
        const int lane = lane_id(), K = bp.K, ld = K | 1;
        const int entries = (int)(t1 - tb < 64 ? t1 - tb : 64) * K;
        const int* const ids = bp.eids + (size_t)tb * K;
        const float* const wts = bp.wts + (size_t)tb * K;
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
        const int nres = bp.nres[tc], b = bp.blocks ? bp.nsh[tc] : 0;
        const bool ok = (bp.valid == nullptr || bp.valid[tc] != 0) && t < t1;
        for (int i = lane; i < 64 * ld; i += kWave) p[i] = 0.f;
        unit[lane] = bp.blocks ? bp.B - b : 1;
        chosen[lane] = ok ? min(nres, K) : -1;
        shared = ok ? (bp.blocks ? b : 1) : 0;
        tokens = ok ? 1 : 0;
        wave_sync();
        int q = lane / K, r = lane - q * K;         // token and rank of entry `lane`
        const int dq = kWave / K, dr = kWave - dq * K;
        for (int i0 = lane; i0 < entries; i0 += kBalBatch * kWave) {
            if (i0 != lane) fetch(i0);
#pragma unroll
            for (int c = 0; c < kBalBatch; ++c) {
                const bool on = i0 + c * kWave < entries;
                if (on && e[c] >= 1 && e[c] <= K && chosen[q] >= 0)
                    p[q * ld + e[c] - 1] =
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
    }

    // dl of the tile's tokens: a lane sums its token's mean slope, then the rows
    // leave side by side.
    __device__ __forceinline__ void write_dl(const BalanceParams& bp, int64_t tb, int64_t t1, const float* slope) {
        const int lane = lane_id(), K = bp.K, ld = K | 1, quads = bp.KP / 4;
        float* const mean = reinterpret_cast<float*>(unit);
        float m = 0.f;
#pragma unroll 8
        for (int j = 0; j < K; ++j) m = fmaf(fabsf(p[lane * ld + j]), slope[j], m);
        wave_sync();
        mean[lane] = m;
        wave_sync();
        const int rows = (int)(t1 - tb < 64 ? t1 - tb : 64);
        for (int i = lane; i < rows * quads; i += kWave) {
            const int q = i / quads, j = 4 * (i - q * quads);
            f32x4 o;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int jc = min(j + c, K - 1);
                const float v = fabsf(p[q * ld + jc]) * (slope[jc] - mean[q]);
                o[c] = j + c < K ? v : 0.f;
            }
            *reinterpret_cast<f32x4*>(bp.dl + (size_t)tb * bp.KP + 4 * (size_t)i) = o;
        }
        wave_sync();
    }
};

// Loads and affinity sums of one piece of a group per workgroup: lane j + w h adds
// expert j's entries of the h-th of 64 / w runs of a tile's tokens, w the experts
// rounded up to a power of two. A group of one piece is finished here, with its dl.
// Latency bound: 50,432 tokens, K = 16: 8.8 us, 0.8 TB/s (entry by entry and token
// by token it took 46).
__global__ __launch_bounds__(kWave* kBalWaves) void balance_count_kernel(BalanceParams p) {
    extern __shared__ float lds[];
    __shared__ double masses[kBalWaves][kWave];
    __shared__ int loads[kBalWaves][kWave + 2];
    __shared__ float slope[kWave];
    const int w = (int)threadIdx.x >> 6, nw = (int)blockDim.x >> 6, lane = lane_id(), K = p.K, ld = K | 1;
    BalTile tile(lds, w, K);
    const int64_t u = (int64_t)flat_block();
    if (u >= (int64_t)p.groups * p.pieces) return;
    const int64_t g = u / p.pieces, g0 = g * p.group, g1 = g0 + p.group < p.N ? g0 + p.group : p.N;
    const int64_t t0 = g0 + (u - g * p.pieces) * p.piece, t1 = t0 + p.piece < g1 ? t0 + p.piece : g1;
    const int wide = K <= 1 ? 1 : 1 << (32 - __builtin_clz(K - 1));
    const int j = lane & (wide - 1), h = lane / wide, run = wide;   // 64 / (64 / wide) tokens per run
    double mass = 0.0;
    int load = 0, shared = 0, tokens = 0;
    for (int64_t tb = t0 + 64 * w; tb < t1; tb += 64 * nw) {
        tile.fill(p, tb, t1);
        shared += tile.shared;
        tokens += tile.tokens;
        if (j < K) {
            float m = 0.f;
#pragma unroll 8
            for (int i = 0; i < run; ++i) {
                const uint32_t v = __float_as_uint(tile.p[(h * run + i) * ld + j]);
                m += __uint_as_float(v & 0x7fffffffu);
                load += (v >> 31) ? tile.unit[h * run + i] : 0;
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
    if (w == 0) {
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
            balance_finish_group(p, g, m, l, s, n, true, slope);
        } else {
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
    }
    if (p.pieces > 1 || p.dl == nullptr) return;
    __syncthreads();
    const bool again = t1 - t0 > 64 * nw;   // the tile in LDS is not the only one
    for (int64_t tb = t0 + 64 * w; tb < t1; tb += 64 * nw) {
        if (again) tile.fill(p, tb, t1);
        tile.write_dl(p, tb, t1, slope);
    }
}

// Groups of several pieces: every workgroup adds its group's pieces, a thread per
// word of a piece's sums and stretch of the pieces (the stretches in order), and
// then forms dl of its own piece; the first piece's writes the group's results
// (with no gradients wanted there is no other). Latency bound: 50,432 tokens, K = 16
// 9.7 us, 131,072, K = 32 22 (loading the first tile beside the sums: 10.4 and 24).
constexpr int kBalStretches = 32;
__global__ __launch_bounds__(kWave* kBalWaves) void balance_slope_kernel(BalanceParams p) {
    extern __shared__ float lds[];
    __shared__ uint64_t stretch[kWave * kBalWaves];
    __shared__ uint64_t total[2 * kWave + 2];
    __shared__ float slope[kWave];
    const int here = p.dl != nullptr ? p.pieces : 1;   // workgroups per group
    const int64_t u = (int64_t)flat_block();
    if (u >= (int64_t)p.groups * here) return;
    const int64_t g = u / here;
    const int K = p.K, words = 2 * K + 2, wide = 1 << (32 - __builtin_clz(words - 1)), tid = (int)threadIdx.x;
    const int n = min(kWave * kBalWaves / wide, kBalStretches), h = tid / wide, c = tid % wide, w = tid >> 6;
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
        stretch[tid] = c < K ? __builtin_bit_cast(uint64_t, m) : l;
    }
    __syncthreads();
    if (tid < words) {
        double m = 0.0;
        uint64_t l = 0;
        for (int i = 0; i < n; ++i) {
            m += __builtin_bit_cast(double, stretch[i * wide + tid]);
            l += stretch[i * wide + tid];
        }
        total[tid] = tid < K ? __builtin_bit_cast(uint64_t, m) : l;
    }
    __syncthreads();
    if (w == 0) {
        const int j = min(tid, K - 1);
        const bool on = tid < K;
        balance_finish_group(p, g, on ? __builtin_bit_cast(double, total[j]) : 0.0, on ? (int64_t)total[K + j] : 0,
                             (int64_t)total[2 * K], (int64_t)total[2 * K + 1], u == g * here, slope);
    }
    if (p.dl == nullptr) return;
    __syncthreads();
    const int64_t g0 = g * p.group, g1 = g0 + p.group < p.N ? g0 + p.group : p.N;
    const int64_t t0 = g0 + (u - g * here) * p.piece, t1 = t0 + p.piece < g1 ? t0 + p.piece : g1;
    BalTile tile(lds, w, K);
    for (int64_t tb = t0 + 64 * w; tb < t1; tb += 64 * kBalWaves) {
        tile.fill(p, tb, t1);
        tile.write_dl(p, tb, t1, slope);
    }
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
// columns each and work apart, lane l the NC consecutive columns from 16-lane
// column l % 16 on, so that one load gives a lane its operand of NC products
// (product i stands for every NC-th column): for v_mfma_f32_16x16x4_f32, X[t + l /
// 16] is the right operand of dl^T X and W_j the one of dl W, whose sums dX_in is
// added to. The experts are dealt to the products' rows and steps so that a lane's
// values of dl lie side by side: row l % 16 of tile kt of dl^T X is expert KT (l %
// 16) + kt, step kk of dl W takes expert 4 KT (l / 16) + kk from lane l. The
// router's rows and the sums of dl^T X stay in registers.
//
// All of the next step's loads are issued between the two products, without a
// branch (a step past the range re-reads the last, rows past the last token the
// last row), and the stores come last: the waits at the next step then name loads
// a whole product old. (The flags of padded tokens loaded ahead of the first product
// instead: 50,000 x 1,024, K = 64, half of them padded, 209 -> 229 us.) Padded tokens
// have dl = 0, their rows of X are not used, and their rows of dX take no product.
// HBM bound: 50,432 x 768 bf16, K = 16 84 us, 4.6 TB/s of 10 bytes an element;
// 131,072 x 1,024, K = 32 279 to 288 us, 4.7 TB/s, the matrix cores busy 40% of it at 153
// TFLOP/s. Past 48 experts the products take as long as the memory (50,000 x 1,024,
// K = 64 175 us against 100), and where dX is added or one gradient is wanted alone the
// kernel spills 12 to 22 registers. The router in LDS and a third wave per SIMD instead:
// 283 -> 345 us; 8 columns a lane: 372 -> 408 in an earlier form.
template <class T, int NC>
struct BalRow {
    typedef T mem __attribute__((ext_vector_type(NC), aligned(sizeof(T))));
};
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(u16 v) { return bf2f(v); }

// Waves that a compute unit holds, by their registers, and the most of a workgroup.
__host__ __device__ constexpr int balance_waves(int K) { return K <= 16 ? 12 : 8; }
constexpr int kBalStrips = 4;

// WHAT 0: by p.dX, p.dX_in and p.dW; 1: all three; 2: dX written and dW.
template <class T, int KT, int NC, int WHAT>
__global__ __launch_bounds__(kBalStrips * kWave, balance_waves(16 * KT) / 4) void balance_grad_kernel(BalanceParams p) {
    constexpr int KP = 16 * KT;
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
    const bool want_x = WHAT != 0 || p.dX != nullptr, want_w = WHAT != 0 || p.dW != nullptr;
    const bool add = WHAT == 1 || (WHAT == 0 && p.dX_in != nullptr), check = p.valid != nullptr;
    // This lane's columns: from col on, loaded from at (the row's last NC where
    // fewer are left); columns before col belong to other lanes, which write them.
    const int col = (((int)blockIdx.y * nw + w) * 16 + lr) * NC;
    const uint32_t at = (uint32_t)min(col, p.d - NC);
    const int own = (int)at >= col ? 0 : min(col - (int)at, NC);   // first own element (NC: none)
    const int64_t first = (int64_t)blockIdx.x * p.steps * 16;
    const int64_t end = first + p.steps * 16 < p.N ? first + p.steps * 16 : p.N;

    f_raw W[4 * KT];
#pragma unroll
    for (int kk = 0; kk < 4 * KT; ++kk) {
        const int j = 4 * KT * lq + kk;
        W[kk] = f_raw{};
        if (want_x && j < K) W[kk] = *reinterpret_cast<const f_mem*>(p.Wr + (size_t)(j + 1) * p.d + at);
    }
    f32x4 dW[KT][NC];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < NC; ++i) dW[kt][i] = f32x4{0.f, 0.f, 0.f, 0.f};

    x_raw x[4];              // rows t + 4 q + lq of X
    float al[4][KT];         // dl of those tokens, this lane's experts of dl^T X
    f_raw s[4], sn[4];       // rows t + 4 lq + r of dX_in
    f32x4 ar[KT], an[KT];    // dl of token t + lr, this lane's experts of dl W
    uint32_t flag = 1;       // token t + lr is real
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = sn[r] = f_raw{};
    // A step's rows have a scalar base and a lane's 32-bit offset, in elements of a
    // row of d; fixed by clamping where the step reaches past the last token.
    auto rows_x = [&](int64_t t) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t row = t + 4 * q < p.N ? t + 4 * q : p.N - 1;
            uint32_t k = (uint32_t)lq;
            if (t + 16 > p.N) k = (uint32_t)min((int64_t)lq, p.N - 1 - row);
            x[q] = *reinterpret_cast<const x_mem*>(static_cast<const char*>(p.X) + (size_t)row * p.d * sizeof(T) +
                                                   (k * p.d + at) * (uint32_t)sizeof(T));
            const float* const dl = reinterpret_cast<const float*>(reinterpret_cast<const char*>(p.dl + (size_t)row * KP) +
                                                                   (k * KP + (uint32_t)lr * KT) * 4u);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) al[q][kt] = dl[kt];
        }
    };
    auto rows_flag = [&](int64_t t) {
        if (check) flag = p.valid[t + lr < p.N ? t + lr : p.N - 1];
    };
    auto rows_s = [&](int64_t t, f_raw (&so)[4], f32x4 (&ao)[KT]) {
        if (add)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t row = t + r < p.N ? t + r : p.N - 1;
                uint32_t k = (uint32_t)lq * 4;
                if (t + 16 > p.N) k = (uint32_t)min((int64_t)lq * 4, p.N - 1 - row);
                so[r] = *reinterpret_cast<const f_mem*>(reinterpret_cast<const char*>(p.dX_in) + (size_t)row * p.d * 4 +
                                                        (k * p.d + at) * 4u);
            }
        uint32_t k = (uint32_t)lr;
        if (t + 16 > p.N) k = (uint32_t)min((int64_t)lr, p.N - 1 - t);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
            ao[kt] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const char*>(p.dl + (size_t)t * KP) +
                                                     (k * KP + (uint32_t)lq * 4 * KT + 4 * kt) * 4u);
    };
    if (want_w) rows_x(first);
    rows_flag(first);
    if (want_x) rows_s(first, s, ar);
    for (int64_t t = first; t < end; t += 16) {
        const int64_t next = t + 16 < end ? t + 16 : t;
        uint32_t mask = 0xffffu;   // the step's real tokens
        if (check) mask = (uint32_t)ballot(flag != 0) & 0xffffu;
        if (t + 16 > end) mask &= (1u << (int)(end - t)) - 1;
        if (want_w) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float b[NC];
#pragma unroll
                for (int i = 0; i < NC; ++i) b[i] = to_f32(x[q][i]);
                if (mask != 0xffffu) {
                    const bool on = mask >> (4 * q + lq) & 1;
#pragma unroll
                    for (int i = 0; i < NC; ++i) b[i] = on ? b[i] : 0.f;
                }
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < NC; ++i)
                        dW[kt][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(al[q][kt], b[i], dW[kt][i], 0, 0, 0);
            }
            rows_x(next);
        }
        rows_flag(next);
        if (want_x) {
            rows_s(next, sn, an);
            f32x4 acc[NC];
#pragma unroll
            for (int i = 0; i < NC; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < 4 * KT; ++kk)
#pragma unroll
                for (int i = 0; i < NC; ++i)
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(ar[kk / 4][kk % 4], W[kk][i], acc[i], 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f_raw v;   // dX_in is added last: one rounding at its magnitude
#pragma unroll
                for (int i = 0; i < NC; ++i) v[i] = s[r][i] + acc[i][r];
                if (mask != 0xffffu && !(mask >> (4 * lq + r) & 1)) v = s[r];   // whatever the router's rows hold
                if (t + 4 * lq + r < end) {
                    char* const out = reinterpret_cast<char*>(p.dX) + (size_t)(t + r) * p.d * 4 + ((uint32_t)lq * 4 * p.d + at) * 4u;
                    if (own == 0 && p.past) __builtin_nontemporal_store(v, reinterpret_cast<f_mem*>(out));
                    else if (own == 0) *reinterpret_cast<f_mem*>(out) = v;
                    else
#pragma unroll
                        for (int i = 0; i < NC; ++i)
                            if (i >= own) reinterpret_cast<float*>(out)[i] = v[i];
                }
                s[r] = sn[r];
            }
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) ar[kt] = an[kt];
        }
    }
    if (!want_w) return;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = (4 * lq + r) * KT + kt;
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
