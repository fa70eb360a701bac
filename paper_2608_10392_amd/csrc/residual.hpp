// The join of a block's branch with the residual stream and the norm in front
// of the next block, v = s x + g N_out(f), y = v, h = N_in(v), and its backward.
//
// Both directions read every element once and keep a token's whole row in
// registers: a team of lanes holds the row, each lane E consecutive columns per
// chunk, so that the statistics (two passes over registers: the mean, then the
// squares of the centred values, which neither an offset nor an outlier
// cancels), the norm and its gradient need no second read. HBM bounds them.
#pragma once
#include "common.hpp"

namespace unifmoe {

constexpr int kNormNone = 0, kNormLayer = 1, kNormRms = 2;

struct ResidualParams {
    int N, d;
    int rows;                  // consecutive tokens per team
    int out_norm, in_norm;
    int group;                 // tokens per gate row (N where one row serves all)
    float out_eps, in_eps, scale, inv_d;
    const float* out_gamma;
    const float* out_beta;
    const float* in_gamma;
    const float* in_beta;
    const float* gate;
    const uint8_t* valid;
    const void* x;             // forward: x; backward: y
    const void* f;
    void* y;
    void* h;
    // backward
    const void* dy;
    const void* dh;
    void* dx;
    void* df;
    float* part;               // [5][workgroups][d]: out_gamma, out_beta, in_gamma, in_beta, gate
    float* gate_part;          // [teams][2][d]: a team's first and last piece of gate groups it shares
    float* dgate;              // [groups][d]: groups that one team holds (NULL: not wanted)
    int want;                  // bit i: parameter i of `part` is wanted
};

typedef u16 u16x8_a2 __attribute__((ext_vector_type(8), aligned(2)));

// E consecutive elements of a row from column c on, as floats; columns past d
// read as 0. Rows start at any element, so the vector loads assume no more
// than the element's alignment.
template <int E>
__device__ __forceinline__ void ld_cols(const float* row, int c, int d, float (&v)[E]) {
    static_assert(E % 4 == 0, "whole vectors");
    if (c + E <= d) {
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            const f32x4 w = ld_f32x4(row + c + 4 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = w[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = c + e < d ? row[c + e] : 0.f;
    }
}
template <int E>
__device__ __forceinline__ void ld_cols(const u16* row, int c, int d, float (&v)[E]) {
    static_assert(E == 8, "one 16-byte vector");
    if (c + E <= d) {
        const u16x8_a2 w = *reinterpret_cast<const u16x8_a2*>(row + c);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = bf2f(w[e]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = c + e < d ? bf2f(row[c + e]) : 0.f;
    }
}

typedef float f32x4_s4 __attribute__((ext_vector_type(4), aligned(4)));
template <int E>
__device__ __forceinline__ void st_cols(float* row, int c, int d, const float (&v)[E]) {
    if (c + E <= d) {
#pragma unroll
        for (int q = 0; q < E / 4; ++q)
            *reinterpret_cast<f32x4_s4*>(row + c + 4 * q) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < d) row[c + e] = v[e];
    }
}
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
template <int E>
__device__ __forceinline__ void st_cols(u16* row, int c, int d, const float (&v)[E]) {
    static_assert(E == 8, "one 16-byte vector");
    if (c + E <= d) {
        u32x4 w;
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = pack_bf16x2(v[2 * q], v[2 * q + 1]);
        *reinterpret_cast<u32x4_a2*>(row + c) = w;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < d) row[c + e] = f2bf(v[e]);
    }
}

// A parameter row, or `other` where there is none.
template <int E>
__device__ __forceinline__ void ld_param(const float* p, int c, int d, float other, float (&v)[E]) {
    if (p != nullptr) {
        ld_cols<E>(p, c, d, v);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = other;
    }
}

// The lanes that hold one row: LPR lanes of a wave, or (LPR = 0) all waves of
// the workgroup. Sums over them end in every lane, the lanes added by a
// butterfly, the waves in order.
template <int LPR>
struct Team {
    static constexpr bool kWide = LPR == 0;
    static constexpr int kLanes = kWide ? kWave : LPR;
    float* red;   // [2][waves][4], wide teams only
    int phase;
    __device__ __forceinline__ int size() const { return kWide ? (int)blockDim.x : LPR; }
    __device__ __forceinline__ int sub() const { return kWide ? (int)threadIdx.x : (int)threadIdx.x % kLanes; }
    __device__ __forceinline__ int index() const {
        return kWide ? (int)blockIdx.x : (int)((blockIdx.x * blockDim.x + threadIdx.x) / kLanes);
    }
    template <int NV>
    __device__ __forceinline__ void sum(float (&v)[NV]) {
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] += __shfl_xor(v[i], o);
        if constexpr (kWide) {
            const int nw = (int)blockDim.x >> 6, w = (int)threadIdx.x >> 6;
            float* r = red + phase * nw * 4;
            phase ^= 1;
            if (lane_id() == 0)
#pragma unroll
                for (int i = 0; i < NV; ++i) r[w * 4 + i] = v[i];
            lds_barrier();
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = 0.f;
            for (int k = 0; k < nw; ++k)
#pragma unroll
                for (int i = 0; i < NV; ++i) v[i] += r[k * 4 + i];
        }
    }
};

// Replaces the row u by its normalised values (mean 0 for RMS) and returns the
// scale they were multiplied with. Columns past d stay out of the sums.
template <int E, int CH, int LPR>
__device__ __forceinline__ float normalise(Team<LPR>& team, int norm, float eps, float inv_d, int d, const int (&col)[CH],
                                           float (&u)[CH][E]) {
    if (norm == kNormLayer) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) s[0] += u[c][e];
        team.sum(s);
        const float mean = s[0] * inv_d;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) u[c][e] = col[c] + e < d ? u[c][e] - mean : 0.f;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) q[0] = fmaf(u[c][e], u[c][e], q[0]);
    team.sum(q);
    const float rstd = 1.0f / sqrtf(fmaf(q[0], inv_d, eps));
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) u[c][e] *= rstd;
    return rstd;
}

// Gradient of a norm's input: a is d loss / d (normalised row), replaced by
// rstd (a - mean(a) - hat mean(a hat)), without the first mean for RMS.
template <int E, int CH, int LPR>
__device__ __forceinline__ void normalise_grad(Team<LPR>& team, int norm, float rstd, float inv_d,
                                               const float (&hat)[CH][E], float (&a)[CH][E]) {
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            s[0] += a[c][e];
            s[1] = fmaf(a[c][e], hat[c][e], s[1]);
        }
    team.sum(s);
    const float m = norm == kNormLayer ? s[0] * inv_d : 0.f, q = s[1] * inv_d;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) a[c][e] = rstd * (fmaf(-hat[c][e], q, a[c][e]) - m);
}

template <class S, class L, int E, int CH, int LPR>
__global__ __launch_bounds__(LPR == 0 ? 512 : 256) void residual_forward_kernel(ResidualParams p) {
    __shared__ float red[2 * 8 * 4];
    Team<LPR> team{red, 0};
    int col[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) col[c] = (c * team.size() + team.sub()) * E;
    const int64_t r0 = (int64_t)team.index() * p.rows;
    const int64_t r1 = r0 + p.rows < p.N ? r0 + p.rows : p.N;
    if (r0 >= r1) return;
    float og[CH][E], ob[CH][E], ig[CH][E], ib[CH][E], gt[CH][E];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        ld_param<E>(p.out_gamma, col[c], p.d, 1.f, og[c]);
        ld_param<E>(p.out_beta, col[c], p.d, 0.f, ob[c]);
        ld_param<E>(p.in_gamma, col[c], p.d, 1.f, ig[c]);
        ld_param<E>(p.in_beta, col[c], p.d, 0.f, ib[c]);
    }
    int64_t gend = r0;   // the gate rows in registers serve the tokens before gend
    for (int64_t r = r0; r < r1; ++r) {
        if (r >= gend) {
            const int64_t g = r / p.group;
            gend = (g + 1) * p.group;
#pragma unroll
            for (int c = 0; c < CH; ++c)
                ld_param<E>(p.gate == nullptr ? nullptr : p.gate + g * p.d, col[c], p.d, 1.f, gt[c]);
        }
        const size_t at = (size_t)r * p.d;
        const bool real = p.valid == nullptr || p.valid[r] != 0;
        float v[CH][E];
        if (real) {
            if (p.f != nullptr) {
#pragma unroll
                for (int c = 0; c < CH; ++c) ld_cols<E>(static_cast<const L*>(p.f) + at, col[c], p.d, v[c]);
                if (p.out_norm != kNormNone) normalise<E, CH, LPR>(team, p.out_norm, p.out_eps, p.inv_d, p.d, col, v);
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) v[c][e] = fmaf(v[c][e], og[c][e], ob[c][e]) * gt[c][e];
            } else {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) v[c][e] = 0.f;
            }
            if (p.x != nullptr) {
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    float x[E];
                    ld_cols<E>(static_cast<const S*>(p.x) + at, col[c], p.d, x);
#pragma unroll
                    for (int e = 0; e < E; ++e) v[c][e] = fmaf(p.scale, x[e], v[c][e]);
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) v[c][e] = 0.f;
        }
        if (p.y != nullptr)
#pragma unroll
            for (int c = 0; c < CH; ++c) st_cols<E>(static_cast<S*>(p.y) + at, col[c], p.d, v[c]);
        if (p.h != nullptr) {
            if (real) {
                normalise<E, CH, LPR>(team, p.in_norm, p.in_eps, p.inv_d, p.d, col, v);
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) v[c][e] = fmaf(v[c][e], ig[c][e], ib[c][e]);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) st_cols<E>(static_cast<L*>(p.h) + at, col[c], p.d, v[c]);
        }
    }
}

// Backward: D = dy + (d N_in)^T dh; dx = s D; dn = g D; df = (d N_out)^T dn. The
// parameters' gradients are sums over the tokens: a team keeps its columns'
// sums in registers for its consecutive tokens, a workgroup adds its teams' and
// writes one partial row per parameter (residual_param_sum_kernel adds those).
// A gate with several rows: a team that reaches the end of a gate's tokens
// writes the sum, straight to the gradient where it held all of them, else as
// its first or last piece (residual_gate_join_kernel).
template <class S, class L, class H, int E, int CH, int LPR>
__global__ __launch_bounds__(LPR == 0 ? 512 : 256) void residual_backward_kernel(ResidualParams p) {
    __shared__ float red[2 * 8 * 4];
    extern __shared__ float sums[];   // [teams of the workgroup][d]
    Team<LPR> team{red, 0};
    int col[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) col[c] = (c * team.size() + team.sub()) * E;
    const int64_t r0 = (int64_t)team.index() * p.rows;
    const int64_t r1 = r0 + p.rows < p.N ? r0 + p.rows : p.N;
    float acc[5][CH][E];
#pragma unroll
    for (int i = 0; i < 5; ++i)
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[i][c][e] = 0.f;
    float og[CH][E], ob[CH][E], ig[CH][E], gt[CH][E];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        ld_param<E>(p.out_gamma, col[c], p.d, 1.f, og[c]);
        ld_param<E>(p.out_beta, col[c], p.d, 0.f, ob[c]);
        ld_param<E>(p.in_gamma, col[c], p.d, 1.f, ig[c]);
    }
    const bool grouped = p.dgate != nullptr;
    int64_t g = -1, gend = r0;
    auto flush = [&]() {
        const int64_t g0 = g * p.group, g1 = gend < p.N ? gend : p.N;
        float* dst = (g0 >= r0 && g1 <= r1) ? p.dgate + g * p.d
                                            : p.gate_part + ((size_t)team.index() * 2 + (g0 > r0 ? 1 : 0)) * p.d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            st_cols<E>(dst, col[c], p.d, acc[4][c]);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[4][c][e] = 0.f;
        }
    };
    for (int64_t r = r0; r < r1; ++r) {
        if (r >= gend) {
            if (grouped && g >= 0) flush();
            g = r / p.group;
            gend = (g + 1) * p.group;
#pragma unroll
            for (int c = 0; c < CH; ++c)
                ld_param<E>(p.gate == nullptr ? nullptr : p.gate + g * p.d, col[c], p.d, 1.f, gt[c]);
        }
        const size_t at = (size_t)r * p.d;
        const bool real = p.valid == nullptr || p.valid[r] != 0;
        float D[CH][E];
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) D[c][e] = 0.f;
        if (real && p.dh != nullptr) {
            float u[CH][E];
#pragma unroll
            for (int c = 0; c < CH; ++c) ld_cols<E>(static_cast<const S*>(p.x) + at, col[c], p.d, u[c]);
            const float rstd = normalise<E, CH, LPR>(team, p.in_norm, p.in_eps, p.inv_d, p.d, col, u);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                ld_cols<E>(static_cast<const H*>(p.dh) + at, col[c], p.d, D[c]);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    acc[2][c][e] = fmaf(D[c][e], u[c][e], acc[2][c][e]);
                    acc[3][c][e] += D[c][e];
                    D[c][e] *= ig[c][e];
                }
            }
            normalise_grad<E, CH, LPR>(team, p.in_norm, rstd, p.inv_d, u, D);
        }
        if (real && p.dy != nullptr) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float y[E];
                ld_cols<E>(static_cast<const S*>(p.dy) + at, col[c], p.d, y);
#pragma unroll
                for (int e = 0; e < E; ++e) D[c][e] += y[e];
            }
        }
        if (p.dx != nullptr) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float o[E];
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = p.scale * D[c][e];
                st_cols<E>(static_cast<S*>(p.dx) + at, col[c], p.d, o);
            }
        }
        if (real && p.f != nullptr) {
            float u[CH][E];
#pragma unroll
            for (int c = 0; c < CH; ++c) ld_cols<E>(static_cast<const L*>(p.f) + at, col[c], p.d, u[c]);
            float rstd = 1.f;
            if (p.out_norm != kNormNone) rstd = normalise<E, CH, LPR>(team, p.out_norm, p.out_eps, p.inv_d, p.d, col, u);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    acc[4][c][e] = fmaf(D[c][e], fmaf(u[c][e], og[c][e], ob[c][e]), acc[4][c][e]);
                    const float dn = D[c][e] * gt[c][e];
                    acc[0][c][e] = fmaf(dn, u[c][e], acc[0][c][e]);
                    acc[1][c][e] += dn;
                    D[c][e] = dn * og[c][e];
                }
            if (p.out_norm != kNormNone) normalise_grad<E, CH, LPR>(team, p.out_norm, rstd, p.inv_d, u, D);
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) D[c][e] *= gt[c][e];
        }
        if (p.df != nullptr)
#pragma unroll
            for (int c = 0; c < CH; ++c) st_cols<E>(static_cast<L*>(p.df) + at, col[c], p.d, D[c]);
    }
    if (grouped && g >= 0) flush();
    const int nteam = (int)blockDim.x / team.size(), me = Team<LPR>::kWide ? 0 : (int)threadIdx.x / Team<LPR>::kLanes;
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        if (!(p.want >> i & 1)) continue;
        float* const dst = p.part + ((size_t)i * gridDim.x + blockIdx.x) * p.d;
        if constexpr (Team<LPR>::kWide) {
#pragma unroll
            for (int c = 0; c < CH; ++c) st_cols<E>(dst, col[c], p.d, acc[i][c]);
        } else {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CH; ++c) st_cols<E>(sums + me * p.d, col[c], p.d, acc[i][c]);
            __syncthreads();
            for (int n = threadIdx.x; n < p.d; n += blockDim.x) {
                float s = 0.f;
                for (int k = 0; k < nteam; ++k) s += sums[k * p.d + n];
                dst[n] = s;
            }
        }
    }
}

struct ResidualSums {
    int d, parts;
    const float* part;   // [5][parts][d]
    float* out[5];       // NULL: not wanted
};

// Parameter blockIdx.y's gradient: 64 columns per workgroup, four waves a
// quarter of the partial rows each, added in order in fp64.
__global__ __launch_bounds__(256) void residual_param_sum_kernel(ResidualSums p) {
    __shared__ double quarter[4][64];
    float* const out = p.out[blockIdx.y];
    if (out == nullptr) return;
    const int lane = lane_id(), w = (int)threadIdx.x >> 6, n = (int)blockIdx.x * 64 + lane;
    const int k0 = (int)((int64_t)w * p.parts / 4), k1 = (int)((int64_t)(w + 1) * p.parts / 4);
    double s = 0.0;
    if (n < p.d)
        for (int k = k0; k < k1; ++k) s += (double)p.part[((size_t)blockIdx.y * p.parts + k) * p.d + n];
    quarter[w][lane] = s;
    __syncthreads();
    if (w == 0 && n < p.d) out[n] = (float)(((quarter[0][lane] + quarter[1][lane]) + quarter[2][lane]) + quarter[3][lane]);
}

struct ResidualGates {
    int N, d, group, rows;
    const float* gate_part;   // [teams][2][d]
    float* dgate;
};

// Gate groups that several teams share: workgroup (x, t - 1) takes the group
// that reaches over the end of team t - 1's tokens, if that is the first such
// end in it, and adds its pieces in order. A team's piece is its first where
// the group holds the team's first token, else its last.
__global__ __launch_bounds__(256) void residual_gate_join_kernel(ResidualGates p) {
    const int64_t t = (int64_t)blockIdx.y + 1, b = t * p.rows;
    const int64_t g = b / p.group, g0 = g * p.group;
    if (b >= p.N || g0 == b || b - p.rows > g0) return;
    const int64_t g1 = g0 + p.group < p.N ? g0 + p.group : p.N;
    const int64_t last = (g1 - 1) / p.rows;
    const int n = (int)(blockIdx.x * blockDim.x + threadIdx.x);
    if (n >= p.d) return;
    double s = (double)p.gate_part[((size_t)(t - 1) * 2 + (g0 > (t - 1) * p.rows ? 1 : 0)) * p.d + n];
    for (int64_t k = t; k <= last; ++k) s += (double)p.gate_part[(size_t)k * 2 * p.d + n];
    p.dgate[(size_t)g * p.d + n] = (float)s;
}

}  // namespace unifmoe
