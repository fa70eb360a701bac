// The join of a block's branch with the residual stream and the norm in front
// of the next block, v = s x + g N_out(f), y = v, h = N_in(v), and its backward.
//
// Both directions read every element once and keep a token's whole row in
// registers: a team of lanes holds the row, each lane E consecutive columns per
// chunk, so that the statistics (two passes over registers: the mean, then the
// squares of the centred values, which neither an offset nor an outlier
// cancels), the norm and its gradient need no second read. HBM bounds them. A
// team works through consecutive tokens, with the next token's loads in flight
// while it computes.
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
    float* part;               // [4][workgroups][d] partial sums (kSum*)
    float* gate_part;          // [teams][2][d]: a team's first and last piece of gate groups it shares
    float* dgate;              // [groups][d]: groups that one team holds (NULL: one gate row, or not wanted)
    int grouped;               // the gate has several rows
    int want;                  // bit i: partial sum i is wanted
};

// E consecutive elements of a row from column c on, E = 4; columns past d read
// as 0. Rows start at any element, so the vector accesses assume no more than
// the element's alignment.
constexpr int E = 4;
typedef u16 u16x4 __attribute__((ext_vector_type(4)));
typedef u16 u16x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
template <class T>
struct Vec;
template <>
struct Vec<float> {
    typedef f32x4 raw;
    typedef f32x4_a4 mem;
    static __device__ __forceinline__ float get(raw v, int e) { return v[e]; }
    static __device__ __forceinline__ raw pack(const float (&v)[E]) { return raw{v[0], v[1], v[2], v[3]}; }
};
template <>
struct Vec<u16> {
    typedef u16x4 raw;
    typedef u16x4_a2 mem;
    static __device__ __forceinline__ float get(raw v, int e) { return bf2f(v[e]); }
    static __device__ __forceinline__ raw pack(const float (&v)[E]) {
        return __builtin_bit_cast(raw, uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])});
    }
};
template <class T>
__device__ __forceinline__ typename Vec<T>::raw ld_raw(const T* row, int c, int d) {
    typename Vec<T>::raw v = {};
    if (c + E <= d) {
        v = *reinterpret_cast<const typename Vec<T>::mem*>(row + c);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < d) v[e] = row[c + e];
    }
    return v;
}
template <class T>
__device__ __forceinline__ void st_cols(T* row, int c, int d, const float (&v)[E]) {
    const typename Vec<T>::raw w = Vec<T>::pack(v);
    if (c + E <= d) {
        *reinterpret_cast<typename Vec<T>::mem*>(row + c) = w;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < d) row[c + e] = w[e];
    }
}

// A parameter row, or `other` where there is none.
__device__ __forceinline__ void ld_param(const float* p, int c, int d, float other, float (&v)[E]) {
    if (p != nullptr) {
        const f32x4 w = ld_raw(p, c, d);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = w[e];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = other;
    }
}

// v plus its value in the lane that the DPP control names.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Sum over the LPR consecutive lanes (a power of two, 8 to 64) that hold v, in
// all of them: quads (quad_perm [1,0,3,2], [2,3,0,1]), then mirrored halves and
// rows of 16 (every lane of a quad, a half already holds its sum), then the
// swapped rows and halves of the wave. No LDS.
template <int LPR>
__device__ __forceinline__ float lanes_sum(float v) {
    v = dpp_add<0xB1>(v);
    v = dpp_add<0x4E>(v);
    v = dpp_add<0x141>(v);
    if constexpr (LPR >= 16) v = dpp_add<0x140>(v);
    if constexpr (LPR >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (LPR >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// The lanes that hold one row: LPR lanes of a wave, or (LPR = 0) all waves of
// the workgroup, whose sums are added in order.
constexpr int kWideWaves = 8;   // most waves of a wide team
template <int LPR>
struct Team {
    static constexpr bool kWide = LPR == 0;
    static constexpr int kLanes = kWide ? kWave : LPR;
    float* red;   // [2][kWideWaves][4], wide teams only: rounds alternate, so that one barrier each suffices
    int phase;
    __device__ __forceinline__ int size() const { return kWide ? (int)blockDim.x : LPR; }
    __device__ __forceinline__ int sub() const { return kWide ? (int)threadIdx.x : (int)threadIdx.x % kLanes; }
    __device__ __forceinline__ int local() const { return kWide ? 0 : (int)threadIdx.x / kLanes; }
    __device__ __forceinline__ int index() const {
        return kWide ? (int)blockIdx.x : (int)((blockIdx.x * blockDim.x + threadIdx.x) / kLanes);
    }
    template <int NV>
    __device__ __forceinline__ void sum(float (&v)[NV]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = lanes_sum<kLanes>(v[i]);
        if constexpr (kWide) {
            const int nw = (int)blockDim.x >> 6, w = (int)threadIdx.x >> 6;
            float* const r = red + phase * kWideWaves * 4;
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

#define UNIF_COLS(c, e)            \
    _Pragma("unroll") for (int c = 0; c < CH; ++c) _Pragma("unroll") for (int e = 0; e < E; ++e)

template <class T, int CH>
struct RowRaw {
    typename Vec<T>::raw v[CH];
    __device__ __forceinline__ void load(const void* p, size_t at, const int (&col)[CH], int d, bool on) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (on && p != nullptr) v[c] = ld_raw(static_cast<const T*>(p) + at, col[c], d);
            else v[c] = typename Vec<T>::raw{};
        }
    }
    __device__ __forceinline__ void get(float (&u)[CH][E]) const { UNIF_COLS(c, e) u[c][e] = Vec<T>::get(v[c], e); }
};

template <int CH>
__device__ __forceinline__ float row_sum(const float (&u)[CH][E]) {
    float s = 0.f;
    UNIF_COLS(c, e) s += u[c][e];
    return s;
}
template <int CH>
__device__ __forceinline__ float row_dot(const float (&a)[CH][E], const float (&b)[CH][E]) {
    float s = 0.f;
    UNIF_COLS(c, e) s = fmaf(a[c][e], b[c][e], s);
    return s;
}
template <int CH>
__device__ __forceinline__ void centre(float mean, int d, const int (&col)[CH], float (&u)[CH][E]) {
    UNIF_COLS(c, e) u[c][e] = col[c] + e < d ? u[c][e] - mean : 0.f;   // columns past d stay out of the sums
}

// Replaces the row u by its normalised values.
template <int CH, int LPR>
__device__ __forceinline__ void normalise(Team<LPR>& team, int norm, float eps, float inv_d, int d,
                                          const int (&col)[CH], float (&u)[CH][E]) {
    if (norm == kNormLayer) {
        float s[1] = {row_sum<CH>(u)};
        team.sum(s);
        centre<CH>(s[0] * inv_d, d, col, u);
    }
    float q[1] = {row_dot<CH>(u, u)};
    team.sum(q);
    const float rstd = rsqrtf(fmaf(q[0], inv_d, eps));
    UNIF_COLS(c, e) u[c][e] *= rstd;
}

// Gradient of a norm's input: a is d loss / d (normalised row), replaced by
// rstd (a - mean(a) - hat mean(a hat)), without the first mean for RMS.
template <int CH, int LPR>
__device__ __forceinline__ void normalise_grad(Team<LPR>& team, int norm, float rstd, float inv_d,
                                               const float (&hat)[CH][E], float (&a)[CH][E]) {
    float s[2] = {row_sum<CH>(a), row_dot<CH>(a, hat)};
    team.sum(s);
    const float m = norm == kNormLayer ? s[0] * inv_d : 0.f, q = s[1] * inv_d;
    UNIF_COLS(c, e) a[c][e] = rstd * (fmaf(-hat[c][e], q, a[c][e]) - m);
}

template <class S, class L, int CH, int LPR>
__global__ __launch_bounds__(LPR == 0 ? 512 : 256) void residual_forward_kernel(ResidualParams p) {
    __shared__ float red[2 * kWideWaves * 4];
    Team<LPR> team{red, 0};
    int col[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) col[c] = (c * team.size() + team.sub()) * E;
    const int64_t r0 = (int64_t)team.index() * p.rows;
    const int64_t r1 = r0 + p.rows < p.N ? r0 + p.rows : p.N;
    if (r0 >= r1) return;
    auto is_real = [&](int64_t r) { return r < r1 && (p.valid == nullptr || p.valid[r] != 0); };
    RowRaw<S, CH> xr;
    RowRaw<L, CH> fr;
    bool real = is_real(r0), next = is_real(r0 + 1);
    xr.load(p.x, (size_t)r0 * p.d, col, p.d, real);
    fr.load(p.f, (size_t)r0 * p.d, col, p.d, real);
    // v = s x + cg f_hat + cb with cg = gate gamma_out, cb = gate beta_out
    float cg[CH][E], cb[CH][E], ig[CH][E], ib[CH][E];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        ld_param(p.in_gamma, col[c], p.d, 1.f, ig[c]);
        ld_param(p.in_beta, col[c], p.d, 0.f, ib[c]);
    }
    int64_t gend = r0;   // cg and cb serve the tokens before gend
    for (int64_t r = r0; r < r1; ++r) {
        if (r >= gend) {
            const int64_t g = r / p.group;
            gend = (g + 1) * p.group;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float gt[E];
                ld_param(p.gate == nullptr ? nullptr : p.gate + g * p.d, col[c], p.d, 1.f, gt);
                ld_param(p.out_gamma, col[c], p.d, 1.f, cg[c]);
                ld_param(p.out_beta, col[c], p.d, 0.f, cb[c]);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    cg[c][e] *= gt[e];
                    cb[c][e] *= gt[e];
                }
            }
        }
        const size_t at = (size_t)r * p.d;
        float v[CH][E], x[CH][E];
        fr.get(v);
        xr.get(x);
        const bool keep = real;
        real = next;
        next = is_real(r + 2);
        xr.load(p.x, at + p.d, col, p.d, real);
        fr.load(p.f, at + p.d, col, p.d, real);
        if (p.out_norm != kNormNone) normalise<CH, LPR>(team, p.out_norm, p.out_eps, p.inv_d, p.d, col, v);
        UNIF_COLS(c, e) v[c][e] = keep ? fmaf(p.scale, x[c][e], fmaf(v[c][e], cg[c][e], cb[c][e])) : 0.f;
        if (p.y != nullptr)
#pragma unroll
            for (int c = 0; c < CH; ++c) st_cols(static_cast<S*>(p.y) + at, col[c], p.d, v[c]);
        if (p.h != nullptr) {
            normalise<CH, LPR>(team, p.in_norm, p.in_eps, p.inv_d, p.d, col, v);
            UNIF_COLS(c, e) v[c][e] = keep ? fmaf(v[c][e], ig[c][e], ib[c][e]) : 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c) st_cols(static_cast<L*>(p.h) + at, col[c], p.d, v[c]);
        }
    }
}

// Backward: D = dy + (d N_in)^T dh; dx = s D; df = (d N_out)^T (g D). The
// parameters' gradients are sums over the tokens of dh, dh v_hat, D and
// D f_hat, which a lane keeps for its columns (padded rows are loaded as zeros
// and so add nothing): with them
//   d in_beta = sum dh, d in_gamma = sum dh v_hat,
//   d out_beta = sum_g g sum D, d out_gamma = sum_g g sum D f_hat,
//   d gate_g = gamma_out sum D f_hat + beta_out sum D over the gate's tokens.
// A workgroup adds its teams' sums and writes one partial row each
// (residual_finish_kernel adds those). A gate with several rows: a team that
// comes to the end of a gate row's tokens adds its two sums, times the gate, to
// its totals in LDS and writes that row's gradient, straight to the result
// where it held all of its tokens, else as its first or last piece.
constexpr int kSumOutGamma = 0, kSumOutBeta = 1, kSumInGamma = 2, kSumInBeta = 3;

template <class S, class L, class H, int CH, int LPR>
__global__ __launch_bounds__(LPR == 0 ? 512 : 256) void residual_backward_kernel(ResidualParams p) {
    __shared__ float red[2 * kWideWaves * 4];
    extern __shared__ float sums[];   // [teams of the workgroup][2][d]
    Team<LPR> team{red, 0};
    int col[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) col[c] = (c * team.size() + team.sub()) * E;
    float* const mine = sums + (size_t)team.local() * 2 * p.d;
    const int64_t r0 = (int64_t)team.index() * p.rows;
    const int64_t r1 = r0 + p.rows < p.N ? r0 + p.rows : p.N;
    auto is_real = [&](int64_t r) { return r < r1 && (p.valid == nullptr || p.valid[r] != 0); };
    RowRaw<S, CH> yr, gr;
    RowRaw<H, CH> hr;
    RowRaw<L, CH> fr;
    bool real = is_real(r0), next = is_real(r0 + 1);
    yr.load(p.x, (size_t)r0 * p.d, col, p.d, real);
    fr.load(p.f, (size_t)r0 * p.d, col, p.d, real);
    hr.load(p.dh, (size_t)r0 * p.d, col, p.d, real);
    gr.load(p.dy, (size_t)r0 * p.d, col, p.d, real);
    float acc[4][CH][E];
#pragma unroll
    for (int i = 0; i < 4; ++i) UNIF_COLS(c, e) acc[i][c][e] = 0.f;
    if (p.grouped) {
        const float zero[E] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            st_cols(mine, col[c], p.d, zero);
            st_cols(mine + p.d, col[c], p.d, zero);
        }
    }
    float ig[CH][E], cg[CH][E];   // cg = gate gamma_out
#pragma unroll
    for (int c = 0; c < CH; ++c) ld_param(p.in_gamma, col[c], p.d, 1.f, ig[c]);
    int64_t g = -1, gend = r0;
    auto flush = [&]() {
        const int64_t g0 = g * p.group, g1 = gend < p.N ? gend : p.N;
        float* const dst = (g0 >= r0 && g1 <= r1) ? p.dgate + g * p.d
                                                  : p.gate_part + ((size_t)team.index() * 2 + (g0 > r0 ? 1 : 0)) * p.d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float og[E], ob[E], gt[E], t0[E], t1[E], dg[E];
            ld_param(p.out_gamma, col[c], p.d, 1.f, og);
            ld_param(p.out_beta, col[c], p.d, 0.f, ob);
            ld_param(p.gate + g * p.d, col[c], p.d, 1.f, gt);
            ld_param(mine, col[c], p.d, 0.f, t0);
            ld_param(mine + p.d, col[c], p.d, 0.f, t1);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                dg[e] = fmaf(og[e], acc[kSumOutGamma][c][e], ob[e] * acc[kSumOutBeta][c][e]);
                t0[e] = fmaf(gt[e], acc[kSumOutGamma][c][e], t0[e]);
                t1[e] = fmaf(gt[e], acc[kSumOutBeta][c][e], t1[e]);
                acc[kSumOutGamma][c][e] = acc[kSumOutBeta][c][e] = 0.f;
            }
            if (p.dgate != nullptr) st_cols(dst, col[c], p.d, dg);
            st_cols(mine, col[c], p.d, t0);
            st_cols(mine + p.d, col[c], p.d, t1);
        }
    };
    const float mask_in = p.in_norm == kNormLayer ? p.inv_d : 0.f, mask_out = p.out_norm == kNormLayer ? p.inv_d : 0.f;
    for (int64_t r = r0; r < r1; ++r) {
        if (r >= gend) {
            if (p.grouped && g >= 0) flush();
            g = r / p.group;
            gend = (g + 1) * p.group;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float gt[E];
                ld_param(p.gate == nullptr ? nullptr : p.gate + g * p.d, col[c], p.d, 1.f, gt);
                ld_param(p.out_gamma, col[c], p.d, 1.f, cg[c]);
#pragma unroll
                for (int e = 0; e < E; ++e) cg[c][e] *= gt[e];
            }
        }
        // Each tensor's next row is loaded as soon as this one's is in use.
        const size_t at = (size_t)r * p.d;
        float y[CH][E], D[CH][E], f[CH][E];
        yr.get(y);
        fr.get(f);
        real = next;
        next = is_real(r + 2);
        yr.load(p.x, at + p.d, col, p.d, real);
        fr.load(p.f, at + p.d, col, p.d, real);
        // both norms' statistics side by side: means, then squares
        if (p.in_norm == kNormLayer || p.out_norm == kNormLayer) {
            float s[2] = {row_sum<CH>(y), row_sum<CH>(f)};
            team.sum(s);
            if (p.in_norm == kNormLayer) centre<CH>(s[0] * mask_in, p.d, col, y);
            if (p.out_norm == kNormLayer) centre<CH>(s[1] * mask_out, p.d, col, f);
        }
        float q[2] = {row_dot<CH>(y, y), row_dot<CH>(f, f)};
        team.sum(q);
        const float r_in = rsqrtf(fmaf(q[0], p.inv_d, p.in_eps));
        const float r_out = p.out_norm == kNormNone ? 1.f : rsqrtf(fmaf(q[1], p.inv_d, p.out_eps));
        hr.get(D);
        hr.load(p.dh, at + p.d, col, p.d, real);
        if (p.dh != nullptr) {
            UNIF_COLS(c, e) {
                y[c][e] *= r_in;
                acc[kSumInGamma][c][e] = fmaf(D[c][e], y[c][e], acc[kSumInGamma][c][e]);
                acc[kSumInBeta][c][e] += D[c][e];
                D[c][e] *= ig[c][e];
            }
            normalise_grad<CH, LPR>(team, p.in_norm, r_in, p.inv_d, y, D);
        }
        UNIF_COLS(c, e) D[c][e] += Vec<S>::get(gr.v[c], e);
        gr.load(p.dy, at + p.d, col, p.d, real);
        if (p.dx != nullptr)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float o[E];
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = p.scale * D[c][e];
                st_cols(static_cast<S*>(p.dx) + at, col[c], p.d, o);
            }
        UNIF_COLS(c, e) {
            f[c][e] *= r_out;
            acc[kSumOutGamma][c][e] = fmaf(D[c][e], f[c][e], acc[kSumOutGamma][c][e]);
            acc[kSumOutBeta][c][e] += D[c][e];
            D[c][e] *= cg[c][e];
        }
        if (p.df != nullptr) {
            if (p.out_norm != kNormNone) normalise_grad<CH, LPR>(team, p.out_norm, r_out, p.inv_d, f, D);
#pragma unroll
            for (int c = 0; c < CH; ++c) st_cols(static_cast<L*>(p.df) + at, col[c], p.d, D[c]);
        }
    }
    if (p.want == 0 && p.dgate == nullptr) return;
    if (p.grouped) {
        if (g >= 0) flush();
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            st_cols(mine, col[c], p.d, acc[kSumOutGamma][c]);
            st_cols(mine + p.d, col[c], p.d, acc[kSumOutBeta][c]);
        }
    }
    // The teams' sums in team order, one partial row each per workgroup.
    const int nteam = (int)blockDim.x / team.size();
    auto add_teams = [&](int first) {
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * p.d; i += blockDim.x) {
            const int k = first + (i >= p.d ? 1 : 0);
            if (!(p.want >> k & 1)) continue;
            float s = 0.f;
            for (int t = 0; t < nteam; ++t) s += sums[(size_t)t * 2 * p.d + i];
            p.part[((size_t)k * gridDim.x + blockIdx.x) * p.d + (i >= p.d ? i - p.d : i)] = s;
        }
    };
    add_teams(kSumOutGamma);
    __syncthreads();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        st_cols(mine, col[c], p.d, acc[kSumInGamma][c]);
        st_cols(mine + p.d, col[c], p.d, acc[kSumInBeta][c]);
    }
    add_teams(kSumInGamma);
}

struct ResidualFinish {
    int N, d, parts, teams, group, rows;
    int64_t groups;          // gate rows
    int grouped;
    const float* part;       // [4][parts][d]
    const float* gate_part;  // [teams][2][d]
    const float* out_gamma;
    const float* out_beta;
    const float* gate;
    float* d_out_gamma;      // NULL: not wanted
    float* d_out_beta;
    float* d_in_gamma;
    float* d_in_beta;
    float* d_gate;
};

// 64 columns per workgroup, the waves a stretch of the partial rows each, the
// stretches added in order, all in fp64. blockIdx.y 0 and 1: the sums of D
// f_hat and D (and with one gate row its gradient, in 0) and of dh v_hat and
// dh; from 2 on: gate rows whose tokens several teams share. Those are found
// from the ends of the teams' tokens, or, where there are fewer, from the gate
// rows: a row belongs to the first team's end that lies inside it.
constexpr int kFinishWaves = 16;

__global__ __launch_bounds__(kFinishWaves* kWave) void residual_finish_kernel(ResidualFinish p) {
    __shared__ double stretch[2][kFinishWaves][kWave];
    const int lane = lane_id(), w = (int)threadIdx.x >> 6, n = (int)blockIdx.x * kWave + lane;
    // sum of count rows of src, `stride` floats apart
    auto column = [&](const float* src, int64_t count, size_t stride) {
        const int64_t k0 = w * count / kFinishWaves, k1 = (w + 1) * count / kFinishWaves;
        double s = 0.0;
        int64_t k = k0;
        for (; k + 8 <= k1; k += 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = src[(size_t)(k + u) * stride];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += (double)v[u];
        }
        for (; k < k1; ++k) s += (double)src[(size_t)k * stride];
        return s;
    };
    auto total = [&](int i) {
        double s = 0.0;
        for (int k = 0; k < kFinishWaves; ++k) s += stretch[i][k][lane];
        return s;
    };
    if (blockIdx.y < 2) {
        const float* const src = p.part + (size_t)blockIdx.y * 2 * p.parts * p.d + n;
        const bool a = blockIdx.y == 1 ? p.d_in_gamma != nullptr : p.d_out_gamma != nullptr || (!p.grouped && p.d_gate != nullptr);
        const bool b = blockIdx.y == 1 ? p.d_in_beta != nullptr : p.d_out_beta != nullptr || (!p.grouped && p.d_gate != nullptr);
        stretch[0][w][lane] = (a && n < p.d) ? column(src, p.parts, p.d) : 0.0;
        stretch[1][w][lane] = (b && n < p.d) ? column(src + (size_t)p.parts * p.d, p.parts, p.d) : 0.0;
        __syncthreads();
        if (w != 0 || n >= p.d) return;
        const double s0 = total(0), s1 = total(1);
        if (blockIdx.y == 1) {
            if (p.d_in_gamma != nullptr) p.d_in_gamma[n] = (float)s0;
            if (p.d_in_beta != nullptr) p.d_in_beta[n] = (float)s1;
            return;
        }
        const double gt = (!p.grouped && p.gate != nullptr) ? (double)p.gate[n] : 1.0;
        if (p.d_out_gamma != nullptr) p.d_out_gamma[n] = (float)(gt * s0);
        if (p.d_out_beta != nullptr) p.d_out_beta[n] = (float)(gt * s1);
        if (!p.grouped && p.d_gate != nullptr)
            p.d_gate[n] = (float)((p.out_gamma != nullptr ? (double)p.out_gamma[n] : 1.0) * s0 +
                                  (p.out_beta != nullptr ? (double)p.out_beta[n] * s1 : 0.0));
        return;
    }
    int64_t g = (int64_t)blockIdx.y - 2;
    if (p.teams - 1 < p.groups) {
        const int64_t end = (g + 1) * p.rows;   // of team blockIdx.y - 2
        g = end / p.group;
        if (end >= p.N || g * p.group == end || end - p.rows > g * p.group) return;
    }
    const int64_t g0 = g * p.group, g1 = g0 + p.group < p.N ? g0 + p.group : p.N;
    const int64_t first = g0 / p.rows, last = (g1 - 1) / p.rows;
    if (first == last) return;
    double s = 0.0;
    if (n < p.d) s = column(p.gate_part + (size_t)(first + 1) * 2 * p.d + n, last - first, (size_t)2 * p.d);
    stretch[0][w][lane] = s;
    __syncthreads();
    if (w == 0 && n < p.d)
        p.d_gate[(size_t)g * p.d + n] =
            (float)((double)p.gate_part[((size_t)first * 2 + (g0 > first * p.rows ? 1 : 0)) * p.d + n] + total(0));
}

#undef UNIF_COLS

}  // namespace unifmoe
