// The join of a block's branch with the residual stream and the norm in front
// of the next block, v = s x + g N_out(f), y = v, h = N_in(v), and its backward.
//
// Both directions read every element once and keep a token's whole row in
// registers: a team of lanes holds the row, each lane kCols consecutive columns per
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
    const void* spare;         // d fp32 values that absent tensors' loads may read
    void* y;
    void* h;
    // backward
    const void* dy;
    const void* dh;
    void* dx;
    void* df;
    float* part;               // [4][workgroups][d] partial sums (kSum*), then a flag per workgroup (kSeen)
    float* gate_part;          // [teams][2][d]: a team's first and last piece of gate groups it shares
    float* dgate;              // [groups][d]: groups that one team holds (NULL: one gate row, or not wanted)
    int grouped;               // the gate has several rows
    int want;                  // bit i: partial sum i is wanted; bit kSeen: the flags, whether one had a real token
};

// kCols consecutive elements of a row, kCols = 4. Rows start at any element, so the
// vector accesses assume no more than the element's alignment.
constexpr int kCols = 4;
typedef u16 u16x4 __attribute__((ext_vector_type(4)));
typedef u16 u16x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
template <class T>
struct Vec;
template <>
struct Vec<float> {
    typedef f32x4 raw;
    typedef f32x4_a4 mem;
    static __device__ __forceinline__ float get(raw v, int e) { return v[e]; }
    static __device__ __forceinline__ raw pack(const float (&v)[kCols]) { return raw{v[0], v[1], v[2], v[3]}; }
};
template <>
struct Vec<u16> {
    typedef u16x4 raw;
    typedef u16x4_a2 mem;
    static __device__ __forceinline__ float get(raw v, int e) { return bf2f(v[e]); }
    static __device__ __forceinline__ raw pack(const float (&v)[kCols]) {
        return __builtin_bit_cast(raw, uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])});
    }
};

#define UNIF_COLS(c, e)            \
    _Pragma("unroll") for (int c = 0; c < CH; ++c) _Pragma("unroll") for (int e = 0; e < kCols; ++e)

// A lane's columns: CH chunks of kCols, those of the row's lanes side by side.
// Loads are issued without a branch, so that the waits for them count exactly
// what is in flight: a chunk that reaches past the row (d >= kCols) reads the row's
// last kCols elements instead, and fix() moves them into place, with 0 past d.
template <int CH>
struct Cols {
    int d;
    uint32_t col[CH], at[CH];   // first column, and where its load starts
    bool full;                  // every lane's columns lie inside the row
    __device__ __forceinline__ Cols(int d_, int lanes, int sub) : d(d_), full(d_ == CH * lanes * kCols) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            col[c] = (uint32_t)(c * lanes + sub) * kCols;
            at[c] = (int)col[c] + kCols <= d ? col[c] : (uint32_t)(d - kCols);
        }
    }
    __device__ __forceinline__ bool in(int c, int e) const { return (int)col[c] + e < d; }
    // What was loaded at at[]: in place, zeros past d and where off.
    __device__ __forceinline__ void fix(bool on, float (&v)[CH][kCols]) const {
        if (full && on) return;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t shift = col[c] - at[c];
            float w[kCols];
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                w[e] = v[c][e];
#pragma unroll
                for (int k = 1; e + k < kCols; ++k) w[e] = shift == (uint32_t)k ? v[c][e + k] : w[e];
            }
#pragma unroll
            for (int e = 0; e < kCols; ++e) v[c][e] = on && in(c, e) ? w[e] : 0.f;
        }
    }
    __device__ __forceinline__ void zero_past(float (&v)[CH][kCols]) const {
        if (!full) UNIF_COLS(c, e) v[c][e] = in(c, e) ? v[c][e] : 0.f;
    }
    // The byte offset is 32 bits wide, so that rows that a wave shares are
    // addressed from scalar registers.
    template <class T>
    __device__ __forceinline__ typename Vec<T>::raw load(int c, const T* row) const {
        return *reinterpret_cast<const typename Vec<T>::mem*>(reinterpret_cast<const char*>(row) +
                                                              at[c] * (uint32_t)sizeof(T));
    }
    // A parameter row, or `other` where there is none.
    __device__ __forceinline__ void param(const float* p, float other, float (&v)[CH][kCols]) const {
        if (p == nullptr) {
            UNIF_COLS(c, e) v[c][e] = other;
            return;
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const f32x4 w = load(c, p);
#pragma unroll
            for (int e = 0; e < kCols; ++e) v[c][e] = w[e];
        }
        fix(true, v);
    }
    template <bool PAST = false, class T>   // PAST: around the caches
    __device__ __forceinline__ void store(T* row, const float (&v)[CH][kCols]) const {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const typename Vec<T>::raw w = Vec<T>::pack(v[c]);
            typename Vec<T>::mem* const out =
                reinterpret_cast<typename Vec<T>::mem*>(reinterpret_cast<char*>(row) + col[c] * (uint32_t)sizeof(T));
            if ((int)col[c] + kCols <= d) {
                if constexpr (PAST) __builtin_nontemporal_store(w, out);
                else *out = w;
            } else
#pragma unroll
                for (int e = 0; e < kCols; ++e)
                    if (in(c, e)) row[col[c] + e] = w[e];
        }
    }
};

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
// the workgroup.
constexpr int kWideWaves = 16;   // most waves of a wide team
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
        // a whole wave's number is scalar, and so are its rows' addresses
        if constexpr (kWide) return (int)blockIdx.x;
        else if constexpr (kLanes == kWave)
            return (int)(blockIdx.x * (blockDim.x / kWave)) + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
        else return (int)((blockIdx.x * blockDim.x + threadIdx.x) / kLanes);
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
            // every 16 lanes read the waves' sums side by side
            const int k = lane_id() & (kWideWaves - 1);
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = lanes_sum<kWideWaves>(k < nw ? r[k * 4 + i] : 0.f);
        }
    }
};

// One row of a tensor on its way. Rows that are not wanted (padded tokens, the
// row past a team's last) and tensors that are absent are loaded from a row that
// is there and read as zeros.
template <class T, int CH>
struct RowRaw {
    const T* base;
    int64_t stride;   // 0: absent
    bool on;
    typename Vec<T>::raw v[CH];
    __device__ __forceinline__ RowRaw(const void* p, const void* other, int d)
        : base(static_cast<const T*>(p != nullptr ? p : other)), stride(p != nullptr ? d : 0), on(false) {}
    __device__ __forceinline__ void load(const Cols<CH>& k, int64_t r, bool real) {
        on = real && stride != 0;
        const T* const row = base + r * stride;
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = k.load(c, row);
    }
    __device__ __forceinline__ void get(const Cols<CH>& k, float (&u)[CH][kCols]) const {
        UNIF_COLS(c, e) u[c][e] = Vec<T>::get(v[c], e);
        k.fix(on, u);
    }
};

// Which of a team's tokens are real, 64 at a time: the lanes read their flags
// side by side.
template <int LANES>
struct RealRows {
    const uint8_t* valid;
    int64_t r0, r1;
    uint64_t bits;
    __device__ __forceinline__ RealRows(const uint8_t* v, int64_t r0_, int64_t r1_) : valid(v), r0(r0_), r1(r1_), bits(0) {}
    // Rows are asked for in order, from r0 on.
    __device__ __forceinline__ bool operator()(int64_t r) {
        if (valid == nullptr) return r < r1;
        const int i = (int)((r - r0) & 63);
        if (i == 0) {
            const int lane = lane_id(), sub = lane % LANES, first = lane - sub;
            bits = 0;
#pragma unroll
            for (int k = 0; k < kWave / LANES; ++k) {
                const int64_t t = r + k * LANES + sub;
                const uint64_t b = ballot(t < r1 && valid[t] != 0) >> first;
                bits |= (LANES == kWave ? b : b & ((1ull << (LANES & 63)) - 1)) << (k * LANES & 63);
            }
        }
        return bits >> i & 1;
    }
};

template <int CH>
__device__ __forceinline__ float row_sum(const float (&u)[CH][kCols]) {
    float s = 0.f;
    UNIF_COLS(c, e) s += u[c][e];
    return s;
}
template <int CH>
__device__ __forceinline__ float row_dot(const float (&a)[CH][kCols], const float (&b)[CH][kCols]) {
    float s = 0.f;
    UNIF_COLS(c, e) s = fmaf(a[c][e], b[c][e], s);
    return s;
}
template <int CH>
__device__ __forceinline__ void centre(const Cols<CH>& k, float mean, float (&u)[CH][kCols]) {
    UNIF_COLS(c, e) u[c][e] -= mean;
    k.zero_past(u);   // columns past d stay out of the sums
}

// Replaces the row u by its normalised values.
template <int CH, int LPR>
__device__ __forceinline__ void normalise(Team<LPR>& team, const Cols<CH>& k, int norm, float eps, float inv_d,
                                          float (&u)[CH][kCols]) {
    if (norm == kNormLayer) {
        float s[1] = {row_sum<CH>(u)};
        team.sum(s);
        centre<CH>(k, s[0] * inv_d, u);
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
                                               const float (&hat)[CH][kCols], float (&a)[CH][kCols]) {
    float s[2] = {0.f, row_dot<CH>(a, hat)};
    if (norm == kNormLayer) s[0] = row_sum<CH>(a);
    team.sum(s);
    const float m = -rstd * inv_d * s[0], q = -rstd * inv_d * s[1];
    UNIF_COLS(c, e) a[c][e] = fmaf(hat[c][e], q, fmaf(a[c][e], rstd, m));
}

// PAST: the outputs are larger than the caches and stored around them.
// 50,432 x 768 bf16, both norms and a gate per 197 tokens: 62 us, 5.0 TB/s of the
// 8 bytes an element (a copy runs at 5.15); 131,072 x 1,024 with an fp32 stream:
// 287 us, 5.6 TB/s of 12 bytes; one token 3.3 us, a launch.
template <class S, class L, bool PAST, int CH, int LPR>
__global__ __launch_bounds__(LPR == 0 ? kWideWaves * kWave : 256) void residual_forward_kernel(ResidualParams p) {
    __shared__ float red[2 * kWideWaves * 4];
    Team<LPR> team{red, 0};
    const Cols<CH> k(p.d, team.size(), team.sub());
    const int64_t r0 = (int64_t)team.index() * p.rows;
    const int64_t r1 = r0 + p.rows < p.N ? r0 + p.rows : p.N;
    if (r0 >= r1) return;
    RealRows<Team<LPR>::kLanes> is_real(p.valid, r0, r1);
    RowRaw<S, CH> x(p.x, p.spare, p.d);
    RowRaw<L, CH> f(p.f, p.spare, p.d);
    bool real = is_real(r0);
    x.load(k, r0, real);
    f.load(k, r0, real);
    // v = s x + cg f_hat + cb with cg = gate gamma_out, cb = gate beta_out
    float cg[CH][kCols], cb[CH][kCols], ig[CH][kCols], ib[CH][kCols];
    k.param(p.in_gamma, 1.f, ig);
    k.param(p.in_beta, 0.f, ib);
    int64_t gend = r0;   // cg and cb serve the tokens before gend
    for (int64_t r = r0; r < r1; ++r) {
        if (r >= gend) {
            const int64_t g = r / p.group;
            gend = (g + 1) * p.group;
            float gt[CH][kCols];
            k.param(p.gate == nullptr ? nullptr : p.gate + g * p.d, 1.f, gt);
            k.param(p.out_gamma, 1.f, cg);
            k.param(p.out_beta, 0.f, cb);
            UNIF_COLS(c, e) cg[c][e] *= gt[c][e];
            UNIF_COLS(c, e) cb[c][e] *= gt[c][e];
        }
        const size_t at = (size_t)r * p.d;
        float v[CH][kCols], u[CH][kCols];
        f.get(k, v);
        x.get(k, u);
        const bool keep = real;
        real = is_real(r + 1);
        x.load(k, real ? r + 1 : r, real);
        f.load(k, real ? r + 1 : r, real);
        if (p.out_norm != kNormNone) normalise<CH, LPR>(team, k, p.out_norm, p.out_eps, p.inv_d, v);
        UNIF_COLS(c, e) v[c][e] = fmaf(p.scale, u[c][e], fmaf(v[c][e], cg[c][e], cb[c][e]));
        if (!keep) UNIF_COLS(c, e) v[c][e] = 0.f;
        if (p.y != nullptr) k.template store<PAST>(static_cast<S*>(p.y) + at, v);
        if (p.h != nullptr) {
            normalise<CH, LPR>(team, k, p.in_norm, p.in_eps, p.inv_d, v);
            UNIF_COLS(c, e) v[c][e] = fmaf(v[c][e], ig[c][e], ib[c][e]);
            if (!keep) UNIF_COLS(c, e) v[c][e] = 0.f;
            k.template store<PAST>(static_cast<L*>(p.h) + at, v);
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
// where it held all of its tokens, else as its first or last piece. Parameters may
// be NaN or infinite where only padded tokens meet them (the gate row of an empty
// sequence, say): they are multiplied only with what real tokens left.
// 50,432 x 768 bf16 with fp32 dh: 119 us of 125, 4.5 TB/s of 14 bytes an element; the
// registers (four sums, two parameter rows, four rows in flight) leave two waves
// per SIMD, which is what keeps it from the copy's rate. Rows of 769 to 1,024 columns (4
// chunks) spill 8 to 24 registers but in bf16 throughout, and wide rows, whose teams may
// have 16 waves and so 128 registers a lane, 17 to 37: 10 of the 109 MB that 4,099 x
// 5,120 writes.
constexpr int kSumOutGamma = 0, kSumOutBeta = 1, kSumInGamma = 2, kSumInBeta = 3, kSeen = 4;

template <class S, class L, class H, int CH, int LPR>
__global__ __launch_bounds__(LPR == 0 ? kWideWaves * kWave : 512) void residual_backward_kernel(ResidualParams p) {
    __shared__ float red[2 * kWideWaves * 4];
    __shared__ int seen_by[kWideWaves];
    extern __shared__ float sums[];   // [teams of the workgroup][2][d]
    Team<LPR> team{red, 0};
    const Cols<CH> k(p.d, team.size(), team.sub());
    float* const mine = sums + (size_t)team.local() * 2 * p.d;
    const int64_t r0 = (int64_t)team.index() * p.rows;
    const int64_t r1 = r0 + p.rows < p.N ? r0 + p.rows : p.N;
    RealRows<Team<LPR>::kLanes> is_real(p.valid, r0, r1);
    RowRaw<S, CH> yr(p.x, p.spare, p.d), gr(p.dy, p.spare, p.d);
    RowRaw<H, CH> hr(p.dh, p.spare, p.d);
    RowRaw<L, CH> fr(p.f, p.spare, p.d);
    bool real = is_real(r0);
    const int64_t start = r0 < p.N ? r0 : 0;
    yr.load(k, start, real);
    fr.load(k, start, real);
    hr.load(k, start, real);
    gr.load(k, start, real);
    float acc[4][CH][kCols];
#pragma unroll
    for (int i = 0; i < 4; ++i) UNIF_COLS(c, e) acc[i][c][e] = 0.f;
    if (p.grouped) {
        k.store(mine, acc[kSumOutGamma]);
        k.store(mine + p.d, acc[kSumOutBeta]);
    }
    float ig[CH][kCols], cg[CH][kCols];   // cg = gate gamma_out
    k.param(p.in_gamma, 1.f, ig);
    int64_t g = -1, gend = r0;
    bool seen = false;   // a real token since the last flush
    auto flush = [&]() {
        const int64_t g0 = g * p.group, g1 = gend < p.N ? gend : p.N;
        float* const dst = (g0 >= r0 && g1 <= r1) ? p.dgate + g * p.d
                                                  : p.gate_part + ((size_t)team.index() * 2 + (g0 > r0 ? 1 : 0)) * p.d;
        float w[CH][kCols], v[CH][kCols];
        if (p.dgate != nullptr) {
            k.param(p.out_gamma, 1.f, w);
            k.param(p.out_beta, 0.f, v);
            UNIF_COLS(c, e) w[c][e] = fmaf(w[c][e], acc[kSumOutGamma][c][e], v[c][e] * acc[kSumOutBeta][c][e]);
            if (!seen) UNIF_COLS(c, e) w[c][e] = 0.f;
            k.store(dst, w);
        }
        if (!seen) return;   // both sums are 0
        seen = false;
        k.param(p.gate + g * p.d, 1.f, w);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            k.param(mine + i * p.d, 0.f, v);
            UNIF_COLS(c, e) v[c][e] = fmaf(w[c][e], acc[i][c][e], v[c][e]);
            k.store(mine + i * p.d, v);
            UNIF_COLS(c, e) acc[i][c][e] = 0.f;
        }
    };
    for (int64_t r = r0; r < r1; ++r) {
        if (r >= gend) {
            if (p.grouped && g >= 0) flush();
            g = r / p.group;
            gend = (g + 1) * p.group;
            float gt[CH][kCols];
            k.param(p.gate == nullptr ? nullptr : p.gate + g * p.d, 1.f, gt);
            k.param(p.out_gamma, 1.f, cg);
            UNIF_COLS(c, e) cg[c][e] *= gt[c][e];
        }
        // Each tensor's next row is loaded as soon as this one's is in use.
        const size_t at = (size_t)r * p.d;
        float y[CH][kCols], D[CH][kCols], f[CH][kCols];
        yr.get(k, y);
        fr.get(k, f);
        const bool keep = real;
        seen |= keep;
        real = is_real(r + 1);
        const int64_t ahead = real ? r + 1 : r;
        yr.load(k, ahead, real);
        fr.load(k, ahead, real);
        // both norms' statistics side by side: means, then squares
        if (p.in_norm == kNormLayer || p.out_norm == kNormLayer) {
            float s[2] = {row_sum<CH>(y), row_sum<CH>(f)};
            team.sum(s);
            if (p.in_norm == kNormLayer) centre<CH>(k, s[0] * p.inv_d, y);
            if (p.out_norm == kNormLayer) centre<CH>(k, s[1] * p.inv_d, f);
        }
        float q[2] = {row_dot<CH>(y, y), row_dot<CH>(f, f)};
        team.sum(q);
        const float r_in = rsqrtf(fmaf(q[0], p.inv_d, p.in_eps));
        const float r_out = p.out_norm == kNormNone ? 1.f : rsqrtf(fmaf(q[1], p.inv_d, p.out_eps));
        hr.get(k, D);
        hr.load(k, ahead, real);
        if (p.dh != nullptr) {
            UNIF_COLS(c, e) {
                y[c][e] *= r_in;
                acc[kSumInGamma][c][e] = fmaf(D[c][e], y[c][e], acc[kSumInGamma][c][e]);
                acc[kSumInBeta][c][e] += D[c][e];
                D[c][e] *= ig[c][e];
            }
            normalise_grad<CH, LPR>(team, p.in_norm, r_in, p.inv_d, y, D);
        }
        float dy[CH][kCols];
        gr.get(k, dy);
        gr.load(k, ahead, real);
        UNIF_COLS(c, e) D[c][e] += dy[c][e];
        if (!keep) UNIF_COLS(c, e) D[c][e] = 0.f;
        if (p.dx != nullptr) {
            UNIF_COLS(c, e) dy[c][e] = p.scale * D[c][e];
            k.store(static_cast<S*>(p.dx) + at, dy);
        }
        UNIF_COLS(c, e) {
            f[c][e] *= r_out;
            acc[kSumOutGamma][c][e] = fmaf(D[c][e], f[c][e], acc[kSumOutGamma][c][e]);
            acc[kSumOutBeta][c][e] += D[c][e];
            D[c][e] *= cg[c][e];
        }
        if (p.df != nullptr) {
            if (p.out_norm != kNormNone) normalise_grad<CH, LPR>(team, p.out_norm, r_out, p.inv_d, f, D);
            if (!keep) UNIF_COLS(c, e) D[c][e] = 0.f;
            k.store(static_cast<L*>(p.df) + at, D);
        }
    }
    if (p.want == 0 && p.dgate == nullptr) return;
    if (p.grouped) {
        if (g >= 0) flush();
    } else {
        k.store(mine, acc[kSumOutGamma]);
        k.store(mine + p.d, acc[kSumOutBeta]);
    }
    if (p.want >> kSeen & 1) {
        const uint64_t b = ballot(seen);
        if (lane_id() == 0) seen_by[threadIdx.x >> 6] = b != 0;
    }
    // The teams' sums in team order, one partial row each per workgroup.
    const int nteam = (int)blockDim.x / team.size();
    auto add_teams = [&](int first) {
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * p.d; i += blockDim.x) {
            const int which = first + (i >= p.d ? 1 : 0);
            if (!(p.want >> which & 1)) continue;
            float s = 0.f;
#pragma unroll 8
            for (int t = 0; t < nteam; ++t) s += sums[(size_t)t * 2 * p.d + i];
            p.part[((size_t)which * gridDim.x + blockIdx.x) * p.d + (i >= p.d ? i - p.d : i)] = s;
        }
    };
    add_teams(kSumOutGamma);
    if ((p.want >> kSeen & 1) && threadIdx.x == 0) {
        int any = 0;
        for (int i = 0; i < (int)blockDim.x >> 6; ++i) any |= seen_by[i];
        reinterpret_cast<int*>(p.part + (size_t)4 * gridDim.x * p.d)[blockIdx.x] = any;
    }
    __syncthreads();
    k.store(mine, acc[kSumInGamma]);
    k.store(mine + p.d, acc[kSumInBeta]);
    add_teams(kSumInGamma);
}

struct ResidualFinish {
    int N, d, parts, teams, group, rows;
    int64_t groups;          // gate rows
    int by_wave;             // a wave takes a gate row (few teams share one), else the workgroup
    int grouped;
    const float* part;       // [4][parts][d]
    const float* gate_part;  // [teams][2][d]
    const float* out_gamma;
    const float* out_beta;
    const float* gate;
    float* d_sum[4];         // gradients of the parameters by their sum (NULL: not wanted)
    float* d_gate;
    const int* seen;         // [parts]: whether a workgroup had a real token (NULL: every one did)
};

// 64 columns per workgroup, the waves a stretch of the partial rows each, the
// stretches added in order, all in fp64. blockIdx.y 0 to 3: the sums (0 also
// forms the gradient of a single gate row, from two of them); from 4 on: gate
// rows whose tokens several teams share. Those are found from the ends of the
// teams' tokens, or, where there are fewer, from the gate rows: a row belongs to
// the first team's end that lies inside it. A gate row that few teams share is
// one wave's, so that a workgroup takes as many as it has waves. A single gate row
// and N_out's parameters are multiplied here and so only where a real token met
// them: `seen` tells, where tokens may be padded. Latency bound: 4 to
// 7 us (253 partial rows of 768, 256 gate rows: 5.0; 16 waves where 4 took 14).
constexpr int kFinishWaves = 16;

__global__ __launch_bounds__(kFinishWaves* kWave) void residual_finish_kernel(ResidualFinish p) {
    __shared__ double stretch[2][kFinishWaves][kWave];
    __shared__ int seen[kFinishWaves];
    const int lane = lane_id(), w = (int)threadIdx.x >> 6, n = (int)blockIdx.x * kWave + lane;
    // sum of rows k0 to k1 of src, `stride` floats apart
    auto column = [&](const float* src, int64_t k0, int64_t k1, size_t stride) {
        double s = 0.0;
        int64_t k = k0;
        for (; k + 16 <= k1; k += 16) {
            float v[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) v[u] = src[(size_t)(k + u) * stride];
#pragma unroll
            for (int u = 0; u < 16; ++u) s += (double)v[u];
        }
        for (; k + 4 <= k1; k += 4) {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = src[(size_t)(k + u) * stride];
#pragma unroll
            for (int u = 0; u < 4; ++u) s += (double)v[u];
        }
        for (; k < k1; ++k) s += (double)src[(size_t)k * stride];
        return s;
    };
    auto part_of = [&](const float* src, int64_t count, size_t stride) {
        return column(src, w * count / kFinishWaves, (w + 1) * count / kFinishWaves, stride);
    };
    auto total = [&](int i) {
        double s = 0.0;
        for (int k = 0; k < kFinishWaves; ++k) s += stretch[i][k][lane];
        return s;
    };
    if (blockIdx.y < 4) {
        const int i = (int)blockIdx.y;
        const bool gate = i == kSumOutGamma && !p.grouped && p.d_gate != nullptr;
        float* const out = p.d_sum[i];
        if (out == nullptr && !gate) return;
        const float* const src = p.part + (size_t)i * p.parts * p.d + n;
        stretch[0][w][lane] = n < p.d ? part_of(src, p.parts, p.d) : 0.0;
        stretch[1][w][lane] = gate && n < p.d ? part_of(src + (size_t)p.parts * p.d, p.parts, p.d) : 0.0;
        if (p.seen != nullptr) {
            int any = 0;
            for (int k = (int)threadIdx.x; k < p.parts; k += (int)blockDim.x) any |= p.seen[k];
            const uint64_t b = ballot(any != 0);
            if (lane == 0) seen[w] = b != 0;
        }
        __syncthreads();
        if (w != 0 || n >= p.d) return;
        if (p.seen != nullptr) {
            int any = 0;
            for (int k = 0; k < kFinishWaves; ++k) any |= seen[k];
            if (any == 0) {
                if (out != nullptr) out[n] = 0.f;
                if (gate) p.d_gate[n] = 0.f;
                return;
            }
        }
        const double s = total(0);
        if (out != nullptr) out[n] = (float)(i <= kSumOutBeta && !p.grouped && p.gate != nullptr ? s * (double)p.gate[n] : s);
        if (gate)
            p.d_gate[n] = (float)((p.out_gamma != nullptr ? (double)p.out_gamma[n] : 1.0) * s +
                                  (p.out_beta != nullptr ? (double)p.out_beta[n] * total(1) : 0.0));
        return;
    }
    int64_t g = (int64_t)blockIdx.y - 4;
    if (p.by_wave) g = g * kFinishWaves + w;
    int64_t first = -1, last = -1;
    if (p.teams - 1 < p.groups) {
        const int64_t end = (g + 1) * p.rows;   // of team number g
        g = end / p.group;
        if (end < p.N && g * p.group < end && end - p.rows <= g * p.group) first = end / p.rows - 1;
    } else if (g < p.groups) {
        first = g * p.group / p.rows;
    }
    const int64_t g0 = g * p.group, g1 = g0 + p.group < p.N ? g0 + p.group : p.N;
    if (first >= 0) last = (g1 - 1) / p.rows;
    const bool shared = first >= 0 && first < last && n < p.d;
    const float* const rest = p.gate_part + (size_t)(first + 1) * 2 * p.d + n;
    double s = 0.0;
    if (p.by_wave) {
        if (shared) s = column(rest, 0, last - first, (size_t)2 * p.d);
    } else {
        stretch[0][w][lane] = shared ? part_of(rest, last - first, (size_t)2 * p.d) : 0.0;
        __syncthreads();
        s = total(0);
    }
    if (shared && (p.by_wave || w == 0))
        p.d_gate[(size_t)g * p.d + n] =
            (float)((double)p.gate_part[((size_t)first * 2 + (g0 > first * p.rows ? 1 : 0)) * p.d + n] + s);
}

#undef UNIF_COLS

}  // namespace unifmoe
