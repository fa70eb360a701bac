// Host side of the operators around the layer (include/unif_moe_ops.h):
// argument validation, workspace planning and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "../../include/unif_moe_ops.h"
#include "balance.hpp"
#include "common.hpp"
#include "host.hpp"
#include "residual.hpp"

using namespace unifmoe;

namespace {

// Quotient rounded up; token counts may be near INT32_MAX.
int div_up(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

size_t elem_size(int32_t dtype) { return dtype == UNIF_BF16 ? 2 : 4; }

bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A tensor as a range of addresses (empty where it is absent).
struct Span {
    uintptr_t b, e;
    Span(const void* p, size_t bytes) : b(reinterpret_cast<uintptr_t>(p)), e(p != nullptr ? b + bytes : b) {}
    bool meets(const Span& o) const { return b < e && o.b < o.e && b < o.e && o.b < e; }
    bool same(const Span& o) const { return b == o.b && e == o.e; }
};

// Whether every output is apart from every input and from the other outputs,
// but for output i being exactly its partner (an input updated in place).
template <int NO, int NI>
bool apart(const Span (&out)[NO], const Span (&partner)[NO], const Span (&in)[NI]) {
    for (int i = 0; i < NO; ++i) {
        for (int j = 0; j < i; ++j)
            if (out[i].meets(out[j])) return false;
        for (int j = 0; j < NO; ++j)
            if (out[i].meets(partner[j]) && !(i == j && out[i].same(partner[j]))) return false;
        for (int j = 0; j < NI; ++j)
            if (out[i].meets(in[j])) return false;
    }
    return true;
}

bool norm_ok(int32_t norm, float eps, const float* gamma, const float* beta) {
    if (norm == UNIF_ROWNORM_NONE) return gamma == nullptr && beta == nullptr;
    if (norm != UNIF_ROWNORM_LAYER && norm != UNIF_ROWNORM_RMS) return false;
    return eps >= FLT_MIN && std::isfinite(eps) && gamma != nullptr;   // 1 / sqrt(eps) is formed in fp32
}

int32_t check_residual(const unif_moe_residual* r) {
    if (r == nullptr) return UNIF_EINVAL;
    if (r->n_tokens < 0 || r->d_model < 1 || r->tokens_per_gate < 0 || !std::isfinite(r->residual_scale))
        return UNIF_EINVAL;
    if (r->dtype != UNIF_F32 && r->dtype != UNIF_BF16) return UNIF_EINVAL;
    if (r->stream_dtype != UNIF_F32 && (r->stream_dtype != UNIF_BF16 || r->dtype != UNIF_BF16)) return UNIF_EINVAL;
    if (!norm_ok(r->out_norm, r->out_eps, r->out_gamma, r->out_beta)) return UNIF_EINVAL;
    if (!norm_ok(r->in_norm, r->in_eps, r->in_gamma, r->in_beta)) return UNIF_EINVAL;
    for (const float* p : {r->out_gamma, r->out_beta, r->in_gamma, r->in_beta, r->gate})
        if (!aligned_to(p, 4)) return UNIF_EINVAL;
    if (r->d_model < UNIF_RESIDUAL_MIN_D || r->d_model > UNIF_RESIDUAL_MAX_D) return UNIF_EUNSUPPORTED;
    return UNIF_OK;
}

int64_t gate_rows(const unif_moe_residual* r) {
    if (r->tokens_per_gate == 0) return 1;
    return ((int64_t)r->n_tokens + r->tokens_per_gate - 1) / r->tokens_per_gate;
}
size_t gate_bytes(const unif_moe_residual* r) { return (size_t)gate_rows(r) * r->d_model * sizeof(float); }
// Several gate rows: their gradients are sums over parts of the tokens.
bool gate_grouped(const unif_moe_residual* r) { return r->gate != nullptr && gate_rows(r) > 1; }

// LDS that the kernels declare beside what their launch asks for.
constexpr size_t kTeamLds = kWideWaves * (8 * sizeof(float) + sizeof(int)), kCountLds = kBalWaves * (kWave * 12 + 8) + 4 * kWave,
                 kSlopeLds = 8 * (kWave * kBalWaves + 2 * kWave + 2) + 4 * kWave;

// Lanes per row (0: the workgroup) and the launch that covers the tokens.
struct RowShape {
    int lpr, chunks, threads, rows, blocks;
    int teams() const { return lpr == 0 ? blocks : blocks * (threads / lpr); }
};
// Rows of up to 1,024 columns are a part of a wave's, 2 or 3 chunks of kCols columns
// per lane (a whole wave's also 4), the fewest columns that cover the row, more
// lanes rather than more chunks: 2 chunks against 4 on half the lanes, 200,000 x
// 128 bf16 42 us and 49, 400,000 x 64 45 and 59, 60,000 x 512 50 and 53; 3 chunks
// against 2 on twice the lanes for 50,432 x 384's gradient: 67 and 79. Wider rows
// take a workgroup, 2 chunks per lane.
RowShape narrow_shape(int d, int threads) {
    RowShape s{};
    s.lpr = 8;
    while (s.lpr < kWave && s.lpr * 3 * kCols < d) s.lpr *= 2;
    s.chunks = s.lpr * 2 * kCols >= d ? 2 : s.lpr * 3 * kCols >= d ? 3 : 4;
    s.threads = threads;
    return s;
}
RowShape wide_shape(int d) {
    RowShape s{};
    s.chunks = 2;
    s.threads = div_up(d, kWave * 2 * kCols) * kWave;
    return s;
}
// The tokens dealt to at most `waves` waves per compute unit.
RowShape cover(RowShape s, int N, int cus, int waves) {
    const int per_block = s.lpr == 0 ? 1 : s.threads / s.lpr;
    const int most = cus * std::max(1, waves / (s.threads / kWave)) * per_block;
    s.rows = std::max(1, div_up(N, most));
    s.blocks = div_up(div_up(N, s.rows), per_block);
    return s;
}

// Outputs past this size do not stay in the L2s (8 x 4 MB) for the next kernel
// and are stored around them: join of 131,072 x 1,024 with an fp32 stream 304 ->
// 286 us, of 50,432 x 768 57 -> 49; balance gradients of 131,072 x 1,024, K = 32,
// 315 -> 306 in an earlier form. (The join's gradients gain nothing: 50,432 x 768
// 125.8 and 127.3.) Together with the kernel that reads the output next it gains
// nothing: the join and a pass over h 390 and 388 us at 131,072 x 1,024, 83 and 85 at
// 50,432 x 768; the balance gradients and the gradient of N_in 609 and 607, 161 and
// 160.
constexpr size_t kCacheBytes = (size_t)32 << 20;

// Calls f(chunks, lanes per row) for a launch's shape.
template <class F>
void with_shape(const RowShape& s, F f) {
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 3> three;
    const std::integral_constant<int, 8> l8;
    const std::integral_constant<int, 16> l16;
    const std::integral_constant<int, 32> l32;
    const std::integral_constant<int, 64> l64;
    if (s.lpr == 0) return f(two, std::integral_constant<int, 0>());
    if (s.chunks == 4) return f(std::integral_constant<int, 4>(), l64);
    if (s.chunks == 3) return s.lpr == 8 ? f(three, l8) : s.lpr == 16 ? f(three, l16) : s.lpr == 32 ? f(three, l32) : f(three, l64);
    return s.lpr == 8 ? f(two, l8) : s.lpr == 16 ? f(two, l16) : s.lpr == 32 ? f(two, l32) : f(two, l64);
}

constexpr int kNarrowD = kWave * 4 * kCols;
// Forward: many more waves than run at once, so that the last ones of a launch
// leave little of the chip idle: 65,536 x 1,024 bf16 113.5 us with 16 waves per
// compute unit, 111 with 32, 108.8 with 64; 200,000 x 128 46.6, 44.9 and 42.5.
// Wide rows' teams are few and come in whole workgroups: about as many waves as run
// at once. 16, 32 and 64 waves: 540 x 6,656 11.8, 15.8 and 16.5 us; 1,068 x 4,400
// 15.7, 22.2 and 25.8; 16,384 x 5,120 149, 158 and 164; but 4,099 x 5,120 47, 45 and
// 47, 16,384 x 2,048 63, 62 and 64.
RowShape forward_shape(const unif_moe_residual* r, int cus) {
    if (r->d_model > kNarrowD) return cover(wide_shape(r->d_model), r->n_tokens, cus, 16);
    return cover(narrow_shape(r->d_model, 256), r->n_tokens, cus, 64);
}
// Backward: as many waves as run at once (two per SIMD by the registers of 3 and 4
// chunks a lane), so that the partial rows are few: 50,432 x 768 134 us with 8 waves
// per compute unit, 168 with 4, 158 with 24. The kernels of 2 chunks a lane take 137
// to 170 registers, and most would run three per SIMD; they are launched alike, which
// was not measured for them. Wide rows in 2 chunks a lane: 16,384 x 4,096 170 us, in 3
// 212, in 4 184; 4,099 x 5,120 72, 78 and 79.
RowShape backward_shape(const unif_moe_residual* r, int cus) {
    return cover(r->d_model > kNarrowD ? wide_shape(r->d_model) : narrow_shape(r->d_model, 512), r->n_tokens, cus, 8);
}

template <class S, class L>
void launch_forward(const RowShape& s, const ResidualParams& p, hipStream_t st) {
    const size_t out = (size_t)p.N * p.d * ((p.y != nullptr ? sizeof(S) : 0) + (p.h != nullptr ? sizeof(L) : 0));
    with_shape(s, [&](auto ch, auto lpr) {
        if (out > kCacheBytes)
            residual_forward_kernel<S, L, true, ch.value, lpr.value><<<(unsigned)s.blocks, (unsigned)s.threads, 0, st>>>(p);
        else
            residual_forward_kernel<S, L, false, ch.value, lpr.value><<<(unsigned)s.blocks, (unsigned)s.threads, 0, st>>>(p);
    });
}
template <class S, class L, class H>
int32_t launch_backward(const RowShape& s, const ResidualParams& p, hipStream_t st) {
    const size_t lds = (size_t)(s.teams() / s.blocks) * 2 * p.d * sizeof(float);
    int32_t status = UNIF_OK;
    with_shape(s, [&](auto ch, auto lpr) {
        status = allow_lds(residual_backward_kernel<S, L, H, ch.value, lpr.value>, lds + kTeamLds);
        if (status != UNIF_OK) return;
        residual_backward_kernel<S, L, H, ch.value, lpr.value>
            <<<(unsigned)s.blocks, (unsigned)s.threads, lds, st>>>(p);
    });
    return status;
}

ResidualParams residual_params(const unif_moe_residual* r, const RowShape& s) {
    ResidualParams p{};
    p.N = r->n_tokens;
    p.d = r->d_model;
    p.rows = s.rows;
    p.out_norm = r->out_norm;
    p.in_norm = r->in_norm;
    p.group = gate_grouped(r) ? r->tokens_per_gate : r->n_tokens;
    p.out_eps = r->out_eps;
    p.in_eps = r->in_eps;
    p.scale = r->residual_scale;
    p.inv_d = (float)(1.0 / r->d_model);
    p.out_gamma = r->out_gamma;
    p.out_beta = r->out_beta;
    p.in_gamma = r->in_gamma;
    p.in_beta = r->in_beta;
    p.gate = r->gate;
    return p;
}

// Workspace of the backward: four partial rows and a flag per workgroup, and a
// team's two pieces of shared gate groups, for the launch of any number of compute
// units up to kMaxCus (the size is known without a device).
constexpr int kMaxCus = 512;
struct ResidualPlan {
    size_t part, gate_part, total;
};
ResidualPlan plan_residual(const unif_moe_residual* r) {
    const RowShape s = backward_shape(r, kMaxCus);
    const size_t row = (size_t)r->d_model * sizeof(float);
    Carver cv;
    ResidualPlan p;
    p.part = cv.take((4 * row + sizeof(int)) * s.blocks);
    p.gate_part = cv.take(gate_grouped(r) ? 2 * row * s.teams() : 0);
    p.total = cv.cur + 256;
    return p;
}

__global__ void zero_floats_kernel(float* p, size_t n) {
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) p[i] = 0.f;
}

}  // namespace

extern "C" {

int32_t unif_moe_residual_forward(const unif_moe_residual* res, const void* x, const void* f, const uint8_t* valid,
                                  void* y, void* h, void* stream) {
    const int32_t s = check_residual(res);
    if (s != UNIF_OK) return s;
    const size_t n = (size_t)res->n_tokens * res->d_model;
    const size_t se = elem_size(res->stream_dtype), le = elem_size(res->dtype);
    if (n > 0) {
        if ((x == nullptr && f == nullptr) || (y == nullptr && h == nullptr)) return UNIF_EINVAL;
        if (f == nullptr && (res->out_norm != UNIF_ROWNORM_NONE || res->gate != nullptr)) return UNIF_EINVAL;
    }
    if (h != nullptr && res->in_norm == UNIF_ROWNORM_NONE) return UNIF_EINVAL;
    if (!aligned_to(x, se) || !aligned_to(y, se) || !aligned_to(f, le) || !aligned_to(h, le)) return UNIF_EINVAL;
    const size_t row = (size_t)res->d_model * 4;
    const Span out[] = {Span(y, n * se), Span(h, n * le)}, partner[] = {Span(x, n * se), Span(nullptr, 0)};
    const Span in[] = {Span(f, n * le), Span(valid, res->n_tokens), Span(res->out_gamma, row),
                       Span(res->out_beta, row), Span(res->in_gamma, row), Span(res->in_beta, row),
                       Span(res->gate, gate_bytes(res))};
    if (!apart(out, partner, in)) return UNIF_EINVAL;
    if (n == 0) return UNIF_OK;
    const RowShape sh = forward_shape(res, std::min(cu_count(), kMaxCus));
    ResidualParams p = residual_params(res, sh);
    p.x = x;
    p.f = f;
    // x is absent only beside h and so in_gamma, or beside y
    p.spare = x != nullptr ? x : y != nullptr ? y : res->in_gamma;
    p.valid = valid;
    p.y = y;
    p.h = h;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (res->dtype == UNIF_F32) launch_forward<float, float>(sh, p, st);
    else if (res->stream_dtype == UNIF_F32) launch_forward<float, u16>(sh, p, st);
    else launch_forward<u16, u16>(sh, p, st);
    UNIF_LAUNCH_CHECK();
    return UNIF_OK;
}

int32_t unif_moe_residual_backward_workspace_size(const unif_moe_residual* res, size_t* bytes) {
    if (bytes == nullptr) return UNIF_EINVAL;
    const int32_t s = check_residual(res);
    if (s != UNIF_OK) return s;
    *bytes = plan_residual(res).total;
    return UNIF_OK;
}

int32_t unif_moe_residual_backward(const unif_moe_residual* res, const void* y, const void* f, const uint8_t* valid,
                                   const void* dy, const void* dh, int32_t dh_dtype, void* dx, void* df,
                                   const unif_moe_residual_grads* grads, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    const int32_t s = check_residual(res);
    if (s != UNIF_OK) return s;
    if (dh_dtype != UNIF_F32 && dh_dtype != res->dtype) return UNIF_EINVAL;
    static const unif_moe_residual_grads none{};
    const unif_moe_residual_grads& gr = grads != nullptr ? *grads : none;
    float* const want[5] = {gr.out_gamma, gr.out_beta, gr.in_gamma, gr.in_beta, gr.gate};
    const float* const have[5] = {res->out_gamma, res->out_beta, res->in_gamma, res->in_beta, res->gate};
    for (int i = 0; i < 5; ++i)
        if (want[i] != nullptr && (have[i] == nullptr || !aligned_to(want[i], 4))) return UNIF_EINVAL;
    const size_t n = (size_t)res->n_tokens * res->d_model;
    const size_t se = elem_size(res->stream_dtype), le = elem_size(res->dtype), he = elem_size(dh_dtype);
    if (n > 0) {
        if (dy == nullptr && dh == nullptr) return UNIF_EINVAL;
        if ((dh == nullptr) != (y == nullptr)) return UNIF_EINVAL;
        if (dh == nullptr && (gr.in_gamma != nullptr || gr.in_beta != nullptr)) return UNIF_EINVAL;
        const bool branch = gr.out_gamma != nullptr || gr.out_beta != nullptr || gr.gate != nullptr ||
                            (df != nullptr && res->out_norm != UNIF_ROWNORM_NONE);
        if (branch && f == nullptr) return UNIF_EINVAL;
    }
    if (dh != nullptr && res->in_norm == UNIF_ROWNORM_NONE) return UNIF_EINVAL;
    if (!aligned_to(y, se) || !aligned_to(dy, se) || !aligned_to(dx, se) || !aligned_to(f, le) ||
        !aligned_to(df, le) || !aligned_to(dh, he))
        return UNIF_EINVAL;
    const ResidualPlan plan = plan_residual(res);
    if (workspace == nullptr || workspace_bytes < plan.total) return UNIF_EWORKSPACE;
    const size_t row = (size_t)res->d_model * 4, gb = gate_bytes(res);
    const Span out[] = {Span(dx, n * se), Span(df, n * le), Span(gr.out_gamma, row), Span(gr.out_beta, row),
                        Span(gr.in_gamma, row), Span(gr.in_beta, row), Span(gr.gate, gb),
                        Span(workspace, plan.total)};
    const Span no(nullptr, 0);
    const Span partner[] = {Span(dy, n * se), no, no, no, no, no, no, no};
    const Span in[] = {Span(y, n * se), Span(f, n * le), Span(valid, res->n_tokens), Span(dh, n * he),
                       Span(res->out_gamma, row), Span(res->out_beta, row), Span(res->in_gamma, row),
                       Span(res->in_beta, row), Span(res->gate, gb)};
    if (!apart(out, partner, in)) return UNIF_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (n == 0) {   // sums over no tokens
        for (int i = 0; i < 5; ++i) {
            const size_t m = i == 4 ? gb / 4 : (size_t)res->d_model;
            if (want[i] == nullptr || m == 0) continue;
            zero_floats_kernel<<<(unsigned)std::min<size_t>(ceil_div_sz(m, 256), 1024), 256, 0, st>>>(want[i], m);
            UNIF_LAUNCH_CHECK();
        }
        return UNIF_OK;
    }
    const RowShape sh = backward_shape(res, std::min(cu_count(), kMaxCus));
    ResidualParams p = residual_params(res, sh);
    char* ws = align_base(workspace);
    p.grouped = gate_grouped(res);
    p.x = y;
    p.f = f;
    p.valid = valid;
    p.dy = dy;
    p.dh = dh;
    p.dx = dx;
    p.df = df;
    p.spare = ws;
    p.part = reinterpret_cast<float*>(ws + plan.part);
    p.gate_part = reinterpret_cast<float*>(ws + plan.gate_part);
    p.dgate = p.grouped ? gr.gate : nullptr;
    const bool one_gate = !p.grouped && gr.gate != nullptr;   // from the sums of out_gamma and out_beta
    p.want = (gr.out_gamma != nullptr || one_gate ? 1 << kSumOutGamma : 0) |
             (gr.out_beta != nullptr || one_gate ? 1 << kSumOutBeta : 0) |
             (gr.in_gamma != nullptr ? 1 << kSumInGamma : 0) | (gr.in_beta != nullptr ? 1 << kSumInBeta : 0);
    // a single gate row's products wait for the finishing launch, which has to know of real tokens
    const bool flags = valid != nullptr && !p.grouped && res->gate != nullptr && (p.want & (1 << kSumOutGamma | 1 << kSumOutBeta)) != 0;
    if (flags) p.want |= 1 << kSeen;
    int32_t status;
    if (res->dtype == UNIF_F32) status = launch_backward<float, float, float>(sh, p, st);
    else if (res->stream_dtype == UNIF_F32 && dh_dtype == UNIF_F32)
        status = launch_backward<float, u16, float>(sh, p, st);
    else if (res->stream_dtype == UNIF_F32) status = launch_backward<float, u16, u16>(sh, p, st);
    else if (dh_dtype == UNIF_F32) status = launch_backward<u16, u16, float>(sh, p, st);
    else status = launch_backward<u16, u16, u16>(sh, p, st);
    if (status != UNIF_OK) return status;
    UNIF_LAUNCH_CHECK();
    if (p.want != 0 || p.dgate != nullptr) {
        const int by_wave = p.group / p.rows <= kFinishWaves;
        const int* const seen = flags ? reinterpret_cast<const int*>(p.part + (size_t)4 * sh.blocks * p.d) : nullptr;
        const ResidualFinish fin{p.N, p.d, sh.blocks, sh.teams(), p.group, p.rows, gate_rows(res), by_wave, p.grouped, p.part,
                                 p.gate_part, res->out_gamma, res->out_beta, res->gate,
                                 {gr.out_gamma, gr.out_beta, gr.in_gamma, gr.in_beta}, gr.gate, seen};
        int64_t shared = p.dgate != nullptr ? std::min<int64_t>(sh.teams() - 1, gate_rows(res)) : 0;
        if (by_wave) shared = (shared + kFinishWaves - 1) / kFinishWaves;
        residual_finish_kernel<<<dim3((unsigned)div_up(p.d, kWave), (unsigned)(4 + shared)), kFinishWaves * kWave, 0,
                                 st>>>(fin);
        UNIF_LAUNCH_CHECK();
    }
    return UNIF_OK;
}

}  // extern "C"

namespace {

int32_t check_balance(const unif_moe_config* c, const unif_moe_balance* b) {
    const int32_t s = check_config(c);
    if (s != UNIF_OK) return s;
    if (b == nullptr || b->tokens_per_group < 0 || !std::isfinite(b->weight)) return UNIF_EINVAL;
    if (c->d_model > 1 << 20) return UNIF_EUNSUPPORTED;   // 32-bit offsets inside 16 rows, threads of a grid
    if (b->unit != UNIF_BALANCE_TOKENS && b->unit != UNIF_BALANCE_BLOCKS) return UNIF_EINVAL;
    return UNIF_OK;
}

constexpr int kBalNC = 4;   // columns per lane
// Groups of up to kBalOnePiece tokens are one workgroup's in the count, which then
// finishes them; longer ones are counted in pieces of at least kBalPiece tokens, at
// most kBalPieces, since every piece's workgroup adds them all before its dl.
constexpr int kBalOnePiece = 1024, kBalPiece = 512, kBalPieces = 256;

struct BalanceShape {
    int group, groups, pieces, piece, waves;   // count
    int cols, slabs, parts, steps;             // gradient
};
int balance_groups(const unif_moe_config* c, const unif_moe_balance* b) {
    return b->tokens_per_group > 0 ? div_up(c->n_tokens, b->tokens_per_group) : 1;
}
BalanceShape balance_shape(const unif_moe_config* c, const unif_moe_balance* b, int cus) {
    BalanceShape s;
    const int N = std::max(c->n_tokens, 1);
    s.group = b->tokens_per_group > 0 ? b->tokens_per_group : N;
    s.groups = balance_groups(c, b);
    const int longest = std::min(s.group, N);
    s.piece = longest <= kBalOnePiece ? longest : std::max(kBalPiece, div_up(div_up(longest, kBalPieces), 64) * 64);
    s.pieces = div_up(longest, s.piece);
    s.waves = std::min(kBalWaves, div_up(s.piece, 64));
    // strips of 16 lanes' columns, a wave each, at most four per workgroup (one per
    // SIMD; with up to eight, 50,000 x 1,152, K = 20 153 -> 161 us, K = 36 92 -> 97)
    const int strips = div_up(c->d_model, 16 * kBalNC);
    s.slabs = div_up(strips, kBalStrips);
    s.cols = div_up(strips, s.slabs);
    // Token ranges of whole 16-token steps, for the waves that run at once: more, of
    // which some run in a second round, cost more than the last ones' idle units, and
    // their partial sums more traffic. In an earlier form, 131,072 x 1,024, K = 32: 64
    // ranges 545 us, 128 (all at once) 328, 170 460, 256 372, 512 387; 50,432 x 768, K
    // = 16: 64 184, 128 125, 170 156, 256 129, 512 138.
    const int steps = div_up(N, 16), ranges = std::max(1, cus * (balance_waves(c->n_experts) / s.cols) / s.slabs);
    s.steps = div_up(steps, ranges);
    s.parts = div_up(steps, s.steps);
    return s;
}

struct BalancePlan {
    size_t sums, gloss, dl, part, total;
};
BalancePlan plan_balance(const unif_moe_config* c, const unif_moe_balance* b) {
    const BalanceShape s = balance_shape(c, b, kMaxCus);
    const size_t K = c->n_experts, units = s.pieces > 1 ? (size_t)s.groups * s.pieces : 0;
    Carver cv;
    BalancePlan p;
    p.sums = cv.take(8 * units * (2 * K + 2));
    p.gloss = cv.take(8 * (size_t)s.groups);
    p.dl = cv.take(4 * (size_t)c->n_tokens * (div_up(c->n_experts, 16) * 16));
    p.part = cv.take(4 * (size_t)s.parts * K * c->d_model);
    p.total = cv.cur + 256;
    return p;
}

template <class T, int KT>
void launch_balance_grad(const BalanceShape& s, const BalanceParams& p, unsigned extra, hipStream_t st) {
    const dim3 grid((unsigned)s.parts + extra, (unsigned)s.slabs);
    const unsigned threads = (unsigned)s.cols * kWave;
    if (p.dX != nullptr && p.dW != nullptr && p.dX_in != nullptr)
        balance_grad_kernel<T, KT, kBalNC, 1><<<grid, threads, 0, st>>>(p);
    else if (p.dX != nullptr && p.dW != nullptr)
        balance_grad_kernel<T, KT, kBalNC, 2><<<grid, threads, 0, st>>>(p);
    else
        balance_grad_kernel<T, KT, kBalNC, 0><<<grid, threads, 0, st>>>(p);
}
template <class T>
void launch_balance_grad(const BalanceShape& s, const BalanceParams& p, unsigned extra, hipStream_t st) {
    switch (div_up(p.K, 16)) {
        case 1: return launch_balance_grad<T, 1>(s, p, extra, st);
        case 2: return launch_balance_grad<T, 2>(s, p, extra, st);
        case 3: return launch_balance_grad<T, 3>(s, p, extra, st);
        default: return launch_balance_grad<T, 4>(s, p, extra, st);
    }
}

}  // namespace

extern "C" {

int32_t unif_moe_balance_loss_workspace_size(const unif_moe_config* cfg, const unif_moe_balance* bal, size_t* bytes) {
    if (bytes == nullptr) return UNIF_EINVAL;
    const int32_t s = check_balance(cfg, bal);
    if (s != UNIF_OK) return s;
    *bytes = plan_balance(cfg, bal).total;
    return UNIF_OK;
}

int32_t unif_moe_balance_loss(const unif_moe_config* cfg, const unif_moe_balance* bal, const unif_moe_routing* record,
                              const uint8_t* valid, const void* X, const float* W_router, float* loss, int64_t* counts,
                              const float* dX_in, float* dX, const float* dW_router_in, float* dW_router,
                              void* workspace, size_t workspace_bytes, void* stream) {
    const int32_t s = check_balance(cfg, bal);
    if (s != UNIF_OK) return s;
    const int N = cfg->n_tokens, d = cfg->d_model, K = cfg->n_experts;
    if (loss == nullptr) return UNIF_EINVAL;
    if (N > 0 && (!record_complete(record) || (dX != nullptr && W_router == nullptr) ||
                  (dW_router != nullptr && X == nullptr)))
        return UNIF_EINVAL;
    if ((dX != nullptr || dW_router != nullptr) && d < UNIF_BALANCE_MIN_D) return UNIF_EUNSUPPORTED;
    if ((dX == nullptr && dX_in != nullptr) || (dW_router == nullptr && dW_router_in != nullptr)) return UNIF_EINVAL;
    if (!aligned_to(X, elem_size(cfg->dtype)) || !aligned_to(counts, 8)) return UNIF_EINVAL;
    for (const void* q : {(const void*)W_router, (const void*)loss, (const void*)dX_in, (const void*)dX,
                          (const void*)dW_router_in, (const void*)dW_router})
        if (!aligned_to(q, 4)) return UNIF_EINVAL;
    const BalancePlan plan = plan_balance(cfg, bal);
    if (workspace == nullptr || workspace_bytes < plan.total) return UNIF_EWORKSPACE;
    const size_t nd = (size_t)N * d, wb = 4 * (size_t)(K + 1) * d;
    static const unif_moe_routing no_record{};
    const unif_moe_routing& rec = N > 0 ? *record : no_record;
    const Span no(nullptr, 0);
    const Span out[] = {Span(loss, 4), Span(counts, 8 * (size_t)balance_groups(cfg, bal) * (K + 1)), Span(dX, 4 * nd),
                        Span(dW_router, wb), Span(workspace, plan.total)};
    const Span partner[] = {no, no, Span(dX_in, 4 * nd), Span(dW_router_in, wb), no};
    const Span in[] = {Span(valid, N), Span(X, nd * elem_size(cfg->dtype)), Span(W_router, wb),
                       Span(rec.alpha, 4 * (size_t)N), Span(rec.n_shared, 4 * (size_t)N),
                       Span(rec.shared_mask, 8 * (size_t)N), Span(rec.n_res, 4 * (size_t)N),
                       Span(rec.expert_ids, 4 * (size_t)N * K), Span(rec.weights, 4 * (size_t)N * K)};
    if (!apart(out, partner, in)) return UNIF_EINVAL;
    const BalanceShape sh = balance_shape(cfg, bal, std::min(cu_count(), kMaxCus));
    char* ws = align_base(workspace);
    BalanceParams p{};
    p.N = N;
    p.d = d;
    p.K = K;
    p.B = cfg->n_blocks;
    p.group = sh.group;
    p.groups = sh.groups;
    p.pieces = sh.pieces;
    p.piece = sh.piece;
    p.blocks = bal->unit == UNIF_BALANCE_BLOCKS;
    p.past = 4 * nd > kCacheBytes;
    p.weight = bal->weight;
    p.valid = valid;
    p.nsh = rec.n_shared;
    p.nres = rec.n_res;
    p.eids = rec.expert_ids;
    p.wts = rec.weights;
    p.X = X;
    p.Wr = W_router;
    p.dX_in = dX_in;
    p.dX = dX;
    p.dW_in = dW_router_in;
    p.dW = dW_router;
    p.loss = loss;
    p.counts = counts;
    p.sums = reinterpret_cast<uint64_t*>(ws + plan.sums);
    p.gloss = reinterpret_cast<double*>(ws + plan.gloss);
    p.part = reinterpret_cast<float*>(ws + plan.part);
    p.parts = N > 0 ? sh.parts : 0;
    p.KP = div_up(K, 16) * 16;
    const bool grads = N > 0 && (dX != nullptr || dW_router != nullptr);
    p.dl = grads ? reinterpret_cast<float*>(ws + plan.dl) : nullptr;
    p.steps = sh.steps;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (sh.groups > 0) {
        const size_t lds = sizeof(float) * sh.waves * (size_t)balance_wave_words(K);
        const int32_t status = allow_lds(balance_count_kernel, lds + kCountLds);
        if (status != UNIF_OK) return status;
        balance_count_kernel<<<flat_grid((size_t)sh.groups * sh.pieces), (unsigned)sh.waves * kWave, lds, st>>>(p);
        UNIF_LAUNCH_CHECK();
        if (sh.pieces > 1) {
            const size_t all = kBalWaves * sizeof(float) * (size_t)balance_wave_words(K);
            const int32_t fits = allow_lds(balance_slope_kernel, (grads ? all : 0) + kSlopeLds);
            if (fits != UNIF_OK) return fits;
            balance_slope_kernel<<<flat_grid((size_t)sh.groups * (grads ? sh.pieces : 1)), kWave * kBalWaves, grads ? all : 0, st>>>(p);
            UNIF_LAUNCH_CHECK();
        }
    }
    // The groups' mean: with one group it is written already, else beside the
    // gradients where those are wanted.
    const bool mean = sh.groups != 1;
    if (mean && !grads) {
        balance_mean_kernel<<<1, 1024, 0, st>>>(p);
        UNIF_LAUNCH_CHECK();
    }
    if (grads) {
        if (cfg->dtype == UNIF_BF16) launch_balance_grad<u16>(sh, p, mean, st);
        else launch_balance_grad<float>(sh, p, mean, st);
        UNIF_LAUNCH_CHECK();
    }
    if (dW_router != nullptr) {
        balance_dw_sum_kernel<<<(unsigned)ceil_div_sz((size_t)(K + 1) * d, kWave), kWave * kBalSumWaves, 0, st>>>(p);
        UNIF_LAUNCH_CHECK();
    }
    return UNIF_OK;
}

}  // extern "C"
