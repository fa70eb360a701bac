// Host helpers that the library's entry points share: configuration checks,
// workspace carving, launch checks.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>
#include <cstdint>

#include "../../include/unif_moe.h"

namespace unifmoe {

// Checks shared by every entry point (host only, no HIP call).
inline int32_t check_config(const unif_moe_config* c) {
    if (c == nullptr) return UNIF_EINVAL;
    if (c->n_tokens < 0 || c->d_model <= 0 || c->n_experts < 1 || c->n_blocks < 1 || c->block_width < 1)
        return UNIF_EINVAL;
    if (c->max_pairs < 0) return UNIF_EINVAL;
    if (c->dtype != UNIF_F32 && c->dtype != UNIF_BF16) return UNIF_EINVAL;
    if (c->alpha_mode != UNIF_ALPHA_ADAPTIVE && c->alpha_mode != UNIF_ALPHA_FIXED) return UNIF_EINVAL;
    if (c->mass_mode != UNIF_MASS_COUPLED && c->mass_mode != UNIF_MASS_FIXED && c->mass_mode != UNIF_MASS_TOPK)
        return UNIF_EINVAL;
    if (c->select_mode != UNIF_SELECT_PROTOTYPE && c->select_mode != UNIF_SELECT_PREFIX) return UNIF_EINVAL;
    if (!(c->mass_threshold > 0.0f && c->mass_threshold <= 1.0f)) return UNIF_EINVAL;
    if (c->max_shared < 0 || c->max_shared > c->n_blocks) return UNIF_EINVAL;
    if (c->alpha_mode == UNIF_ALPHA_ADAPTIVE && c->n_blocks < 2) return UNIF_EINVAL;
    if (c->alpha_mode == UNIF_ALPHA_FIXED && !(c->alpha_fixed >= 0.0f && c->alpha_fixed <= 1.0f))
        return UNIF_EINVAL;
    if (c->mass_mode == UNIF_MASS_TOPK && (c->fixed_k < 1 || c->fixed_k > c->n_experts)) return UNIF_EINVAL;
    if (!std::isnan(c->tau) && !(c->tau >= 0.0f && c->tau < 0.5f)) return UNIF_EINVAL;
    if (c->n_blocks > 64 || c->n_experts > 64) return UNIF_EUNSUPPORTED;
    const int64_t N = c->n_tokens, K = c->n_experts, B = c->n_blocks;
    if (N * (K + 1) > INT32_MAX || N * K * B > INT32_MAX) return UNIF_EUNSUPPORTED;
    if (c->dtype == UNIF_BF16 && c->d_model % 32 != 0) return UNIF_EUNSUPPORTED;
    return UNIF_OK;
}

// Workspace carving: regions aligned to 256 bytes.
struct Carver {
    size_t cur = 0;
    size_t take(size_t bytes) {
        cur = (cur + 255) & ~(size_t)255;
        const size_t o = cur;
        cur += bytes;
        return o;
    }
};

inline size_t ceil_div_sz(size_t a, size_t b) { return (a + b - 1) / b; }

// A grid of at least `blocks` workgroups, numbered by flat_block(): the threads
// of a grid's x dimension are limited to 2^32 - 1.
inline dim3 flat_grid(size_t blocks) {
    const size_t x = (size_t)1 << 22;
    return blocks <= x ? dim3((unsigned)blocks) : dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

inline char* align_base(void* ws) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(ws);
    return reinterpret_cast<char*>((a + 255) & ~(uintptr_t)255);
}

// Compute units of the current device (queried at each call; the grids of
// the persistent kernels are sized by it).
inline int cu_count() {
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess) return 256;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
    return n;
}

inline bool record_complete(const unif_moe_routing* r) {
    return r && r->alpha && r->n_shared && r->shared_mask && r->n_res && r->expert_ids && r->weights;
}

#define UNIF_LAUNCH_CHECK()                              \
    do {                                                 \
        if (hipGetLastError() != hipSuccess) return UNIF_EDEVICE; \
    } while (0)

template <class F>
int32_t allow_lds(F* kernel, size_t bytes) {
    if (bytes <= 64 * 1024) return UNIF_OK;
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                            (int)bytes) != hipSuccess)
        return UNIF_EDEVICE;
    return UNIF_OK;
}

}  // namespace unifmoe
