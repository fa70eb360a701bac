/* Drives the host code of the operators around the layer with a stand-in for
 * the HIP runtime that launches nothing: every call of a grid of sizes is
 * validated, planned and "launched", and each launch is checked against the
 * limits of the device (threads of a workgroup and of a grid's dimensions, LDS)
 * and of the call's workspace query. Built with the host code under
 * AddressSanitizer by tests/test_ops_host_asan.py; device pointers are
 * addresses that nothing on the host may touch. Prints "ops host paths ok
 * <calls> <launches>" at the end. */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "unif_moe_ops.h"

static long calls = 0, launches = 0, bad = 0;
static char what[160];

/* The HIP calls that the host code makes. */
typedef struct { uint32_t x, y, z; } dim3_t;
static dim3_t grid_s, block_s;
static size_t lds_s;
static void* stream_s;

void** __hipRegisterFatBinary(const void* d) { static void* h; (void)d; return &h; }
void __hipUnregisterFatBinary(void** h) { (void)h; }
void __hipRegisterFunction(void** m, const void* f, char* n, const char* d, unsigned t, void* a, void* b, void* c, void* e,
                           int* w) { (void)m; (void)f; (void)n; (void)d; (void)t; (void)a; (void)b; (void)c; (void)e; (void)w; }
void __hipRegisterVar(void** m, void* v, char* n, const char* d, int e, size_t s, int c, int g) {
    (void)m; (void)v; (void)n; (void)d; (void)e; (void)s; (void)c; (void)g;
}
int __hipPushCallConfiguration(dim3_t g, dim3_t b, size_t lds, void* st) { grid_s = g; block_s = b; lds_s = lds; stream_s = st; return 0; }
int __hipPopCallConfiguration(dim3_t* g, dim3_t* b, size_t* lds, void** st) { *g = grid_s; *b = block_s; *lds = lds_s; *st = stream_s; return 0; }
int hipLaunchKernel(const void* f, dim3_t g, dim3_t b, void** args, size_t lds, void* st) {
    (void)f; (void)args; (void)st;
    ++launches;
    const uint64_t threads = (uint64_t)b.x * b.y * b.z;
    if (threads == 0 || threads > 1024 || g.x == 0 || g.y == 0 || g.z == 0 || (uint64_t)g.x * b.x > 0xffffffffull ||
        g.y > 65535 || g.z > 65535 || lds > 160 * 1024 - 16 * 1024) {
        ++bad;
        printf("%s: grid %u x %u x %u, block %u, lds %zu\n", what, g.x, g.y, g.z, b.x, lds);
    }
    return 0;
}
int hipGetLastError(void) { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipDeviceGetAttribute(int* v, int a, int d) { (void)a; (void)d; *v = 256; return 0; }
int hipFuncSetAttribute(const void* f, int a, int v) { (void)f; (void)a; (void)v; return 0; }

static void expect(int32_t got, int32_t want) {
    ++calls;
    if (got != want) {
        ++bad;
        printf("%s: returned %d, expected %d\n", what, (int)got, (int)want);
    }
}

/* Device addresses far apart: 2^48 bytes each. */
static void* at(int i) { return (void*)(((uintptr_t)i + 1) << 48); }

static void residual(int n, int d, int dtype, int stream, int dh, int per, int gate, int out, int in) {
    unif_moe_residual r;
    memset(&r, 0, sizeof r);
    r.n_tokens = n; r.d_model = d; r.dtype = dtype; r.stream_dtype = stream; r.out_norm = out; r.in_norm = in;
    r.tokens_per_gate = per; r.out_eps = r.in_eps = 1e-6f; r.residual_scale = 1.0f;
    if (out) { r.out_gamma = at(0); r.out_beta = at(1); }
    if (in) { r.in_gamma = at(2); r.in_beta = at(3); }
    if (gate) r.gate = at(4);
    snprintf(what, sizeof what, "residual n=%d d=%d dtype=%d stream=%d dh=%d per=%d", n, d, dtype, stream, dh, per);
    expect(unif_moe_residual_forward(&r, at(5), at(6), at(7), at(8), in ? at(9) : NULL, NULL), UNIF_OK);
    size_t bytes = 0;
    expect(unif_moe_residual_backward_workspace_size(&r, &bytes), UNIF_OK);
    unif_moe_residual_grads g;
    memset(&g, 0, sizeof g);
    if (out) { g.out_gamma = at(10); g.out_beta = at(11); }
    if (in) { g.in_gamma = at(12); g.in_beta = at(13); }
    if (gate) g.gate = at(14);
    expect(unif_moe_residual_backward(&r, in ? at(5) : NULL, at(6), at(7), at(15), in ? at(16) : NULL, dh, at(17), at(18),
                                      &g, at(19), bytes, NULL), UNIF_OK);
    expect(unif_moe_residual_backward(&r, in ? at(5) : NULL, at(6), at(7), at(15), in ? at(16) : NULL, dh, at(17), at(18),
                                      &g, at(19), bytes - 1, NULL), UNIF_EWORKSPACE);
}

static void balance(int n, int d, int K, int dtype, int per, int unit, int32_t want) {
    unif_moe_config c;
    memset(&c, 0, sizeof c);
    c.n_tokens = n; c.d_model = d; c.n_experts = K; c.n_blocks = 4; c.block_width = 64; c.dtype = dtype;
    c.tau = 0.1f; c.mass_threshold = 0.6f; c.max_shared = 4;
    unif_moe_balance b = {per, unit, 0.5f};
    unif_moe_routing rec = {at(0), at(1), at(2), at(3), at(4), at(5)};
    snprintf(what, sizeof what, "balance n=%d d=%d K=%d dtype=%d per=%d", n, d, K, dtype, per);
    size_t bytes = 0;
    expect(unif_moe_balance_loss_workspace_size(&c, &b, &bytes), want == UNIF_EUNSUPPORTED && d < 8 ? UNIF_OK : want);
    if (want != UNIF_OK) bytes = (size_t)1 << 42;
    expect(unif_moe_balance_loss(&c, &b, &rec, at(6), at(7), at(8), at(9), at(10), at(11), at(12), at(13), at(14), at(15),
                                 bytes, NULL), want);
    if (want != UNIF_OK) return;
    expect(unif_moe_balance_loss(&c, &b, &rec, at(6), NULL, NULL, at(9), NULL, NULL, NULL, NULL, NULL, at(15), bytes, NULL),
           UNIF_OK);
    expect(unif_moe_balance_loss(&c, &b, &rec, at(6), at(7), at(8), at(9), at(10), at(11), at(11), at(13), at(13), at(15),
                                 bytes - 1, NULL), UNIF_EWORKSPACE);
}

int main(void) {
    const int ns[] = {0, 1, 2, 63, 64, 1000, 50432, 131072, 10000019, 2147483647};
    const int ds[] = {4, 5, 31, 32, 33, 96, 97, 200, 384, 512, 513, 768, 769, 1000, 1024, 1025, 5120, 8191, 8192};
    const int types[][3] = {{1, 1, 0}, {1, 1, 1}, {1, 0, 0}, {1, 0, 1}, {0, 0, 0}};
    for (size_t i = 0; i < sizeof ns / sizeof *ns; ++i)
        for (size_t j = 0; j < sizeof ds / sizeof *ds; ++j)
            for (int t = 0; t < 5; ++t)
                for (int v = 0; v < 6; ++v) {
                    const int pers[] = {0, 1, 3, 197, 100000, 2147483647};
                    residual(ns[i], ds[j], types[t][0], types[t][1], types[t][2], pers[v], v != 0 || t != 0, (v + t) % 3, v % 3);
                }
    const int Ks[] = {1, 2, 15, 16, 17, 32, 33, 64};
    const int bd[] = {8, 9, 63, 64, 384, 768, 1000, 1024, 4096, 1 << 20};
    for (size_t i = 0; i < sizeof ns / sizeof *ns; ++i)
        for (size_t j = 0; j < sizeof bd / sizeof *bd; ++j)
            for (size_t k = 0; k < sizeof Ks / sizeof *Ks; ++k)
                for (int v = 0; v < 5; ++v) {
                    const int pers[] = {0, 1, 128, 1025, 5000000};
                    const int fits = (int64_t)ns[i] * (Ks[k] + 1) <= 2147483647 && (int64_t)ns[i] * Ks[k] * 4 <= 2147483647;
                    balance(ns[i], bd[j], Ks[k], v % 2 && bd[j] % 32 == 0, pers[v], v & 1, fits ? UNIF_OK : UNIF_EUNSUPPORTED);
                }
    balance(100, 7, 4, 0, 0, 0, UNIF_EUNSUPPORTED);
    balance(100, (1 << 20) + 32, 4, 1, 0, 0, UNIF_EUNSUPPORTED);
    if (bad == 0) printf("ops host paths ok %ld %ld\n", calls, launches);
    return bad != 0;
}
