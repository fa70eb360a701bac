/* Calls of the operators around the layer that are refused, against a stand-in
 * for the HIP runtime that counts every call made of it: a refused call makes
 * none. Built and run by tests/test_ops_refusals.py; device pointers are
 * addresses that nothing on the host may touch. Prints "ops refusals ok
 * <refused calls>" at the end. */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "unif_moe_ops.h"

static long hip_calls = 0, refused = 0, bad = 0;

/* The HIP calls that the host code makes. */
typedef struct { uint32_t x, y, z; } dim3_t;
void** __hipRegisterFatBinary(const void* d) { static void* h; (void)d; return &h; }
void __hipUnregisterFatBinary(void** h) { (void)h; }
void __hipRegisterFunction(void** m, const void* f, char* n, const char* d, unsigned t, void* a, void* b, void* c, void* e,
                           int* w) { (void)m; (void)f; (void)n; (void)d; (void)t; (void)a; (void)b; (void)c; (void)e; (void)w; }
void __hipRegisterVar(void** m, void* v, char* n, const char* d, int e, size_t s, int c, int g) {
    (void)m; (void)v; (void)n; (void)d; (void)e; (void)s; (void)c; (void)g;
}
int __hipPushCallConfiguration(dim3_t g, dim3_t b, size_t lds, void* st) { (void)g; (void)b; (void)lds; (void)st; ++hip_calls; return 0; }
int __hipPopCallConfiguration(dim3_t* g, dim3_t* b, size_t* lds, void** st) { (void)g; (void)b; *lds = 0; *st = NULL; ++hip_calls; return 0; }
int hipLaunchKernel(const void* f, dim3_t g, dim3_t b, void** args, size_t lds, void* st) {
    (void)f; (void)g; (void)b; (void)args; (void)lds; (void)st;
    ++hip_calls;
    return 0;
}
int hipGetLastError(void) { ++hip_calls; return 0; }
int hipGetDevice(int* d) { *d = 0; ++hip_calls; return 0; }
int hipDeviceGetAttribute(int* v, int a, int d) { (void)a; (void)d; *v = 256; ++hip_calls; return 0; }
int hipFuncSetAttribute(const void* f, int a, int v) { (void)f; (void)a; (void)v; ++hip_calls; return 0; }

static void expect(const char* what, int32_t got, int32_t want) {
    if (got != want || (want != UNIF_OK && hip_calls != 0) || (want == UNIF_OK && hip_calls == 0)) {
        ++bad;
        printf("%s: returned %d, expected %d, %ld HIP calls\n", what, (int)got, (int)want, hip_calls);
    }
    refused += want != UNIF_OK;
    hip_calls = 0;
}

/* Device addresses far apart. */
#define AT(i) ((void*)(((uintptr_t)(i) + 1) << 40))
#define OFF(p, n) ((void*)((char*)(p) + (n)))

static unif_moe_residual res;
static unif_moe_residual_grads grads;
static const void *x, *f, *y_in, *dy, *dh;
static const uint8_t* valid;
static void *y, *h, *dx, *df, *ws;
static size_t bytes;

static void join_defaults(void) {
    memset(&res, 0, sizeof res);
    res.n_tokens = 100; res.d_model = 64; res.dtype = res.stream_dtype = UNIF_BF16;
    res.out_norm = UNIF_ROWNORM_LAYER; res.in_norm = UNIF_ROWNORM_RMS; res.out_eps = res.in_eps = 1e-6f; res.residual_scale = 1.f;
    res.out_gamma = AT(0); res.out_beta = AT(1); res.in_gamma = AT(2); res.in_beta = AT(3); res.gate = AT(4);
    x = AT(5); f = AT(6); valid = AT(7); y = AT(8); h = AT(9);
    y_in = AT(10); dy = AT(11); dh = AT(12); dx = AT(13); df = AT(14); ws = AT(15);
    grads.out_gamma = AT(16); grads.out_beta = AT(17); grads.in_gamma = AT(18); grads.in_beta = AT(19); grads.gate = AT(20);
    unif_moe_residual_backward_workspace_size(&res, &bytes);
}
static int32_t forward(void) { return unif_moe_residual_forward(&res, x, f, valid, y, h, NULL); }
static int32_t backward(void) {
    return unif_moe_residual_backward(&res, y_in, f, valid, dy, dh, UNIF_F32, dx, df, &grads, ws, bytes, NULL);
}
#define FWD(change, want) do { join_defaults(); change; expect("forward " #change, forward(), want); } while (0)
#define BWD(change, want) do { join_defaults(); change; expect("backward " #change, backward(), want); } while (0)

static unif_moe_config cfg;
static unif_moe_balance bal;
static unif_moe_routing rec;
static const unif_moe_routing* record;
static const void* X;
static const float *W, *dX_in, *dW_in;
static float *loss, *dX, *dW;
static int64_t* counts;

static void balance_defaults(void) {
    memset(&cfg, 0, sizeof cfg);
    cfg.n_tokens = 100; cfg.d_model = 64; cfg.n_experts = 4; cfg.n_blocks = 8; cfg.block_width = 64; cfg.dtype = UNIF_BF16;
    cfg.tau = 0.1f; cfg.mass_threshold = 0.6f; cfg.max_shared = 8;
    bal.tokens_per_group = 0; bal.unit = 0; bal.weight = 1.f;
    rec.alpha = AT(0); rec.n_shared = AT(1); rec.shared_mask = AT(2); rec.n_res = AT(3); rec.expert_ids = AT(4); rec.weights = AT(5);
    record = &rec; valid = AT(6); X = AT(7); W = AT(8); loss = AT(9); counts = AT(10); dX_in = AT(11); dX = AT(12); dW_in = AT(13);
    dW = AT(14); ws = AT(15);
    unif_moe_balance_loss_workspace_size(&cfg, &bal, &bytes);
}
static int32_t balance(void) {
    return unif_moe_balance_loss(&cfg, &bal, record, valid, X, W, loss, counts, dX_in, dX, dW_in, dW, ws, bytes, NULL);
}
#define BAL(change, want) do { balance_defaults(); change; expect("balance " #change, balance(), want); } while (0)

int main(void) {
    FWD((void)0, UNIF_OK);
    FWD(res.dtype = 7, UNIF_EINVAL);
    FWD(res.d_model = 9000, UNIF_EUNSUPPORTED);
    FWD(x = f = NULL, UNIF_EINVAL);
    FWD(y = h = NULL, UNIF_EINVAL);
    FWD(y = (void*)f, UNIF_EINVAL);
    FWD(h = (void*)x, UNIF_EINVAL);
    FWD(y = OFF(x, 2), UNIF_EINVAL);
    FWD(h = OFF(res.gate, 128), UNIF_EINVAL);
    FWD(y = (void*)x, UNIF_OK);
    BWD((void)0, UNIF_OK);
    BWD(res.in_gamma = NULL, UNIF_EINVAL);
    BWD(dy = dh = NULL, UNIF_EINVAL);
    BWD(y_in = NULL, UNIF_EINVAL);
    BWD(bytes -= 1, UNIF_EWORKSPACE);
    BWD(ws = NULL, UNIF_EWORKSPACE);
    BWD(df = dx, UNIF_EINVAL);
    BWD(df = (void*)dy, UNIF_EINVAL);
    BWD(dx = OFF(dy, 2), UNIF_EINVAL);
    BWD(ws = (void*)dh, UNIF_EINVAL);
    BWD(grads.gate = (float*)res.gate, UNIF_EINVAL);
    BWD(dx = (void*)dy, UNIF_OK);
    BAL((void)0, UNIF_OK);
    BAL(bal.unit = 2, UNIF_EINVAL);
    BAL(cfg.n_experts = 65, UNIF_EUNSUPPORTED);
    BAL(loss = NULL, UNIF_EINVAL);
    BAL(record = NULL, UNIF_EINVAL);
    BAL(dX = NULL, UNIF_EINVAL);
    BAL(bytes -= 1, UNIF_EWORKSPACE);
    BAL(ws = NULL, UNIF_EWORKSPACE);
    /* overlaps: with inputs, in part with the tensor that is added, with each other */
    BAL(dX = (float*)X, UNIF_EINVAL);
    BAL(dX = OFF(dX_in, 4), UNIF_EINVAL);
    BAL(dW = (float*)W, UNIF_EINVAL);
    BAL(loss = (float*)counts, UNIF_EINVAL);
    BAL(loss = OFF(counts, 8 * 5 - 4), UNIF_EINVAL);
    BAL(loss = OFF(counts, 8 * 5), UNIF_OK);
    BAL(bal.tokens_per_group = 10; loss = OFF(counts, 8 * 5 * 10 - 4), UNIF_EINVAL);
    BAL(bal.tokens_per_group = 10; loss = OFF(counts, 8 * 5 * 10), UNIF_OK);
    BAL(ws = rec.weights, UNIF_EINVAL);
    BAL(dX = dW, UNIF_EINVAL);
    BAL(dX = (float*)dX_in; dW = (float*)dW_in, UNIF_OK);
    if (bad == 0) printf("ops refusals ok %ld\n", refused);
    return bad != 0;
}
