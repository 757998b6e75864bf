/* The operators of a worker's own training step from plain C (no Python, no tensor library): one step of a small policy, a dense
 * layer's logits, the policy loss with its gradient, the layer's backward pass and AdamW, against the same in double. */
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <hip/hip_runtime_api.h>

#include "adpsgd.h"

#define CHECK(cond, code) do { if (!(cond)) { fprintf(stderr, "check failed: %s (line %d): %s\n", #cond, __LINE__, adpsgd_last_error(NULL)); return code; } } while (0)

enum { M = 6, K = 40, N = 24 };

static float up(uint16_t h) {
    const uint32_t u = (uint32_t)h << 16;
    float f;
    memcpy(&f, &u, 4);
    return f;
}
static uint16_t down(float f) {             /* finite: to the nearest, ties to even */
    uint32_t u;
    memcpy(&u, &f, 4);
    return (uint16_t)((u + 0x7FFFu + (u >> 16 & 1u)) >> 16);
}
static void* on_gpu(const void* from, size_t bytes) {
    void* p = NULL;
    if (hipMalloc(&p, bytes) != hipSuccess) return NULL;
    if ((from ? hipMemcpy(p, from, bytes, hipMemcpyHostToDevice) : hipMemset(p, 0, bytes)) != hipSuccess) return NULL;
    return p;
}

int main(void) {
    static uint16_t x[M * K], w[N * K], b[N], z[M * N], dz[M * N], dw[N * K], db[N];
    static float adv[M], logp[M], master[N * K], old[M], norm;
    static double zz[M * N], lp[M], dzz[M * N];
    int64_t tokens[M];
    uint32_t s = 12345;
    for (int i = 0; i < M * K; ++i) x[i] = down((float)((s = s * 1664525u + 1013904223u) >> 16 & 1023) / 512.0f - 1.0f);
    for (int i = 0; i < N * K; ++i) w[i] = down((float)((s = s * 1664525u + 1013904223u) >> 16 & 1023) / 1024.0f - 0.5f);
    for (int i = 0; i < N; ++i) b[i] = down((float)i / 64.0f);
    for (int i = 0; i < M; ++i) {
        tokens[i] = i == 2 ? -1 : (i * 7) % N;
        adv[i] = (float)i - 2.5f;
    }
    for (int i = 0; i < N * K; ++i) master[i] = up(w[i]);

    void *dx_ = on_gpu(x, sizeof x), *dw_ = on_gpu(w, sizeof w), *db_ = on_gpu(b, sizeof b), *dz_ = on_gpu(NULL, sizeof z), *dtok = on_gpu(tokens, sizeof tokens);
    void *dgrad = on_gpu(NULL, sizeof dz), *dadv = on_gpu(adv, sizeof adv), *dold = on_gpu(NULL, sizeof old), *dlogp = on_gpu(NULL, sizeof logp), *dloss = on_gpu(NULL, 4);
    void *dgw = on_gpu(NULL, sizeof dw), *dgb = on_gpu(NULL, sizeof db), *dmaster = on_gpu(master, sizeof master), *dnorm = on_gpu(NULL, 4);
    int64_t dense_bytes = adpsgd_dense_workspace_bytes(M, N, K, 0), back_bytes = adpsgd_dense_workspace_bytes(M, N, K, 1), loss_bytes = adpsgd_loss_workspace_bytes(M, N);
    if (back_bytes > dense_bytes) dense_bytes = back_bytes;
    CHECK(dense_bytes > 0 && loss_bytes > 0, 1);
    void *space = on_gpu(NULL, (size_t)dense_bytes), *loss_space = on_gpu(NULL, (size_t)loss_bytes);
    CHECK(dx_ && dw_ && db_ && dz_ && dtok && dgrad && dadv && dold && dlogp && dloss && dgw && dgb && dmaster && dnorm && space && loss_space, 2);
    hipStream_t stream;
    CHECK(hipStreamCreate(&stream) == hipSuccess, 3);

    adpsgd_dense_t o = {0};
    o.type = ADPSGD_TYPE_BF16;
    o.M = M; o.N = N; o.K = K;
    o.x = dx_; o.ldx = K; o.w = dw_; o.ldw = K; o.b = db_;
    o.workspace = space; o.workspace_bytes = dense_bytes;
    CHECK(adpsgd_dense_forward(&o, dz_, NULL, stream) == ADPSGD_OK, 4);
    adpsgd_logits_t l = {0};
    l.type = ADPSGD_TYPE_BF16;
    l.rows = M; l.vocab = N; l.z = dz_; l.ld = N; l.tokens = dtok;
    l.workspace = loss_space; l.workspace_bytes = loss_bytes;
    CHECK(adpsgd_token_log_probs(&l, dold, stream) == ADPSGD_OK, 5);
    CHECK(adpsgd_policy_loss(&l, dold, dadv, NULL, 0.2f, 0.2f, 0.0f, dloss, dgrad, dlogp, stream) == ADPSGD_OK, 6);
    CHECK(adpsgd_dense_backward(&o, dgrad, N, NULL, NULL, dgw, dgb, stream) == ADPSGD_OK, 7);
    adpsgd_adamw_opts_t a = {0};
    const int64_t size = N * K;
    void* const params[] = {dw_};
    const void* const grads[] = {dgw};
    float* const masters[] = {dmaster};
    const float decay[] = {0.1f};
    a.tensors = 1;
    a.param_type = a.grad_type = ADPSGD_TYPE_BF16;
    a.state_bits = 32;
    a.sizes = &size; a.params = params; a.grads = grads; a.masters = masters; a.weight_decay = decay;
    a.beta1 = 0.9; a.beta2 = 0.999; a.eps = 1e-8;
    const size_t state = sizeof(float) * (size_t)adpsgd_adamw_state_length(&size, 1);
    a.m = on_gpu(NULL, state);
    a.v = on_gpu(NULL, state);
    adpsgd_adamw_t* opt = NULL;
    CHECK(a.m && a.v && adpsgd_adamw_create(&opt, &a) == ADPSGD_OK, 8);
    CHECK(adpsgd_adamw_step(opt, 1e-2, 1e6, 1.0, dnorm, stream) == ADPSGD_OK, 9);
    CHECK(hipStreamSynchronize(stream) == hipSuccess, 10);
    float loss = 0.0f;
    static uint16_t w1[N * K];
    CHECK(hipMemcpy(z, dz_, sizeof z, hipMemcpyDeviceToHost) == hipSuccess && hipMemcpy(dz, dgrad, sizeof dz, hipMemcpyDeviceToHost) == hipSuccess &&
          hipMemcpy(dw, dgw, sizeof dw, hipMemcpyDeviceToHost) == hipSuccess && hipMemcpy(db, dgb, sizeof db, hipMemcpyDeviceToHost) == hipSuccess &&
          hipMemcpy(logp, dlogp, sizeof logp, hipMemcpyDeviceToHost) == hipSuccess && hipMemcpy(old, dold, sizeof old, hipMemcpyDeviceToHost) == hipSuccess &&
          hipMemcpy(&loss, dloss, 4, hipMemcpyDeviceToHost) == hipSuccess && hipMemcpy(master, dmaster, sizeof master, hipMemcpyDeviceToHost) == hipSuccess &&
          hipMemcpy(w1, dw_, sizeof w1, hipMemcpyDeviceToHost) == hipSuccess && hipMemcpy(&norm, dnorm, 4, hipMemcpyDeviceToHost) == hipSuccess, 11);

    const double h = 1.0 / 256.0;           /* half a step of bfloat16, relative to the value */
    double mean = 0.0;
    for (int i = 0; i < M; ++i) {
        for (int j = 0; j < N; ++j) {
            double sum = up(b[j]), most = fabs(sum);
            for (int k = 0; k < K; ++k) {
                sum += (double)up(x[i * K + k]) * up(w[j * K + k]);
                most += fabs((double)up(x[i * K + k]) * up(w[j * K + k]));
            }
            CHECK(fabs(up(z[i * N + j]) - sum) <= h * fabs(sum) + 1e-5 * most, 12);
            zz[i * N + j] = up(z[i * N + j]);           /* what the losses read */
        }
        double total = 0.0;
        for (int j = 0; j < N; ++j) total += exp(zz[i * N + j]);
        lp[i] = tokens[i] < 0 ? 0.0 : zz[i * N + tokens[i]] - log(total);
        CHECK(fabs(logp[i] - lp[i]) <= 2e-6 && fabs(old[i] - lp[i]) <= 2e-6, 13);
        for (int j = 0; j < N; ++j) {       /* the ratio is 1 but for roundings: nothing is clipped */
            const double c = tokens[i] < 0 ? 0.0 : -adv[i] / (M - 1.0);
            dzz[i * N + j] = c * ((j == tokens[i]) - exp(zz[i * N + j]) / total);
            CHECK(fabs(up(dz[i * N + j]) - dzz[i * N + j]) <= h * fabs(dzz[i * N + j]) + 4e-6 * fabs(c), 14);
        }
        mean -= tokens[i] < 0 ? 0.0 : adv[i] / (M - 1.0);
    }
    CHECK(fabs(loss - mean) <= 1e-5, 15);
    double squares = 0.0;
    for (int j = 0; j < N; ++j) {
        double sb = 0.0, mb = 0.0;
        for (int i = 0; i < M; ++i) {
            sb += up(dz[i * N + j]);
            mb += fabs(up(dz[i * N + j]));
        }
        CHECK(fabs(up(db[j]) - sb) <= h * fabs(sb) + 1e-6 * mb, 16);
        for (int k = 0; k < K; ++k) {
            double sum = 0.0, most = 0.0;
            for (int i = 0; i < M; ++i) {
                sum += (double)up(dz[i * N + j]) * up(x[i * K + k]);
                most += fabs((double)up(dz[i * N + j]) * up(x[i * K + k]));
            }
            const double g = up(dw[j * K + k]), before = up(w[j * K + k]);
            CHECK(fabs(g - sum) <= h * fabs(sum) + 1e-5 * most, 17);
            squares += g * g;
            const double u = g / (fabs(g) + 1e-8);       /* the first step: m and v over their bias are g and g^2 */
            const double want = before - 1e-2 * (u + 0.1f * before);
            CHECK(fabs(master[j * K + k] - want) <= 1e-7 + (fabs(g) < 1e-12 ? 1e-2 : 0.0), 18);
            CHECK(w1[j * K + k] == down(master[j * K + k]), 19);
        }
    }
    CHECK(fabs(norm - sqrt(squares)) <= 1e-6 * sqrt(squares), 20);
    int64_t steps = 0;
    CHECK(adpsgd_adamw_get_steps(opt, &steps) == ADPSGD_OK && steps == 1, 21);
    CHECK(adpsgd_adamw_step(opt, 1e-2, -1.0, 1.0, NULL, stream) == ADPSGD_ERR_ARG && strstr(adpsgd_last_error(NULL), "max_norm"), 22);
    adpsgd_adamw_destroy(opt);
    void* all[] = {dx_, dw_, db_, dz_, dtok, dgrad, dadv, dold, dlogp, dloss, dgw, dgb, dmaster, dnorm, space, loss_space, a.m, a.v};
    for (size_t i = 0; i < sizeof all / sizeof *all; ++i) CHECK(hipFree(all[i]) == hipSuccess, 23);
    CHECK(hipStreamDestroy(stream) == hipSuccess, 24);
    puts("c abi operators ok");
    return 0;
}
