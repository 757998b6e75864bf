/* Layer norm, gated projections and the distillation loss from plain C (no Python, no tensor library): h = gated(layer_norm(x)), logits a dense layer
 * of h, the distillation loss with its gradient and all backward calls, against the same in double. */
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <hip/hip_runtime_api.h>

#include "adpsgd.h"

#define CHECK(cond, code) do { if (!(cond)) { fprintf(stderr, "check failed: %s (line %d): %s\n", #cond, __LINE__, adpsgd_last_error(NULL)); return code; } } while (0)

enum { M = 7, D = 40, H = 24, V = 50, E = 5 };

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
static uint32_t seed = 12345;
static float next(void) { return (float)((seed = seed * 1664525u + 1013904223u) >> 16 & 1023) / 512.0f - 1.0f; }
static void* on_gpu(const void* from, size_t bytes) {
    void* p = NULL;
    if (hipMalloc(&p, bytes) != hipSuccess) return NULL;
    if ((from ? hipMemcpy(p, from, bytes, hipMemcpyHostToDevice) : hipMemset(p, 0, bytes)) != hipSuccess) return NULL;
    return p;
}
static int back(void* to, const void* from, size_t bytes) { return hipMemcpy(to, from, bytes, hipMemcpyDeviceToHost) == hipSuccess; }
/* within half a step of bfloat16 and `part` of the sum of magnitudes */
static int near(float got, double want, double most, double part) { return fabs(got - want) <= fabs(want) / 256.0 + part * most + 1e-12; }

int main(void) {
    static uint16_t x[M * D], w[2 * H * D], o[V * H], n[M * D], h[M * H], z[M * V], dz[M * V], dh[M * H], dwo[V * H], dn[M * D], dwg[2 * H * D], dx[M * D];
    static float s[D], t[D], ds[D], dt[D], told[M * E], kl[M], logp[M], loss;
    int64_t tokens[M], entries[M * E];
    for (int i = 0; i < M * D; ++i) x[i] = down(next() + 0.25f);
    for (int i = 0; i < 2 * H * D; ++i) w[i] = down(next() / 4.0f);
    for (int i = 0; i < V * H; ++i) o[i] = down(next() / 2.0f);
    for (int i = 0; i < D; ++i) {
        s[i] = 1.0f + next() / 8.0f;
        t[i] = next() / 8.0f;
    }
    for (int i = 0; i < M; ++i) {
        tokens[i] = i == 3 ? -1 : (i * 11) % V;
        for (int j = 0; j < E; ++j) {
            entries[i * E + j] = i == 5 && j > 2 ? -1 : (i * 13 + j * 7) % V;
            told[i * E + j] = 2.0f * next();
        }
    }
    void *gx = on_gpu(x, sizeof x), *gs = on_gpu(s, sizeof s), *gt = on_gpu(t, sizeof t), *gw = on_gpu(w, sizeof w), *go = on_gpu(o, sizeof o), *gtok = on_gpu(tokens, sizeof tokens);
    void *gent = on_gpu(entries, sizeof entries), *gtold = on_gpu(told, sizeof told), *gn = on_gpu(NULL, sizeof n), *gstats = on_gpu(NULL, 3 * M * 4), *gh = on_gpu(NULL, sizeof h);
    void *gz = on_gpu(NULL, sizeof z), *gdz = on_gpu(NULL, sizeof dz), *gdh = on_gpu(NULL, sizeof dh), *gdo = on_gpu(NULL, sizeof dwo), *gdn = on_gpu(NULL, sizeof dn);
    void *gdw = on_gpu(NULL, sizeof dwg), *gdx = on_gpu(NULL, sizeof dx), *gds = on_gpu(NULL, sizeof ds), *gdt = on_gpu(NULL, sizeof dt), *gkl = on_gpu(NULL, sizeof kl);
    void *glogp = on_gpu(NULL, sizeof logp), *gloss = on_gpu(NULL, 4);
    const int64_t slope_bytes = adpsgd_gated_slopes_bytes(ADPSGD_TYPE_BF16, M, H);
    const int64_t sizes[] = {adpsgd_layer_norm_workspace_bytes(ADPSGD_TYPE_BF16, M, D), adpsgd_gated_workspace_bytes(M, H, D, 0), adpsgd_gated_workspace_bytes(M, H, D, 1),
                             adpsgd_dense_workspace_bytes(M, V, H, 0), adpsgd_dense_workspace_bytes(M, V, H, 1), adpsgd_distillation_workspace_bytes(M, V, E)};
    int64_t bytes = 16;
    for (size_t i = 0; i < sizeof sizes / sizeof *sizes; ++i) {
        CHECK(sizes[i] >= 0, 1);
        if (sizes[i] > bytes) bytes = sizes[i];
    }
    CHECK(slope_bytes == 4 * M * H, 1);
    void *space = on_gpu(NULL, (size_t)bytes), *slopes = on_gpu(NULL, (size_t)slope_bytes);      /* one workspace for all: they follow each other on one stream */
    void* all[] = {gx, gs, gt, gw, go, gtok, gent, gtold, gn, gstats, gh, gz, gdz, gdh, gdo, gdn, gdw, gdx, gds, gdt, gkl, glogp, gloss, space, slopes};
    for (size_t i = 0; i < sizeof all / sizeof *all; ++i) CHECK(all[i], 2);
    hipStream_t stream;
    CHECK(hipStreamCreate(&stream) == hipSuccess, 3);

    adpsgd_layer_norm_t norm = {0};
    norm.type = ADPSGD_TYPE_BF16;
    norm.param_type = ADPSGD_TYPE_F32;
    norm.rows = M; norm.n = D; norm.x = gx; norm.ldx = D; norm.w = gs; norm.b = gt; norm.eps = 1e-5;
    norm.workspace = space; norm.workspace_bytes = bytes;
    adpsgd_dense_t gate = {0}, out = {0};
    gate.type = out.type = ADPSGD_TYPE_BF16;
    gate.activation = ADPSGD_ACT_SILU;
    gate.M = M; gate.N = H; gate.K = D; gate.x = gn; gate.ldx = D; gate.w = gw; gate.ldw = D;
    out.M = M; out.N = V; out.K = H; out.x = gh; out.ldx = H; out.w = go; out.ldw = H;
    gate.workspace = out.workspace = space; gate.workspace_bytes = out.workspace_bytes = bytes;
    adpsgd_logits_t logits = {0};
    logits.type = ADPSGD_TYPE_BF16;
    logits.rows = M; logits.vocab = V; logits.z = gz; logits.ld = V; logits.tokens = gtok;
    logits.workspace = space; logits.workspace_bytes = bytes;
    adpsgd_teacher_t teacher = {0};
    teacher.type = ADPSGD_TYPE_F32;
    teacher.k = E; teacher.tokens = gent; teacher.ld_tokens = E; teacher.z = gtold; teacher.ld = E;
    const double T = 2.0, a = 0.25;
    CHECK(adpsgd_layer_norm_forward(&norm, gn, gstats, stream) == ADPSGD_OK, 4);
    CHECK(adpsgd_gated_forward(&gate, gh, slopes, stream) == ADPSGD_OK, 5);
    CHECK(adpsgd_dense_forward(&out, gz, NULL, stream) == ADPSGD_OK, 6);
    CHECK(adpsgd_distillation_loss(&logits, &teacher, T, a, 1.0, gloss, gdz, gkl, glogp, stream) == ADPSGD_OK, 7);
    CHECK(adpsgd_dense_backward(&out, gdz, V, NULL, gdh, gdo, NULL, stream) == ADPSGD_OK, 8);
    CHECK(adpsgd_gated_backward(&gate, gdh, H, slopes, gdn, gdw, NULL, stream) == ADPSGD_OK, 9);
    CHECK(adpsgd_layer_norm_backward(&norm, gdn, D, gstats, gdx, gds, gdt, stream) == ADPSGD_OK, 10);
    CHECK(hipStreamSynchronize(stream) == hipSuccess, 11);
    CHECK(back(n, gn, sizeof n) && back(h, gh, sizeof h) && back(z, gz, sizeof z) && back(dz, gdz, sizeof dz) && back(dh, gdh, sizeof dh) && back(dn, gdn, sizeof dn) &&
          back(dwg, gdw, sizeof dwg) && back(dx, gdx, sizeof dx) && back(ds, gds, sizeof ds) && back(dt, gdt, sizeof dt) && back(kl, gkl, sizeof kl) &&
          back(logp, glogp, sizeof logp) && back(&loss, gloss, 4), 12);

    /* each call from what the one before it left */
    static double hat[M * D], r[M], g[M * H], u[M * H], dgu[M * 2 * H];
    for (int i = 0; i < M; ++i) {
        double mean = 0.0, var = 0.0;
        for (int k = 0; k < D; ++k) mean += up(x[i * D + k]) / (double)D;
        for (int k = 0; k < D; ++k) var += (up(x[i * D + k]) - mean) * (up(x[i * D + k]) - mean) / D;
        r[i] = 1.0 / sqrt(var + 1e-5);
        for (int k = 0; k < D; ++k) {
            hat[i * D + k] = (up(x[i * D + k]) - mean) * r[i];
            CHECK(near(up(n[i * D + k]), hat[i * D + k] * s[k] + t[k], 4.0, 1e-6), 13);
        }
        for (int j = 0; j < H; ++j) {
            double most = 0.0;
            g[i * H + j] = u[i * H + j] = 0.0;
            for (int k = 0; k < D; ++k) {
                g[i * H + j] += (double)up(n[i * D + k]) * up(w[j * D + k]);
                u[i * H + j] += (double)up(n[i * D + k]) * up(w[(H + j) * D + k]);
                most += fabs((double)up(n[i * D + k]) * up(w[(H + j) * D + k]));
            }
            const double sig = 1.0 / (1.0 + exp(-g[i * H + j])), act = g[i * H + j] * sig;
            CHECK(near(up(h[i * H + j]), act * u[i * H + j], most * (fabs(g[i * H + j]) + 1.0), 1e-5), 14);
            dgu[i * 2 * H + j] = up(dh[i * H + j]) * u[i * H + j] * (sig + act * (1.0 - sig));
            dgu[i * 2 * H + H + j] = up(dh[i * H + j]) * act;
        }
    }
    double total = 0.0;
    for (int i = 0; i < M; ++i) {
        double sT = 0.0, s1 = 0.0, Z = 0.0, div = 0.0;
        for (int v = 0; v < V; ++v) {
            sT += exp(up(z[i * V + v]) / T);
            s1 += exp(up(z[i * V + v]));
        }
        for (int j = 0; j < E; ++j) Z += entries[i * E + j] < 0 ? 0.0 : exp(told[i * E + j] / T);
        static double want[V];
        const int counts = tokens[i] >= 0;
        for (int v = 0; v < V; ++v) want[v] = (1.0 - a) * T * exp(up(z[i * V + v]) / T) / sT + a * exp(up(z[i * V + v])) / s1;
        for (int j = 0; j < E; ++j) {
            const int64_t v = entries[i * E + j];
            if (v < 0) continue;
            const double p = exp(told[i * E + j] / T) / Z;
            div += p * (log(p) - (up(z[i * V + v]) / T - log(sT)));
            want[v] -= (1.0 - a) * T * p;
        }
        if (counts) want[tokens[i]] -= a;
        const double l = counts ? up(z[i * V + tokens[i]]) - log(s1) : 0.0;
        CHECK(fabs(kl[i] - (counts ? div : 0.0)) <= 4e-6 && fabs(logp[i] - l) <= 4e-6, 15);
        total += counts ? ((1.0 - a) * T * T * div - a * l) / (M - 1.0) : 0.0;
        for (int v = 0; v < V; ++v) CHECK(near(up(dz[i * V + v]), counts ? want[v] / (M - 1.0) : 0.0, 1.0, 2e-6), 16);
    }
    CHECK(fabs(loss - total) <= 1e-5, 17);
    for (int j = 0; j < 2 * H; ++j)
        for (int k = 0; k < D; ++k) {
            double sum = 0.0, most = 0.0;
            for (int i = 0; i < M; ++i) {
                sum += dgu[i * 2 * H + j] * up(n[i * D + k]);
                most += fabs(dgu[i * 2 * H + j] * up(n[i * D + k]));
            }
            CHECK(near(up(dwg[j * D + k]), sum, most, 1.0 / 900.0), 18);          /* slopes: 2^-10 */
        }
    for (int i = 0; i < M; ++i) {
        double mg = 0.0, mgh = 0.0;
        for (int k = 0; k < D; ++k) {
            double sum = 0.0, most = 0.0;
            for (int j = 0; j < 2 * H; ++j) {
                sum += dgu[i * 2 * H + j] * up(w[j * D + k]);
                most += fabs(dgu[i * 2 * H + j] * up(w[j * D + k]));
            }
            CHECK(near(up(dn[i * D + k]), sum, most, 1.0 / 900.0), 19);
            mg += (double)up(dn[i * D + k]) * s[k] / D;
            mgh += (double)up(dn[i * D + k]) * s[k] * hat[i * D + k] / D;
        }
        for (int k = 0; k < D; ++k) {
            const double want = r[i] * ((double)up(dn[i * D + k]) * s[k] - mg - hat[i * D + k] * mgh);
            CHECK(near(up(dx[i * D + k]), want, r[i] * (fabs((double)up(dn[i * D + k])) + fabs(mg) + fabs(mgh)), 1e-5), 20);
        }
    }
    for (int k = 0; k < D; ++k) {
        double sw = 0.0, sb = 0.0, most = 0.0;
        for (int i = 0; i < M; ++i) {
            sw += up(dn[i * D + k]) * hat[i * D + k];
            sb += up(dn[i * D + k]);
            most += fabs((double)up(dn[i * D + k])) * (1.0 + fabs(hat[i * D + k]));
        }
        CHECK(fabs(ds[k] - sw) <= 1e-5 * most + 1e-12 && fabs(dt[k] - sb) <= 1e-5 * most + 1e-12, 21);
    }
    CHECK(adpsgd_distillation_loss(&logits, &teacher, -1.0, a, 1.0, gloss, gdz, gkl, glogp, stream) == ADPSGD_ERR_ARG && strstr(adpsgd_last_error(NULL), "temperature"), 22);
    for (size_t i = 0; i < sizeof all / sizeof *all; ++i) CHECK(hipFree(all[i]) == hipSuccess, 23);
    CHECK(hipStreamDestroy(stream) == hipSuccess, 24);
    puts("c abi more operators ok");
    return 0;
}
