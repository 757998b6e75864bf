// C entries of the operators of a worker's own training step (include/adpsgd.h): checks of arguments, then launches.
#include <cmath>
#include <cstring>
#include <limits>
#include <new>
#include <string>
#include <vector>

#include "handle.hpp"
#include "operators.hpp"

using namespace adpsgd_impl;

namespace {

int refuse(const char* what) { return fail(nullptr, ADPSGD_ERR_ARG, what); }
int ended(hipError_t e, const char* what) { return e == hipSuccess ? ADPSGD_OK : hip_fail(nullptr, e, what); }
// Nothing is thrown across the C boundary.
template <class F>
int guarded(const F& f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return ADPSGD_ERR_ARG;
    } catch (...) {
        return ADPSGD_ERR_STATE;
    }
}

int64_t size_of(int32_t type) { return type == ADPSGD_TYPE_F32 ? 4 : 2; }
bool is_type(int32_t t) { return t == ADPSGD_TYPE_F32 || t == ADPSGD_TYPE_BF16 || t == ADPSGD_TYPE_F16; }
bool aligned_to(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }

// ---- dense ----
constexpr int64_t kMostSide = int64_t(1) << 31;        // of M, N and K
constexpr int64_t kMostStride = int64_t(1) << 22;      // a tile's rows are addressed with 32-bit offsets from its first
constexpr int64_t kMostTiles = int64_t(1) << 22;       // of 64 x 64, and with them blocks of a launch

bool dense_sizes(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 1 || K < 1 || M >= kMostSide || N >= kMostSide || K >= kMostSide) return false;
    const int64_t m = (M + 63) / 64, n = (N + 63) / 64, k = (K + 63) / 64;
    return m <= kMostTiles && n <= kMostTiles && k <= kMostTiles && m * n <= kMostTiles && m * k <= kMostTiles && n * k <= kMostTiles;
}
int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

struct BackwardSpace {
    int64_t dz, sums, partial, bytes;       // where they begin
};
BackwardSpace backward_space(int64_t M, int64_t N, int64_t K) {
    BackwardSpace b{};
    b.dz = 0;
    b.sums = up256(2 * M * N);
    b.partial = b.sums + up256(dense_sums_bytes(M, N));
    b.bytes = b.partial + up256(std::max(dense_partial_bytes(M, K, N), dense_partial_bytes(N, K, M)));
    return b;
}

const char* dense_fault(const adpsgd_dense_t* o) {
    if (!o) return "dense: no arguments";
    if (o->type != ADPSGD_TYPE_BF16 && o->type != ADPSGD_TYPE_F16) return "dense: type must be BF16 or F16";
    if (o->activation < ADPSGD_ACT_NONE || o->activation > ADPSGD_ACT_SILU) return "dense: unknown activation";
    if (!dense_sizes(o->M, o->N, o->K)) return "dense: M >= 0, N >= 1, K >= 1, and no product of two of them over 2^34";
    if (o->ldx < o->K || o->ldw < (o->w_transposed ? o->N : o->K) || (o->r && o->ldr < o->N)) return "dense: a leading dimension is too small";
    if (o->ldx > kMostStride || o->ldw > kMostStride || o->ldr > kMostStride || o->N > kMostStride || o->K > kMostStride)
        return "dense: rows of more than 2^22 elements";
    if (!o->w || (o->M > 0 && !o->x)) return "dense: x or w is NULL";
    if (!aligned_to(o->x, 2) || !aligned_to(o->w, 2) || !aligned_to(o->b, 2) || !aligned_to(o->r, 2)) return "dense: a tensor is not aligned to its type";
    return nullptr;
}

// ---- losses ----
bool loss_sizes(int64_t rows, int64_t vocab) {
    return rows >= 0 && vocab >= 1 && vocab <= (int64_t(1) << 30) && rows <= (int64_t(1) << 21) && rows * ((vocab + 4095) / 4096) <= (int64_t(1) << 23);
}
const char* logits_fault(const adpsgd_logits_t* o) {
    if (!o) return "logits: no arguments";
    if (!is_type(o->type)) return "logits: unknown type";
    if (!loss_sizes(o->rows, o->vocab)) return "logits: rows <= 2^21, 1 <= vocab <= 2^30 and rows * ceil(vocab / 4096) <= 2^23";
    if (o->ld < o->vocab) return "logits: the leading dimension is smaller than the vocabulary";
    if (o->ld > (int64_t(1) << 40)) return "logits: the leading dimension is too large";
    if (o->rows > 0 && (!o->z || !o->tokens)) return "logits: z or tokens is NULL";
    if (!aligned_to(o->z, size_of(o->type)) || !aligned_to(o->tokens, 8)) return "logits: a tensor is not aligned to its type";
    if (!o->workspace || !aligned16(o->workspace) || o->workspace_bytes < loss_workspace_bytes(o->rows, o->vocab)) return "logits: workspace missing, not 16-byte aligned or too small";
    return nullptr;
}
LossRows rows_of(const adpsgd_logits_t* o) { return LossRows{o->type, o->rows, o->vocab, o->ld, o->z, o->tokens}; }

}  // namespace

extern "C" int64_t adpsgd_dense_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t backward) {
    if (!dense_sizes(M, N, K)) return -1;
    return backward ? backward_space(M, N, K).bytes : up256(dense_partial_bytes(M, N, K));
}

extern "C" int adpsgd_dense_forward(const adpsgd_dense_t* o, void* y, uint16_t* slope, void* stream) {
    return guarded([&]() -> int {
        if (const char* why = dense_fault(o)) return refuse(why);
        if (o->M == 0) return ADPSGD_OK;
        if (!y || !aligned_to(y, 2) || !aligned_to(slope, 2)) return refuse("dense: y is NULL, or not aligned to its type");
        const int64_t bytes = up256(dense_partial_bytes(o->M, o->N, o->K));
        if (o->workspace_bytes < bytes || (bytes > 0 && (!o->workspace || !aligned16(o->workspace)))) return refuse("dense: workspace missing, not 16-byte aligned or too small");
        DenseGemm g{};
        g.a = o->x; g.lda = o->ldx; g.a_outer = false;
        g.b = o->w; g.ldb = o->ldw; g.b_outer = o->w_transposed != 0;
        g.I = o->M; g.J = o->N; g.K = o->K;
        g.act = o->activation;
        g.bias = o->b; g.res = o->r; g.ldres = o->ldr;
        g.out = y; g.slope = slope;
        g.partial = static_cast<float*>(o->workspace); g.partial_bytes = bytes;
        return ended(launch_dense_gemm(o->type, g, static_cast<hipStream_t>(stream)), "dense forward");
    });
}

extern "C" int adpsgd_dense_backward(const adpsgd_dense_t* o, const void* dy, int64_t lddy, const uint16_t* slope, void* dx, void* dw, void* db,
                                     void* stream) {
    return guarded([&]() -> int {
        if (const char* why = dense_fault(o)) return refuse(why);
        if (o->M > 0 && !dy) return refuse("dense: dy is NULL");
        if (lddy < o->N || lddy > kMostStride) return refuse("dense: the leading dimension of dy is not N .. 2^22");
        if (!slope && o->M > 0 && o->activation != ADPSGD_ACT_NONE) return refuse("dense: the backward call of an activation needs the slopes of the forward call");
        if (!aligned_to(dy, 2) || !aligned_to(slope, 2) || !aligned_to(dx, 2) || !aligned_to(dw, 2) || !aligned_to(db, 2)) return refuse("dense: a tensor is not aligned to its type");
        const BackwardSpace at = backward_space(o->M, o->N, o->K);
        if (o->workspace_bytes < at.bytes || (at.bytes > 0 && (!o->workspace || !aligned16(o->workspace)))) return refuse("dense: workspace missing, not 16-byte aligned or too small");
        hipStream_t s = static_cast<hipStream_t>(stream);
        char* ws = static_cast<char*>(o->workspace);
        const void* dz = dy;
        int64_t lddz = lddy;
        const bool own = o->activation != ADPSGD_ACT_NONE && (dx || dw);
        if (own) {
            dz = ws + at.dz;
            lddz = o->N;
        }
        if (own || db) {
            const uint16_t* of = o->activation == ADPSGD_ACT_NONE ? nullptr : slope;
            hipError_t e = launch_dense_dz(o->type, dy, lddy, of, own ? ws + at.dz : nullptr, db, reinterpret_cast<double*>(ws + at.sums), o->M, o->N, s);
            if (e != hipSuccess) return hip_fail(nullptr, e, "dense backward");
        }
        DenseGemm g{};
        g.act = ADPSGD_ACT_NONE;
        g.partial = reinterpret_cast<float*>(ws + at.partial);
        g.partial_bytes = at.bytes - at.partial;
        if (dx && o->M > 0) {
            g.a = dz; g.lda = lddz; g.a_outer = false;
            g.b = o->w; g.ldb = o->ldw; g.b_outer = o->w_transposed == 0;
            g.I = o->M; g.J = o->K; g.K = o->N;
            g.out = dx;
            hipError_t e = launch_dense_gemm(o->type, g, s);
            if (e != hipSuccess) return hip_fail(nullptr, e, "dense backward");
        }
        if (dw) {
            g.a_outer = g.b_outer = true;
            g.K = o->M;
            g.out = dw;
            if (o->w_transposed) {
                g.a = o->x; g.lda = o->ldx; g.I = o->K;
                g.b = dz; g.ldb = lddz; g.J = o->N;
            } else {
                g.a = dz; g.lda = lddz; g.I = o->N;
                g.b = o->x; g.ldb = o->ldx; g.J = o->K;
            }
            hipError_t e = launch_dense_gemm(o->type, g, s);
            if (e != hipSuccess) return hip_fail(nullptr, e, "dense backward");
        }
        return ADPSGD_OK;
    });
}

extern "C" int64_t adpsgd_loss_workspace_bytes(int64_t rows, int64_t vocab) { return loss_sizes(rows, vocab) ? loss_workspace_bytes(rows, vocab) : -1; }

extern "C" int adpsgd_token_log_probs(const adpsgd_logits_t* o, float* log_probs, void* stream) {
    return guarded([&]() -> int {
        if (const char* why = logits_fault(o)) return refuse(why);
        if (o->rows > 0 && (!log_probs || !aligned_to(log_probs, 4))) return refuse("token_log_probs: log_probs is NULL or not aligned");
        return ended(launch_log_probs(rows_of(o), log_probs, o->workspace, static_cast<hipStream_t>(stream)), "token_log_probs");
    });
}

extern "C" int adpsgd_policy_loss(const adpsgd_logits_t* o, const float* old_log_probs, const float* advantages, const float* ref_log_probs, float clip_low,
                                  float clip_high, float kl_coef, float* loss, void* dlogits, float* log_probs, void* stream) {
    return guarded([&]() -> int {
        if (const char* why = logits_fault(o)) return refuse(why);
        if (!(clip_low >= 0.0f && clip_low <= 1.0f && clip_high >= 0.0f && clip_high < INFINITY)) return refuse("policy_loss: 0 <= clip_low <= 1, 0 <= clip_high");
        if (!(kl_coef >= 0.0f && kl_coef < INFINITY)) return refuse("policy_loss: kl_coef must not be negative");
        if (kl_coef > 0.0f && o->rows > 0 && !ref_log_probs) return refuse("policy_loss: a KL term needs ref_log_probs");
        if (!loss || (o->rows > 0 && (!old_log_probs || !advantages || !dlogits || !log_probs))) return refuse("policy_loss: a tensor is NULL");
        if (!aligned_to(old_log_probs, 4) || !aligned_to(advantages, 4) || !aligned_to(ref_log_probs, 4) || !aligned_to(loss, 4) || !aligned_to(log_probs, 4) ||
            !aligned_to(dlogits, size_of(o->type)))
            return refuse("policy_loss: a tensor is not aligned to its type");
        const PolicyTerms t{old_log_probs, advantages, kl_coef > 0.0f ? ref_log_probs : nullptr, clip_low, clip_high, kl_coef};
        return ended(launch_policy(rows_of(o), t, loss, dlogits, log_probs, o->workspace, static_cast<hipStream_t>(stream)), "policy_loss");
    });
}

extern "C" int adpsgd_preference_loss(const adpsgd_logits_t* o, const int64_t* offsets, int64_t pairs, const float* ref_log_probs, float beta,
                                      float label_smoothing, float* loss, void* dlogits, float* log_probs, float* margins, void* stream) {
    return guarded([&]() -> int {
        if (const char* why = logits_fault(o)) return refuse(why);
        if (pairs < 1 || pairs > (int64_t(1) << 23)) return refuse("preference_loss: 1 <= pairs <= 2^23");
        if (!(beta > 0.0f && beta < INFINITY)) return refuse("preference_loss: beta must be positive");
        if (!(label_smoothing >= 0.0f && label_smoothing < 0.5f)) return refuse("preference_loss: 0 <= label_smoothing < 1/2");
        if (!offsets || !ref_log_probs || !loss || !log_probs || !margins || (o->rows > 0 && !dlogits)) return refuse("preference_loss: a tensor is NULL");
        if (!aligned_to(offsets, 8) || !aligned_to(ref_log_probs, 4) || !aligned_to(loss, 4) || !aligned_to(log_probs, 4) || !aligned_to(margins, 4) ||
            !aligned_to(dlogits, size_of(o->type)))
            return refuse("preference_loss: a tensor is not aligned to its type");
        return ended(launch_preference(rows_of(o), offsets, pairs, ref_log_probs, beta, label_smoothing, loss, dlogits, log_probs, margins, o->workspace,
                                       static_cast<hipStream_t>(stream)),
                     "preference_loss");
    });
}

// ---- AdamW ----
struct adpsgd_adamw {
    DevBuf tables;                  // chunks, norm parts, factor, norm
    AdamwArgs a{};
    float* own_norm = nullptr;
    double beta1 = 0.0, beta2 = 0.0;
    int64_t state_length = 0, steps = 0;
};

extern "C" int64_t adpsgd_adamw_state_length(const int64_t* sizes, int32_t tensors) {
    if (tensors < 0 || (tensors > 0 && !sizes)) return -1;
    int64_t n = 0;
    for (int32_t i = 0; i < tensors; ++i) {
        if (sizes[i] < 0 || sizes[i] > (int64_t(1) << 40)) return -1;
        n += (sizes[i] + kAdamwBlock - 1) / kAdamwBlock * kAdamwBlock;
    }
    return n;
}

extern "C" int adpsgd_adamw_create(adpsgd_adamw_t** out, const adpsgd_adamw_opts_t* o) {
    if (out) *out = nullptr;
    return guarded([&]() -> int {
        if (!out || !o) return refuse("adamw: no arguments");
        if (o->tensors < 0 || !is_type(o->param_type) || !is_type(o->grad_type)) return refuse("adamw: unknown type, or a negative number of tensors");
        if (o->state_bits != 8 && o->state_bits != 32) return refuse("adamw: state_bits must be 8 or 32");
        if (!(o->beta1 >= 0.0 && o->beta1 < 1.0 && o->beta2 >= 0.0 && o->beta2 < 1.0 && o->eps > 0.0 && o->eps < INFINITY)) return refuse("adamw: 0 <= beta < 1 and eps > 0");
        if (!(static_cast<float>(o->eps) >= std::numeric_limits<float>::min())) return refuse("adamw: eps is under 2^-126, the smallest normal number of 32 bits");
        const int64_t length = adpsgd_adamw_state_length(o->sizes, o->tensors);
        if (length < 0) return refuse("adamw: a size is negative or over 2^40");
        if (o->tensors > 0 && (!o->params || !o->grads || !o->weight_decay)) return refuse("adamw: params, grads or weight_decay is NULL");
        if (length > 0 && (!o->m || !o->v || !aligned16(o->m) || !aligned16(o->v))) return refuse("adamw: m or v is NULL or not 16-byte aligned");
        if (length > 0 && o->state_bits == 8 && (!o->exponents || !aligned_to(o->exponents, 2))) return refuse("adamw: exponents is NULL or not aligned to 2 bytes");
        std::vector<AdamwChunk> chunks;
        int64_t state = 0;
        const int64_t p_size = size_of(o->param_type), g_size = size_of(o->grad_type);
        for (int32_t i = 0; i < o->tensors; ++i) {
            const int64_t n = o->sizes[i];
            char* p = static_cast<char*>(o->params[i]);
            const char* g = static_cast<const char*>(o->grads[i]);
            float* master = o->masters ? o->masters[i] : nullptr;
            float* to = o->out ? o->out[i] : nullptr;
            const float decay = o->weight_decay[i];
            if (!std::isfinite(decay)) return refuse("adamw: weight_decay is not finite");
            if (n > 0 && (!p || !g || (o->masters && !master) || (o->out && !to))) return refuse("adamw: a tensor is NULL");
            if (!aligned_to(p, p_size) || !aligned_to(g, g_size) || !aligned_to(master, 4) || !aligned_to(to, 4)) return refuse("adamw: a tensor is not aligned to its type");
            if (static_cast<int64_t>(chunks.size()) + n / kAdamwChunk >= (int64_t(1) << 23)) return refuse("adamw: more than 2^35 elements");
            for (int64_t at = 0; at < n; at += kAdamwChunk)
                chunks.push_back(AdamwChunk{p + at * p_size, g + at * g_size, master ? master + at : nullptr, to ? to + at : nullptr, state + at,
                                            static_cast<int32_t>(std::min<int64_t>(n - at, kAdamwChunk)), decay});
            state += (n + kAdamwBlock - 1) / kAdamwBlock * kAdamwBlock;
        }
        const size_t cb = chunks.size() * sizeof(AdamwChunk);
        const size_t own = (kAdamwNormBlocks + 1) * sizeof(double) + sizeof(float);
        std::vector<char> image(cb + own, 0);
        if (cb) std::memcpy(image.data(), chunks.data(), cb);
        adpsgd_adamw* h = new adpsgd_adamw;
        hipError_t e = h->tables.reserve(image.size());
        if (e == hipSuccess) e = hipMemcpy(h->tables.p, image.data(), image.size(), hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            h->tables.release();
            delete h;
            return hip_fail(nullptr, e, "adamw: tables");
        }
        char* at = static_cast<char*>(h->tables.p);
        h->a.chunks = reinterpret_cast<const AdamwChunk*>(at);
        h->a.n_chunks = static_cast<int64_t>(chunks.size());
        h->a.norm_parts = reinterpret_cast<double*>(at + cb);
        h->a.factor = h->a.norm_parts + kAdamwNormBlocks;
        h->own_norm = reinterpret_cast<float*>(h->a.factor + 1);
        h->a.param_type = o->param_type;
        h->a.grad_type = o->grad_type;
        h->a.bits = o->state_bits;
        h->a.masters = o->masters != nullptr;
        h->a.direction = o->out != nullptr;
        h->a.m = o->m;
        h->a.v = o->v;
        h->a.exponents = o->exponents;
        h->a.beta1 = static_cast<float>(o->beta1);
        h->a.beta2 = static_cast<float>(o->beta2);
        h->a.beta1_64 = o->beta1;
        h->a.beta2_64 = o->beta2;
        h->a.rest1_64 = 1.0 - o->beta1;
        h->a.rest2_64 = 1.0 - o->beta2;
        h->a.rest1 = static_cast<float>(1.0 - o->beta1);
        h->a.rest2 = static_cast<float>(1.0 - o->beta2);
        h->a.eps = static_cast<float>(o->eps);
        h->a.root = o->eps < 1e-18 ? 0x1p-15f : 1.0f;
        h->a.seed = o->seed;
        h->beta1 = o->beta1;
        h->beta2 = o->beta2;
        h->state_length = length;
        *out = h;
        return ADPSGD_OK;
    });
}

extern "C" void adpsgd_adamw_destroy(adpsgd_adamw_t* h) {
    if (!h) return;
    h->tables.release();
    delete h;
}

extern "C" int adpsgd_adamw_step(adpsgd_adamw_t* h, double lr, double max_norm, double grad_scale, float* norm, void* stream) {
    return guarded([&]() -> int {
        if (!h) return refuse("adamw: no handle");
        if (!(max_norm >= 0.0 && max_norm < INFINITY)) return refuse("adamw: max_norm must be finite and not negative");
        if (!std::isfinite(lr) || !std::isfinite(grad_scale)) return refuse("adamw: lr and grad_scale must be finite");
        if (norm && !(max_norm > 0.0)) return refuse("adamw: the norm is computed where gradients are clipped only");
        if (!aligned_to(norm, 4)) return refuse("adamw: norm is not aligned");
        hipStream_t s = static_cast<hipStream_t>(stream);
        hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
        hipError_t e = hipStreamIsCapturing(s, &capture);
        if (e != hipSuccess) return hip_fail(nullptr, e, "adamw: stream");
        if (capture != hipStreamCaptureStatusNone) return fail(nullptr, ADPSGD_ERR_STATE, "adamw: the stream is being captured, and the number of a step is the host's");
        AdamwArgs a = h->a;
        a.lr = static_cast<float>(lr);
        a.grad_scale = static_cast<float>(grad_scale);
        a.grad_scale_64 = grad_scale;
        a.max_norm = max_norm;
        a.norm = norm ? norm : h->own_norm;
        const int64_t t = h->steps + 1;
        a.step = static_cast<uint64_t>(t);
        a.inv_c1 = static_cast<float>(1.0 / (1.0 - std::pow(h->beta1, static_cast<double>(t))));
        a.inv_c2 = static_cast<float>(1.0 / (1.0 - std::pow(h->beta2, static_cast<double>(t)))) / (a.root * a.root);
        e = launch_adamw(a, s);
        if (e != hipSuccess) return hip_fail(nullptr, e, "adamw step");
        h->steps = t;
        return ADPSGD_OK;
    });
}

extern "C" int adpsgd_adamw_get_steps(const adpsgd_adamw_t* h, int64_t* out) {
    if (!h || !out) return refuse("adamw: no handle, or nowhere to write");
    *out = h->steps;
    return ADPSGD_OK;
}
extern "C" int adpsgd_adamw_set_steps(adpsgd_adamw_t* h, int64_t steps) {
    if (!h || steps < 0) return refuse("adamw: no handle, or a negative number of steps");
    h->steps = steps;
    return ADPSGD_OK;
}

extern "C" int adpsgd_adamw_get_moments(adpsgd_adamw_t* h, uint16_t* m, uint16_t* v, void* stream) {
    return guarded([&]() -> int {
        if (!h || (h->state_length > 0 && (!m || !v))) return refuse("adamw: no handle, or nowhere to write");
        if (h->a.bits != 8) return fail(nullptr, ADPSGD_ERR_STATE, "adamw: a state of 32 bits is the caller's own m and v");
        if (!aligned_to(m, 2) || !aligned_to(v, 2)) return refuse("adamw: a tensor is not aligned to its type");
        return ended(launch_adamw_get(h->a.m, h->a.v, h->a.exponents, h->state_length, m, v, static_cast<hipStream_t>(stream)), "adamw moments");
    });
}
extern "C" int adpsgd_adamw_set_moments(adpsgd_adamw_t* h, const float* m, const float* v, void* stream) {
    return guarded([&]() -> int {
        if (!h || (h->state_length > 0 && (!m || !v))) return refuse("adamw: no handle, or nothing to read");
        if (h->a.bits != 8) return fail(nullptr, ADPSGD_ERR_STATE, "adamw: a state of 32 bits is the caller's own m and v");
        if (!aligned_to(m, 4) || !aligned_to(v, 4)) return refuse("adamw: a tensor is not aligned to its type");
        return ended(launch_adamw_set(m, v, h->state_length, h->a.m, h->a.v, h->a.exponents, static_cast<hipStream_t>(stream)), "adamw moments");
    });
}
