// What the C entries of the training-step operators (api_operators.cpp) and their kernels share.
#pragma once

#include "internal.hpp"

namespace adpsgd_impl {

// ---- dense layers (kernels_dense.hip) ----
struct DenseGemm {                  // D[i][j] = sum_k A(i, k) B(j, k), i < I, j < J, k < K
    const void *a, *b;
    int64_t lda, ldb;
    bool a_outer, b_outer;          // false: (i, k) at a + i lda + k;  true: at a + k lda + i.  b likewise
    const void *a_low, *b_low;      // what a's or b's rounding has left, laid out as a or b; nullptr but for small results of a gated projection's backward pass
    bool a_padded, b_padded;        // rows begin at whole pieces and have zeros up to one behind them
    int64_t b_up;                   // gated products (kernels_gated.hip) only: elements from a gate's weight to its partner's
    int64_t I, J, K;
    int32_t act;
    const void* bias;               // J, or nullptr
    const void* res;                // I x J, or nullptr
    int64_t ldres;
    void* out;                      // I x J, contiguous
    uint16_t* slope;                // I x J, or nullptr
    float* partial;                 // workspace for sums of parts of k
    int64_t partial_bytes;
};
hipError_t launch_dense_gemm(int32_t type, const DenseGemm& g, hipStream_t s);
int64_t dense_partial_bytes(int64_t I, int64_t J, int64_t K);      // of the workspace such a product may ask for
// dz = dy slope (dz may be nullptr: only db), db = column sums of the unrounded dz (db may be nullptr)
hipError_t launch_dense_dz(int32_t type, const void* dy, int64_t lddy, const uint16_t* slope, void* dz, void* db, double* sums, int64_t M, int64_t N,
                           hipStream_t s);
int64_t dense_sums_bytes(int64_t M, int64_t N);

// ---- gated projections (kernels_gated.hip): g of J gates with their partners, act(gate) partner ----
hipError_t launch_gated_gemm(int32_t type, const DenseGemm& g, hipStream_t s);      // b_up is set here
int64_t gated_partial_bytes(int64_t I, int64_t J, int64_t K);
int64_t gated_sums_bytes(int64_t M, int64_t N);
// dz = [dh slope | dh slope'], rows of lddz >= 2 N with zeros at their ends (dz may be nullptr: only db), low (or nullptr) what its rounding has left, db = column sums of the unrounded dz (db may be nullptr)
hipError_t launch_gated_dz(int32_t type, const void* dh, int64_t lddh, const uint16_t* slopes, void* dz, void* low, int64_t lddz, void* db, double* sums, int64_t M,
                           int64_t N, hipStream_t s);
// w and x as the products of the backward pass want them, in rows of whole pieces
struct GatedCopies {
    const void* w;
    int64_t ldw;
    const void* x;
    int64_t ldx;
};
bool gated_copies(int64_t M, int64_t N, int64_t K, bool w_transposed);      // whether both products want them
int64_t gated_copies_bytes(int64_t M, int64_t N, int64_t K);
void launch_gated_copies(const void* w, int64_t ldw, bool w_transposed, const void* x, int64_t ldx, int64_t M, int64_t N, int64_t K, void* to, GatedCopies* copies, hipStream_t s);
bool gated_padded(int64_t M, int64_t N, int64_t K);        // whether dz is written in rows of whole pieces
bool gated_low(int64_t of_result, int64_t of_dz);   // whether a result of so many elements is computed from dz in two parts

// ---- layer norm (kernels_norm.hip) ----
struct NormRows {
    int32_t type, param_type;
    int64_t rows, n;
    const void* x;
    int64_t ldx;
    const void* w;                  // n, or nullptr
};
int64_t norm_workspace_bytes(int32_t type, int64_t rows, int64_t n);       // of a gradient
hipError_t launch_norm(const NormRows& r, const void* b, double eps, void* y, float* stats, hipStream_t s);
hipError_t launch_norm_gradient(const NormRows& r, const void* dy, int64_t lddy, const float* stats, void* dx, void* dw, void* db, void* ws, hipStream_t s);

// ---- losses over a vocabulary (kernels_losses.hip) ----
struct LossRows {
    int32_t type;
    int64_t rows, vocab, ld;
    const void* z;
    const int64_t* tokens;
};
int64_t loss_workspace_bytes(int64_t rows, int64_t vocab);
hipError_t launch_log_probs(const LossRows& a, float* logp, void* ws, hipStream_t s);
struct PolicyTerms {
    const float *old, *adv, *ref;
    float clip_low, clip_high, kl;
};
hipError_t launch_policy(const LossRows& a, const PolicyTerms& t, float* loss, void* dz, float* logp, void* ws, hipStream_t s);
hipError_t launch_preference(const LossRows& a, const int64_t* offsets, int64_t pairs, const float* ref, double beta, double smoothing, float* loss,
                             void* dz, float* sums, float* margins, void* ws, hipStream_t s);

struct TeacherRows {                // kernels_distill.hip
    int32_t type;
    int64_t k;
    const int64_t* tokens;
    int64_t ld_tokens;
    const void* z;
    int64_t ld;
};
int64_t distill_workspace_bytes(int64_t rows, int64_t k);
hipError_t launch_distill(const LossRows& r, const TeacherRows& t, double temperature, double hard_weight, double loss_scale, float* loss, void* dz, float* kl,
                          float* logp, void* ws, hipStream_t s);

// ---- AdamW (kernels_adamw.hip) ----
constexpr int kAdamwBlock = 256;    // elements that share an exponent
constexpr int kAdamwChunk = 4096;   // elements of one thread block
struct AdamwChunk {                 // of one tensor: where it begins
    void* p;
    const void* g;
    float* master;
    float* out;
    int64_t state;                  // a multiple of 256
    int32_t n;
    float decay;
};
struct AdamwArgs {
    const AdamwChunk* chunks;
    int64_t n_chunks;
    int32_t param_type, grad_type, bits;
    bool masters, direction;
    void *m, *v;
    int8_t* exponents;
    double beta1_64, beta2_64, rest1_64, rest2_64;
    float beta1, beta2, rest1, rest2, eps, lr, inv_c1, inv_c2;     // rest: 1 - beta, inv_c: 1 / (1 - beta^step), inv_c2 divided by root^2
    float root;                     // times the root of v inv_c2
    float grad_scale;
    double grad_scale_64, max_norm;
    uint64_t seed, step;
    double* norm_parts;             // kAdamwNormBlocks ...
    int32_t norm_blocks;            // ... of which so many are used
    double* factor;                 // of the gradients in this step
    float* norm;
};
constexpr int kAdamwNormBlocks = 2048;      // eight for a compute unit: all are there at once
hipError_t launch_adamw(const AdamwArgs& a, hipStream_t s);
hipError_t launch_adamw_get(const void* m, const void* v, const int8_t* exponents, int64_t length, uint16_t* m_out, uint16_t* v_out, hipStream_t s);
hipError_t launch_adamw_set(const float* m, const float* v, int64_t length, void* m_out, void* v_out, int8_t* exponents, hipStream_t s);

}  // namespace adpsgd_impl
