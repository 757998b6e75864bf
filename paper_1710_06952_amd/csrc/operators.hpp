// What the C entries of the training-step operators (api_operators.cpp) and their kernels share.
#pragma once

#include "internal.hpp"

namespace adpsgd_impl {

// ---- dense layers (kernels_dense.hip) ----
struct DenseGemm {                  // D[i][j] = sum_k A(i, k) B(j, k), i < I, j < J, k < K
    const void *a, *b;
    int64_t lda, ldb;
    bool a_outer, b_outer;          // false: (i, k) at a + i lda + k;  true: at a + k lda + i.  b likewise
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
