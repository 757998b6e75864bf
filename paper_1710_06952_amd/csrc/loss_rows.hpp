// What the losses over a vocabulary share: how a row is cut into vectors, the largest value and the sum of exponentials and how they
// join, logarithm and exponential of their own, the rows that count and the mean over them.
#pragma once

#include <algorithm>

#include "elements.hpp"

namespace adpsgd_impl {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = 1.925963033500e-8f;
constexpr int kT = 256;

// How a row of V elements is cut: vectors of kN whose addresses are multiples of 16 bytes, and what is left in front of and behind them,
// less than a vector each, which the first threads of a block take as one element each.  (Ends taken inside of the vectors' code
// made kernels of 40 KB whose registers did not suffice.)
template <class E>
struct Cut {
    int head, vectors, tail;
    __device__ __forceinline__ Cut(const void* row, int V) {
        const int off = static_cast<int>(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(typename E::Raw));
        head = off == 0 ? 0 : E::kN - off;
        head = head < V ? head : V;
        vectors = (V - head) / E::kN;
        tail = V - head - vectors * E::kN;
    }
    __device__ __forceinline__ int at(int v) const { return head + v * E::kN; }
    // The vector that covers element e, or -1.
    __device__ __forceinline__ int vector_of(int e) const { return e >= head && e < at(vectors) ? (e - head) / E::kN : -1; }
    // The element that a thread takes beside its vectors, or -1.
    __device__ __forceinline__ int single() const {
        const int t = threadIdx.x;
        return t < E::kN ? (t < head ? t : -1) : t < 2 * E::kN && t - E::kN < tail ? at(vectors) + t - E::kN : -1;
    }
};
// Past the caches unless a later pass of the same call reads them again; gradients always.  8000 x 32 000 in fp16: 74 us for 84;
// preference loss of 8 pairs over 50 001 tokens: 163 us for 198, and 183 where the first pass reads past the caches as well.
template <class E, bool kAgain>
__device__ __forceinline__ v4u load_vector(const typename E::Raw* row, int at) {
    const v4u_any* p = reinterpret_cast<const v4u_any*>(row + at);
    return kAgain ? *p : __builtin_nontemporal_load(p);
}
template <class E>
__device__ __forceinline__ void store_vector(typename E::Raw* row, int at, const float* f) {
    __builtin_nontemporal_store(E::pack(f), reinterpret_cast<v4u_any*>(row + at));
}
template <class E>
constexpr uint32_t kNothing = E::kN == 4 ? 0xFF800000u : 0u;       // two halves of -infinity ...
template <>
constexpr uint32_t kNothing<Bf16> = 0xFF80FF80u;
template <>
constexpr uint32_t kNothing<F16> = 0xFC00FC00u;

struct Stat {
    float m, s;                 // the largest value, and the sum of exp(z - m)
};
// exp(d).  (2^(z log2 e - m') by an FMA is an instruction less, but a rounded m' stands for no m: at 1e9 its rounding is e^20.)
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// ... kFine: log2 e in two parts.  Its rounding to 32 bits is 1.3e-8 of d in every term of a sum, in the same direction, and sums of
// log-probabilities over a sequence add that up: l is off by 2e-8 in the mean without it, and by less than 3e-9 with it.
template <bool kFine>
__device__ __forceinline__ float exp_in_sum(float d) { return __builtin_amdgcn_exp2f(kFine ? fmaf(d, kLog2e, d * kLog2eRest) : d * kLog2e); }
// What the sum over values up to m is taken relative to: m, or 0 where there is nothing but -infinity.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ Stat joined(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m), base = base_of(m);
    return Stat{m, a.s * exp_in_sum<true>(a.m - base) + b.s * exp_in_sum<true>(b.m - base)};
}
__device__ __forceinline__ Stat of_one(float z) { return Stat{z, exp_of(z - base_of(z))}; }
// Of each group of kLanes neighbouring lanes, to all of them.
template <int kLanes>
__device__ __forceinline__ Stat lanes_joined(Stat a) {
    float m = a.m;
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    float s = a.s * exp_in_sum<true>(a.m - base_of(m));
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
    return Stat{m, s};
}
// Of a block of kWaves wavefronts, to all threads; `at`: kWaves places in LDS.
template <int kWaves>
__device__ __forceinline__ Stat block_joined(Stat a, Stat* at) {
    a = lanes_joined<64>(a);
    if (kWaves == 1) return a;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = a;
    __syncthreads();
    return lanes_joined<kWaves>(at[threadIdx.x % kWaves]);
}

// log s.  Rows of the same length have about the same s, so what a logarithm is off by is the same for all of them and adds up over a
// sequence (logf: 5e-8): the series of 2 atanh((f - 1) / (f + 1)) in 64 bits, to 1e-11, in few registers (the library's takes 40, which the
// kernel that holds a row in registers does not have).
__device__ __forceinline__ double log_of(float s) {
    int k;
    float f = frexpf(s, &k);                             // 1/2 <= f < 1
    if (f < 0.70710678f) {
        f *= 2.0f;
        --k;
    }
    const double x = static_cast<double>(f) - 1.0, w = x + 2.0;
    double r = static_cast<double>(__builtin_amdgcn_rcpf(static_cast<float>(w)));
    r = r * fma(-w, r, 2.0);
    const double u = x * r, y = u * u;                   // |u| <= 0.172
    double p = fma(y, 1.0 / 13.0, 1.0 / 11.0);
    p = fma(y, p, 1.0 / 9.0);
    p = fma(y, p, 1.0 / 7.0);
    p = fma(y, p, 1.0 / 5.0);
    p = fma(y, p, 1.0 / 3.0);
    return fma(static_cast<double>(k), 0.6931471805599453, 2.0 * u * fma(y, p, 1.0));
}
// In the gradient the rounding of log2 e is 1.3e-8 of z - m, in the same direction in every element: 1e-7 where fp32 holds it, nothing in 16 bits.
template <class E>
__device__ __forceinline__ float exp_in_gradient(float d) { return exp_in_sum<E::kN == 4>(d); }

// Rows that count, to all threads of a block of kWaves wavefronts.
template <int kWaves>
__device__ __forceinline__ float counted_rows(const int64_t* tokens, int64_t rows, float* at) {
    float n = 0.0f;                                      // up to 2^21: exact
    for (int64_t i = threadIdx.x; i < rows; i += kWaves * 64) n += tokens[i] >= 0 ? 1.0f : 0.0f;
    n = wave_sum(n);
    if (kWaves == 1) return n;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = n;
    __syncthreads();
    n = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) n += at[w];
    return n;
}
// 1 / max(1, counted rows).
__global__ __launch_bounds__(1024) void count_rows_kernel(const int64_t* tokens, int64_t rows, float* share) {
    __shared__ float at[16];
    const float n = counted_rows<16>(tokens, rows, at);
    if (threadIdx.x == 0) *share = 1.0f / fmaxf(n, 1.0f);
}
// The mean of the loss terms, in an order that the number of rows gives.
__global__ __launch_bounds__(1024) void mean_terms_kernel(const double* term, const int64_t* tokens, int64_t rows, float* loss) {
    __shared__ float counts[16];
    __shared__ double at[16];
    const float n = counted_rows<16>(tokens, rows, counts);
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) sum += term[i];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) sum += at[w];
        *loss = static_cast<float>(sum / static_cast<double>(fmaxf(n, 1.0f)));
    }
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

}  // namespace
}  // namespace adpsgd_impl
