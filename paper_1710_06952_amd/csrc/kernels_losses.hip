// Log-probabilities and losses over a vocabulary, and their gradients for the logits.
//
// Of a row z the softmax needs the largest value m and s = sum exp(z - m).  Both come from one pass: every thread keeps its own
// (m, s), rescaled when m grows, and two such pairs join as (max, s exp(m - max) + s' exp(m' - max)).  With l = z[token] - m -
// log s and a coefficient c = dL/dl of the row, the gradient is  c (onehot - exp(z - m) / s).
//
//   row_stats         (m, s) of parts of rows, one thread block each; whole rows end in `finish_row` at once
//   join_stats        joins the parts of a row (few rows over a large vocabulary), one wavefront a row
//   policy_rows       statistics, coefficient and gradient with the row held in registers: the logits are read once
//   logit_gradient    the gradient from stored statistics and coefficients
//   preference_pairs  sums over sequences, margins, coefficients
//
// Bound: memory, 2 or 4 bytes an element in and, with a gradient, out.  The instructions for an element (conversion, difference,
// product, v_exp_f32, sum, twice for a gradient) take about half of the time that its bytes take.
//
// Rows begin at any multiple of the element (odd vocabularies): vectors of 16 bytes are read and written at such addresses too.
// Exponentials, sums and the gradient are in 32 bits, what there is one of in a row (l, ratios, loss terms, coefficients) in 64,
// as a ratio may stand next to the border of the clipping.  A row is summed in an order that depends on the sizes alone.
#include <algorithm>

#include "device_common.hpp"
#include "operators.hpp"

namespace adpsgd_impl {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kT = 256;
constexpr int kUnroll = 4;              // vectors of a thread on their way at once
constexpr int64_t kSplitBlocks = 1024;  // blocks that fill the chip: rows are split over the vocabulary up to this many

typedef v4u v4u_any __attribute__((aligned(2)));       // 16 bytes at any multiple of an element

struct F32 {
    using Raw = float;
    static constexpr int kN = 4;
    __device__ static float get(const Raw* p) { return *p; }
    __device__ static void unpack(v4u v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    __device__ static v4u pack(const float* f) {
        return v4u{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
    __device__ static void put(Raw* p, float f) { *p = f; }
};
struct Bf16 {
    using Raw = uint16_t;
    static constexpr int kN = 8;
    __device__ static float get(const Raw* p) { return bf16_to_float(*p); }
    __device__ static void unpack(v4u v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        }
    }
    __device__ static v4u pack(const float* f) {
        typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
        v4u v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, v2bf{static_cast<__bf16>(f[2 * i]), static_cast<__bf16>(f[2 * i + 1])});
        return v;
    }
    __device__ static void put(Raw* p, float f) { *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
};
struct F16 {
    using Raw = uint16_t;
    static constexpr int kN = 8;
    typedef _Float16 v2hf __attribute__((ext_vector_type(2)));
    __device__ static float get(const Raw* p) { return static_cast<float>(__builtin_bit_cast(_Float16, *p)); }
    __device__ static void unpack(v4u v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2hf h = __builtin_bit_cast(v2hf, static_cast<uint32_t>(v[i]));
            f[2 * i] = static_cast<float>(h.x);
            f[2 * i + 1] = static_cast<float>(h.y);
        }
    }
    __device__ static v4u pack(const float* f) {
        v4u v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, v2hf{static_cast<_Float16>(f[2 * i]), static_cast<_Float16>(f[2 * i + 1])});
        return v;
    }
    __device__ static void put(Raw* p, float f) { *p = __builtin_bit_cast(uint16_t, static_cast<_Float16>(f)); }
};

// Elements v kN .. of a row of V; beyond the end: `fill`, as bits of 32.
template <class E>
__device__ __forceinline__ v4u load_vector(const typename E::Raw* row, int64_t v, int64_t V, uint32_t fill) {
    const int64_t at = v * E::kN;
    if (at + E::kN <= V) return *reinterpret_cast<const v4u_any*>(row + at);
    v4u x = {fill, fill, fill, fill};
    typename E::Raw part[E::kN];
    __builtin_memcpy(part, &x, 16);
#pragma unroll
    for (int i = 0; i < E::kN; ++i)
        if (at + i < V) part[i] = row[at + i];
    __builtin_memcpy(&x, part, 16);
    return x;
}
template <class E>
__device__ __forceinline__ void store_vector(typename E::Raw* row, int64_t v, int64_t V, const float* f) {
    const int64_t at = v * E::kN;
    if (at + E::kN <= V) {
        *reinterpret_cast<v4u_any*>(row + at) = E::pack(f);
        return;
    }
#pragma unroll
    for (int i = 0; i < E::kN; ++i)
        if (at + i < V) E::put(row + at + i, f[i]);
}
template <class E>
constexpr uint32_t kNothing = E::kN == 4 ? 0xFF800000u : 0u;       // two halves of -infinity ...
template <>
constexpr uint32_t kNothing<Bf16> = 0xFF80FF80u;
template <>
constexpr uint32_t kNothing<F16> = 0xFC00FC00u;

struct Stat {
    float m, s;
};
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// What the sum over values up to m is taken relative to: m, or 0 where there is nothing but -infinity.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ Stat joined(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m), base = base_of(m);
    return Stat{m, a.s * exp_of(a.m - base) + b.s * exp_of(b.m - base)};
}
__device__ __forceinline__ Stat wave_joined(Stat a) {
    float m = a.m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    return Stat{m, wave_sum(a.s * exp_of(a.m - base_of(m)))};
}
// Of a block of kWaves wavefronts, to all threads; `at`: kWaves places in LDS.
template <int kWaves>
__device__ __forceinline__ Stat block_joined(Stat a, Stat* at) {
    a = wave_joined(a);
    if (kWaves == 1) return a;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = a;
    __syncthreads();
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, at[w].m);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += at[w].s * exp_of(at[w].m - base_of(m));
    return Stat{m, s};
}

enum Mode { kScore, kPolicy, kPreference };

// What one thread does once for a row.
struct RowArgs {
    const void* z;
    const int64_t* tokens;
    int64_t rows, vocab, ld;
    Mode mode;
    float* logp;            // kScore, kPolicy
    PolicyTerms policy;
    const float* share;     // kPolicy: 1 / counted rows
    Stat* stat;             // kPolicy, kPreference
    float* coef;
    double* term;           // kPolicy: of the loss, kPreference: log-probabilities
    Stat* parts;            // [row][split]
    int splits;
};

__device__ __forceinline__ double log_prob(float at, Stat st) { return static_cast<double>(at - st.m) - log(static_cast<double>(st.s)); }

// dL/dl and the loss term of one row, both times the number of counted rows.
__device__ __forceinline__ void policy_row(const PolicyTerms& t, int64_t row, double l, double& slope, double& term) {
    const double A = t.adv[row], rho = exp(l - static_cast<double>(t.old[row]));
    const double free = rho * A;
    // fmin and fmax pass over a NaN: the ratio is kept as it is unless it is outside
    const double inside = rho < 1.0 - t.clip_low ? 1.0 - t.clip_low : rho > 1.0 + t.clip_high ? 1.0 + t.clip_high : rho;
    const double held = inside * A;
    term = held < free ? -held : -free;
    slope = held < free ? 0.0 : -free;
    if (t.ref) {
        const double d = static_cast<double>(t.ref[row]) - l, e = exp(d);
        term += t.kl * (e - d - 1.0);
        slope += t.kl * (1.0 - e);
    }
}

template <class E>
__device__ __forceinline__ void finish_row(const RowArgs& a, int64_t row, Stat st) {
    const int64_t token = a.tokens[row];
    double l = 0.0;
    if (token >= 0) {
        const float at = token < a.vocab ? E::get(static_cast<const typename E::Raw*>(a.z) + row * a.ld + token) : NAN;
        l = log_prob(at, st);
    }
    if (a.mode == kScore) {
        a.logp[row] = static_cast<float>(l);
        return;
    }
    a.stat[row] = st;
    if (a.mode == kPreference) {
        a.term[row] = l;
        a.coef[row] = 0.0f;
        return;
    }
    double slope = 0.0, term = 0.0;
    if (token >= 0) policy_row(a.policy, row, l, slope, term);
    a.logp[row] = static_cast<float>(l);
    a.term[row] = term;
    a.coef[row] = static_cast<float>(slope * *a.share);
}

// (m, s) of the vectors v0 <= v < v1 of a row that this thread takes
template <class E>
__device__ __forceinline__ Stat thread_stat(const typename E::Raw* row, int64_t v0, int64_t v1, int64_t V) {
    Stat st{-INFINITY, 0.0f};
    for (int64_t v = v0 + threadIdx.x; v < v1; v += kT * kUnroll) {
        v4u x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            x[u] = v4u{kNothing<E>, kNothing<E>, kNothing<E>, kNothing<E>};
            if (v + u * kT < v1) x[u] = load_vector<E>(row, v + u * kT, V, kNothing<E>);
        }
        float f[kUnroll][E::kN], m = st.m;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            E::unpack(x[u], f[u]);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) m = fmaxf(m, f[u][i]);
        }
        const float base = base_of(m);
        float s = st.s * exp_of(st.m - base);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < E::kN; ++i) s += exp_of(f[u][i] - base);
        st = Stat{m, s};
    }
    return st;
}

// grid: rows * splits.
template <class E>
__global__ __launch_bounds__(kT) void row_stats_kernel(const RowArgs a) {
    __shared__ Stat at[kT / 64];
    const int64_t row = blockIdx.x / a.splits;
    const int part = blockIdx.x % a.splits;
    if (a.tokens[row] < 0) {
        if (a.splits == 1 && threadIdx.x == 0) finish_row<E>(a, row, Stat{0.0f, 1.0f});
        return;
    }
    const int64_t vectors = (a.vocab + E::kN - 1) / E::kN, each = (vectors + a.splits - 1) / a.splits;
    const int64_t v0 = part * each, v1 = v0 + each < vectors ? v0 + each : vectors;
    const Stat st = block_joined<kT / 64>(thread_stat<E>(static_cast<const typename E::Raw*>(a.z) + row * a.ld, v0, v1, a.vocab), at);
    if (threadIdx.x == 0) {
        if (a.splits == 1) finish_row<E>(a, row, st);
        else a.parts[row * a.splits + part] = st;
    }
}

// One wavefront a row.
template <class E>
__global__ __launch_bounds__(kT) void join_stats_kernel(const RowArgs a) {
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kT / 64) + (threadIdx.x >> 6);
    if (row >= a.rows) return;
    Stat st{-INFINITY, 0.0f};
    if (a.tokens[row] >= 0)
        for (int q = threadIdx.x & 63; q < a.splits; q += 64) st = joined(st, a.parts[row * a.splits + q]);
    st = wave_joined(st);
    if ((threadIdx.x & 63) == 0) finish_row<E>(a, row, st);
}

// d[i] = exp(z[i] - m) scale, and coef more at the token.
template <class E>
__device__ __forceinline__ void gradient_of(v4u x, int64_t v, int64_t token, float m, float scale, float coef, float* d) {
    E::unpack(x, d);
#pragma unroll
    for (int i = 0; i < E::kN; ++i) d[i] = exp_of(d[i] - m) * scale;
    const int64_t here = token - v * E::kN;
    if (here >= 0 && here < E::kN) {
#pragma unroll
        for (int i = 0; i < E::kN; ++i) d[i] += here == i ? coef : 0.0f;
    }
}

struct GradientArgs {
    RowArgs row;
    void* dz;               // rows x vocab
    int64_t blocks;         // of a row
    const float* margins;   // preference: the loss of these goes to `loss`
    int64_t pairs;
    double smoothing;
    float* loss;
};

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }      // NaN: below

// grid: rows * blocks.  The last rows first: they are the ones that the pass before has left in the last-level cache.
template <class E>
__global__ __launch_bounds__(kT) void logit_gradient_kernel(const GradientArgs g) {
    const RowArgs& a = g.row;
    if (g.margins && blockIdx.x == 0 && threadIdx.x < 64) {
        double sum = 0.0;
        for (int64_t q = threadIdx.x; q < g.pairs; q += 64) {
            const double x = g.margins[q];
            sum += x == x ? (1.0 - g.smoothing) * softplus(-x) + g.smoothing * softplus(x) : x;
        }
        sum = wave_sum(sum);
        if (threadIdx.x == 0) *g.loss = static_cast<float>(sum / static_cast<double>(g.pairs));
    }
    const int64_t row = a.rows - 1 - blockIdx.x / g.blocks;
    const int64_t vectors = (a.vocab + E::kN - 1) / E::kN;
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    typename E::Raw* dz = static_cast<typename E::Raw*>(g.dz) + row * a.vocab;
    const int64_t token = a.tokens[row];
    const float coef = token < 0 ? 0.0f : a.coef[row];
    const Stat st = token < 0 ? Stat{0.0f, 1.0f} : a.stat[row];
    const float scale = -coef / st.s;
    const int64_t v0 = (blockIdx.x % g.blocks) * (kT * kUnroll) + threadIdx.x;
    v4u x[kUnroll];
    float d[E::kN];
    if (coef == 0.0f) {                 // nothing to read
#pragma unroll
        for (int i = 0; i < E::kN; ++i) d[i] = 0.0f;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (v0 + u * kT < vectors) store_vector<E>(dz, v0 + u * kT, a.vocab, d);
        return;
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
        if (v0 + u * kT < vectors) x[u] = load_vector<E>(z, v0 + u * kT, a.vocab, 0);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
        if (v0 + u * kT < vectors) {
            gradient_of<E>(x[u], v0 + u * kT, token, st.m, scale, coef, d);
            store_vector<E>(dz, v0 + u * kT, a.vocab, d);
        }
}

// ---- policy ----------------------------------------------------------------------------------------------
// 1 / max(1, counted rows), and the ticket of the last block at zero.
__global__ __launch_bounds__(1024) void count_rows_kernel(const int64_t* tokens, int64_t rows, float* share, uint32_t* ticket) {
    __shared__ double at[16];
    double n = 0.0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) n += tokens[i] >= 0 ? 1.0 : 0.0;
    n = wave_sum(n);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) n += at[w];
        *share = static_cast<float>(1.0 / fmax(n, 1.0));
        share[1] = static_cast<float>(fmax(n, 1.0));
        *ticket = 0;
    }
}

// The mean of the loss terms, by one block, in an order that the number of rows gives.
template <int kThreads>
__device__ __forceinline__ void sum_terms(const double* term, int64_t rows, const float* share, float* loss, double* at) {
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < rows; i += kThreads) sum += __hip_atomic_load(term + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 64; ++w) sum += at[w];
        *loss = static_cast<float>(sum / static_cast<double>(share[1]));
    }
}
__global__ __launch_bounds__(kT) void mean_terms_kernel(const double* term, int64_t rows, const float* share, float* loss) {
    __shared__ double at[kT / 64];
    sum_terms<kT>(term, rows, share, loss, at);
}

// kWaves wavefronts a row, up to kHeld vectors a thread in registers; the last block to end adds the loss.
template <class E, int kWaves, int kHeld>
__global__ __launch_bounds__(kWaves * 64) void policy_rows_kernel(const GradientArgs g, uint32_t* ticket) {
    constexpr int kThreads = kWaves * 64;
    __shared__ Stat at[kWaves];
    __shared__ double sums[kWaves];
    __shared__ float of_row[2];
    __shared__ uint32_t turn;
    const RowArgs& a = g.row;
    const int64_t row = blockIdx.x, vectors = (a.vocab + E::kN - 1) / E::kN;
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    typename E::Raw* dz = static_cast<typename E::Raw*>(g.dz) + row * a.vocab;
    const int64_t token = a.tokens[row];
    float coef = 0.0f, m = 0.0f, scale = 0.0f;
    v4u x[kHeld];
    if (token >= 0) {                   // uniform over the block
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int64_t v = u * kThreads + threadIdx.x;
            x[u] = v4u{kNothing<E>, kNothing<E>, kNothing<E>, kNothing<E>};
            if (v < vectors) x[u] = load_vector<E>(z, v, a.vocab, kNothing<E>);
        }
        float f[E::kN];
        Stat st{-INFINITY, 0.0f};
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            E::unpack(x[u], f);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) st.m = fmaxf(st.m, f[i]);
        }
        const float base = base_of(st.m);
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            E::unpack(x[u], f);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) st.s += exp_of(f[i] - base);
        }
        st = block_joined<kWaves>(st, at);
        if (threadIdx.x < 64) {         // 64-bit logarithm and exponentials: one wavefront's time, not the block's
            const float value = token < a.vocab ? E::get(z + token) : NAN;
            const double l = log_prob(value, st);
            double slope, term;
            policy_row(a.policy, row, l, slope, term);
            if (threadIdx.x == 0) {
                a.logp[row] = static_cast<float>(l);
                __hip_atomic_store(a.term + row, term, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                of_row[0] = static_cast<float>(slope * *a.share);
            }
        }
        __syncthreads();
        coef = of_row[0];
        m = st.m;
        scale = -coef / st.s;
    } else if (threadIdx.x == 0) {
        a.logp[row] = 0.0f;
        __hip_atomic_store(a.term + row, 0.0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    const bool zero = coef == 0.0f;     // NaN is not
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        const int64_t v = u * kThreads + threadIdx.x;
        if (v < vectors) {
            float d[E::kN];
            if (zero) {
#pragma unroll
                for (int i = 0; i < E::kN; ++i) d[i] = 0.0f;
            } else {
                gradient_of<E>(x[u], v, token, m, scale, coef, d);
            }
            store_vector<E>(dz, v, a.vocab, d);
        }
    }
    if (threadIdx.x == 0) {             // its term is in memory before it counts as done
        __threadfence();
        turn = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (turn + 1 == gridDim.x) {
        __threadfence();
        sum_terms<kThreads>(a.term, a.rows, a.share, g.loss, sums);
    }
}

// ---- preference ------------------------------------------------------------------------------------------
// One block a pair.  Offsets that do not ascend from 0 to `rows` are never followed: the margin is NaN, and with it the loss.
__global__ __launch_bounds__(kT) void preference_pairs_kernel(const double* logp, const int64_t* offsets, int64_t pairs, int64_t rows, const float* ref,
                                                             double beta, double smoothing, float* sums, float* margins, float* coef) {
    __shared__ double at[2][kT / 64];
    __shared__ float slope;
    const int64_t q = blockIdx.x;
    int64_t from[2], to[2];
    bool good = offsets[0] == 0 && offsets[2 * pairs] == rows;
    double part[2] = {0.0, 0.0};
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        from[side] = offsets[q + side * pairs];
        to[side] = offsets[q + side * pairs + 1];
        good = good && 0 <= from[side] && from[side] <= to[side] && to[side] <= rows;
    }
    if (good)                            // uniform over the block
        for (int side = 0; side < 2; ++side)
            for (int64_t i = from[side] + threadIdx.x; i < to[side]; i += kT) part[side] += logp[i];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        part[side] = wave_sum(part[side]);
        if ((threadIdx.x & 63) == 0) at[side][threadIdx.x >> 6] = part[side];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double s[2];
        for (int side = 0; side < 2; ++side) {
            s[side] = good ? 0.0 : NAN;
            for (int w = 0; w < kT / 64; ++w) s[side] += at[side][w];
            sums[q + side * pairs] = static_cast<float>(s[side]);
        }
        const double margin = beta * ((s[0] - ref[q]) - (s[1] - ref[pairs + q]));
        margins[q] = static_cast<float>(margin);
        slope = static_cast<float>(beta / static_cast<double>(pairs) * (smoothing - 1.0 / (1.0 + exp(margin))));
    }
    __syncthreads();
    if (good)
        for (int side = 0; side < 2; ++side)
            for (int64_t i = from[side] + threadIdx.x; i < to[side]; i += kT) coef[i] = side == 0 ? slope : -slope;
}

// ---- host ------------------------------------------------------------------------------------------------
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// Few rows are split over the vocabulary, but into no parts under 2048 vectors (two turns of a block's threads).
int split_of(int64_t rows, int64_t vectors) {
    const int64_t most = kSplitBlocks / std::max<int64_t>(rows, 1);
    return static_cast<int>(std::max<int64_t>(1, std::min(most, vectors / (2 * kT))));
}

struct Workspace {
    Stat* stat;
    double* term;
    float* coef;
    float* share;           // 1 / counted and counted
    uint32_t* ticket;
    Stat* parts;
    int64_t bytes;
};
Workspace laid_out(void* at, int64_t rows) {
    char* p = static_cast<char*>(at);
    Workspace w{};
    auto take = [&](int64_t bytes) {
        char* q = p + w.bytes;
        w.bytes += up16(bytes);
        return q;
    };
    w.stat = reinterpret_cast<Stat*>(take(rows * sizeof(Stat)));
    w.term = reinterpret_cast<double*>(take(rows * sizeof(double)));
    w.coef = reinterpret_cast<float*>(take(rows * sizeof(float)));
    w.share = reinterpret_cast<float*>(take(2 * sizeof(float)));
    w.ticket = reinterpret_cast<uint32_t*>(take(sizeof(uint32_t)));
    w.parts = reinterpret_cast<Stat*>(take(std::max(rows, kSplitBlocks) * sizeof(Stat)));      // rows * split_of(rows, .) at most
    return w;
}

RowArgs row_args(const LossRows& a, Mode mode, const Workspace& w) {
    RowArgs r{};
    r.z = a.z;
    r.tokens = a.tokens;
    r.rows = a.rows;
    r.vocab = a.vocab;
    r.ld = a.ld;
    r.mode = mode;
    r.stat = w.stat;
    r.term = w.term;
    r.coef = w.coef;
    r.share = w.share;
    r.parts = w.parts;
    return r;
}

template <class E>
void launch_stats(RowArgs r, hipStream_t s) {
    r.splits = split_of(r.rows, (r.vocab + E::kN - 1) / E::kN);
    hipLaunchKernelGGL(row_stats_kernel<E>, dim3(static_cast<uint32_t>(r.rows * r.splits)), dim3(kT), 0, s, r);
    if (r.splits > 1) hipLaunchKernelGGL(join_stats_kernel<E>, dim3(static_cast<uint32_t>((r.rows + kT / 64 - 1) / (kT / 64))), dim3(kT), 0, s, r);
}
template <class E>
void launch_gradient(GradientArgs g, hipStream_t s) {
    const int64_t vectors = (g.row.vocab + E::kN - 1) / E::kN;
    g.blocks = (vectors + kT * kUnroll - 1) / (kT * kUnroll);
    hipLaunchKernelGGL(logit_gradient_kernel<E>, dim3(static_cast<uint32_t>(g.row.rows * g.blocks)), dim3(kT), 0, s, g);
}

template <class E>
void launch_policy_of(GradientArgs g, uint32_t* ticket, hipStream_t s) {
    const int64_t rows = g.row.rows, vectors = (g.row.vocab + E::kN - 1) / E::kN;
    const dim3 grid(static_cast<uint32_t>(rows));
    hipLaunchKernelGGL(count_rows_kernel, dim3(1), dim3(1024), 0, s, g.row.tokens, rows, const_cast<float*>(g.row.share), ticket);
    if (vectors <= 256) hipLaunchKernelGGL((policy_rows_kernel<E, 1, 4>), grid, dim3(64), 0, s, g, ticket);
    else if (vectors <= 1024) hipLaunchKernelGGL((policy_rows_kernel<E, 4, 4>), grid, dim3(256), 0, s, g, ticket);
    else if (vectors <= 4096) hipLaunchKernelGGL((policy_rows_kernel<E, 8, 8>), grid, dim3(512), 0, s, g, ticket);
    else if (vectors <= 8192) hipLaunchKernelGGL((policy_rows_kernel<E, 16, 8>), grid, dim3(1024), 0, s, g, ticket);
    else if (vectors <= 16384) hipLaunchKernelGGL((policy_rows_kernel<E, 16, 16>), grid, dim3(1024), 0, s, g, ticket);
    else {                               // more than a block's registers hold
        launch_stats<E>(g.row, s);
        hipLaunchKernelGGL(mean_terms_kernel, dim3(1), dim3(kT), 0, s, g.row.term, rows, g.row.share, g.loss);
        launch_gradient<E>(g, s);
    }
}
template <class E>
void launch_preference_of(const GradientArgs& g, const int64_t* offsets, const float* ref, double beta, float* sums, float* margins, hipStream_t s) {
    if (g.row.rows > 0) launch_stats<E>(g.row, s);
    hipLaunchKernelGGL(preference_pairs_kernel, dim3(static_cast<uint32_t>(g.pairs)), dim3(kT), 0, s, g.row.term, offsets, g.pairs, g.row.rows, ref, beta,
                       g.smoothing, sums, margins, g.row.coef);
    if (g.row.rows > 0) launch_gradient<E>(g, s);
}

__global__ __launch_bounds__(64) void preference_loss_kernel(const float* margins, int64_t pairs, double smoothing, float* loss) {
    double sum = 0.0;
    for (int64_t q = threadIdx.x; q < pairs; q += 64) {
        const double x = margins[q];
        sum += x == x ? (1.0 - smoothing) * softplus(-x) + smoothing * softplus(x) : x;
    }
    sum = wave_sum(sum);
    if (threadIdx.x == 0) *loss = static_cast<float>(sum / static_cast<double>(pairs));
}

}  // namespace

int64_t loss_workspace_bytes(int64_t rows, int64_t) { return laid_out(nullptr, rows).bytes; }

hipError_t launch_log_probs(const LossRows& a, float* logp, void* ws, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    RowArgs r = row_args(a, kScore, laid_out(ws, a.rows));
    r.logp = logp;
    if (a.type == ADPSGD_TYPE_F32) launch_stats<F32>(r, s);
    else if (a.type == ADPSGD_TYPE_BF16) launch_stats<Bf16>(r, s);
    else launch_stats<F16>(r, s);
    return hipGetLastError();
}

hipError_t launch_policy(const LossRows& a, const PolicyTerms& t, float* loss, void* dz, float* logp, void* ws, hipStream_t s) {
    const Workspace w = laid_out(ws, a.rows);
    GradientArgs g{};
    g.row = row_args(a, kPolicy, w);
    g.row.logp = logp;
    g.row.policy = t;
    g.dz = dz;
    g.loss = loss;
    if (a.rows == 0) {
        hipLaunchKernelGGL(count_rows_kernel, dim3(1), dim3(1024), 0, s, a.tokens, a.rows, w.share, w.ticket);
        hipLaunchKernelGGL(mean_terms_kernel, dim3(1), dim3(kT), 0, s, w.term, a.rows, w.share, loss);
    } else if (a.type == ADPSGD_TYPE_F32) launch_policy_of<F32>(g, w.ticket, s);
    else if (a.type == ADPSGD_TYPE_BF16) launch_policy_of<Bf16>(g, w.ticket, s);
    else launch_policy_of<F16>(g, w.ticket, s);
    return hipGetLastError();
}

hipError_t launch_preference(const LossRows& a, const int64_t* offsets, int64_t pairs, const float* ref, double beta, double smoothing, float* loss,
                             void* dz, float* sums, float* margins, void* ws, hipStream_t s) {
    GradientArgs g{};
    g.row = row_args(a, kPreference, laid_out(ws, a.rows));
    g.dz = dz;
    g.margins = margins;
    g.pairs = pairs;
    g.smoothing = smoothing;
    g.loss = loss;
    if (a.type == ADPSGD_TYPE_F32) launch_preference_of<F32>(g, offsets, ref, beta, sums, margins, s);
    else if (a.type == ADPSGD_TYPE_BF16) launch_preference_of<Bf16>(g, offsets, ref, beta, sums, margins, s);
    else launch_preference_of<F16>(g, offsets, ref, beta, sums, margins, s);
    if (a.rows == 0) hipLaunchKernelGGL(preference_loss_kernel, dim3(1), dim3(64), 0, s, margins, pairs, smoothing, loss);
    return hipGetLastError();
}

}  // namespace adpsgd_impl
