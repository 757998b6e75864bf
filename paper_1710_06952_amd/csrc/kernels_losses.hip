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
// product, v_exp_f32, sum, twice for a gradient) take about half of the time that its bytes take.  Measured: log-probabilities of
// 8000 x 32 000 in fp16 73 us (6.3 TB/s), policy loss of 4096 x 65 536 in bf16 172 us (5.6 TB/s of what the counted rows need), preference
// loss of 8 pairs over 50 001 tokens 61 + 102 us: its gradient needs sums over whole sequences first, so the logits are read twice, the
// second time in reverse and partly from the last-level cache.
//
// Rows begin at any multiple of the element (odd vocabularies).
// Exponentials, sums and the gradient are in 32 bits, log-probabilities, their sums over a sequence and the loss in 64.  A row is summed in an
// order that depends on the sizes and the alignment of the rows alone.
#include <algorithm>

#include "device_common.hpp"
#include "operators.hpp"

namespace adpsgd_impl {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = 1.925963033500e-8f;
constexpr int kT = 256;
constexpr int64_t kCountHere = 1024;    // rows that a block of the policy kernel counts itself: a launch less where launches are the time
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
__device__ __forceinline__ double log_prob(float at, Stat st) {
    const double l = static_cast<double>(at) - static_cast<double>(st.m) - log_of(st.s);
    return st.s < INFINITY ? l : NAN;                    // NaN too, of which frexp says nothing
}
// Exponentials of what there is one of in a row: s is off by 1e-7, so 32 bits lose nothing.
__device__ __forceinline__ float exp_near(float x) {     // the rounding of x log2 e made good
    const float t = x * kLog2e, rest = fmaf(x, kLog2e, -t) + x * kLog2eRest, e = __builtin_amdgcn_exp2f(t);
    return fabsf(t) < 126.0f ? fmaf(e, rest * 0.6931471805599453f, e) : e;
}
// exp(d) - 1 - d
__device__ __forceinline__ float exp_less_line(float d) {
    if (fabsf(d) > 0.25f) return exp_near(d) - 1.0f - d;
    float p = fmaf(d, 1.0f / 40320.0f, 1.0f / 5040.0f);
    p = fmaf(d, p, 1.0f / 720.0f);
    p = fmaf(d, p, 1.0f / 120.0f);
    p = fmaf(d, p, 1.0f / 24.0f);
    p = fmaf(d, p, 1.0f / 6.0f);
    p = fmaf(d, p, 0.5f);
    return d * d * p;
}
// dL/dl and the loss term of one row, both times the number of counted rows.
struct RowNumbers {
    float old, adv, ref;
    __device__ __forceinline__ RowNumbers(const PolicyTerms& t, int64_t row) : old(t.old[row]), adv(t.adv[row]), ref(t.ref ? t.ref[row] : 0.0f) {}
};
__device__ __forceinline__ void policy_row(const PolicyTerms& t, const RowNumbers& n, double l, float& slope, float& term) {
    const float A = n.adv, rho = exp_near(static_cast<float>(l - static_cast<double>(n.old)));
    const float free = rho * A;
    // fmin and fmax pass over a NaN: the ratio is kept as it is unless it is outside
    const float lo = 1.0f - t.clip_low, hi = 1.0f + t.clip_high, held = (rho < lo ? lo : rho > hi ? hi : rho) * A;
    term = held < free ? -held : -free;
    slope = held < free ? 0.0f : -free;
    if (t.ref) {
        const float d = static_cast<float>(static_cast<double>(n.ref) - l), q = exp_less_line(d);
        term = fmaf(t.kl, q, term);
        slope = fmaf(-t.kl, q + d, slope);
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
    float slope = 0.0f, term = 0.0f;
    if (token >= 0) policy_row(a.policy, RowNumbers(a.policy, row), l, slope, term);
    a.logp[row] = static_cast<float>(l);
    a.term[row] = term;
    a.coef[row] = slope * *a.share;
}

// (m, s) of the vectors v0 <= v < v1 of a row that this thread takes
template <class E, bool kFine>
__device__ __forceinline__ Stat thread_stat(const typename E::Raw* row, const Cut<E>& cut, int v0, int v1) {
    // 32 terms at a time in 32 bits, their sums in 64: one long sum in 32 bits is too large by 3e-8 after 200 terms and 5e-8 after 500
    float most = -INFINITY;
    double sum = 0.0;
    for (int v = v0 + static_cast<int>(threadIdx.x); v < v1; v += kT * kUnroll) {
        v4u x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            x[u] = v4u{kNothing<E>, kNothing<E>, kNothing<E>, kNothing<E>};
            if (v + u * kT < v1) x[u] = load_vector<E, kFine>(row, cut.at(v + u * kT));
        }
        float f[kUnroll][E::kN], top = -INFINITY;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            E::unpack(x[u], f[u]);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) top = fmaxf(top, f[u][i]);
        }
        const float m = fmaxf(most, top), base = base_of(m);
        float part[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            part[u] = 0.0f;
#pragma unroll
            for (int i = 0; i < E::kN; ++i) part[u] += exp_in_sum<kFine>(f[u][i] - base);
        }
        sum = sum * static_cast<double>(exp_in_sum<true>(most - base)) + static_cast<double>((part[0] + part[1]) + (part[2] + part[3]));
        most = m;
    }
    static_assert(kUnroll == 4, "");
    return Stat{most, static_cast<float>(sum)};
}

// grid: rows * splits.
template <class E, bool kFine>
__global__ __launch_bounds__(kT) void row_stats_kernel(const RowArgs a) {
    __shared__ Stat at[kT / 64];
    const int64_t row = blockIdx.x / a.splits;
    const int part = blockIdx.x % a.splits;
    if (a.tokens[row] < 0) {
        if (a.splits == 1 && threadIdx.x == 0) finish_row<E>(a, row, Stat{0.0f, 1.0f});
        return;
    }
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    const Cut<E> cut(z, static_cast<int>(a.vocab));
    const int each = (cut.vectors + a.splits - 1) / a.splits, v0 = part * each, v1 = v0 + each < cut.vectors ? v0 + each : cut.vectors;
    Stat st = thread_stat<E, kFine>(z, cut, v0, v1);
    if (part == 0 && cut.single() >= 0) st = joined(st, of_one(E::get(z + cut.single())));
    st = block_joined<kT / 64>(st, at);
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
    st = lanes_joined<64>(st);
    if ((threadIdx.x & 63) == 0) finish_row<E>(a, row, st);
}

// In the gradient the rounding of log2 e is 1.3e-8 of z - m, in the same direction in every element: 1e-7 where fp32 holds it, nothing in 16 bits.
template <class E>
__device__ __forceinline__ float exp_in_gradient(float d) { return exp_in_sum<E::kN == 4>(d); }
template <class E>
__device__ __forceinline__ float gradient_at(float z, bool hot, float m, float scale, float coef) {
    return exp_in_gradient<E>(z - m) * scale + (hot ? coef : 0.0f);
}
// d[i] = exp(z[i] - m) scale
template <class E>
__device__ __forceinline__ void gradient_of(v4u x, float m, float scale, float* d) {
    E::unpack(x, d);
#pragma unroll
    for (int i = 0; i < E::kN; ++i) d[i] = exp_in_gradient<E>(d[i] - m) * scale;
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
// The loss of the margins, by one wavefront.
__device__ __forceinline__ void preference_loss(const float* margins, int64_t pairs, double smoothing, float* loss) {
    double sum = 0.0;
    for (int64_t q = threadIdx.x; q < pairs; q += 64) {
        const double x = margins[q];
        sum += x == x ? (1.0 - smoothing) * softplus(-x) + smoothing * softplus(x) : x;
    }
    sum = wave_sum(sum);
    if (threadIdx.x == 0) *loss = static_cast<float>(sum / static_cast<double>(pairs));
}

// grid: rows * blocks.  The last rows first: they are the ones that the pass before has left in the last-level cache.
template <class E>
__global__ __launch_bounds__(kT) void logit_gradient_kernel(const GradientArgs g) {
    const RowArgs& a = g.row;
    if (g.margins && blockIdx.x == 0 && threadIdx.x < 64) preference_loss(g.margins, g.pairs, g.smoothing, g.loss);
    const int64_t row = a.rows - 1 - blockIdx.x / g.blocks;
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    typename E::Raw* dz = static_cast<typename E::Raw*>(g.dz) + row * a.vocab;
    const Cut<E> cut(dz, static_cast<int>(a.vocab));     // stores aligned; loads too where rows of both lie alike
    const int64_t token = a.tokens[row];
    const float coef = token < 0 ? 0.0f : a.coef[row];
    const Stat st = token < 0 ? Stat{0.0f, 1.0f} : a.stat[row];
    const float scale = -coef / st.s;
    const int v0 = static_cast<int>(blockIdx.x % g.blocks) * (kT * kUnroll) + static_cast<int>(threadIdx.x);
    const int hot = token < a.vocab ? static_cast<int>(token) : -1, single = blockIdx.x % g.blocks == 0 ? cut.single() : -1;
    if (single >= 0) E::put(dz + single, coef == 0.0f ? 0.0f : gradient_at<E>(E::get(z + single), single == hot, st.m, scale, coef));
    v4u x[kUnroll];
    float d[E::kN];
    if (coef == 0.0f) {                 // nothing to read
#pragma unroll
        for (int i = 0; i < E::kN; ++i) d[i] = 0.0f;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (v0 + u * kT < cut.vectors) store_vector<E>(dz, cut.at(v0 + u * kT), d);
        return;
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
        if (v0 + u * kT < cut.vectors) x[u] = load_vector<E, false>(z, cut.at(v0 + u * kT));
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
        if (v0 + u * kT < cut.vectors) {
            gradient_of<E>(x[u], st.m, scale, d);
            store_vector<E>(dz, cut.at(v0 + u * kT), d);
        }
    // the token's element once more, by the thread that has stored it without coef
    const int back = cut.vector_of(hot) - v0;
    if (cut.vector_of(hot) >= 0 && back >= 0 && back < kT * kUnroll && back % kT == 0) E::put(dz + hot, gradient_at<E>(E::get(z + hot), true, st.m, scale, coef));
}

// ---- policy ----------------------------------------------------------------------------------------------
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

// kWaves wavefronts a row, up to kHeld vectors a thread in registers.  kPerSimd wavefronts a SIMD:
// with two blocks on a compute unit one loads or stores while the other computes, which its registers have to leave room for.
template <class E, int kWaves, int kHeld, int kPerSimd>
__global__ __launch_bounds__(kWaves * 64, kPerSimd) void policy_rows_kernel(const GradientArgs g) {
    constexpr int kThreads = kWaves * 64;
    __shared__ Stat at[kWaves];
    __shared__ float counts[kWaves];
    __shared__ float of_row;
    const RowArgs& a = g.row;
    const int64_t row = blockIdx.x;
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    typename E::Raw* dz = static_cast<typename E::Raw*>(g.dz) + row * a.vocab;
    const Cut<E> cut(dz, static_cast<int>(a.vocab));
    const int64_t token = a.tokens[row];
    const int single = cut.single();
    float coef = 0.0f, m = 0.0f, scale = 0.0f, alone = -INFINITY, value = 0.0f;
    v4u x[kHeld];
    if (token >= 0) {                   // uniform over the block
        // in front of the row: behind it they would be waited for, and with them the whole row
        value = token < a.vocab ? E::get(z + token) : NAN;
        float share = a.rows <= kCountHere ? 0.0f : *a.share;
        const RowNumbers numbers(a.policy, row);
        if (single >= 0) alone = E::get(z + single);
        __builtin_amdgcn_sched_barrier(0);
        // No load under a condition (places beyond the end read the last vector), so that each is waited for by itself: behind
        // branches all are waited for before the first is used.
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int v = u * kThreads + static_cast<int>(threadIdx.x);
            x[u] = load_vector<E, false>(z, cut.at(v < cut.vectors ? v : cut.vectors - 1));
        }
        if (a.rows <= kCountHere) share = 1.0f / fmaxf(counted_rows<kWaves>(a.tokens, a.rows, counts), 1.0f);
        __builtin_amdgcn_sched_barrier(0);
        Stat st{-INFINITY, 0.0f};
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            float f[E::kN], top = -INFINITY;
            if ((u + 1) * kThreads > cut.vectors)        // uniform
                x[u] = u * kThreads + static_cast<int>(threadIdx.x) < cut.vectors ? x[u] : v4u{kNothing<E>, kNothing<E>, kNothing<E>, kNothing<E>};
            asm volatile("" : "+v"(x[u]));               // held packed, however it was come by
            E::unpack(x[u], f);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) top = fmaxf(top, f[i]);
            const float m = fmaxf(st.m, top), base = base_of(m);
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < E::kN; ++i) part += exp_in_sum<false>(f[i] - base);
            st.s = fmaf(st.s, exp_in_sum<true>(st.m - base), part);
            st.m = m;
            __builtin_amdgcn_sched_barrier(0);           // one vector after the other: unpacked, they would not all fit
        }
        if (single >= 0) st = joined(st, of_one(alone));
        st = block_joined<kWaves>(st, at);
        if (threadIdx.x < 64) {
            const double l = log_prob(value, st);
            float slope, term;
            policy_row(a.policy, numbers, l, slope, term);
            if (threadIdx.x == 0) {
                a.logp[row] = static_cast<float>(l);
                a.term[row] = term;
                of_row = slope * share;
            }
        }
        __syncthreads();
        coef = of_row;
        m = st.m;
        scale = -coef / st.s;
    } else if (threadIdx.x == 0) {
        a.logp[row] = 0.0f;
        a.term[row] = 0.0;
    }
    const int hot = token < a.vocab ? static_cast<int>(token) : -1;
    const bool zero = coef == 0.0f;     // NaN is not
    if (single >= 0) E::put(dz + single, zero ? 0.0f : gradient_at<E>(alone, single == hot, m, scale, coef));
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        const int v = u * kThreads + static_cast<int>(threadIdx.x);
        if (v < cut.vectors) {
            float d[E::kN];
            if (zero) {
#pragma unroll
                for (int i = 0; i < E::kN; ++i) d[i] = 0.0f;
            } else {
                asm volatile("" : "+v"(x[u]));           // unpacked anew, not kept unpacked since the sum
                gradient_of<E>(x[u], m, scale, d);
            }
            store_vector<E>(dz, cut.at(v), d);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // the token's element once more, by the thread that has stored it without coef
    if (cut.vector_of(hot) >= 0 && cut.vector_of(hot) % kThreads == static_cast<int>(threadIdx.x)) E::put(dz + hot, gradient_at<E>(value, true, m, scale, coef));
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
    float* share;           // 1 / counted
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
    w.share = reinterpret_cast<float*>(take(sizeof(float)));
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
    r.splits = split_of(r.rows, r.vocab / E::kN);
    const dim3 grid(static_cast<uint32_t>(r.rows * r.splits));
    if (r.mode == kPreference) hipLaunchKernelGGL((row_stats_kernel<E, true>), grid, dim3(kT), 0, s, r);
    else hipLaunchKernelGGL((row_stats_kernel<E, false>), grid, dim3(kT), 0, s, r);
    if (r.splits > 1) hipLaunchKernelGGL(join_stats_kernel<E>, dim3(static_cast<uint32_t>((r.rows + kT / 64 - 1) / (kT / 64))), dim3(kT), 0, s, r);
}
template <class E>
void launch_gradient(GradientArgs g, hipStream_t s) {
    const int64_t vectors = g.row.vocab / E::kN;
    g.blocks = std::max<int64_t>(1, (vectors + kT * kUnroll - 1) / (kT * kUnroll));
    hipLaunchKernelGGL(logit_gradient_kernel<E>, dim3(static_cast<uint32_t>(g.row.rows * g.blocks)), dim3(kT), 0, s, g);
}

template <class E>
void launch_policy_of(GradientArgs g, hipStream_t s) {
    const int64_t rows = g.row.rows, vectors = g.row.vocab / E::kN;
    const dim3 grid(static_cast<uint32_t>(rows));
    const bool apart = vectors < 2 || vectors > 16384;
    if (apart || rows > kCountHere) hipLaunchKernelGGL(count_rows_kernel, dim3(1), dim3(1024), 0, s, g.row.tokens, rows, const_cast<float*>(g.row.share));
    if (apart) {                         // perhaps none behind the first 16-byte address, or more than a block's registers hold
        launch_stats<E>(g.row, s);
        launch_gradient<E>(g, s);
    } else if (vectors <= 256) hipLaunchKernelGGL((policy_rows_kernel<E, 1, 4, 4>), grid, dim3(64), 0, s, g);
    else if (vectors <= 1024) hipLaunchKernelGGL((policy_rows_kernel<E, 4, 4, 8>), grid, dim3(256), 0, s, g);
    else if (vectors <= 4096) hipLaunchKernelGGL((policy_rows_kernel<E, 8, 8, 8>), grid, dim3(512), 0, s, g);
    else if (vectors <= 8192) hipLaunchKernelGGL((policy_rows_kernel<E, 16, 8, 8>), grid, dim3(1024), 0, s, g);
    else hipLaunchKernelGGL((policy_rows_kernel<E, 16, 16, 4>), grid, dim3(1024), 0, s, g);
    hipLaunchKernelGGL(mean_terms_kernel, dim3(1), dim3(1024), 0, s, g.row.term, g.row.tokens, rows, g.loss);
}
template <class E>
void launch_preference_of(const GradientArgs& g, const int64_t* offsets, const float* ref, double beta, float* sums, float* margins, hipStream_t s) {
    if (g.row.rows > 0) launch_stats<E>(g.row, s);
    hipLaunchKernelGGL(preference_pairs_kernel, dim3(static_cast<uint32_t>(g.pairs)), dim3(kT), 0, s, g.row.term, offsets, g.pairs, g.row.rows, ref, beta,
                       g.smoothing, sums, margins, g.row.coef);
    if (g.row.rows > 0) launch_gradient<E>(g, s);
}

__global__ __launch_bounds__(64) void preference_loss_kernel(const float* margins, int64_t pairs, double smoothing, float* loss) {
    preference_loss(margins, pairs, smoothing, loss);
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
        hipLaunchKernelGGL(mean_terms_kernel, dim3(1), dim3(1024), 0, s, w.term, a.tokens, a.rows, loss);
    } else if (a.type == ADPSGD_TYPE_F32) launch_policy_of<F32>(g, s);
    else if (a.type == ADPSGD_TYPE_BF16) launch_policy_of<Bf16>(g, s);
    else launch_policy_of<F16>(g, s);
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
