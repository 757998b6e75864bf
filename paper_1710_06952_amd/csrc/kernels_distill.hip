// Distillation from a teacher's top logits, and its gradient for the logits.
//
// A row has logits z and up to k entries (v_j, t_j) of the teacher.  With p = softmax(t / T) over its entries, q_T = softmax(z / T), q = softmax(z):
//   KL = sum_j p_j (log p_j - log q_T[v_j])
//      = [sum_j p_j t_j / T - log Z + sum_j p_j (b - z[v_j]) / T] + (m - b) / T + log s        Z and b = max z[v_j] of the entries, m and s of the row
//   The first part needs no pass over z.  b is what z[v_j] and m are taken from: neither sum of differences has another sign in it, while p_j z[v_j] / T and m / T of
//   their own would leave 2^-53 |m| / T of each other.
//   dL/dz = cs (q_T - sum_j p_j onehot(v_j)) + ch (q - onehot(token)),   cs = (1 - a) T / counted,  ch = a / counted
//
//   teacher_row      p and the first part of KL by one wavefront; entries of the same token become one, and the token itself is the last
//   distill_rows     all of a row with its logits held in registers: they are read once
//   stats, gradient  the same in two passes, for rows that registers do not hold, and for few rows, which are split over the chip
//
// The gradient of all elements is stored without the entries first; behind a barrier the few that have an entry are stored again.  (The pass
// would have to look for its own elements among the entries.)
//
// Exponentials, sums of a row and the gradient are in 32 bits, what there is one of in a row or an entry in 64.  Where a teacher and a row are sure of the same token,
// q - p there is what is left of two numbers next to 1: in fp32 it is computed in 64 bits, and the sums of a row are in 64 bits too (2^-25 of a sum of
// 1 + 10^-3 would be 3e-5 of that; 1 to 5 % of the time).  Orders depend on the sizes and the alignment of the gradient alone.
//
// Bound: memory, 2 or 4 bytes an element in and out: 4096 x 65 536 in bf16, a fifth of the rows not counted, 172 us (5.6 TB/s).  With labels at another
// temperature the instructions: two softmaxes of 2001 x 50 001 in fp16 84 us (4.5 TB/s).
#include <cmath>

#include "loss_rows.hpp"

namespace adpsgd_impl {
namespace {

constexpr int kUnroll = 4;              // vectors of a thread on their way at once
constexpr int64_t kCountHere = 1024;    // rows that a block counts itself: a launch less where launches are the time
constexpr int64_t kSplitBlocks = 1024;  // blocks that fill the chip: rows are split over the vocabulary up to this many

struct Entry {
    int v;                      // of the vocabulary, or -1: nothing
    float p, rest;              // p in two parts
};
// log2 e / T as it rounds, and in two parts, the second positive: a difference of -infinity is e^-infinity by both.
struct Heat {
    float near, hi, lo;
};
template <class E>
using Sum = std::conditional_t<E::kN == 4, double, float>;
template <class S>
struct Stat2 {
    float m;
    S s, s1;                    // the largest value, sum exp((z - m) / T), sum exp(z - m)
};
struct DistillArgs {
    const void* z;
    const int64_t* tokens;
    int64_t rows, vocab, ld;
    const void* t;              // teacher
    int32_t t_type;
    const int64_t* t_tokens;
    int64_t k, ld_t, ld_tokens;
    double T, inv_T, soft, hard;        // soft: 1 - a, hard: a
    float cs, ch;               // times 1 / counted
    Heat heat;
    const float* share;         // 1 / counted, where rows > kCountHere
    Entry* entries;             // [row][k + 1]
    double* first;              // of KL: its first part ...
    float* best;                // ... and the largest of a row's logits that have an entry
    double* term;
    void* parts;                // in passes: Stat2 of parts of rows
    int splits, together;       // ... of a row; teacher's rows of a block
    float* loss;
    int64_t blocks;             // of a row, in the gradient's pass
    void* dz;
    float *kl, *logp;           // logp may be nullptr
};

template <bool kFine>
__device__ __forceinline__ float warm(float d, const Heat& h) { return __builtin_amdgcn_exp2f(kFine ? fmaf(d, h.hi, d * h.lo) : d * h.near); }
// In the sums of a row: 32-bit logits take the second part as well.  Beside 16 bits its 3e-8 of z / T is left out: 2e-7 of log s, which is 5 to 15.
template <class E>
__device__ __forceinline__ float warm_in_sum(float d, const Heat& h) { return warm<E::kN == 4>(d, h); }
template <bool kTwo, class S>
__device__ __forceinline__ Stat2<S> joined2(Stat2<S> a, Stat2<S> b, const Heat& h) {
    const float m = fmaxf(a.m, b.m), base = base_of(m);
    Stat2<S> r{m, a.s * warm<true>(a.m - base, h) + b.s * warm<true>(b.m - base, h), 0};
    if (kTwo) r.s1 = a.s1 * exp_in_sum<true>(a.m - base) + b.s1 * exp_in_sum<true>(b.m - base);
    return r;
}
template <class S>
__device__ __forceinline__ Stat2<S> of_one2(float z, const Heat& h) { return Stat2<S>{z, warm<true>(z - base_of(z), h), exp_in_sum<true>(z - base_of(z))}; }
template <bool kTwo, int kLanes, class S>
__device__ __forceinline__ Stat2<S> lanes_joined2(Stat2<S> a, const Heat& h) {
    float m = a.m;
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    S s = a.s * warm<true>(a.m - base_of(m), h), s1 = kTwo ? a.s1 * exp_in_sum<true>(a.m - base_of(m)) : 0;
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) {
        s += __shfl_xor(s, off, 64);
        if (kTwo) s1 += __shfl_xor(s1, off, 64);
    }
    return Stat2<S>{m, s, s1};
}
template <bool kTwo, int kWaves, class S>
__device__ __forceinline__ Stat2<S> block_joined2(Stat2<S> a, const Heat& h, Stat2<S>* at) {
    a = lanes_joined2<kTwo, 64>(a, h);
    if (kWaves == 1) return a;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = a;
    __syncthreads();
    return lanes_joined2<kTwo, kWaves>(at[threadIdx.x % kWaves], h);
}

// ---- the teacher's rows ------------------------------------------------------------------------------------
// exp(x) of what there is one of in an entry: x in 64 bits as a rounding and its rest.
__device__ __forceinline__ float exp_of_entry(double x) {
    const float hi = static_cast<float>(x), t = hi * kLog2e;
    const float rest = fmaf(hi, kLog2e, -t) + hi * kLog2eRest + static_cast<float>(x - static_cast<double>(hi)) * kLog2e, e = __builtin_amdgcn_exp2f(t);
    return fabsf(t) < 126.0f ? fmaf(e, rest * 0.6931471805599453f, e) : e;
}
// ... in 64 bits, x <= 0 or NaN: 2^n e^r with |r| <= ln 2 / 2, the series up to r^11 (the next term is 6e-15).
__device__ __forceinline__ double exp64(double x) {
    if (x < -745.0) return 0.0;
    const double n = rint(x * 1.4426950408889634), r = fma(-n, 0x1.ef35793c7673p-45, fma(-n, 0x1.62e42fefa38p-1, x));
    double p = 1.0 / 39916800.0;
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    return x == x ? ldexp(fma(p, r, 1.0), static_cast<int>(n)) : x;
}
__device__ __forceinline__ float teacher_logit(const void* t, int32_t type, int64_t at) {
    if (type == ADPSGD_TYPE_F32) return F32::get(static_cast<const float*>(t) + at);
    const uint16_t* p = static_cast<const uint16_t*>(t) + at;
    return type == ADPSGD_TYPE_BF16 ? Bf16::get(p) : F16::get(p);
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}

// Words of LDS for a row: entries (token, value, place in the table) and a table of twice as many places (token, first entry).
__host__ __device__ constexpr int teacher_places(int k) {
    int n = 64;
    while (n < 2 * (k + 1)) n *= 2;
    return n;
}
static_assert(60 * 1024 > 4 * (3 * 1025 + 2 * 4096) + 12 * 1025, "the words of 1024 entries, and the entries, beside what a block has of its own");
__host__ __device__ constexpr int teacher_words(int k) { return 3 * (k + 1) + 2 * teacher_places(k); }

// One wavefront, a row: leaves its entries in `out` (k + 1 of them), with `words` of LDS, and gives the first part of KL: NaN where there is none, -infinity where
// there is no entry.  best: the largest logit that has an entry, 0 where there is none but -infinity.
template <class E>
__device__ __forceinline__ double teacher_row(const DistillArgs& a, int64_t row, int64_t token, int* words, Entry* out, float& best) {
    const int lane = threadIdx.x & 63, k = static_cast<int>(a.k), places = teacher_places(k);
    int* token_of = words;
    float* value = reinterpret_cast<float*>(token_of + (k + 1));
    int *place_of_entry = token_of + 2 * (k + 1), *key = token_of + 3 * (k + 1), *owner = key + places;
    for (int i = lane; i < places; i += 64) {
        key[i] = -1;
        owner[i] = k + 1;
    }
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    bool beyond = false, some = false;
    float top = -INFINITY;
    for (int j = lane; j < k; j += 64) {
        const int64_t v = a.t_tokens[row * a.ld_tokens + j];
        const float t = v < 0 ? -INFINITY : teacher_logit(a.t, a.t_type, row * a.ld_t + j);
        token_of[j] = v < 0 || v >= a.vocab ? -1 : static_cast<int>(v);
        value[j] = t;
        beyond = beyond || v >= a.vocab;
        some = some || v >= 0;
        top = t != t ? NAN : top != top ? top : fmaxf(top, t);       // fmax passes over a NaN
    }
    if (lane == 0) {                                     // the row's own token, an entry that weighs nothing
        token_of[k] = token < a.vocab ? static_cast<int>(token) : -1;
        value[k] = 0.0f;
    }
    beyond = __any(beyond || top != top);
    some = __any(some);
    top = wave_max(top);
    wave_lds_sync();
    double Z = 0.0, with_t = 0.0, with_z = 0.0;          // with_z: from a lane's largest logit so far
    float most = -INFINITY;
    for (int j = lane; j < k; j += 64) {
        const int v = token_of[j];
        const double x = (static_cast<double>(value[j]) - static_cast<double>(top)) * a.inv_T;
        const float e = v < 0 ? 0.0f : exp_of_entry(x);
        value[j] = e;
        if (e != 0.0f) {
            const float own = E::get(z + v), was = most == -INFINITY ? own : most;
            most = fmaxf(was, own);
            const double from = base_of(most);
            with_z += Z * (from - static_cast<double>(base_of(was))) + static_cast<double>(e) * (from - static_cast<double>(own));
            Z += static_cast<double>(e);
            with_t += static_cast<double>(e) * x;
        }
    }
    best = base_of(wave_max(most));
    if (most > -INFINITY) with_z += Z * (static_cast<double>(best) - static_cast<double>(most));
    Z = wave_sum(Z);
    with_t = wave_sum(with_t);
    with_z = wave_sum(with_z);
    // one entry for each token: the first of its entries
    for (int j = lane; j <= k; j += 64) {
        const int v = token_of[j];
        int at = -1;
        if (v >= 0) {
            at = static_cast<int>(static_cast<uint32_t>(v) * 2654435761u >> 7) & (places - 1);
            for (;;) {                                   // less than half of the places are taken
                const int was = atomicCAS(&key[at], -1, v);
                if (was == -1 || was == v) break;
                at = (at + 1) & (places - 1);
            }
            atomicMin(&owner[at], j);
        }
        place_of_entry[j] = at;
    }
    wave_lds_sync();
    bool twice = false;
    for (int j = lane; j < k; j += 64) twice = twice || (place_of_entry[j] >= 0 && owner[place_of_entry[j]] != j);      // the token adds nothing
    twice = __any(twice);
    const double scale = 1.0 / Z;
    for (int j = lane; j <= k; j += 64) {
        const int at = place_of_entry[j];
        Entry e{at >= 0 && owner[at] == j ? token_of[j] : -1, 0.0f, 0.0f};
        if (e.v >= 0) {
            double w = value[j];
            if (twice)
                for (int i = j + 1; i <= k; ++i) w += place_of_entry[i] == at ? static_cast<double>(value[i]) : 0.0;
            if (some) {
                e.p = static_cast<float>(w * scale);
                e.rest = static_cast<float>(w * scale - static_cast<double>(e.p));
            }
        }
        out[j] = e;
    }
    if (beyond || (some && !(Z > 0.0 && Z < INFINITY))) return NAN;
    if (!some) return -INFINITY;
    const float near = static_cast<float>(Z);
    return with_t * scale - (log_of(near) + (Z - static_cast<double>(near)) * scale) + with_z * scale * a.inv_T;
}

// ---- what one thread does once for a row --------------------------------------------------------------------
struct RowEnd {
    float cs, ch;               // of exp((z - m) / T) and exp(z - m): cs / s, ch / s1
    float cp, ct;               // of an entry's p, of the token
    double q, q1;               // 1 / s and 1 / s1, for entries
};
// log s.
__device__ __forceinline__ double log_of_sum(float s) { return log_of(s); }
__device__ __forceinline__ double log_of_sum(double s) {
    const float near = static_cast<float>(s);
    return log_of(near) + (s - static_cast<double>(near)) / s;
}
__device__ __forceinline__ void empty_row(const DistillArgs& a, int64_t row) {
    a.kl[row] = 0.0f;
    if (a.logp) a.logp[row] = 0.0f;
    a.term[row] = 0.0;
}
template <bool kTwo, class S>
__device__ __forceinline__ RowEnd end_of_row(const DistillArgs& a, int64_t row, double first, float best, float at, const Stat2<S>& st, float share, bool writes, double& term) {
    const bool there = first != static_cast<double>(-INFINITY), good = st.s > 0 && st.s < static_cast<S>(INFINITY);
    double kl = there ? first + (static_cast<double>(st.m) - static_cast<double>(best)) * a.inv_T + log_of_sum(st.s) : 0.0, logp = 0.0;
    if (!good || first != first) kl = NAN;
    if (a.hard > 0.0) {
        const S s1 = kTwo ? st.s1 : st.s;
        logp = static_cast<double>(at) - static_cast<double>(st.m) - log_of_sum(s1);
        if (!(s1 > 0 && s1 < static_cast<S>(INFINITY))) logp = NAN;
    } else if (at != at) {
        kl = NAN;                                        // the token is beyond the vocabulary
    }
    term = a.soft * a.T * a.T * kl - (a.hard > 0.0 ? a.hard * logp : 0.0);
    if (writes) {
        a.kl[row] = static_cast<float>(kl);
        if (a.logp) a.logp[row] = static_cast<float>(logp);
        a.term[row] = term;
    }
    RowEnd e;
    e.cp = there ? a.cs * share : 0.0f;
    e.ct = a.ch * share;
    if (kl != kl || logp != logp) e.cp = NAN;
    e.cs = e.cp / static_cast<float>(st.s);
    e.ch = kTwo ? e.ct / static_cast<float>(st.s1) : 0.0f;
    if (!kTwo) e.cs += e.ct / static_cast<float>(st.s);  // one softmax for both
    e.q = 1.0 / static_cast<double>(st.s);
    e.q1 = kTwo ? 1.0 / static_cast<double>(st.s1) : 0.0;
    return e;
}
template <class E, bool kTwo>
__device__ __forceinline__ float slope_at(float z, float m, const RowEnd& e, const Heat& h) {
    float d = warm<E::kN == 4>(z - m, h) * e.cs;
    if (kTwo) d = fmaf(exp_in_gradient<E>(z - m), e.ch, d);
    return d;
}
template <class E, bool kTwo>
__device__ __forceinline__ void slopes_of(v4u x, float m, const RowEnd& e, const Heat& h, float* d) {
    E::unpack(x, d);
#pragma unroll
    for (int i = 0; i < E::kN; ++i) d[i] = slope_at<E, kTwo>(d[i], m, e, h);
}
// An element that has an entry.
template <class E, bool kTwo>
__device__ __forceinline__ void store_entry(const DistillArgs& a, const Entry& n, int64_t row, int64_t token, float m, const RowEnd& e) {
    const float z = E::get(static_cast<const typename E::Raw*>(a.z) + row * a.ld + n.v);
    typename E::Raw* to = static_cast<typename E::Raw*>(a.dz) + row * a.vocab + n.v;
    if (E::kN == 8) {                                    // 16 bits hold no more than this
        E::put(to, slope_at<E, kTwo>(z, m, e, a.heat) - e.cp * n.p - (n.v == token ? e.ct : 0.0f));
        return;
    }
    const double x = static_cast<double>(z) - static_cast<double>(m), q = exp64(x * a.inv_T) * e.q;
    double d = static_cast<double>(e.cp) * ((q - static_cast<double>(n.p)) - static_cast<double>(n.rest));
    if (e.ct != 0.0f) d += static_cast<double>(e.ct) * ((kTwo ? exp64(x) * e.q1 : q) - (n.v == token ? 1.0 : 0.0));
    E::put(to, static_cast<float>(d));
}

// ---- rows held in registers -----------------------------------------------------------------------------------
// What lanes behind the end of a row read: 16 bytes of -infinity.
__device__ const uint32_t kNone[3][4] = {{kNothing<F32>, kNothing<F32>, kNothing<F32>, kNothing<F32>},
                                         {kNothing<Bf16>, kNothing<Bf16>, kNothing<Bf16>, kNothing<Bf16>},
                                         {kNothing<F16>, kNothing<F16>, kNothing<F16>, kNothing<F16>}};
template <class E>
constexpr int kTypeOf = E::kN == 4 ? 0 : 1;
template <>
constexpr int kTypeOf<F16> = 2;

// The gradient beside 16 bits: cs exp((z - m) / T) = 2^(z log2 e / T + c), c = log2 cs - m log2 e / T, is one FMA and one exponential.  c is rounded, which makes
// all of a row's q too large or small by 2^-24 |c|: under 1e-5 for |m log2 e / T| < 128.  Other rows, and signs, take the long way.
struct RowLine {
    float c, c1;
    bool short_way;
};
template <class E, bool kTwo>
__device__ __forceinline__ RowLine line_of(const RowEnd& e, float m, const Heat& h) {
    const float at = m * h.near, at1 = m * kLog2e;
    const bool good = E::kN == 8 && fabsf(at) < 128.0f && (!kTwo || fabsf(at1) < 128.0f) && e.cs >= 0.0f && e.ch >= 0.0f;
    return RowLine{__builtin_amdgcn_logf(e.cs) - at, __builtin_amdgcn_logf(e.ch) - at1, good};
}

// kWaves wavefronts a row, up to kHeld vectors a thread; as policy_rows_kernel of the policy loss.  The first wavefront does the teacher's row in front of
// its own loads, while those of the others are on their way.
template <class E, bool kTwo, int kWaves, int kHeld, int kPerSimd>
__global__ __launch_bounds__(kWaves * 64, kPerSimd) void distill_rows_kernel(const DistillArgs a) {
    constexpr int kThreads = kWaves * 64;
    extern __shared__ int words[];                       // the entries, and the teacher's words
    __shared__ Stat2<Sum<E>> at[kWaves];
    __shared__ float counts[kWaves];
    __shared__ RowEnd of_row;
    const int64_t row = blockIdx.x;
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    typename E::Raw* dz = static_cast<typename E::Raw*>(a.dz) + row * a.vocab;
    const Cut<E> cut(dz, static_cast<int>(a.vocab));
    const int64_t token = a.tokens[row];
    const int single = cut.single();
    RowEnd end{};
    float m = 0.0f, alone = -INFINITY;
    Entry* list = reinterpret_cast<Entry*>(words);
    v4u x[kHeld];
    if (token >= 0) {                   // uniform over the block
        double first = 0.0;
        float best = 0.0f;
        if (threadIdx.x < 64) first = teacher_row<E>(a, row, token, words + sizeof(Entry) / sizeof(int) * (a.k + 1), list, best);
        const float value = token < a.vocab ? E::get(z + token) : NAN;
        float share = a.rows <= kCountHere ? 0.0f : *a.share;
        if (single >= 0) alone = E::get(z + single);
        __builtin_amdgcn_sched_barrier(0);
        // no load under a condition: each is waited for by itself
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int v = u * kThreads + static_cast<int>(threadIdx.x);
            const typename E::Raw* from = v < cut.vectors ? z + cut.at(v) : reinterpret_cast<const typename E::Raw*>(kNone[kTypeOf<E>]);
            x[u] = load_vector<E, false>(from, 0);
        }
        if (a.rows <= kCountHere) share = 1.0f / fmaxf(counted_rows<kWaves>(a.tokens, a.rows, counts), 1.0f);
        __builtin_amdgcn_sched_barrier(0);
        Stat2<Sum<E>> st{-INFINITY, 0, 0};
        const float e1 = in_vector(kLog2e);              // in vector registers: an operand in a scalar one costs most of an instruction more
        Heat h = a.heat;
        h.near = in_vector(h.near);
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            float f[E::kN], top = -INFINITY;
            asm volatile("" : "+v"(x[u]));               // held packed
            E::unpack(x[u], f);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) top = fmaxf(top, f[i]);
            const float most = fmaxf(st.m, top), base = base_of(most);
            Sum<E> part = 0, part1 = 0;
#pragma unroll
            for (int i = 0; i < E::kN; ++i) {
                part += warm_in_sum<E>(f[i] - base, h);
                if (kTwo) part1 += __builtin_amdgcn_exp2f((f[i] - base) * e1);
            }
            st.s = fma(st.s, static_cast<Sum<E>>(warm<true>(st.m - base, a.heat)), part);
            if (kTwo) st.s1 = fma(st.s1, static_cast<Sum<E>>(exp_in_sum<true>(st.m - base)), part1);
            st.m = most;
            __builtin_amdgcn_sched_barrier(0);           // one vector after the other: unpacked, they would not all fit
        }
        if (single >= 0) st = joined2<kTwo>(st, of_one2<Sum<E>>(alone, a.heat), a.heat);
        st = block_joined2<kTwo, kWaves>(st, a.heat, at);
        if (threadIdx.x < 64) {
            double term;
            const RowEnd e = end_of_row<kTwo>(a, row, first, best, value, st, share, threadIdx.x == 0, term);
            if (threadIdx.x == 0) of_row = e;
        }
        __syncthreads();
        end = of_row;
        m = st.m;
    } else if (threadIdx.x == 0) {
        empty_row(a, row);
    }
    const bool zero = end.cs == 0.0f && end.ch == 0.0f;  // NaN is not
    if (single >= 0) E::put(dz + single, zero ? 0.0f : slope_at<E, kTwo>(alone, m, end, a.heat));
    auto store = [&](const auto& of) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int v = u * kThreads + static_cast<int>(threadIdx.x);
            if (v < cut.vectors) {
                float d[E::kN];
                of(u, d);
                store_vector<E>(dz, cut.at(v), d);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const RowLine line = line_of<E, kTwo>(end, m, a.heat);
    if (zero) {
        store([&](int, float* d) {
#pragma unroll
            for (int i = 0; i < E::kN; ++i) d[i] = 0.0f;
        });
    } else if (line.short_way) {
        const float near = in_vector(a.heat.near), e1 = in_vector(kLog2e);
        store([&](int u, float* d) {
            asm volatile("" : "+v"(x[u]));               // unpacked anew, not kept unpacked since the sum
            E::unpack(x[u], d);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) {
                const float z = d[i];
                d[i] = __builtin_amdgcn_exp2f(fmaf(z, near, line.c));
                if (kTwo) d[i] += __builtin_amdgcn_exp2f(fmaf(z, e1, line.c1));
            }
        });
    } else {
        store([&](int u, float* d) {
            asm volatile("" : "+v"(x[u]));
            slopes_of<E, kTwo>(x[u], m, end, a.heat, d);
        });
    }
    if (token < 0) return;
    __syncthreads();
    for (int j = threadIdx.x; j <= a.k; j += kThreads)
        if (list[j].v >= 0) store_entry<E, kTwo>(a, list[j], row, token, m, end);
}

// ---- in passes ------------------------------------------------------------------------------------------------
// grid: the teacher's rows, one wavefront each, a.together in a block; then rows * splits.
template <class E, bool kTwo>
__global__ __launch_bounds__(kT) void distill_stats_kernel(const DistillArgs a, const int64_t teachers) {
    extern __shared__ int words[];
    __shared__ Stat2<Sum<E>> at[kT / 64];
    if (blockIdx.x < teachers) {
        const int wave = threadIdx.x >> 6;
        const int64_t row = static_cast<int64_t>(blockIdx.x) * a.together + wave;
        if (wave >= a.together || row >= a.rows) return;
        const int64_t token = a.tokens[row];
        if (token < 0) return;                           // nothing of the row is read
        float best;
        const double first = teacher_row<E>(a, row, token, words + wave * teacher_words(static_cast<int>(a.k)), a.entries + row * (a.k + 1), best);
        if ((threadIdx.x & 63) == 0) {
            a.first[row] = first;
            a.best[row] = best;
        }
        return;
    }
    const int64_t id = blockIdx.x - teachers, row = id / a.splits;
    const int part = static_cast<int>(id % a.splits);
    if (a.tokens[row] < 0) return;
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    const Cut<E> cut(static_cast<const typename E::Raw*>(a.dz) + row * a.vocab, static_cast<int>(a.vocab));    // as the gradient's pass
    const int each = (cut.vectors + a.splits - 1) / a.splits, v0 = part * each, v1 = v0 + each < cut.vectors ? v0 + each : cut.vectors;
    float most = -INFINITY;
    double sum = 0.0, sum1 = 0.0;                        // 32 terms at a time in 32 bits, their sums in 64
    for (int v = v0 + static_cast<int>(threadIdx.x); v < v1; v += kT * kUnroll) {
        v4u x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            x[u] = v4u{kNothing<E>, kNothing<E>, kNothing<E>, kNothing<E>};
            if (v + u * kT < v1) x[u] = load_vector<E, true>(z, cut.at(v + u * kT));
        }
        float f[kUnroll][E::kN], top = -INFINITY;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            E::unpack(x[u], f[u]);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) top = fmaxf(top, f[u][i]);
        }
        const float m = fmaxf(most, top), base = base_of(m);
        Sum<E> part[kUnroll], part1[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            part[u] = part1[u] = 0;
#pragma unroll
            for (int i = 0; i < E::kN; ++i) {
                part[u] += warm_in_sum<E>(f[u][i] - base, a.heat);
                if (kTwo) part1[u] += exp_in_sum<true>(f[u][i] - base);
            }
        }
        static_assert(kUnroll == 4, "");
        sum = sum * static_cast<double>(warm<true>(most - base, a.heat)) + static_cast<double>((part[0] + part[1]) + (part[2] + part[3]));
        if (kTwo) sum1 = sum1 * static_cast<double>(exp_in_sum<true>(most - base)) + static_cast<double>((part1[0] + part1[1]) + (part1[2] + part1[3]));
        most = m;
    }
    Stat2<Sum<E>> st{most, static_cast<Sum<E>>(sum), static_cast<Sum<E>>(sum1)};
    if (part == 0 && cut.single() >= 0) st = joined2<kTwo>(st, of_one2<Sum<E>>(E::get(z + cut.single()), a.heat), a.heat);
    st = block_joined2<kTwo, kT / 64>(st, a.heat, at);
    if (threadIdx.x == 0) static_cast<Stat2<Sum<E>>*>(a.parts)[row * a.splits + part] = st;
}

// A row's parts joined, by every wavefront for itself, and what follows from them.
template <class E, bool kTwo>
__device__ __forceinline__ RowEnd joined_row(const DistillArgs& a, int64_t row, int64_t token, float share, bool writes, float& m, double& term) {
    Stat2<Sum<E>> st{-INFINITY, 0, 0};
    for (int q = threadIdx.x & 63; q < a.splits; q += 64) st = joined2<kTwo>(st, static_cast<const Stat2<Sum<E>>*>(a.parts)[row * a.splits + q], a.heat);
    st = lanes_joined2<kTwo, 64>(st, a.heat);
    m = st.m;
    const float at = token < a.vocab ? E::get(static_cast<const typename E::Raw*>(a.z) + row * a.ld + token) : NAN;
    return end_of_row<kTwo>(a, row, a.first[row], a.best[row], at, st, share, writes, term);
}

constexpr int64_t kLossHere = 8;        // rows whose loss terms one more block of the gradient's pass adds up: a launch less, but a quarter of a microsecond a row

// grid: rows * blocks, and the block for the loss.  The last rows first: they are the ones that the pass before has left in the last-level cache.
template <class E, bool kTwo>
__global__ __launch_bounds__(kT) void distill_gradient_kernel(const DistillArgs a) {
    __shared__ float counts[kT / 64];
    __shared__ double terms[kT / 64];
    const float counted = a.rows <= kCountHere ? fmaxf(counted_rows<kT / 64>(a.tokens, a.rows, counts), 1.0f) : 0.0f;
    const float share = a.rows <= kCountHere ? 1.0f / counted : *a.share;
    const int64_t row = a.rows - 1 - blockIdx.x / a.blocks;
    float m = 0.0f;
    double term = 0.0;
    if (row < 0) {                                       // the block for the loss
        double sum = 0.0;
        for (int64_t i = threadIdx.x >> 6; i < a.rows; i += kT / 64)
            if (a.tokens[i] >= 0) {
                joined_row<E, kTwo>(a, i, a.tokens[i], share, false, m, term);
                sum += term;
            }
        if ((threadIdx.x & 63) == 0) terms[threadIdx.x >> 6] = sum;
        __syncthreads();
        if (threadIdx.x == 0) *a.loss = static_cast<float>((((terms[0] + terms[1]) + terms[2]) + terms[3]) / static_cast<double>(counted));
        static_assert(kT / 64 == 4, "");
        return;
    }
    const int part = static_cast<int>(blockIdx.x % a.blocks);
    const int64_t token = a.tokens[row];
    const bool writes = part == 0 && threadIdx.x == 0;
    RowEnd e{};
    if (token >= 0) e = joined_row<E, kTwo>(a, row, token, share, writes, m, term);
    else if (writes) empty_row(a, row);
    const typename E::Raw* z = static_cast<const typename E::Raw*>(a.z) + row * a.ld;
    typename E::Raw* dz = static_cast<typename E::Raw*>(a.dz) + row * a.vocab;
    const Cut<E> cut(dz, static_cast<int>(a.vocab));
    const bool zero = e.cs == 0.0f && e.ch == 0.0f;
    const int v0 = part * (kT * kUnroll) + static_cast<int>(threadIdx.x);
    const int single = part == 0 ? cut.single() : -1;
    if (single >= 0) E::put(dz + single, zero ? 0.0f : slope_at<E, kTwo>(E::get(z + single), m, e, a.heat));
    v4u x[kUnroll];
    float d[E::kN];
    if (zero) {                         // nothing to read
#pragma unroll
        for (int i = 0; i < E::kN; ++i) d[i] = 0.0f;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (v0 + u * kT < cut.vectors) store_vector<E>(dz, cut.at(v0 + u * kT), d);
    } else {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (v0 + u * kT < cut.vectors) x[u] = load_vector<E, true>(z, cut.at(v0 + u * kT));
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (v0 + u * kT < cut.vectors) {
                slopes_of<E, kTwo>(x[u], m, e, a.heat, d);
                store_vector<E>(dz, cut.at(v0 + u * kT), d);
            }
    }
    if (token < 0) return;
    __syncthreads();
    const Entry* list = a.entries + row * (a.k + 1);
    for (int j = threadIdx.x; j <= a.k; j += kT) {       // those of this part
        const Entry n = list[j];
        if (n.v < 0) continue;
        const int v = cut.vector_of(n.v);
        if ((v < 0 ? 0 : v / (kT * kUnroll)) == part) store_entry<E, kTwo>(a, n, row, token, m, e);
    }
}

// ---- host -----------------------------------------------------------------------------------------------------
int split_of(int64_t rows, int64_t vectors) {
    const int64_t most = kSplitBlocks / std::max<int64_t>(rows, 1);
    return static_cast<int>(std::max<int64_t>(1, std::min(most, vectors / (2 * kT))));
}

struct Workspace {
    Entry* entries;
    double *first, *term;
    void* parts;
    float *share, *best;
    int64_t bytes;
};
Workspace laid_out(void* at, int64_t rows, int64_t k) {
    char* p = static_cast<char*>(at);
    Workspace w{};
    auto take = [&](int64_t bytes) {
        char* q = p + w.bytes;
        w.bytes += up16(bytes);
        return q;
    };
    w.entries = reinterpret_cast<Entry*>(take(rows * (k + 1) * sizeof(Entry)));
    w.first = reinterpret_cast<double*>(take(rows * sizeof(double)));
    w.term = reinterpret_cast<double*>(take(rows * sizeof(double)));
    w.parts = take(std::max(rows, kSplitBlocks) * sizeof(Stat2<double>));    // rows * split_of(rows, .) at most
    w.share = reinterpret_cast<float*>(take(sizeof(float)));
    w.best = reinterpret_cast<float*>(take(rows * sizeof(float)));
    return w;
}

// Whether the loss is there as well.
template <class E, bool kTwo>
bool launch_rows(DistillArgs a, hipStream_t s) {
    const int64_t rows = a.rows, vectors = a.vocab / E::kN;
    const dim3 grid(static_cast<uint32_t>(rows));
    // Microseconds held and in passes, bf16, 64 entries:  1 row of 8192 9.9 and 9.5, 16 384 11.8 and 9.7, 65 536 15 and 10, 131 072 20 and 10;  8 rows of 8192
    // 10.3 and 10.8, 16 384 12.2 and 10.8;  16 rows (the loss is a launch more) of 32 768 12.8 and 13.0, 65 536 16.8 and 13.0;  64 rows of 65 536 17.5 and
    // 14.3, 131 072 24 and 16;  96 rows 17.8 and 16.2, 24.2 and 22.5;  128 rows 17.8 and 16.0, 24.1 and 25.8;  256 rows 20 and 26, 34 and 42.
    const bool few = rows <= 8 ? vectors >= 2048 : rows <= 96 && vectors >= 8192;
    const bool apart = vectors < 2 || vectors > 16384 || few;
    const int bytes = teacher_words(static_cast<int>(a.k)) * static_cast<int>(sizeof(int)), held = bytes + static_cast<int>((a.k + 1) * sizeof(Entry));
    if (apart) {                         // perhaps none behind the first 16-byte address, or more than a block's registers hold, or few rows
        a.together = 4;
        while (a.together > 1 && a.together * bytes > 16 * 1024) a.together /= 2;      // of LDS, which all blocks of the pass get
        const int64_t teachers = (rows + a.together - 1) / a.together;
        a.splits = split_of(rows, vectors);
        a.blocks = std::max<int64_t>(1, (vectors + kT * kUnroll - 1) / (kT * kUnroll));
        const bool loss = rows <= kLossHere;
        hipLaunchKernelGGL((distill_stats_kernel<E, kTwo>), dim3(static_cast<uint32_t>(teachers + rows * a.splits)), dim3(kT), a.together * bytes, s, a, teachers);
        hipLaunchKernelGGL((distill_gradient_kernel<E, kTwo>), dim3(static_cast<uint32_t>(rows * a.blocks + (loss ? 1 : 0))), dim3(kT), 0, s, a);
        return loss;
    } else if (vectors <= 256) hipLaunchKernelGGL((distill_rows_kernel<E, kTwo, 1, 4, 4>), grid, dim3(64), held, s, a);
    else if (vectors <= 1024) hipLaunchKernelGGL((distill_rows_kernel<E, kTwo, 4, 4, 8>), grid, dim3(256), held, s, a);
    else if (vectors <= 4096) hipLaunchKernelGGL((distill_rows_kernel<E, kTwo, 8, 8, 8>), grid, dim3(512), held, s, a);
    else if (vectors <= 8192) hipLaunchKernelGGL((distill_rows_kernel<E, kTwo, 16, 8, 8>), grid, dim3(1024), held, s, a);
    else hipLaunchKernelGGL((distill_rows_kernel<E, kTwo, 16, 16, 4>), grid, dim3(1024), held, s, a);
    return false;
}
template <class E>
bool launch_of(const DistillArgs& a, hipStream_t s) { return a.hard > 0.0 && a.T != 1.0 ? launch_rows<E, true>(a, s) : launch_rows<E, false>(a, s); }

}  // namespace

int64_t distill_workspace_bytes(int64_t rows, int64_t k) { return laid_out(nullptr, rows, k).bytes; }

hipError_t launch_distill(const LossRows& r, const TeacherRows& t, double temperature, double hard_weight, double loss_scale, float* loss, void* dz, float* kl,
                          float* logp, void* ws, hipStream_t s) {
    const Workspace w = laid_out(ws, r.rows, t.k);
    DistillArgs a{};
    a.z = r.z; a.tokens = r.tokens; a.rows = r.rows; a.vocab = r.vocab; a.ld = r.ld;
    a.t = t.z; a.t_type = t.type; a.t_tokens = t.tokens; a.k = t.k; a.ld_t = t.ld; a.ld_tokens = t.ld_tokens;
    a.T = temperature; a.inv_T = 1.0 / temperature; a.soft = 1.0 - hard_weight; a.hard = hard_weight;
    a.cs = static_cast<float>((1.0 - hard_weight) * temperature * loss_scale);
    a.ch = static_cast<float>(hard_weight * loss_scale);
    const double heat = 1.4426950408889634 / temperature;
    a.heat.near = a.heat.hi = static_cast<float>(heat);
    if (static_cast<double>(a.heat.hi) >= heat) a.heat.hi = std::nextafterf(a.heat.hi, 0.0f);
    a.heat.lo = static_cast<float>(heat - static_cast<double>(a.heat.hi));
    a.share = w.share;
    a.entries = w.entries; a.first = w.first; a.best = w.best; a.term = w.term; a.parts = w.parts;
    a.dz = dz; a.kl = kl; a.logp = logp; a.loss = loss;
    if (r.rows > kCountHere) hipLaunchKernelGGL(count_rows_kernel, dim3(1), dim3(1024), 0, s, r.tokens, r.rows, w.share);
    const bool done = r.rows > 0 && (r.type == ADPSGD_TYPE_F32 ? launch_of<F32>(a, s) : r.type == ADPSGD_TYPE_BF16 ? launch_of<Bf16>(a, s) : launch_of<F16>(a, s));
    if (!done) hipLaunchKernelGGL(mean_terms_kernel, dim3(1), dim3(1024), 0, s, w.term, r.tokens, r.rows, loss);
    return hipGetLastError();
}

}  // namespace adpsgd_impl
