// Layer norm over rows of n elements, and its gradients.
//
//   m = mean x,  v = mean (x - m)^2,  r = 1 / sqrt(v + eps),  h = (x - m) r,  y = h w + b
//   g = dy w,  dx = r (g - mean g - h mean(g h)),  dw = sum over rows of dy h,  db = sum over rows of dy
//
// A team of lanes holds a row in registers, so it is read once: 8 to 64 lanes of a wavefront, or a block.  Teams walk over the rows with w and b
// (backward: and their columns' sums for dw and db) in registers, and the next row's loads are on their way while one is computed.
// Rows too long for that are read again for every pass (`long`); sums of columns are then a kernel of their own.
//
// The mean is taken in two parts: m1 = sum x / n as it rounds, then c = x - m1, which is exact where it matters, and m2 = mean c.  The
// variance is mean c^2 - m2^2, and (c - m2) r has the accuracy of 32 bits where the mean is 10^4 standard deviations away too
// (with m1 alone: 10^-3 of them).  The backward pass gets m1, m2 and r.  Two kinds of rows are summed again, with mean (c - m2)^2 for the variance: those whose
// spread is a few roundings of their mean, for which the difference of the squares is another rounding (the largest gradients: 1 / sqrt(eps)), and those whose
// squares or sum overflow 32 bits, which are taken times 2^-90.
//
// Columns' sums are in 32 bits over kChain rows of a team and over the teams of a block, and in 64 over the blocks; their order depends on the sizes alone.
//
// Bound: memory, 2 to 4 bytes an element and tensor: x in, y out;  x and dy in, dx out.  16 384 x 8192 in bf16: 95 us forward (5.7 TB/s), 140 and 5 for the
// join of the columns' sums backward (5.8); the sizes of the teams are at `Shape`.
#include <algorithm>
#include <limits>

#include "elements.hpp"

namespace adpsgd_impl {
namespace {

constexpr float kSmall = 0x1p-90f;      // squares of 2^38 and sums of 2^30 of them are there in 32 bits
constexpr int kChain = 128;

// kN neighbouring parameters (w or b) from element `at` on.
template <class E, class W>
__device__ __forceinline__ void load_params(const void* p, int at, float* f) {
    const typename W::Raw* q = static_cast<const typename W::Raw*>(p) + at;
#pragma unroll
    for (int i = 0; i < E::kN; i += W::kN) W::unpack(*reinterpret_cast<const v4u_any*>(q + i), f + i);
}
template <class E>
__device__ __forceinline__ v4u load_row(const typename E::Raw* row, int at) {
    return __builtin_nontemporal_load(reinterpret_cast<const v4u_any*>(row + at));
}
template <class E>
__device__ __forceinline__ void store_row(typename E::Raw* row, int at, const float* f) {
    __builtin_nontemporal_store(E::pack(f), reinterpret_cast<v4u_any*>(row + at));
}

// Sums of two values over a team, to all of it.  A team of several wavefronts is a block: `at` has 2 turns of its wavefronts' sums, taken
// alternately, so that one barrier a sum is enough.
template <int kLanes>
struct Team {
    static constexpr int kWaves = kLanes / 64;
    float2 (*at)[kWaves ? kWaves : 1];
    int turn = 0;
    __device__ __forceinline__ float2 sum(float a, float b) {
#pragma unroll
        for (int off = (kLanes < 64 ? kLanes : 64) / 2; off > 0; off >>= 1) {
            a += __shfl_xor(a, off, 64);
            b += __shfl_xor(b, off, 64);
        }
        if (kWaves > 1) {
            if ((threadIdx.x & 63) == 0) at[turn][threadIdx.x >> 6] = make_float2(a, b);
            __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                a += at[turn][w].x;
                b += at[turn][w].y;
            }
            turn ^= 1;
        }
        return make_float2(a, b);
    }
};

struct RowStat {
    float m1, m2, r, scale;             // (x scale - m1 - m2) r
};
// each(f, s): s += f(element) over a thread's elements of the row, absent ones passed over
template <class Sums, class Each>
__device__ __forceinline__ RowStat row_stat(Sums& team, float n, float eps, const Each& each) {
    float s = 0.0f, c1 = 0.0f, c2 = 0.0f;
    each([&](float x) { s += x; });
    float m1 = team.sum(s, 0.0f).x / n;
    each([&](float x) {
        const float c = x - m1;
        c1 += c;
        c2 = fmaf(c, c, c2);
    });
    const float2 t = team.sum(c1, c2);
    float m2 = t.x / n;
    const float v = t.y / n - m2 * m2;
    if (v >= m2 * m2 && t.y < INFINITY) return RowStat{m1, m2, __builtin_amdgcn_rsqf(v + eps), 1.0f};
    // Nearly one value, of which the difference is what the sums were rounded by or little more; or squares or a sum that 32 bits do not hold.
    constexpr float kMost = std::numeric_limits<float>::max() * kSmall;
    const float scale = t.y < INFINITY ? 1.0f : kSmall;
    s = c1 = c2 = 0.0f;
    each([&](float x) { s = fmaf(x, scale, s); });
    m1 = team.sum(s, 0.0f).x / n;
    if (scale != 1.0f) m1 = fminf(fmaxf(m1, -kMost), kMost);         // the mean of the largest numbers may round to more than they are
    each([&](float x) { c1 += fmaf(x, scale, -m1); });
    m2 = team.sum(c1, 0.0f).x / n;
    asm volatile("" : "+v"(m1));        // x - m1 computed anew, not kept since the sum
    each([&](float x) {
        const float c = fmaf(x, scale, -m1) - m2;
        c2 = fmaf(c, c, c2);
    });
    const float rest = team.sum(c2, 0.0f).x / n, up = scale == 1.0f ? 1.0f : 1.0f / kSmall;
    if (rest == 0.0f) return RowStat{m1 * up, m2 * up, __builtin_amdgcn_rsqf(eps), 1.0f};        // one value only: eps times 2^-180 would be 0, and r infinite
    return RowStat{m1, m2, rest < INFINITY ? __builtin_amdgcn_rsqf(rest + eps * scale * scale) : NAN, scale};
}
__device__ __forceinline__ float normed(float x, const RowStat& st) { return (fmaf(x, st.scale, -st.m1) - st.m2) * st.r; }

struct NormArgs {
    const void *x, *w, *b;
    int64_t ldx, rows;
    int n;
    float eps;
    void* y;
    float* stats;               // [3][rows]: m1, m2, r; or nullptr
};
__device__ __forceinline__ void keep_stat(const NormArgs& a, int64_t row, const RowStat& st) {
    const float up = 1.0f / st.scale;
    a.stats[row] = st.m1 * up;
    a.stats[a.rows + row] = st.m2 * up;
    a.stats[2 * a.rows + row] = st.r * st.scale;
}

constexpr int block_of(int lanes, int least) { return lanes > least ? lanes : least; }
// Wavefronts of a SIMD that the registers have to leave room for, where row_stat's second way would just take it (a wavefront less: 65 536 x 1024 in
// bf16 57 us for 52).
constexpr int waves_of(int lanes, int held, int elements) { return held == 1 ? 8 : lanes == 256 && held * elements == 8 ? 6 : 1; }

// Vectors v = u kLanes + lane, u < kHeld, and the elements behind the last whole vector one for each of the first lanes.  kKeep: w and b
// stay in registers; blocks of 1024 threads have none left for them and read them for every row, from the caches.
template <class E, class W, int kLanes, int kHeld>
__global__ __launch_bounds__(block_of(kLanes, 256), waves_of(kLanes, kHeld, E::kN)) void norm_kernel(const NormArgs a) {
    constexpr bool kKeep = kLanes < 1024, kLate = kLanes * kHeld == 4096;
    constexpr int kTeams = block_of(kLanes, 256) / kLanes;
    __shared__ float2 at[2][Team<kLanes>::kWaves ? Team<kLanes>::kWaves : 1];
    Team<kLanes> team{at};
    const int lane = threadIdx.x % kLanes, vectors = a.n / E::kN, tail = a.n - vectors * E::kN, last = vectors * E::kN + lane;
    const bool single = lane < tail;
    float w[kHeld][E::kN], b[kHeld][E::kN], w1 = 1.0f, b1 = 0.0f;
    auto params = [&](int u) {
        const int v = u * kLanes + lane;
#pragma unroll
        for (int i = 0; i < E::kN; ++i) {
            w[u][i] = 1.0f;
            b[u][i] = 0.0f;
        }
        if (a.w && v < vectors) load_params<E, W>(a.w, v * E::kN, w[u]);
        if (a.b && v < vectors) load_params<E, W>(a.b, v * E::kN, b[u]);
    };
    if (kKeep) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) params(u);
    }
    if (a.w && single) w1 = W::get(static_cast<const typename W::Raw*>(a.w) + last);
    if (a.b && single) b1 = W::get(static_cast<const typename W::Raw*>(a.b) + last);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kTeams;
    v4u x[kHeld];
    float x1 = 0.0f;
    auto load = [&](int64_t first) {
        if (first >= a.rows) return;                     // uniform over the block, as `first` is
        const int64_t row = first + threadIdx.x / kLanes;
        const typename E::Raw* from = static_cast<const typename E::Raw*>(a.x) + (row < a.rows ? row : a.rows - 1) * a.ldx;
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int v = u * kLanes + lane;
            if (vectors > 0) x[u] = load_row<E>(from, (v < vectors ? v : vectors - 1) * E::kN);
        }
        if (single) x1 = E::get(from + last);
    };
    int64_t first = static_cast<int64_t>(blockIdx.x) * kTeams;
    load(first);
    for (; first < a.rows; first += stride) {
        const int64_t row = first + threadIdx.x / kLanes;
        float f[kHeld][E::kN];
        const float f1 = x1;
#pragma unroll
        for (int u = 0; u < kHeld; ++u) E::unpack(x[u], f[u]);
        if (!kLate) load(first + stride);
        const RowStat st = row_stat(team, static_cast<float>(a.n), a.eps, [&](const auto& add) {
#pragma unroll
            for (int u = 0; u < kHeld; ++u)
                if (u * kLanes + lane < vectors) {
#pragma unroll
                    for (int i = 0; i < E::kN; ++i) add(f[u][i]);
                }
            if (single) add(f1);
        });
        if (kLate) load(first + stride);
        if (row >= a.rows) continue;
        typename E::Raw* y = static_cast<typename E::Raw*>(a.y) + row * a.n;
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int v = u * kLanes + lane;
            float o[E::kN];
            if (!kKeep) params(u);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) o[i] = fmaf(normed(f[u][i], st), w[u][i], b[u][i]);
            if (v < vectors) store_row<E>(y, v * E::kN, o);
        }
        if (single) E::put(y + last, fmaf(normed(f1, st), w1, b1));
        if (a.stats && lane == 0) keep_stat(a, row, st);
    }
}

constexpr int kLongThreads = 1024;

// Rows of any length, read once for each of three passes.  grid: rows, at most.
template <class E, class W>
__global__ __launch_bounds__(kLongThreads) void norm_long_kernel(const NormArgs a) {
    __shared__ float2 at[2][kLongThreads / 64];
    Team<kLongThreads> team{at};
    const int vectors = a.n / E::kN, tail = a.n - vectors * E::kN, last = vectors * E::kN + static_cast<int>(threadIdx.x);
    const bool single = static_cast<int>(threadIdx.x) < tail;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const typename E::Raw* p = static_cast<const typename E::Raw*>(a.x) + row * a.ldx;
        const RowStat st = row_stat(team, static_cast<float>(a.n), a.eps, [&](const auto& add) {
            for (int v = threadIdx.x; v < vectors; v += kLongThreads) {
                float f[E::kN];
                E::unpack(*reinterpret_cast<const v4u_any*>(p + v * E::kN), f);
#pragma unroll
                for (int i = 0; i < E::kN; ++i) add(f[i]);
            }
            if (single) add(E::get(p + last));
        });
        typename E::Raw* y = static_cast<typename E::Raw*>(a.y) + row * a.n;
        for (int v = threadIdx.x; v < vectors; v += kLongThreads) {
            float f[E::kN], w[E::kN], b[E::kN];
            E::unpack(load_row<E>(p, v * E::kN), f);
            if (a.w) load_params<E, W>(a.w, v * E::kN, w);
            if (a.b) load_params<E, W>(a.b, v * E::kN, b);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) f[i] = fmaf(normed(f[i], st), a.w ? w[i] : 1.0f, a.b ? b[i] : 0.0f);
            store_row<E>(y, v * E::kN, f);
        }
        if (single) {
            const float w = a.w ? W::get(static_cast<const typename W::Raw*>(a.w) + last) : 1.0f;
            E::put(y + last, fmaf(normed(E::get(p + last), st), w, a.b ? W::get(static_cast<const typename W::Raw*>(a.b) + last) : 0.0f));
        }
        if (a.stats && threadIdx.x == 0) keep_stat(a, row, st);
    }
}

// ---- gradients -------------------------------------------------------------------------------------------
struct NormGradArgs {
    const void *dy, *x, *w;
    int64_t lddy, ldx, rows;
    int n;
    const float* stats;
    void* dx;                   // or nullptr
    float* sums;                // [parts][2][n] columns' sums of dy h and dy; nullptr: dw and db are written as they are
    void *dw, *db;              // either may be nullptr
};
__device__ __forceinline__ RowStat kept_stat(const NormGradArgs& a, int64_t row) {
    return RowStat{a.stats[row], a.stats[a.rows + row], a.stats[2 * a.rows + row], 1.0f};
}
// Where 1 / r is so large that a value may be further from the mean than the largest number (no further than sqrt n / r, n <= 2^28), the row is taken times
// 1/4.  Not a part of kept_stat: what is loaded is not waited for there.
__device__ __forceinline__ RowStat within_reach(const RowStat& st) {
    const bool far = st.r < 0x1p-100f;
    const float scale = far ? 0.25f : 1.0f;
    return RowStat{st.m1 * scale, st.m2 * scale, far ? 4.0f * st.r : st.r, scale};
}
__device__ __forceinline__ float unscaled(const RowStat& st) { return st.r * st.scale; }

// As norm_kernel; a thread's columns are the same in every row.
template <class E, class W, int kLanes, int kHeld, int kBlock>
__global__ __launch_bounds__(kBlock) void norm_gradient_kernel(const NormGradArgs a) {
    constexpr bool kAgain = kHeld == 4, kKeep = !kAgain;
    constexpr int kTeams = kBlock / kLanes, kWide = kLanes * kHeld * E::kN + E::kN;
    __shared__ float2 at[2][Team<kLanes>::kWaves ? Team<kLanes>::kWaves : 1];
    __shared__ float joined[kTeams > 1 ? 2 : 1][kTeams > 1 ? kWide : 1];
    static_assert(kTeams == 1 || kLanes <= 64, "a team of several wavefronts is a block");
    Team<kLanes> team{at};
    const int lane = threadIdx.x % kLanes, vectors = a.n / E::kN, tail = a.n - vectors * E::kN, last = vectors * E::kN + lane;
    const bool single = lane < tail;
    const float inv = 1.0f / static_cast<float>(a.n);
    float w[kHeld][E::kN], w1 = 1.0f;
    auto params = [&](int u) {
        const int v = u * kLanes + lane;
#pragma unroll
        for (int i = 0; i < E::kN; ++i) w[u][i] = 1.0f;
        if (a.w && v < vectors) load_params<E, W>(a.w, v * E::kN, w[u]);
    };
    if (kKeep) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) params(u);
    }
    if (a.w && single) w1 = W::get(static_cast<const typename W::Raw*>(a.w) + last);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kTeams;
    v4u x[kHeld], d[kHeld];
    float x1 = 0.0f, d1 = 0.0f;
    RowStat next{};
    auto load = [&](int64_t first) {
        if (first >= a.rows) return;                     // uniform over the block, as `first` is
        const int64_t row = first + threadIdx.x / kLanes, from = row < a.rows ? row : a.rows - 1;
        const typename E::Raw* of_x = static_cast<const typename E::Raw*>(a.x) + from * a.ldx;
        const typename E::Raw* of_d = static_cast<const typename E::Raw*>(a.dy) + from * a.lddy;
        next = kept_stat(a, from);
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int v = u * kLanes + lane, e = (v < vectors ? v : vectors - 1) * E::kN;
            if (vectors > 0) {
                x[u] = load_row<E>(of_x, e);
                d[u] = load_row<E>(of_d, e);
            }
        }
        if (single) {
            x1 = E::get(of_x + last);
            d1 = E::get(of_d + last);
        }
    };
    float sw[kHeld][E::kN] = {}, sb[kHeld][E::kN] = {}, sw1 = 0.0f, sb1 = 0.0f;
    int64_t first = static_cast<int64_t>(blockIdx.x) * kTeams;
    load(first);
    for (; first < a.rows; first += stride) {
        const int64_t row = first + threadIdx.x / kLanes;
        const bool there = row < a.rows;
        const RowStat st = within_reach(next);
        float h[kHeld][E::kN], g[kHeld][E::kN], h1 = 0.0f, g1 = 0.0f, p = 0.0f, q = 0.0f;
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const bool mine = there && u * kLanes + lane < vectors;
            if (kAgain) __builtin_amdgcn_sched_barrier(0);           // one vector after the other: unpacked, they would not all fit
            if (!kKeep) params(u);
            E::unpack(x[u], h[u]);
            E::unpack(d[u], g[u]);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) {
                h[u][i] = normed(h[u][i], st);
                const float dy = mine ? g[u][i] : 0.0f, hh = mine ? h[u][i] : 0.0f;
                sw[u][i] = fmaf(dy, hh, sw[u][i]);
                sb[u][i] += dy;
                g[u][i] = dy * w[u][i];
                p += g[u][i];
                q = fmaf(g[u][i], hh, q);
            }
        }
        if (single && there) {
            h1 = normed(x1, st);
            sw1 = fmaf(d1, h1, sw1);
            sb1 += d1;
            g1 = d1 * w1;
            p += g1;
            q = fmaf(g1, h1, q);
        }
        if (!kAgain) load(first + stride);
        const float2 t = team.sum(p, q);
        const float mp = t.x * inv, mq = t.y * inv, r = unscaled(st);
        if (there && a.dx) {
            typename E::Raw* dx = static_cast<typename E::Raw*>(a.dx) + row * a.n;
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                const int v = u * kLanes + lane;
                float o[E::kN];
                if (kAgain) {                            // unpacked and computed anew, not kept since the sum
                    __builtin_amdgcn_sched_barrier(0);
                    asm volatile("" : "+v"(x[u]), "+v"(d[u]));
                    params(u);
                    E::unpack(x[u], h[u]);
                    E::unpack(d[u], g[u]);
#pragma unroll
                    for (int i = 0; i < E::kN; ++i) {
                        h[u][i] = normed(h[u][i], st);
                        g[u][i] *= w[u][i];
                    }
                }
#pragma unroll
                for (int i = 0; i < E::kN; ++i) o[i] = r * (g[u][i] - mp - h[u][i] * mq);
                if (v < vectors) store_row<E>(dx, v * E::kN, o);
            }
            if (single) E::put(dx + last, r * (g1 - mp - h1 * mq));
        }
        if (kAgain) load(first + stride);
    }
    if (!a.dw && !a.db) return;
    auto finish = [&](int e, float s, float c) {
        if (a.sums) {
            float* out = a.sums + static_cast<int64_t>(blockIdx.x) * 2 * a.n;
            out[e] = s;
            out[a.n + e] = c;
        } else {                                         // the only block
            if (a.dw) W::put(static_cast<typename W::Raw*>(a.dw) + e, s);
            if (a.db) W::put(static_cast<typename W::Raw*>(a.db) + e, c);
        }
    };
    auto columns = [&](const auto& f) {                  // a thread's own
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int v = u * kLanes + lane;
            if (v < vectors) {
#pragma unroll
                for (int i = 0; i < E::kN; ++i) f(v * E::kN + i, sw[u][i], sb[u][i]);
            }
        }
        if (single) f(last, sw1, sb1);
    };
    if constexpr (kTeams == 1) {
        columns(finish);
    } else {                                             // one team after the other, in their order
        for (int t = 0; t < kTeams; ++t) {
            if (static_cast<int>(threadIdx.x) / kLanes == t)
                columns([&](int e, float s, float c) {
                    joined[0][e] = t == 0 ? s : joined[0][e] + s;
                    joined[1][e] = t == 0 ? c : joined[1][e] + c;
                });
            __syncthreads();
        }
        for (int e = threadIdx.x; e < a.n; e += kBlock) finish(e, joined[0][e], joined[1][e]);
    }
}

// Rows of any length: sums, then dx.
template <class E, class W>
__global__ __launch_bounds__(kLongThreads) void norm_gradient_long_kernel(const NormGradArgs a) {
    __shared__ float2 at[2][kLongThreads / 64];
    Team<kLongThreads> team{at};
    const int vectors = a.n / E::kN, tail = a.n - vectors * E::kN, last = vectors * E::kN + static_cast<int>(threadIdx.x);
    const bool single = static_cast<int>(threadIdx.x) < tail;
    const float inv = 1.0f / static_cast<float>(a.n);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const typename E::Raw* x = static_cast<const typename E::Raw*>(a.x) + row * a.ldx;
        const typename E::Raw* dy = static_cast<const typename E::Raw*>(a.dy) + row * a.lddy;
        const RowStat st = within_reach(kept_stat(a, row));
        auto both = [&](int v, float* g, float* h) {
            float w[E::kN];
            E::unpack(*reinterpret_cast<const v4u_any*>(x + v * E::kN), h);
            E::unpack(*reinterpret_cast<const v4u_any*>(dy + v * E::kN), g);
            if (a.w) load_params<E, W>(a.w, v * E::kN, w);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) {
                h[i] = normed(h[i], st);
                g[i] = a.w ? g[i] * w[i] : g[i];
            }
        };
        float p = 0.0f, q = 0.0f, h1 = 0.0f, g1 = 0.0f;
        for (int v = threadIdx.x; v < vectors; v += kLongThreads) {
            float g[E::kN], h[E::kN];
            both(v, g, h);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) {
                p += g[i];
                q = fmaf(g[i], h[i], q);
            }
        }
        if (single) {
            h1 = normed(E::get(x + last), st);
            g1 = E::get(dy + last) * (a.w ? W::get(static_cast<const typename W::Raw*>(a.w) + last) : 1.0f);
            p += g1;
            q = fmaf(g1, h1, q);
        }
        const float2 t = team.sum(p, q);
        const float mp = t.x * inv, mq = t.y * inv, r = unscaled(st);
        typename E::Raw* dx = static_cast<typename E::Raw*>(a.dx) + row * a.n;
        for (int v = threadIdx.x; v < vectors; v += kLongThreads) {
            float g[E::kN], h[E::kN];
            both(v, g, h);
#pragma unroll
            for (int i = 0; i < E::kN; ++i) g[i] = r * (g[i] - mp - h[i] * mq);
            store_row<E>(dx, v * E::kN, g);
        }
        if (single) E::put(dx + last, r * (g1 - mp - h1 * mq));
    }
}
// ... and the columns' sums of a strip of rows, a column a thread.  grid: (ceil(n / kColumns), parts), as many strips as fill the chip: with min(rows, 512) of
// them, whatever n is, the sums of 512 x 2^20 in bf16 took 4.3 GB beside 1.07 GB of x, and the backward pass 3880 us for 1710 (2000 x 32 768: 236 us for 148).
constexpr int kColumns = 256;
constexpr int64_t kColumnBlocks = 2048;
template <class E>
__global__ __launch_bounds__(kColumns) void norm_columns_kernel(const NormGradArgs a) {
    const int64_t e = static_cast<int64_t>(blockIdx.x) * kColumns + threadIdx.x;
    if (e >= a.n) return;
    double sw = 0.0, sb = 0.0;
    for (int64_t row = a.rows * blockIdx.y / gridDim.y, end = a.rows * (blockIdx.y + 1) / gridDim.y; row < end; ++row) {
        const float dy = E::get(static_cast<const typename E::Raw*>(a.dy) + row * a.lddy + e);
        sw += static_cast<double>(dy) * normed(E::get(static_cast<const typename E::Raw*>(a.x) + row * a.ldx + e), within_reach(kept_stat(a, row)));
        sb += dy;
    }
    float* out = a.sums + static_cast<int64_t>(blockIdx.y) * 2 * a.n;
    out[e] = static_cast<float>(sw);
    out[a.n + e] = static_cast<float>(sb);
}

// The parts in their order: kJoin threads a column, each every kJoin-th part.  grid: (ceil(n / 64), 2).
constexpr int kJoin = 16;
template <class W>
__global__ __launch_bounds__(64 * kJoin) void norm_join_kernel(const float* sums, int64_t parts, int n, void* dw, void* db) {
    __shared__ double at[kJoin][64];
    const int64_t e = static_cast<int64_t>(blockIdx.x) * 64 + (threadIdx.x & 63);
    const int turn = threadIdx.x >> 6;
    typename W::Raw* out = static_cast<typename W::Raw*>(blockIdx.y ? db : dw);
    if (!out) return;                                    // uniform
    double s = 0.0;
    if (e < n) {
#pragma unroll 4
        for (int64_t p = turn; p < parts; p += kJoin) s += sums[(2 * p + blockIdx.y) * n + e];
    }
    at[turn][threadIdx.x & 63] = s;
    __syncthreads();
    if (turn == 0 && e < n) {
#pragma unroll
        for (int t = 1; t < kJoin; ++t) s += at[t][threadIdx.x];
        W::put(out + e, static_cast<float>(s));
    }
}

// ---- host ------------------------------------------------------------------------------------------------
// The team for rows of so many vectors (lanes, vectors of a lane; lanes 0: `long`), threads of a block, and blocks at most.  Microseconds for 2^27
// elements in bf16 (537 MB forward, 805 backward, 6.1 TB/s at most), forward:
//   1024 vectors  256 lanes of 4 in 2048 blocks 94 (8192 blocks 98, all rows at once 114), 512 of 2 96, 1024 of 1 134
//    512          256 of 2 in 8192 blocks 90 (1024 blocks 93, all 111), 512 of 1 106, 64 of 8 104
//    256          64 of 4 in 8192 blocks 89, 256 of 1 97;    128: 64 of 2 91;    64: 64 of 1 98;    16: 98 to 103
// backward, where every block costs its columns' sums:
//   1024 vectors  1024 lanes of 1 in 256 blocks 139 (512 blocks 147), 512 of 2 152
//    512          512 of 1 in 512 blocks 138, 256 of 2 143;    256: 256 of 1 in 1024 blocks 140 (512: 154);    128: 64 of 2 in 512 blocks 138
//     64          64 of 1, blocks of 512 threads, 512 of them 135 (256 threads, 1024 blocks 139)
// A second row under way: 92 for 94 and 135 for 139 at 1024 vectors, and slower at most others.
struct Shape {
    int lanes, held, block;
    int64_t blocks;
};
Shape forward_shape(int64_t vectors) {
    for (int lanes : {8, 16, 32, 64})
        if (vectors <= lanes) return Shape{lanes, 1, 256, 8192};
    if (vectors <= 128) return Shape{64, 2, 256, 8192};
    if (vectors <= 256) return Shape{64, 4, 256, 8192};
    if (vectors <= 512) return Shape{256, 2, 256, 8192};
    if (vectors <= 1024) return Shape{256, 4, 256, 2048};
    if (vectors <= 2048) return Shape{1024, 2, 1024, 512};
    if (vectors <= 4096) return Shape{1024, 4, 1024, 512};
    return Shape{0, 0, kLongThreads, 512};
}
Shape gradient_shape(int64_t vectors) {
    for (int lanes : {8, 16, 32, 64})
        if (vectors <= lanes) return Shape{lanes, 1, 512, 512};
    if (vectors <= 128) return Shape{64, 2, 256, 512};
    if (vectors <= 256) return Shape{256, 1, 256, 1024};
    if (vectors <= 512) return Shape{512, 1, 512, 512};
    if (vectors <= 1024) return Shape{1024, 1, 1024, 256};
    if (vectors <= 2048) return Shape{512, 4, 512, 256};
    return Shape{0, 0, kLongThreads, 512};
}
int64_t vectors_of(int32_t type, int64_t n) { return n / (type == ADPSGD_TYPE_F32 ? F32::kN : Bf16::kN); }
// Blocks of the gradient's pass, and parts of the columns' sums.  Up to eight rows of a team are left to one block, which writes dw and db itself: a
// launch and a workspace less (128 x 128 in fp32: 5 us of host time, and on the GPU eight turns take no longer than one and the join).
int64_t parts_of(int32_t type, int64_t rows, int64_t n) {
    const Shape s = gradient_shape(vectors_of(type, n));
    if (s.lanes == 0) return std::max<int64_t>(1, std::min(rows, kColumnBlocks / ((n + kColumns - 1) / kColumns)));
    const int64_t teams = s.block / s.lanes, turns = (rows + teams - 1) / teams;
    if (turns <= 8) return 1;
    return std::max<int64_t>(std::min(turns, s.blocks), (turns + kChain - 1) / kChain);
}

template <class E, class W>
void launch_norm_of(const NormArgs& a, hipStream_t s) {
    const Shape shape = forward_shape(a.n / E::kN);
    const int64_t teams = shape.lanes ? shape.block / shape.lanes : 1, blocks = std::min<int64_t>((a.rows + teams - 1) / teams, shape.blocks);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(shape.block), 0, s, a); };
    switch (shape.lanes * 8 + shape.held) {
        case 8 * 8 + 1: return go(norm_kernel<E, W, 8, 1>);
        case 16 * 8 + 1: return go(norm_kernel<E, W, 16, 1>);
        case 32 * 8 + 1: return go(norm_kernel<E, W, 32, 1>);
        case 64 * 8 + 1: return go(norm_kernel<E, W, 64, 1>);
        case 64 * 8 + 2: return go(norm_kernel<E, W, 64, 2>);
        case 64 * 8 + 4: return go(norm_kernel<E, W, 64, 4>);
        case 256 * 8 + 2: return go(norm_kernel<E, W, 256, 2>);
        case 256 * 8 + 4: return go(norm_kernel<E, W, 256, 4>);
        case 1024 * 8 + 2: return go(norm_kernel<E, W, 1024, 2>);
        case 1024 * 8 + 4: return go(norm_kernel<E, W, 1024, 4>);
        default: return go(norm_long_kernel<E, W>);
    }
}

template <class E, class W>
void launch_norm_gradient_of(int32_t type, const NormGradArgs& a, hipStream_t s) {
    const Shape shape = gradient_shape(a.n / E::kN);
    const int64_t parts = parts_of(type, a.rows, a.n);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(parts)), dim3(shape.block), 0, s, a); };
    if (a.rows > 0) switch (shape.lanes * 8 + shape.held) {
        case 8 * 8 + 1: go(norm_gradient_kernel<E, W, 8, 1, 512>); break;
        case 16 * 8 + 1: go(norm_gradient_kernel<E, W, 16, 1, 512>); break;
        case 32 * 8 + 1: go(norm_gradient_kernel<E, W, 32, 1, 512>); break;
        case 64 * 8 + 1: go(norm_gradient_kernel<E, W, 64, 1, 512>); break;
        case 64 * 8 + 2: go(norm_gradient_kernel<E, W, 64, 2, 256>); break;
        case 256 * 8 + 1: go(norm_gradient_kernel<E, W, 256, 1, 256>); break;
        case 512 * 8 + 1: go(norm_gradient_kernel<E, W, 512, 1, 512>); break;
        case 1024 * 8 + 1: go(norm_gradient_kernel<E, W, 1024, 1, 1024>); break;
        case 512 * 8 + 4: go(norm_gradient_kernel<E, W, 512, 4, 512>); break;
        default:
            if (a.dx) hipLaunchKernelGGL((norm_gradient_long_kernel<E, W>), dim3(static_cast<uint32_t>(std::min<int64_t>(a.rows, 512))), dim3(kLongThreads), 0, s, a);
            if (a.sums) hipLaunchKernelGGL(norm_columns_kernel<E>, dim3(static_cast<uint32_t>((a.n + kColumns - 1) / kColumns), static_cast<uint32_t>(parts)), dim3(kColumns), 0, s, a);
    }
    if ((a.dw || a.db) && (a.sums || a.rows == 0))
        hipLaunchKernelGGL(norm_join_kernel<W>, dim3(static_cast<uint32_t>((a.n + 63) / 64), 2), dim3(64 * kJoin), 0, s, a.sums, a.rows > 0 ? parts : 0, a.n, a.dw, a.db);
}

// f(E, W) for the two types
template <class F>
void with_types(int32_t type, int32_t params, const F& f) {
    if (type == ADPSGD_TYPE_F32) f(F32(), F32());
    else if (type == ADPSGD_TYPE_BF16) params == ADPSGD_TYPE_F32 ? f(Bf16(), F32()) : f(Bf16(), Bf16());
    else params == ADPSGD_TYPE_F32 ? f(F16(), F32()) : f(F16(), F16());
}

}  // namespace

int64_t norm_workspace_bytes(int32_t type, int64_t rows, int64_t n) {
    const int64_t parts = rows > 0 ? parts_of(type, rows, n) : 0;
    return parts > 1 || gradient_shape(vectors_of(type, n)).lanes == 0 ? parts * 2 * n * static_cast<int64_t>(sizeof(float)) : 0;
}

hipError_t launch_norm(const NormRows& r, const void* b, double eps, void* y, float* stats, hipStream_t s) {
    NormArgs a{};
    a.x = r.x; a.w = r.w; a.b = b;
    a.ldx = r.ldx; a.rows = r.rows; a.n = static_cast<int>(r.n);
    a.eps = static_cast<float>(eps);
    a.y = y; a.stats = stats;
    with_types(r.type, r.param_type, [&](auto e, auto w) { launch_norm_of<decltype(e), decltype(w)>(a, s); });
    return hipGetLastError();
}

hipError_t launch_norm_gradient(const NormRows& r, const void* dy, int64_t lddy, const float* stats, void* dx, void* dw, void* db, void* ws, hipStream_t s) {
    NormGradArgs a{};
    a.dy = dy; a.x = r.x; a.w = r.w;
    a.lddy = lddy; a.ldx = r.ldx; a.rows = r.rows; a.n = static_cast<int>(r.n);
    a.stats = stats;
    a.dx = dx;
    a.dw = dw; a.db = db;
    a.sums = (dw || db) && norm_workspace_bytes(r.type, r.rows, r.n) > 0 ? static_cast<float*>(ws) : nullptr;
    with_types(r.type, r.param_type, [&](auto e, auto w) { launch_norm_gradient_of<decltype(e), decltype(w)>(r.type, a, s); });
    return hipGetLastError();
}

}  // namespace adpsgd_impl
