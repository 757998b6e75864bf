// Gated projections with few rows, I <= 64: the products of dense_narrow.hpp with gates and their partners side by side.  The weights are read once and
// their bytes are the time.
//
// A block owns 16 kV gates and their partners for all rows; a lane holds the matrix operands of both kinds, so both sums end in the same block, and the
// activation and the product are in its end.
#pragma once

#include "dense_narrow.hpp"

namespace adpsgd_impl {
namespace {

// kTI: tiles of 16 rows; kV: gates of a lane's operands, 16 kV of a block; kCorner: relu with slopes (its end in the other calls' code as well: 27.4 us
// for 26.5 of 1 x 4096 x (2 x 8192))
template <class T, bool kBOuter, int kTI, int kV, bool kCorner>
__global__ __launch_bounds__(kNarrowWaves * 64, kTI == 1 && !kBOuter ? 4 : 2) void gated_narrow_kernel(const DenseGemm g, const int splits) {
    constexpr int kColumns = 16 * kV, kStep = kBOuter ? 32 : 64, kPitch = 2 * kColumns + 4;
    static_assert(kBOuter || kV == 1, "");
    extern __shared__ __attribute__((aligned(16))) float sums[];         // [wave][16 kTI][kPitch]: gates, partners
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 15, q = threadIdx.x >> 4 & 3;
    int64_t none, tile, split;
    if (kBOuter) {
        place_of(blockIdx.x, gridDim.x, 1, gridDim.x / splits, none, tile, split);      // neighbouring columns on one XCD: they share lines
    } else {                                             // rows of their own; in their order over the XCDs 25.8 us for 27.3
        tile = blockIdx.x / splits;
        split = blockIdx.x % splits;
    }
    const int64_t j0 = tile * kColumns;
    const uint16_t* a[kTI];
#pragma unroll
    for (int m = 0; m < kTI; ++m) {
        const int64_t i = 16 * m + l;
        a[m] = static_cast<const uint16_t*>(g.a) + (i < g.I ? i : g.I - 1) * g.lda;
    }
    v4f acc[2][kTI][kV];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
        for (int m = 0; m < kTI; ++m)
#pragma unroll
            for (int n = 0; n < kV; ++n) acc[kind][m][n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t whole = g.K / kStep, until = whole * (split + 1) / splits;          // this block's steps, wavefronts in turn
    if constexpr (!kBOuter) {
        const int64_t j = j0 + l < g.J ? j0 + l : g.J - 1;
        const uint16_t* b[2] = {static_cast<const uint16_t*>(g.b) + j * g.ldb, static_cast<const uint16_t*>(g.b) + j * g.ldb + g.b_up};
        // kDeep steps are on their way while one is multiplied, so that the loads of a wavefront never run dry.  1 x 4096 x (2 x 8192): three steps
        // 25.8 us, two 27, four (of which registers spill) 32; two steps that are waited for together 31.
        constexpr int kDeep = kTI == 1 ? 3 : 2;
        v4u fb[kDeep][2][2], fa[kDeep][2][kTI];
        auto load = [&](int64_t s, auto place, auto last) {
            constexpr int u = decltype(place)::value;
            constexpr bool kLast = decltype(last)::value;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t k = s * kStep + 16 * q + 8 * h;
#pragma unroll
                for (int kind = 0; kind < 2; ++kind) fb[u][h][kind] = kLast ? load_cut(b[kind], k, g.K) : *reinterpret_cast<const v4u_any*>(b[kind] + k);
#pragma unroll
                for (int m = 0; m < kTI; ++m) fa[u][h][m] = kLast ? load_cut(a[m], k, g.K) : *reinterpret_cast<const v4u_any*>(a[m] + k);
            }
        };
        auto multiply = [&](auto place) {
            constexpr int u = decltype(place)::value;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int m = 0; m < kTI; ++m)
#pragma unroll
                    for (int kind = 0; kind < 2; ++kind) acc[kind][m][0] = T::mfma(fb[u][h][kind], fa[u][h][m], acc[kind][m][0]);
        };
        auto each = [&](const auto& f) {                 // of the kDeep places
            f(std::integral_constant<int, 0>());
            f(std::integral_constant<int, 1>());
            if constexpr (kDeep == 3) f(std::integral_constant<int, 2>());
        };
        const std::false_type inside;
        const int64_t first = whole * split / splits + wave;
        int64_t groups = first < until ? ((until - first + kNarrowWaves - 1) / kNarrowWaves) / kDeep : 0, s = first;
        if (groups > 0) {
            each([&](auto place) { load(s + place * kNarrowWaves, place, inside); });
            for (s += kDeep * kNarrowWaves; groups > 1; --groups, s += kDeep * kNarrowWaves)
                each([&](auto place) {
                    multiply(place);
                    load(s + place * kNarrowWaves, place, inside);
                });
            each([&](auto place) { multiply(place); });
        }
        const std::integral_constant<int, 0> one;
#pragma unroll 1
        for (; s < until; s += kNarrowWaves) {
            load(s, one, inside);
            multiply(one);
        }
        if (whole * kStep < g.K && split + 1 == splits && wave == 0) {
            load(whole, one, std::true_type());
            multiply(one);
        }
    } else {
        constexpr int kTogether = kTI == 1 ? 2 : 1;
        auto walk = [&](auto go) {
            int64_t s = whole * split / splits + wave;
            if (kTogether > 1)
                for (; s + (kTogether - 1) * kNarrowWaves < until; s += kTogether * kNarrowWaves) go(s, std::integral_constant<int, kTogether>(), std::false_type());
#pragma unroll 1
            for (; s < until; s += kNarrowWaves) go(s, std::integral_constant<int, 1>(), std::false_type());
            if (whole * kStep < g.K && split + 1 == splits && wave == 0) go(whole, std::integral_constant<int, 1>(), std::true_type());
        };
        const int64_t j = j0 + l * kV;
        const bool cut = j + kV > g.J;
        auto go = [&](int64_t s, auto some, auto last) {
            constexpr int kSome = decltype(some)::value;
            constexpr bool kLast = decltype(last)::value;
            v2u r[kSome][2][8];
            v4u fa[kSome][kTI];
#pragma unroll
            for (int u = 0; u < kSome; ++u) {
                const int64_t k = (s + u * kNarrowWaves) * kStep + 8 * q;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t at = kLast && k + e >= g.K ? g.K - 1 : k + e;
                    const uint16_t* p = static_cast<const uint16_t*>(g.b) + at * g.ldb;
#pragma unroll
                    for (int kind = 0; kind < 2; ++kind) {
                        r[u][kind][e] = load_some<kV>(p + kind * g.b_up, j, g.J, cut);
                        if (kLast && k + e >= g.K) r[u][kind][e] = v2u{0, 0};
                    }
                }
#pragma unroll
                for (int m = 0; m < kTI; ++m) fa[u][m] = kLast ? load_cut(a[m], k, g.K) : *reinterpret_cast<const v4u_any*>(a[m] + k);
            }
#pragma unroll
            for (int u = 0; u < kSome; ++u)
#pragma unroll
                for (int kind = 0; kind < 2; ++kind)
#pragma unroll
                    for (int n = 0; n < kV; ++n) {
                        v4u fb;                          // element n of rows k .. k + 7
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            fb[e] = __builtin_amdgcn_perm(r[u][kind][2 * e + 1][n / 2], r[u][kind][2 * e][n / 2], n % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                        for (int m = 0; m < kTI; ++m) acc[kind][m][n] = T::mfma(fb, fa[u][m], acc[kind][m][n]);
                    }
        };
        walk(go);
    }
    // a lane's results of a kind: columns 4 kV q + 4 n + v, v kV + n of them with k outer
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
        for (int m = 0; m < kTI; ++m)
#pragma unroll
            for (int n = 0; n < kV; ++n) {
                v4f x;
#pragma unroll
                for (int v = 0; v < 4; ++v) x[v] = kBOuter ? acc[kind][m][(4 * n + v) % kV][(4 * n + v) / kV] : acc[kind][m][n][v];
                *reinterpret_cast<v4f*>(&sums[(wave * 16 * kTI + 16 * m + l) * kPitch + kind * kColumns + 4 * kV * q + 4 * n]) = x;
            }
    __syncthreads();
    constexpr int kEights = kColumns / 8;
    for (int id = threadIdx.x; id < 16 * kTI * kEights; id += kNarrowWaves * 64) {
        const int i = id / kEights, c = id % kEights * 8;
        if (i >= g.I || j0 + c >= g.J) continue;
        const GatedEnding<T, false> end(g, j0 + c, 32);
        float f[2][8] = {};
#pragma unroll
        for (int w = 0; w < kNarrowWaves; ++w)
#pragma unroll
            for (int kind = 0; kind < 2; ++kind)
#pragma unroll
                for (int v = 0; v < 8; ++v) f[kind][v] += sums[(w * 16 * kTI + i) * kPitch + kind * kColumns + c + v];
        if (splits > 1) store_gated_part(g, split, i, j0 + c, f[0], f[1]);
        else
            end.template finish<kCorner>(i, f[0], f[1], [&](const float* gate, float* scale) {
                if constexpr (kCorner) {
                    end.of_parts(kNarrowWaves, [&](int w, int v) { return sums[(w * 16 * kTI + i) * kPitch + c + v]; }, scale);
                    if (end.n == 1) {                    // alone: where one part is all there is, its other rows tell (else all of them are added again: 67 us for 6 of 64 x 64 x 1)
                        float rows[8];
                        end.template of_columns<kEights, 64 / kEights>(gate, rows);
                        scale[0] = scale[0] < INFINITY ? scale[0] : rows[0];
                    }
                }
            });
    }
}

template <class T, bool kBOuter, int kTI, int kV, bool kCorner>
hipError_t launch_gated_narrow_of(const DenseGemm& g, int splits, hipStream_t s) {
    constexpr int kBytes = kNarrowWaves * 16 * kTI * (2 * 16 * kV + 4) * 4;
    const dim3 grid(static_cast<uint32_t>((g.J + 16 * kV - 1) / (16 * kV) * splits));
    auto kernel = gated_narrow_kernel<T, kBOuter, kTI, kV, kCorner>;
    static std::atomic<uint64_t> allowed{0};
    const hipError_t e = allow_lds(allowed, reinterpret_cast<const void*>(kernel), kBytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(kNarrowWaves * 64), kBytes, s, g, splits);
    return hipSuccess;
}
template <class T, bool kCorner>
hipError_t launch_gated_narrow_as(const DenseGemm& g, int splits, hipStream_t s) {
    if (g.b_outer) return g.I <= 16 ? launch_gated_narrow_of<T, true, 1, 2, kCorner>(g, splits, s) : launch_gated_narrow_of<T, true, 4, 2, kCorner>(g, splits, s);
    return g.I <= 16 ? launch_gated_narrow_of<T, false, 1, 1, kCorner>(g, splits, s) : launch_gated_narrow_of<T, false, 4, 1, kCorner>(g, splits, s);
}
template <class T>
hipError_t launch_gated_narrow(const DenseGemm& g, int splits, hipStream_t s) {
    return g.act == ADPSGD_ACT_RELU && g.slope && splits == 1 ? launch_gated_narrow_as<T, true>(g, splits, s) : launch_gated_narrow_as<T, false>(g, splits, s);
}

}  // namespace
}  // namespace adpsgd_impl
