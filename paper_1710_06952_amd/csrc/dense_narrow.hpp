// Products with few rows, D[i][j] = sum_k A(i, k) B(j, k), I <= 64 (few_rows in kernels_dense.hip): B is read once and its bytes are the time.
//
// A block owns up to 64 columns and all rows; its eight wavefronts take steps of k in turn and their sums are joined through LDS, so a call is
// one launch, unless columns are few and k is long: then several blocks share the steps, and dense_join_kernel adds their sums.  Matrix operands come from memory straight into registers, no LDS in between: B is used once.
//   k inner  a lane reads 16 neighbouring k of a row in two loads; four lanes together 128 bytes, a line.  Which 8 of 32 k a lane holds is
//            of no account as long as A's lanes hold the same.
//   k outer  a lane reads kV neighbouring j at 8 k (16 lanes 128 or 64 bytes of a k) and exchanges halves of registers, 4 v_perm_b32 a
//            j: then it holds 8 k of kV rows j, which are matrix operands of rows (l % 16) kV + f.
// Either way a lane ends with neighbouring j of one i (dense_tiles.hpp).
//
// 1 x 4096 x 8192 in bf16: 13 to 15.6 us, 4.3 to 5.2 TB/s of weights (9.3 at the rate of a long read): two blocks on a compute unit with eight
// steps a wavefront, of which launch, first loads and the join are 5 us.  64 x 784 x 1024 6.5 to 7 us in a graph of such calls (tiles of 64: 9 to 10),
// 8.5 to 10 between other kernels.
#pragma once

#include "dense_tiles.hpp"

namespace adpsgd_impl {
namespace {

constexpr int kNarrowWaves = 8;

// kV elements from `start` on of a row that ends at `end`, zero beyond.
template <int kV>
__device__ __forceinline__ v2u load_some(const uint16_t* row, int64_t start, int64_t end, bool cut) {
    static_assert(kV == 2 || kV == 4, "");
    uint64_t x = 0;
    if (!cut) {
        __builtin_memcpy(&x, row + start, 2 * kV);
    } else if (end < kV) {
#pragma unroll
        for (int i = 0; i < kV; ++i)
            if (start + i < end) x |= static_cast<uint64_t>(row[start + i]) << (16 * i);
    } else {
        const int64_t at = start < end - kV ? start : end - kV, by = start - at;
        __builtin_memcpy(&x, row + at, 2 * kV);
        x = by >= kV ? 0 : x >> (16 * by);
    }
    return v2u{static_cast<uint32_t>(x), static_cast<uint32_t>(x >> 32)};
}

// kTI: tiles of 16 rows; kV: columns of a lane's operands, 16 kV of a block
template <class T, bool kBOuter, int kTI, int kV>
__global__ __launch_bounds__(kNarrowWaves * 64) void dense_narrow_kernel(const DenseGemm g, const int splits) {
    constexpr int kColumns = 16 * kV, kStep = kBOuter ? 32 : 64, kPitch = kColumns + 4;
    __shared__ __attribute__((aligned(16))) float sums[kNarrowWaves][16 * kTI][kPitch];
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 15, q = threadIdx.x >> 4 & 3;
    int64_t none, tile, split;
    place_of(blockIdx.x, gridDim.x, 1, gridDim.x / splits, none, tile, split);        // neighbouring columns on one XCD: they share lines where k is outer
    const int64_t j0 = tile * kColumns;
    const uint16_t* a[kTI];
#pragma unroll
    for (int m = 0; m < kTI; ++m) {
        const int64_t i = 16 * m + l;
        a[m] = static_cast<const uint16_t*>(g.a) + (i < g.I ? i : g.I - 1) * g.lda;
    }
    v4f acc[kTI][kV];
#pragma unroll
    for (int m = 0; m < kTI; ++m)
#pragma unroll
        for (int n = 0; n < kV; ++n) acc[m][n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // this wavefront's steps: kTogether at a time, then one by one, and the end of k where it is not a whole step
    constexpr int kTogether = kTI == 1 && !kBOuter ? 4 : 2;
    const int64_t whole = g.K / kStep, until = whole * (split + 1) / splits;
    auto walk = [&](auto go) {
        int64_t s = whole * split / splits + wave;
        for (; s + (kTogether - 1) * kNarrowWaves < until; s += kTogether * kNarrowWaves) go(s, std::integral_constant<int, kTogether>(), std::false_type());
#pragma unroll 1
        for (; s < until; s += kNarrowWaves) go(s, std::integral_constant<int, 1>(), std::false_type());
        if (whole * kStep < g.K && split + 1 == splits && wave == 0) go(whole, std::integral_constant<int, 1>(), std::true_type());
    };

    if constexpr (!kBOuter) {
        const uint16_t* b[kV];
#pragma unroll
        for (int n = 0; n < kV; ++n) {
            const int64_t j = j0 + (l >> 2) * (4 * kV) + 4 * n + (l & 3);
            b[n] = static_cast<const uint16_t*>(g.b) + (j < g.J ? j : g.J - 1) * g.ldb;
        }
        // `some` steps at once, all their loads in front of the products
        auto go = [&](int64_t s, auto some, auto last) {
            constexpr int kSome = decltype(some)::value;
            constexpr bool kLast = decltype(last)::value;
            v4u fb[kSome][2][kV], fa[kSome][2][kTI];
#pragma unroll
            for (int u = 0; u < kSome; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t k = (s + u * kNarrowWaves) * kStep + 16 * q + 8 * h;
#pragma unroll
                    for (int n = 0; n < kV; ++n) fb[u][h][n] = kLast ? load_cut(b[n], k, g.K) : *reinterpret_cast<const v4u_any*>(b[n] + k);
#pragma unroll
                    for (int m = 0; m < kTI; ++m) fa[u][h][m] = kLast ? load_cut(a[m], k, g.K) : *reinterpret_cast<const v4u_any*>(a[m] + k);
                }
#pragma unroll
            for (int u = 0; u < kSome; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int m = 0; m < kTI; ++m)
#pragma unroll
                        for (int n = 0; n < kV; ++n) acc[m][n] = T::mfma(fb[u][h][n], fa[u][h][m], acc[m][n]);
        };
        walk(go);
    } else {
        const int64_t j = j0 + l * kV;
        const bool cut = j + kV > g.J;
        auto go = [&](int64_t s, auto some, auto last) {
            constexpr int kSome = decltype(some)::value;
            constexpr bool kLast = decltype(last)::value;
            v2u r[kSome][8];
            v4u fa[kSome][kTI];
#pragma unroll
            for (int u = 0; u < kSome; ++u) {
                const int64_t k = (s + u * kNarrowWaves) * kStep + 8 * q;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t at = kLast && k + e >= g.K ? g.K - 1 : k + e;
                    r[u][e] = load_some<kV>(static_cast<const uint16_t*>(g.b) + at * g.ldb, j, g.J, cut);
                    if (kLast && k + e >= g.K) r[u][e] = v2u{0, 0};
                }
#pragma unroll
                for (int m = 0; m < kTI; ++m) fa[u][m] = kLast ? load_cut(a[m], k, g.K) : *reinterpret_cast<const v4u_any*>(a[m] + k);
            }
#pragma unroll
            for (int u = 0; u < kSome; ++u)
#pragma unroll
                for (int n = 0; n < kV; ++n) {
                    v4u fb;                              // element n of rows k .. k + 7
#pragma unroll
                    for (int e = 0; e < 4; ++e) fb[e] = __builtin_amdgcn_perm(r[u][2 * e + 1][n / 2], r[u][2 * e][n / 2], n % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                    for (int m = 0; m < kTI; ++m) acc[m][n] = T::mfma(fb, fa[u][m], acc[m][n]);
                }
        };
        walk(go);
    }
    // neighbouring j of a lane: 4 n + v with k inner, v kV + n with k outer
#pragma unroll
    for (int m = 0; m < kTI; ++m)
#pragma unroll
        for (int n = 0; n < kV; ++n) {
            v4f x;
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = kBOuter ? acc[m][(4 * n + v) % kV][(4 * n + v) / kV] : acc[m][n][v];
            *reinterpret_cast<v4f*>(&sums[wave][16 * m + l][4 * kV * q + 4 * n]) = x;
        }
    __syncthreads();
    constexpr int kEights = kColumns / 8;                // kV 1: two of them
    for (int id = threadIdx.x; id < 16 * kTI * kEights; id += kNarrowWaves * 64) {
        const int i = id / kEights, c = id % kEights * 8;
        if (i >= g.I || j0 + c >= g.J) continue;
        const Ending<T, false> end(g, j0 + c);
        const v4u r = end.residual(i);
        float f[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) f[v] = sums[0][i][c + v];
#pragma unroll
        for (int w = 1; w < kNarrowWaves; ++w)
#pragma unroll
            for (int v = 0; v < 8; ++v) f[v] += sums[w][i][c + v];
        if (splits > 1) store_part(g, split, i, j0 + c, f);
        else end.finish(i, f, r);
    }
}

template <class T, bool kBOuter, int kTI, int kV>
void launch_narrow_of(const DenseGemm& g, int splits, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>((g.J + 16 * kV - 1) / (16 * kV) * splits));
    hipLaunchKernelGGL((dense_narrow_kernel<T, kBOuter, kTI, kV>), grid, dim3(kNarrowWaves * 64), 0, s, g, splits);
}
template <class T>
void launch_narrow(const DenseGemm& g, int splits, hipStream_t s) {
    if (g.b_outer) {
        if (narrow_columns(g.I, g.J) == 64) launch_narrow_of<T, true, 1, 4>(g, splits, s);
        else if (g.I <= 16) launch_narrow_of<T, true, 1, 2>(g, splits, s);
        else launch_narrow_of<T, true, 4, 2>(g, splits, s);
    } else {                                             // every block reads all of A: more columns where that is not little
        if (g.I <= 16) launch_narrow_of<T, false, 1, 1>(g, splits, s);
        else launch_narrow_of<T, false, 4, 2>(g, splits, s);
    }
}

}  // namespace
}  // namespace adpsgd_impl
