// Gated projections, the first half of a feed-forward block:  g = x Wg^T + bg,  u = x Wu^T + bu,  h = act(g) u.
//
// Both products are one pass over x: a tile holds eight gates, their eight partners, eight gates ... (gated_row in dense_tiles.hpp), so that a gate
// and its partner end in the same lane, and activation and product are the epilogue of the matrix product of dense layers.  Neither g nor u goes to memory; a
// backward pass gets dh/dg = u act'(g) and dh/du = act(g) in 16 or 24 bits each.  Then
//   dz = [dh u act'(g) | dh act(g)],  db = sum over rows of dz      (this file)
//   dx = dz w,  dw = dz^T x                                         the products of dense layers, over 2 N
//
// dz is rounded to 16 bits once for these products, which puts dx and dw sqrt 2 as far from 64 bits as their own rounding: 2.4e-3 for 1.7e-3 in bf16.  Results of
// up to 2^13 elements, and those of up to 2^12 elements of dz, are computed from dz in two parts (its rounding, and the rounding of what that has left): their products
// take little time, and few elements, or those that few roundings go into, are up to 1.6 times as far in the one form, which is 1.0 in the other.
//
// Bound: the matrix cores, with few rows the bytes of the weights.  8192 x 2048 x (2 x 8192) in bf16, one call after the other: 452 us without an activation, 490 with
// silu, and 38 more where slopes are kept (520 to 530);  between the products of the backward pass 570 to 580, where a library product of that size without an end takes 417 by
// itself.  1 x 4096 x (2 x 8192): 26 us.
#include <algorithm>

#include "dense_tiles.hpp"

namespace adpsgd_impl {
namespace {

constexpr int kT = 256;

int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

// Strips of rows of the pass over dh: 1024 blocks of 256 columns, but none of under 32 rows; up to 64 rows are one.
int gated_strips(int64_t M, int64_t N) {
    if (M <= 64) return M > 0 ? 1 : 0;
    const int64_t across = (N + 255) / 256;
    return static_cast<int>(std::max<int64_t>(2, std::min((M + 31) / 32, std::max<int64_t>(1024 / across, 1))));
}

}  // namespace

bool gated_padded(int64_t M, int64_t N, int64_t K) { return 2 * N % 8 != 0 && worth_packing(M, 2 * N, K); }
bool gated_low(int64_t of_result, int64_t of_dz) { return of_result <= 8192 || of_dz <= 4096; }
int64_t gated_sums_bytes(int64_t M, int64_t N) { return gated_strips(M, N) * 2 * N * static_cast<int64_t>(sizeof(double)); }

int64_t gated_partial_bytes(int64_t I, int64_t J, int64_t K) {
    int64_t parts = 0;
    for (bool direct : {false, true}) parts = std::max<int64_t>(parts, plan_of(I, 2 * J, K, false, direct).splits);
    if (I <= 64) parts = std::max<int64_t>(parts, plan_of(I, 2 * J, K, true, false).splits);
    const bool pack = (J % 8 || K % 8) && worth_packing(I, 2 * J, K);
    const int64_t copies = pack ? packed_bytes(I, K) + std::max(packed_bytes(2 * J, K), packed_bytes(K, 2 * up8(J))) : 0;
    return (parts > 1 ? up256(parts * I * 2 * J * static_cast<int64_t>(sizeof(float))) : 0) + copies;
}

// Copies of w and x for the two products of a backward pass in one launch, where launch_dense_gemm would make one in front of each.  Sizes decide, so that
// the products are cut alike.
bool gated_copies(int64_t M, int64_t N, int64_t K, bool w_transposed) {
    if (K % 8 == 0 || (w_transposed && 2 * N % 8 == 0) || M <= 64 || !worth_packing(M, 2 * N, K)) return false;
    const DensePlan of_dw = w_transposed ? plan_of(K, 2 * N, M, false, true) : plan_of(2 * N, K, M, false, true);
    return of_dw.side >= 128 && plan_of(M, K, 2 * N, false, true).side >= 128;
}
int64_t gated_copies_bytes(int64_t M, int64_t N, int64_t K) {
    int64_t bytes = 0;
    if (gated_copies(M, N, K, false)) bytes = packed_bytes(2 * N, K);
    if (gated_copies(M, N, K, true)) bytes = std::max(bytes, packed_bytes(K, 2 * N));
    return bytes > 0 ? bytes + packed_bytes(M, K) : 0;
}
void launch_gated_copies(const void* w, int64_t ldw, bool w_transposed, const void* x, int64_t ldx, int64_t M, int64_t N, int64_t K, void* to, GatedCopies* copies, hipStream_t s) {
    const int64_t rows = w_transposed ? K : 2 * N, inner = w_transposed ? 2 * N : K;
    *copies = GatedCopies{to, up8(inner), static_cast<char*>(to) + packed_bytes(rows, inner), up8(K)};
    const PackJob jobs[2] = {{w, ldw, to, up8(inner), rows, inner}, {x, ldx, static_cast<char*>(to) + packed_bytes(rows, inner), up8(K), M, K}};
    launch_pack(jobs, 2, s);
}

// As launch_dense_gemm, for 2 J columns.
hipError_t launch_gated_gemm(int32_t type, const DenseGemm& given, hipStream_t s) {
    DenseGemm g = given;
    g.b_up = g.b_outer ? g.J : g.J * g.ldb;
    const bool a_whole = whole_pieces(g.a, g.lda, g.K), b_whole = whole_pieces(g.b, g.ldb, g.b_outer ? g.J : g.K);
    const bool pack = !(a_whole && b_whole) && (g.J % 8 || g.K % 8) && worth_packing(g.I, 2 * g.J, g.K);
    const DensePlan p = plan_of(g.I, 2 * g.J, g.K, few_rows(g.I, 2 * g.J, g.K, g.b_outer, b_whole), (a_whole && b_whole) || pack);
    if (p.side >= 128 && pack) {
        char* at = reinterpret_cast<char*>(g.partial) + (p.splits > 1 ? up256(p.splits * g.I * 2 * g.J * static_cast<int64_t>(sizeof(float))) : 0);
        PackJob jobs[kMostPacks];
        int n = 0;
        if (!a_whole) {
            jobs[n++] = PackJob{g.a, g.lda, at, up8(g.K), g.I, g.K};
            g.a = at;
            g.lda = up8(g.K);
            at += packed_bytes(g.I, g.K);
        }
        if (!b_whole && g.b_outer) {                     // gates and partners each in whole pieces
            const int64_t half = up8(g.J);
            for (int kind = 0; kind < 2; ++kind)
                jobs[n++] = PackJob{static_cast<const uint16_t*>(g.b) + kind * g.J, g.ldb, at + kind * 2 * half, 2 * half, g.K, g.J};
            g.b = at;
            g.ldb = 2 * half;
            g.b_up = half;
        } else if (!b_whole) {
            jobs[n++] = PackJob{g.b, g.ldb, at, up8(g.K), 2 * g.J, g.K};
            g.b = at;
            g.ldb = up8(g.K);
            g.b_up = g.J * g.ldb;
        }
        launch_pack(jobs, n, s);
    }
    return type == ADPSGD_TYPE_BF16 ? launch_gated_tiles<Bf16>(g, p, s) : launch_gated_tiles<F16>(g, p, s);
}

namespace {

// The elements skip .. 7 of a vector, to + 8 the end of their row: pieces of four, two and one from behind.
__device__ __forceinline__ void store_end(uint16_t* to, v4u p, int skip) {
    const int n = 8 - skip;
    int at = 8;
    if (n & 4) {
        at = 4;
        __builtin_memcpy(to + 4, reinterpret_cast<const char*>(&p) + 8, 8);
    }
    if (n & 2) {
        at -= 2;
        const uint32_t w = at == 6 ? p.w : p.y;
        __builtin_memcpy(to + at, &w, 4);
    }
    if (n & 1) {
        at -= 1;                         // odd: the upper half of its word
        to[at] = static_cast<uint16_t>((at == 7 ? p.w : at == 5 ? p.z : at == 3 ? p.y : p.x) >> 16);
    }
}

// dz = [dh slope | dh slope'], rounded once, and sums of the unrounded dz over a strip of rows (32 bits for up to 4 rows of a thread, then 64).
// Memory: 2 + 4 + 4 bytes a result (fp16: 2 more); 8192 x 8192 in bf16 109 us, 6.1 TB/s.  kAcross threads of eight columns in a block.  grid: (ceil(N / (8 kAcross)), strips).
template <class T, int kAcross>
__global__ __launch_bounds__(kT) void gated_dz_kernel(const uint16_t* dh, int64_t lddh, const uint16_t* slopes, uint16_t* dz, uint16_t* rest, int64_t lddz, double* sums, uint16_t* db, int64_t M,
                                                     int64_t N) {
    constexpr int kColumns = 8 * kAcross, kRowsAtOnce = kT / kAcross;
    __shared__ double at[kRowsAtOnce][kColumns];
    const int cx = threadIdx.x % kAcross, ry = threadIdx.x / kAcross;
    const int64_t j = static_cast<int64_t>(blockIdx.x) * kColumns + 8 * cx;
    const int64_t m0 = M * blockIdx.y / gridDim.y, m1 = M * (blockIdx.y + 1) / gridDim.y;
    double sum[2][8] = {};
    const GatedSlopes<T> kept(const_cast<uint16_t*>(slopes), M, N);
    // A vector that the end of the row cuts is the last whole one, of which the first `skip` columns are its neighbour's: it stores the others and counts
    // them only.  (A way of its own for it, element by element, doubled the time of its block: 151 us for 2003 x 2731 in fp16, 30 with shifted loads, 20 so.)
    const int skip = N >= 8 && j < N && j + 8 > N ? static_cast<int>(j + 8 - N) : 0;
    const int64_t from_j = j - skip;
    auto rows = [&](auto vectors) {
        constexpr bool kVectors = decltype(vectors)::value;      // else there are less than eight columns in all
        auto load = [&](const uint16_t* p) { return kVectors ? static_cast<v4u>(__builtin_nontemporal_load(reinterpret_cast<const v4u_any*>(p))) : load_cut(p, 0, N); };
        auto load_low = [&](const uint8_t* p) {
            uint64_t x = 0;
            if (kVectors) {
                __builtin_memcpy(&x, p, 8);
            } else {
                for (int i = 0; i < 8; ++i)
                    if (i < N) x |= static_cast<uint64_t>(p[i]) << (8 * i);
            }
            return v2u{static_cast<uint32_t>(x), static_cast<uint32_t>(x >> 32)};
        };
        for (int64_t first = m0 + ry; first < m1; first += 4 * kRowsAtOnce) {
            float part[2][8] = {};
            v4u d[4], w[4][2];
            v2u low[4][2] = {};
#pragma unroll
            for (int u = 0; u < 4; ++u) {                // rows beyond the strip: its last one again, which counts nothing
                const int64_t m = first + u * kRowsAtOnce < m1 ? first + u * kRowsAtOnce : m1 - 1;
                d[u] = load(dh + m * lddh + from_j);
#pragma unroll
                for (int kind = 0; kind < 2; ++kind) {
                    const int64_t from = (2 * m + kind) * N + from_j;
                    w[u][kind] = load(kept.high + from);
                    if (GatedSlopes<T>::kLow) low[u][kind] = load_low(kept.low + from);
                }
            }
            uint32_t words = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int kind = 0; kind < 2; ++kind) words |= GatedSlopes<T>::large_in(w[u][kind]);
            const bool large = !GatedSlopes<T>::kLow && __ballot(words & 0x80008000u) != 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t m = first + u * kRowsAtOnce;
                if (m >= m1) break;
                float dy[8];
                unpack8<T>(d[u], dy);
#pragma unroll
                for (int kind = 0; kind < 2; ++kind) {
                    float f[8];
                    GatedSlopes<T>::slopes(w[u][kind], low[u][kind], large, f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        f[i] *= dy[i];
                        part[kind][i] += f[i];
                    }
                    if (!dz) continue;
                    auto write = [&](uint16_t* to, v4u p) {
                        to += m * lddz + kind * N + from_j;
                        if (!kVectors) {
                            const v8h h = __builtin_bit_cast(v8h, p);
                            for (int i = 0; i < 8; ++i)
                                if (i < N) to[i] = h[i];
                        } else if (skip == 0) {
                            *reinterpret_cast<v4u_any*>(to) = p;
                        } else {
                            store_end(to, p, skip);
                        }
                        if (kind == 1 && j + 8 >= N)
                            for (int64_t i = 2 * N; i < lddz; ++i) to[i - N - from_j] = 0;
                    };
                    const v4u p = pack8<T>(f);
                    write(dz, p);
                    if (rest) {
                        float near[8];
                        unpack8<T>(p, near);
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[i] = fabsf(near[i]) < INFINITY ? f[i] - near[i] : 0.0f;
                        write(rest, pack8<T>(f));
                    }
                }
            }
#pragma unroll
            for (int kind = 0; kind < 2; ++kind)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[kind][i] += static_cast<double>(part[kind][i]);
        }
    };
    if (N < 8) {
        if (j == 0) rows(std::false_type());
    } else if (j < N) {
        rows(std::true_type());
    }
    if (!sums && !db) return;
    for (int kind = 0; kind < 2; ++kind) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= skip) at[ry][8 * cx + i - skip] = sum[kind][i];
        __syncthreads();
        const int64_t column = static_cast<int64_t>(blockIdx.x) * kColumns + threadIdx.x;
        if (static_cast<int>(threadIdx.x) < kColumns && column < N) {
            double s = 0.0;
            for (int r = 0; r < kRowsAtOnce; ++r) s += at[r][threadIdx.x];
            if (db) db[kind * N + column] = T::down(static_cast<float>(s));      // the only strip
            else sums[(2 * blockIdx.y + kind) * N + column] = s;
        }
    }
}

template <class T>
void launch_dz_of(const void* dh, int64_t lddh, const uint16_t* slopes, void* dz, void* low, int64_t lddz, void* db, double* sums, int64_t M, int64_t N, hipStream_t s) {
    const int strips = gated_strips(M, N);
    auto go = [&](auto kernel, int64_t columns) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>((N + columns - 1) / columns), strips), dim3(kT), 0, s, static_cast<const uint16_t*>(dh), lddh, slopes,
                           static_cast<uint16_t*>(dz), static_cast<uint16_t*>(low), lddz, db ? sums : nullptr, strips == 1 ? static_cast<uint16_t*>(db) : nullptr, M, N);
    };
    if (strips == 1) go(gated_dz_kernel<T, 8>, 64);
    else if (strips > 1) go(gated_dz_kernel<T, 32>, 256);
    if (db && strips != 1) launch_dense_db<T>(sums, strips, 2 * N, db, s);
}

}  // namespace

hipError_t launch_gated_dz(int32_t type, const void* dh, int64_t lddh, const uint16_t* slopes, void* dz, void* low, int64_t lddz, void* db, double* sums, int64_t M,
                           int64_t N, hipStream_t s) {
    if (type == ADPSGD_TYPE_BF16) launch_dz_of<Bf16>(dh, lddh, slopes, dz, low, lddz, db, sums, M, N, s);
    else launch_dz_of<F16>(dh, lddh, slopes, dz, low, lddz, db, sums, M, N, s);
    return hipGetLastError();
}

}  // namespace adpsgd_impl
