// Dense layers: how a product is cut, and the pass over dy in front of the backward products.
#include <algorithm>

#include "dense.hpp"

namespace adpsgd_impl {

namespace {

constexpr int kT = 256;
constexpr int kColumns = 256;           // of a block: 32 threads of eight
constexpr int kRowsAtOnce = 8;

// dz = dy slope, rounded once, and sums of the unrounded dz over a strip of rows (32 bits for up to 8 rows of a thread, then 64).
// Memory: 6 bytes an element.  grid: (ceil(N / 256), strips).
template <class T>
__global__ __launch_bounds__(kT) void dense_dz_kernel(const uint16_t* dy, int64_t lddy, const uint16_t* slope, uint16_t* dz, double* sums, int64_t M, int64_t N) {
    __shared__ double at[kRowsAtOnce][kColumns];
    const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
    const int64_t j = static_cast<int64_t>(blockIdx.x) * kColumns + 8 * cx;
    const int64_t m0 = M * blockIdx.y / gridDim.y, m1 = M * (blockIdx.y + 1) / gridDim.y;
    const bool whole = j + 8 <= N;
    double sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t first = m0 + ry; first < m1; first += 4 * kRowsAtOnce) {
        float part[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        v4u d[4], w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t m = first + u * kRowsAtOnce;
            d[u] = w[u] = v4u{0, 0, 0, 0};
            if (m >= m1 || j >= N) continue;
            if (whole) {
                d[u] = *reinterpret_cast<const v4u_any*>(dy + m * lddy + j);
                if (slope) w[u] = *reinterpret_cast<const v4u_any*>(slope + m * N + j);
            } else {
                v8h a = {0, 0, 0, 0, 0, 0, 0, 0}, b = a;
                for (int i = 0; i < 8; ++i)
                    if (j + i < N) {
                        a[i] = dy[m * lddy + j + i];
                        if (slope) b[i] = slope[m * N + j + i];
                    }
                d[u] = __builtin_bit_cast(v4u, a);
                w[u] = __builtin_bit_cast(v4u, b);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t m = first + u * kRowsAtOnce;
            if (m >= m1 || j >= N) continue;
            float f[8];
            unpack8<T>(d[u], f);
            if (slope) {
                const v8h s = __builtin_bit_cast(v8h, w[u]);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= slope_of(s[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) part[i] += f[i];
            if (dz) {
                const v4u p = pack8<T>(f);
                if (whole) {
                    *reinterpret_cast<v4u_any*>(dz + m * N + j) = p;
                } else {
                    const v8h h = __builtin_bit_cast(v8h, p);
                    for (int i = 0; i < 8; ++i)
                        if (j + i < N) dz[m * N + j + i] = h[i];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += static_cast<double>(part[i]);
    }
    if (!sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) at[ry][8 * cx + i] = sum[i];
    __syncthreads();
    const int64_t column = static_cast<int64_t>(blockIdx.x) * kColumns + threadIdx.x;
    if (column < N) {
        double s = 0.0;
        for (int r = 0; r < kRowsAtOnce; ++r) s += at[r][threadIdx.x];
        sums[blockIdx.y * N + column] = s;
    }
}
template <class T>
__global__ __launch_bounds__(kT) void dense_db_kernel(const double* sums, int strips, int64_t N, uint16_t* db) {
    const int64_t j = static_cast<int64_t>(blockIdx.x) * kT + threadIdx.x;
    if (j >= N) return;
    double s = 0.0;
    for (int r = 0; r < strips; ++r) s += sums[r * N + j];
    db[j] = T::down(static_cast<float>(s));
}

// Strips of 256 rows, as many as 64: with N = 8192 four blocks for a compute unit.
int strips_of(int64_t M) { return static_cast<int>(std::min<int64_t>((M + 255) / 256, 64)); }

template <class T>
void launch_dz_of(const void* dy, int64_t lddy, const uint16_t* slope, void* dz, void* db, double* sums, int64_t M, int64_t N, hipStream_t s) {
    const int strips = strips_of(M);
    if (strips > 0)
        hipLaunchKernelGGL(dense_dz_kernel<T>, dim3(static_cast<uint32_t>((N + kColumns - 1) / kColumns), strips), dim3(kT), 0, s,
                           static_cast<const uint16_t*>(dy), lddy, slope, static_cast<uint16_t*>(dz), db ? sums : nullptr, M, N);
    if (db) hipLaunchKernelGGL(dense_db_kernel<T>, dim3(static_cast<uint32_t>((N + kT - 1) / kT)), dim3(kT), 0, s, sums, strips, N, static_cast<uint16_t*>(db));
}

}  // namespace

int64_t dense_sums_bytes(int64_t M, int64_t N) { return strips_of(M) * N * static_cast<int64_t>(sizeof(double)); }

hipError_t launch_dense_dz(int32_t type, const void* dy, int64_t lddy, const uint16_t* slope, void* dz, void* db, double* sums, int64_t M, int64_t N,
                           hipStream_t s) {
    if (type == ADPSGD_TYPE_BF16) launch_dz_of<Bf16>(dy, lddy, slope, dz, db, sums, M, N, s);
    else launch_dz_of<F16>(dy, lddy, slope, dz, db, sums, M, N, s);
    return hipGetLastError();
}

DensePlan dense_plan(int64_t I, int64_t J, int64_t K, bool aligned) {
    auto tiles = [&](int64_t side) { return ((I + side - 1) / side) * ((J + side - 1) / side); };
    if (aligned && tiles(256) >= 128) return DensePlan{256, 1};
    if (tiles(128) >= 128) return DensePlan{128, 1};
    const int64_t steps = (K + 63) / 64, n = tiles(64);
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({512 / std::max<int64_t>(n, 1), steps / 4, 32}));
    return DensePlan{64, static_cast<int>(splits)};
}
int64_t dense_partial_bytes(int64_t I, int64_t J, int64_t K) {
    const DensePlan p = dense_plan(I, J, K, false);       // aligned operands are cut into as many parts or none
    return p.splits > 1 ? p.splits * I * J * static_cast<int64_t>(sizeof(float)) : 0;
}

hipError_t launch_dense_gemm(int32_t type, const DenseGemm& g, hipStream_t s) {
    if (g.I == 0 || g.J == 0) return hipSuccess;
    const DensePlan p = dense_plan(g.I, g.J, g.K, large_fits(g));
    if (type == ADPSGD_TYPE_BF16) launch_dense_tiles<Bf16>(g, p, s);
    else launch_dense_tiles<F16>(g, p, s);
    return hipGetLastError();
}

}  // namespace adpsgd_impl
