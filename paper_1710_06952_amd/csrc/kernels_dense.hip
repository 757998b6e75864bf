// Dense layers: how a product is cut, and the pass over dy in front of the backward products.
#include <algorithm>

#include "dense.hpp"

namespace adpsgd_impl {

namespace {

constexpr int kT = 256;

// dz = dy slope, rounded once, and sums of the unrounded dz over a strip of rows (32 bits for up to 4 rows of a thread, then 64).  dz has 16 bits as
// the matrix instructions take them: dx and dw are sqrt 2 as far from 64 bits as their own rounding (2.35e-3 for 1.66e-3 in bf16); dz in two parts
// of 16 bits would make each of their products two, 215 us more at 8192 x 2048 x 8192.
// Memory: 6 bytes an element.  kAcross threads of eight columns in a block: 32, or 8 where there is one strip only (64 x 1024: a quarter of
// the rows for a thread and four times the blocks).  grid: (ceil(N / (8 kAcross)), strips).
template <class T, int kAcross>
__global__ __launch_bounds__(kT) void dense_dz_kernel(const uint16_t* dy, int64_t lddy, const uint16_t* slope, uint16_t* dz, double* sums, uint16_t* db, int64_t M,
                                                     int64_t N) {
    constexpr int kColumns = 8 * kAcross, kRowsAtOnce = kT / kAcross;
    __shared__ double at[kRowsAtOnce][kColumns];
    const int cx = threadIdx.x % kAcross, ry = threadIdx.x / kAcross;
    const int64_t j = static_cast<int64_t>(blockIdx.x) * kColumns + 8 * cx;
    const int64_t m0 = M * blockIdx.y / gridDim.y, m1 = M * (blockIdx.y + 1) / gridDim.y;
    double sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    // Four rows at a time; rows beyond the strip are its last one again and count nothing, so that no load stands behind a condition
    // (there they are waited for together with the stores before).
    auto rows = [&](auto whole_columns) {
        constexpr bool kWhole = decltype(whole_columns)::value;
        auto load = [&](const uint16_t* p) {
            if (kWhole) return static_cast<v4u>(__builtin_nontemporal_load(reinterpret_cast<const v4u_any*>(p)));
            v8h h = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int i = 0; i < 8; ++i)
                if (j + i < N) h[i] = p[i];
            return __builtin_bit_cast(v4u, h);
        };
        for (int64_t first = m0 + ry; first < m1; first += 4 * kRowsAtOnce) {
            float part[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            v4u d[4], w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t m = first + u * kRowsAtOnce < m1 ? first + u * kRowsAtOnce : m1 - 1;
                d[u] = load(dy + m * lddy + j);
                if (slope) w[u] = load(slope + m * N + j);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t m = first + u * kRowsAtOnce;
                if (m >= m1) break;
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
                    if (kWhole) {
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
    };
    if (j + 8 <= N) rows(std::true_type());
    else if (j < N) rows(std::false_type());
    if (!sums && !db) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) at[ry][8 * cx + i] = sum[i];
    __syncthreads();
    const int64_t column = static_cast<int64_t>(blockIdx.x) * kColumns + threadIdx.x;
    if (static_cast<int>(threadIdx.x) < kColumns && column < N) {
        double s = 0.0;
        for (int r = 0; r < kRowsAtOnce; ++r) s += at[r][threadIdx.x];
        if (db) db[column] = T::down(static_cast<float>(s));        // the only strip
        else sums[blockIdx.y * N + column] = s;
    }
}
// Sums of the strips, four threads a column.  grid: ceil(N / 64).
template <class T>
__global__ __launch_bounds__(kT) void dense_db_kernel(const double* sums, int strips, int64_t N, uint16_t* db) {
    __shared__ double at[4][64];
    const int64_t j = static_cast<int64_t>(blockIdx.x) * 64 + (threadIdx.x & 63);
    const int part = threadIdx.x >> 6;
    double s = 0.0;
    if (j < N) {
#pragma unroll 8
        for (int r = part; r < strips; r += 4) s += sums[r * N + j];
    }
    at[part][threadIdx.x & 63] = s;
    __syncthreads();
    if (part == 0 && j < N) db[j] = T::down(static_cast<float>(((s + at[1][threadIdx.x]) + at[2][threadIdx.x]) + at[3][threadIdx.x]));
}

}  // namespace

int strips_of(int64_t M) { return static_cast<int>(std::min<int64_t>((M + 255) / 256, 64)); }
template <class T>
void launch_dense_db(const double* sums, int strips, int64_t N, void* db, hipStream_t s) {
    hipLaunchKernelGGL(dense_db_kernel<T>, dim3(static_cast<uint32_t>((N + 63) / 64)), dim3(kT), 0, s, sums, strips, N, static_cast<uint16_t*>(db));
}
template void launch_dense_db<Bf16>(const double* sums, int strips, int64_t N, void* db, hipStream_t s);
template void launch_dense_db<F16>(const double* sums, int strips, int64_t N, void* db, hipStream_t s);

namespace {

template <class T>
void launch_dz_of(const void* dy, int64_t lddy, const uint16_t* slope, void* dz, void* db, double* sums, int64_t M, int64_t N, hipStream_t s) {
    const int strips = strips_of(M);
    auto go = [&](auto kernel, int64_t columns) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>((N + columns - 1) / columns), strips), dim3(kT), 0, s, static_cast<const uint16_t*>(dy), lddy, slope,
                           static_cast<uint16_t*>(dz), db ? sums : nullptr, strips == 1 ? static_cast<uint16_t*>(db) : nullptr, M, N);
    };
    if (strips == 1) go(dense_dz_kernel<T, 8>, 64);
    else if (strips > 1) go(dense_dz_kernel<T, 32>, 256);
    if (db && strips != 1) launch_dense_db<T>(sums, strips, N, db, s);
}

}  // namespace

int64_t dense_sums_bytes(int64_t M, int64_t N) { return strips_of(M) * N * static_cast<int64_t>(sizeof(double)); }

hipError_t launch_dense_dz(int32_t type, const void* dy, int64_t lddy, const uint16_t* slope, void* dz, void* db, double* sums, int64_t M, int64_t N,
                           hipStream_t s) {
    if (type == ADPSGD_TYPE_BF16) launch_dz_of<Bf16>(dy, lddy, slope, dz, db, sums, M, N, s);
    else launch_dz_of<F16>(dy, lddy, slope, dz, db, sums, M, N, s);
    return hipGetLastError();
}

namespace {

int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

// The estimate of a cut, in microseconds, from measured calls: a step of 64 k of a block, with so many of them on a compute unit, and both ends
// of a block.  Tiles of 256 take 1.5 a step and 24; of 128 0.65 alone and 1.0 by two, and 6; of 64 0.5 alone to 0.93 by four, and 3.
// Against 4096^3: 120 (measured 125), 140 (151) and 260 (260); 2048^3: 72 (50), 27 (29), 33 (35); 1024^3: 48 (33), 16 (14), 11 (10.5);
// 512 x 8192 x 512 in eight parts of tiles of 64: 20.  Parts of k are written and read in 32 bits at 5 TB/s, and a launch more.
double estimate(int side, int splits, int64_t I, int64_t J, int64_t K) {
    constexpr double kUnits = 256.0;
    const double tiles = static_cast<double>((I + side - 1) / side) * static_cast<double>((J + side - 1) / side) * splits;
    const double steps = static_cast<double>(((K + 63) / 64 + splits - 1) / splits);
    const double most = side == 256 ? 1.0 : side == 128 ? 2.0 : 4.0, ends = side == 256 ? 24.0 : side == 128 ? 6.0 : 3.0;
    const double together = std::min(most, std::max(1.0, tiles / kUnits)), turns = std::max(1.0, tiles / (kUnits * most));
    const double step = side == 256 ? 1.5 : side == 128 ? 0.30 + 0.35 * together : 0.357 + 0.143 * together;
    return turns * (steps * step + ends) + (splits > 1 ? 4.0 + 8.0 * splits * static_cast<double>(I) * static_cast<double>(J) / 5e6 : 0.0);
}
// Whether a product goes to the kernel for few rows; `b_whole`: B's rows are whole 16-byte pieces.  Microseconds there and in tiles, I x K x J:
//   up to 16 rows: 1 x 4096 x 6144 14 and 19, 16 x 1024 x 1024 4.8 and 9, 16 x 2048 x 8192 11 and 16, 8 x 8192 x 12288 48 and 53, 16 x 16384 x 16384
//     136 and 141; the other way round between 2^25 and 2^26 weights with nearly 16 rows (16 x 8192 x 8192 41 and 34, 8 rows 36 and 34)
//   up to 64 rows, to 2^24 weights: 64 x 4096 x 6144 27 and 22, 64 x 8192 x 8192 52 and 39; 64 x 4096 x 4096 19.1 and 18.7, 64 x 2048 x 4096 14.4 and
//     14.0, 17 x 4096 x 4096 16 and 19, 64 x 1024 x 8192 9.2 and 13.2; whole pieces only: 32 x 2001 x 5003 27 and 21, 64 x 255 x 1021 9.3 and 6.3;
//     64 x 504 x 504 (whole) 5.8 and 7.1
//   k outer, a last block that the end of the columns cuts and K over 1024: 1 x 3000 x 5008 30 and 17, 16 x 3001 x 3001 52 and 21,
//     1 x 4096 x 16416 52 and 42; 1 x 3000 x 5024 (not cut) 9.7 and 16, 16 x 1000 x 1000 9.1 and 10.1
}  // namespace
bool few_rows(int64_t I, int64_t J, int64_t K, bool b_outer, bool b_whole) {
    if (I > 64 || (I > 16 && (!b_whole || J * K > (int64_t(1) << 24)))) return false;
    return !(b_outer && J % narrow_columns(I, J) != 0 && K > 1024);
}
// `few`: for the kernel of few rows.  `direct`: the tiles of 256 and 128, whose operands go straight to LDS, can be had.
DensePlan plan_of(int64_t I, int64_t J, int64_t K, bool few, bool direct) {
    const int64_t steps = std::max<int64_t>(1, (K + 63) / 64);
    if (few) {                           // a wavefront's steps of 64 k take 1 to 2 us each with few blocks: shared from eight on (64 x 8192 x 1024: 15 us, 45 unshared)
        const int64_t blocks = (J + 31) / 32, shares = std::min<int64_t>(std::min<int64_t>(256 / blocks, steps / 16), 32);
        return DensePlan{0, steps >= 64 && shares > 1 ? static_cast<int>(shares) : 1};
    }
    DensePlan best{64, 1};
    double least = 1e30;
    for (int side : {64, 128, 256}) {
        if (side > 64 && !direct) continue;
        for (int splits : {1, 2, 4, 8, 16, 32}) {
            if (splits > 1 && steps / splits < 4) break;
            const double t = estimate(side, splits, I, J, K);
            if (t < least) {
                least = t;
                best = DensePlan{side, splits};
            }
        }
    }
    return best;
}

namespace {
// Rows of `inner` elements as whole 16-byte pieces with zeros at their ends, of several matrices in one launch.  grid: the sum of ceil(rows ceil(inner / 8) / 256).
struct PackJobs {
    PackJob job[kMostPacks];
    uint32_t blocks[kMostPacks];
};
__global__ __launch_bounds__(kT) void dense_pack_kernel(const PackJobs jobs) {
    uint32_t block = blockIdx.x;
    int n = 0;
    while (n + 1 < kMostPacks && block >= jobs.blocks[n]) block -= jobs.blocks[n++];
    const PackJob& j = jobs.job[n];
    const int64_t pieces = (j.inner + 7) / 8, id = static_cast<int64_t>(block) * kT + threadIdx.x;
    const int64_t row = id / pieces, c = id % pieces * 8;
    if (row >= j.rows) return;
    const uint16_t* p = static_cast<const uint16_t*>(j.from) + row * j.ld + c;
    v8h h = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c + 8 <= j.inner) {
        h = __builtin_bit_cast(v8h, *reinterpret_cast<const v4u_any*>(p));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < j.inner) h[i] = p[i];
    }
    *reinterpret_cast<v4u*>(static_cast<uint16_t*>(j.to) + (row * j.ldto + c)) = __builtin_bit_cast(v4u, h);
}
}  // namespace

bool whole_pieces(const void* p, int64_t ld, int64_t inner) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && inner % 8 == 0; }
// Copies of operands whose rows are no whole pieces: they pay where the direct tiles do, from about 2^32 products on (2100 x 1030 x 4097:
// dx 60 us with the copies, 257 with tiles of 64 from the operands as they are).
bool worth_packing(int64_t I, int64_t J, int64_t K) { return static_cast<double>(I) * static_cast<double>(J) * static_cast<double>(K) >= 4294967296.0; }
int64_t packed_bytes(int64_t rows, int64_t inner) { return up256(2 * rows * up8(inner)); }
void launch_pack(const PackJob* job, int jobs, hipStream_t s) {
    constexpr uint32_t kMostBlocks = (uint32_t(1) << 24) - 1;        // under 2^32 threads; one matrix has up to 2^23 blocks
    PackJobs all{};
    uint32_t blocks = 0;
    int n = 0;
    auto go = [&]() {
        if (blocks > 0) hipLaunchKernelGGL(dense_pack_kernel, dim3(blocks), dim3(kT), 0, s, all);
        all = PackJobs{};
        blocks = 0;
        n = 0;
    };
    for (int i = 0; i < jobs; ++i) {
        const uint32_t more = static_cast<uint32_t>((job[i].rows * (up8(job[i].inner) / 8) + kT - 1) / kT);
        if (blocks + more > kMostBlocks) go();
        all.job[n] = job[i];
        all.blocks[n++] = more;
        blocks += more;
    }
    go();
}

// Both ways of storing an operand, and operands that begin anywhere: what any of them may ask for.
int64_t dense_partial_bytes(int64_t I, int64_t J, int64_t K) {
    int64_t parts = 0;
    for (bool direct : {false, true}) parts = std::max<int64_t>(parts, plan_of(I, J, K, false, direct).splits);
    if (I <= 64) parts = std::max<int64_t>(parts, plan_of(I, J, K, true, false).splits);
    const bool pack = (I % 8 || J % 8 || K % 8) && worth_packing(I, J, K);
    const int64_t copies = pack ? std::max(packed_bytes(I, K), packed_bytes(K, I)) + std::max(packed_bytes(J, K), packed_bytes(K, J)) : 0;
    return (parts > 1 ? up256(parts * I * J * static_cast<int64_t>(sizeof(float))) : 0) + copies;
}

hipError_t launch_dense_gemm(int32_t type, const DenseGemm& given, hipStream_t s) {
    if (given.I == 0 || given.J == 0) return hipSuccess;
    DenseGemm g = given;
    if (g.a_low || g.b_low) {                       // small results: tiles of 64 take operands as they are
        const DensePlan p = plan_of(g.I, g.J, g.K, false, false);
        return type == ADPSGD_TYPE_BF16 ? launch_low_tiles<Bf16>(g, p, s) : launch_low_tiles<F16>(g, p, s);
    }
    const int64_t a_inner = g.a_outer ? g.I : g.K, a_rows = g.a_outer ? g.K : g.I, b_inner = g.b_outer ? g.J : g.K, b_rows = g.b_outer ? g.K : g.J;
    const bool a_whole = g.a_padded || whole_pieces(g.a, g.lda, a_inner), b_whole = g.b_padded || whole_pieces(g.b, g.ldb, b_inner);
    const bool pack = !(a_whole && b_whole) && (g.I % 8 || g.J % 8 || g.K % 8) && worth_packing(g.I, g.J, g.K);
    const bool direct = g.K >= 1 && ((a_whole && b_whole) || pack);
    const DensePlan p = plan_of(g.I, g.J, g.K, !g.a_outer && few_rows(g.I, g.J, g.K, g.b_outer, b_whole), direct);
    if (p.side >= 128 && pack) {
        char* at = reinterpret_cast<char*>(g.partial) + (p.splits > 1 ? up256(p.splits * g.I * g.J * static_cast<int64_t>(sizeof(float))) : 0);
        PackJob jobs[2];
        int n = 0;
        auto copy = [&](const void*& from, int64_t& ld, int64_t rows, int64_t inner) {
            jobs[n++] = PackJob{from, ld, at, up8(inner), rows, inner};
            from = at;
            ld = up8(inner);
            at += packed_bytes(rows, inner);
        };
        if (!a_whole) copy(g.a, g.lda, a_rows, a_inner);
        if (!b_whole) copy(g.b, g.ldb, b_rows, b_inner);
        launch_pack(jobs, n, s);
    }
    return type == ADPSGD_TYPE_BF16 ? launch_dense_tiles<Bf16>(g, p, s) : launch_dense_tiles<F16>(g, p, s);
}

}  // namespace adpsgd_impl
