// Large tiled products D[i][j] = sum_k A(i, k) B(j, k), for operands whose rows begin at multiples of 16 bytes: tiles of 256 x 256 by four
// wavefronts of 128 x 128, or of 128 x 128 by four of 64 x 64, two blocks on a compute unit, where the large ones are too few.
//
// Of the large tiles a wavefront is alone on its SIMD and has 512 registers: 256 hold its results, and both halves of a step of 64 k fit
// beside them, so the loads of one half are under way while the other is multiplied.  128 x 128 results of a wavefront read 128 KB of a
// step's operands from LDS a compute unit, 64 x 128 would read 192.
//
// Operands go from memory straight to LDS (buffer loads with the lds bit: 16 bytes a lane, a wavefront's 1024 bytes in a row), so
// they cost no registers.  Two steps' operands are in LDS.  A turn of the loop:
//     request half 1 of step s from LDS;  multiply half 0;
//     wait for the loads of step s + 1 (requested a turn ago);  barrier: nobody reads step s any more, and step s + 1 is there for all;
//     request step s + 2 from memory into the place of step s;  request half 0 of step s + 1 from LDS;  multiply half 1.
// The pieces of 16 bytes are exchanged as in dense_tiles.hpp, here by the addresses that the lanes load from.
//
// Bound: the matrix cores, at the clock that their power leaves.  8192^3 in bf16 takes 850 us, 1.30 PFLOP/s (a library's product 680 to 790); a tile
// of 256 takes 1.45 us a step, 1.5 PFLOP/s over the chip, and 24 us at its ends, which with four tiles of K = 2048 for a compute unit
// are a third of the time (274 us; with gelu, slopes and a residual 327, 343 to 368 between other kernels: the activation is 25 instructions an element).  Two blocks on a
// compute unit would hide the ends, but tiles of 128 take 1.4 times as long for the same products: their fragments come from LDS twice as often.
//
// What lies beyond the ends: rows of an operand with k inner are the last row again; pieces beyond the end of k, and rows of k beyond the
// end where k is outer, are out of the buffer's range, for which the load delivers zeros.
#pragma once

#include "dense_tiles.hpp"

namespace adpsgd_impl {
namespace {

typedef uint32_t v4su __attribute__((ext_vector_type(4)));

// 16 bytes a lane from `rsrc` + offset to LDS at `lds` + 16 lane.  No register is written; the wait is `wait_loads`.  Between the write of M0
// and the load that reads it the hardware wants another instruction.
__device__ __forceinline__ void load_to_lds(v4su rsrc, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(offset), "s"(rsrc), "s"(lds) : "memory");
}
// ... and for this wavefront's reads of the LDS that the next loads go to.
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory"); }

// 16 bytes from accumulation registers to LDS: written out, as the compiler would copy all results to vector registers in front of the loop.
__device__ __forceinline__ void write_result(uint32_t lds, v4f c) { asm volatile("ds_write_b128 %0, %1" : : "v"(lds), "a"(c) : "memory"); }
__device__ __forceinline__ void wait_results() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

constexpr uint32_t kOutOfRange = 0x80000000u;

// Rows are whole pieces: where a row's length is no multiple of 8 it has been copied with zeros behind it (dense_pack_kernel).
__device__ __forceinline__ int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

template <bool kOuter, int kSide, int kStep>
struct DirectOperand {
    static constexpr int kThreads = 256, kLoads = kSide * kBK / 8 / kThreads;
    typedef Operand<kOuter, kSide, kThreads, kStep> Form;
    uint64_t base, end;         // bytes
    uint64_t advance;           // of a step
    uint32_t offset[kLoads];
    uint32_t beyond[2];         // k inner: out of range in the last step, for even and odd loads
    v4su rsrc;                  // of the step that is being loaded ...
    uint32_t to, cut, none;     // ... its place in LDS, all ones in the last step, and kOutOfRange behind it

    __device__ void start(const void* p, int64_t ld, int64_t first, int64_t all, int64_t K) {
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        const uint32_t pitch = static_cast<uint32_t>(ld * 2);
        if (!kOuter) {
            base = at + static_cast<uint64_t>(first) * pitch;
            end = at + static_cast<uint64_t>(all - 1) * pitch + 2 * up8(K);
            advance = 2 * kBK;
            const int there = static_cast<int>(up8(K - (K - 1) / kBK * kBK) / 8);    // pieces of the last step
#pragma unroll
            for (int s = 0; s < 2; ++s) beyond[s] = ((threadIdx.x & 7) ^ Form::turn_of(s * 32 + (threadIdx.x >> 3))) < there ? 0u : kOutOfRange;
        } else {
            base = at + 2 * first;
            end = at + static_cast<uint64_t>(K - 1) * pitch + 2 * up8(all);
            advance = static_cast<uint64_t>(kBK) * pitch;
        }
        const int rows = static_cast<int>(all - first < kSide ? all - first : kSide);
#pragma unroll
        for (int s = 0; s < kLoads; ++s) {
            const int id = s * kThreads + static_cast<int>(threadIdx.x);
            if (!kOuter) {
                const int row = id >> 3, piece = (id & 7) ^ Form::turn_of(row);
                offset[s] = static_cast<uint32_t>(row < rows ? row : rows - 1) * pitch + piece * 16;
            } else {
                const int k = id / Form::kPieces, piece = (id % Form::kPieces) ^ Form::piece_of(k);
                offset[s] = static_cast<uint32_t>(k) * pitch + piece * 16;
            }
        }
    }
    __device__ __forceinline__ void aim(int64_t step, int64_t steps, int64_t until, uint32_t lds) {
        const uint64_t from = base + static_cast<uint64_t>(step) * advance;
        const uint64_t left = end - from;
        const uint32_t range = left < kOutOfRange - 1 ? static_cast<uint32_t>(left) : kOutOfRange - 1;
        rsrc = v4su{static_cast<uint32_t>(from), static_cast<uint32_t>(from >> 32) & 0xFFFFu, range, 0x00020000u};
        to = lds;
        cut = step == steps - 1 ? 0xFFFFFFFFu : 0u;
        none = step < until ? 0u : kOutOfRange;
    }
    __device__ __forceinline__ void load(int s) const {
        const uint32_t at = offset[s] | (kOuter ? none : (beyond[s & 1] & cut) | none);
        load_to_lds(rsrc, at, to + s * kThreads * 16u);
    }
};

// Where a lane reads its fragments of 16 rows and 32 k: what differs between fragments t and halves h by exchanged bits is a register,
// the rest an immediate.  `flip` goes to the other step's operands.
template <bool kOuter, int kSide, int kStep>
struct FragmentReader {
    typedef Operand<kOuter, kSide, 256, kStep> Form;
    static constexpr int kTiles = kSide / 32, kPlaces = !kOuter ? 2 : kStep == 0 ? kTiles : kTiles / 2;
    uint32_t at[kPlaces];

    __device__ void start(uint32_t lds, int row0) {
        const int l = threadIdx.x & 15, q = threadIdx.x >> 4 & 3;
#pragma unroll
        for (int p = 0; p < kPlaces; ++p) {
            if (!kOuter) {                               // the same exchange for all t
                const int row = kStep == 0 ? row0 + l : row0 + (l >> 2) * kStep + (l & 3);
                at[p] = lds + (row * 8 + ((4 * p + q) ^ Form::turn_of(row))) * 16;
            } else {                                     // the same for both h and both fours of k
                const int k = 8 * q + (l >> 2), row = kStep == 0 ? row0 + 16 * p + (l & 3) * 4 : row0 + (l & 3) * kStep + 8 * p;
                at[p] = lds + (k * Form::kPieces + ((row >> 3) ^ Form::piece_of(k))) * 16 + (row & 4) * 2;
            }
        }
    }
    __device__ __forceinline__ void flip() {
#pragma unroll
        for (int p = 0; p < kPlaces; ++p) at[p] ^= 4u * kSide * kBK;       // the operands lie at the beginning of LDS
    }
    __device__ __forceinline__ v4u read(int t, int h) const {
        if (!kOuter) {
            constexpr uint32_t kBytes = (kStep == 0 ? 16 : 4) * 128;
            return *(const __attribute__((address_space(3))) v4u*)(static_cast<uintptr_t>(at[h] + t * kBytes));
        }
        typedef short v4s __attribute__((ext_vector_type(4)));
        const uint32_t from = (kStep == 0 ? at[t] : at[t / 2] + t % 2 * 8) + h * (32 * 2 * kSide);
        v2u half[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
            half[e] = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(static_cast<uintptr_t>(from + e * (4 * 2 * kSide)))));
        return v4u{half[0].x, half[0].y, half[1].x, half[1].y};
    }
};

template <class T, bool kAOuter, bool kBOuter, int kSide>
__global__ __launch_bounds__(256, kSide == 256 ? 1 : 2) void dense_large_kernel(const DenseGemm g, const int splits) {
    constexpr int kTI = kSide / 32, kTJ = kTI, kHalf = kSide * kBK;
    typedef DirectOperand<kAOuter, kSide, 0> OpA;
    typedef DirectOperand<kBOuter, kSide, 4 * kTJ> OpB;
    extern __shared__ __attribute__((aligned(16))) uint16_t lds[];       // [2][A | B]
    const int64_t tiles_i = (g.I + kSide - 1) / kSide, tiles_j = (g.J + kSide - 1) / kSide;
    int64_t ti, tj, split;
    place_of(blockIdx.x, gridDim.x, tiles_i, tiles_j, ti, tj, split);
    const int64_t steps = (g.K + kBK - 1) / kBK, s0 = steps * split / splits, s1 = steps * (split + 1) / splits;
    OpA a;
    OpB b;
    a.start(g.a, g.lda, ti * kSide, g.I, g.K);
    b.start(g.b, g.ldb, tj * kSide, g.J, g.K);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = (wave >> 1) * (kSide / 2), wj = (wave & 1) * (kSide / 2);
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint16_t*)lds)), place = at + wave * 1024;
    FragmentReader<kAOuter, kSide, 0> read_a;
    FragmentReader<kBOuter, kSide, 4 * kTJ> read_b;
    read_a.start(at, wi);
    read_b.start(at + 2 * kHalf, wj);
    v4f acc[kTI][kTJ];
#pragma unroll
    for (int m = 0; m < kTI; ++m)
#pragma unroll
        for (int n = 0; n < kTJ; ++n) acc[m][n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    v4u fa[2][kTI], fb[2][kTJ];

    auto aim = [&](int64_t step) {
        const uint32_t to = place + static_cast<uint32_t>((step - s0) & 1) * (4 * kHalf);
        a.aim(step, steps, s1, to);
        b.aim(step, steps, s1, to + 2 * kHalf);
    };
    auto request = [&](int h, int n) {                   // fragment n of 16, from LDS: those of B first, all products need them
        if (n < kTJ) fb[h][n] = read_b.read(n, h);
        else fa[h][n - kTJ] = read_a.read(n - kTJ, h);
    };
    auto other_step = [&]() {
        read_a.flip();
        read_b.flip();
    };
    // The results take all 256 accumulation registers, so the products are written as instructions that leave a result where it is: the
    // compiler's own form takes a new place for it, and with none left over moves results around (200 to 560 moves a step).
    // Multiplies half h; between the products of one row of fragments and the next: three fragments of the other half, and four
    // loads.  The order is the one written: a block of loads or reads in front of the products would hold them up.
    auto multiply = [&](int h, bool loads) {
#pragma unroll
        for (int m = 0; m < kTI; ++m) {
#pragma unroll
            for (int n = 3 * m; n < 3 * m + 3; ++n)
                if (n < kTI + kTJ) request(1 - h, n);
            if (loads && m < kTI / 2) {
#pragma unroll
                for (int s = 2 * m; s < 2 * m + 2; ++s) {
                    a.load(s);
                    b.load(s);
                }
            }
#pragma unroll
            for (int n = 0; n < kTJ; ++n) {
                T::mfma_in_place(fb[h][n], fa[h][m], acc[m][n]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto all_loads = [&]() {
#pragma unroll
        for (int s = 0; s < OpA::kLoads; ++s) {
            a.load(s);
            b.load(s);
        }
    };
    aim(s0);
    all_loads();
    wait_loads();
    __syncthreads();
    aim(s0 + 1);
    all_loads();
#pragma unroll
    for (int n = 0; n < kTI + kTJ; ++n) request(0, n);
    // Behind the last step nothing is loaded (out of range), and what is requested is not used: one loop without ends of its own.
    for (int64_t step = s0; step < s1; ++step) {
        multiply(0, false);
        wait_loads();
        __syncthreads();
        aim(step + 2);
        other_step();
        multiply(1, true);
    }
    wait_loads();
    wait_mfma();                                         // the compiler may copy a result in front of it, but none of the last eight: a test looks

    // The end.  A store is waited for together with the loads behind it, so the residual's rows are loaded in front of the first store, into
    // the LDS that the operands have left; with loads two turns ahead every turn waited for the stores of the one before, 25 us a tile with
    // gelu.  The results go through LDS, 16 rows of a wavefront at a time: one short loop over eight neighbouring results a lane, which
    // stores rows of 128 or 256 bytes.  As 32 copies of the loop's body it took 60 us a tile: the instructions had to come from memory.
    __syncthreads();                                     // the operands in LDS have been read by all
    constexpr int kColumns = 16 * kTJ, kLanes = kColumns / 8, kRows = 64 / kLanes, kTurns = 16 * kTI / kRows, kMask = kColumns / 4 - 1;
    const int lane = threadIdx.x & 63, l = lane & 15, q = lane >> 4, c = lane % kLanes, at_row = lane / kLanes;
    v4u* kept = reinterpret_cast<v4u*>(lds) + wave * (kTurns * 64) + lane;                     // a lane's own
    float* own = reinterpret_cast<float*>(reinterpret_cast<v4u*>(lds) + 4 * kTurns * 64) + wave * (16 * kColumns);
    const uint32_t stage = at + (4 * kTurns * 64) * 16 + wave * (16 * kColumns * 4) + l * (kColumns * 4) + (((q * kTJ) ^ (l & kMask)) * 16);
    const int64_t i0 = ti * kSide + wi + at_row, j = tj * kSide + wj + 8 * c;
    auto finish_rows = [&](auto whole) {
        const Ending<T, decltype(whole)::value> end(g, j);
        if (g.res) {
            if (end.n > 0) {
                v4u r[kTurns];
#pragma unroll
                for (int t = 0; t < kTurns; ++t) r[t] = end.residual_row(i0 + kRows * t);
#pragma unroll
                for (int t = 0; t < kTurns; ++t) kept[t * 64] = r[t];
            }
        }
#pragma unroll 1
        for (int m = 0; m < kTI; ++m) {
#pragma unroll
            for (int k = 0; k < kTI; ++k)
                if (m == k) {
#pragma unroll
                    for (int n = 0; n < kTJ; ++n) write_result(stage ^ (n * 16), acc[k][n]);      // pieces exchanged by the row
                }
            wait_results();
#pragma unroll 1
            for (int turn = 0; turn < 16 / kRows; ++turn) {
                const int row = turn * kRows + at_row, t = m * (16 / kRows) + turn;
                const v4f f0 = *reinterpret_cast<const v4f*>(own + row * kColumns + ((2 * c) ^ (row & kMask)) * 4);
                const v4f f1 = *reinterpret_cast<const v4f*>(own + row * kColumns + ((2 * c + 1) ^ (row & kMask)) * 4);
                const v4u r = kept[t * 64];
                float f[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
                if (splits > 1) store_part(g, split, i0 + kRows * t, j, f);
                else end.finish(i0 + kRows * t, f, r);
            }
            wave_lds_sync();
        }
    };
    if (g.J % 8 == 0) finish_rows(std::true_type());
    else finish_rows(std::false_type());
}

template <class T, bool kAOuter, bool kBOuter, int kSide>
hipError_t launch_large(const DenseGemm& g, int splits, hipStream_t s) {
    const int64_t tiles = (g.I + kSide - 1) / kSide * ((g.J + kSide - 1) / kSide);
    constexpr int kBytes = kSide == 256 ? 160 * 1024 : 4 * kSide * kBK * 2;       // two steps' operands; the end of the large tiles needs more
    auto kernel = dense_large_kernel<T, kAOuter, kBOuter, kSide>;
    static std::atomic<uint64_t> allowed{0};
    const hipError_t e = allow_lds(allowed, reinterpret_cast<const void*>(kernel), kBytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(tiles * splits)), dim3(256), kBytes, s, g, splits);
    return hipSuccess;
}

}  // namespace
}  // namespace adpsgd_impl
