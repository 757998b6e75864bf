// Tiled products D[i][j] = sum_k A(i, k) B(j, k) on the matrix cores, operands stored either way round, any sizes and strides.
//
// A block owns a tile of D and walks k in steps of 64: the next step's operands are on their way from memory into registers while
// the present ones are multiplied out of LDS, then they go to the other half of the LDS; one barrier a step.
//
// Loads are 16 bytes wide at any multiple of two bytes, so odd leading dimensions take the same path.  Rows beyond the end of A
// or B are the last row again (their results are not stored); what lies beyond the end of k is zero in both operands.  A vector
// that the end cuts is read ending there and shifted, so nothing outside of a row is ever read.
//
// The kernel of this file, tiles of 64, is for what the others do not take: operands that begin anywhere, small products, parts of k.  It is bound
// by the way from memory through registers to LDS (one step takes 0.5 to 0.9 us; 8192 x 2048 x 8192: 493 us, 560 TFLOP/s, where the
// direct tiles take 274).
//
// LDS.  An operand with k inner is kept [row][64 k]; its rows of 128 bytes hold their 16-byte pieces exchanged by bits of the row, so
// that the 16 rows of a matrix operand come from different banks.  One with k outer is kept [k][row] and read by ds_read_b64_tr_b16,
// which gives 16 lanes the transpose of 4 k times 16 rows; pieces are exchanged by bits of k.
//
// Operand layout of v_mfma_f32_16x16x32 (D = A B + C): lane l supplies A[l % 16][8 (l / 16) ..+7] and B[8 (l / 16) ..+7][l % 16], and
// receives D[4 (l / 16) + v][l % 16].  Here B's rows j go in as the instruction's A, and the wavefront's 16 TJ values of j are dealt to its
// TJ instructions so that a lane ends with 4 TJ neighbouring j of one row i: with TJ = 4 a row's 64 results are 128 bytes from 4 lanes.
#pragma once

#include "dense.hpp"

namespace adpsgd_impl {
namespace {

constexpr int kBK = 64;

// Elements start .. start + 7 of a row that ends at `end` (zero beyond it; start may lie beyond).
__device__ __forceinline__ v4u load_cut(const uint16_t* row, int64_t start, int64_t end) {
    if (end < 8) {
        v8h h = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (start + i < end) h[i] = row[start + i];
        return __builtin_bit_cast(v4u, h);
    }
    const int64_t at = start < end - 8 ? start : end - 8;
    const v4u x = *reinterpret_cast<const v4u_any*>(row + at);
    const int64_t by = start - at;                      // elements to drop
    if (by == 0) return x;
    if (by >= 8) return v4u{0, 0, 0, 0};
    uint64_t lo = x.x | static_cast<uint64_t>(x.y) << 32, hi = x.z | static_cast<uint64_t>(x.w) << 32;
    const int bits = static_cast<int>(by) * 16;
    if (bits >= 64) {
        lo = hi >> (bits - 64);
        hi = 0;
    } else {
        lo = lo >> bits | hi << (64 - bits);
        hi >>= bits;
    }
    return v4u{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
}

// Rows of a tile of gated weights: eight gates, their eight partners, eight gates ...  Row r is the partner of a gate or a gate itself
// (kind), and the number of that gate in the tile.
__device__ __forceinline__ int gated_kind(int r) { return r >> 3 & 1; }
__device__ __forceinline__ int gated_row(int r) { return (r >> 4) * 8 + (r & 7); }

// One operand: kRows rows (of i or j) by 64 k, loaded by kThreads threads; kStep: 4 TJ of the permuted operand, or 0.  kGated: kRows / 2 gates
// and their partners `up` elements behind them.
template <bool kOuter, int kRows, int kThreads, int kStep, bool kGated = false>
struct Operand {
    static constexpr int kVectors = kRows * kBK / 8 / kThreads;      // of a thread
    static constexpr int kPieces = kRows / 8;                        // of a k where k is outer
    static_assert(kRows * kBK / 8 % kThreads == 0, "");
    const uint16_t* base;       // row 0 of the tile at k 0
    int64_t ld, rows, depth;    // rows of the tile that are there
    int64_t up;
    bool edge;
    v4u x[kVectors];

    __device__ void start(const void* p, int64_t stride, int64_t first, int64_t all, int64_t K, int64_t partner = 0) {
        constexpr int kMost = kGated ? kRows / 2 : kRows;
        ld = stride;
        up = partner;
        rows = all - first < kMost ? all - first : kMost;
        edge = rows < kMost;
        depth = K;
        base = static_cast<const uint16_t*>(p) + (kOuter ? first : first * stride);
    }
    __device__ static int piece_of(int k) {             // exchange of the 16-byte pieces of a k
        if (kStep == 0) return ((k & 3) << 1 | ((k >> 3 & 1) << 3)) & (kPieces - 1);
        if (kStep == 32) return k & 3;
        if (kStep == 16) return ((k & 1) | (k >> 1 & 1) << 3 | (k >> 3 & 1) << 4) & (kPieces - 1);
        return ((k & 3) << 2) & (kPieces - 1);
    }
    __device__ static int turn_of(int row) { return kStep == 0 ? row & 7 : (row & 3) | (row / (kStep ? kStep : 1) & 1) << 2; }

    // k step `step`; `last`: it reaches the end of k
    __device__ __forceinline__ void load(int64_t step, bool last) {
#pragma unroll
        for (int s = 0; s < kVectors; ++s) {
            const int id = s * kThreads + static_cast<int>(threadIdx.x);
            if (!kOuter) {
                int row = kGated ? gated_row(id >> 3) : id >> 3;
                row = row < rows ? row : static_cast<int>(rows) - 1;
                const int64_t k = step * kBK + (id & 7) * 8;
                const uint16_t* p = base + static_cast<int64_t>(row) * ld + (kGated && gated_kind(id >> 3) ? up : 0);
                x[s] = last ? load_cut(p, k, depth) : *reinterpret_cast<const v4u_any*>(p + k);
            } else {
                const int64_t k = step * kBK + id / kPieces;
                const int at = kGated ? gated_row(id % kPieces * 8) : id % kPieces * 8;
                if (last && k >= depth) {
                    x[s] = v4u{0, 0, 0, 0};
                } else {
                    const uint16_t* p = base + k * ld + (kGated && gated_kind(id % kPieces * 8) ? up : 0);
                    x[s] = edge ? load_cut(p, at, rows) : *reinterpret_cast<const v4u_any*>(p + at);
                }
            }
        }
    }
    __device__ __forceinline__ void store(uint16_t* lds) const {
#pragma unroll
        for (int s = 0; s < kVectors; ++s) {
            const int id = s * kThreads + static_cast<int>(threadIdx.x);
            int place;
            if (!kOuter) {
                const int row = id >> 3;
                place = row * 8 + ((id & 7) ^ turn_of(row));
            } else {
                const int k = id / kPieces;
                place = k * kPieces + ((id % kPieces) ^ piece_of(k));
            }
            *reinterpret_cast<v4u*>(lds + place * 8) = x[s];
        }
    }
    // The matrix operand of 16 rows and 32 k (half `h` of the 64): rows row0 + l % 16, or with kStep the rows
    // row0 + (l % 16 / 4) kStep + 4 t + l % 4.
    __device__ static __forceinline__ v4u fragment(const uint16_t* lds, int row0, int t, int h) {
        const int l = threadIdx.x & 15, q = threadIdx.x >> 4 & 3;
        if (!kOuter) {
            const int row = kStep == 0 ? row0 + 16 * t + l : row0 + (l >> 2) * kStep + 4 * t + (l & 3);
            return *reinterpret_cast<const v4u*>(lds + (row * 8 + ((4 * h + q) ^ turn_of(row))) * 8);
        }
        typedef short v4s __attribute__((ext_vector_type(4)));
        const int row = kStep == 0 ? row0 + 16 * t + (l & 3) * 4 : row0 + (l & 3) * kStep + 4 * t;     // four from here on, at k + l / 4
        v2u half[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int k = 32 * h + 8 * q + 4 * e + (l >> 2);
            const uint16_t* p = lds + (k * kPieces + ((row >> 3) ^ piece_of(k))) * 8 + (row & 4);
            half[e] = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(p)));
        }
        return v4u{half[0].x, half[0].y, half[1].x, half[1].y};
    }
};

// bias, activation, slope, residual and rounding of up to kN neighbouring results (4 or 8) of row i from column j on
template <int kN>
__device__ __forceinline__ void load_up_to(const uint16_t* p, int64_t n, uint16_t* h) {
    if (n >= kN) {
        __builtin_memcpy(h, p, 2 * kN);
        return;
    }
#pragma unroll
    for (int v = 0; v < kN; ++v) h[v] = v < n ? p[v] : 0;
}
template <int kN>
__device__ __forceinline__ void store_up_to(uint16_t* p, int64_t n, const uint16_t* h) {
    if (n >= kN) {
        __builtin_memcpy(p, h, 2 * kN);
        return;
    }
#pragma unroll
    for (int v = 0; v < kN; ++v)
        if (v < n) p[v] = h[v];
}
// Eight activations at once: the choice outside, so that their steps interleave.
template <bool kSlope>
__device__ __forceinline__ void activate8(float* f, float* slope, int act) {
    auto all = [&](auto which) {
#pragma unroll
        for (int v = 0; v < 8; ++v) f[v] = activated<kSlope, decltype(which)::value>(f[v], slope[v]);
    };
    if (act == ADPSGD_ACT_RELU) all(std::integral_constant<int, ADPSGD_ACT_RELU>());
    else if (act == ADPSGD_ACT_GELU) all(std::integral_constant<int, ADPSGD_ACT_GELU>());
    else all(std::integral_constant<int, ADPSGD_ACT_SILU>());
}

// The end of eight neighbouring columns from j on: what all rows share is read once.  kWhole: J is a multiple of 8.
template <class T, bool kWhole>
struct Ending {
    const DenseGemm& g;
    int64_t j;
    int n;                      // columns that are there, up to 8
    float bias[8];

    __device__ __forceinline__ Ending(const DenseGemm& gemm, int64_t column) : g(gemm), j(column) {
        n = g.J - j < 0 ? 0 : g.J - j < 8 ? static_cast<int>(g.J - j) : 8;
        uint16_t h[8];
        if (g.bias && n > 0) load(static_cast<const uint16_t*>(g.bias) + j, h);
#pragma unroll
        for (int v = 0; v < 8; ++v) bias[v] = g.bias && v < n ? T::up(h[v]) : 0.0f;
    }
    __device__ __forceinline__ void load(const uint16_t* p, uint16_t* h) const {
        if (kWhole) __builtin_memcpy(h, p, 16);
        else load_up_to<8>(p, n, h);
    }
    __device__ __forceinline__ void store(uint16_t* p, const uint16_t* h) const {
        if (kWhole) __builtin_memcpy(p, h, 16);
        else store_up_to<8>(p, n, h);
    }
    // Where there is a residual and a column (n > 0); a row beyond the end reads the last one.
    __device__ __forceinline__ v4u residual_row(int64_t i) const {
        uint16_t h[8];
        load(static_cast<const uint16_t*>(g.res) + (i < g.I ? i : g.I - 1) * g.ldres + j, h);
        v4u r;
        __builtin_memcpy(&r, h, 16);
        return r;
    }
    __device__ __forceinline__ v4u residual(int64_t i) const {
        uint16_t h[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (g.res && i < g.I && n > 0) load(static_cast<const uint16_t*>(g.res) + i * g.ldres + j, h);
        v4u r;
        __builtin_memcpy(&r, h, 16);
        return r;
    }
    __device__ __forceinline__ void finish(int64_t i, float* f, v4u r) const {
        if (i >= g.I || n <= 0) return;
        const int64_t at = i * g.J + j;
        uint16_t h[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) f[v] += bias[v];
        if (g.act != ADPSGD_ACT_NONE) {
            float slope[8];
            if (g.slope) {
                activate8<true>(f, slope, g.act);
                const v4u w = slope_words(slope);
                __builtin_memcpy(h, &w, 16);
                store(g.slope + at, h);
            } else {
                activate8<false>(f, slope, g.act);
            }
        }
        if (g.res) {
            float add[8];
            unpack8<T>(r, add);
#pragma unroll
            for (int v = 0; v < 8; ++v) f[v] += add[v];
        }
#pragma unroll
        for (int v = 0; v < 8; ++v) h[v] = T::down(f[v]);
        store(static_cast<uint16_t*>(g.out) + at, h);
    }
};

// Eight neighbouring sums of a part of k, for dense_join_kernel.
__device__ __forceinline__ void store_part(const DenseGemm& g, int64_t split, int64_t i, int64_t j, const float* f) {
    if (i >= g.I || j >= g.J) return;
    float* out = g.partial + (split * g.I + i) * g.J + j;
    if (j + 8 <= g.J) {
        __builtin_memcpy(out, f, 32);
        return;
    }
#pragma unroll
    for (int v = 0; v < 8; ++v)
        if (j + v < g.J) out[v] = f[v];
}

// ---- gated projections: act(gate) partner ----
// What lane `lane` has, to all; lane is the same for all, and one of those that are here.
template <class V>
__device__ __forceinline__ V read_lane(V value, int lane) {
    constexpr int kWords = sizeof(V) / 4;
    struct Words {
        int w[kWords];
    };
    Words x = __builtin_bit_cast(Words, value);
#pragma unroll
    for (int i = 0; i < kWords; ++i) x.w[i] = __builtin_amdgcn_readlane(x.w[i], lane);
    return __builtin_bit_cast(V, x);
}
// The end of eight neighbouring results from column j on.  kWhole: J is a multiple of 8.
template <class T, bool kWhole>
struct GatedEnding {
    const DenseGemm& g;
    int64_t j;
    int n;                      // columns that are there, up to 8
    float bias[2][8];
    mutable int walks, idle;    // gates that this wavefront may still add again, and those of 0 that may come out as 0

    // most: of `walks`
    __device__ __forceinline__ GatedEnding(const DenseGemm& gemm, int64_t column, int most) : g(gemm), j(column), walks(most), idle(4) {
        n = g.J - j < 0 ? 0 : g.J - j < 8 ? static_cast<int>(g.J - j) : 8;
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            uint16_t h[8];
            if (g.bias && n > 0) load_up_to<8>(static_cast<const uint16_t*>(g.bias) + kind * g.J + j, n, h);
#pragma unroll
            for (int v = 0; v < 8; ++v) bias[kind][v] = g.bias && v < n ? T::up(h[v]) : 0.0f;
        }
    }
    __device__ __forceinline__ void store(uint16_t* p, const uint16_t* h) const {
        if (kWhole) __builtin_memcpy(p, h, 16);
        else store_up_to<8>(p, n, h);
    }
    // The slope of relu jumps at 0, and a gate that is 0 but for the rounding of its sum has either sign: one such gate in a million puts the gradients
    // of a layer twice as far from 64 bits as their other roundings do.  Gates under sqrt(K + 64) 2^-25 of the largest of their eight neighbours and of their
    // column's scale (about ten times what sums are off by; six of 2003 x 2731), a column alone in its eight of the latter, are added again in 64 bits by all lanes that are here.
    // The column's scale keeps out the gates whose weights are all 0 or tiny, each of which would be one of them.  Sums that are 0 because no product is anything (one-hot
    // rows of x beside pruned weights) are among their row's and column's ordinary gates: a wavefront adds those that are 0 again only until four of them were 0 after
    // all, and no more than `walks` gates in all, those that are not 0 first; the others keep the side that 32 bits give them.
    // 8192 x 2048 x 8192 in bf16, forward with slopes, one call after the other: 527 us (silu 520 to 530);  a tenth of the columns tiny 690;  half of the gates sums of zeros
    // 700 (95 ms if all of them are added again);  half of them sums that cancel to what they are rounded by 1465 (99 ms).  2003 x 1021 x 2731 in fp16: 57 (silu 56), 62, 82.
    // scales(gate, s): s[v], infinite where there is nothing to tell it by.
    template <class Scales>
    __device__ __forceinline__ void settle(int64_t i, float* gate, const Scales& scales) const {
        const float corner = 0x1p-25f * __builtin_amdgcn_sqrtf(static_cast<float>(g.K + 64));
        float least = INFINITY, top = 0.0f;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            least = kWhole || v < n ? fminf(least, fabsf(gate[v])) : least;
            top = kWhole || v < n ? fmaxf(top, fabsf(gate[v])) : top;
        }
        const bool alone = !kWhole && n == 1;            // no neighbours: its column tells
        const bool some = (alone || least < top * corner) && top < INFINITY;
        if (__ballot(some) == 0) return;
        float scale[8];
        scales(gate, scale);
        uint32_t near = 0, zero = 0;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            near |= fabsf(gate[v]) < corner * (alone ? scale[v] : fminf(top, scale[v])) ? 1u << v : 0u;
            zero |= gate[v] == 0.0f ? 1u << v : 0u;
        }
        near &= some ? (1u << n) - 1u : 0u;
        uint32_t open = near & ~zero;
        zero &= near;
        const int me = threadIdx.x & 63;
        const uint64_t here = __ballot(1);
        int may = __builtin_amdgcn_readfirstlane(walks), vain = __builtin_amdgcn_readfirstlane(idle);       // rows ascend: who is here now was here before
        for (; may > 0; --may) {
            uint64_t left = __ballot(open != 0);
            const bool zeros = left == 0;
            if (zeros) left = vain > 0 ? __ballot(zero != 0) : 0;
            if (left == 0) break;
            const int lane = __builtin_ctzll(left), v = __builtin_ctz(read_lane(zeros ? zero : open, lane));
            const int64_t row = read_lane(i, lane), column = read_lane(j, lane) + v;
            const uint16_t* a = static_cast<const uint16_t*>(g.a) + row * g.lda;
            const uint16_t* b = static_cast<const uint16_t*>(g.b) + (g.b_outer ? column : column * g.ldb);
            const int rank = __builtin_popcountll(here & ((uint64_t(1) << me) - 1)), lanes = __builtin_popcountll(here);
            double part = 0.0, sum = 0.0;
#pragma unroll 1
            for (int64_t k = rank; k < g.K; k += 8 * lanes) {
                uint16_t ha[8], hb[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {            // all on their way at once
                    const int64_t at = k + e * lanes < g.K ? k + e * lanes : g.K - 1;
                    ha[e] = a[at];
                    hb[e] = b[g.b_outer ? at * g.ldb : at];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) part = fma(k + e * lanes < g.K ? static_cast<double>(T::up(ha[e])) : 0.0, static_cast<double>(T::up(hb[e])), part);
            }
            if (lanes == 64) sum = wave_sum(part);
            else
                for (uint64_t l = here; l; l &= l - 1) sum += read_lane(part, __builtin_ctzll(l));
            bool still = false;
            if (me == lane) {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    gate[u] = u == v ? static_cast<float>(sum + static_cast<double>(bias[0][u])) : gate[u];
                    still = still || (u == v && gate[u] == 0.0f);
                }
                if (zeros) zero &= zero - 1;
                else open &= open - 1;
            }
            vain -= zeros && __ballot(still) != 0;
        }
        walks = may;
        idle = vain;
    }
    // Scales of a tile: the largest of the wavefront's other rows, kLanes lanes kApart apart.
    template <int kApart, int kLanes>
    __device__ __forceinline__ static void of_columns(const float* gate, float* scale) {
        const uint64_t here = __ballot(1);
        const int me = threadIdx.x & 63;
        uint64_t others = 0;
#pragma unroll
        for (int r = 0; r < kLanes; ++r) others |= uint64_t(1) << (r * kApart);
        others <<= me & ~((kLanes - 1) * kApart);
        const bool alone = (here & others) == uint64_t(1) << me;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            float s = fabsf(gate[v]);
#pragma unroll
            for (int off = kApart; off < kApart * kLanes; off *= 2) {
                const float theirs = __shfl_xor(s, off, 64);
                s = here >> (me ^ off) & 1u ? fmaxf(s, theirs) : s;
            }
            scale[v] = alone ? INFINITY : s;
        }
    }
    // Scales of sums of `parts` parts: the largest of them.  part(p, v): part p of gate v.
    template <class Part>
    __device__ __forceinline__ static void of_parts(int parts, const Part& part, float* scale) {
        for (int v = 0; v < 8; ++v) {
            float most = 0.0f;
            int some = 0;
            for (int p = 0; p < parts; ++p) {
                const float f = part(p, v);
                most = fmaxf(most, fabsf(f));
                some += f != 0.0f;
            }
            scale[v] = some == 1 ? INFINITY : most;
        }
    }
    template <bool kCorner = true, class Scales>
    __device__ __forceinline__ void finish(int64_t i, float* gate, float* up, const Scales& scales) const {
        if (i >= g.I || n <= 0) return;
        uint16_t h[8];
        float slope[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            gate[v] += bias[0][v];
            up[v] += bias[1][v];
            slope[v] = 1.0f;
        }
        if (g.slope) {
            if (kCorner && g.act == ADPSGD_ACT_RELU) settle(i, gate, scales);
            if (g.act != ADPSGD_ACT_NONE) activate8<true>(gate, slope, g.act);
            const GatedSlopes<T> kept(g.slope, g.I, g.J);
#pragma unroll
            for (int v = 0; v < 8; ++v) slope[v] *= up[v];
#pragma unroll
            for (int kind = 0; kind < 2; ++kind) {
                const int64_t at = (2 * i + kind) * g.J + j;
                uint32_t w[8];
#pragma unroll
                for (int v = 0; v < 8; ++v) w[v] = GatedSlopes<T>::word(kind ? gate[v] : slope[v]);
#pragma unroll
                for (int v = 0; v < 8; ++v) h[v] = static_cast<uint16_t>(w[v] >> 8);
                store(kept.high + at, h);
                if (!GatedSlopes<T>::kLow) continue;
                if (kWhole || n == 8) {
                    const uint32_t low[2] = {(w[0] & 255u) | (w[1] & 255u) << 8 | (w[2] & 255u) << 16 | w[3] << 24,
                                             (w[4] & 255u) | (w[5] & 255u) << 8 | (w[6] & 255u) << 16 | w[7] << 24};
                    __builtin_memcpy(kept.low + at, low, 8);
                } else {
#pragma unroll
                    for (int v = 0; v < 8; ++v)
                        if (v < n) kept.low[at + v] = static_cast<uint8_t>(w[v]);
                }
            }
            if (__builtin_expect(GatedSlopes<T>::some_large(slope, gate), 0)) kept.put_large(slope, gate, i, j, g.J, n);
        } else if (g.act != ADPSGD_ACT_NONE) {
            activate8<false>(gate, slope, g.act);
        }
#pragma unroll
        for (int v = 0; v < 8; ++v) h[v] = T::down(gate[v] * up[v]);
        store(static_cast<uint16_t*>(g.out) + i * g.J + j, h);
    }
};
// Eight neighbouring sums of a part of k, gates [split][i][j] and their partners J behind them, for gated_join_kernel.
__device__ __forceinline__ void store_gated_part(const DenseGemm& g, int64_t split, int64_t i, int64_t j, const float* gate, const float* up) {
    if (i >= g.I || j >= g.J) return;
    float* out = g.partial + (split * g.I + i) * (2 * g.J) + j;
    const int n = g.J - j < 8 ? static_cast<int>(g.J - j) : 8;
    if (n == 8) {
        __builtin_memcpy(out, gate, 32);
        __builtin_memcpy(out + g.J, up, 32);
        return;
    }
#pragma unroll
    for (int v = 0; v < 8; ++v)
        if (v < n) {
            out[v] = gate[v];
            out[g.J + v] = up[v];
        }
}

// Blocks go to the eight XCDs in turn, each with an L2 of its own: block b takes the tile that gives every XCD a run of neighbouring
// ones, and a run goes through 4 tiles of j before it moves on in i, so that the tiles at work on an XCD share rows of both and
// those at work on all of them write whole rows of D.
__device__ __forceinline__ void place_of(int64_t b, int64_t blocks, int64_t tiles_i, int64_t tiles_j, int64_t& ti, int64_t& tj, int64_t& split) {
    const int64_t q = blocks / 8, r = blocks % 8, xcd = b % 8;
    const int64_t id = xcd * q + (xcd < r ? xcd : r) + b / 8;
    split = id / (tiles_i * tiles_j);
    const int64_t t = id % (tiles_i * tiles_j), group = t / (4 * tiles_i), first = group * 4;
    const int64_t size = tiles_j - first < 4 ? tiles_j - first : 4, in = t % (4 * tiles_i);
    tj = first + in % size;
    ti = in / size;
}

// kSide x kSide tiles, kWI x kWJ wavefronts.  kGated: of kSide / 2 results and their partners.  kLow: A (1) or B (2) is in two
// parts, whose products are added.
template <class T, bool kAOuter, bool kBOuter, int kSide, int kWI, int kWJ, bool kGated = false, int kLow = 0>
__global__ __launch_bounds__(kWI * kWJ * 64) void dense_tile_kernel(const DenseGemm g, const int splits) {
    constexpr int kThreads = kWI * kWJ * 64, kTI = kSide / kWI / 16, kTJ = kSide / kWJ / 16;
    typedef Operand<kAOuter, kSide, kThreads, 0> OpA;
    typedef Operand<kBOuter, kSide, kThreads, 4 * kTJ, kGated> OpB;
    constexpr int kSideJ = kGated ? kSide / 2 : kSide;
    extern __shared__ __attribute__((aligned(16))) uint16_t lds[];       // [2][A | B | the low part]
    constexpr int kHalf = kSide * kBK, kAll = (kLow ? 3 : 2) * kHalf;    // elements of one operand's step, of all operands'

    const int64_t tiles_i = (g.I + kSide - 1) / kSide, tiles_j = (g.J + kSideJ - 1) / kSideJ;
    int64_t ti, tj, split;
    place_of(blockIdx.x, gridDim.x, tiles_i, tiles_j, ti, tj, split);
    const int64_t steps = (g.K + kBK - 1) / kBK, s0 = steps * split / splits, s1 = steps * (split + 1) / splits;
    OpA a;
    OpB b;
    typename std::conditional<kLow == 2, OpB, OpA>::type low;
    a.start(g.a, g.lda, ti * kSide, g.I, g.K);
    if (kLow == 1) low.start(g.a_low, g.lda, ti * kSide, g.I, g.K);
    if (kLow == 2) low.start(g.b_low, g.ldb, tj * kSideJ, g.J, g.K);
    b.start(g.b, g.ldb, tj * kSideJ, g.J, g.K, g.b_up);
    const int wave = threadIdx.x >> 6, wi = wave / kWJ * (kTI * 16), wj = wave % kWJ * (kTJ * 16);
    v4f acc[kTI][kTJ];
#pragma unroll
    for (int m = 0; m < kTI; ++m)
#pragma unroll
        for (int n = 0; n < kTJ; ++n) acc[m][n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    auto fetch = [&](int64_t step) {
        const bool last = step == steps - 1;             // uniform
        if (last) {
            a.load(step, true);
            b.load(step, true);
            if (kLow) low.load(step, true);
        } else {
            a.load(step, false);
            b.load(step, false);
            if (kLow) low.load(step, false);
        }
    };
    auto put = [&](uint16_t* to) {
        a.store(to);
        b.store(to + kHalf);
        if (kLow) low.store(to + 2 * kHalf);
    };
    if (s0 < s1) {
        fetch(s0);
        put(lds);
        __syncthreads();
    }
    for (int64_t step = s0; step < s1; ++step) {
        const uint16_t* now = lds + ((step - s0) & 1) * kAll;
        if (step + 1 < s1) fetch(step + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4u fa[kTI], fb[kTJ];
#pragma unroll
            for (int n = 0; n < kTJ; ++n) fb[n] = OpB::fragment(now + kHalf, wj, n, h);
#pragma unroll
            for (int m = 0; m < kTI; ++m) fa[m] = OpA::fragment(now, wi, m, h);
#pragma unroll
            for (int m = 0; m < kTI; ++m)
#pragma unroll
                for (int n = 0; n < kTJ; ++n) acc[m][n] = T::mfma(fb[n], fa[m], acc[m][n]);
            if constexpr (kLow != 0) {
                if constexpr (kLow == 1) {
#pragma unroll
                    for (int m = 0; m < kTI; ++m) fa[m] = OpA::fragment(now + 2 * kHalf, wi, m, h);
                } else {
#pragma unroll
                    for (int n = 0; n < kTJ; ++n) fb[n] = OpB::fragment(now + 2 * kHalf, wj, n, h);
                }
#pragma unroll
                for (int m = 0; m < kTI; ++m)
#pragma unroll
                    for (int n = 0; n < kTJ; ++n) acc[m][n] = T::mfma(fb[n], fa[m], acc[m][n]);
            }
        }
        if (step + 1 < s1) put(lds + ((step + 1 - s0) & 1) * kAll);
        __syncthreads();
    }

    const int l = threadIdx.x & 15, q = threadIdx.x >> 4 & 3;
    if constexpr (kGated) {                              // a lane has eight neighbouring gates and their partners
        static_assert(kTJ == 4 && kWJ == 1, "");
        const GatedEnding<T, false> end(g, tj * kSideJ + q * 8, 8);
#pragma unroll
        for (int m = 0; m < kTI; ++m) {
            const int64_t i = ti * kSide + wi + l + m * 16;
            float f[2][8];
#pragma unroll
            for (int v = 0; v < 16; ++v) f[v / 8][v % 8] = acc[m][v / 4][v % 4];
            if (splits > 1) store_gated_part(g, split, i, end.j, f[0], f[1]);
            else end.finish(i, f[0], f[1], [](const float* gate, float* scale) { GatedEnding<T, false>::template of_columns<1, 16>(gate, scale); });
        }
        return;
    }
    const int64_t j = tj * kSide + wj + q * (4 * kTJ), i0 = ti * kSide + wi + l;
    if (j >= g.J) return;
#pragma unroll
    for (int n = 0; n < kTJ; n += 2) {
        const Ending<T, false> end(g, j + 4 * n);
        v4u r[kTI];
#pragma unroll
        for (int m = 0; m < kTI; ++m) r[m] = end.residual(i0 + m * 16);
#pragma unroll
        for (int m = 0; m < kTI; ++m) {
            float f[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) f[v] = acc[m][n + v / 4][v % 4];
            if (splits > 1) store_part(g, split, i0 + m * 16, j + 4 * n, f);
            else end.finish(i0 + m * 16, f, r[m]);
        }
    }
}

// The parts of k in their order, then the same end.  grid: ceil(I ceil(J / 8) / 256).
template <class T>
__global__ __launch_bounds__(256) void dense_join_kernel(const DenseGemm g, const int splits) {
    const int64_t eights = (g.J + 7) / 8, id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t i = id / eights, j = id % eights * 8;
    if (i >= g.I) return;
    const Ending<T, false> end(g, j);
    const v4u r = end.residual(i);
    float f[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < splits; ++s) {
        const float* p = g.partial + (s * g.I + i) * g.J + j;
        if (end.n == 8) {
            float part[8];
            __builtin_memcpy(part, p, sizeof part);
#pragma unroll
            for (int v = 0; v < 8; ++v) f[v] += part[v];
        } else {
#pragma unroll
            for (int v = 0; v < 8; ++v)
                if (v < end.n) f[v] += p[v];
        }
    }
    end.finish(i, f, r);
}

// The same for gated projections.
template <class T>
__global__ __launch_bounds__(256) void gated_join_kernel(const DenseGemm g, const int splits) {
    const int64_t eights = (g.J + 7) / 8, id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t i = id / eights, j = id % eights * 8;
    if (i >= g.I) return;
    const GatedEnding<T, false> end(g, j, 32);
    float f[2][8] = {}, most[8] = {};
    int some[8] = {};
    for (int s = 0; s < splits; ++s) {
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            const float* p = g.partial + (s * g.I + i) * (2 * g.J) + kind * g.J + j;
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                const float part = v < end.n ? p[v] : 0.0f;
                f[kind][v] += part;
                if (kind == 1) continue;
                most[v] = fmaxf(most[v], fabsf(part));
                some[v] += part != 0.0f;
            }
        }
    }
    end.finish(i, f[0], f[1], [&](const float*, float* scale) {          // as of_parts: read again for it, 32 parts are 10 us
#pragma unroll
        for (int v = 0; v < 8; ++v) scale[v] = some[v] == 1 ? INFINITY : most[v];
    });
}

template <class T, bool kAOuter, bool kBOuter, int kSide, int kWI, int kWJ, bool kGated = false, int kLow = 0>
hipError_t launch_tile(const DenseGemm& g, int splits, hipStream_t s) {
    constexpr int kSideJ = kGated ? kSide / 2 : kSide;
    const int64_t tiles = (g.I + kSide - 1) / kSide * ((g.J + kSideJ - 1) / kSideJ);
    constexpr int kBytes = (kLow ? 6 : 4) * kSide * kBK * 2;
    auto kernel = dense_tile_kernel<T, kAOuter, kBOuter, kSide, kWI, kWJ, kGated, kLow>;
    static std::atomic<uint64_t> allowed{0};
    const hipError_t e = allow_lds(allowed, reinterpret_cast<const void*>(kernel), kBytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(tiles * splits)), dim3(kWI * kWJ * 64), kBytes, s, g, splits);
    return hipSuccess;
}
}  // namespace
}  // namespace adpsgd_impl
