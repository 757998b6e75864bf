// Shared by the kernels of dense layers: their two types, the activations with their slopes, and the 16-bit form of a slope.
#pragma once

#include <type_traits>

#include "device_common.hpp"
#include "operators.hpp"
#include "per_device.hpp"

namespace adpsgd_impl {

typedef v4u v4u_any __attribute__((aligned(2)));        // 16 bytes at any multiple of an element
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint16_t v8h __attribute__((ext_vector_type(8)));

struct Bf16 {
    typedef __bf16 V8 __attribute__((ext_vector_type(8)));
    __device__ static float up(uint16_t h) { return bf16_to_float(h); }
    __device__ static uint16_t down(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
    __device__ static v4f mfma(v4u a, v4u b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
    }
    // c in accumulation registers, and in the same ones before and after; wait_mfma before c is read
    __device__ static void mfma_in_place(v4u a, v4u b, v4f& c) { asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};
struct F16 {
    typedef _Float16 V8 __attribute__((ext_vector_type(8)));
    __device__ static float up(uint16_t h) { return static_cast<float>(__builtin_bit_cast(_Float16, h)); }
    __device__ static uint16_t down(float f) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(f)); }
    __device__ static v4f mfma(v4u a, v4u b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
    }
    __device__ static void mfma_in_place(v4u a, v4u b, v4f& c) { asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};

// An instruction that reads the result of a matrix instruction has to come some cycles later, which the compiler sees to for its
// own only: 32 cycles cover every form.
__device__ __forceinline__ void wait_mfma() { asm volatile("s_nop 15\n\ts_nop 15"); }

// Eight values rounded.
template <class T>
__device__ __forceinline__ v4u pack8(const float* f) {
    v4u v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = T::down(f[2 * i]) | static_cast<uint32_t>(T::down(f[2 * i + 1])) << 16;
    return v;
}
template <class T>
__device__ __forceinline__ void unpack8(v4u v, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = T::up(static_cast<uint16_t>(v[i] & 0xFFFFu));
        f[2 * i + 1] = T::up(static_cast<uint16_t>(v[i] >> 16));
    }
}

// act(z) and its derivative.  gelu: the upper tail of the normal distribution is exp(-t^2 / 2) P(1 / (1 + 0.38 t)), P of degree 7
// fitted to the least largest relative error over t >= 0, 2.6e-6: the tail keeps its relative accuracy, unlike 1 + erf.
template <bool kSlope, int kAct>
__device__ __forceinline__ float activated(float z, float& slope) {
    if (kAct == ADPSGD_ACT_RELU) {
        slope = z > 0.0f ? 1.0f : 0.0f;
        return z <= 0.0f ? 0.0f : z;                     // NaN stays
    }
    if (kAct == ADPSGD_ACT_GELU) {
        const float t = fabsf(z), u = __builtin_amdgcn_rcpf(fmaf(0.38f, t, 1.0f));
        const float e = __builtin_amdgcn_exp2f(z * z * -0.7213475204444817f);
        float p = fmaf(u, 0.04894981298366624f, -0.16002513951519665f);
        p = fmaf(p, u, 0.11438935044517826f);
        p = fmaf(p, u, 0.05999139163590317f);
        p = fmaf(p, u, 0.1337908999955492f);
        p = fmaf(p, u, 0.15129931401177749f);
        p = fmaf(p, u, 0.15160565325274758f);
        const float tail = e * u * p, phi = z < 0.0f ? tail : 1.0f - tail;
        if (kSlope) slope = fmaf(z * 0.3989422804014327f, e, phi);
        return z * phi;
    }
    const float sig = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f)), y = z * sig;
    if (kSlope) slope = fmaf(y, 1.0f - sig, sig);
    return y;
}

// Slopes in 16 bits for the backward pass: their roots, signs kept, in steps of 1 / 46000 (roots are from -0.359 to 1.063: words 80 to 65479), and 0
// for NaN, which no slope comes to.  A slope s is within 2.2e-5 |s|^1/2 (1.2e-10 where its word is that of 0): 2^-15.5 at 1, and no more than half a step
// of fp16 down to 2^-9, of bf16 to 2^-15; beside the rounding of dz to its type that is little.  In steps of s itself (2^-15) the same 16 bits
// were coarser than fp16 under 2^-5, and in the tails of gelu and silu nothing was left.  0 and 1 are exact.
constexpr float kRootSteps = 46000.0f, kRootZero = 16600.0f;
__device__ __forceinline__ v4u slope_words(const float* s) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = fmaf(copysignf(__builtin_amdgcn_sqrtf(fabsf(s[i])), s[i]), kRootSteps / 65535.0f, kRootZero / 65535.0f);
    v4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pknorm_u16(r[2 * i], r[2 * i + 1]));
    return w;
}
__device__ __forceinline__ float slope_of(uint32_t w) {
    const float r = (static_cast<float>(w) - kRootZero) * (1.0f / kRootSteps);
    return w == 0u ? NAN : r * fabsf(r);
}

// Slopes of gated projections.  What the backward pass needs of a result h = act(g) u is dh/dg = u act'(g) and dh/du = act(g).
// bf16: 16 bits each, the fp16 roots of their magnitudes with their signs: a slope is within 2^-10 of itself from 4e-9 to 65504^2 (in larger steps down to
// 2^-50, 0 below), where bf16 would add 2^-8 to what dz is rounded by.  Above, where the root is over what fp16 holds, fp16's 1024 words for infinity and NaN are 1022
// numbers in equal ratios up to 2^128, within 3.4 %, and those two: so that a slope is infinite where it is, and not the whole gradient with it.
// fp16: the first 24 bits of fp32, within 2^-16; 16 bits of them in one plane, eight in another behind it.  Slopes in fp16 as they are
// would add as much as dz is rounded by: dx and dw sqrt 3 as far from 64 bits as their own rounding, with these sqrt 2.
template <class T>
struct GatedSlopes {
    static constexpr bool kLow = std::is_same<T, F16>::value;
    uint16_t* high;             // M x 2 N
    uint8_t* low;               // M x 2 N, kLow only
    __device__ __forceinline__ GatedSlopes(uint16_t* p, int64_t M, int64_t N) : high(p), low(reinterpret_cast<uint8_t*>(p + M * 2 * N)) {}

    static constexpr float kMostRoot = 65504.0f * 65504.0f;
    static constexpr uint32_t kLarge = 0x7C00u, kInfinite = 0x7FFEu, kNaN = 0x7FFFu;
    static constexpr float kRatio = 96.0f / 1022.0f;         // of an octave from 2^32 on
    __device__ static __forceinline__ uint32_t large_word(float s) {
        const float f = fabsf(s), at = (__builtin_amdgcn_logf(f) - 32.0f) * (1.0f / kRatio);
        const uint32_t finite = kLarge + static_cast<uint32_t>(fminf(fmaxf(at, 0.0f), 1021.0f));
        return (__float_as_uint(s) >> 16 & 0x8000u) | (s != s ? kNaN : f == INFINITY ? kInfinite : finite);
    }
    __device__ static __forceinline__ float large_slope(uint32_t w) {
        const uint32_t word = w & 0x7FFFu;
        const float f = __builtin_amdgcn_exp2f(fmaf(static_cast<float>(word - kLarge) + 0.5f, kRatio, 32.0f));
        return word == kNaN ? NAN : copysignf(word == kInfinite ? INFINITY : f, __uint_as_float(w << 16));
    }
    // Whether one of eight slopes of each kind may have no root in fp16.
    __device__ static __forceinline__ bool some_large(const float* s, const float* t) {
        if (kLow) return false;
        float all[2] = {0.0f, 0.0f};                     // NaN where one is
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            all[0] += fabsf(s[v]);
            all[1] += fabsf(t[v]);
        }
        return !(all[0] + all[1] < kMostRoot);
    }
    // A slope's word of 24 bits, the last eight of them `low`; large ones' are put in its place afterwards.
    __device__ static __forceinline__ uint32_t word(float s) {
        if (!kLow) return static_cast<uint32_t>(F16::down(copysignf(__builtin_amdgcn_sqrtf(fabsf(s)), s))) << 8;
        const uint32_t bits = __float_as_uint(s);
        return s != s ? bits >> 8 | 0x4000u : (bits + 0x80u) >> 8;       // the largest round to infinity
    }
    // ... one after the other: this is code that few calls come to, and must not be long beside what all of them run.
    __device__ __forceinline__ void put_large(const float* s, const float* t, int64_t i, int64_t j, int64_t N, int n) const {
        uint32_t large = 0;
#pragma unroll
        for (int v = 0; v < 8; ++v) large |= (fabsf(s[v]) < kMostRoot ? 0u : 1u << v) | (fabsf(t[v]) < kMostRoot ? 0u : 256u << v);
        large &= 257u * ((1u << n) - 1u);
#pragma unroll 1
        for (; large; large &= large - 1) {
            const int which = __builtin_ctz(large);
            float f = 0.0f;
#pragma unroll
            for (int v = 0; v < 8; ++v) f = which == v ? s[v] : which == v + 8 ? t[v] : f;
            high[(2 * i + (which >> 3)) * N + j + (which & 7)] = static_cast<uint16_t>(large_word(f));
        }
    }
    // Words of large slopes: bit 15 or 31.
    __device__ static __forceinline__ uint32_t large_in(v4u high) {
        uint32_t of = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) of |= (high[i] & 0x7C007C00u) + 0x04000400u;
        return of;
    }
    // Eight slopes from their high and low parts.  large: of all lanes, whether there may be a large one.
    __device__ static __forceinline__ void slopes(v4u high, v2u low, bool large, float* s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t h = high[i / 2] >> (16 * (i % 2)) & 0xFFFFu;
            if (kLow) {
                s[i] = __uint_as_float(h << 16 | (low[i / 4] >> (8 * (i % 4)) & 255u) << 8);
            } else {
                const float r = F16::up(static_cast<uint16_t>(h));
                s[i] = r * fabsf(r);
            }
        }
        if (kLow || !large) return;
        uint32_t at = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) at |= (high[i / 2] >> (16 * (i % 2)) & kLarge) == kLarge ? 1u << i : 0u;
#pragma unroll 1
        for (; at; at &= at - 1) {
            const int which = __builtin_ctz(at);
            const uint32_t pair = which < 4 ? (which < 2 ? high.x : high.y) : (which < 6 ? high.z : high.w);
            const float f = large_slope(pair >> (16 * (which & 1)));
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = which == i ? f : s[i];
        }
    }
};

// How a product is cut: tiles of side x side (0: columns, dense_narrow.hpp), `splits` parts of k whose sums are joined afterwards.
struct DensePlan {
    int side;
    int splits;
};

// Columns of a block of the kernel for few rows with k outer: lines of 128 bytes where that leaves a block for every compute unit.
inline int64_t narrow_columns(int64_t I, int64_t J) { return I <= 16 && J >= 64 * 256 ? 64 : 32; }

// Dynamic LDS over 64 KB for a kernel, on the current device; `done`: the kernel's own.
inline hipError_t allow_lds(std::atomic<uint64_t>& done, const void* kernel, int bytes) {
    int device = -1;
    const hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    return once_a_device(done, device, hipSuccess, [&] { return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
}

// Whether a product goes to the kernel for few rows, how it is cut, and copies of operands whose rows are no whole pieces (kernels_dense.hip).
bool few_rows(int64_t I, int64_t J, int64_t K, bool b_outer, bool b_whole);
DensePlan plan_of(int64_t I, int64_t J, int64_t K, bool few, bool direct);
bool whole_pieces(const void* p, int64_t ld, int64_t inner);
bool worth_packing(int64_t I, int64_t J, int64_t K);
int64_t packed_bytes(int64_t rows, int64_t inner);
// rows x inner at `from` to rows of ldto elements at `to`, whole pieces with zeros at their ends; up to kMostPacks of them in a launch
struct PackJob {
    const void* from;
    int64_t ld;
    void* to;
    int64_t ldto, rows, inner;
};
constexpr int kMostPacks = 3;
void launch_pack(const PackJob* job, int jobs, hipStream_t s);

// Strips that a pass over dy sums by itself (256 rows each, as many as 64: with N = 8192 four blocks for a compute unit), and their sums.
int strips_of(int64_t M);
template <class T>
void launch_dense_db(const double* sums, int strips, int64_t N, void* db, hipStream_t s);

template <class T>
hipError_t launch_dense_tiles(const DenseGemm& g, const DensePlan& p, hipStream_t s);

template <class T>
hipError_t launch_low_tiles(const DenseGemm& g, const DensePlan& p, hipStream_t s);
template <class T>
hipError_t launch_gated_tiles(const DenseGemm& g, const DensePlan& p, hipStream_t s);

}  // namespace adpsgd_impl
