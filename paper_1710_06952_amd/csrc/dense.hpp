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

template <class T>
hipError_t launch_dense_tiles(const DenseGemm& g, const DensePlan& p, hipStream_t s);

}  // namespace adpsgd_impl
