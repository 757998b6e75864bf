// The three element types of rows, 16 bytes at a time: unpacked to 32 bits and rounded from there.
#pragma once

#include "device_common.hpp"
#include "operators.hpp"

namespace adpsgd_impl {
namespace {

typedef v4u v4u_any __attribute__((aligned(2)));       // 16 bytes at any multiple of an element

struct F32 {
    using Raw = float;
    static constexpr int kN = 4;
    __device__ static float get(const Raw* p) { return *p; }
    __device__ static void unpack(v4u v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    __device__ static v4u pack(const float* f) {
        return v4u{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
    __device__ static void put(Raw* p, float f) { *p = f; }
};
struct Bf16 {
    using Raw = uint16_t;
    static constexpr int kN = 8;
    __device__ static float get(const Raw* p) { return bf16_to_float(*p); }
    __device__ static void unpack(v4u v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        }
    }
    __device__ static v4u pack(const float* f) {
        typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
        v4u v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, v2bf{static_cast<__bf16>(f[2 * i]), static_cast<__bf16>(f[2 * i + 1])});
        return v;
    }
    __device__ static void put(Raw* p, float f) { *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
};
struct F16 {
    using Raw = uint16_t;
    static constexpr int kN = 8;
    typedef _Float16 v2hf __attribute__((ext_vector_type(2)));
    __device__ static float get(const Raw* p) { return static_cast<float>(__builtin_bit_cast(_Float16, *p)); }
    __device__ static void unpack(v4u v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2hf h = __builtin_bit_cast(v2hf, static_cast<uint32_t>(v[i]));
            f[2 * i] = static_cast<float>(h.x);
            f[2 * i + 1] = static_cast<float>(h.y);
        }
    }
    __device__ static v4u pack(const float* f) {
        v4u v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, v2hf{static_cast<_Float16>(f[2 * i]), static_cast<_Float16>(f[2 * i + 1])});
        return v;
    }
    __device__ static void put(Raw* p, float f) { *p = __builtin_bit_cast(uint16_t, static_cast<_Float16>(f)); }
};

}  // namespace
}  // namespace adpsgd_impl
