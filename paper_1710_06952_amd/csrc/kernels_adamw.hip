// AdamW over all tensors of a model in one launch, or two where the gradients are clipped by their global norm.
//
//   g' = f g;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2;  u = (m / c1) / (sqrt(v / c2) + eps);  p = p - lr (u + wd p)
//
// A table cuts the tensors into chunks of 4096 elements, one thread block each: a model of many small tensors is one grid, as a
// single large tensor is.  A wavefront takes 256 consecutive elements at a time, four a lane, which is the block of elements that
// shares an exponent where the state has 8 bits: its largest magnitude is a reduction over the wavefront.
//
// Bound: memory, 28 bytes an element with everything in 32 bits (gradient 4, parameter 8, moments 16), 16 with bf16 parameters and
// gradients, fp32 masters and 8-bit moments.  With clipping the gradients are read once more before that, by adamw_norm_kernel.
//
// 8 bits.  A block's scale is 2^k, so that its largest value y 2^k has 128 <= y < 256 (k >= -50).  The codes are e4m3, not
// negative: between two neighbours lo and hi the share of the way is
//   for m     (y - lo) / (hi - lo)               the bits of y below the third of its fraction, so rounding up is an addition
//   for v     (v - lo^2) / (hi^2 - lo^2)         in units of 4^k: what is kept is the root, and v keeps its mean
// and hi is taken where share + (word + 1/2) / 2^16 >= 1, with 16 bits of a counter generator's word for each.  v > 0 is never
// rounded to 0, so a direction is never divided by eps alone.
#include <algorithm>

#include "device_common.hpp"
#include "operators.hpp"

namespace adpsgd_impl {
namespace {

constexpr int kT = 256;
constexpr int kPerThread = 4;                                     // consecutive elements
constexpr int kTurns = kAdamwChunk / (kT * kPerThread);
constexpr uint32_t kStreamMoments = 3u << 24;

typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t v4h_any __attribute__((ext_vector_type(4), aligned(2)));

struct TypeF32 {
    using Raw = float;
    __device__ static v4f load4(const void* p, int64_t at) { return *reinterpret_cast<const v4f_any*>(static_cast<const float*>(p) + at); }
    __device__ static void store4(void* p, int64_t at, v4f x) { *reinterpret_cast<v4f_any*>(static_cast<float*>(p) + at) = x; }
    __device__ static float load(const void* p, int64_t at) { return static_cast<const float*>(p)[at]; }
    __device__ static void store(void* p, int64_t at, float x) { static_cast<float*>(p)[at] = x; }
};
struct TypeBf16 {
    __device__ static v4f load4(const void* p, int64_t at) {
        const v4h_any h = *reinterpret_cast<const v4h_any*>(static_cast<const uint16_t*>(p) + at);
        return v4f{bf16_to_float(h.x), bf16_to_float(h.y), bf16_to_float(h.z), bf16_to_float(h.w)};
    }
    __device__ static void store4(void* p, int64_t at, v4f x) {
        *reinterpret_cast<v4h_any*>(static_cast<uint16_t*>(p) + at) = v4h_any{bf16_rne(x.x), bf16_rne(x.y), bf16_rne(x.z), bf16_rne(x.w)};
    }
    __device__ static float load(const void* p, int64_t at) { return bf16_to_float(static_cast<const uint16_t*>(p)[at]); }
    __device__ static void store(void* p, int64_t at, float x) { static_cast<uint16_t*>(p)[at] = bf16_rne(x); }
};
struct TypeF16 {
    __device__ static float up(uint16_t h) { return static_cast<float>(__builtin_bit_cast(_Float16, h)); }
    __device__ static uint16_t down(float x) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x)); }
    __device__ static v4f load4(const void* p, int64_t at) {
        const v4h_any h = *reinterpret_cast<const v4h_any*>(static_cast<const uint16_t*>(p) + at);
        return v4f{up(h.x), up(h.y), up(h.z), up(h.w)};
    }
    __device__ static void store4(void* p, int64_t at, v4f x) {
        *reinterpret_cast<v4h_any*>(static_cast<uint16_t*>(p) + at) = v4h_any{down(x.x), down(x.y), down(x.z), down(x.w)};
    }
    __device__ static float load(const void* p, int64_t at) { return up(static_cast<const uint16_t*>(p)[at]); }
    __device__ static void store(void* p, int64_t at, float x) { static_cast<uint16_t*>(p)[at] = down(x); }
};

// Four elements from `at` on of a tensor that ends at n; 0 beyond.
template <class T>
__device__ __forceinline__ v4f load_up_to(const void* p, int64_t at, int64_t n) {
    if (at + 4 <= n) return T::load4(p, at);
    v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < n) x[i] = T::load(p, at + i);
    return x;
}
template <class T>
__device__ __forceinline__ void store_up_to(void* p, int64_t at, int64_t n, v4f x) {
    if (at + 4 <= n) {
        T::store4(p, at, x);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < n) T::store(p, at + i, x[i]);
}

// ---- e4m3 codes and exponents ----
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
    return x;
}
__device__ __forceinline__ float finite_or_0(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.0f; }
__device__ __forceinline__ float largest(v4f x) {
    return fmaxf(fmaxf(finite_or_0(x.x), finite_or_0(x.y)), fmaxf(finite_or_0(x.z), finite_or_0(x.w)));
}
// floor(log2 x), x finite and not negative; -1 for 0
__device__ __forceinline__ int exponent_of(float x) { return x > 0.0f ? __builtin_amdgcn_frexp_expf(x) - 1 : -1; }
__device__ __forceinline__ int scale_exponent(int top) { return (top < -43 ? -43 : top) - 7; }
constexpr uint32_t kNanCode = 0x7F;

// e4m3 code of y, 0 <= y < 256, rounded up where its share of the way to the next code and (word + 1/2) / 2^16 come to one
__device__ __forceinline__ uint32_t code_up(float y, uint32_t word) {
    const bool low = y < 0x1p-6f;                       // no exponent of their own: shifted to where the steps are the same
    const uint32_t bits = __float_as_uint(low ? y + 0x1p-6f : y) + (word << 4) + 8u;
    return (bits >> 20) - (low ? 121u << 3 : 120u << 3);
}
__device__ __forceinline__ float value_of(uint32_t code) { return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(code), 0); }
__device__ __forceinline__ uint32_t moment_code(float m, int k, uint32_t word) {
    const uint32_t sign = __float_as_uint(m) >> 31 << 7;
    const uint32_t code = code_up(ldexpf(fabsf(m), -k), word);
    return sign | (fabsf(m) < INFINITY ? code : kNanCode);
}
__device__ __forceinline__ uint32_t square_code(float v, int k, uint32_t word) {
    const float y2 = ldexpf(v, -2 * k);
    const float y = sqrtf(y2);
    const bool low = y < 0x1p-6f;
    const uint32_t below = (__float_as_uint(low ? y + 0x1p-6f : y) >> 20) - (low ? 121u << 3 : 120u << 3);
    const float lo = value_of(below), hi = value_of(below + 1);
    const float way = hi * hi - lo * lo, up = (static_cast<float>(word) + 0.5f) * 0x1p-16f;
    uint32_t code = below + ((y2 - lo * lo) + up * way >= way ? 1u : 0u);
    code = v > 0.0f && code == 0u ? 1u : code;
    return v < INFINITY ? code : kNanCode;              // NaN too
}
// The values of four codes, times 2^k.
__device__ __forceinline__ v4f moments_of(uint32_t codes, int k) {
    return v4f{ldexpf(__builtin_amdgcn_cvt_f32_fp8(codes, 0), k), ldexpf(__builtin_amdgcn_cvt_f32_fp8(codes, 1), k),
               ldexpf(__builtin_amdgcn_cvt_f32_fp8(codes, 2), k), ldexpf(__builtin_amdgcn_cvt_f32_fp8(codes, 3), k)};
}
__device__ __forceinline__ v4f squares_of(uint32_t codes, int k) {
    v4f v = moments_of(codes, 0);
    v *= v;                                             // exact: 8 bits
    return v4f{ldexpf(v.x, 2 * k), ldexpf(v.y, 2 * k), ldexpf(v.z, 2 * k), ldexpf(v.w, 2 * k)};
}
// What a wavefront keeps of 256 moments: codes of its lanes' four, and the exponents.
struct Kept {
    uint32_t m, v;
    int km, kv;
};
__device__ __forceinline__ Kept kept_of(v4f m, v4f v, v4u words) {
    Kept k;
    k.km = scale_exponent(exponent_of(wave_max(largest(m))));
    const float top = wave_max(largest(v));
    k.kv = scale_exponent(top > 0.0f ? exponent_of(top) >> 1 : -1);     // floor(log2 sqrt v)
    k.m = k.v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k.m |= moment_code(m[i], k.km, words[i] >> 16) << (8 * i);
        k.v |= square_code(v[i], k.kv, words[i] & 0xFFFFu) << (8 * i);
    }
    return k;
}

// ---- the norm ----
// Sums of squares in 64 bits, block by block and then by the last block, in an order that the sizes give.
template <class G>
__global__ __launch_bounds__(kT) void adamw_norm_kernel(const AdamwArgs a) {
    __shared__ double at[kT / 64];
    __shared__ uint32_t turn;
    double sum = 0.0;
    for (int64_t c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
        const AdamwChunk chunk = a.chunks[c];
        const AdamwTensor& t = a.tensors[chunk.tensor];
        const int64_t first = static_cast<int64_t>(chunk.index) * kAdamwChunk + threadIdx.x * kPerThread;
        v4f g[kTurns];
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            const int64_t e = first + u * kT * kPerThread;
            g[u] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            if (e < t.n) g[u] = load_up_to<G>(t.g, e, t.n);
        }
#pragma unroll
        for (int u = 0; u < kTurns; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = fma(static_cast<double>(g[u][i]), static_cast<double>(g[u][i]), sum);
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kT / 64; ++w) sum += at[w];
        __hip_atomic_store(a.norm_parts + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        turn = count_done(a.ticket);
    }
    __syncthreads();
    if (turn + 1 != gridDim.x) return;
    sum = 0.0;
    for (uint32_t b = threadIdx.x; b < gridDim.x; b += kT) sum += __hip_atomic_load(a.norm_parts + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kT / 64; ++w) sum += at[w];
        const double norm = sqrt(sum) * fabs(static_cast<double>(a.grad_scale));
        const double f = a.max_norm / (norm + 1e-6);
        *a.norm = static_cast<float>(norm);
        *a.factor = static_cast<float>(f > 1.0 ? 1.0 : f);           // NaN stays
        *a.ticket = 0;                                               // for the next step
    }
}

// ---- the step ----
template <class P, class G, bool kBytes, bool kMaster, bool kDirection>
__global__ __launch_bounds__(kT) void adamw_step_kernel(const AdamwArgs a) {
    const AdamwChunk chunk = a.chunks[blockIdx.x];
    const AdamwTensor t = a.tensors[chunk.tensor];
    const float f = a.max_norm > 0.0 ? *a.factor : 1.0f;
    const int64_t first = static_cast<int64_t>(chunk.index) * kAdamwChunk + threadIdx.x * kPerThread;
    v4f g[kTurns], p[kTurns], m32[kTurns], v32[kTurns];
    uint32_t m8[kTurns], v8[kTurns];
    int km[kTurns], kv[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int64_t e = first + u * kT * kPerThread;
        const int64_t at = t.state + e;                   // the state is whole blocks of 256: no end inside four elements
        if (e < (t.n + kAdamwBlock - 1) / kAdamwBlock * kAdamwBlock) {      // uniform over a wavefront
            if (kBytes) {
                m8[u] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.m) + at);
                v8[u] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.v) + at);
                const uint16_t k = *reinterpret_cast<const uint16_t*>(a.exponents + 2 * (at / kAdamwBlock));
                km[u] = static_cast<int8_t>(k & 0xFF);
                kv[u] = static_cast<int8_t>(k >> 8);
            } else {
                m32[u] = *reinterpret_cast<const v4f*>(static_cast<const float*>(a.m) + at);
                v32[u] = *reinterpret_cast<const v4f*>(static_cast<const float*>(a.v) + at);
            }
            g[u] = load_up_to<G>(t.g, e, t.n);
            p[u] = kMaster ? load_up_to<TypeF32>(t.master, e, t.n) : load_up_to<P>(t.p, e, t.n);
        }
    }
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int64_t e = first + u * kT * kPerThread;
        const int64_t at = t.state + e;
        if (e >= (t.n + kAdamwBlock - 1) / kAdamwBlock * kAdamwBlock) continue;
        v4f m = kBytes ? moments_of(m8[u], km[u]) : m32[u], v = kBytes ? squares_of(v8[u], kv[u]) : v32[u], q;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float gi = g[u][i] * a.grad_scale * f;
            m[i] = fmaf(a.beta1, m[i], a.rest1 * gi);
            v[i] = fmaf(a.beta2, v[i], a.rest2 * gi * gi);
            const float dir = m[i] * a.inv_c1 / (sqrtf(v[i] * a.inv_c2) + a.eps) + t.decay * p[u][i];
            q[i] = kDirection ? dir : p[u][i] - a.lr * dir;
        }
        if (kDirection) {
            store_up_to<TypeF32>(t.out, e, t.n, q);
        } else {
            if (kMaster) store_up_to<TypeF32>(t.master, e, t.n, q);
            store_up_to<P>(t.p, e, t.n, q);
        }
        if (kBytes) {
            const uint64_t lane = static_cast<uint64_t>(at) / 4;
            const v4u words = philox4x32_rounds<10>(static_cast<uint32_t>(lane), static_cast<uint32_t>(lane >> 32), static_cast<uint32_t>(a.step),
                                                    (static_cast<uint32_t>(a.step >> 32) & 0x00FFFFFFu) | kStreamMoments,
                                                    philox_keys<10>(static_cast<uint32_t>(a.seed), static_cast<uint32_t>(a.seed >> 32)));
            const Kept k = kept_of(m, v, words);
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.m) + at) = k.m;
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.v) + at) = k.v;
            if ((threadIdx.x & 63) == 0)
                *reinterpret_cast<uint16_t*>(a.exponents + 2 * (at / kAdamwBlock)) = static_cast<uint16_t>((k.km & 0xFF) | (k.kv & 0xFF) << 8);
        } else {
            *reinterpret_cast<v4f*>(static_cast<float*>(a.m) + at) = m;
            *reinterpret_cast<v4f*>(static_cast<float*>(a.v) + at) = v;
        }
    }
}

// ---- the state in 8 bits from and to values; grid: ceil(length / 1024) ----
__global__ __launch_bounds__(kT) void adamw_get_kernel(const uint8_t* m, const uint8_t* v, const int8_t* exponents, int64_t length, uint16_t* m_out, uint16_t* v_out) {
    const int64_t at = 4 * (static_cast<int64_t>(blockIdx.x) * kT + threadIdx.x);
    if (at >= length) return;
    const int8_t* k = exponents + 2 * (at / kAdamwBlock);
    const v4f x = moments_of(*reinterpret_cast<const uint32_t*>(m + at), k[0]), y = squares_of(*reinterpret_cast<const uint32_t*>(v + at), k[1]);
    TypeBf16::store4(m_out, at, x);
    TypeBf16::store4(v_out, at, y);
}
__global__ __launch_bounds__(kT) void adamw_set_kernel(const float* m, const float* v, int64_t length, uint8_t* m_out, uint8_t* v_out, int8_t* exponents) {
    const int64_t at = 4 * (static_cast<int64_t>(blockIdx.x) * kT + threadIdx.x);
    if (at >= length) return;                            // whole wavefronts: the length is a multiple of 256
    const v4u half = {0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu};      // (word + 1/2) / 2^16 just under 1/2: to the nearest
    const Kept k = kept_of(TypeF32::load4(m, at), TypeF32::load4(v, at), half);
    *reinterpret_cast<uint32_t*>(m_out + at) = k.m;
    *reinterpret_cast<uint32_t*>(v_out + at) = k.v;
    if ((threadIdx.x & 63) == 0) {
        exponents[2 * (at / kAdamwBlock)] = static_cast<int8_t>(k.km);
        exponents[2 * (at / kAdamwBlock) + 1] = static_cast<int8_t>(k.kv);
    }
}

template <class P, class G>
void launch_step_of(const AdamwArgs& a, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>(a.n_chunks));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kT), 0, s, a); };
    const int form = (a.bits == 8 ? 4 : 0) | (a.masters ? 2 : 0) | (a.direction ? 1 : 0);
    switch (form) {
        case 0: go(adamw_step_kernel<P, G, false, false, false>); break;
        case 1: go(adamw_step_kernel<P, G, false, false, true>); break;
        case 2: go(adamw_step_kernel<P, G, false, true, false>); break;
        case 3: go(adamw_step_kernel<P, G, false, true, true>); break;
        case 4: go(adamw_step_kernel<P, G, true, false, false>); break;
        case 5: go(adamw_step_kernel<P, G, true, false, true>); break;
        case 6: go(adamw_step_kernel<P, G, true, true, false>); break;
        case 7: go(adamw_step_kernel<P, G, true, true, true>); break;
    }
}
template <class P>
void launch_step(const AdamwArgs& a, hipStream_t s) {
    if (a.grad_type == ADPSGD_TYPE_F32) launch_step_of<P, TypeF32>(a, s);
    else if (a.grad_type == ADPSGD_TYPE_BF16) launch_step_of<P, TypeBf16>(a, s);
    else launch_step_of<P, TypeF16>(a, s);
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, hipStream_t s) {
    if (a.max_norm > 0.0) {
        const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(std::max<int64_t>(a.n_chunks, 1), kAdamwNormBlocks)));
        if (a.grad_type == ADPSGD_TYPE_F32) hipLaunchKernelGGL(adamw_norm_kernel<TypeF32>, grid, dim3(kT), 0, s, a);
        else if (a.grad_type == ADPSGD_TYPE_BF16) hipLaunchKernelGGL(adamw_norm_kernel<TypeBf16>, grid, dim3(kT), 0, s, a);
        else hipLaunchKernelGGL(adamw_norm_kernel<TypeF16>, grid, dim3(kT), 0, s, a);
    }
    if (a.n_chunks > 0) {
        if (a.param_type == ADPSGD_TYPE_F32) launch_step<TypeF32>(a, s);
        else if (a.param_type == ADPSGD_TYPE_BF16) launch_step<TypeBf16>(a, s);
        else launch_step<TypeF16>(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_adamw_get(const void* m, const void* v, const int8_t* exponents, int64_t length, uint16_t* m_out, uint16_t* v_out, hipStream_t s) {
    if (length > 0)
        hipLaunchKernelGGL(adamw_get_kernel, dim3(static_cast<uint32_t>((length + 4 * kT - 1) / (4 * kT))), dim3(kT), 0, s, static_cast<const uint8_t*>(m),
                           static_cast<const uint8_t*>(v), exponents, length, m_out, v_out);
    return hipGetLastError();
}
hipError_t launch_adamw_set(const float* m, const float* v, int64_t length, void* m_out, void* v_out, int8_t* exponents, hipStream_t s) {
    if (length > 0)
        hipLaunchKernelGGL(adamw_set_kernel, dim3(static_cast<uint32_t>((length + 4 * kT - 1) / (4 * kT))), dim3(kT), 0, s, m, v, length,
                           static_cast<uint8_t*>(m_out), static_cast<uint8_t*>(v_out), exponents);
    return hipGetLastError();
}

}  // namespace adpsgd_impl
