// AdamW over all tensors of a model in one launch, or two where the gradients are clipped by their global norm.
//
//   g' = f g;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2;  u = (m / c1) / (sqrt(v / c2) + eps);  p = p - lr (u + wd p)
//
// A table cuts the tensors into chunks of up to 4096 elements, one thread block each: a model of many small tensors is one grid, as a
// single large tensor is.  A whole chunk has no condition in front of its loads, so that all are on their way at once.  A wavefront
// takes 256 consecutive elements at a time, four a lane, which is the block of elements that shares an exponent where the state has 8
// bits: its largest magnitude is a reduction over the wavefront.
//
// Bound: memory, 28 bytes an element with everything in 32 bits (gradient 4, parameter 8, moments 16), 16 with bf16 parameters and
// gradients, fp32 masters and 8-bit moments.  With clipping the gradients are read once more before that, by adamw_norm_kernel.
// Measured: 25.6 M parameters in 32 bits 118 us (6.1 TB/s) and 16 + 5 for the norm; 67 M with 8-bit moments 190 to 240 us (5.6 to 4.5 TB/s:
// 440 instructions for four elements a lane are as long as their bytes) and 28 + 5 for the norm.
//
// 8 bits.  A block's scale is 2^k, so that its largest value y 2^k has 128 <= y < 256 (k >= -50).  The codes are e4m3, not
// negative: between two neighbours lo and hi the share of the way is
//   for m     (y - lo) / (hi - lo)               the bits of y below the third of its fraction, so rounding up is an addition
//   for v     (v - lo^2) / (hi^2 - lo^2)         in units of 4^k: what is kept is the root, and v keeps its mean
// and hi is taken where share + (word + 1/2) / 2^16 >= 1, with 16 bits of a counter generator's word for each.  v > 0 is never
// rounded to 0, so a direction is never divided by eps alone.
#include <algorithm>
#include <type_traits>

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
    __device__ static v4f load4(const void* p, int64_t at) { return __builtin_nontemporal_load(reinterpret_cast<const v4f_any*>(static_cast<const float*>(p) + at)); }
    __device__ static void store4(void* p, int64_t at, v4f x) { __builtin_nontemporal_store(x, reinterpret_cast<v4f_any*>(static_cast<float*>(p) + at)); }
    __device__ static float load(const void* p, int64_t at) { return static_cast<const float*>(p)[at]; }
    __device__ static void store(void* p, int64_t at, float x) { static_cast<float*>(p)[at] = x; }
};
struct TypeBf16 {
    __device__ static v4f load4(const void* p, int64_t at) {
        const v4h_any h = *reinterpret_cast<const v4h_any*>(static_cast<const uint16_t*>(p) + at);
        return v4f{bf16_to_float(h.x), bf16_to_float(h.y), bf16_to_float(h.z), bf16_to_float(h.w)};
    }
    __device__ static void store4(void* p, int64_t at, v4f x) {
        __builtin_nontemporal_store(v4h_any{bf16_rne(x.x), bf16_rne(x.y), bf16_rne(x.z), bf16_rne(x.w)}, reinterpret_cast<v4h_any*>(static_cast<uint16_t*>(p) + at));
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

// Four elements from `at` on of n; beyond the end 0, or nothing.  kWhole: all of them are there.
template <class T, bool kWhole>
__device__ __forceinline__ v4f load_up_to(const void* p, int at, int n) {
    if (kWhole || at + 4 <= n) return T::load4(p, at);
    v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < n) x[i] = T::load(p, at + i);
    return x;
}
template <class T, bool kWhole>
__device__ __forceinline__ void store_up_to(void* p, int at, int n, v4f x) {
    if (kWhole || at + 4 <= n) {
        T::store4(p, at, x);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < n) T::store(p, at + i, x[i]);
}

// ---- e4m3 codes and exponents ----
// The largest of a wavefront's magnitudes, NaN if there is one, by moves between lanes of a row and between rows (no LDS).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_largest(v4f v) {
    float x = larger(larger(fabsf(v.x), fabsf(v.y)), larger(fabsf(v.z), fabsf(v.w)));
    auto with = [&](auto control) {
        const int moved = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(control)::value, 0xF, 0xF, false);
        x = larger(x, __builtin_bit_cast(float, moved));
    };
    with(std::integral_constant<int, 0x111>());          // one lane up, two, four, eight within rows of 16
    with(std::integral_constant<int, 0x112>());
    with(std::integral_constant<int, 0x114>());
    with(std::integral_constant<int, 0x118>());
    with(std::integral_constant<int, 0x142>());          // the last of a row to the next, of two rows to the others
    with(std::integral_constant<int, 0x143>());
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ v4f finite_or_0(v4f x) {
    return v4f{fabsf(x.x) < INFINITY ? x.x : 0.0f, fabsf(x.y) < INFINITY ? x.y : 0.0f, fabsf(x.z) < INFINITY ? x.z : 0.0f, fabsf(x.w) < INFINITY ? x.w : 0.0f};
}
// floor(log2 x), x finite and not negative; -1 for 0
__device__ __forceinline__ int exponent_of(float x) { return x > 0.0f ? __builtin_amdgcn_frexp_expf(x) - 1 : -1; }
__device__ __forceinline__ int scale_exponent(int top) { return (top < -43 ? -43 : top) - 7; }
constexpr uint32_t kNanCode = 0x7F;

__device__ __forceinline__ float value_of(uint32_t code) { return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(code), 0); }
// The draw decides by 2^-16 of a step, and a 32-bit m is off by up to 2^-20 of one: one element in a million would go the other way.
// So gradients are scaled and moments added in 64 bits here, of which the upper word is enough: 20 bits of fraction, 3 of them the code's, and what the other
// 17 come to with 2 word + 1 is the carry.
__device__ __forceinline__ uint32_t moment_code(double m, int k, uint32_t word) {
    const double y = __builtin_amdgcn_ldexp(fabs(m), -k);
    const bool low = y < 0x1p-6;                        // no exponent of their own: shifted to where the steps are the same
    const uint32_t bits = static_cast<uint32_t>(__builtin_bit_cast(uint64_t, low ? y + 0x1p-6 : y) >> 32) + 2 * word + 1;
    const uint32_t code = ((bits >> 17) - (low ? 1017u << 3 : 1016u << 3)) & 0x7Fu;
    const uint32_t sign = static_cast<uint32_t>(__builtin_bit_cast(uint64_t, m) >> 63) << 7;
    return sign | code;
}
// v finite and not negative: another one has no code of seven bits, and its upper bits would be those of the next element.
__device__ __forceinline__ uint32_t square_code(double v, int k, uint32_t word) {
    const double y2 = __builtin_amdgcn_ldexp(v, -2 * k);
    const float y = __builtin_amdgcn_sqrtf(static_cast<float>(y2));     // a step too far or too short is made good by the share
    const bool low = y < 0x1p-6f;
    const uint32_t below = (__float_as_uint(low ? y + 0x1p-6f : y) >> 20) - (low ? 121u << 3 : 120u << 3);
    const float lo = value_of(below), hi = value_of(below + 1);
    const float way = hi * hi - lo * lo, up = (static_cast<float>(word) + 0.5f) * 0x1p-16f;
    uint32_t code = below + (fmaf(up, way, static_cast<float>(y2 - static_cast<double>(lo * lo))) >= way ? 1u : 0u);
    return v > 0.0 && code == 0u ? 1u : code;
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
typedef double v4d __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v4f rounded(v4d x) {
    return v4f{static_cast<float>(x.x), static_cast<float>(x.y), static_cast<float>(x.z), static_cast<float>(x.w)};
}
// What a wavefront keeps of 256 moments: codes of its lanes' four, and the exponents.
struct Kept {
    uint32_t m, v;
    int km, kv;
};
// kAgain: the values may be what a state stood for, and are kept as they are then.  Its largest may be a code that was rounded up to 256; with
// the exponent one higher that 256 gives, the smallest codes of its block would not all be there.
template <bool kAgain>
__device__ __forceinline__ Kept kept_of(v4d m, v4d v, v4u words) {
    const v4f m32 = rounded(m), v32 = rounded(v);
    float top_m = wave_largest(m32), top_v = wave_largest(v32);
    const bool all_finite = top_m < INFINITY && top_v < INFINITY;       // uniform; else the others decide, and NaN is kept as its code
    if (!all_finite) {
        top_m = wave_largest(finite_or_0(m32));
        top_v = wave_largest(finite_or_0(v32));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!(v32[i] < INFINITY)) v[i] = 0.0;
    }
    Kept k;
    int em = exponent_of(top_m), ev = exponent_of(top_v);
    if (kAgain) {                                        // 2^n as if it were a little less
        if (top_m > 0.0f && ldexpf(1.0f, em) == top_m) --em;
        if (top_v > 0.0f && ldexpf(1.0f, ev) == top_v) --ev;
    }
    k.km = scale_exponent(em);
    k.kv = scale_exponent(top_v > 0.0f ? ev >> 1 : -1);     // floor(log2 sqrt v)
    if (top_v == 0.0f && __ballot(v[0] > 0.0 || v[1] > 0.0 || v[2] > 0.0 || v[3] > 0.0) != 0)
        k.kv = scale_exponent(-75);                      // squares that 32 bits do not hold are no block of zeros
    k.m = k.v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k.m |= moment_code(m[i], k.km, words[i] >> 16) << (8 * i);
        k.v |= square_code(v[i], k.kv, words[i] & 0xFFFFu) << (8 * i);
    }
    if (!all_finite) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!(fabsf(m32[i]) < INFINITY)) k.m |= kNanCode << (8 * i);
            if (!(v32[i] < INFINITY)) k.v |= kNanCode << (8 * i);
        }
    }
    return k;
}

// ---- the norm ----
// Sums of squares in 64 bits, block by block, then over the blocks, in an order that the sizes give.  The second sum is taken by a kernel of one
// block, or, where the blocks are few, by every block of the step itself (a launch less).  A last block that takes it, found by a
// counter that all blocks increment, cost 20 to 30 us with 1024 and 2048 of them.
__device__ __forceinline__ double block_sum(double x, double* at) {
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
    __syncthreads();
    x = at[0];
#pragma unroll
    for (int w = 1; w < kT / 64; ++w) x += at[w];
    return x;
}
// The gradients' norm and their factor from the blocks' sums, to all threads.
__device__ __forceinline__ double factor_of(const AdamwArgs& a, double* at, float& norm) {
    double sum = 0.0;
    for (int b = threadIdx.x; b < a.norm_blocks; b += kT) sum += a.norm_parts[b];
    const double of = sqrt(block_sum(sum, at)) * fabs(a.grad_scale_64), f = a.max_norm / (of + 1e-6);
    norm = static_cast<float>(of);
    return f > 1.0 ? 1.0 : f;                            // NaN stays
}
__global__ __launch_bounds__(kT) void adamw_factor_kernel(const AdamwArgs a) {
    __shared__ double at[kT / 64];
    float norm;
    const double f = factor_of(a, at, norm);
    if (threadIdx.x == 0) {
        *a.norm = norm;
        *a.factor = f;
    }
}
template <class G>
__global__ __launch_bounds__(kT) void adamw_norm_kernel(const AdamwArgs a) {
    __shared__ double at[kT / 64];
    double sum = 0.0;
    auto add = [&](const AdamwChunk& c, auto whole) {
        v4f g[kTurns];
#pragma unroll
        for (int u = 0; u < kTurns; ++u) g[u] = load_up_to<G, decltype(whole)::value>(c.g, (u * kT + static_cast<int>(threadIdx.x)) * kPerThread, c.n);
#pragma unroll
        for (int u = 0; u < kTurns; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = fma(static_cast<double>(g[u][i]), static_cast<double>(g[u][i]), sum);
    };
    if (blockIdx.x < a.n_chunks) {
        AdamwChunk next = a.chunks[blockIdx.x];
        for (int64_t c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
            const AdamwChunk chunk = next;
            if (c + gridDim.x < a.n_chunks) next = a.chunks[c + gridDim.x];
            if (chunk.n == kAdamwChunk) add(chunk, std::true_type());
            else add(chunk, std::false_type());
        }
    }
    sum = block_sum(sum, at);
    if (threadIdx.x == 0) a.norm_parts[blockIdx.x] = sum;
}

// ---- the step ----
// Root and quotient by v_sqrt_f32 and v_rcp_f32, within 2^-22.  v_sqrt_f32 takes a v under 2^-126 as 0, whose root an eps over 1e-18 does not feel;
// beside a smaller one v is taken times 2^30 and the root times 2^-15 (inv_c2 and root), which v up to 2^98 allow.
template <class P, class G, bool kBytes, bool kMaster, bool kDirection, bool kWhole>
__device__ __forceinline__ void step_chunk(const AdamwArgs& a, const AdamwChunk& t, double* sums) {
    const int first = static_cast<int>(threadIdx.x) * kPerThread, padded = (t.n + kAdamwBlock - 1) / kAdamwBlock * kAdamwBlock;
    v4f g[kTurns], p[kTurns], m32[kTurns], v32[kTurns];
    uint32_t m8[kTurns], v8[kTurns];
    uint16_t k8[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int e = first + u * kT * kPerThread;
        const int64_t at = t.state + e;                   // the state is whole blocks of 256: no end inside four elements
        if (kWhole || e < padded) {                       // uniform over a wavefront
            g[u] = load_up_to<G, kWhole>(t.g, e, t.n);
            p[u] = kMaster ? load_up_to<TypeF32, kWhole>(t.master, e, t.n) : load_up_to<P, kWhole>(t.p, e, t.n);
            if (kBytes) {
                m8[u] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.m) + at));
                v8[u] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.v) + at));
                k8[u] = *reinterpret_cast<const uint16_t*>(a.exponents + 2 * (at / kAdamwBlock));
            } else {
                m32[u] = __builtin_nontemporal_load(reinterpret_cast<const v4f*>(static_cast<const float*>(a.m) + at));
                v32[u] = __builtin_nontemporal_load(reinterpret_cast<const v4f*>(static_cast<const float*>(a.v) + at));
            }
        }
    }
    double f = 1.0;                                       // the loads are on their way
    if (a.max_norm > 0.0) {
        if (a.norm_blocks <= kT) {
            float norm;
            f = factor_of(a, sums, norm);
            if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
        } else {
            f = *a.factor;
        }
    }
    const float f32 = static_cast<float>(f);
    const double scale = a.grad_scale_64 * f;
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int e = first + u * kT * kPerThread;
        const int64_t at = t.state + e;
        if (!kWhole && e >= padded) continue;
        v4f m, v, q;
        v4d m64, v64;
        if (kBytes) {
            const v4f m_old = moments_of(m8[u], static_cast<int8_t>(k8[u] & 0xFF)), v_old = squares_of(v8[u], static_cast<int8_t>(k8[u] >> 8));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double gi = scale * static_cast<double>(g[u][i]);
                m64[i] = fma(a.beta1_64, static_cast<double>(m_old[i]), a.rest1_64 * gi);
                v64[i] = fma(a.beta2_64, static_cast<double>(v_old[i]), a.rest2_64 * gi * gi);
            }
            m = rounded(m64);
            v = rounded(v64);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float gi = g[u][i] * a.grad_scale * f32;
                m[i] = fmaf(a.beta1, m32[u][i], a.rest1 * gi);
                v[i] = fmaf(a.beta2, v32[u][i], a.rest2 * gi * gi);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float dir = m[i] * a.inv_c1 * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[i] * a.inv_c2), a.root, a.eps)) + t.decay * p[u][i];
            q[i] = kDirection ? dir : p[u][i] - a.lr * dir;
            asm volatile("" : "+v"(q[i]));                // rounded to 32 bits, as the master is, before the parameter's rounding
        }
        if (kDirection) {
            store_up_to<TypeF32, kWhole>(t.out, e, t.n, q);
        } else {
            if (kMaster) store_up_to<TypeF32, kWhole>(t.master, e, t.n, q);
            store_up_to<P, kWhole>(t.p, e, t.n, q);
        }
        if (kBytes) {
            const uint64_t lane = static_cast<uint64_t>(at) / 4;
            const v4u words = philox4x32_rounds<10>(static_cast<uint32_t>(lane), static_cast<uint32_t>(lane >> 32), static_cast<uint32_t>(a.step),
                                                    (static_cast<uint32_t>(a.step >> 32) & 0x00FFFFFFu) | kStreamMoments,
                                                    philox_keys<10>(static_cast<uint32_t>(a.seed), static_cast<uint32_t>(a.seed >> 32)));
            const Kept k = kept_of<false>(m64, v64, words);
            __builtin_nontemporal_store(k.m, reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.m) + at));
            __builtin_nontemporal_store(k.v, reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.v) + at));
            if ((threadIdx.x & 63) == 0)
                *reinterpret_cast<uint16_t*>(a.exponents + 2 * (at / kAdamwBlock)) = static_cast<uint16_t>((k.km & 0xFF) | (k.kv & 0xFF) << 8);
        } else {
            __builtin_nontemporal_store(m, reinterpret_cast<v4f*>(static_cast<float*>(a.m) + at));
            __builtin_nontemporal_store(v, reinterpret_cast<v4f*>(static_cast<float*>(a.v) + at));
        }
    }
}
template <class P, class G, bool kBytes, bool kMaster, bool kDirection>
__global__ __launch_bounds__(kT) void adamw_step_kernel(const AdamwArgs a) {
    __shared__ double sums[kT / 64];
    const AdamwChunk chunk = a.chunks[blockIdx.x];
    if (chunk.n == kAdamwChunk) step_chunk<P, G, kBytes, kMaster, kDirection, true>(a, chunk, sums);
    else step_chunk<P, G, kBytes, kMaster, kDirection, false>(a, chunk, sums);
}

// ---- the state in 8 bits from and to values; grid: ceil(length / 2048), ceil(length / 1024) ----
__global__ __launch_bounds__(kT) void adamw_get_kernel(const uint8_t* m, const uint8_t* v, const int8_t* exponents, int64_t length, uint16_t* m_out, uint16_t* v_out) {
    typedef uint16_t v8h_any __attribute__((ext_vector_type(8), aligned(2)));
    const int64_t at = 8 * (static_cast<int64_t>(blockIdx.x) * kT + threadIdx.x);
    if (at >= length) return;
    const int8_t* k = exponents + 2 * (at / kAdamwBlock);
    const uint64_t cm = *reinterpret_cast<const uint64_t*>(m + at), cv = *reinterpret_cast<const uint64_t*>(v + at);
    v8h_any x, y;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const v4f p = moments_of(static_cast<uint32_t>(cm >> (32 * h)), k[0]), q = squares_of(static_cast<uint32_t>(cv >> (32 * h)), k[1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[4 * h + i] = bf16_rne(p[i]);
            y[4 * h + i] = bf16_rne(q[i]);
        }
    }
    __builtin_nontemporal_store(x, reinterpret_cast<v8h_any*>(m_out + at));
    __builtin_nontemporal_store(y, reinterpret_cast<v8h_any*>(v_out + at));
}
__global__ __launch_bounds__(kT) void adamw_set_kernel(const float* m, const float* v, int64_t length, uint8_t* m_out, uint8_t* v_out, int8_t* exponents) {
    const int64_t at = 4 * (static_cast<int64_t>(blockIdx.x) * kT + threadIdx.x);
    if (at >= length) return;                            // whole wavefronts: the length is a multiple of 256
    const v4u half = {0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu};      // (word + 1/2) / 2^16 just under 1/2: to the nearest
    const v4f x = TypeF32::load4(m, at);
    v4f y = TypeF32::load4(v, at);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = y[i] < 0.0f ? NAN : y[i];         // what its root is
    const Kept k = kept_of<true>(v4d{x.x, x.y, x.z, x.w}, v4d{y.x, y.y, y.z, y.w}, half);
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

hipError_t launch_adamw(const AdamwArgs& args, hipStream_t s) {
    AdamwArgs a = args;
    if (a.max_norm > 0.0) {
        a.norm_blocks = static_cast<int32_t>(std::min<int64_t>(a.n_chunks, kAdamwNormBlocks));
        const dim3 grid(static_cast<uint32_t>(a.norm_blocks));
        if (a.n_chunks > 0) {
            if (a.grad_type == ADPSGD_TYPE_F32) hipLaunchKernelGGL(adamw_norm_kernel<TypeF32>, grid, dim3(kT), 0, s, a);
            else if (a.grad_type == ADPSGD_TYPE_BF16) hipLaunchKernelGGL(adamw_norm_kernel<TypeBf16>, grid, dim3(kT), 0, s, a);
            else hipLaunchKernelGGL(adamw_norm_kernel<TypeF16>, grid, dim3(kT), 0, s, a);
        }
        if (a.n_chunks == 0 || a.norm_blocks > kT) hipLaunchKernelGGL(adamw_factor_kernel, dim3(1), dim3(kT), 0, s, a);
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
        hipLaunchKernelGGL(adamw_get_kernel, dim3(static_cast<uint32_t>((length + 8 * kT - 1) / (8 * kT))), dim3(kT), 0, s, static_cast<const uint8_t*>(m),
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
