// Which kernel a gated projection goes to; instantiated once for each type (kernels_gated_bf16.hip, kernels_gated_f16.hip: compiled side by side).
#pragma once

#include "dense_large.hpp"
#include "gated_narrow.hpp"

namespace adpsgd_impl {
namespace {

template <class T, bool kBOuter>
hipError_t launch_gated_of(const DenseGemm& g, const DensePlan& p, hipStream_t s) {
    if (p.side == 256) return launch_large<T, false, kBOuter, 256, true>(g, p.splits, s);
    if (p.side == 128) return launch_large<T, false, kBOuter, 128, true>(g, p.splits, s);
    return launch_tile<T, false, kBOuter, 64, 4, 1, true>(g, p.splits, s);
}

}  // namespace

// The products of the backward pass with dz in two parts.
template <class T>
hipError_t launch_low_tiles(const DenseGemm& g, const DensePlan& p, hipStream_t s) {
    const hipError_t e = g.b_low     ? launch_tile<T, true, true, 64, 2, 2, false, 2>(g, p.splits, s)       // dw as in x 2 N: dz is the right operand
                         : g.a_outer ? launch_tile<T, true, true, 64, 2, 2, false, 1>(g, p.splits, s)
                         : g.b_outer ? launch_tile<T, false, true, 64, 2, 2, false, 1>(g, p.splits, s)
                                     : launch_tile<T, false, false, 64, 2, 2, false, 1>(g, p.splits, s);
    if (e != hipSuccess) return e;
    if (p.splits > 1)
        hipLaunchKernelGGL(dense_join_kernel<T>, dim3(static_cast<uint32_t>((g.I * ((g.J + 7) / 8) + 255) / 256)), dim3(256), 0, s, g, p.splits);
    return hipGetLastError();
}

template <class T>
hipError_t launch_gated_tiles(const DenseGemm& g, const DensePlan& p, hipStream_t s) {
    const hipError_t e = p.side == 0 ? launch_gated_narrow<T>(g, p.splits, s) : g.b_outer ? launch_gated_of<T, true>(g, p, s) : launch_gated_of<T, false>(g, p, s);
    if (e != hipSuccess) return e;
    if (p.splits > 1)
        hipLaunchKernelGGL(gated_join_kernel<T>, dim3(static_cast<uint32_t>((g.I * ((g.J + 7) / 8) + 255) / 256)), dim3(256), 0, s, g, p.splits);
    return hipGetLastError();
}

}  // namespace adpsgd_impl
