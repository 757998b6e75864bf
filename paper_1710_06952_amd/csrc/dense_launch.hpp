// Which kernel a product goes to; instantiated once for each type (kernels_dense_bf16.hip, kernels_dense_f16.hip: compiled side by side).
#pragma once

#include "dense_large.hpp"
#include "dense_narrow.hpp"

namespace adpsgd_impl {
namespace {

template <class T, bool kAOuter, bool kBOuter>
hipError_t launch_tiles_of(const DenseGemm& g, const DensePlan& p, hipStream_t s) {
    if (p.side == 256) return launch_large<T, kAOuter, kBOuter, 256>(g, p.splits, s);
    if (p.side == 128) return launch_large<T, kAOuter, kBOuter, 128>(g, p.splits, s);
    return launch_tile<T, kAOuter, kBOuter, 64, 2, 2>(g, p.splits, s);
}

}  // namespace

template <class T>
hipError_t launch_dense_tiles(const DenseGemm& g, const DensePlan& p, hipStream_t s) {
    hipError_t e = hipSuccess;
    if (p.side == 0) launch_narrow<T>(g, p.splits, s);
    else if (g.a_outer) e = launch_tiles_of<T, true, true>(g, p, s);
    else if (g.b_outer) e = launch_tiles_of<T, false, true>(g, p, s);
    else e = launch_tiles_of<T, false, false>(g, p, s);
    if (e != hipSuccess) return e;
    if (p.splits > 1)
        hipLaunchKernelGGL(dense_join_kernel<T>, dim3(static_cast<uint32_t>((g.I * ((g.J + 7) / 8) + 255) / 256)), dim3(256), 0, s, g, p.splits);
    return hipGetLastError();
}

}  // namespace adpsgd_impl
