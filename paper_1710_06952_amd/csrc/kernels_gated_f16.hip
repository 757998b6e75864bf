// Gated projections in float16.
#include "gated_launch.hpp"

namespace adpsgd_impl {

template hipError_t launch_low_tiles<F16>(const DenseGemm& g, const DensePlan& p, hipStream_t s);
template hipError_t launch_gated_tiles<F16>(const DenseGemm& g, const DensePlan& p, hipStream_t s);

}  // namespace adpsgd_impl
