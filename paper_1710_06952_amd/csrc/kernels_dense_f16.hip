// The products of dense layers in float16.
#include "dense_launch.hpp"

namespace adpsgd_impl {

template hipError_t launch_dense_tiles<F16>(const DenseGemm& g, const DensePlan& p, hipStream_t s);

}  // namespace adpsgd_impl
