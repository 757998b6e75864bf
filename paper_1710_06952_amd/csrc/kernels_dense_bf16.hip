// The products of dense layers in bfloat16.
#include "dense_launch.hpp"

namespace adpsgd_impl {

template hipError_t launch_dense_tiles<Bf16>(const DenseGemm& g, const DensePlan& p, hipStream_t s);

}  // namespace adpsgd_impl
