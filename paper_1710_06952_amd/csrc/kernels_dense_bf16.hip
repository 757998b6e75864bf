// The tiled products of dense layers in one of their types (dense_tiles.hpp).
#include "dense_tiles.hpp"

namespace adpsgd_impl {

template void launch_dense_tiles<Bf16>(const DenseGemm& g, const DensePlan& p, hipStream_t s);

}  // namespace adpsgd_impl
