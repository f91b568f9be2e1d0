// The products Z = X W: X along the contraction, W across it.  See dense_kernel.hpp.
#include "dense_kernel.hpp"

namespace ftc {
template void launch_dense<false, true>(const DenseArgs &a, int dtype, int tile, hipStream_t s);
}
