// The products dX = dP W^T: both along the contraction.  See dense_kernel.hpp.
#include "dense_kernel.hpp"

namespace ftc {
template void launch_dense<false, false>(const DenseArgs &a, int dtype, int tile, hipStream_t s);
}
