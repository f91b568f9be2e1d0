// The products dW = X^T dP: both across the contraction.  See dense_kernel.hpp.
#include "dense_kernel.hpp"

namespace ftc {
template void launch_dense<true, true>(const DenseArgs &a, int dtype, int tile, hipStream_t s);
}
