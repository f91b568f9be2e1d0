// Weight gradients by group.  See grouped_kernel.hpp.
#include "grouped_kernel.hpp"

namespace ftc {

template <class T, bool FAST>
static void dw_t(const GroupedArgs &g, int tile, hipStream_t s)
{
    const int64_t chunks = (grouped_numbers(g.a.K, g.groups, g.a.k_each) + 7) / 8 * 8;
    const dim3 grid(static_cast<unsigned>(chunks * dense_tiles(g.a.M, g.a.N, tile)));
    if (tile == DENSE_64) {
        hipLaunchKernelGGL((grouped_dw_kernel<T, FAST, 2, 2, 1, 1>), grid, dim3(256), 0, s, g);
    } else if (tile == DENSE_128) {
        hipLaunchKernelGGL((grouped_dw_kernel<T, FAST, 2, 2, 2, 2>), grid, dim3(256), 0, s, g);
    } else if constexpr (FAST && T::BYTES == 2) {
        hipLaunchKernelGGL((grouped_dw_kernel<T, FAST, 2, 4, 4, 2>), grid, dim3(512), 0, s, g);
    }
}

void launch_grouped_dw(const GroupedArgs &g, int dtype, int tile, hipStream_t s)
{
    const bool fast = grouped_dw_fast(g.a, dtype);
    if (dtype == FTC_F32) FTC_GROUPED(dw_t, F32);
    else if (dtype == FTC_F16) FTC_GROUPED(dw_t, F16);
    else FTC_GROUPED(dw_t, BF16);
}

}  // namespace ftc
