// Weight gradients by group.  See grouped_kernel.hpp.
#include "grouped_kernel.hpp"

namespace ftc {

int64_t grouped_dw_groups(int n, int groups, int k_each, int64_t tiles)
{
    const int64_t turn = 8 * dw_unit(static_cast<int>(tiles < DW_EIGHT ? tiles : DW_EIGHT));
    return (grouped_most(n, groups, k_each) * tiles + turn - 1) / turn * turn;
}

template <class T, bool FAST>
static void dw_t(const GroupedArgs &g, int tile, hipStream_t s)
{
    const dim3 grid(static_cast<unsigned>(grouped_dw_groups(g.a.K, g.groups, g.a.k_each, dense_tiles(g.a.M, g.a.N, tile))));
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
