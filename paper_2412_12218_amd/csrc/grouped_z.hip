// Grouped products with W across the contraction.  See grouped_kernel.hpp.
#include "grouped_kernel.hpp"

namespace ftc {

template <class T, bool FAST>
static void rows_t(const GroupedArgs &g, int tile, hipStream_t s) { launch_grouped_rows_t<T, true, FAST>(g, tile, s); }

template <>
void launch_grouped_rows<true>(const GroupedArgs &g, int dtype, int tile, hipStream_t s)
{
    const bool fast = grouped_rows_fast(g.a, true, dtype);
    if (dtype == FTC_F32) FTC_GROUPED(rows_t, F32);
    else if (dtype == FTC_F16) FTC_GROUPED(rows_t, F16);
    else FTC_GROUPED(rows_t, BF16);
}

}  // namespace ftc
