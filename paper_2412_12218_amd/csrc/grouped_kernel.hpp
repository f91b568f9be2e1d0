// The product kernels of the grouped dense layer (grouped_linear.hip): the dense layer's tiles, each of one group.
//
// The groups' rows are known on the device only, so a launch has as many workgroups as groups could ever need (grouped_plan.hpp) and each looks up what it is
// for: a wave looks at 64 offsets at once, one step for up to 64 groups, two up to 4096.
#pragma once
#include "dense_kernel.hpp"
#include "grouped_plan.hpp"

namespace ftc {

struct GroupedArgs {
    DenseArgs a;  // M: all rows (Z, dX); K: all rows (dW)
    const int *group_ptr;
    int groups;
};

// Z: A along the contraction, W across it.  dX: both along it.  dW: both across it, k_each rows a chunk, a.splits > 1 where groups may have several.
template <bool BX>
void launch_grouped_rows(const GroupedArgs &g, int dtype, int tile, hipStream_t s);
void launch_grouped_dw(const GroupedArgs &g, int dtype, int tile, hipStream_t s);

// Whether the rows of both operands are whole pieces (dense_kernel.hpp); a group's first ones are at 16 bytes then, too.
inline bool grouped_rows_fast(const DenseArgs &a, bool across, int dtype)
{
    return dense_whole_pieces(a.A, a.lda, a.K, dtype) && dense_whole_pieces(a.B, a.ldb, across ? a.N : a.K, dtype);
}
inline bool grouped_dw_fast(const DenseArgs &a, int dtype)
{
    return dense_whole_pieces(a.A, a.lda, a.M, dtype) && dense_whole_pieces(a.B, a.ldb, a.N, dtype);
}

#if defined(__HIPCC__)

struct GroupSpan {
    int group, start, len, at;  // at: which of the group's tiles
};
__device__ __forceinline__ int group_offset(const int *ptr, int i, int n) { return min(max(ptr[i], 0), n); }

// What number `id` stands for (grouped_numbers); group -1: nothing.
__device__ __forceinline__ GroupSpan group_span(const int *ptr, int groups, int n, int side, int id)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = groups;  // the last group whose numbers begin at or before id is in lo .. hi - 1
    do {
        const int stride = (hi - lo + 63) / 64, i = lo + lane * stride;
        const bool before = i < hi && group_offset(ptr, i, n) / side + i <= id;
        const int count = __popcll(__builtin_amdgcn_ballot_w64(before));
        if (count == 0) return {-1, 0, 0, 0};  // in front of the first group
        lo += (count - 1) * stride;
        hi = min(lo + stride, hi);
    } while (hi - lo > 1);
    const int start = __builtin_amdgcn_readfirstlane(group_offset(ptr, lo, n)), end = __builtin_amdgcn_readfirstlane(group_offset(ptr, lo + 1, n));
    const int at = id - start / side - lo;
    return {at < 0 ? -1 : lo, start, max(end - start, 0), at};  // below 0: offsets that decrease
}

__device__ __forceinline__ const void *moved(const void *p, int64_t bytes) { return p ? static_cast<const char *>(p) + bytes : nullptr; }
__device__ __forceinline__ void *moved(void *p, int64_t bytes) { return p ? static_cast<char *>(p) + bytes : nullptr; }
__device__ __forceinline__ int out_bytes(int dtype) { return dtype == FTC_F32 ? 4 : 2; }

template <class T, bool BX, bool FAST, int RW, int CW, int WM, int WN>
__global__ __launch_bounds__(64 * RW * CW, 2) void grouped_rows_kernel(GroupedArgs g)
{
    constexpr int TM = 32 * WM * RW, TN = 32 * WN * CW;
    DenseArgs a = g.a;
    int id, tn;
    dense_tile(blockIdx.x, a.M / TM + g.groups, (a.N + TN - 1) / TN, id, tn);
    const GroupSpan span = group_span(g.group_ptr, g.groups, a.M, TM, id);
    if (span.group < 0 || static_cast<int64_t>(span.at) * TM >= span.len) return;
    const int64_t first = span.start;
    const int k_begin = static_cast<int>(blockIdx.y) * a.k_each, k_end = min(a.K, k_begin + a.k_each);
    float *part = a.splits > 1 ? a.part + (static_cast<int64_t>(blockIdx.y) * a.M + first) * a.N : nullptr;
    a.M = span.len;
    a.A = moved(a.A, first * a.lda * T::BYTES);
    a.B = moved(a.B, static_cast<int64_t>(span.group) * a.N * a.K * T::BYTES);
    a.bias = moved(a.bias, static_cast<int64_t>(span.group) * a.N * T::BYTES);
    a.residual = moved(a.residual, first * a.ldr * T::BYTES);
    a.slope = moved(a.slope, first * a.lds * T::BYTES);
    a.out = moved(a.out, first * a.ldo * out_bytes(a.out_dtype));
    dense_product<T, false, BX, FAST, RW, CW, WM, WN>(a, span.at, tn, k_begin, k_end, part);
}

// Chunks go round the XCDs; all the tiles of a chunk, which share its rows, are of one.
template <class T, bool FAST, int RW, int CW, int WM, int WN>
__global__ __launch_bounds__(64 * RW * CW, 2) void grouped_dw_kernel(GroupedArgs g)
{
    constexpr int TM = 32 * WM * RW, TN = 32 * WN * CW;
    DenseArgs a = g.a;
    const int tiles_m = (a.M + TM - 1) / TM, tiles_n = (a.N + TN - 1) / TN, tiles = tiles_m * tiles_n, k = blockIdx.x / 8;
    int tm, tn;
    dense_band(k % tiles, tiles_m, tiles_n, tm, tn);
    const GroupSpan span = group_span(g.group_ptr, g.groups, a.K, a.k_each, k / tiles * 8 + static_cast<int>(blockIdx.x) % 8);
    const int chunks = span.len > a.k_each ? (span.len + a.k_each - 1) / a.k_each : 1;  // a group without rows has zeros to write
    if (span.group < 0 || span.at >= chunks) return;
    const int64_t first = span.start + static_cast<int64_t>(span.at) * a.k_each;
    float *part = chunks > 1 ? a.part + (2ll * (span.start / a.k_each) + span.at) * a.M * a.N : nullptr;
    a.K = min(a.k_each, span.len - span.at * a.k_each);
    a.A = moved(a.A, first * a.lda * T::BYTES);
    a.B = moved(a.B, first * a.ldb * T::BYTES);
    a.out = moved(a.out, static_cast<int64_t>(span.group) * a.M * a.N * out_bytes(a.out_dtype));
    dense_product<T, true, true, FAST, RW, CW, WM, WN>(a, tm, tn, 0, a.K, part);
}

template <class T, bool BX, bool FAST>
void launch_grouped_rows_t(const GroupedArgs &g, int tile, hipStream_t s)
{
    const dim3 grid(static_cast<unsigned>(grouped_numbers(g.a.M, g.groups, grouped_rows(tile)) * ceil_div(g.a.N, grouped_columns(tile))), g.a.splits);
    if (tile == DENSE_64) {
        hipLaunchKernelGGL((grouped_rows_kernel<T, BX, FAST, 2, 2, 1, 1>), grid, dim3(256), 0, s, g);
    } else if (tile == DENSE_128) {
        hipLaunchKernelGGL((grouped_rows_kernel<T, BX, FAST, 2, 2, 2, 2>), grid, dim3(256), 0, s, g);
    } else if (tile == GROUPED_THIN) {
        hipLaunchKernelGGL((grouped_rows_kernel<T, BX, FAST, 1, 4, 1, 1>), grid, dim3(256), 0, s, g);
    } else if constexpr (FAST && T::BYTES == 2) {
        hipLaunchKernelGGL((grouped_rows_kernel<T, BX, FAST, 2, 4, 4, 2>), grid, dim3(512), 0, s, g);
    }
}

#define FTC_GROUPED(launch, T)                  \
    do {                                        \
        if (fast) launch<T, true>(g, tile, s);  \
        else launch<T, false>(g, tile, s);      \
    } while (0)

#endif  // __HIPCC__
}  // namespace ftc
