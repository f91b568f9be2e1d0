// The product kernels of the grouped dense layer (grouped_linear.hip): the dense layer's tiles, each of one group.
//
// The groups' rows are known on the device only, so a launch has as many workgroups as groups could ever need (grouped_plan.hpp), and each of them looks up which tile of
// which group it is for, or that it is not needed.
//
// As fast as the dense layer's tiles: 48 000 rows in 16 groups, 4096 -> 1024 in fp16 430 to 453 us from card to card (937 to 889 TFLOP/s; a library product of 8192^3 1086), 20 000 in 8 groups, 768 -> 768 in bf16 Z 48,
// dX 38, dW 48 us.  24 rows of 64 groups, 1024 -> 4096 in bf16: 24 us, 135 MB of weights at 5.6 TB/s.
#pragma once
#include "dense_kernel.hpp"
#include "grouped_plan.hpp"

namespace ftc {

struct GroupedArgs {
    DenseArgs a;  // M: all rows (Z, dX); K: all rows (dW)
    const int *group_ptr;
    int groups, tail;  // tail: whether there may be one (grouped_tail_on)
};

// Z: A along the contraction, W across it.  dX: both along it.  dW: both across it, in chunks of at most k_each rows.
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

// Workgroups of a weight gradient's launch.
int64_t grouped_dw_groups(int n, int groups, int k_each, int64_t tiles);

#if defined(__HIPCC__)

// What a workgroup is for: tile (chunk) `at` of the rows start .. start + len - 1 of a group; group -1: nothing.
struct GroupSpan {
    int group, start, len, at;
};
__device__ __forceinline__ int group_offset(const int *ptr, int i, int n) { return min(max(ptr[i], 0), n); }
// Tiles of a group; EMPTY: one of a group without rows, too.
template <bool EMPTY>
__device__ __forceinline__ int group_tiles(int start, int end, int side)
{
    const int len = max(end - start, 0);
    return EMPTY && len == 0 ? 1 : len / side + (len % side != 0);
}

// The tile `number` of the tiles of all groups, counted in their order; number(tiles): it, from how many there are.  Every wave counts for itself, lane l the groups from
// l each on, `each` = ceil(groups / 64): one load for up to 64 groups, and a scan over the lanes.  Beyond GROUPS_COUNTED groups nothing is counted: a group's
// tiles have the numbers of grouped_plan.hpp, some of which stand for nothing, and the group is found by looking at 64 offsets at a time.
constexpr int GROUPS_COUNTED = 512;
template <bool EMPTY, class Number>
__device__ __forceinline__ GroupSpan group_span(const int *ptr, int groups, int n, int side, const Number &number)
{
    const int lane = threadIdx.x & 63;
    if (groups > GROUPS_COUNTED) {
        const int tiles = n / side + groups, wanted = number(tiles);
        if (wanted < 0 || wanted >= tiles) return {-1, 0, 0, 0};
        int lo = 0, hi = groups;  // the last group whose numbers begin at or before it is in lo .. hi - 1
        do {
            const int stride = (hi - lo + 63) / 64, i = lo + lane * stride;
            const bool before = i < hi && group_offset(ptr, i, n) / side + i <= wanted;
            const int count = __popcll(__builtin_amdgcn_ballot_w64(before));
            if (count == 0) return {-1, 0, 0, 0};  // in front of the first group
            lo += (count - 1) * stride;
            hi = min(lo + stride, hi);
        } while (hi - lo > 1);
        const int s = __builtin_amdgcn_readfirstlane(group_offset(ptr, lo, n)), e = __builtin_amdgcn_readfirstlane(group_offset(ptr, lo + 1, n)), at = wanted - s / side - lo;
        return {at >= 0 && at < group_tiles<EMPTY>(s, e, side) ? lo : -1, s, max(e - s, 0), at};
    }
    const int each = (groups + 63) / 64, from = min(lane * each, groups), to = min(from + each, groups);
    int own = 0, start = group_offset(ptr, from, n), last = start;
#pragma unroll 4
    for (int g = from; g < to; ++g) {
        const int end = group_offset(ptr, g + 1, n);
        own += group_tiles<EMPTY>(last, end, side);
        last = end;
    }
    const int upto = wave_inclusive_scan(own), tiles = __builtin_amdgcn_readlane(upto, 63), wanted = number(tiles);
    if (wanted < 0 || wanted >= tiles) return {-1, 0, 0, 0};
    const int at_lane = __popcll(__builtin_amdgcn_ballot_w64(upto <= wanted));  // the first lane that has more
    int g = min(at_lane * each, groups - 1), at = wanted - __builtin_amdgcn_readlane(upto - own, at_lane);
    int s = __builtin_amdgcn_readlane(start, at_lane), e = each == 1 ? __builtin_amdgcn_readlane(last, at_lane) : group_offset(ptr, g + 1, n);
    for (int k = 1; k < each; ++k) {  // uniform
        const int there = group_tiles<EMPTY>(s, e, side);
        if (at < there) break;
        at -= there;
        s = e;
        g = min(g + 1, groups - 1);
        e = group_offset(ptr, g + 1, n);
    }
    return {at >= 0 && at < group_tiles<EMPTY>(s, e, side) ? g : -1, s, max(e - s, 0), at};  // else: offsets that decrease
}

__device__ __forceinline__ const void *moved(const void *p, int64_t bytes) { return p ? static_cast<const char *>(p) + bytes : nullptr; }
__device__ __forceinline__ void *moved(void *p, int64_t bytes) { return p ? static_cast<char *>(p) + bytes : nullptr; }
__device__ __forceinline__ int out_bytes(int dtype) { return dtype == FTC_F32 ? 4 : 2; }

// The product of a group, out of that of all rows.
template <class T>
__device__ __forceinline__ DenseArgs of_group(const DenseArgs &all, const GroupSpan &span)
{
    const int64_t first = span.start;
    DenseArgs a = all;
    a.M = span.len;
    a.A = moved(a.A, first * a.lda * T::BYTES);
    a.B = moved(a.B, static_cast<int64_t>(span.group) * a.N * a.K * T::BYTES);
    a.bias = moved(a.bias, static_cast<int64_t>(span.group) * a.N * T::BYTES);
    a.residual = moved(a.residual, first * a.ldr * T::BYTES);
    a.slope = moved(a.slope, first * a.lds * T::BYTES);
    a.out = moved(a.out, first * a.ldo * out_bytes(a.out_dtype));
    return a;
}

template <class T, bool BX, bool FAST, int RW, int CW, int WM, int WN>
__global__ __launch_bounds__(64 * RW * CW, 2) void grouped_rows_kernel(GroupedArgs g)
{
    constexpr int TM = 32 * WM * RW, TN = 32 * WN * CW;
    const int tiles_n = (g.a.N + TN - 1) / TN;
    int tn = 0, part_of = -1;  // which of the parts of a tile of the tail
    GroupedTail tail = {0, 0, 1};
    // groups of few rows are bound by reading their weights, which no two tiles share: those of a group go round the XCDs
    const GroupSpan span = group_span<false>(g.group_ptr, g.groups, g.a.M, TM, [&](int tiles) {
        int tm = -1, id = blockIdx.x;
        if (TM == 32) {
            tm = id / tiles_n;
            tn = id % tiles_n;
            return tm;
        }
        if (TM == 256 && g.tail) {
            tail = grouped_tail(static_cast<int64_t>(tiles) * tiles_n, g.a.K);
            if (id >= tail.full && tail.rest) {
                part_of = (id - tail.full) % tail.parts;
                id = tail.full + (id - tail.full) / tail.parts;
            }
        }
        if (id < tiles * tiles_n) dense_tile(id, tiles, tiles_n, tm, tn);
        return tm;
    });
    if (span.group < 0) return;
    const DenseArgs a = of_group<T>(g.a, span);
    int k_begin = static_cast<int>(blockIdx.y) * a.k_each, k_end = min(a.K, k_begin + a.k_each);
    float *part = a.splits > 1 ? a.part + (static_cast<int64_t>(blockIdx.y) * g.a.M + span.start) * a.N : nullptr;
    int64_t part_ld = a.N;
    if (TM == 256 && part_of >= 0) {
        const int each = tail_each(a.K, tail.parts);
        k_begin = min(part_of * each, a.K);
        k_end = min(k_begin + each, a.K);
        // the workgroup's place, as one tile
        part_ld = TN;
        part = a.part + static_cast<int64_t>(blockIdx.x - tail.full) * TM * TN - (static_cast<int64_t>(span.at) * TM * TN + static_cast<int64_t>(tn) * TN);
    }
    dense_product<T, false, BX, FAST, RW, CW, WM, WN>(a, span.at, tn, k_begin, k_end, part, part_ld);
}

// The sums of the tail's parts: 32 workgroups a tile, eight columns of a row a thread.
template <class T>
__global__ __launch_bounds__(256) void grouped_tail_kernel(GroupedArgs g)
{
    constexpr int TM = 256, TN = 256;
    const int tiles_n = (g.a.N + TN - 1) / TN, which = blockIdx.x / 32;
    int tn = 0;
    GroupedTail tail = {0, 0, 1};
    const GroupSpan span = group_span<false>(g.group_ptr, g.groups, g.a.M, TM, [&](int tiles) {
        int tm = -1;
        tail = grouped_tail(static_cast<int64_t>(tiles) * tiles_n, g.a.K);
        if (which < tail.rest) dense_tile(tail.full + which, tiles, tiles_n, tm, tn);
        return tm;
    });
    if (span.group < 0) return;
    const DenseArgs a = of_group<T>(g.a, span);
    const int id = blockIdx.x % 32 * 256 + threadIdx.x, r = id / (TN / 8), c = id % (TN / 8) * 8, row = span.at * TM + r, col = tn * TN + c, left = a.N - col;
    if (row >= a.M || left <= 0) return;
    float x[8], bias[8];
    load_eight_numbers<T>(a.bias, col, a.bias ? left : 0, bias);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.f;
#pragma unroll
    for (int p = 0; p < TAIL_PARTS; ++p) {
        if (p >= tail.parts) break;
        float v[8];
        load_eight_numbers<F32>(a.part, (static_cast<int64_t>(which * tail.parts + p) * TM + r) * TN + c, left, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += v[j];
    }
    epilogue<T>(a, row, col, left, bias, x);
}

// Eight tiles of a chunk (a band's column, dense_band: they share the rows of both operands) are of one XCD, the eights go round the XCDs.
constexpr int DW_EIGHT = 8;
inline __host__ __device__ int dw_unit(int tiles) { return tiles < DW_EIGHT ? tiles : DW_EIGHT; }
template <class T, bool FAST, int RW, int CW, int WM, int WN>
__global__ __launch_bounds__(64 * RW * CW, 2) void grouped_dw_kernel(GroupedArgs g)
{
    constexpr int TM = 32 * WM * RW, TN = 32 * WN * CW;
    DenseArgs a = g.a;
    const int tiles_m = (a.M + TM - 1) / TM, tiles_n = (a.N + TN - 1) / TN, tiles = tiles_m * tiles_n, unit = dw_unit(tiles), k = blockIdx.x / 8;
    const int item = (k / unit * 8 + static_cast<int>(blockIdx.x) % 8) * unit + k % unit;
    int tm, tn;
    dense_band(item % tiles, tiles_m, tiles_n, tm, tn);
    const GroupSpan span = group_span<true>(g.group_ptr, g.groups, a.K, a.k_each, [&](int) { return item / tiles; });
    if (span.group < 0) return;
    const int chunks = group_tiles<true>(span.start, span.start + span.len, a.k_each);  // a group without rows has zeros to write
    const int64_t first = span.start + static_cast<int64_t>(span.at) * a.k_each;
    float *part = chunks > 1 ? a.part + (2ll * (span.start / a.k_each) + span.at) * a.M * a.N : nullptr;
    a.K = min(a.k_each, span.len - span.at * a.k_each);
    a.A = moved(a.A, first * a.lda * T::BYTES);
    a.B = moved(a.B, first * a.ldb * T::BYTES);
    a.out = moved(a.out, static_cast<int64_t>(span.group) * a.M * a.N * out_bytes(a.out_dtype));
    dense_product<T, true, true, FAST, RW, CW, WM, WN>(a, tm, tn, 0, a.K, part, a.N);
}

template <class T, bool BX, bool FAST>
void launch_grouped_rows_t(const GroupedArgs &g, int tile, hipStream_t s)
{
    const int64_t most = grouped_most(g.a.M, g.groups, grouped_rows(tile)) * ceil_div(g.a.N, grouped_columns(tile));
    const dim3 grid(static_cast<unsigned>(most + (g.tail ? 256 : 0)), g.a.splits);  // 256: the tail's parts
    if (tile == DENSE_64) {
        hipLaunchKernelGGL((grouped_rows_kernel<T, BX, FAST, 2, 2, 1, 1>), grid, dim3(256), 0, s, g);
    } else if (tile == DENSE_128) {
        hipLaunchKernelGGL((grouped_rows_kernel<T, BX, FAST, 2, 2, 2, 2>), grid, dim3(256), 0, s, g);
    } else if (tile == GROUPED_THIN) {
        hipLaunchKernelGGL((grouped_rows_kernel<T, BX, FAST, 1, 4, 1, 1>), grid, dim3(256), 0, s, g);
    } else if constexpr (FAST && T::BYTES == 2) {
        hipLaunchKernelGGL((grouped_rows_kernel<T, BX, FAST, 2, 4, 4, 2>), grid, dim3(512), 0, s, g);
        if (g.tail) hipLaunchKernelGGL(grouped_tail_kernel<T>, dim3(128 * 32), dim3(256), 0, s, g);
    }
}

#define FTC_GROUPED(launch, T)                  \
    do {                                        \
        if (fast) launch<T, true>(g, tile, s);  \
        else launch<T, false>(g, tile, s);      \
    } while (0)

#endif  // __HIPCC__
}  // namespace ftc
