// Dense layer with weights for each group of rows, Z_g = act(X_g W_g + b_g) + R_g, and its gradients
//   dP = dZ act'(P),  dX_g = dP_g W_g^T,  dW_g = X_g^T dP_g,  db_g = column sums of dP_g.
//
// The products are the dense layer's tiles, each of one group (grouped_kernel.hpp), all groups in one launch.  What is kept of the activation, and the
// roundings, are the dense layer's (linear.hip): act' is 16 bits of fixed point for 16-bit types (db 2e-4 to 3e-4 of its norm from one of unrounded slopes), dP is rounded to X's type, once, for both
// of its products, which the matrix instructions have in that type: 2.3e-3 of their norms in bf16, 1.7e-3 without, which are the results' own roundings.
#include "grouped_kernel.hpp"
#include "stream_piece.hpp"

namespace ftc {

// Group of a row, or -1.
__device__ __forceinline__ int group_of_row(const int *ptr, int groups, int row)
{
    int lo = 0, hi = groups;  // the last one that begins at or before it
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (ptr[mid] <= row) lo = mid;
        else hi = mid;
    }
    return ptr[lo] <= row && row < ptr[lo + 1] ? lo : -1;
}

// The sums of Z's or dX's parts, eight columns of a row a thread.
template <class T>
__global__ __launch_bounds__(256) void grouped_join_kernel(GroupedArgs g)
{
    const DenseArgs &a = g.a;
    const int eights = (a.N + 7) / 8;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (id >= static_cast<int64_t>(a.M) * eights) return;
    const int row = static_cast<int>(id / eights), col = static_cast<int>(id % eights) * 8, left = a.N - col;
    const int group = group_of_row(g.group_ptr, g.groups, row);
    if (group < 0) return;
    float x[8], bias[8];
    load_eight_numbers<T>(a.bias, static_cast<int64_t>(group) * a.N + col, a.bias ? left : 0, bias);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.f;
#pragma unroll 8
    for (int z = 0; z < a.splits; ++z) {
        float v[8];
        load_eight_numbers<F32>(a.part, (static_cast<int64_t>(z) * a.M + row) * a.N + col, left, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += v[j];
    }
    epilogue<T>(a, row, col, left, bias, x);
}

// dP = dZ act'(P) (dP NULL: not written) and, for the rows of a workgroup, which are of one group, its column sums (sums NULL: none), by the tile's number
// (grouped_plan.hpp).  2^log_lanes threads have the 16 bytes of VEC columns each of a row; a thread has DP_ROWS rows, all of them on their way at once.
constexpr int DP_ROWS = 4;
static int dp_lanes(int width, int vec)
{
    int b = 0;
    while (b < 5 && (vec << b) < width) ++b;
    return b;
}
static int dp_rows(int log_lanes) { return (256 >> log_lanes) * DP_ROWS; }  // of a workgroup
template <class T>
__global__ __launch_bounds__(256) void grouped_dp_kernel(int n, const int *__restrict__ ptr, int groups, int width, const void *__restrict__ dZ, int64_t ldz,
                                                         const void *__restrict__ slope, int64_t lds, void *__restrict__ dP, float *__restrict__ sums, int log_lanes)
{
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16, V = T::VEC;
    __shared__ float part[256 * V];
    const int lanes = 1 << log_lanes, subs = 256 >> log_lanes, side = subs * DP_ROWS;
    const GroupSpan span = group_span<false>(ptr, groups, n, side, [&](int) { return static_cast<int>(blockIdx.x); });
    if (span.group < 0) return;
    const int lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> log_lanes, col = (blockIdx.y * lanes + lane) * V, left = width - col;
    const int64_t row0 = span.start + static_cast<int64_t>(span.at) * side + sub, end = span.start + span.len;
    ftc_u32x4 w[DP_ROWS], u[DP_ROWS];
    // with a slope both are read for the last time, as dP takes their place; without one dZ itself is what dX and dW read next
    // (backward pass of 48 000 x 1024 -> 1024 in 16 groups in fp16 without a slope 322 us with the hint on dZ, 306 without; 46 000 x 100 -> 128 in 118 groups in fp32 65, 62)
    if ((span.at + 1) * side <= span.len && static_cast<int>((blockIdx.y + 1) * lanes * V) <= width) {  // uniform: all of the rows and columns are there
#pragma unroll
        for (int i = 0; i < DP_ROWS; ++i) {
            const int64_t row = row0 + i * subs;
            if (slope) {
                w[i] = load_piece_nt<T>(dZ, row * ldz + col);
                u[i] = load_piece_nt<T>(slope, row * lds + col);
            } else {
                w[i] = load_piece<T>(dZ, row * ldz + col, V);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < DP_ROWS; ++i) {
            const int64_t row = row0 + i * subs;
            w[i] = load_piece<T>(dZ, row * ldz + col, row < end ? left : 0);
            if (slope) u[i] = load_piece<T>(slope, row * lds + col, row < end ? left : 0);
        }
    }
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.f;
#pragma unroll
    for (int i = 0; i < DP_ROWS; ++i) {
        const int64_t row = row0 + i * subs;
        RawVec<T, V> r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r.w[j] = w[i][j];
        float g[V];
        unpack<T, V>(r, g);
        if (slope) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if constexpr (T::BYTES == 4) g[j] *= __uint_as_float(u[i][j]);
                else g[j] *= slope_value(static_cast<int16_t>(u[i][j / 2] >> (16 * (j & 1))));
            }
        }
        if (row >= end) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += g[j];
        if (dP && left > 0) {
            const int64_t at = row * width + col;
            if (left >= V) {
                store_piece<T>(dP, at, g);
            } else {
#pragma unroll
                for (int j = 0; j < V - 1; ++j)
                    if (j < left) store_elem(dP, at + j, DT, g[j]);
            }
        }
    }
    if (!sums) return;
#pragma unroll
    for (int j = 0; j < V; ++j) part[(sub * lanes + lane) * V + j] = sum[j];
    __syncthreads();
    // halves of the rows' sums onto the other half, in the same order every time
    const int columns = lanes * V;
    for (int half = subs / 2; half > 0; half /= 2) {
        for (int i = threadIdx.x; i < half * columns; i += 256) part[i] += part[i + half * columns];
        __syncthreads();
    }
    for (int i = threadIdx.x; i < columns; i += 256)
        if (blockIdx.y * columns + i < static_cast<unsigned>(width)) sums[static_cast<int64_t>(span.start / side + span.group + span.at) * width + blockIdx.y * columns + i] = part[i];
}

// What is added up last, in one launch: db_g = sum of the sums of the group's rows, 16 columns an item, 16 threads a column, items taken in turn by the first `groups` workgroups; and by the
// others, `across` of them along y, dW's parts.  11 us in a training step of 20 000 x 768 -> 768 in 8 groups, 5 and 9 by a launch each.
constexpr int JOIN_THREADS = 256, DB_MOST = 4096;  // workgroups for db
struct GroupedSums {
    const float *sums;
    void *db;
    int side, width, dtype;
    int64_t items;
    int groups, across;
};
__device__ __forceinline__ void group_bias(int n, const int *__restrict__ ptr, const GroupedSums &b, int64_t item, float (*part)[17])
{
    constexpr int EACH = JOIN_THREADS / 16;
    const int columns = (b.width + 15) / 16, group = static_cast<int>(item / columns), start = group_offset(ptr, group, n), len = max(group_offset(ptr, group + 1, n) - start, 0);
    const int c = threadIdx.x & 15, sub = threadIdx.x >> 4, col = static_cast<int>(item % columns) * 16 + c;
    const int64_t first = start / b.side + group, end = first + (len + b.side - 1) / b.side;
    float x = 0.f;
    if (col < b.width) {
#pragma unroll 8
        for (int64_t p = first + sub; p < end; p += EACH) x += b.sums[p * b.width + col];
    }
    part[sub][c] = x;
    __syncthreads();
    if (sub < 4) {
        x = 0.f;
#pragma unroll
        for (int k = 0; k < EACH / 4; ++k) x += part[sub * (EACH / 4) + k][c];
        x += __shfl_xor(x, 16, 64);
        x += __shfl_xor(x, 32, 64);
        if (sub == 0 && col < b.width) store_elem(b.db, static_cast<int64_t>(group) * b.width + col, b.dtype, x);
    }
    __syncthreads();
}

// The sums of dW's parts, for groups of several chunks.  Such a group has rows on both sides of the first multiple of k_each behind its start, and of those
// multiples there are n / k_each, one for each y.
__device__ __forceinline__ void join_weights(const GroupedArgs &g, int x0, int y)
{
    const DenseArgs &a = g.a;
    const int row = (y + 1) * a.k_each;
    const int group = row < a.K ? group_of_row(g.group_ptr, g.groups, row) : -1;
    if (group < 0) return;
    const int start = group_offset(g.group_ptr, group, a.K), end = group_offset(g.group_ptr, group + 1, a.K);
    if (end - start <= a.k_each || start == row || row - start > a.k_each) return;
    const int64_t id = (static_cast<int64_t>(x0) * JOIN_THREADS + threadIdx.x) * 4, all = static_cast<int64_t>(a.M) * a.N;
    if (id >= all) return;
    const int chunks = (end - start + a.k_each - 1) / a.k_each, left = static_cast<int>(all - id < 4 ? all - id : 4);
    const float *from = a.part + 2ll * (start / a.k_each) * all + id;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int c = 0; c < chunks; ++c) {
        const ftc_u32x4 v = load_piece<F32>(from, c * all, left);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += __uint_as_float(v[j]);
    }
    const int64_t to = group * all + id;
    if (left == 4) {
        store_vec_any<4>(a.out, to, a.out_dtype, x);
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < left) store_elem(a.out, to + j, a.out_dtype, x[j]);
    }
}

__global__ __launch_bounds__(JOIN_THREADS) void grouped_sums_kernel(GroupedArgs g, GroupedSums b)
{
    __shared__ float part[JOIN_THREADS / 16][17];
    const int id = static_cast<int>(blockIdx.x) - b.groups;
    if (id < 0) {  // uniform
        for (int64_t item = blockIdx.x; item < b.items; item += b.groups) group_bias(g.a.K, g.group_ptr, b, item, part);
    } else {
        join_weights(g, id % b.across, id / b.across);
    }
}

// ---- launches --------------------------------------------------------------------------------------------------
static size_t rows_ws(int n, int groups, int N, int K)
{
    size_t most = 0;
    for (int v = 0; v < 4; ++v) {
        const DensePlan p = grouped_plan(n, groups, N, K, v & 1, v & 2);
        const size_t tail = p.tile == DENSE_256 && grouped_tail_on(n, groups, N, K) ? 256ull * 256 * 256 : 0, own = p.splits > 1 ? static_cast<size_t>(p.splits) * n * N : tail;
        if (own > most) most = own;
    }
    return align_up(most * sizeof(float), 256);
}
static size_t dw_ws(int n, int groups, int M, int N)
{
    int64_t most = 0;
    for (int v = 0; v < 4; ++v) {
        const int64_t parts = grouped_dw_parts(n, grouped_dw_plan(n, groups, M, N, v & 1, v & 2));
        if (parts > most) most = parts;
    }
    return align_up(static_cast<size_t>(most) * M * N * sizeof(float), 256);
}

template <bool BX>
static void grouped(GroupedArgs g, int dtype, void *ws, hipStream_t s)
{
    const DensePlan p = grouped_plan(g.a.M, g.groups, g.a.N, g.a.K, dtype == FTC_F32, grouped_rows_fast(g.a, BX, dtype));
    g.a.splits = p.splits;
    g.a.k_each = p.k_each;
    g.a.part = static_cast<float *>(ws);
    g.tail = p.tile == DENSE_256 && p.splits == 1 && grouped_tail_on(g.a.M, g.groups, g.a.N, g.a.K);
    launch_grouped_rows<BX>(g, dtype, p.tile, s);
    if (p.splits > 1) {
        const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(g.a.M) * ceil_div(g.a.N, 8) + 255) / 256));
        if (dtype == FTC_F32) hipLaunchKernelGGL(grouped_join_kernel<F32>, grid, dim3(256), 0, s, g);
        else if (dtype == FTC_F16) hipLaunchKernelGGL(grouped_join_kernel<F16>, grid, dim3(256), 0, s, g);
        else hipLaunchKernelGGL(grouped_join_kernel<BF16>, grid, dim3(256), 0, s, g);
    }
}

static void add_rows_size(LaunchSize &z, int n, int groups, int N, int K)
{
    for (int v = 0; v < 4; ++v) {
        const DensePlan p = grouped_plan(n, groups, N, K, v & 1, v & 2);
        z.add(grouped_most(n, groups, grouped_rows(p.tile)) * dense_parts(N, grouped_columns(p.tile)) * grouped_threads(p.tile) + 256 * 512, p.splits);
    }
    z.add(static_cast<int64_t>(n) * ceil_div(N, 8), 1);
}
LaunchSize grouped_linear_size(int n, int groups, int d_in, int d_out)
{
    LaunchSize z;
    add_rows_size(z, n, groups, d_out, d_in);
    return z;
}
LaunchSize grouped_linear_backward_size(int n, int groups, int d_in, int d_out)
{
    LaunchSize z;
    add_rows_size(z, n, groups, d_in, d_out);
    for (int v = 0; v < 4; ++v) {
        const DensePlan p = grouped_dw_plan(n, groups, d_in, d_out, v & 1, v & 2);
        z.add(grouped_dw_groups(n, groups, p.k_each, dense_tiles(d_in, d_out, p.tile)) * grouped_threads(p.tile), n / p.k_each);
    }
    z.add(static_cast<int64_t>(d_in) * d_out / 4, 1);
    for (int vec = 4; vec <= 8; vec *= 2) {
        const int lanes = dp_lanes(d_out, vec);
        z.add(256ll * grouped_most(n, groups, dp_rows(lanes)), ceil_div(d_out, vec << lanes));
    }
    return z;
}

size_t grouped_linear_ws(int n, int groups, int d_in, int d_out) { return rows_ws(n, groups, d_out, d_in); }

static size_t sums_bytes(int n, int groups, int d_out)
{
    const int rows = dp_rows(dp_lanes(d_out, 4));  // those of fp32 are at most as many as those of 16 bits
    return align_up(static_cast<size_t>(grouped_most(n, groups, rows)) * d_out * sizeof(float), 256);
}

size_t grouped_linear_backward_ws(int n, int groups, int d_in, int d_out)
{
    const size_t x = rows_ws(n, groups, d_in, d_out), w = dw_ws(n, groups, d_in, d_out);
    return align_up(static_cast<size_t>(n) * d_out * sizeof(float), 256) + sums_bytes(n, groups, d_out) + (x > w ? x : w);
}

int32_t launch_grouped_linear(const LinearShape &p, const int *group_ptr, int groups, void *ws, hipStream_t s)
{
    GroupedArgs g = {};
    g.group_ptr = group_ptr;
    g.groups = groups;
    DenseArgs &a = g.a;
    a.A = p.X; a.lda = p.ldx; a.B = p.W; a.ldb = p.d_out;
    a.M = p.n; a.N = p.d_out; a.K = p.d_in;
    a.bias = p.bias; a.act = p.act; a.residual = p.residual; a.ldr = p.ldr;
    a.slope = p.slope; a.lds = p.lds; a.out = p.Z; a.ldo = p.ldz; a.out_dtype = p.z_dtype;
    grouped<true>(g, p.dtype, ws, s);
    return launch_status("grouped linear");
}

template <class T>
static void grouped_backward_t(const LinearShape &p, const LinearGrads &k, const int *group_ptr, int groups, void *ws, hipStream_t s)
{
    char *q = static_cast<char *>(ws);
    void *dP = q; q += align_up(static_cast<size_t>(p.n) * p.d_out * sizeof(float), 256);
    float *sums = reinterpret_cast<float *>(q); q += sums_bytes(p.n, groups, p.d_out);
    const int lanes = dp_lanes(p.d_out, T::VEC), side = dp_rows(lanes);
    const void *G = p.slope ? dP : k.dZ;
    const int64_t ldg = p.slope ? p.d_out : k.lddz;
    if ((p.slope || k.db) && p.n > 0) {
        const dim3 grid(static_cast<unsigned>(grouped_most(p.n, groups, side)), ceil_div(p.d_out, T::VEC << lanes));
        hipLaunchKernelGGL(grouped_dp_kernel<T>, grid, dim3(256), 0, s, p.n, group_ptr, groups, p.d_out, k.dZ, static_cast<int64_t>(k.lddz), p.slope,
                           static_cast<int64_t>(p.lds), p.slope ? dP : nullptr, k.db ? sums : nullptr, lanes);
    }
    GroupedArgs g = {};
    g.group_ptr = group_ptr;
    g.groups = groups;
    DenseArgs &a = g.a;
    const int64_t items = k.db ? static_cast<int64_t>(groups) * ceil_div(p.d_out, 16) : 0;
    GroupedSums last = {sums, k.db, side, p.d_out, k.dw_dtype, items, static_cast<int>(items < DB_MOST ? items : DB_MOST), 1};
    int64_t joins = 0;
    if (k.dX && p.n > 0) {
        a.A = G; a.lda = ldg; a.B = p.W; a.ldb = p.d_out;
        a.M = p.n; a.N = p.d_in; a.K = p.d_out;
        a.residual = k.dX_add; a.ldr = k.ldda; a.out = k.dX; a.ldo = k.lddx; a.out_dtype = k.dx_dtype;
        grouped<false>(g, p.dtype, q, s);
    }
    if (k.dW) {
        a = {};
        a.A = p.X; a.lda = p.ldx; a.B = G; a.ldb = ldg;
        a.M = p.d_in; a.N = p.d_out; a.K = p.n;
        a.out = k.dW; a.ldo = p.d_out; a.out_dtype = k.dw_dtype;
        const DensePlan plan = grouped_dw_plan(p.n, groups, p.d_in, p.d_out, p.dtype == FTC_F32, grouped_dw_fast(a, p.dtype));
        a.k_each = plan.k_each;
        a.part = reinterpret_cast<float *>(q);
        launch_grouped_dw(g, p.dtype, plan.tile, s);
        if (grouped_dw_parts(p.n, plan) > 0) {
            last.across = static_cast<int>((static_cast<int64_t>(p.d_in) * p.d_out + 4 * JOIN_THREADS - 1) / (4 * JOIN_THREADS));
            joins = static_cast<int64_t>(last.across) * (p.n / plan.k_each);  // of parts of at most 2 GB
        }
    }
    a.K = p.n;
    if (last.groups + joins > 0) hipLaunchKernelGGL(grouped_sums_kernel, dim3(static_cast<unsigned>(last.groups + joins)), dim3(JOIN_THREADS), 0, s, g, last);
}

int32_t launch_grouped_linear_backward(const LinearShape &p, const LinearGrads &g, const int *group_ptr, int groups, void *ws, hipStream_t s)
{
    if (p.dtype == FTC_F32) grouped_backward_t<F32>(p, g, group_ptr, groups, ws, s);
    else if (p.dtype == FTC_F16) grouped_backward_t<F16>(p, g, group_ptr, groups, ws, s);
    else grouped_backward_t<BF16>(p, g, group_ptr, groups, ws, s);
    return launch_status("grouped linear backward");
}

}  // namespace ftc
