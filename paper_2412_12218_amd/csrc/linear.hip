// Dense layer with its epilogue, Z = act(X W + b) + R, and its gradients
//   dP = dZ act'(P),  dX = dP W^T,  dW = X^T dP,  db = column sums of dP   (P = X W + b).
//
// All three products run on one kernel (dense_kernel.hpp).  Few tiles and a long contraction (a single row; a weight gradient): the
// contraction is split over workgroups, whose parts are added up in order by a second kernel, which has the epilogue then.
//
// The forward pass keeps act'(P), not P: it is between -0.13 and 1.13, so 16 bits of fixed point with 14 of fraction hold it to 2^-15
// (P in bf16 would move dP by a third of its own rounding), and the backward pass needs no activation function.  dP is rounded to the type of
// X for the products; db is the sum of the unrounded ones.
//
// A training step of 20 000 x 768 -> 768 in bf16 (SiLU, bias, residual) takes 164 us: Z 53, dP and its sums 21 (92 MB at 4.4 TB/s), db 5, dX 35, dW 42 in twelve
// parts and 8 to join them.
#include "dense_kernel.hpp"

namespace ftc {

// The parts' sums, eight columns of a row for LANES neighbouring lanes, which take the parts in turn.
template <class T, int LANES>
__global__ __launch_bounds__(256) void dense_join_kernel(DenseArgs a)
{
    const int eights = (a.N + 7) / 8, z0 = threadIdx.x % LANES;
    const int64_t id = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / LANES;
    const bool there = id < static_cast<int64_t>(a.M) * eights;
    const int row = there ? static_cast<int>(id / eights) : 0, col = there ? static_cast<int>(id % eights) * 8 : 0, left = a.N - col;
    float x[8], bias[8];
    load_eight_numbers<T>(a.bias, col, a.bias ? left : 0, bias);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.f;
#pragma unroll 8
    for (int z = z0; z < a.splits; z += LANES) {
        float v[8];
        load_eight_numbers<F32>(a.part, (static_cast<int64_t>(z) * a.M + row) * a.N + col, left, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += v[j];
    }
#pragma unroll
    for (int m = 1; m < LANES; m *= 2)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += __shfl_xor(x[j], m, 64);
    if (there && z0 == 0) epilogue<T>(a, row, col, left, bias, x);
}

// dP = dZ act'(P) (dP NULL: not written) and, for the rows of a workgroup, its column sums (sums NULL: none).  2^log_lanes threads have the 16
// bytes of VEC columns each of a row; a thread has DP_ROWS rows, all of them on their way at once.
constexpr int DP_ROWS = 4;
static int dp_lanes(int width, int vec)
{
    int b = 0;
    while (b < 5 && (vec << b) < width) ++b;
    return b;
}
static int dp_rows(int log_lanes) { return (256 >> log_lanes) * DP_ROWS; }  // of a workgroup
template <class T>
__global__ __launch_bounds__(256) void linear_dp_kernel(int n, int width, const void *__restrict__ dZ, int64_t ldz, const void *__restrict__ slope,
                                                        int64_t lds, void *__restrict__ dP, float *__restrict__ sums, int log_lanes)
{
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16, V = T::VEC;
    __shared__ float part[256 * V];
    const int lanes = 1 << log_lanes, groups = 256 >> log_lanes;
    const int lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> log_lanes, col = (blockIdx.y * lanes + lane) * V, left = width - col;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * groups * DP_ROWS + sub;
    ftc_u32x4 w[DP_ROWS], u[DP_ROWS];
#pragma unroll
    for (int i = 0; i < DP_ROWS; ++i) {
        const int64_t row = row0 + i * groups;
        w[i] = load_piece<T>(dZ, row * ldz + col, row < n ? left : 0);
        if (slope) u[i] = load_piece<T>(slope, row * lds + col, row < n ? left : 0);
    }
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.f;
#pragma unroll
    for (int i = 0; i < DP_ROWS; ++i) {
        const int64_t row = row0 + i * groups;
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
        if (row >= n) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += g[j];
        if (dP && left > 0) {
            const int64_t at = row * width + col;
            if (left >= V) {
                store_vec_any<V>(dP, at, DT, g);
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
    for (int half = groups / 2; half > 0; half /= 2) {
        for (int i = threadIdx.x; i < half * columns; i += 256) part[i] += part[i + half * columns];
        __syncthreads();
    }
    for (int i = threadIdx.x; i < columns; i += 256)
        if (blockIdx.y * columns + i < static_cast<unsigned>(width)) sums[static_cast<int64_t>(blockIdx.x) * width + blockIdx.y * columns + i] = part[i];
}

// db = sum of the rows' sums: 16 columns a workgroup, 64 threads a column (20 000 x 768: 16 of them 5.8 us, 64 4.6).
constexpr int DB_THREADS = 1024;
__global__ __launch_bounds__(DB_THREADS) void linear_db_kernel(int parts, int width, const float *__restrict__ sums, void *db, int dtype)
{
    constexpr int EACH = DB_THREADS / 16;
    __shared__ float part[EACH][17];
    const int c = threadIdx.x & 15, sub = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float x = 0.f;
    if (col < width) {
#pragma unroll 8
        for (int p = sub; p < parts; p += EACH) x += sums[static_cast<int64_t>(p) * width + col];
    }
    part[sub][c] = x;
    __syncthreads();
    if (sub < 4) {
        x = 0.f;
#pragma unroll
        for (int k = 0; k < EACH / 4; ++k) x += part[sub * (EACH / 4) + k][c];
        x += __shfl_xor(x, 16, 64);
        x += __shfl_xor(x, 32, 64);
        if (sub == 0 && col < width) store_elem(db, col, dtype, x);
    }
}

// ---- launches --------------------------------------------------------------------------------------------------
extern template void launch_dense<false, true>(const DenseArgs &a, int dtype, int tile, hipStream_t s);
extern template void launch_dense<false, false>(const DenseArgs &a, int dtype, int tile, hipStream_t s);
extern template void launch_dense<true, true>(const DenseArgs &a, int dtype, int tile, hipStream_t s);

static size_t dense_ws(int M, int N, int K)
{
    int most = 1;
    for (int v = 0; v < 4; ++v) {
        const DensePlan p = dense_plan(M, N, K, v & 1, v & 2);
        if (p.splits > most) most = p.splits;
    }
    return most > 1 ? align_up(static_cast<size_t>(most) * M * N * sizeof(float), 256) : 0;
}

template <bool AX, bool BX>
static void dense(DenseArgs a, int dtype, void *ws, hipStream_t s)
{
    if (!AX && dense_few_rows(a.M, a.N, a.K, dtype == FTC_F32, BX)) {
        launch_dense_rows(a, dtype, BX, s);
        return;
    }
    const bool fast = dense_whole_pieces(a.A, a.lda, AX ? a.M : a.K, dtype) && dense_whole_pieces(a.B, a.ldb, BX ? a.N : a.K, dtype);
    const DensePlan p = dense_plan(a.M, a.N, a.K, dtype == FTC_F32, fast);
    a.splits = p.splits;
    a.k_each = p.k_each;
    a.part = static_cast<float *>(ws);
    launch_dense<AX, BX>(a, dtype, p.tile, s);
    if (p.splits > 1) {
        // a lane a result where there are many, eight for a few results of many parts.  us with one / eight, bf16: 300 x 2000 -> 300 in eight parts
        // 13.6 / 11.3, 1000 x 3000 -> 100 in twelve 16.7 / 13.3, 512 x 4096 -> 1024 in four 15.9 / 17.8, 768 x 20 000 -> 768 in twelve 50.5 / 51.5
        const int64_t results = static_cast<int64_t>(a.M) * ceil_div(a.N, 8);
        const bool many = results >= (1 << 15) || p.splits < 8;
        const dim3 grid(static_cast<unsigned>(((many ? results : 8 * results) + 255) / 256));
#define FTC_JOIN(T)                                                                                \
    do {                                                                                           \
        if (many) hipLaunchKernelGGL((dense_join_kernel<T, 1>), grid, dim3(256), 0, s, a);          \
        else hipLaunchKernelGGL((dense_join_kernel<T, 8>), grid, dim3(256), 0, s, a);               \
    } while (0)
        if (dtype == FTC_F32) FTC_JOIN(F32);
        else if (dtype == FTC_F16) FTC_JOIN(F16);
        else FTC_JOIN(BF16);
#undef FTC_JOIN
    }
}

static void add_dense_size(LaunchSize &z, int M, int N, int K)
{
    for (int v = 0; v < 4; ++v) {
        const DensePlan p = dense_plan(M, N, K, v & 1, v & 2);
        z.add(dense_tiles(M, N, p.tile) * (p.tile == DENSE_256 ? 512 : 256), p.splits);
    }
    if (M <= 4) z.add(16ll * N, 1);  // linear_rows.hip
    z.add(static_cast<int64_t>(M) * ceil_div(N, 8), 1);  // the join of parts
}
// Of ftc_linear, and of its backward pass.
LaunchSize linear_size(int n, int d_in, int d_out)
{
    LaunchSize z;
    add_dense_size(z, n, d_out, d_in);
    return z;
}
LaunchSize linear_backward_size(int n, int d_in, int d_out)
{
    LaunchSize z;
    add_dense_size(z, n, d_in, d_out);
    add_dense_size(z, d_in, d_out, n);
    for (int vec = 4; vec <= 8; vec *= 2) {
        const int lanes = dp_lanes(d_out, vec);
        z.add(256ll * ceil_div(n, dp_rows(lanes)), ceil_div(d_out, vec << lanes));
    }
    z.add(DB_THREADS / 16ll * d_out, 1);
    return z;
}

size_t linear_ws(int n, int d_in, int d_out) { return dense_ws(n, d_out, d_in); }

static size_t linear_sums_bytes(int n, int d_out)
{
    const int rows = dp_rows(dp_lanes(d_out, 4));  // those of fp32 are at most as many as those of 16 bits
    return align_up(static_cast<size_t>(ceil_div(n, rows)) * d_out * sizeof(float), 256);
}

size_t linear_backward_ws(int n, int d_in, int d_out)
{
    const size_t x = dense_ws(n, d_in, d_out), w = dense_ws(d_in, d_out, n);
    return align_up(static_cast<size_t>(n) * d_out * sizeof(float), 256) + linear_sums_bytes(n, d_out) + (x > w ? x : w);
}

int32_t launch_linear(const LinearShape &p, void *ws, hipStream_t s)
{
    DenseArgs a = {};
    a.A = p.X; a.lda = p.ldx; a.B = p.W; a.ldb = p.d_out;
    a.M = p.n; a.N = p.d_out; a.K = p.d_in;
    a.bias = p.bias; a.act = p.act; a.residual = p.residual; a.ldr = p.ldr;
    a.slope = p.slope; a.lds = p.lds; a.out = p.Z; a.ldo = p.ldz; a.out_dtype = p.z_dtype;
    dense<false, true>(a, p.dtype, ws, s);
    return launch_status("linear");
}

template <class T>
static void linear_backward_t(const LinearShape &p, const LinearGrads &g, void *ws, hipStream_t s)
{
    char *q = static_cast<char *>(ws);
    void *dP = q; q += align_up(static_cast<size_t>(p.n) * p.d_out * sizeof(float), 256);
    float *sums = reinterpret_cast<float *>(q); q += linear_sums_bytes(p.n, p.d_out);
    const int lanes = dp_lanes(p.d_out, T::VEC), parts = ceil_div(p.n, dp_rows(lanes));
    const void *G = p.slope ? dP : g.dZ;
    const int64_t ldg = p.slope ? p.d_out : g.lddz;
    if (p.slope || g.db) {
        const dim3 grid(parts, ceil_div(p.d_out, T::VEC << lanes));
        if (p.n > 0) hipLaunchKernelGGL(linear_dp_kernel<T>, grid, dim3(256), 0, s, p.n, p.d_out, g.dZ, static_cast<int64_t>(g.lddz), p.slope,
                           static_cast<int64_t>(p.lds), p.slope ? dP : nullptr, g.db ? sums : nullptr, lanes);
    }
    if (g.db)
        hipLaunchKernelGGL(linear_db_kernel, dim3(ceil_div(p.d_out, 16)), dim3(DB_THREADS), 0, s, parts, p.d_out, sums, g.db, g.dw_dtype);
    if (g.dX && p.n > 0) {
        DenseArgs a = {};
        a.A = G; a.lda = ldg; a.B = p.W; a.ldb = p.d_out;
        a.M = p.n; a.N = p.d_in; a.K = p.d_out;
        a.residual = g.dX_add; a.ldr = g.ldda; a.out = g.dX; a.ldo = g.lddx; a.out_dtype = g.dx_dtype;
        dense<false, false>(a, p.dtype, q, s);
    }
    if (g.dW) {
        DenseArgs a = {};
        a.A = p.X; a.lda = p.ldx; a.B = G; a.ldb = ldg;
        a.M = p.d_in; a.N = p.d_out; a.K = p.n;
        a.out = g.dW; a.ldo = p.d_out; a.out_dtype = g.dw_dtype;
        dense<true, true>(a, p.dtype, q, s);
    }
}

int32_t launch_linear_backward(const LinearShape &p, const LinearGrads &g, void *ws, hipStream_t s)
{
    if (p.dtype == FTC_F32) linear_backward_t<F32>(p, g, ws, s);
    else if (p.dtype == FTC_F16) linear_backward_t<F16>(p, g, ws, s);
    else linear_backward_t<BF16>(p, g, ws, s);
    return launch_status("linear backward");
}

}  // namespace ftc
