// Dense layer with its epilogue, Z = act(X W + b) + R, and its gradients
//   dP = dZ act'(P),  dX = dP W^T,  dW = X^T dP,  db = column sums of dP   (P = X W + b).
//
// All three products run on one kernel: a workgroup of four waves computes a tile of the result, a wave 32 x 32 blocks of it
// (matrix_frag.hpp).  An operand whose memory rows run along the contraction is a tile of rows read along rows, one whose
// memory rows run across it is read along columns, so nothing is transposed in memory:
//   Z   X along, W across;   dX   dP along, W along;   dW   X across, dP across.
// A lane holds one row and four neighbouring columns of the result at a time: bias, activation, residual and the store work on
// four numbers.  Few tiles and a long contraction (a single row; a weight gradient): the contraction is split over
// workgroups, whose parts are added up in order by a second kernel, which has the epilogue then.
//
// The forward pass keeps act'(P), not P: it is between -0.13 and 1.13, so 16 bits of fixed point with 14 of fraction hold it to 2^-15
// (P in bf16 would move dP by a third of its own rounding), and the backward pass needs no activation function.  dP is rounded to the type of
// X for the products; db is the sum of the unrounded ones.
#include "matrix_frag.hpp"

namespace ftc {

constexpr int SLOPE_BITS = 14;

struct DenseArgs {
    const void *A, *B;  // M x K, K x N
    int64_t lda, ldb;
    int M, N, K, splits, k_each;
    float *part;  // splits x M x N
    const void *bias, *residual;
    void *slope, *out;
    int64_t ldr, lds, ldo;
    int act, out_dtype;
};

// act(p); slope: act'(p).  Infinite p: the limits.
__device__ __forceinline__ float activation(float p, int act, float &slope)
{
    slope = 1.f;
    if (act == FTC_ACT_RELU) {
        slope = p > 0.f ? 1.f : p != p ? p : 0.f;
        return p > 0.f ? p : p != p ? p : 0.f;
    }
    if (act == FTC_ACT_GELU) {
        const float q = p < -40.f ? -40.f : p > 40.f ? 40.f : p;
        const float cdf = 0.5f * (1.f + erff(q * 0.70710678118654752f));
        slope = cdf + q * 0.39894228040143268f * expf(-0.5f * q * q);
        return p > 40.f ? p : q * cdf;
    }
    if (act == FTC_ACT_SILU) {
        const float q = p < -80.f ? -80.f : p > 80.f ? 80.f : p;
        const float g = 1.f / (1.f + expf(-q));
        slope = g * (1.f + q * (1.f - g));
        return p > 80.f ? p : p < -80.f ? 0.f : q * g;
    }
    return p;
}

__device__ __forceinline__ int16_t slope_code(float s)
{
    return s != s ? INT16_MIN : static_cast<int16_t>(rintf(s * (1 << SLOPE_BITS)));
}
__device__ __forceinline__ float slope_value(int16_t c)
{
    return c == INT16_MIN ? __builtin_nanf("") : c * (1.f / (1 << SLOPE_BITS));
}

// Four neighbouring numbers of a row of the result.
template <class T>
__device__ __forceinline__ void epilogue(const DenseArgs &a, int row, int col, float (&x)[4])
{
    const int left = a.N - col;
    float add[4] = {0.f, 0.f, 0.f, 0.f}, slope[4];
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    if (a.bias) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) x[j] += load_elem(a.bias, col + j, DT);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = activation(x[j], a.act, slope[j]);
    if (a.residual) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) add[j] = load_elem(a.residual, row * a.ldr + col + j, DT);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] += add[j];
    if (a.slope) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) {
                if constexpr (T::BYTES == 4) static_cast<float *>(a.slope)[row * a.lds + col + j] = slope[j];
                else static_cast<int16_t *>(a.slope)[row * a.lds + col + j] = slope_code(slope[j]);
            }
    }
    if (left >= 4) {
        store_vec_any<4>(a.out, row * a.ldo + col, a.out_dtype, x);
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < left) store_elem(a.out, row * a.ldo + col + j, a.out_dtype, x[j]);
    }
}

// One operand's tile: SIDE rows of the result's side and STEP of the contraction.
template <class T, int SIDE, int STEP, bool ACROSS>
struct Operand {
    static constexpr int ROWS = ACROSS ? STEP : SIDE, COLS = ACROSS ? SIDE : STEP;
    typedef LdsTile<T, COLS> L;
    static constexpr int BYTES = ROWS * L::ROW, EACH = ROWS * L::PIECES / 256;
    static_assert(ROWS * L::PIECES % 256 == 0, "whole pieces a thread");
    ftc_u32x4 v[EACH];
    // side0, k0: the tile's first row; `side`, `k_end`: their ends
    __device__ __forceinline__ void load(const void *base, int64_t ld, int side0, int side, int k0, int k_end)
    {
        const int row0 = ACROSS ? k0 : side0, rows = ACROSS ? k_end : side, col0 = ACROSS ? side0 : k0, cols = ACROSS ? side : k_end;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * 256 + static_cast<int>(threadIdx.x), r = row0 + id / L::PIECES, c = col0 + id % L::PIECES * T::VEC;
            v[e] = load_piece<T>(base, r * ld + c, r < rows ? cols - c : 0);
        }
    }
    __device__ __forceinline__ void store(char *tile) const
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * 256 + static_cast<int>(threadIdx.x);
            L::store(tile, id / L::PIECES, id % L::PIECES, v[e]);
        }
    }
    // the 32 from side0 on, indices 16 s .. of the step
    static __device__ __forceinline__ Frag<T> frag(const char *tile, int side0, int s, int lane)
    {
        const int half = lane >> 5;
        if constexpr (ACROSS) return L::along_column(tile, 16 * s + 8 * half, 16 * s + 8 * half + 4, side0);
        else return L::along_row(tile, side0 + (lane & 31), 2 * s + half);
    }
};

// Result tiles of 64 WM x 64 WN: 2 x 2 waves of WM x WN blocks.
template <class T, bool AX, bool BX, int WM, int WN>
__global__ __launch_bounds__(256, WM * WN >= 16 ? 1 : 2) void dense_kernel(DenseArgs a)
{
    constexpr int TM = 64 * WM, TN = 64 * WN, STEP = T::BYTES == 4 ? 32 : 64, KS = STEP / 16;
    typedef Operand<T, TM, STEP, AX> OA;
    typedef Operand<T, TN, STEP, BX> OB;
    __shared__ __align__(16) char As[2][OA::BYTES], Bs[2][OB::BYTES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tiles_n = (a.N + TN - 1) / TN;
    const int m0 = static_cast<int>(blockIdx.x) / tiles_n * TM, n0 = static_cast<int>(blockIdx.x) % tiles_n * TN;
    const int wm = (wave >> 1) * 32 * WM, wn = (wave & 1) * 32 * WN;
    const int k_begin = static_cast<int>(blockIdx.y) * a.k_each, k_end = min(a.K, k_begin + a.k_each);
    f32x16 c[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) c[i][j] = zero16();
    OA oa;
    OB ob;
    oa.load(a.A, a.lda, m0, a.M, k_begin, k_end);
    ob.load(a.B, a.ldb, n0, a.N, k_begin, k_end);
    oa.store(As[0]);
    ob.store(Bs[0]);
    __syncthreads();
    int buf = 0;
    for (int k = k_begin; k < k_end; k += STEP) {
        const bool more = k + STEP < k_end;
        if (more) {
            oa.load(a.A, a.lda, m0, a.M, k + STEP, k_end);
            ob.load(a.B, a.ldb, n0, a.N, k + STEP, k_end);
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            Frag<T> fa[WM], fb[WN];
#pragma unroll
            for (int i = 0; i < WM; ++i) fa[i] = OA::frag(As[buf], wm + 32 * i, s, lane);
#pragma unroll
            for (int j = 0; j < WN; ++j) fb[j] = OB::frag(Bs[buf], wn + 32 * j, s, lane);
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int j = 0; j < WN; ++j) mma<T>(c[i][j], fb[j], fa[i]);
        }
        if (more) {
            oa.store(As[buf ^ 1]);
            ob.store(Bs[buf ^ 1]);
        }
        __syncthreads();
        buf ^= 1;
    }
#pragma unroll
    for (int i = 0; i < WM; ++i) {
        const int row = m0 + wm + 32 * i + (lane & 31);
        if (row >= a.M) continue;
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int col = n0 + wn + 32 * j + 8 * b + 4 * (lane >> 5);
                if (col >= a.N) continue;
                float x[4] = {c[i][j][4 * b], c[i][j][4 * b + 1], c[i][j][4 * b + 2], c[i][j][4 * b + 3]};
                if (a.splits > 1)
                    store_four<F32>(a.part, (static_cast<int64_t>(blockIdx.y) * a.M + row) * a.N + col, a.N - col, x);
                else
                    epilogue<T>(a, row, col, x);
            }
    }
}

template <class T>
__global__ __launch_bounds__(256) void dense_join_kernel(DenseArgs a)
{
    const int quads = (a.N + 3) / 4;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (id >= static_cast<int64_t>(a.M) * quads) return;
    const int row = static_cast<int>(id / quads), col = static_cast<int>(id % quads) * 4;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    for (int z = 0; z < a.splits; ++z) {
        const ftc_u32x4 v = load_piece<F32>(a.part, (static_cast<int64_t>(z) * a.M + row) * a.N + col, a.N - col);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += __uint_as_float(v[j]);
    }
    epilogue<T>(a, row, col, x);
}

// dP = dZ act'(P) (dP NULL: not written) and, for BIAS_ROWS rows at a time, its column sums (sums NULL: none).  A thread has the 16
// bytes of VEC columns of every eighth row.
constexpr int BIAS_ROWS = 128;
template <class T>
__global__ __launch_bounds__(256) void linear_dp_kernel(int n, int width, const void *__restrict__ dZ, int64_t ldz, const void *__restrict__ slope,
                                                        int64_t lds, void *__restrict__ dP, float *__restrict__ sums)
{
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16, V = T::VEC;
    __shared__ float part[8][32 * V];
    const int lane = threadIdx.x & 31, sub = threadIdx.x >> 5, col = (blockIdx.y * 32 + lane) * V, left = width - col;
    const int row0 = blockIdx.x * BIAS_ROWS, row1 = row0 + min(n - row0, BIAS_ROWS);
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.f;
    if (left > 0) {
#pragma unroll 4
        for (int row = row0 + sub; row < row1; row += 8) {
            const ftc_u32x4 w = load_piece<T>(dZ, row * ldz + col, left);
            RawVec<T, V> r;
#pragma unroll
            for (int j = 0; j < 4; ++j) r.w[j] = w[j];
            float g[V];
            unpack<T, V>(r, g);
            if (slope) {
                const ftc_u32x4 u = load_piece<T>(slope, row * lds + col, left);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if constexpr (T::BYTES == 4) g[j] *= __uint_as_float(u[j]);
                    else g[j] *= slope_value(static_cast<int16_t>(u[j / 2] >> (16 * (j & 1))));
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += g[j];
            if (dP) {
                const int64_t at = static_cast<int64_t>(row) * width + col;
                if (left >= V) {
                    store_vec_any<V>(dP, at, DT, g);
                } else {
#pragma unroll
                    for (int j = 0; j < V - 1; ++j)
                        if (j < left) store_elem(dP, at + j, DT, g[j]);
                }
            }
        }
    }
    if (!sums) return;
#pragma unroll
    for (int j = 0; j < V; ++j) part[sub][lane * V + j] = sum[j];
    __syncthreads();
    const int c = blockIdx.y * 32 * V + threadIdx.x;
    if (static_cast<int>(threadIdx.x) < 32 * V && c < width) {
        float x = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) x += part[k][threadIdx.x];
        sums[static_cast<int64_t>(blockIdx.x) * width + c] = x;
    }
}

// db = sum of the rows' sums: 16 columns a workgroup, 16 threads a column.
__global__ __launch_bounds__(256) void linear_db_kernel(int parts, int width, const float *__restrict__ sums, void *db, int dtype)
{
    __shared__ float part[16][17];
    const int c = threadIdx.x & 15, sub = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float x = 0.f;
    if (col < width) {
#pragma unroll 4
        for (int p = sub; p < parts; p += 16) x += sums[static_cast<int64_t>(p) * width + col];
    }
    part[sub][c] = x;
    __syncthreads();
    if (sub == 0 && col < width) {
        float y = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) y += part[k][c];
        store_elem(db, col, dtype, y);
    }
}

// ---- launches --------------------------------------------------------------------------------------------------
struct DensePlan {
    int blocks;  // 32 x 32 blocks of a wave along each side: 1 or 2
    int splits, k_each;
};

static int64_t dense_tiles(int M, int N, int blocks)
{
    const int t = 64 * blocks;
    return static_cast<int64_t>(ceil_div(M, t)) * ceil_div(N, t);
}

// The large tile where it gives every compute unit one; else the small one, and parts of the contraction of 128 indices at least
// until there are two workgroups a compute unit.
static DensePlan dense_plan(int M, int N, int K)
{
    DensePlan p = {1, 1, 64};
    if (M < 1 || N < 1) return p;
    p.blocks = dense_tiles(M, N, 2) >= 256 ? 2 : 1;
    const int64_t tiles = dense_tiles(M, N, p.blocks);
    int64_t s = tiles >= 512 ? 1 : (512 + tiles - 1) / tiles;
    const int most = K > 128 ? ceil_div(K, 128) : 1;
    if (s > most) s = most;
    if (s > 64) s = 64;
    p.k_each = static_cast<int>(align_up(K > 0 ? ceil_div(K, static_cast<int>(s)) : 1, 64));
    p.splits = K > 0 ? ceil_div(K, p.k_each) : 1;
    return p;
}
static size_t dense_ws(int M, int N, int K)
{
    const DensePlan p = dense_plan(M, N, K);
    return p.splits > 1 ? align_up(static_cast<size_t>(p.splits) * M * N * sizeof(float), 256) : 0;
}

template <class T, bool AX, bool BX>
static int32_t dense_t(DenseArgs a, void *ws, hipStream_t s)
{
    const DensePlan p = dense_plan(a.M, a.N, a.K);
    a.splits = p.splits;
    a.k_each = p.k_each;
    a.part = static_cast<float *>(ws);
    const dim3 grid(static_cast<unsigned>(dense_tiles(a.M, a.N, p.blocks)), p.splits);
    if (p.blocks == 2) hipLaunchKernelGGL((dense_kernel<T, AX, BX, 2, 2>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((dense_kernel<T, AX, BX, 1, 1>), grid, dim3(256), 0, s, a);
    if (p.splits > 1) {
        const int64_t quads = static_cast<int64_t>(a.M) * ceil_div(a.N, 4);
        hipLaunchKernelGGL(dense_join_kernel<T>, dim3(static_cast<unsigned>((quads + 255) / 256)), dim3(256), 0, s, a);
    }
    return FTC_OK;
}

size_t linear_ws(int n, int d_in, int d_out) { return dense_ws(n, d_out, d_in); }

static size_t linear_sums_bytes(int n, int d_out) { return align_up(static_cast<size_t>(ceil_div(n, BIAS_ROWS)) * d_out * sizeof(float), 256); }

size_t linear_backward_ws(int n, int d_in, int d_out)
{
    const size_t x = dense_ws(n, d_in, d_out), w = dense_ws(d_in, d_out, n);
    return align_up(static_cast<size_t>(n) * d_out * sizeof(float), 256) + linear_sums_bytes(n, d_out) + (x > w ? x : w);
}

template <class T>
static int32_t linear_t(const LinearShape &p, void *ws, hipStream_t s)
{
    DenseArgs a = {};
    a.A = p.X; a.lda = p.ldx; a.B = p.W; a.ldb = p.d_out;
    a.M = p.n; a.N = p.d_out; a.K = p.d_in;
    a.bias = p.bias; a.act = p.act; a.residual = p.residual; a.ldr = p.ldr;
    a.slope = p.slope; a.lds = p.lds; a.out = p.Z; a.ldo = p.ldz; a.out_dtype = p.z_dtype;
    return dense_t<T, false, true>(a, ws, s);
}

int32_t launch_linear(const LinearShape &p, void *ws, hipStream_t s)
{
    if (p.dtype == FTC_F32) linear_t<F32>(p, ws, s);
    else if (p.dtype == FTC_F16) linear_t<F16>(p, ws, s);
    else linear_t<BF16>(p, ws, s);
    return launch_status("linear");
}

template <class T>
static void linear_backward_t(const LinearShape &p, const LinearGrads &g, void *ws, hipStream_t s)
{
    char *q = static_cast<char *>(ws);
    void *dP = q; q += align_up(static_cast<size_t>(p.n) * p.d_out * sizeof(float), 256);
    float *sums = reinterpret_cast<float *>(q); q += linear_sums_bytes(p.n, p.d_out);
    const void *G = p.slope ? dP : g.dZ;
    const int64_t ldg = p.slope ? p.d_out : g.lddz;
    if (p.slope || g.db) {
        const dim3 grid(ceil_div(p.n, BIAS_ROWS), ceil_div(p.d_out, 32 * T::VEC));
        if (p.n > 0) hipLaunchKernelGGL(linear_dp_kernel<T>, grid, dim3(256), 0, s, p.n, p.d_out, g.dZ, static_cast<int64_t>(g.lddz), p.slope,
                           static_cast<int64_t>(p.lds), p.slope ? dP : nullptr, g.db ? sums : nullptr);
    }
    if (g.db)
        hipLaunchKernelGGL(linear_db_kernel, dim3(ceil_div(p.d_out, 16)), dim3(256), 0, s, ceil_div(p.n, BIAS_ROWS), p.d_out, sums, g.db, g.dw_dtype);
    if (g.dX && p.n > 0) {
        DenseArgs a = {};
        a.A = G; a.lda = ldg; a.B = p.W; a.ldb = p.d_out;
        a.M = p.n; a.N = p.d_in; a.K = p.d_out;
        a.out = g.dX; a.ldo = g.lddx; a.out_dtype = g.dx_dtype;
        dense_t<T, false, false>(a, q, s);
    }
    if (g.dW) {
        DenseArgs a = {};
        a.A = p.X; a.lda = p.ldx; a.B = G; a.ldb = ldg;
        a.M = p.d_in; a.N = p.d_out; a.K = p.n;
        a.out = g.dW; a.ldo = p.d_out; a.out_dtype = g.dw_dtype;
        dense_t<T, true, true>(a, q, s);
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
