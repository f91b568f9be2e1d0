// Products of a few rows: Z = X W (W across the contraction) and dX = dP W^T (W along it).  What they cost is reading W once, and one
// launch, so the whole contraction of a result stays in one workgroup (wave) on the vector units.  dense_few_rows() (dense_plan.hpp) says which
// products come here, with the times of both sides; tiles of 64 rows there have the contraction in parts and a second kernel.
#include "dense_kernel.hpp"

namespace ftc {

// ---- W across: 512 threads have 8 * LANES columns, LANES lanes of 8 columns each for every row of W that the others skip ----------------
constexpr int ROWS_THREADS = 512, ROWS_STAGE = 4096;  // numbers of X in LDS
template <class T, int R, int LANES>
__global__ __launch_bounds__(ROWS_THREADS) void dense_rows_across_kernel(DenseArgs a)
{
    constexpr int SLICES = ROWS_THREADS / LANES, STAGE = ROWS_STAGE / R, WAVES = ROWS_THREADS / 64, AHEAD = 4;
    __shared__ __align__(16) float xs[ROWS_STAGE], part[WAVES][LANES][R * 8];
    const int lane = threadIdx.x % LANES, slice = threadIdx.x / LANES, col = (blockIdx.x * LANES + lane) * 8, left = a.N - col;
    float acc[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[r][j] = 0.f;
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    for (int base = 0; base < a.K; base += STAGE) {
        const int count = min(STAGE, a.K - base);
        __syncthreads();
        for (int i = threadIdx.x; i < count * R; i += ROWS_THREADS) {
            const int r = i / count, k = i % count;
            xs[k * R + r] = r < a.M ? load_elem(a.A, r * a.lda + base + k, DT) : 0.f;
        }
        __syncthreads();
        for (int k0 = slice; k0 < count; k0 += SLICES * AHEAD) {
            Frag<T> w[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int k = k0 + i * SLICES;
                w[i] = load_frag<T>(a.B, (base + k) * a.ldb + col, k < count ? left : 0);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int k = k0 + i * SLICES;
                if (k >= count) break;
                float f[8];
                frag_numbers<T>(w[i], f);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[r][j] = fmaf(xs[k * R + r], f[j], acc[r][j]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int m = LANES; m < 64; m *= 2) acc[r][j] += __shfl_xor(acc[r][j], m, 64);
            if ((threadIdx.x & 63) < LANES) part[threadIdx.x / 64][lane][r * 8 + j] = acc[r][j];
        }
    __syncthreads();
    const int row = threadIdx.x / LANES;
    if (row >= a.M || left <= 0) return;  // row: of the result now
    float x[8], bias[8];
    load_eight_numbers<T>(a.bias, col, a.bias ? left : 0, bias);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += part[w][lane][row * 8 + j];
    epilogue<T>(a, row, col, left, bias, x);
}

// ---- W along: a wave has EACH rows of W, that is columns of the result ---------------------------------------------------------------
template <class T, int R, int EACH>
__global__ __launch_bounds__(256) void dense_rows_along_kernel(DenseArgs a)
{
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    const int lane = threadIdx.x & 63, col = (blockIdx.x * 4 + (threadIdx.x >> 6)) * EACH;
    if (col >= a.N) return;
    float acc[R][EACH];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < EACH; ++e) acc[r][e] = 0.f;
#pragma unroll 2
    for (int k = lane * 8; k < a.K; k += 512) {
        const int left = a.K - k;
        Frag<T> w[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) w[e] = load_frag<T>(a.B, min(col + e, a.N - 1) * a.ldb + k, left);
        float x[R][8];
#pragma unroll
        for (int r = 0; r < R; ++r) load_eight_numbers<T>(a.A, min(r, a.M - 1) * a.lda + k, left, x[r]);
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            float f[8];
            frag_numbers<T>(w[e], f);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[r][e] = fmaf(x[r][j], f[j], acc[r][e]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            float v = acc[r][e];
            v += __shfl_xor(v, 32, 64);
            v = group_sum_dpp<32>(v);
            if (lane == r * EACH + e && r < a.M && col + e < a.N) {
                if (a.residual) v += load_elem(a.residual, r * a.ldr + col + e, DT);
                store_elem(a.out, r * a.ldo + col + e, a.out_dtype, v);
            }
        }
}

template <class T>
static void rows_t(const DenseArgs &a, bool across, hipStream_t s)
{
    if (across) {
        // 64 columns a workgroup, or 32 where that leaves compute units without one
        const bool wide = a.N >= 64 * 256;
        const dim3 grid(ceil_div(a.N, wide ? 64 : 32));
#define FTC_ROWS(R)                                                                                                             \
    do {                                                                                                                       \
        if (wide) hipLaunchKernelGGL((dense_rows_across_kernel<T, R, 8>), grid, dim3(ROWS_THREADS), 0, s, a);                   \
        else hipLaunchKernelGGL((dense_rows_across_kernel<T, R, 4>), grid, dim3(ROWS_THREADS), 0, s, a);                        \
    } while (0)
        if (a.M == 1) FTC_ROWS(1);
        else FTC_ROWS(2);
#undef FTC_ROWS
    } else {
        const dim3 grid(ceil_div(a.N, 16));
        if (a.M == 1) hipLaunchKernelGGL((dense_rows_along_kernel<T, 1, 4>), grid, dim3(256), 0, s, a);
        else if (a.M == 2) hipLaunchKernelGGL((dense_rows_along_kernel<T, 2, 4>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((dense_rows_along_kernel<T, 4, 4>), grid, dim3(256), 0, s, a);
    }
}

void launch_dense_rows(const DenseArgs &a, int dtype, bool across, hipStream_t s)
{
    if (dtype == FTC_F32) rows_t<F32>(a, across, s);
    else if (dtype == FTC_F16) rows_t<F16>(a, across, s);
    else rows_t<BF16>(a, across, s);
}

}  // namespace ftc
