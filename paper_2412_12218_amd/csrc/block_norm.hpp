// Rows of the norms around a block (block_norm.hip, block_norm_backward.hip): which lanes have a row, its sums, its statistics.
//
// A row is in the registers of L lanes, C pieces of eight numbers each, lane l having the pieces l, l + L, ...; it is read once whatever is computed
// of it.  Up to 64 lanes are lanes of one wave and their sums stay in registers; more are waves of one workgroup, whose sums meet in LDS.
#pragma once
#include "matrix_frag.hpp"

namespace ftc {

constexpr int row_threads(int lanes) { return lanes > 64 ? lanes : 256; }  // of a workgroup

struct BlockArgs {
    int n, d, post, pre;
    float eps, x_scale;
    const void *X, *F, *gate, *post_w, *post_b, *pre_w, *pre_b;
    int64_t ldx, ldf, ldg;  // ldg: 0 where all rows have one gate
};

#if defined(__HIPCC__)

// Totals of K sums over the L lanes of a row, in each of them.  `area`: 2 x K x 16 floats of LDS, `turn`: which half, the other one at the next call
// (a wave that writes a half again has passed the barrier of the call between, and so have all that read it).
template <int L, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float *area, int &turn)
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if constexpr (L >= 64) v[k] += __shfl_xor(v[k], 32, 64);
        v[k] = group_sum_dpp<(L < 64 ? L : 32)>(v[k]);
    }
    if constexpr (L > 64) {
        constexpr int WAVES = L / 64;
        const int wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;  // of the row
        float *half = area + turn * K * 16;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) half[k * 16 + wave] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[k] += half[k * 16 + first + w];
        }
        turn ^= 1;
    }
}

// A lane's C pieces of rows of d numbers.  WHOLE: d is a multiple of eight, so a piece is there or it is not.
template <class T, int L, int C, bool WHOLE>
struct RowPieces {
    int d, lane;
    __device__ __forceinline__ int col(int c) const { return 8 * (c * L + lane); }
    __device__ __forceinline__ int left(int c) const { return d - col(c); }
    __device__ __forceinline__ bool has(int c, int j) const { return WHOLE ? left(c) > 0 : j < left(c); }
    // there: whether there is such a row
    __device__ __forceinline__ void load(const void *base, int64_t at, bool there, Frag<T> (&f)[C]) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (WHOLE) f[c] = load_frag<T>(base, at + col(c), there && left(c) > 0 ? 8 : 0);
            else f[c] = load_frag<T>(base, at + col(c), there ? left(c) : 0);
        }
    }
    __device__ __forceinline__ void store(void *base, int64_t at, bool there, const float (&x)[C][8]) const
    {
        constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (WHOLE) {
                if (there && left(c) > 0) store_eight_numbers(base, at + col(c), DT, 8, x[c]);
            } else {
                if (there) store_eight_numbers(base, at + col(c), DT, left(c), x[c]);
            }
        }
    }
};

// Mean (0 for FTC_NORM_RMS) of a row and what its distance from there is multiplied by.  The squares are those of the distances, from registers, so
// a mean that is large beside the spread costs nothing.  Distances from 1e19 on, whose squares are infinite in fp32, once more times 2^-96.
template <class T, int L, int C, bool WHOLE>
__device__ __forceinline__ void row_statistics(const RowPieces<T, L, C, WHOLE> &r, int kind, float eps, const float (&x)[C][8], float *area, int &turn, float &mean, float &rstd)
{
    const float each = 1.f / static_cast<float>(r.d);
    mean = 0.f;
    if (kind == FTC_NORM_LAYER) {  // uniform
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] = fmaf(x[c][j], each, s[0]);  // zeros behind the row; no sum beyond the largest number
        row_sums<L, 1>(s, area, turn);
        mean = s[0];
    }
    auto squares = [&](float scale) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = r.has(c, j) ? (x[c][j] - mean) * scale : 0.f;
                s[0] = fmaf(v, v, s[0]);
            }
        row_sums<L, 1>(s, area, turn);
        return s[0] * each;
    };
    const float s = squares(1.f);
    rstd = 1.f / sqrtf(s + eps);
    // lanes that meet in row_sums go the same way: those of a wave, or of a workgroup, which has one row then
    const bool wide = s == INFINITY;
    if (L > 64 ? wide : __builtin_amdgcn_ballot_w64(wide) != 0) {
        const float t = squares(0x1p-96f);
        if (wide) rstd = 0x1p-96f / sqrtf(t);
    }
}

#endif  // __HIPCC__
}  // namespace ftc
