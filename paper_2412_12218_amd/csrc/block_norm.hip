// The norms around a block, with its gate and its residual connection, in one pass over the rows:
//   p = Npost(F),  h = x_scale X + gate p,  u = Npre(h),  N(t) = (t - mean) / sqrt(mean((t - mean)^2) + eps) w + b   (RMS: without the mean).
// All of a row is in registers (block_norm.hpp); h is normalised before it is rounded.
//
// Bound by memory: 50 000 x 1024 in fp16 with both norms and a gate 75 us (410 MB at 5.4 TB/s; a copy with the same hint reaches 6.3, without 5.6), 46 000 x 200 in fp32, one
// norm, 13 us (74 MB, in cache in part), 20 000 x 768 in bf16 with two layer norms 35 (123 MB at 3.5 TB/s: four sums across the two waves of a row, in which 96 of 128 lanes have numbers; two of
// them are of two numbers, as a mean in two steps has it, 2 us).  Rows above 4096, layer norms and biases around a block: 8000 x 4100 in fp32 105 us, 2000 x 16 384 203.  A row is a lane's eight numbers wide, not more: two pieces a lane (one wave a row of 1024) take as long, with three waves a SIMD instead of
// four.  What is not kept: registers for F in a norm without a block (66 instead of 131 in fp32, 13 us for 19).
#include <algorithm>

#include "block_norm.hpp"

namespace ftc {

// BLOCK: with F
template <class T, int L, int C, bool BLOCK, bool WHOLE, bool NT>
__global__ __launch_bounds__(row_threads(L)) void block_norm_kernel(BlockArgs a, void *H, int64_t ldh, void *U, int64_t ldu, float *stats)
{
    constexpr int GROUPS = row_threads(L) / L;
    __shared__ float area[64];
    int turn = 0;
    const RowPieces<T, L, C, WHOLE, NT> r = {a.d, static_cast<int>(threadIdx.x) % L, L < 64 ? static_cast<int>(threadIdx.x) / L : __builtin_amdgcn_readfirstlane(threadIdx.x / L)};
    auto scaled = [&](float (&x)[C][8], float mean, float rstd, const float (&w)[C][8], const float (&b)[C][8]) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[c][j] = fmaf((x[c][j] - mean) * rstd, w[c][j], b[c][j]);
    };
    // the next rows are on their way while these are worked on
    const int64_t step = static_cast<int64_t>(gridDim.x) * GROUPS;
    Frag<T> next_x[C], next_f[C], next_gate[C];
    r.clear(next_x);
    r.clear(next_f);
    r.clear(next_gate);
    auto fetch = [&](int64_t row0) {
        const bool there = row0 + r.sub < a.n;
        if (row0 + GROUPS > a.n) {  // uniform
            r.clear(next_x);
            r.clear(next_f);
        }
        r.load(a.X, a.ldx, row0, there, next_x);
        if (BLOCK) r.load(a.F, a.ldf, row0, there, next_f);
        if (BLOCK && a.ldg) r.load(a.gate, a.ldg, row0, there, next_gate);
    };
    fetch(static_cast<int64_t>(blockIdx.x) * GROUPS);
    Frag<T> raw_post_w[C], raw_post_b[C], raw_pre_w[C], raw_pre_b[C], raw_gate[C];
    r.fetch(a.post_w, raw_post_w);
    r.fetch(a.post_b, raw_post_b);
    r.fetch(a.pre_w, raw_pre_w);
    r.fetch(a.pre_b, raw_pre_b);
    r.fetch(a.ldg ? nullptr : a.gate, raw_gate);
    float post_w[C][8], post_b[C][8], pre_w[C][8], pre_b[C][8], one_gate[C][8];
    r.vector(a.post_w, raw_post_w, 1.f, post_w);
    r.vector(a.post_b, raw_post_b, 0.f, post_b);
    r.vector(a.pre_w, raw_pre_w, 1.f, pre_w);
    r.vector(a.pre_b, raw_pre_b, 0.f, pre_b);
    r.vector(a.ldg ? nullptr : a.gate, raw_gate, 1.f, one_gate);
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * GROUPS; row0 < a.n; row0 += step) {
        const bool there = row0 + r.sub < a.n;
        float h[C][8], p[C][8], gate[C][8], m[4] = {0.f, 1.f, 0.f, 1.f};
        r.numbers(next_x, h);
        r.numbers(next_f, p);
        if (BLOCK && a.ldg) {
            r.numbers(next_gate, gate);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) gate[c][j] = one_gate[c][j];
        }
        if (row0 + step < a.n) fetch(row0 + step);
        if constexpr (BLOCK) {
            if (a.post != FTC_NORM_NONE) {
                row_statistics(r, a.post, a.eps, p, area, turn, m[0], m[1]);
                scaled(p, m[0], m[1], post_w, post_b);
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    h[c][j] = fmaf(a.x_scale, h[c][j], gate[c][j] * p[c][j]);
                    if (!r.has(c, j)) h[c][j] = 0.f;
                }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) h[c][j] *= a.x_scale;
        }
        if (H) r.store(H, ldh, row0, there, h);
        if (a.pre != FTC_NORM_NONE) {
            row_statistics(r, a.pre, a.eps, h, area, turn, m[2], m[3]);
            if (U) {
                scaled(h, m[2], m[3], pre_w, pre_b);
                r.store(U, ldu, row0, there, h);
            }
        }
        if (stats && there && r.lane == 0) *reinterpret_cast<ftc_f32x4 *>(stats + 4 * (row0 + r.sub)) = ftc_f32x4{m[0], m[1], m[2], m[3]};
    }
}

template <class T, int L, int C, bool BLOCK>
static void forward_t(const BlockArgs &a, void *H, int ldh, void *U, int ldu, float *stats, hipStream_t s)
{
    const dim3 grid(row_groups(a.n, L, BLOCK ? 1024 : 2048)), threads(row_threads(L));
    const bool whole = a.d % T::VEC == 0, nt = row_stream(a.n, a.d, T::BYTES, {a.X, a.F, a.ldg ? a.gate : nullptr, H, U});
#define FTC_GO(WHOLE, NT) \
    hipLaunchKernelGGL((block_norm_kernel<T, L, C, BLOCK, WHOLE, NT>), grid, threads, 0, s, a, H, static_cast<int64_t>(ldh), U, static_cast<int64_t>(ldu), stats)
    if (whole && nt) FTC_GO(true, true);
    else if (whole) FTC_GO(true, false);
    else if (nt) FTC_GO(false, true);
    else FTC_GO(false, false);
#undef FTC_GO
}

int32_t launch_block_norm(const ftc_block &b, void *H, int ldh, void *U, int ldu, float *stats, hipStream_t s)
{
    const BlockArgs a = {b.n, b.d, b.F ? b.post : FTC_NORM_NONE, b.pre, b.eps, b.x_scale, b.X, b.F, b.gate, b.post_w, b.post_b, b.pre_w, b.pre_b, b.ldx, b.ldf, b.ldg};
    const int64_t lds[5] = {b.ldx, b.ldf, b.ldg, ldh, ldu};
    const int lanes = row_lanes(b.d, *std::max_element(lds, lds + 5), elem_size(b.dtype));
#define FTC_ROWS(T, L, C)                                                     \
    do {                                                                      \
        if (a.F) forward_t<T, L, C, true>(a, H, ldh, U, ldu, stats, s);       \
        else forward_t<T, L, C, false>(a, H, ldh, U, ldu, stats, s);          \
    } while (0)
#define FTC_WIDTHS(T)                                                     \
    do {                                                                  \
        switch (lanes) {                                                  \
        case 4: FTC_ROWS(T, 4, 1); break;                                 \
        case 8: FTC_ROWS(T, 8, 1); break;                                 \
        case 16: FTC_ROWS(T, 16, 1); break;                               \
        case 32: FTC_ROWS(T, 32, 1); break;                               \
        case 64: FTC_ROWS(T, 64, 1); break;                               \
        case 128: FTC_ROWS(T, 128, 1); break;                             \
        case 192: FTC_ROWS(T, 192, 1); break;                             \
        case 256: FTC_ROWS(T, 256, 1); break;                             \
        case 384: FTC_ROWS(T, 384, 1); break;                             \
        case 512:                                                         \
            if (b.d <= 4096) FTC_ROWS(T, 512, 1);                         \
            else FTC_ROWS(T, 512, 2);                                     \
            break;                                                        \
        default: FTC_ROWS(T, 1024, 2);                                    \
        }                                                                 \
    } while (0)
    if (b.dtype == FTC_F32) FTC_WIDTHS(F32);
    else if (b.dtype == FTC_F16) FTC_WIDTHS(F16);
    else FTC_WIDTHS(BF16);
#undef FTC_WIDTHS
#undef FTC_ROWS
    return launch_status("block norm");
}

}  // namespace ftc
