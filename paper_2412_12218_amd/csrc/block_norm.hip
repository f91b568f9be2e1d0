// The norms around a block, with its gate and its residual connection, in one pass over the rows:
//   p = Npost(F),  h = x_scale X + gate p,  u = Npre(h),  N(t) = (t - mean) / sqrt(mean((t - mean)^2) + eps) w + b   (RMS: without the mean).
// All of a row is in registers (block_norm.hpp); h is normalised before it is rounded.
#include "block_norm.hpp"

namespace ftc {

template <class T, int L, int C, bool WHOLE>
__global__ __launch_bounds__(row_threads(L)) void block_norm_kernel(BlockArgs a, void *H, int64_t ldh, void *U, int64_t ldu, float *stats)
{
    constexpr int GROUPS = row_threads(L) / L;
    __shared__ float area[32];
    int turn = 0;
    const RowPieces<T, L, C, WHOLE> r = {a.d, static_cast<int>(threadIdx.x) % L};
    const int sub = threadIdx.x / L;
    // weights: from memory once, for all rows
    Frag<T> post_w[C], post_b[C], pre_w[C], pre_b[C], gate[C];
    r.load(a.post_w, 0, a.post_w != nullptr, post_w);
    r.load(a.post_b, 0, a.post_b != nullptr, post_b);
    r.load(a.pre_w, 0, a.pre_w != nullptr, pre_w);
    r.load(a.pre_b, 0, a.pre_b != nullptr, pre_b);
    r.load(a.gate, 0, a.gate && a.ldg == 0, gate);
    auto scaled = [&](float (&x)[C][8], float mean, float rstd, const void *w, const Frag<T> (&wf)[C], const Frag<T> (&bf)[C]) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float wn[8], bn[8];
            frag_numbers<T>(wf[c], wn);
            frag_numbers<T>(bf[c], bn);  // zeros where there are none
#pragma unroll
            for (int j = 0; j < 8; ++j) x[c][j] = fmaf((x[c][j] - mean) * rstd, w ? wn[j] : 1.f, bn[j]);
        }
    };
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * GROUPS; row0 < a.n; row0 += static_cast<int64_t>(gridDim.x) * GROUPS) {
        const int64_t row = row0 + sub;
        const bool there = row < a.n;
        Frag<T> x[C], f[C];
        r.load(a.X, row * a.ldx, there, x);
        r.load(a.F, row * a.ldf, there && a.F, f);
        if (a.ldg) r.load(a.gate, row * a.ldg, there, gate);
        float h[C][8], m[4] = {0.f, 1.f, 0.f, 1.f};
        if (a.F) {
            float p[C][8];
#pragma unroll
            for (int c = 0; c < C; ++c) frag_numbers<T>(f[c], p[c]);
            if (a.post != FTC_NORM_NONE) {
                row_statistics(r, a.post, a.eps, p, area, turn, m[0], m[1]);
                scaled(p, m[0], m[1], a.post_w, post_w, post_b);
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float xn[8], g[8];
                frag_numbers<T>(x[c], xn);
                frag_numbers<T>(gate[c], g);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[c][j] = r.has(c, j) ? fmaf(a.x_scale, xn[j], a.gate ? g[j] * p[c][j] : p[c][j]) : 0.f;
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                frag_numbers<T>(x[c], h[c]);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[c][j] *= a.x_scale;
            }
        }
        if (H) r.store(H, row * ldh, there, h);
        if (a.pre != FTC_NORM_NONE) {
            row_statistics(r, a.pre, a.eps, h, area, turn, m[2], m[3]);
            if (U) {
                scaled(h, m[2], m[3], a.pre_w, pre_w, pre_b);
                r.store(U, row * ldu, there, h);
            }
        }
        if (stats && there && r.lane == 0) *reinterpret_cast<ftc_f32x4 *>(stats + 4 * row) = ftc_f32x4{m[0], m[1], m[2], m[3]};
    }
}

template <class T, int L, int C>
static void forward_t(const BlockArgs &a, void *H, int ldh, void *U, int ldu, float *stats, hipStream_t s)
{
    constexpr int THREADS = row_threads(L), GROUPS = THREADS / L, MOST = 256 * 2048 / THREADS;
    const int64_t groups = (static_cast<int64_t>(a.n) + GROUPS - 1) / GROUPS;
    const dim3 grid(static_cast<unsigned>(groups < MOST ? groups : MOST));
    if (a.d % 8 == 0) hipLaunchKernelGGL((block_norm_kernel<T, L, C, true>), grid, dim3(THREADS), 0, s, a, H, static_cast<int64_t>(ldh), U, static_cast<int64_t>(ldu), stats);
    else hipLaunchKernelGGL((block_norm_kernel<T, L, C, false>), grid, dim3(THREADS), 0, s, a, H, static_cast<int64_t>(ldh), U, static_cast<int64_t>(ldu), stats);
}

int32_t launch_block_norm(const ftc_block &b, void *H, int ldh, void *U, int ldu, float *stats, hipStream_t s)
{
    const BlockArgs a = {b.n, b.d, b.F ? b.post : FTC_NORM_NONE, b.pre, b.eps, b.x_scale, b.X, b.F, b.gate, b.post_w, b.post_b, b.pre_w, b.pre_b, b.ldx, b.ldf, b.ldg};
#define FTC_ROWS(T, L, C) forward_t<T, L, C>(a, H, ldh, U, ldu, stats, s)
#define FTC_WIDTHS(T)                                \
    do {                                             \
        if (b.d <= 32) FTC_ROWS(T, 4, 1);            \
        else if (b.d <= 64) FTC_ROWS(T, 8, 1);       \
        else if (b.d <= 128) FTC_ROWS(T, 16, 1);     \
        else if (b.d <= 256) FTC_ROWS(T, 32, 1);     \
        else if (b.d <= 512) FTC_ROWS(T, 64, 1);     \
        else if (b.d <= 1024) FTC_ROWS(T, 128, 1);   \
        else if (b.d <= 2048) FTC_ROWS(T, 256, 1);   \
        else if (b.d <= 4096) FTC_ROWS(T, 512, 1);   \
        else if (b.d <= 8192) FTC_ROWS(T, 512, 2);   \
        else FTC_ROWS(T, 1024, 2);                   \
    } while (0)
    if (b.dtype == FTC_F32) FTC_WIDTHS(F32);
    else if (b.dtype == FTC_F16) FTC_WIDTHS(F16);
    else FTC_WIDTHS(BF16);
#undef FTC_WIDTHS
#undef FTC_ROWS
    return launch_status("block norm");
}

}  // namespace ftc
