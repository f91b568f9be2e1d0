// Gradients of the norms around a block.  With h and p computed again from the inputs and the statistics that the forward pass kept, fh, hh the
// normalised rows and mean() that of a row,
//   dh = dH + Npre'(dU),  dX = x_scale dh,  dgate = dh p,  dp = gate dh,  dF = Npost'(dp),
//   N'(g) = rstd (g w - mean(g w xh) xh - mean(g w)),  dw = sum over the rows of g xh,  db = sum of g   (RMS: without the mean of g w).
// A workgroup keeps the sums over its rows in registers, adds them up over its row groups and writes one row of each; a second kernel adds
// these in order.
#include "block_norm.hpp"

namespace ftc {

enum { SUM_GATE = 0, SUM_POST_W, SUM_POST_B, SUM_PRE_W, SUM_PRE_B, SUMS };

struct BlockGradArgs {
    const float *stats;
    const void *dH, *dU;
    void *dX, *dF, *dgate;  // dgate: rows; one gate of all rows is a sum
    int64_t lddh, lddu, lddx, lddf, lddg;
    float *part[SUMS];  // gridDim.x rows of d each, or NULL
};

template <class T, int L, int C, bool WHOLE>
__global__ __launch_bounds__(row_threads(L)) void block_norm_backward_kernel(BlockArgs a, BlockGradArgs g)
{
    constexpr int THREADS = row_threads(L), GROUPS = THREADS / L;
    __shared__ float area[64];
    __shared__ __align__(16) float joined[GROUPS > 1 ? THREADS * C * 8 : 1];
    int turn = 0;
    const RowPieces<T, L, C, WHOLE> r = {a.d, static_cast<int>(threadIdx.x) % L};
    const int sub = threadIdx.x / L;
    const float each = 1.f / static_cast<float>(a.d);
    Frag<T> post_w[C], post_b[C], pre_w[C], gate[C];
    r.load(a.post_w, 0, a.post_w != nullptr, post_w);
    r.load(a.post_b, 0, a.post_b != nullptr, post_b);
    r.load(a.pre_w, 0, a.pre_w != nullptr, pre_w);
    r.load(a.gate, 0, a.gate && a.ldg == 0, gate);
    float sum[SUMS][C][8];
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[k][c][j] = 0.f;
    // N'(gr) for the weights wf, its sums on the way; gr is replaced
    auto back = [&](int kind, const float (&xh)[C][8], float rstd, const void *w, const Frag<T> (&wf)[C], float (&sw)[C][8], float (&sb)[C][8], float (&gr)[C][8]) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float wn[8];
            frag_numbers<T>(wf[c], wn);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sw[c][j] = fmaf(gr[c][j], xh[c][j], sw[c][j]);
                sb[c][j] += gr[c][j];
                if (w) gr[c][j] *= wn[j];
                s[0] = fmaf(gr[c][j], xh[c][j], s[0]);
                s[1] += gr[c][j];
            }
        }
        row_sums<L, 2>(s, area, turn);
        s[0] *= each;
        s[1] = kind == FTC_NORM_LAYER ? s[1] * each : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) gr[c][j] = r.has(c, j) ? rstd * (gr[c][j] - fmaf(xh[c][j], s[0], s[1])) : 0.f;
    };
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * GROUPS; row0 < a.n; row0 += static_cast<int64_t>(gridDim.x) * GROUPS) {
        const int64_t row = row0 + sub;
        const bool there = row < a.n;
        Frag<T> x[C], f[C], dh[C], du[C];
        r.load(a.X, row * a.ldx, there, x);
        r.load(a.F, row * a.ldf, there && a.F, f);
        r.load(g.dH, row * g.lddh, there && g.dH, dh);
        r.load(g.dU, row * g.lddu, there && g.dU, du);
        if (a.ldg) r.load(a.gate, row * a.ldg, there, gate);
        ftc_f32x4 m = {0.f, 0.f, 0.f, 0.f};
        if (there && g.stats) m = *reinterpret_cast<const ftc_f32x4 *>(g.stats + 4 * row);
        // numbers behind a row's end are zeros all the way: normalised ones are made so
        float fh[C][8], p[C][8], hh[C][8], gr[C][8];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float xn[8], gn[8], w[8], b[8];
            frag_numbers<T>(x[c], xn);
            frag_numbers<T>(f[c], fh[c]);
            frag_numbers<T>(gate[c], gn);
            frag_numbers<T>(post_w[c], w);
            frag_numbers<T>(post_b[c], b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (a.post != FTC_NORM_NONE) {
                    fh[c][j] = r.has(c, j) ? (fh[c][j] - m[0]) * m[1] : 0.f;
                    p[c][j] = fmaf(fh[c][j], a.post_w ? w[j] : 1.f, b[j]);
                } else {
                    p[c][j] = fh[c][j];
                }
                float h = a.x_scale * xn[j];
                if (a.F) h = fmaf(a.x_scale, xn[j], a.gate ? gn[j] * p[c][j] : p[c][j]);
                hh[c][j] = r.has(c, j) ? (h - m[2]) * m[3] : 0.f;
            }
            frag_numbers<T>(du[c], gr[c]);
        }
        if (a.pre != FTC_NORM_NONE) back(a.pre, hh, m[3], a.pre_w, pre_w, sum[SUM_PRE_W], sum[SUM_PRE_B], gr);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float v[8];
            frag_numbers<T>(dh[c], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) gr[c][j] += v[j];  // dh now
        }
        if (g.dX) {
            float v[C][8];
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = a.x_scale * gr[c][j];
            r.store(g.dX, row * g.lddx, there, v);
        }
        if (!a.F) continue;
        if (a.gate) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float gn[8];
                frag_numbers<T>(gate[c], gn);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[c][j] *= gr[c][j];  // dgate
                    sum[SUM_GATE][c][j] += p[c][j];
                    gr[c][j] *= gn[j];
                }
            }
            if (g.dgate) r.store(g.dgate, row * g.lddg, there, p);
        }
        if (a.post != FTC_NORM_NONE) back(a.post, fh, m[1], a.post_w, post_w, sum[SUM_POST_W], sum[SUM_POST_B], gr);
        if (g.dF) r.store(g.dF, row * g.lddf, there, gr);
    }
#pragma unroll
    for (int k = 0; k < SUMS; ++k) {
        if (!g.part[k]) continue;  // uniform
        float *to = g.part[k] + static_cast<int64_t>(blockIdx.x) * a.d;
        if constexpr (GROUPS == 1) {
#pragma unroll
            for (int c = 0; c < C; ++c) store_eight_numbers(to, r.col(c), FTC_F32, r.left(c), sum[k][c]);
        } else {
            constexpr int COLS = L * C * 8;
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; j += 4)
                    *reinterpret_cast<ftc_f32x4 *>(joined + sub * COLS + r.col(c) + j) = ftc_f32x4{sum[k][c][j], sum[k][c][j + 1], sum[k][c][j + 2], sum[k][c][j + 3]};
            __syncthreads();
            for (int i = threadIdx.x; i < COLS && i < a.d; i += THREADS) {
                float v = 0.f;
                for (int q = 0; q < GROUPS; ++q) v += joined[q * COLS + i];
                to[i] = v;
            }
        }
    }
}

// Sums of the workgroups' rows: 16 columns a workgroup, 64 threads a column.
struct BlockSums {
    const float *part[SUMS];
    void *out[SUMS];
};
constexpr int SUM_THREADS = 1024;
__global__ __launch_bounds__(SUM_THREADS) void block_norm_sums_kernel(int parts, int d, BlockSums a, int dtype)
{
    constexpr int EACH = SUM_THREADS / 16;
    __shared__ float part[EACH][17];
    const float *from = nullptr;
    void *out = nullptr;
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
        if (static_cast<int>(blockIdx.y) == k) {
            from = a.part[k];
            out = a.out[k];
        }
    if (!out) return;  // uniform
    const int c = threadIdx.x & 15, sub = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float x = 0.f;
    if (col < d) {
#pragma unroll 8
        for (int p = sub; p < parts; p += EACH) x += from[static_cast<int64_t>(p) * d + col];
    }
    part[sub][c] = x;
    __syncthreads();
    if (sub < 4) {
        x = 0.f;
#pragma unroll
        for (int k = 0; k < EACH / 4; ++k) x += part[sub * (EACH / 4) + k][c];
        x += __shfl_xor(x, 16, 64);
        x += __shfl_xor(x, 32, 64);
        if (sub == 0 && col < d) store_elem(out, col, dtype, x);
    }
}

// Workgroups of a launch, which are the rows of the sums' parts.
static int backward_groups(int n, int lanes)
{
    const int threads = row_threads(lanes), most = 256 * 512 / threads, groups = ceil_div(n, threads / lanes);
    return groups < most ? groups : most;
}
static int lanes_of(int d)
{
    int lanes = 4;
    while (lanes < 512 && lanes * 8 < d) lanes *= 2;
    return d > 8192 ? 1024 : lanes;
}

size_t block_norm_backward_ws(int n, int d)
{
    return align_up(static_cast<size_t>(SUMS) * backward_groups(n, lanes_of(d)) * d * sizeof(float), 256);
}

template <class T, int L, int C>
static void backward_t(const BlockArgs &a, const BlockGradArgs &g, int groups, hipStream_t s)
{
    constexpr int THREADS = row_threads(L);
    if (a.d % 8 == 0) hipLaunchKernelGGL((block_norm_backward_kernel<T, L, C, true>), dim3(groups), dim3(THREADS), 0, s, a, g);
    else hipLaunchKernelGGL((block_norm_backward_kernel<T, L, C, false>), dim3(groups), dim3(THREADS), 0, s, a, g);
}

int32_t launch_block_norm_backward(const ftc_block &b, const float *stats, const void *dH, int lddh, const void *dU, int lddu,
                                   const ftc_block_grads &g, void *ws, hipStream_t s)
{
    const BlockArgs a = {b.n, b.d, b.F ? b.post : FTC_NORM_NONE, b.pre, b.eps, b.x_scale, b.X, b.F, b.gate, b.post_w, b.post_b, b.pre_w, b.pre_b, b.ldx, b.ldf, b.ldg};
    const bool rows = b.gate && b.ldg != 0;
    const int groups = backward_groups(b.n, lanes_of(b.d));
    BlockGradArgs k = {stats, dH, dU, g.dX, g.dF, rows ? g.dgate : nullptr, lddh, lddu, g.lddx, g.lddf, g.lddg, {}};
    BlockSums sums = {};
    void *const outs[SUMS] = {rows ? nullptr : g.dgate, g.dpost_w, g.dpost_b, g.dpre_w, g.dpre_b};
    bool any = false;
    for (int i = 0; i < SUMS; ++i) {
        if (!outs[i]) continue;
        any = true;
        sums.out[i] = outs[i];
        sums.part[i] = k.part[i] = static_cast<float *>(ws) + static_cast<size_t>(i) * groups * b.d;
    }
    if (b.n > 0) {
#define FTC_ROWS(T, L, C) backward_t<T, L, C>(a, k, groups, s)
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
    }
    if (any) hipLaunchKernelGGL(block_norm_sums_kernel, dim3(ceil_div(b.d, 16), SUMS), dim3(SUM_THREADS), 0, s, b.n > 0 ? groups : 0, b.d, sums, g.dw_dtype);
    return launch_status("block norm backward");
}

}  // namespace ftc
