// Gradients of the norms around a block.  With h and p computed again from the inputs and the statistics that the forward pass kept, fh, hh the
// normalised rows and mean() that of a row,
//   dh = dH + Npre'(dU),  dX = x_scale dh,  dgate = dh p,  dp = gate dh,  dF = Npost'(dp),
//   N'(g) = rstd (g w - mean(g w xh) xh - mean(g w)),  dw = sum over the rows of g xh,  db = sum of g   (RMS: without the mean of g w).
// A workgroup keeps the sums over its rows in registers, adds them up over its row groups and writes one row of each; a second kernel adds
// these in order.
//
// 20 000 x 768 in bf16 with layer norms, biases and a gate 46 us (184 MB at 4.0 TB/s, 430 vector instructions for eight numbers of a lane at two waves a SIMD: both count) and
// 7 for the sums; 200 000 x 128 with a gate a row 72 us (410 MB at 5.7 TB/s) and 5.
// Wide rows in fp32, layer norms and biases around a block, with the sums: 4000 x 8192 233 us (786 MB at 3.4 TB/s), 2000 x 16 384 603 (1.3 TB/s: 1024 lanes have 128 registers each, up to 1036 bytes a lane are in
// scratch memory).  One row to 300 rows of 768 in bf16: 16 us a call, two launches from Python.
#include <algorithm>

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

// BLOCK: with F
template <class T, int L, int C, bool BLOCK, bool WHOLE, bool NT>
__global__ __launch_bounds__(row_threads(L), 2) void block_norm_backward_kernel(BlockArgs a, BlockGradArgs g)
{
    constexpr int THREADS = row_threads(L), GROUPS = THREADS / L;
    constexpr bool LEAN = C > 1;  // registers: no rows ahead, weights out of the caches for every row
    __shared__ float area[64];
    __shared__ __align__(16) float joined[GROUPS > 1 ? THREADS * C * 8 : 1];
    int turn = 0;
    const RowPieces<T, L, C, WHOLE, NT> r = {a.d, static_cast<int>(threadIdx.x) % L, L < 64 ? static_cast<int>(threadIdx.x) / L : __builtin_amdgcn_readfirstlane(threadIdx.x / L)};
    const int sub = r.sub;
    const float each = 1.f / static_cast<float>(a.d);
    float post_w[C][8], post_b[C][8], pre_w[C][8], one_gate[C][8], sum[SUMS][C][8];
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[k][c][j] = 0.f;
    // N'(gr), its sums on the way; gr is replaced.  Numbers behind a row's end are zeros all the way
    auto back = [&](int kind, const float (&xh)[C][8], float rstd, const float (&w)[C][8], float (&sw)[C][8], float (&sb)[C][8], float (&gr)[C][8]) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sw[c][j] = fmaf(gr[c][j], xh[c][j], sw[c][j]);
                sb[c][j] += gr[c][j];
                gr[c][j] *= w[c][j];
                s[0] = fmaf(gr[c][j], xh[c][j], s[0]);
                s[1] += gr[c][j];
            }
        row_sums<L, 2>(s, area, turn);
        s[0] *= each;
        s[1] = kind == FTC_NORM_LAYER ? s[1] * each : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) gr[c][j] = (r.has(c, j) ? rstd : 0.f) * (gr[c][j] - fmaf(xh[c][j], s[0], s[1]));
    };
    // the next rows are on their way while these are worked on
    const int64_t step = static_cast<int64_t>(gridDim.x) * GROUPS;
    Frag<T> next_x[C], next_f[C], next_dh[C], next_du[C], next_gate[C];
    ftc_f32x4 next_m = {0.f, 0.f, 0.f, 0.f};
    r.clear(next_x);
    r.clear(next_f);
    r.clear(next_dh);
    r.clear(next_du);
    r.clear(next_gate);
    auto fetch = [&](int64_t row0) {
        const bool there = row0 + sub < a.n;
        if (row0 + GROUPS > a.n) {  // uniform: rows that are not there add nothing
            r.clear(next_x);
            r.clear(next_f);
            r.clear(next_dh);
            r.clear(next_du);
            r.clear(next_gate);
            next_m = ftc_f32x4{0.f, 0.f, 0.f, 0.f};
        }
        r.load(a.X, a.ldx, row0, there, next_x);
        if (BLOCK) r.load(a.F, a.ldf, row0, there, next_f);
        if (g.dH) r.load(g.dH, g.lddh, row0, there, next_dh);
        if (g.dU) r.load(g.dU, g.lddu, row0, there, next_du);
        if (BLOCK && a.ldg) r.load(a.gate, a.ldg, row0, there, next_gate);
        if (there && g.stats) next_m = *reinterpret_cast<const ftc_f32x4 *>(g.stats + 4 * (row0 + sub));
    };
    if constexpr (!LEAN) fetch(static_cast<int64_t>(blockIdx.x) * GROUPS);
    auto weights = [&] {
        Frag<T> raw_post_w[C], raw_post_b[C], raw_pre_w[C], raw_gate[C];
        r.fetch(a.post_w, raw_post_w);
        r.fetch(a.post_b, raw_post_b);
        r.fetch(a.pre_w, raw_pre_w);
        r.fetch(a.ldg ? nullptr : a.gate, raw_gate);
        r.vector(a.post_w, raw_post_w, 1.f, post_w);
        r.vector(a.post_b, raw_post_b, 0.f, post_b);
        r.vector(a.pre_w, raw_pre_w, 1.f, pre_w);
        r.vector(a.ldg ? nullptr : a.gate, raw_gate, 1.f, one_gate);
    };
    if constexpr (!LEAN) weights();
    // LEAN: one of them, where it is used
    auto weight = [&](const void *base, float none, float (&x)[C][8]) {
        if constexpr (LEAN) {
            asm volatile("" ::: "memory");  // not before the loop
            Frag<T> raw[C];
            r.fetch(base, raw);
            r.vector(base, raw, none, x);
        }
    };
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * GROUPS; row0 < a.n; row0 += step) {
        const bool there = row0 + sub < a.n;
        if constexpr (LEAN) fetch(row0);
        const ftc_f32x4 m = next_m;
        float fh[C][8], p[C][8], hh[C][8], gr[C][8], gate[C][8];
        Frag<T> dh[C];
        r.numbers(next_x, hh);
        r.numbers(next_f, fh);
        r.numbers(next_du, gr);
#pragma unroll
        for (int c = 0; c < C; ++c) dh[c] = next_dh[c];
        if (BLOCK && a.ldg) {
            r.numbers(next_gate, gate);
        } else {
            weight(a.gate, 1.f, one_gate);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) gate[c][j] = one_gate[c][j];
        }
        if (!LEAN && row0 + step < a.n) fetch(row0 + step);
        if (BLOCK && a.post != FTC_NORM_NONE) {
            weight(a.post_w, 1.f, post_w);
            weight(a.post_b, 0.f, post_b);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    fh[c][j] = (fh[c][j] - m[0]) * (r.has(c, j) ? m[1] : 0.f);
                    p[c][j] = fmaf(fh[c][j], post_w[c][j], post_b[c][j]);
                }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) p[c][j] = fh[c][j];
        }
        if (a.pre != FTC_NORM_NONE) {
            // as the forward pass has h
            if constexpr (BLOCK) {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) hh[c][j] = fmaf(a.x_scale, hh[c][j], gate[c][j] * p[c][j]);
            } else {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) hh[c][j] *= a.x_scale;
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) hh[c][j] = (hh[c][j] - m[2]) * (r.has(c, j) ? m[3] : 0.f);
            weight(a.pre_w, 1.f, pre_w);
            back(a.pre, hh, m[3], pre_w, sum[SUM_PRE_W], sum[SUM_PRE_B], gr);
        }
        {
            float v[C][8];
            r.numbers(dh, v);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) gr[c][j] += v[c][j];  // dh now
        }
        if (g.dX) {
            float v[C][8];
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = a.x_scale * gr[c][j];
            r.store(g.dX, g.lddx, row0, there, v);
        }
        if constexpr (!BLOCK) continue;
        if (a.gate) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[c][j] *= gr[c][j];  // dgate
                    sum[SUM_GATE][c][j] += p[c][j];
                    gr[c][j] *= gate[c][j];
                }
            if (g.dgate) r.store(g.dgate, g.lddg, row0, there, p);
        }
        if (a.post != FTC_NORM_NONE) {
            weight(a.post_w, 1.f, post_w);
            back(a.post, fh, m[1], post_w, sum[SUM_POST_W], sum[SUM_POST_B], gr);
        }
        if (g.dF) r.store(g.dF, g.lddf, row0, there, gr);
    }
#pragma unroll
    for (int k = 0; k < SUMS; ++k) {
        if (!g.part[k]) continue;  // uniform
        float *to = g.part[k] + static_cast<int64_t>(blockIdx.x) * a.d;
        if constexpr (GROUPS == 1) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (r.has(c, j)) to[r.col(c, j / T::VEC) + j % T::VEC] = sum[k][c][j];
        } else {
            constexpr int COLS = L * C * 8;
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; j += 4)
                    *reinterpret_cast<ftc_f32x4 *>(joined + sub * COLS + r.col(c, j / T::VEC) + j % T::VEC) = ftc_f32x4{sum[k][c][j], sum[k][c][j + 1], sum[k][c][j + 2], sum[k][c][j + 3]};
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
static int backward_groups(int n, int lanes) { return row_groups(n, lanes, 512); }

size_t block_norm_backward_ws(int n, int d)
{
    // narrow rows far apart have 64 lanes
    const int near = backward_groups(n, row_lanes(d, d, 4)), far = backward_groups(n, row_lanes(d, INT32_MAX, 4));
    return align_up(static_cast<size_t>(SUMS) * (near > far ? near : far) * d * sizeof(float), 256);
}

template <class T, int L, int C, bool BLOCK>
static void backward_t(const BlockArgs &a, const BlockGradArgs &g, int groups, hipStream_t s)
{
    const bool whole = a.d % T::VEC == 0, nt = row_stream(a.n, a.d, T::BYTES, {a.X, a.F, a.ldg ? a.gate : nullptr, g.dH, g.dU, g.dX, g.dF, g.dgate});
#define FTC_GO(WHOLE, NT) hipLaunchKernelGGL((block_norm_backward_kernel<T, L, C, BLOCK, WHOLE, NT>), dim3(groups), dim3(row_threads(L)), 0, s, a, g)
    if (whole && nt) FTC_GO(true, true);
    else if (whole) FTC_GO(true, false);
    else if (nt) FTC_GO(false, true);
    else FTC_GO(false, false);
#undef FTC_GO
}

int32_t launch_block_norm_backward(const ftc_block &b, const float *stats, const void *dH, int lddh, const void *dU, int lddu,
                                   const ftc_block_grads &g, void *ws, hipStream_t s)
{
    const BlockArgs a = {b.n, b.d, b.F ? b.post : FTC_NORM_NONE, b.pre, b.eps, b.x_scale, b.X, b.F, b.gate, b.post_w, b.post_b, b.pre_w, b.pre_b, b.ldx, b.ldf, b.ldg};
    const bool rows = b.gate && b.ldg != 0;
    const int64_t lds[8] = {b.ldx, b.ldf, b.ldg, lddh, lddu, g.lddx, g.lddf, g.lddg};
    const int lanes = row_lanes(b.d, *std::max_element(lds, lds + 8), elem_size(b.dtype)), groups = backward_groups(b.n, lanes);
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
#define FTC_ROWS(T, L, C)                                       \
    do {                                                        \
        if (a.F) backward_t<T, L, C, true>(a, k, groups, s);    \
        else backward_t<T, L, C, false>(a, k, groups, s);       \
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
    }
    if (any) hipLaunchKernelGGL(block_norm_sums_kernel, dim3(ceil_div(b.d, 16), SUMS), dim3(SUM_THREADS), 0, s, b.n > 0 ? groups : 0, b.d, sums, g.dw_dtype);
    return launch_status("block norm backward");
}

}  // namespace ftc
