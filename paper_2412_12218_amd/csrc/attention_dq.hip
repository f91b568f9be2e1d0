// Attention between all nodes of a graph: the kernel of dQ.  See attention_common.hpp.
//
// delta' = <dO, out> carries the rounding of a 16-bit out, which in dQ shows beside that of ds (D = 8, graphs of 65 to 140 nodes: 1.62 times
// the error of a result that is only rounded; 1.5 without it).  What is wrong with it is the sum of ds, which should be zero:
// delta = delta' + sum_j ds'_j, which the dK / dV kernel finds in its place, and dQ = scale (sum_j ds'_j k_j - (sum_j ds'_j) sum_j p_j k_j), for which
// the kernels with D up to 32 add up p k in one more product (keys in parts: attention_settle_kernel puts the sums together; D = 64, 48 x 400 nodes: 1.46 times the error without and 1.43 with it, but
// 75 and 93 us).  Where one tile holds all keys delta is the sum of
// p <dO, v> from the start: one key gives ds = 0 exactly.
//
// Measured as the forward kernel: D = 64 73 us, 400 TFLOP/s; D = 128 1040 us, 936 TFLOP/s (three products).
#include "attention_common.hpp"

namespace ftc {

template <class T, int DP, int NW>
constexpr bool scores_kept() { return key_rows<T, NW>() == 32 || DP == 32; }

template <class T, int DP, int NW, bool WHOLE>
__global__ __launch_bounds__(64 * NW, DP == 128 && (T::BYTES == 4 || NW == 1) ? 1 : 2) void attention_dq_kernel(AttnArgs a)
{
    constexpr int TQ = 32 * NW, TK = key_rows<T, NW>(), SUB = TK / 32, KS = DP / 16, DT = DP / 32, BUFFERS = tile_buffers<NW>();
    typedef LdsTile<T, DP> L;
    typedef Keys<T, DP, TK, 64 * NW, WHOLE> Tiles;
    __shared__ __align__(16) char Ks[BUFFERS][Tiles::BYTES], Vs[BUFFERS][Tiles::BYTES];
    __shared__ __align__(16) float biases[BUFFERS][TK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const Place here = place_of(a);
    const Tile tile = find_tile<TQ>(a.q_ptr, a.graphs, a.n_q, a.group, here.tile, a.tiles);
    if (tile.graph < 0) return;
    const int q0 = tile.begin, q1 = tile.end;
    const int rows = (q1 - q0) * a.group;
    if (q1 <= q0 || static_cast<int64_t>(tile.index) * TQ >= rows) return;
    const bool same = a.kv_ptr == a.q_ptr && a.n_kv == a.n_q;  // uniform
    const int k0 = same ? q0 : clamped(a.kv_ptr, tile.graph, a.n_kv), k1 = same ? q1 : clamped(a.kv_ptr, tile.graph + 1, a.n_kv);
    const int keys = max(k1 - k0, 0), tiles = (keys + TK - 1) / TK;
    const int each = (tiles + a.splits - 1) / a.splits, first = here.part * each, last = min(tiles, first + each);

    Tiles next;
    next.look(a, k0 + first * TK, first < last ? k1 : 0);
    const int r = tile.index * TQ + wave * 32 + col;
    const bool there = r < rows, busy = tile.index * TQ + wave * 32 < rows;  // busy: uniform in the wave, which has rows
    int query, head;
    split_row(a, there ? r : 0, query, head);
    query += q0;
    head += here.share * a.group;
    const char *q_row = head_of<T>(a.Q, query, a.ldq, head * a.D), *g_row = head_of<T>(a.dO, query, a.lddo, head * a.D);
    Frag<T> q[KS], g[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + 8 * half;
        q[s] = operand_at<T, WHOLE>(q_row, c, a.D, there);
        g[s] = operand_at<T, WHOLE>(g_row, c, a.D, there);
    }
    // scale has the sign of + (turn_query), which the -infinity of hidden keys keeps
    const float scale2 = size_of_scale(a);
    const int64_t at = static_cast<int64_t>(query) * a.heads + head;
    const float lse = there ? a.lse[at] : -INFINITY;
    const float minus_lse2 = lse == -INFINITY ? -INFINITY : -lse * LOG2E;  // a row without keys has no probabilities
    float delta = there && tiles > 1 ? a.delta[at] : 0.f;
    constexpr bool MEAN = ds_in_two<T, DP>();
    f32x16 dq[DT], mean[MEAN ? DT : 1];  // mean: sum of p k
    float rest = 0.f;                    // sum of ds (a half's keys)
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[d] = zero16();
    if constexpr (MEAN) {
#pragma unroll
        for (int d = 0; d < DT; ++d) mean[d] = zero16();
    }

    // p and <dO, v> of 32 keys
    auto scores = [&](const char *K, const char *V, const float *bias, int u, f32x16 &p, f32x16 &dp) {
        p = bias_of(bias + 32 * u, half);
        dp = zero16();
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            mma<T>(p, L::along_row(K + 32 * u * L::ROW, col, 2 * k + half), q[k]);
            mma<T>(dp, L::along_row(V + 32 * u * L::ROW, col, 2 * k + half), g[k]);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], scale2, minus_lse2));
    };
    // delta of a row whose keys are all here, from p and <dO, v> of SUB 32 keys, which are kept where they fit in registers
    auto settle = [&](auto get_scores) {
        float sum = 0.f, d = 0.f;
        f32x16 p, dp;
#pragma unroll (scores_kept<T, DP, NW>() ? key_rows<T, NW>() / 32 : 1)
        for (int u = 0; u < SUB; ++u) {
            get_scores(u, p, dp);
#pragma unroll
            for (int e = 0; e < 16; ++e) sum += p[e];
        }
        sum = both_halves_sum(sum);
#pragma unroll (scores_kept<T, DP, NW>() ? key_rows<T, NW>() / 32 : 1)
        for (int u = 0; u < SUB; ++u) {
            get_scores(u, p, dp);
#pragma unroll
            for (int e = 0; e < 16; ++e) d = p[e] != 0.f ? fmaf(p[e] / sum, dp[e], d) : d;
        }
        delta = both_halves_sum(d);
        if (there && half == 0) a.delta[at] = delta;
    };
    auto gather = [&](const char *K, int u, const f32x16 &p, f32x16 &ds) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            ds[e] = p[e] * (ds[e] - delta);
            if constexpr (MEAN) rest += ds[e];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Frag<T> df = operand_of<T>(ds, k);
            Frag<T> pf, low;
            if constexpr (MEAN) pf = operand_of<T>(p, k);
            const bool two = ds_in_two<T, DP>() || (T::BYTES == 2 && NW == 1 && tiles == 1);
            if (two) low = rest_of<T>(ds, k, df);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const Frag<T> kf = L::along_column(K + (32 * u + 16 * k) * L::ROW, 4 * half, 4 * half + 8, 32 * d);
                mma<T>(dq[d], kf, df);
                if (two) mma<T>(dq[d], kf, low);
                if constexpr (MEAN) mma<T>(mean[d], kf, pf);
            }
        }
    };
    auto attend = [&](const char *K, const char *V, const float *bias) {
        if (!busy) return;
        if constexpr (scores_kept<T, DP, NW>()) {
            f32x16 p[SUB], dp[SUB];
#pragma unroll
            for (int u = 0; u < SUB; ++u) scores(K, V, bias, u, p[u], dp[u]);
            if (tiles == 1) settle([&](int u, f32x16 &x, f32x16 &y) { x = p[u]; y = dp[u]; });
#pragma unroll
            for (int u = 0; u < SUB; ++u) gather(K, u, p[u], dp[u]);
        } else {
            if (tiles == 1) settle([&](int u, f32x16 &x, f32x16 &y) { scores(K, V, bias, u, x, y); });
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                f32x16 p, dp;
                scores(K, V, bias, u, p, dp);
                gather(K, u, p, dp);
            }
        }
    };
    auto get = [&](int t, char *K, char *V, float *bias) {
        if (t >= last) return;
        next.get(a, K, V, bias, k0 + t * TK, keys - t * TK, here.share);
        next.look(a, k0 + (t + 1) * TK, k1);
    };
    auto put = [&](int t, char *K, char *V, float *bias) {
        if (t < last) next.put(a, K, V, bias);
        if constexpr (WHOLE) wait_for_lds_loads();
        __syncthreads();
    };
    for (int b = 0; b < BUFFERS; ++b) Tiles::clear(a, Ks[b], Vs[b]);
    if (WHOLE && a.D < DP) __syncthreads();
    // the first tile is on its way before the query is waited for, except through the registers of a single wave
    constexpr bool EARLY = WHOLE || BUFFERS == 2;
    if constexpr (EARLY) get(first, Ks[0], Vs[0], biases[0]);
    turn_query<T>(q, a.scale);
    if constexpr (BUFFERS == 1) {
        for (int t = first; t < last; ++t) {
            if constexpr (!EARLY) get(t, Ks[0], Vs[0], biases[0]);
            put(t, Ks[0], Vs[0], biases[0]);
            attend(Ks[0], Vs[0], biases[0]);
            __syncthreads();
            if constexpr (EARLY) get(t + 1, Ks[0], Vs[0], biases[0]);
        }
    } else {
        // one buffer is read while the next tile is on its way to the other (restrict: its arrival need not be waited for before)
        auto turn = [&](int t, const char *__restrict__ K, const char *__restrict__ V, const float *__restrict__ bias, char *__restrict__ Kn,
                        char *__restrict__ Vn, float *__restrict__ bias_n) {
            get(t + 1, Kn, Vn, bias_n);
            attend(K, V, bias);
            put(t + 1, Kn, Vn, bias_n);
        };
        put(first, Ks[0], Vs[0], biases[0]);
        for (int t = first, b = 0; t < last; ++t, b ^= 1) turn(t, Ks[b], Vs[b], biases[b], Ks[b ^ 1], Vs[b ^ 1], biases[b ^ 1]);
    }
    if (MEAN && tiles > 1 && a.splits == 1) {
        rest = both_halves_sum(rest);
        if (there && half == 0) a.delta[at] = delta + rest;
#pragma unroll
        for (int d = 0; d < DT; ++d) dq[d] -= rest * mean[MEAN ? d : 0];
    }
    if (MEAN && a.splits > 1) rest = both_halves_sum(rest);
    if (!there) return;
    const int64_t part = static_cast<int64_t>(here.part) * a.n_q * a.heads + at;
    const bool none = lse == -INFINITY;  // without a key dq is zero, and not what hidden ones, zeros in LDS, make of a query of NaN or infinities
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int c = 32 * d + 8 * b + 4 * half;
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = none ? 0.f : dq[d][4 * b + i] * a.scale;
            if (a.splits > 1) store_four<F32>(a.part, part * a.D + c, a.D - c, x);
            else store_four<T>(a.dQ, query * a.lddq + head * a.D + c, a.D - c, x);
            if constexpr (MEAN) {
                if (a.splits > 1) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = none ? 0.f : mean[d][4 * b + i] * a.scale;
                    store_four<F32>(a.part_mean, part * a.D + c, a.D - c, x);
                }
            }
        }
    if (MEAN && a.splits > 1 && half == 0) a.part_rest[part] = none || tiles == 1 ? 0.f : rest;
}

template <class T, int DP, int NW>
constexpr int attention_dq_kernel_threads() { return 64 * NW; }

void launch_attention_dq(const AttnArgs &a, int dtype, int nw, bool whole, unsigned grid, hipStream_t s) { FTC_ATTN_TYPES(attention_dq_kernel); }

}  // namespace ftc
