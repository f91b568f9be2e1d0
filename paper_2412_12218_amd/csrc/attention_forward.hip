// Attention between all nodes of a graph: the forward kernel.  See attention_common.hpp.
//
// A workgroup has 32 queries a wave and walks over the keys of their graph in tiles, the next one on its way to LDS while
// this one is multiplied.
//
// Bound by the exponentials and what a softmax does beside the products for D up to 64 (48 graphs of 1 to 799 nodes, 8 heads, D = 64, bf16 62 us, 313
// TFLOP/s), for D = 128 by both (5 graphs of 1 to 7999 nodes, 12 heads over 4, fp16 805 us, 806 TFLOP/s); readouts by the rows' bytes (12 graphs of 1 to 19 999 nodes, 17 us, 3.6 TB/s,
// and 4 to join 39 parts); batches of small graphs by the latency of three dependent loads a workgroup (2000 molecules, fp32 38 us).
#include "attention_common.hpp"

namespace ftc {

// Five waves a SIMD for the narrowest heads in 16 bits (48 graphs of 1 to 799 nodes, 8 heads, D = 32, bf16 38 us; with four 43).
template <class T, int DP, int NW, bool WHOLE>
__global__ __launch_bounds__(64 * NW, T::BYTES == 4 && DP == 128 ? 1 : T::BYTES == 2 && DP == 32 && WHOLE ? 5 : 2) void attention_forward_kernel(AttnArgs a)
{
#pragma clang fp contract(off)  // m scale2 is the same rounded number wherever it is used
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
    const int rows = (q1 - q0) * a.group;  // virtual rows of the graph
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
    // scale has the sign of + (turn_query): the maximum of the products is then that of the scores
    const float scale2 = size_of_scale(a);
    const char *q_row = head_of<T>(a.Q, query, a.ldq, head * a.D);
    Frag<T> q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + 8 * half;
        q[s] = operand_at<T, WHOLE>(q_row, c, a.D, there);
    }
    float m = -INFINITY, l = 0.f;  // maximum of the products, sum of the exponentials (a half's keys)
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = zero16();

    auto attend = [&](const char *K, const char *V, const float *bias) {
        if (!busy) return;
        f32x16 s[SUB];
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            s[u] = bias_of(bias + 32 * u, half);
#pragma unroll
            for (int k = 0; k < KS; ++k) mma<T>(s[u], L::along_row(K + 32 * u * L::ROW, col, 2 * k + half), q[k]);
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
        }
        const float m_new = fmaxf(m, both_halves_max(top)), shift = m_new == -INFINITY ? 0.f : m_new * scale2;
        if (__builtin_amdgcn_ballot_w64(m_new != m)) {
            // between the shifts that the exponentials were and will be taken with, as they are rounded: exactly one where the maximum stays
            // (fma(m, scale2, -shift) is the residue of a rounding there, which each tile that another row of the wave needs it for would leave in l and o: lse off by 6e-4 after 8000 keys, 1e-5 so)
            const float fade = __builtin_amdgcn_exp2f(m * scale2 - shift);
            l *= fade;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= fade;
            m = m_new;
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[u][e] = __builtin_amdgcn_exp2f(fmaf(s[u][e], scale2, p_bits<T>() - shift));
                l += s[u][e];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Frag<T> p = operand_of<T>(s[u], k);
#pragma unroll
                for (int d = 0; d < DT; ++d) mma<T>(o[d], L::along_column(V + (32 * u + 16 * k) * L::ROW, 4 * half, 4 * half + 8, 32 * d), p);
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
    l = both_halves_sum(l);
    // A query that holds NaN or an infinity makes NaN of hidden keys, which are zeros in LDS.  Where a key is seen the row is NaN anyway; where none is, as
    // in a graph of padding, the row has no weights.
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(l != l) != 0, 0)) {
        bool sees = false;
        const int end = min(k1, k0 + last * TK);
        for (int j = k0 + first * TK + lane; j < end; j += 64) sees = sees || !a.mask || a.mask[j];
        if (!__builtin_amdgcn_ballot_w64(sees)) {
            m = -INFINITY;
            l = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = zero16();
        }
    }
    m *= scale2;
    if (!there) return;
    if (a.splits > 1) {
        const int64_t row = (static_cast<int64_t>(here.part) * a.n_q + query) * a.heads + head;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int c = 32 * d + 8 * b + 4 * half;
                const float x[4] = {o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
                store_four<F32>(a.part, row * a.D + c, a.D - c, x);
            }
        if (half == 0) {
            a.part_ml[2 * row] = m;
            a.part_ml[2 * row + 1] = l;
        }
        return;
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int c = 32 * d + 8 * b + 4 * half;
            const float x[4] = {o[d][4 * b] * inv, o[d][4 * b + 1] * inv, o[d][4 * b + 2] * inv, o[d][4 * b + 3] * inv};
            store_four<T>(a.out, query * a.ldo + head * a.D + c, a.D - c, x);
        }
    if (a.lse && half == 0) a.lse[static_cast<int64_t>(query) * a.heads + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l) - p_bits<T>()) * LN2;
}

template <class T, int DP, int NW>
constexpr int attention_forward_kernel_threads() { return 64 * NW; }

void launch_attention_forward(const AttnArgs &a, int dtype, int nw, bool whole, unsigned grid, hipStream_t s) { FTC_ATTN_TYPES(attention_forward_kernel); }

}  // namespace ftc
