// Attention between all nodes of a graph, over a batch of graphs packed one behind the other, and its gradients.
//
// For the queries i and the unmasked keys j of one graph, head by head:
//   s_ij = scale <q_i, k_j>,  lse_i = log sum_j exp(s_ij),  p_ij = exp(s_ij - lse_i),  out_i = sum_j p_ij v_j
//   delta_i = sum_j p_ij <dO_i, v_j> = <dO_i, out_i>,  ds_ij = p_ij (<dO_i, v_j> - delta_i)
//   dV_j = sum_i p_ij dO_i,  dQ_i = scale sum_j ds_ij k_j,  dK_j = scale sum_i ds_ij q_i
// Nothing of the size queries x keys is ever in memory: the forward pass keeps the maximum and the sum of a row while it
// walks over the keys, the backward pass computes the probabilities again from lse.
//
// A wave has 32 columns of every product it takes part in (see matrix_frag.hpp): 32 queries in the forward and dQ kernels,
// whose scores come as S^T (keys x queries), so that maximum, sum, lse and delta are one number a lane and the probabilities
// are the second product's operand as they lie; 32 keys in the dK / dV kernel, whose scores come as S (queries x keys) for the
// same reason.  The other side goes through LDS in tiles that all waves of a workgroup share.  Query heads that share a
// K/V head are rows of the same tiles ("virtual rows": query r / group, head r % group), so a tile of K and V serves them all.
//
// dQ and dK / dV are sums over different axes; two kernels (seven products a pair for five) add them up in a fixed order, where one would need
// atomics.  Few queries (keys) and long graphs: the other axis is split over workgroups, whose parts join_*() adds up, in order.
//
// Probabilities and ds are rounded to the type of the inputs for the second product; scores, softmax statistics and sums are fp32.
#include "matrix_frag.hpp"

namespace ftc {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct AttnArgs {
    const void *Q, *K, *V, *O, *dO;
    void *out, *dQ, *dK, *dV;
    float *lse;       // n_q x heads
    float *delta;     // n_q x heads
    float *part;      // parts of split sums
    float *part_ml;   // their maxima and sums
    const int *q_ptr, *kv_ptr;
    const uint8_t *mask;
    int64_t ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;
    int n_q, n_kv, graphs, heads, kv_heads, group, D, splits;
    float scale;
};

// Tile b of the tiles of all graphs: graph g has its tiles from [ptr[g] mult / rows] + g on, which leaves room for the rows of
// every graph without a pass over the lengths.  Wave-uniform; a 64-way search.  -1: no graph.
struct Tile {
    int graph, index;
};
__device__ __forceinline__ int clamped(const int *ptr, int i, int n)
{
    const int v = ptr[i];
    return v < 0 ? 0 : v > n ? n : v;
}
__device__ __forceinline__ Tile find_tile(const int *__restrict__ ptr, int graphs, int n, int mult, int rows, int b)
{
    const int lane = threadIdx.x & 63;
    auto start = [&](int g) { return static_cast<int>(static_cast<int64_t>(clamped(ptr, g, n)) * mult / rows) + g; };
    int lo = 0, hi = graphs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, g = lo + lane * step;
        const uint64_t below = __builtin_amdgcn_ballot_w64(g < hi && start(g) <= b);
        const int count = __popcll(below);
        const int next = lo + (count > 0 ? count - 1 : 0) * step;
        hi = min(hi, next + step);
        lo = next;
    }
    Tile t;
    const int s = start(lo);
    t.graph = __builtin_amdgcn_readfirstlane(s <= b ? lo : -1);
    t.index = __builtin_amdgcn_readfirstlane(b - s);
    return t;
}

// A tile of ROWS rows of a matrix on its way to LDS: loaded into registers a tile ahead.
template <class T, int DP, int ROWS, int THREADS>
struct Staged {
    static constexpr int PIECES = LdsTile<T, DP>::PIECES, EACH = ROWS * PIECES / THREADS;
    static_assert(ROWS * PIECES % THREADS == 0, "whole pieces a thread");
    ftc_u32x4 v[EACH];
    // row(r): element index of row r of the tile, negative: a row of zeros
    template <class Row>
    __device__ __forceinline__ void load(const void *base, int D, Row row)
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * THREADS + static_cast<int>(threadIdx.x), r = id / PIECES, c = id % PIECES * T::VEC;
            const int64_t at = row(r);
            v[e] = load_piece<T>(base, at + c, at < 0 ? 0 : D - c);
        }
    }
    __device__ __forceinline__ void store(char *tile) const
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * THREADS + static_cast<int>(threadIdx.x);
            LdsTile<T, DP>::store(tile, id / PIECES, id % PIECES, v[e]);
        }
    }
};

__device__ __forceinline__ float both_halves_max(float v) { return fmaxf(v, __shfl_xor(v, 32, 64)); }
__device__ __forceinline__ float both_halves_sum(float v) { return v + __shfl_xor(v, 32, 64); }

// Element b 4 + i of a 32-row result belongs to row 8 b + 4 half + i.
__device__ __forceinline__ int result_row(int e, int half) { return (e >> 2) * 8 + half * 4 + (e & 3); }

template <class T>
__device__ __forceinline__ Frag<T> operand_of(const f32x16 &c, int step)  // rows 16 step .. of a result as an operand
{
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = step == 0 ? c[j] : c[8 + j];
    return frag_of<T>(x);
}

// Waves a SIMD that the registers are shared out for.
template <class T, int DP, int NW>
constexpr int attn_occupancy() { return DP == 128 || (T::BYTES == 4 && NW == 1) ? 1 : 2; }

// Keys in a tile of the kernels whose waves own queries.
template <class T, int NW>
constexpr int key_rows() { return T::BYTES == 4 || NW == 1 ? 32 : 64; }

// ---- forward ------------------------------------------------------------------------------------------------
template <class T, int DP, int NW>
__global__ __launch_bounds__(64 * NW, (attn_occupancy<T, DP, NW>())) void attention_forward_kernel(AttnArgs a)
{
    constexpr int TQ = 32 * NW, TK = key_rows<T, NW>(), SUB = TK / 32, KS = DP / 16, DT = DP / 32;
    typedef LdsTile<T, DP> L;
    __shared__ __align__(16) char Ks[TK * L::ROW], Vs[TK * L::ROW];
    __shared__ __align__(16) float bias[TK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int share = blockIdx.y;
    const Tile tile = find_tile(a.q_ptr, a.graphs, a.n_q, a.group, TQ, blockIdx.x);
    if (tile.graph < 0) return;
    const int q0 = clamped(a.q_ptr, tile.graph, a.n_q), q1 = clamped(a.q_ptr, tile.graph + 1, a.n_q);
    const int rows = (q1 - q0) * a.group;  // virtual rows of the graph
    if (q1 <= q0 || static_cast<int64_t>(tile.index) * TQ >= rows) return;
    const int k0 = clamped(a.kv_ptr, tile.graph, a.n_kv), k1 = clamped(a.kv_ptr, tile.graph + 1, a.n_kv);
    const int keys = max(k1 - k0, 0), tiles = (keys + TK - 1) / TK;
    const int each = (tiles + a.splits - 1) / a.splits, first = blockIdx.z * each, last = min(tiles, first + each);

    const int r = tile.index * TQ + wave * 32 + col;
    const bool there = r < rows;
    const int query = q0 + (there ? r / a.group : 0), head = share * a.group + (there ? r % a.group : 0);
    Frag<T> q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + 8 * half;
        q[s] = load_frag<T>(a.Q, query * a.ldq + head * a.D + c, there ? a.D - c : 0);
    }
    const float scale2 = a.scale * LOG2E;
    float m = -INFINITY, l = 0.f;
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = zero16();

    Staged<T, DP, TK, 64 * NW> ks, vs;
    float kb = 0.f;
    auto fetch = [&](int t) {
        const int base = k0 + t * TK;
        auto seen = [&](int j) { return base + j < k1 && (!a.mask || a.mask[base + j]); };
        ks.load(a.K, a.D, [&](int j) { return seen(j) ? (base + j) * a.ldk + share * a.D : int64_t(-1); });
        vs.load(a.V, a.D, [&](int j) { return seen(j) ? (base + j) * a.ldv + share * a.D : int64_t(-1); });
        if (static_cast<int>(threadIdx.x) < TK) kb = seen(threadIdx.x) ? 0.f : -INFINITY;
    };
    if (first < last) fetch(first);
    for (int t = first; t < last; ++t) {
        __syncthreads();
        ks.store(Ks);
        vs.store(Vs);
        if (static_cast<int>(threadIdx.x) < TK) bias[threadIdx.x] = kb;
        __syncthreads();
        if (t + 1 < last) fetch(t + 1);
        f32x16 s[SUB];
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            s[u] = zero16();
#pragma unroll
            for (int k = 0; k < KS; ++k) mma<T>(s[u], L::along_row(Ks + 32 * u * L::ROW, col, 2 * k + half), q[k]);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const ftc_f32x4 w = *reinterpret_cast<const ftc_f32x4 *>(&bias[32 * u + 8 * b + 4 * half]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[u][4 * b + i] = fmaf(s[u][4 * b + i], scale2, w[i]);
                    top = fmaxf(top, s[u][4 * b + i]);
                }
            }
        }
        const float m_new = fmaxf(m, both_halves_max(top)), shift = m_new == -INFINITY ? 0.f : m_new;
        const float fade = __builtin_amdgcn_exp2f(m - shift);
        l *= fade;
        if (__builtin_amdgcn_ballot_w64(m_new != m)) {
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= fade;
        }
        m = m_new;
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[u][e] = __builtin_amdgcn_exp2f(s[u][e] - shift);
                l += s[u][e];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Frag<T> p = operand_of<T>(s[u], k);
                const int r0 = (32 * u + 16 * k) * L::ROW;
#pragma unroll
                for (int d = 0; d < DT; ++d) mma<T>(o[d], L::along_column(Vs + r0, 4 * half, 4 * half + 8, 32 * d), p);
            }
        }
    }
    l = both_halves_sum(l);
    if (!there) return;
    if (a.splits > 1) {
        const int64_t row = (static_cast<int64_t>(blockIdx.z) * a.n_q + query) * a.heads + head;
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
    if (a.lse && half == 0) a.lse[static_cast<int64_t>(query) * a.heads + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// Adds up the parts of the forward pass, one wave a query and head.  Rows that belong to no graph stay as they are.
__device__ __forceinline__ bool in_a_graph(const int *__restrict__ ptr, int graphs, int n, int row)
{
    return row >= clamped(ptr, 0, n) && row < clamped(ptr, graphs, n);
}
template <class T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a)
{
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6), all = static_cast<int64_t>(a.n_q) * a.heads;
    const int lane = threadIdx.x & 63;
    if (row >= all) return;
    const int query = static_cast<int>(row / a.heads), head = static_cast<int>(row % a.heads);
    if (!in_a_graph(a.q_ptr, a.graphs, a.n_q, query)) return;
    float m = -INFINITY;
    for (int z = 0; z < a.splits; ++z) m = fmaxf(m, a.part_ml[2 * (z * all + row)]);
    const float shift = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    for (int z = 0; z < a.splits; ++z) {
        const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (z * all + row));
        l += ml.y * __builtin_amdgcn_exp2f(ml.x - shift);
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    for (int c = lane; c < a.D; c += 64) {
        float x = 0.f;
        for (int z = 0; z < a.splits; ++z)
            x = fmaf(a.part[(z * all + row) * a.D + c], __builtin_amdgcn_exp2f(a.part_ml[2 * (z * all + row)] - shift), x);
        store_elem(a.out, query * a.ldo + head * a.D + c, DT, x * inv);
    }
    if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// ---- backward: delta -----------------------------------------------------------------------------------------
// 16 lanes a query and head.
template <class T>
__global__ __launch_bounds__(256) void attention_delta_kernel(AttnArgs a)
{
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4), all = static_cast<int64_t>(a.n_q) * a.heads;
    const int lane = threadIdx.x & 15;
    const bool there = row < all;
    const int query = there ? static_cast<int>(row / a.heads) : 0, head = there ? static_cast<int>(row % a.heads) : 0;
    float sum = 0.f;
    for (int c = lane * T::VEC; c < a.D; c += 16 * T::VEC) {
        const int left = there ? a.D - c : 0;
        const ftc_u32x4 x = load_piece<T>(a.O, query * a.ldo + head * a.D + c, left), y = load_piece<T>(a.dO, query * a.lddo + head * a.D + c, left);
        RawVec<T, T::VEC> u, v;
#pragma unroll
        for (int j = 0; j < 4; ++j) { u.w[j] = x[j]; v.w[j] = y[j]; }
        float f[T::VEC], g[T::VEC];
        unpack<T, T::VEC>(u, f);
        unpack<T, T::VEC>(v, g);
#pragma unroll
        for (int j = 0; j < T::VEC; ++j) sum = fmaf(f[j], g[j], sum);
    }
    sum = group_sum_dpp<16>(sum);
    if (there && lane == 0) a.delta[row] = sum;
}

// ---- backward: dQ ----------------------------------------------------------------------------------------------
// delta = <dO, out> carries the rounding of out.  Where one tile holds all keys of a graph it is the sum of p <dO, v> instead, in fp32,
// which the dK / dV kernel then finds in its place: one key gives ds = 0 exactly, and few keys, whose ds is small against delta, lose nothing.
template <class T, int DP, int NW>
__global__ __launch_bounds__(64 * NW, (attn_occupancy<T, DP, NW>())) void attention_dq_kernel(AttnArgs a)
{
    constexpr int TQ = 32 * NW, TK = key_rows<T, NW>(), SUB = TK / 32, KS = DP / 16, DT = DP / 32;
    typedef LdsTile<T, DP> L;
    __shared__ __align__(16) char Ks[TK * L::ROW], Vs[TK * L::ROW];
    __shared__ __align__(16) float bias[TK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int share = blockIdx.y;
    const Tile tile = find_tile(a.q_ptr, a.graphs, a.n_q, a.group, TQ, blockIdx.x);
    if (tile.graph < 0) return;
    const int q0 = clamped(a.q_ptr, tile.graph, a.n_q), q1 = clamped(a.q_ptr, tile.graph + 1, a.n_q);
    const int rows = (q1 - q0) * a.group;
    if (q1 <= q0 || static_cast<int64_t>(tile.index) * TQ >= rows) return;
    const int k0 = clamped(a.kv_ptr, tile.graph, a.n_kv), k1 = clamped(a.kv_ptr, tile.graph + 1, a.n_kv);
    const int keys = max(k1 - k0, 0), tiles = (keys + TK - 1) / TK;
    const int each = (tiles + a.splits - 1) / a.splits, first = blockIdx.z * each, last = min(tiles, first + each);

    const int r = tile.index * TQ + wave * 32 + col;
    const bool there = r < rows;
    const int query = q0 + (there ? r / a.group : 0), head = share * a.group + (there ? r % a.group : 0);
    Frag<T> q[KS], g[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + 8 * half;
        q[s] = load_frag<T>(a.Q, query * a.ldq + head * a.D + c, there ? a.D - c : 0);
        g[s] = load_frag<T>(a.dO, query * a.lddo + head * a.D + c, there ? a.D - c : 0);
    }
    const float scale2 = a.scale * LOG2E;
    const int64_t at = static_cast<int64_t>(query) * a.heads + head;
    const float lse = there ? a.lse[at] : -INFINITY;
    const float minus_lse2 = lse == -INFINITY ? -INFINITY : -lse * LOG2E;  // a row without keys has no probabilities
    float delta = there && tiles > 1 ? a.delta[at] : 0.f;
    f32x16 dq[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[d] = zero16();

    Staged<T, DP, TK, 64 * NW> ks, vs;
    float kb = 0.f;
    auto fetch = [&](int t) {
        const int base = k0 + t * TK;
        auto seen = [&](int j) { return base + j < k1 && (!a.mask || a.mask[base + j]); };
        ks.load(a.K, a.D, [&](int j) { return seen(j) ? (base + j) * a.ldk + share * a.D : int64_t(-1); });
        vs.load(a.V, a.D, [&](int j) { return seen(j) ? (base + j) * a.ldv + share * a.D : int64_t(-1); });
        if (static_cast<int>(threadIdx.x) < TK) kb = seen(threadIdx.x) ? 0.f : -INFINITY;
    };
    if (first < last) fetch(first);
    for (int t = first; t < last; ++t) {
        __syncthreads();
        ks.store(Ks);
        vs.store(Vs);
        if (static_cast<int>(threadIdx.x) < TK) bias[threadIdx.x] = kb;
        __syncthreads();
        if (t + 1 < last) fetch(t + 1);
        f32x16 p[SUB], dp[SUB];
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            p[u] = zero16();
            dp[u] = zero16();
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                mma<T>(p[u], L::along_row(Ks + 32 * u * L::ROW, col, 2 * k + half), q[k]);
                mma<T>(dp[u], L::along_row(Vs + 32 * u * L::ROW, col, 2 * k + half), g[k]);
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const ftc_f32x4 w = *reinterpret_cast<const ftc_f32x4 *>(&bias[32 * u + 8 * b + 4 * half]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    p[u][4 * b + i] = __builtin_amdgcn_exp2f(fmaf(p[u][4 * b + i], scale2, w[i] + minus_lse2));
            }
        }
        if (tiles == 1) {
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum += p[u][e];
            sum = both_halves_sum(sum);
            float d = 0.f;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) d = p[u][e] != 0.f ? fmaf(p[u][e] / sum, dp[u][e], d) : d;
            delta = both_halves_sum(d);
            if (there && half == 0) a.delta[at] = delta;
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
#pragma unroll
            for (int e = 0; e < 16; ++e) p[u][e] *= dp[u][e] - delta;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Frag<T> ds = operand_of<T>(p[u], k);
                const int r0 = (32 * u + 16 * k) * L::ROW;
#pragma unroll
                for (int d = 0; d < DT; ++d) mma<T>(dq[d], L::along_column(Ks + r0, 4 * half, 4 * half + 8, 32 * d), ds);
            }
        }
    }
    if (!there) return;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int c = 32 * d + 8 * b + 4 * half;
            const float x[4] = {dq[d][4 * b] * a.scale, dq[d][4 * b + 1] * a.scale, dq[d][4 * b + 2] * a.scale, dq[d][4 * b + 3] * a.scale};
            if (a.splits > 1) store_four<F32>(a.part, (static_cast<int64_t>(blockIdx.z) * a.n_q * a.heads + at) * a.D + c, a.D - c, x);
            else store_four<T>(a.dQ, query * a.lddq + head * a.D + c, a.D - c, x);
        }
}

// ---- backward: dK, dV ------------------------------------------------------------------------------------------
template <class T, int DP>
constexpr int query_rows() { return T::BYTES == 2 && DP <= 64 ? 64 : 32; }

template <class T, int DP, int NW>
__global__ __launch_bounds__(64 * NW, (attn_occupancy<T, DP, NW>())) void attention_dkv_kernel(AttnArgs a)
{
    constexpr int TK = 32 * NW, TQ = query_rows<T, DP>(), SUB = TQ / 32, KS = DP / 16, DT = DP / 32;
    typedef LdsTile<T, DP> L;
    __shared__ __align__(16) char Qs[TQ * L::ROW], Gs[TQ * L::ROW];
    __shared__ __align__(16) float row_lse[TQ], row_delta[TQ];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int share = blockIdx.y;
    const Tile tile = find_tile(a.kv_ptr, a.graphs, a.n_kv, 1, TK, blockIdx.x);
    if (tile.graph < 0) return;
    const int k0 = clamped(a.kv_ptr, tile.graph, a.n_kv), k1 = clamped(a.kv_ptr, tile.graph + 1, a.n_kv);
    if (k1 <= k0 || static_cast<int64_t>(tile.index) * TK >= k1 - k0) return;
    const int q0 = clamped(a.q_ptr, tile.graph, a.n_q), q1 = clamped(a.q_ptr, tile.graph + 1, a.n_q);
    const int rows = max(q1 - q0, 0) * a.group, tiles = (rows + TQ - 1) / TQ;
    const int each = (tiles + a.splits - 1) / a.splits, first = blockIdx.z * each, last = min(tiles, first + each);

    const int key = k0 + tile.index * TK + wave * 32 + col;
    const bool there = key < k1, seen = there && (!a.mask || a.mask[key]);
    Frag<T> k[KS], v[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + 8 * half;
        k[s] = load_frag<T>(a.K, (seen ? key : 0) * a.ldk + share * a.D + c, seen ? a.D - c : 0);
        v[s] = load_frag<T>(a.V, (seen ? key : 0) * a.ldv + share * a.D + c, seen ? a.D - c : 0);
    }
    const float scale2 = a.scale * LOG2E, bias = seen ? 0.f : -INFINITY;
    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) { dk[d] = zero16(); dv[d] = zero16(); }

    Staged<T, DP, TQ, 64 * NW> qs, gs;
    float my_lse = 0.f, my_delta = 0.f;
    auto fetch = [&](int t) {
        auto place = [&](int j, int64_t ld) {
            const int r = t * TQ + j;
            return r < rows ? (q0 + r / a.group) * ld + (share * a.group + r % a.group) * a.D : int64_t(-1);
        };
        qs.load(a.Q, a.D, [&](int j) { return place(j, a.ldq); });
        gs.load(a.dO, a.D, [&](int j) { return place(j, a.lddo); });
        if (static_cast<int>(threadIdx.x) < TQ) {
            const int r = t * TQ + threadIdx.x;
            my_lse = -INFINITY;
            my_delta = 0.f;
            if (r < rows) {
                const int64_t at = static_cast<int64_t>(q0 + r / a.group) * a.heads + share * a.group + r % a.group;
                const float lse = a.lse[at];
                my_lse = lse == -INFINITY ? -INFINITY : -lse * LOG2E;
                my_delta = a.delta[at];
            }
        }
    };
    if (first < last) fetch(first);
    for (int t = first; t < last; ++t) {
        __syncthreads();
        qs.store(Qs);
        gs.store(Gs);
        if (static_cast<int>(threadIdx.x) < TQ) {
            row_lse[threadIdx.x] = my_lse;
            row_delta[threadIdx.x] = my_delta;
        }
        __syncthreads();
        if (t + 1 < last) fetch(t + 1);
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            f32x16 p = zero16(), ds = zero16();
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                mma<T>(p, L::along_row(Qs + 32 * u * L::ROW, col, 2 * s + half), k[s]);
                mma<T>(ds, L::along_row(Gs + 32 * u * L::ROW, col, 2 * s + half), v[s]);
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const ftc_f32x4 w = *reinterpret_cast<const ftc_f32x4 *>(&row_lse[32 * u + 8 * b + 4 * half]);
                const ftc_f32x4 x = *reinterpret_cast<const ftc_f32x4 *>(&row_delta[32 * u + 8 * b + 4 * half]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[4 * b + i] = __builtin_amdgcn_exp2f(fmaf(p[4 * b + i], scale2, w[i] + bias));
                    ds[4 * b + i] = p[4 * b + i] * (ds[4 * b + i] - x[i]);
                }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const Frag<T> pf = operand_of<T>(p, s), df = operand_of<T>(ds, s);
                const int r0 = (32 * u + 16 * s) * L::ROW;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    mma<T>(dv[d], L::along_column(Gs + r0, 4 * half, 4 * half + 8, 32 * d), pf);
                    mma<T>(dk[d], L::along_column(Qs + r0, 4 * half, 4 * half + 8, 32 * d), df);
                }
            }
        }
    }
    if (!there) return;
    const int64_t all = static_cast<int64_t>(a.n_kv) * a.kv_heads;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int c = 32 * d + 8 * b + 4 * half;
            const float x[4] = {dk[d][4 * b] * a.scale, dk[d][4 * b + 1] * a.scale, dk[d][4 * b + 2] * a.scale, dk[d][4 * b + 3] * a.scale};
            const float y[4] = {dv[d][4 * b], dv[d][4 * b + 1], dv[d][4 * b + 2], dv[d][4 * b + 3]};
            if (a.splits > 1) {
                const int64_t row = (static_cast<int64_t>(blockIdx.z) * 2 * a.n_kv + key) * a.kv_heads + share;
                store_four<F32>(a.part, row * a.D + c, a.D - c, x);
                store_four<F32>(a.part, (row + all) * a.D + c, a.D - c, y);
            } else {
                store_four<T>(a.dK, key * a.lddk + share * a.D + c, a.D - c, x);
                store_four<T>(a.dV, key * a.lddv + share * a.D + c, a.D - c, y);
            }
        }
}

// out[row, :] = sum over the parts, for the rows of the graphs; `width` elements a row, parts `stride` elements apart.
template <class T>
__global__ __launch_bounds__(256) void attention_sum_kernel(const float *__restrict__ part, int64_t stride, int splits, const int *__restrict__ ptr,
                                                            int graphs, int n, int width, void *out, int64_t ld)
{
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int row = static_cast<int>(id / width), c = static_cast<int>(id % width);
    if (id >= static_cast<int64_t>(n) * width || !in_a_graph(ptr, graphs, n, row)) return;
    float x = 0.f;
    for (int z = 0; z < splits; ++z) x += part[z * stride + id];
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    store_elem(out, row * ld + c, DT, x);
}

// ---- launches ----------------------------------------------------------------------------------------------------
// Waves of a workgroup: one where a graph's rows are hardly more than a wave's, else four.
static int attn_waves(int64_t rows, int graphs) { return rows <= 48ll * graphs ? 1 : 4; }
static int attn_tiles(int64_t rows, int graphs, int waves) { return static_cast<int>(rows / (32 * waves)) + graphs; }
// Parts of the other axis where there are fewer workgroups than two for each compute unit; a part is four tiles at least.
static int attn_splits(int64_t rows, int64_t other, int graphs, int kv_heads)
{
    const int64_t groups = static_cast<int64_t>(attn_tiles(rows, graphs, attn_waves(rows, graphs))) * kv_heads;
    if (groups < 1) return 1;
    const int64_t want = (512 + groups - 1) / groups, most = other / 256;
    const int64_t s = want < most ? want : most;
    return static_cast<int>(s < 1 ? 1 : s > 64 ? 64 : s);
}

size_t attention_ws(int n_q, int n_kv, int graphs, int heads, int kv_heads, int D)
{
    const int64_t rows = static_cast<int64_t>(n_q) * heads;
    const int s = attn_splits(static_cast<int64_t>(n_q) * (heads / kv_heads), n_kv, graphs, kv_heads);
    if (s == 1) return 0;
    return align_up(static_cast<size_t>(s) * rows * D * sizeof(float), 256) + align_up(static_cast<size_t>(s) * rows * 2 * sizeof(float), 256);
}

size_t attention_backward_ws(int n_q, int n_kv, int graphs, int heads, int kv_heads, int D)
{
    const int64_t rows = static_cast<int64_t>(n_q) * heads, group = heads / kv_heads;
    const int sq = attn_splits(n_q * group, n_kv, graphs, kv_heads), sk = attn_splits(n_kv, n_q * group, graphs, kv_heads);
    const size_t parts_q = sq > 1 ? static_cast<size_t>(sq) * rows * D * sizeof(float) : 0;
    const size_t parts_k = sk > 1 ? static_cast<size_t>(sk) * 2 * n_kv * kv_heads * D * sizeof(float) : 0;
    return align_up(static_cast<size_t>(rows) * sizeof(float), 256) + align_up(parts_q > parts_k ? parts_q : parts_k, 256);
}

#define FTC_ATTN_WIDTHS(KERNEL, T, NW, GRID)                                                                          \
    do {                                                                                                             \
        if (a.D <= 32) hipLaunchKernelGGL((KERNEL<T, 32, NW>), GRID, dim3(64 * NW), 0, s, a);                         \
        else if (a.D <= 64) hipLaunchKernelGGL((KERNEL<T, 64, NW>), GRID, dim3(64 * NW), 0, s, a);                    \
        else hipLaunchKernelGGL((KERNEL<T, 128, NW>), GRID, dim3(64 * NW), 0, s, a);                                  \
    } while (0)
#define FTC_ATTN_LAUNCH(KERNEL, ROWS)                                                                                 \
    do {                                                                                                             \
        const int nw = attn_waves(ROWS, a.graphs);                                                                   \
        const dim3 grid(attn_tiles(ROWS, a.graphs, nw), a.kv_heads, a.splits);                                       \
        if (nw == 1) FTC_ATTN_WIDTHS(KERNEL, T, 1, grid);                                                            \
        else FTC_ATTN_WIDTHS(KERNEL, T, 4, grid);                                                                    \
    } while (0)

template <class T>
static void forward_t(AttnArgs a, void *ws, hipStream_t s)
{
    const int64_t rows = static_cast<int64_t>(a.n_q) * a.heads, virt = static_cast<int64_t>(a.n_q) * a.group;
    a.splits = attn_splits(virt, a.n_kv, a.graphs, a.kv_heads);
    a.part = static_cast<float *>(ws);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(ws) + align_up(static_cast<size_t>(a.splits) * rows * a.D * sizeof(float), 256));
    FTC_ATTN_LAUNCH(attention_forward_kernel, virt);
    if (a.splits > 1) hipLaunchKernelGGL(attention_join_kernel<T>, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, s, a);
}

template <class T>
static void backward_t(AttnArgs a, void *ws, hipStream_t s)
{
    const int64_t rows = static_cast<int64_t>(a.n_q) * a.heads, virt = static_cast<int64_t>(a.n_q) * a.group;
    a.delta = static_cast<float *>(ws);
    a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + align_up(static_cast<size_t>(rows) * sizeof(float), 256));
    if (rows > 0) {
        hipLaunchKernelGGL(attention_delta_kernel<T>, dim3(static_cast<unsigned>((rows + 15) / 16)), dim3(256), 0, s, a);
        a.splits = attn_splits(virt, a.n_kv, a.graphs, a.kv_heads);
        FTC_ATTN_LAUNCH(attention_dq_kernel, virt);
        const int width = a.heads * a.D;
        if (a.splits > 1)
            hipLaunchKernelGGL(attention_sum_kernel<T>, dim3(static_cast<unsigned>((static_cast<int64_t>(a.n_q) * width + 255) / 256)), dim3(256), 0, s,
                               a.part, static_cast<int64_t>(a.n_q) * width, a.splits, a.q_ptr, a.graphs, a.n_q, width, a.dQ, a.lddq);
    }
    if (a.n_kv > 0) {
        a.splits = attn_splits(a.n_kv, virt, a.graphs, a.kv_heads);
        FTC_ATTN_LAUNCH(attention_dkv_kernel, static_cast<int64_t>(a.n_kv));
        const int width = a.kv_heads * a.D;
        const int64_t count = static_cast<int64_t>(a.n_kv) * width;
        if (a.splits > 1) {
            const dim3 grid(static_cast<unsigned>((count + 255) / 256));
            hipLaunchKernelGGL(attention_sum_kernel<T>, grid, dim3(256), 0, s, a.part, 2 * count, a.splits, a.kv_ptr, a.graphs, a.n_kv, width, a.dK, a.lddk);
            hipLaunchKernelGGL(attention_sum_kernel<T>, grid, dim3(256), 0, s, a.part + count, 2 * count, a.splits, a.kv_ptr, a.graphs, a.n_kv, width, a.dV,
                               a.lddv);
        }
    }
}

static AttnArgs attn_args(const AttnShape &p)
{
    AttnArgs a = {};
    a.Q = p.Q; a.K = p.K; a.V = p.V;
    a.ldq = p.ldq; a.ldk = p.ldk; a.ldv = p.ldv;
    a.q_ptr = p.q_ptr; a.kv_ptr = p.kv_ptr; a.mask = p.kv_mask;
    a.n_q = p.n_q; a.n_kv = p.n_kv; a.graphs = p.graphs; a.heads = p.heads; a.kv_heads = p.kv_heads;
    a.group = p.heads / p.kv_heads; a.D = p.D; a.scale = p.scale;
    return a;
}

int32_t launch_attention(const AttnShape &p, void *out, int ldo, float *lse, void *ws, hipStream_t s)
{
    AttnArgs a = attn_args(p);
    a.out = out; a.ldo = ldo; a.lse = lse;
    if (p.dtype == FTC_F32) forward_t<F32>(a, ws, s);
    else if (p.dtype == FTC_F16) forward_t<F16>(a, ws, s);
    else forward_t<BF16>(a, ws, s);
    return launch_status("graph attention");
}

int32_t launch_attention_backward(const AttnShape &p, const void *out, int ldo, const float *lse, const void *dO, int lddo, void *dQ, int lddq,
                                  void *dK, int lddk, void *dV, int lddv, void *ws, hipStream_t s)
{
    AttnArgs a = attn_args(p);
    a.O = out; a.ldo = ldo; a.lse = const_cast<float *>(lse); a.dO = dO; a.lddo = lddo;
    a.dQ = dQ; a.lddq = lddq; a.dK = dK; a.lddk = lddk; a.dV = dV; a.lddv = lddv;
    if (p.dtype == FTC_F32) backward_t<F32>(a, ws, s);
    else if (p.dtype == FTC_F16) backward_t<F16>(a, ws, s);
    else backward_t<BF16>(a, ws, s);
    return launch_status("graph attention backward");
}

}  // namespace ftc
