// What the kernels of attention between all nodes of a graph share (graph_attention.hip: the entry points' launches).
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
// Probabilities and ds are rounded to the type of the inputs for the second product (see ds_in_two() and p_bits()); scores, softmax statistics and sums are fp32.
#pragma once
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
    float *part_mean, *part_rest;  // dQ in parts, D up to 32 in 16 bits: of p k, and of ds
    const int *q_ptr, *kv_ptr;
    const uint8_t *mask;
    int64_t ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;
    int n_q, n_kv, graphs, heads, kv_heads, group, D, splits;
    uint32_t group_magic;  // ceil(2^32 / group)
    int tiles;             // of all graphs: the workgroups of a K/V head and part
    float scale;
};

// Virtual row -> query row and head of the group: the quotient by the magic number is right or one too large (row < 2^31).
__device__ __forceinline__ void split_row(const AttnArgs &a, int row, int &query, int &head)
{
    if (a.group == 1) {
        query = row;
        head = 0;
        return;
    }
    query = static_cast<int>(__umulhi(static_cast<uint32_t>(row), a.group_magic));
    head = row - query * a.group;
    if (head < 0) {
        --query;
        head += a.group;
    }
}

// Tile b of the tiles of all graphs: graph g has its tiles from [ptr[g] mult / rows] + g on, which leaves room for the rows of
// every graph without a pass over the lengths.  Wave-uniform.  The 63 graphs around the place where b is among `tiles` are looked at first: it is one of
// them where the graphs' sizes are alike, and small graphs have little else to wait for.  Else a 64-way search.
struct Tile {
    int graph, index, begin, end;  // graph -1: none; begin, end: ptr of the graph
};
__device__ __forceinline__ int clamped(const int *ptr, int i, int n)
{
    const int v = ptr[i];
    return v < 0 ? 0 : v > n ? n : v;
}
template <int ROWS>
__device__ __forceinline__ Tile find_tile(const int *__restrict__ ptr, int graphs, int n, int mult, int b, int tiles)
{
    const int lane = threadIdx.x & 63;
    auto start = [&](int p, int g) { return static_cast<int>(static_cast<uint64_t>(p) * mult / ROWS) + g; };
    int lo = static_cast<int>(static_cast<int64_t>(b) * graphs / tiles) - 31;
    lo = max(min(lo, graphs - 63), 0);
    Tile t;
    for (int first = 0, end = graphs;;) {  // the graph is in [first, end), if there is one; twice at most
        const int g = min(lo + lane, graphs), p = clamped(ptr, g, n), s = start(p, g);
        const uint64_t below = __builtin_amdgcn_ballot_w64(g < end && s <= b);
        const int last = below ? 63 - __builtin_clzll(below) : -1;
        if ((last >= 0 || lo == first) && last < 63) {  // lane 63 does not know its graph's end
            const int at = max(last, 0);
            t.begin = __builtin_amdgcn_readlane(p, at);
            t.end = __builtin_amdgcn_readlane(p, min(at + 1, 63));
            t.index = b - __builtin_amdgcn_readlane(s, at);
            t.graph = last >= 0 ? lo + at : -1;
            return t;
        }
        if (last < 0) end = lo;
        else first = lo + 63;
        while (end - first > 63) {
            const int step = (end - first + 63) / 64, h = first + lane * step;
            const uint64_t under = __builtin_amdgcn_ballot_w64(h < end && start(clamped(ptr, h, n), h) <= b);
            first += max(__popcll(under) - 1, 0) * step;
            end = min(end, first + step);
        }
        lo = first;
    }
}

// A tile of ROWS rows in LDS, and this thread's pieces of it: piece number e * threads + thread, as it lies there.
//   WHOLE  rows of whole 16-byte pieces at 16-byte alignment go straight to LDS (global_load_lds); rows that are not to be seen are written
//          as zeros instead, columns from D on once, by clear()
//   else   through registers: get() loads, put() stores
template <class T, int DP, int ROWS, int THREADS, bool WHOLE>
struct Rows {
    typedef LdsTile<T, DP> L;
    static constexpr int BYTES = ROWS * L::ROW, EACH = BYTES / 16 / THREADS;
    static_assert(BYTES % (16 * THREADS) == 0, "whole pieces a thread");
    static __device__ __forceinline__ int row(int e) { return (e * THREADS + static_cast<int>(threadIdx.x)) / L::PIECES; }
    static __device__ __forceinline__ int col(int e)
    {
        return (((e * THREADS + static_cast<int>(threadIdx.x)) % L::PIECES) ^ L::swizzle(row(e))) * T::VEC;
    }
    static __device__ __forceinline__ ftc_u32x4 *place(char *tile, int e)
    {
        return reinterpret_cast<ftc_u32x4 *>(tile + (e * THREADS + static_cast<int>(threadIdx.x)) * 16);
    }
    static __device__ __forceinline__ void clear(char *tile, int D)
    {
        if (WHOLE && D < DP) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) *place(tile, e) = ftc_u32x4{0u, 0u, 0u, 0u};
        }
    }

    ftc_u32x4 v[WHOLE ? 1 : EACH];
    typedef typename std::conditional<WHOLE, uint32_t, int64_t>::type Offset;  // WHOLE: below 2^32 bytes (attn_whole)
    // base: the tile's rows begin there, at: this piece from there (elements), both of head columns
    __device__ __forceinline__ void get(char *tile, int e, const void *base, Offset at, int D)
    {
        if constexpr (WHOLE) {
            typedef __attribute__((address_space(3))) void *lds_ptr;
            typedef const __attribute__((address_space(1))) void *global_ptr;
            if (col(e) < D) {
                const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
                __builtin_amdgcn_global_load_lds((global_ptr)(static_cast<const char *>(base) + at * T::BYTES),
                                                 (lds_ptr)(tile + e * THREADS * 16 + wave * 1024), 16, 0, 0);
            }
        } else {
            // the last piece of a row is the last 16 bytes of the row; put() moves them, so that no load is waited for here
            if (D < T::VEC) {
                v[e] = load_piece<T>(base, at, D - col(e));
            } else {
                RawVec<T, T::VEC> r;
                load_raw_any<T>(base, at - max(col(e) + T::VEC - D, 0), r);
                v[e] = ftc_u32x4{r.w[0], r.w[1], r.w[2], r.w[3]};
            }
        }
    }
    __device__ __forceinline__ void get_zeros(char *tile, int e)
    {
        if constexpr (WHOLE) *place(tile, e) = ftc_u32x4{0u, 0u, 0u, 0u};
        else v[e] = ftc_u32x4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ void put(char *tile, int D)
    {
        if constexpr (!WHOLE) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                if (D >= T::VEC && col(e) + T::VEC > D) move_down<T>(v[e], col(e) + T::VEC - D);
                *place(tile, e) = v[e];
            }
        }
    }
};

// This wave's loads to LDS have arrived.  The barrier of several waves comes with that; a single wave has none, and the compiler does not see from one turn
// of a loop to the next that what a load writes is read.
__device__ __forceinline__ void wait_for_lds_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The first element of a row of a head, and an operand of it: elements c .. c + 7, zeros if the row is not `there`.
template <class T>
__device__ __forceinline__ const char *head_of(const void *p, int64_t row, int64_t ld, int col)
{
    return static_cast<const char *>(p) + (row * ld + col) * T::BYTES;
}
template <class T, bool WHOLE>
__device__ __forceinline__ Frag<T> operand_at(const char *row, int c, int D, bool there)
{
    Frag<T> a;
    if constexpr (!WHOLE) {
        const ftc_u32x4 x = load_piece_of_row<T>(row, c, D);
        if constexpr (T::BYTES == 4) {
            const ftc_u32x4 y = load_piece_of_row<T>(row, c + 4, D);
#pragma unroll
            for (int j = 0; j < 4; ++j) { a.f[j] = there ? __uint_as_float(x[j]) : 0.f; a.f[4 + j] = there ? __uint_as_float(y[j]) : 0.f; }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) a.w[j] = there ? x[j] : 0u;
        }
        return a;
    }
    if constexpr (T::BYTES == 4) {
        const bool x_ok = there && c < D, y_ok = there && c + 4 < D;
        const ftc_f32x4 x = *reinterpret_cast<const ftc_f32x4 *>(row + (x_ok ? c : 0) * 4), y = *reinterpret_cast<const ftc_f32x4 *>(row + (y_ok ? c + 4 : 0) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) { a.f[j] = x_ok ? x[j] : 0.f; a.f[4 + j] = y_ok ? y[j] : 0.f; }
    } else {
        const bool ok = there && c < D;
        const ftc_u32x4 x = *reinterpret_cast<const ftc_u32x4 *>(row + (ok ? c : 0) * 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) a.w[j] = ok ? x[j] : 0u;
    }
    return a;
}

// A query for a scale that is not positive: the kernels multiply by its size, so that -infinity stays what hides a key.  Zero leaves nothing of a product but NaN.
template <class T, int N>
__device__ __forceinline__ void turn_query(Frag<T> (&q)[N], float scale)
{
    if (__builtin_expect(scale > 0.f, 1)) return;  // uniform
#pragma unroll
    for (int s = 0; s < N; ++s) {
        float x[8];
        frag_numbers<T>(q[s], x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = scale < 0.f ? -x[j] : x[j] * 0.f;
        q[s] = frag_of<T>(x);
    }
}
// For exponentials in base two; a normal number, so that -infinity times it is one.
__device__ __forceinline__ float size_of_scale(const AttnArgs &a) { return fmaxf(fabsf(a.scale) * LOG2E, 0x1p-126f); }

// The keys of a graph, tile by tile, K and V with what is added to their scores (0, or -infinity for keys that are not seen).
template <class T, int DP, int TK, int THREADS, bool WHOLE>
struct Keys {
    typedef Rows<T, DP, TK, THREADS, WHOLE> R;
    static constexpr int BYTES = R::BYTES;
    R k, v;
    float mine;
    uint32_t hidden;  // by the mask: bit e of the pieces, bit 31 of the key of this thread
    static __device__ __forceinline__ void clear(const AttnArgs &a, char *K, char *V)
    {
        R::clear(K, a.D);
        R::clear(V, a.D);
    }
    // what the mask hides of a tile; a tile ahead of get(), which needs it
    __device__ __forceinline__ void look(const AttnArgs &a, int first, int end)
    {
        hidden = 0;
        if (!a.mask) return;
#pragma unroll
        for (int e = 0; e < R::EACH; ++e) {
            const int j = first + R::row(e);
            hidden |= (j < end && !a.mask[j] ? 1u : 0u) << e;
        }
        const int j = first + static_cast<int>(threadIdx.x);
        if (static_cast<int>(threadIdx.x) < TK && j < end && !a.mask[j]) hidden |= 1u << 31;
    }
    // keys first .. of which `count` are the graph's; writes the bias unless the tile is whole and nothing is hidden
    __device__ __forceinline__ void get(const AttnArgs &a, char *K, char *V, float *bias, int first, int count, int share)
    {
        static_assert(R::EACH < 31, "a bit for every piece");
        const char *kp = head_of<T>(a.K, first, a.ldk, share * a.D), *vp = head_of<T>(a.V, first, a.ldv, share * a.D);
        const typename R::Offset ldk = a.ldk, ldv = a.ldv;
        if (count >= TK && !a.mask) {
#pragma unroll
            for (int e = 0; e < R::EACH; ++e) {
                k.get(K, e, kp, R::row(e) * ldk + R::col(e), a.D);
                v.get(V, e, vp, R::row(e) * ldv + R::col(e), a.D);
            }
            mine = 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < R::EACH; ++e) {
                if (R::row(e) < count && !(hidden >> e & 1u)) {
                    k.get(K, e, kp, R::row(e) * ldk + R::col(e), a.D);
                    v.get(V, e, vp, R::row(e) * ldv + R::col(e), a.D);
                } else {
                    k.get_zeros(K, e);
                    v.get_zeros(V, e);
                }
            }
            mine = static_cast<int>(threadIdx.x) < count && !(hidden >> 31) ? 0.f : -INFINITY;
        }
        if (WHOLE && static_cast<int>(threadIdx.x) < TK) bias[threadIdx.x] = mine;
    }
    __device__ __forceinline__ void put(const AttnArgs &a, char *K, char *V, float *bias)
    {
        k.put(K, a.D);
        v.put(V, a.D);
        if (!WHOLE && static_cast<int>(threadIdx.x) < TK) bias[threadIdx.x] = mine;
    }
};

// What is added to the scores of 32 keys, as the result that their product begins with.
__device__ __forceinline__ f32x16 bias_of(const float *bias, int half)
{
    f32x16 c;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const ftc_f32x4 w = *reinterpret_cast<const ftc_f32x4 *>(&bias[8 * b + 4 * half]);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[4 * b + i] = w[i];
    }
    return c;
}

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

template <class T>
__device__ __forceinline__ Frag<T> rest_of(const f32x16 &c, int step, const Frag<T> &rounded)  // what the rounding left of them
{
    float x[8], y[8];
    frag_numbers<T>(rounded, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (step == 0 ? c[j] : c[8 + j]) - y[j];
    return frag_of<T>(x);
}

// ds adds up to zero over a row's keys, so with few columns its rounding shows more than that of the result: for D up to 32 in 16
// bits its products take what the rounding left as a second operand (dQ against 64 bits, fp16, D = 8: 1.58 times the error of a result that
// is only rounded, 1.1 so; the exponentials, not the matrix cores, bound these kernels).  So do those of any D in one wave's workgroups for graphs
// of one tile, whose few sums do not average it (three nodes, D = 37, bf16: 1.69 times), and which are bound by latency.
template <class T, int DP>
constexpr bool ds_in_two() { return T::BYTES == 2 && DP == 32; }
constexpr bool delta_settled(int D) { return D <= 32; }  // by the dQ kernel, in 16 bits

// Probabilities are 2^p_bits() times as large in fp16: one key of a hundred thousand has 1e-5, which fp16 holds with 8 bits, and 2^15 p with 11; the
// largest is 2^15.  Sums of them are taken back in fp32.
template <class T>
constexpr int p_bits() { return std::is_same<T, F16>::value ? 15 : 0; }

// Tiles of the other side in LDS: one wave has no others that read while it waits, so it has one, and more workgroups find room beside it (D = 20,
// fp32, 2000 graphs of 1 to 45 nodes, 4 heads, the forward pass: 48 us with two, 38 with one; the readout of 12 graphs of 1 to 19 999 nodes 16 and 17).
template <int NW>
constexpr int tile_buffers() { return NW == 1 ? 1 : 2; }

// Keys in a tile of the kernels whose waves own queries.
template <class T, int NW>
constexpr int key_rows() { return T::BYTES == 4 || NW == 1 ? 32 : 64; }

__device__ __forceinline__ bool in_a_graph(const int *__restrict__ ptr, int graphs, int n, int row)
{
    return row >= clamped(ptr, 0, n) && row < clamped(ptr, graphs, n);
}

// Which K/V head, tile and part a workgroup has: neighbouring tiles of a head, which read the same keys, mostly on one XCD.
struct Place {
    int tile, share, part;
};
__device__ __forceinline__ Place place_of(const AttnArgs &a)
{
    const int b = xcd_chunked_block(blockIdx.x, gridDim.x);
    Place p;
    p.tile = b % a.tiles;
    p.share = b / a.tiles % a.kv_heads;
    p.part = b / a.tiles / a.kv_heads;
    return p;
}

// Whether a matrix' rows are whole pieces at 16-byte alignment, head by head, and those of a tile within 2^32 bytes.
inline bool attn_whole(const void *p, int64_t ld, int D, int dtype)
{
    return aligned16(p) && ld * elem_size(dtype) % 16 == 0 && D * elem_size(dtype) % 16 == 0 &&
           ld * elem_size(dtype) < (1 << 24);
}

// dtype, width and waves of a workgroup to template arguments.
#define FTC_ATTN_WIDTHS(KERNEL, T, NW, WHOLE)                                                                              \
    do {                                                                                                                  \
        if (a.D <= 32) hipLaunchKernelGGL((KERNEL<T, 32, NW, WHOLE>), dim3(grid), dim3((KERNEL##_threads<T, 32, NW>())), 0, s, a); \
        else if (a.D <= 64) hipLaunchKernelGGL((KERNEL<T, 64, NW, WHOLE>), dim3(grid), dim3((KERNEL##_threads<T, 64, NW>())), 0, s, a); \
        else hipLaunchKernelGGL((KERNEL<T, 128, NW, WHOLE>), dim3(grid), dim3((KERNEL##_threads<T, 128, NW>())), 0, s, a);  \
    } while (0)
#define FTC_ATTN_LAUNCH(KERNEL, T)                                                                                        \
    do {                                                                                                                  \
        if (nw == 1 && whole) FTC_ATTN_WIDTHS(KERNEL, T, 1, true);                                                         \
        else if (nw == 1) FTC_ATTN_WIDTHS(KERNEL, T, 1, false);                                                            \
        else if (whole) FTC_ATTN_WIDTHS(KERNEL, T, 4, true);                                                               \
        else FTC_ATTN_WIDTHS(KERNEL, T, 4, false);                                                                         \
    } while (0)
#define FTC_ATTN_TYPES(KERNEL)                                                                                            \
    do {                                                                                                                  \
        if (dtype == FTC_F32) FTC_ATTN_LAUNCH(KERNEL, F32);                                                                \
        else if (dtype == FTC_F16) FTC_ATTN_LAUNCH(KERNEL, F16);                                                           \
        else FTC_ATTN_LAUNCH(KERNEL, BF16);                                                                                \
    } while (0)

// nw: waves of a workgroup that have rows of their own, 1 or 4; grid: a.tiles * a.kv_heads * a.splits workgroups
void launch_attention_forward(const AttnArgs &a, int dtype, int nw, bool whole, unsigned grid, hipStream_t s);
void launch_attention_dq(const AttnArgs &a, int dtype, int nw, bool whole, unsigned grid, hipStream_t s);
void launch_attention_dkv(const AttnArgs &a, int dtype, int nw, bool whole, unsigned grid, hipStream_t s);

}  // namespace ftc
