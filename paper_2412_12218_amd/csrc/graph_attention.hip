// Attention between all nodes of a graph, over a batch of graphs packed one behind the other, and its gradients: the launches, and the
// kernels that are bound by memory.  The formulas and how the products are laid out: attention_common.hpp.
#include "attention_common.hpp"

namespace ftc {

// Adds up the parts of the forward pass, WAVES waves a query and head, which take the parts in turn, at most JOIN_EACH each: all of them on their way before
// anything is known about them (7.2 us for 96 rows of 39 parts, 3.9 so).  Lane z has the maximum and the sum of part z.  Rows that belong to no graph stay as they are.
constexpr int JOIN_EACH = 16;
template <class T, int WAVES>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, mine = __builtin_amdgcn_readfirstlane(wave % WAVES);
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (4 / WAVES) + wave / WAVES, all = static_cast<int64_t>(a.n_q) * a.heads;
    if (row >= all) return;
    float v[2][JOIN_EACH];  // columns lane and lane + 64
#pragma unroll
    for (int i = 0; i < JOIN_EACH; ++i) {
        const int z = mine + i * WAVES;
        const float *part = a.part + (z * all + row) * a.D;
        v[0][i] = z < a.splits ? part[lane < a.D ? lane : 0] : 0.f;
        v[1][i] = z < a.splits && a.D > 64 ? part[lane + 64 < a.D ? lane + 64 : 0] : 0.f;
    }
    float2 ml = {-INFINITY, 0.f};
    if (lane < a.splits) ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (lane * all + row));
    const int query = static_cast<int>(row / a.heads), head = static_cast<int>(row % a.heads);
    if (!in_a_graph(a.q_ptr, a.graphs, a.n_q, query)) return;  // of WAVES = 4 the whole workgroup
    float m = ml.x;
#pragma unroll
    for (int b = 1; b < 64; b *= 2) m = fmaxf(m, __shfl_xor(m, b, 64));
    const float shift = m == -INFINITY ? 0.f : m, weight = __builtin_amdgcn_exp2f(ml.x - shift);
    float l = ml.y * weight;
#pragma unroll
    for (int b = 1; b < 64; b *= 2) l += __shfl_xor(l, b, 64);
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    __shared__ float sums[WAVES][128];
    float x[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < JOIN_EACH; ++i) {
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), mine + i * WAVES));  // 0 behind the last part
        x[0] = fmaf(v[0][i], w, x[0]);
        x[1] = fmaf(v[1][i], w, x[1]);
    }
    if constexpr (WAVES > 1) {
        sums[mine][lane] = x[0];
        sums[mine][lane + 64] = x[1];
        __syncthreads();
        if (mine > 0) return;
#pragma unroll
        for (int k = 1; k < WAVES; ++k) {
            x[0] += sums[k][lane];
            x[1] += sums[k][lane + 64];
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = lane + 64 * k;
        if (c < a.D) store_elem(a.out, query * a.ldo + head * a.D + c, DT, x[k] * inv);
    }
    if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l) - p_bits<T>()) * LN2;
}

// ---- backward: delta -----------------------------------------------------------------------------------------
// 16 lanes a query and head; DELTA_GROUPS workgroups at most, which go on with the next rows.
constexpr int DELTA_GROUPS = 1 << 20;
template <class T>
__global__ __launch_bounds__(256) void attention_delta_kernel(AttnArgs a)
{
    const int64_t all = static_cast<int64_t>(a.n_q) * a.heads;
    const int lane = threadIdx.x & 15;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * 16; first < all; first += static_cast<int64_t>(gridDim.x) * 16) {
        const int64_t row = first + (threadIdx.x >> 4);
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
#pragma unroll 8
    for (int z = 0; z < splits; ++z) x += part[z * stride + id];
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    store_elem(out, row * ld + c, DT, x);
}

// dQ of parts with their sums of ds, and delta with them (attention_dq.hip).
template <class T>
__global__ __launch_bounds__(256) void attention_settle_kernel(AttnArgs a)
{
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, rows = static_cast<int64_t>(a.n_q) * a.heads;
    const int64_t row = id / a.D;
    const int c = static_cast<int>(id % a.D), query = static_cast<int>(row / a.heads), head = static_cast<int>(row % a.heads);
    if (row >= rows || !in_a_graph(a.q_ptr, a.graphs, a.n_q, query)) return;
    float x = 0.f, mean = 0.f, rest = 0.f;
#pragma unroll 8
    for (int z = 0; z < a.splits; ++z) {
        x += a.part[z * rows * a.D + id];
        mean += a.part_mean[z * rows * a.D + id];
        rest += a.part_rest[z * rows + row];
    }
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    store_elem(a.dQ, query * a.lddq + head * a.D + c, DT, fmaf(-rest, mean, x));
    if (c == 0) a.delta[row] += rest;
}

// ---- launches ----------------------------------------------------------------------------------------------------
// Waves of a workgroup: one for short graphs, whose rows would not fill four, else four, which share the other side's tiles.  us of the forward and
// backward passes with one and four, 50 000 nodes, 8 heads: bf16, D = 64, graphs of 80 nodes 49 / 59 and 197 / 220, of 100 57 / 52 and 223 / 198,
// of 160 60 / 66 and 232 / 237, of 300 97 / 80 and 309 / 267; fp32, D = 16, of 160 100 / 124 and 339 / 429.  With D = 128, where K, V and
// their gradients leave a SIMD one wave, of 160 135 / 135 and 710 / 579.
static int attn_waves(int64_t rows, int64_t other, int graphs, int D)
{
    const int64_t most = (D <= 64 ? 160ll : 64ll) * graphs;
    return rows <= 64ll * graphs || (rows <= most && other <= most) ? 1 : 4;
}
static int attn_tiles(int64_t rows, int graphs, int waves) { return static_cast<int>(rows / (32 * waves)) + graphs; }
// Parts of the other axis where there are at most four waves for each compute unit, up to eight (parts and their join cost a pass over fp32 results: 8
// graphs of 799 nodes, 8 heads, D = 64, bf16, in two parts 47 us, whole 27).  A part of a graph of the mean size has at least two tiles of one
// wave's workgroups (parts of 64 / 128 / 256: 121 graphs of 557 nodes, one query, D = 37, bf16 18 / 26 / 54 us, 19 of 350, D = 96, fp32 47 / 87 / 157),
// four of four waves'.
static int attn_splits(int64_t rows, int64_t other, int graphs, int kv_heads, int D)
{
    const int nw = attn_waves(rows, other, graphs, D);
    const int64_t groups = static_cast<int64_t>(attn_tiles(rows, graphs, nw)) * kv_heads;
    if (groups < 1 || graphs < 1) return 1;
    const int64_t want = 2048 / nw / groups, most = other / graphs / (nw == 1 ? 64 : 256);
    const int64_t s = want < most ? want : most;
    return static_cast<int>(s < 1 ? 1 : s > 64 ? 64 : s);
}

LaunchSize attention_size(int n_q, int n_kv, int graphs, int heads, int kv_heads, int D)
{
    const int64_t virt = static_cast<int64_t>(n_q) * (heads / kv_heads);
    LaunchSize z;
    for (int side = 0; side < 2; ++side) {
        const int64_t rows = side ? n_kv : virt, other = side ? virt : n_kv;
        const int nw = attn_waves(rows, other, graphs, D), splits = attn_splits(rows, other, graphs, kv_heads, D);
        z.add(static_cast<int64_t>(attn_tiles(rows, graphs, nw)) * kv_heads * splits * (nw == 1 ? 64 : 512), 1);
        if (splits > 1) z.add((side ? static_cast<int64_t>(n_kv) * kv_heads : static_cast<int64_t>(n_q) * heads) * (D > 64 ? D : 64), 1);
    }
    return z;
}

size_t attention_ws(int n_q, int n_kv, int graphs, int heads, int kv_heads, int D)
{
    const int64_t rows = static_cast<int64_t>(n_q) * heads;
    const int s = attn_splits(static_cast<int64_t>(n_q) * (heads / kv_heads), n_kv, graphs, kv_heads, D);
    if (s == 1) return 0;
    return align_up(static_cast<size_t>(s) * rows * D * sizeof(float), 256) + align_up(static_cast<size_t>(s) * rows * 2 * sizeof(float), 256);
}

size_t attention_backward_ws(int n_q, int n_kv, int graphs, int heads, int kv_heads, int D)
{
    const int64_t rows = static_cast<int64_t>(n_q) * heads, group = heads / kv_heads;
    const int sq = attn_splits(n_q * group, n_kv, graphs, kv_heads, D), sk = attn_splits(n_kv, n_q * group, graphs, kv_heads, D);
    const size_t parts_q = sq > 1 ? static_cast<size_t>(sq) * rows * (delta_settled(D) ? 2 * D + 1 : D) * sizeof(float) : 0;
    const size_t parts_k = sk > 1 ? static_cast<size_t>(sk) * 2 * n_kv * kv_heads * D * sizeof(float) : 0;
    return align_up(static_cast<size_t>(rows) * sizeof(float), 256) + align_up(parts_q > parts_k ? parts_q : parts_k, 256);
}

// a.splits is set; rows: those that waves have 32 of each
static unsigned attn_grid(AttnArgs &a, int64_t rows, int nw)
{
    a.tiles = attn_tiles(rows, a.graphs, nw);
    return static_cast<unsigned>(a.tiles) * a.kv_heads * a.splits;  // attention_size()
}

#define FTC_ATTN_TYPED_N(KERNEL, N, GRID, ...)                                                                         \
    do {                                                                                                               \
        const dim3 grid__(static_cast<unsigned>(GRID));                                                                \
        if (dtype == FTC_F32) hipLaunchKernelGGL((KERNEL<F32, N>), grid__, dim3(256), 0, s, __VA_ARGS__);               \
        else if (dtype == FTC_F16) hipLaunchKernelGGL((KERNEL<F16, N>), grid__, dim3(256), 0, s, __VA_ARGS__);          \
        else hipLaunchKernelGGL((KERNEL<BF16, N>), grid__, dim3(256), 0, s, __VA_ARGS__);                               \
    } while (0)
#define FTC_ATTN_TYPED(KERNEL, GRID, ...)                                                                              \
    do {                                                                                                               \
        const dim3 grid__(static_cast<unsigned>(GRID));                                                                \
        if (dtype == FTC_F32) hipLaunchKernelGGL(KERNEL<F32>, grid__, dim3(256), 0, s, __VA_ARGS__);                    \
        else if (dtype == FTC_F16) hipLaunchKernelGGL(KERNEL<F16>, grid__, dim3(256), 0, s, __VA_ARGS__);               \
        else hipLaunchKernelGGL(KERNEL<BF16>, grid__, dim3(256), 0, s, __VA_ARGS__);                                    \
    } while (0)

static void forward(AttnArgs a, int dtype, void *ws, hipStream_t s)
{
    const int64_t rows = static_cast<int64_t>(a.n_q) * a.heads, virt = static_cast<int64_t>(a.n_q) * a.group;
    const bool whole = attn_whole(a.Q, a.ldq, a.D, dtype) && attn_whole(a.K, a.ldk, a.D, dtype) && attn_whole(a.V, a.ldv, a.D, dtype);
    const int nw = attn_waves(virt, a.n_kv, a.graphs, a.D);
    a.splits = attn_splits(virt, a.n_kv, a.graphs, a.kv_heads, a.D);
    a.part = static_cast<float *>(ws);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(ws) + align_up(static_cast<size_t>(a.splits) * rows * a.D * sizeof(float), 256));
    const unsigned grid = attn_grid(a, virt, nw);
    launch_attention_forward(a, dtype, nw, whole, grid, s);
    if (a.splits > JOIN_EACH) FTC_ATTN_TYPED_N(attention_join_kernel, 4, rows, a);
    else if (a.splits > 1) FTC_ATTN_TYPED_N(attention_join_kernel, 1, (rows + 3) / 4, a);
}

static void backward(AttnArgs a, int dtype, void *ws, hipStream_t s)
{
    const int64_t rows = static_cast<int64_t>(a.n_q) * a.heads, virt = static_cast<int64_t>(a.n_q) * a.group;
    const bool whole = attn_whole(a.Q, a.ldq, a.D, dtype) && attn_whole(a.K, a.ldk, a.D, dtype) && attn_whole(a.V, a.ldv, a.D, dtype) &&
                       attn_whole(a.dO, a.lddo, a.D, dtype);
    a.delta = static_cast<float *>(ws);
    a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + align_up(static_cast<size_t>(rows) * sizeof(float), 256));
    if (rows > 0) {
        FTC_ATTN_TYPED(attention_delta_kernel, (rows + 15) / 16 < DELTA_GROUPS ? (rows + 15) / 16 : DELTA_GROUPS, a);
        const int nw = attn_waves(virt, a.n_kv, a.graphs, a.D);
        a.splits = attn_splits(virt, a.n_kv, a.graphs, a.kv_heads, a.D);
        a.part_mean = a.part + a.splits * rows * a.D;
        a.part_rest = a.part_mean + a.splits * rows * a.D;
        const unsigned grid = attn_grid(a, virt, nw);
        launch_attention_dq(a, dtype, nw, whole, grid, s);
        const int width = a.heads * a.D;
        const int64_t count = static_cast<int64_t>(a.n_q) * width;
        const dim3 elements(static_cast<unsigned>((count + 255) / 256));
        if (a.splits > 1 && dtype != FTC_F32 && delta_settled(a.D)) {
            if (dtype == FTC_F16) hipLaunchKernelGGL(attention_settle_kernel<F16>, elements, dim3(256), 0, s, a);
            else hipLaunchKernelGGL(attention_settle_kernel<BF16>, elements, dim3(256), 0, s, a);
        } else if (a.splits > 1) {
            FTC_ATTN_TYPED(attention_sum_kernel, elements.x, a.part, count, a.splits, a.q_ptr, a.graphs, a.n_q, width, a.dQ, a.lddq);
        }
    }
    if (a.n_kv > 0) {
        const int nw = attn_waves(a.n_kv, virt, a.graphs, a.D);
        a.splits = attn_splits(a.n_kv, virt, a.graphs, a.kv_heads, a.D);
        const unsigned grid = attn_grid(a, a.n_kv, nw);
        launch_attention_dkv(a, dtype, nw, whole, grid, s);
        const int width = a.kv_heads * a.D;
        const int64_t count = static_cast<int64_t>(a.n_kv) * width;
        if (a.splits > 1) {
            FTC_ATTN_TYPED(attention_sum_kernel, (count + 255) / 256, a.part, 2 * count, a.splits, a.kv_ptr, a.graphs, a.n_kv, width, a.dK, a.lddk);
            FTC_ATTN_TYPED(attention_sum_kernel, (count + 255) / 256, a.part + count, 2 * count, a.splits, a.kv_ptr, a.graphs, a.n_kv, width, a.dV, a.lddv);
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
    a.group_magic = static_cast<uint32_t>(((1ull << 32) + a.group - 1) / a.group);
    return a;
}

int32_t launch_attention(const AttnShape &p, void *out, int ldo, float *lse, void *ws, hipStream_t s)
{
    AttnArgs a = attn_args(p);
    a.out = out; a.ldo = ldo; a.lse = lse;
    forward(a, p.dtype, ws, s);
    return launch_status("graph attention");
}

int32_t launch_attention_backward(const AttnShape &p, const void *out, int ldo, const float *lse, const void *dO, int lddo, void *dQ, int lddq,
                                  void *dK, int lddk, void *dV, int lddv, void *ws, hipStream_t s)
{
    AttnArgs a = attn_args(p);
    a.O = out; a.ldo = ldo; a.lse = const_cast<float *>(lse); a.dO = dO; a.lddo = lddo;
    a.dQ = dQ; a.lddq = lddq; a.dK = dK; a.lddk = lddk; a.dV = dV; a.lddv = lddv;
    backward(a, p.dtype, ws, s);
    return launch_status("graph attention backward");
}

}  // namespace ftc
