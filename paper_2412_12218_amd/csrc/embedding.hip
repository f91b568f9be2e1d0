// Rows of a table by id, out_i = scale E[id_i], and the gradient of the table, dE_v = scale sum over {i: id_i = v} of dOut_i.
//
// Both only move rows: bound by memory.  A group of lanes (a power of two, 16 bytes each) has a row, or 64 lanes a part of a long one.
//
// The gradient adds the rows of an id in the order of their positions, whatever the ids: positions sorted by id (a stable radix
// sort, reorder.hip) lie in chunks; a group adds up the runs of equal ids in its chunk in fp32 and writes those that begin and
// end there.  What a run has in other chunks is kept as partial rows, at most two a chunk (the run it begins with and the one it ends with), and a
// second kernel adds them up, the chunks of a run spread over a workgroup and joined in order: an id that every second token has costs no more
// than others.  Rows without an id are zeros.
#include "matrix_frag.hpp"

namespace ftc {

template <class T>
__device__ __forceinline__ void piece_values(const ftc_u32x4 &w, float (&f)[T::VEC])
{
    RawVec<T, T::VEC> r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r.w[j] = w[j];
    unpack<T, T::VEC>(r, f);
}

// NV numbers at element idx in a run-time type, those from `left` on not written.
template <int NV>
__device__ __forceinline__ void store_left(void *base, int64_t idx, int dtype, int left, const float (&f)[NV])
{
    if (left >= NV) {
        store_vec_any<NV>(base, idx, dtype, f);
    } else {
#pragma unroll
        for (int j = 0; j < NV - 1; ++j)
            if (j < left) store_elem(base, idx + j, dtype, f[j]);
    }
}

// Lanes of a row: the power of two that holds its pieces, 64 at most.
static int row_lanes(int D, int vec)
{
    int l = 1;
    while (l < 64 && l * vec < D) l *= 2;
    return l;
}

constexpr int LOOKUP_ROWS = 4;  // rows of a group: loads in flight
template <class T>
__global__ __launch_bounds__(256) void embedding_kernel(int n, const int *__restrict__ ids, int vocab, const void *__restrict__ E, int64_t lde, int D,
                                                        float scale, void *__restrict__ out, int64_t ldo, int odt, int log_lanes)
{
    const int groups = 256 >> log_lanes, group = threadIdx.x >> log_lanes, lane = threadIdx.x & ((1 << log_lanes) - 1);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * groups * LOOKUP_ROWS + group;
    const int col = ((blockIdx.y << log_lanes) + lane) * T::VEC, left = D - col;
    if (left <= 0) return;
    int id[LOOKUP_ROWS];
#pragma unroll
    for (int k = 0; k < LOOKUP_ROWS; ++k) {
        const int64_t i = first + k * groups;
        id[k] = i < n ? ids[i] : -1;
    }
    ftc_u32x4 w[LOOKUP_ROWS];
#pragma unroll
    for (int k = 0; k < LOOKUP_ROWS; ++k) {
        const bool ok = id[k] >= 0 && id[k] < vocab;
        w[k] = load_piece<T>(E, (ok ? id[k] : 0) * lde + col, ok ? left : 0);
    }
#pragma unroll
    for (int k = 0; k < LOOKUP_ROWS; ++k) {
        const int64_t i = first + k * groups;
        if (i >= n) return;
        float f[T::VEC];
        piece_values<T>(w[k], f);
        const bool ok = id[k] >= 0 && id[k] < vocab;
#pragma unroll
        for (int j = 0; j < T::VEC; ++j) f[j] = ok ? f[j] * scale : 0.f;
        store_left<T::VEC>(out, i * ldo + col, odt, left, f);
    }
}

// Sorted positions of a chunk.
static int chunk_tokens(int n) { return n <= (1 << 15) ? 16 : n <= (1 << 17) ? 32 : 64; }

struct GradArgs {
    const uint32_t *keys, *order;
    const void *G;
    float *head, *tail;  // partial rows of the chunks, `pad` numbers apart
    void *dE;
    int64_t ldg, lde;
    int n, vocab, D, pad, chunk, chunks, de_dt;
    float scale;
};

template <class T>
__global__ __launch_bounds__(256) void embedding_runs_kernel(GradArgs a, int log_lanes)
{
    const int groups = 256 >> log_lanes, group = threadIdx.x >> log_lanes, lane = threadIdx.x & ((1 << log_lanes) - 1);
    const int64_t chunk = static_cast<int64_t>(blockIdx.x) * groups + group;
    const int col = ((blockIdx.y << log_lanes) + lane) * T::VEC, left = a.D - col;
    if (chunk >= a.chunks || left <= 0) return;
    const int64_t begin = chunk * a.chunk, end = min(static_cast<int64_t>(a.n), begin + a.chunk);
    const uint32_t none = static_cast<uint32_t>(a.vocab);
    bool from_before = begin > 0 && a.keys[begin - 1] == a.keys[begin];
    float sum[T::VEC];
#pragma unroll
    for (int j = 0; j < T::VEC; ++j) sum[j] = 0.f;
    constexpr int AHEAD = 8;
    for (int64_t i = begin; i < end; i += AHEAD) {
        uint32_t key[AHEAD + 1];
        ftc_u32x4 w[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const bool in = i + k < end;
            key[k] = in ? a.keys[i + k] : none;
            const int64_t row = in ? a.order[i + k] : 0;
            w[k] = load_piece<T>(a.G, row * a.ldg + col, key[k] != none ? left : 0);
        }
        key[AHEAD] = i + AHEAD < end ? a.keys[i + AHEAD] : none;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (key[k] == none) break;  // padded positions are the last ones
            float f[T::VEC];
            piece_values<T>(w[k], f);
#pragma unroll
            for (int j = 0; j < T::VEC; ++j) sum[j] += f[j];
            const bool last = i + k + 1 == end;
            if (!last && key[k + 1] == key[k]) continue;
            const bool goes_on = last && end < a.n && a.keys[end] == key[k];
            if (from_before || goes_on) {
                float *to = (from_before ? a.head : a.tail) + chunk * a.pad + col;
#pragma unroll
                for (int j = 0; j < T::VEC; j += 4) *reinterpret_cast<float4 *>(to + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
            } else {
#pragma unroll
                for (int j = 0; j < T::VEC; ++j) sum[j] *= a.scale;
                store_left<T::VEC>(a.dE, key[k] * a.lde + col, a.de_dt, left, sum);
            }
            from_before = false;
#pragma unroll
            for (int j = 0; j < T::VEC; ++j) sum[j] = 0.f;
        }
    }
}

// First place of the sorted keys that is not below `key`.
__device__ __forceinline__ int lower_place(const uint32_t *__restrict__ keys, int lo, int hi, uint32_t key)
{
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (keys[mid] < key) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// The run that chunk blockIdx.x ends with, where it began there and goes on: its tail and the heads of the chunks after it.
__global__ __launch_bounds__(256) void embedding_join_kernel(GradArgs a, int log_lanes)
{
    __shared__ float4 part[256];
    const int64_t chunk = blockIdx.x, end = (chunk + 1) * a.chunk;
    if (end >= a.n) return;
    const uint32_t key = a.keys[end - 1];
    if (a.keys[end] != key || key == static_cast<uint32_t>(a.vocab)) return;
    const int64_t begin = chunk * a.chunk;
    if (a.keys[begin] == key && begin > 0 && a.keys[begin - 1] == key) return;  // it began before
    const int run_end = lower_place(a.keys, static_cast<int>(end), a.n, key + 1), last = (run_end - 1) / a.chunk;
    const int lanes = 1 << log_lanes, groups = 256 >> log_lanes, group = threadIdx.x >> log_lanes, lane = threadIdx.x & (lanes - 1);
    const int col = ((blockIdx.y << log_lanes) + lane) * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < a.D) {
        const int each = (last - static_cast<int>(chunk) + groups - 1) / groups;
        const int c0 = static_cast<int>(chunk) + 1 + group * each, c1 = min(last + 1, c0 + each);
#pragma unroll 8
        for (int c = c0; c < c1; ++c) {
            const float4 x = *reinterpret_cast<const float4 *>(a.head + static_cast<int64_t>(c) * a.pad + col);
            sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
        }
    }
    part[threadIdx.x] = sum;
    __syncthreads();
    if (group > 0 || col >= a.D) return;
    sum = *reinterpret_cast<const float4 *>(a.tail + chunk * a.pad + col);
    for (int g = 0; g < groups; ++g) {
        const float4 x = part[g * lanes + lane];
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    const float f[4] = {sum.x * a.scale, sum.y * a.scale, sum.z * a.scale, sum.w * a.scale};
    store_left<4>(a.dE, key * a.lde + col, a.de_dt, a.D - col, f);
}

__global__ __launch_bounds__(256) void embedding_absent_kernel(GradArgs a, int log_lanes)
{
    const int groups = 256 >> log_lanes, lanes = 1 << log_lanes, lane = threadIdx.x & (lanes - 1);
    const int64_t v = static_cast<int64_t>(blockIdx.x) * groups + (threadIdx.x >> log_lanes);
    if (v >= a.vocab) return;
    const int at = lower_place(a.keys, 0, a.n, static_cast<uint32_t>(v));
    if (at < a.n && a.keys[at] == static_cast<uint32_t>(v)) return;
    const float zeros[4] = {0.f, 0.f, 0.f, 0.f};
    for (int col = lane * 4; col < a.D; col += lanes * 4) store_left<4>(a.dE, v * a.lde + col, a.de_dt, a.D - col, zeros);
}

static int log_of(int x)
{
    int b = 0;
    while ((1 << b) < x) ++b;
    return b;
}

int32_t launch_embedding(int n, const int *ids, int vocab, const void *E, int lde, int dt, int D, float scale, void *out, int ldo, int odt,
                         hipStream_t s)
{
    const int vec = dt == FTC_F32 ? 4 : 8, lanes = row_lanes(D, vec), groups = 256 / lanes;
    const dim3 grid(ceil_div(n, groups * LOOKUP_ROWS), ceil_div(D, lanes * vec));
#define FTC_LOOKUP(T) hipLaunchKernelGGL(embedding_kernel<T>, grid, dim3(256), 0, s, n, ids, vocab, E, static_cast<int64_t>(lde), D, scale, out, \
                                         static_cast<int64_t>(ldo), odt, log_of(lanes))
    if (dt == FTC_F32) FTC_LOOKUP(F32);
    else if (dt == FTC_F16) FTC_LOOKUP(F16);
    else FTC_LOOKUP(BF16);
#undef FTC_LOOKUP
    return launch_status("embedding");
}

static size_t partial_row_bytes(int n, int D)
{
    return align_up(static_cast<size_t>(ceil_div(n, chunk_tokens(n))) * align_up(D, 8) * sizeof(float), 256);
}

size_t embedding_backward_ws(int n, int vocab, int D)
{
    (void)vocab;
    return id_sort_ws(n) + 2 * partial_row_bytes(n, D);
}

int32_t launch_embedding_backward(int n, const int *ids, int vocab, const void *G, int ldg, int dt, int D, float scale, void *dE, int lde,
                                  int de_dt, void *ws, hipStream_t s)
{
    GradArgs a = {};
    const int32_t st = launch_sort_ids(n, ids, vocab, &a.keys, &a.order, ws, s);
    if (st != FTC_OK) return st;
    char *p = static_cast<char *>(ws) + id_sort_ws(n);
    a.head = reinterpret_cast<float *>(p);
    a.tail = reinterpret_cast<float *>(p + partial_row_bytes(n, D));
    a.G = G; a.ldg = ldg; a.dE = dE; a.lde = lde;
    a.n = n; a.vocab = vocab; a.D = D; a.pad = static_cast<int>(align_up(D, 8)); a.de_dt = de_dt; a.scale = scale;
    a.chunk = chunk_tokens(n);
    a.chunks = ceil_div(n, a.chunk);
    const int vec = dt == FTC_F32 ? 4 : 8, lanes = row_lanes(D, vec), lanes4 = row_lanes(D, 4);
    if (n > 0) {
        const dim3 grid(ceil_div(a.chunks, 256 / lanes), ceil_div(D, lanes * vec));
        if (dt == FTC_F32) hipLaunchKernelGGL(embedding_runs_kernel<F32>, grid, dim3(256), 0, s, a, log_of(lanes));
        else if (dt == FTC_F16) hipLaunchKernelGGL(embedding_runs_kernel<F16>, grid, dim3(256), 0, s, a, log_of(lanes));
        else hipLaunchKernelGGL(embedding_runs_kernel<BF16>, grid, dim3(256), 0, s, a, log_of(lanes));
        if (a.chunks > 1)
            hipLaunchKernelGGL(embedding_join_kernel, dim3(a.chunks - 1, ceil_div(D, lanes4 * 4)), dim3(256), 0, s, a, log_of(lanes4));
    }
    hipLaunchKernelGGL(embedding_absent_kernel, dim3(ceil_div(vocab, 256 / lanes4)), dim3(256), 0, s, a, log_of(lanes4));
    return launch_status("embedding backward");
}

}  // namespace ftc
