// Rows of a table by id, out_i = scale E[id_i], and the gradient of the table, dE_v = scale sum over {i: id_i = v} of dOut_i.
//
// Both only move rows: bound by memory.  A group of lanes (a power of two, 16 bytes each) has a row, or 64 lanes a part of a long one.
//
// The gradient adds the rows of an id in the order of their positions, whatever the ids: positions sorted by id (a stable radix
// sort, reorder.hip) lie in chunks, one for each group of a workgroup; a group adds up the runs of equal ids in its chunk in fp32 and writes
// those that begin and end there.  What a run has in other chunks is kept as partial rows, at most two a chunk (the run it begins with and
// the one it ends with): the workgroup adds up those of its chunks, in order, and leaves two at most of its own, which a second kernel
// adds up, those of a long run spread over a workgroup and joined in order: an id that every second position has costs no more than others.
// Rows without an id are zeros.
//
// Measured: 300 000 look-ups in 200 000 x 128, fp16, 29.4 us, 154 MB with the rows that several ids share at 5.2 TB/s (a large copy: 5.1).  Gradient of 131 072
// x 512 into 50 000 rows, bf16, 86 us: sort 26 (launches of 3 to 6 us, two digits), runs 37 (the rows of dOut from memory in the ids' order, 3.6 TB/s), finish 15
// (25 000 joins and zeros); of 46 000 x 200 into 118 rows, fp32, 31 us: sort 12, runs and finish 11 each.
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

struct GradArgs {
    const uint32_t *keys, *order;
    const void *G;
    float *head, *tail;  // partial rows of the workgroups of embedding_runs_kernel, `pad` numbers apart
    void *dE;
    int64_t ldg, lde;
    int n, vocab, D, pad, chunk, span, spans, de_dt;  // positions of a group, of a workgroup; workgroups
    float scale;
};

__device__ __forceinline__ void add4(float4 &a, const float4 &b)
{
    a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
}
__device__ __forceinline__ void store_joined(const GradArgs &a, uint32_t key, int col, const float4 &sum)
{
    const float f[4] = {sum.x * a.scale, sum.y * a.scale, sum.z * a.scale, sum.w * a.scale};
    store_left<4>(a.dE, key * a.lde + col, a.de_dt, a.D - col, f);
}
// Sorted positions of a workgroup, kept in LDS: a chunk for each of its groups.
constexpr int RUN_TOKENS = 2048;

template <class T>
__global__ __launch_bounds__(256) void embedding_runs_kernel(GradArgs a, int log_lanes)
{
    __shared__ uint32_t keys[RUN_TOKENS + 2], order[RUN_TOKENS];  // keys: from the one before on
    __shared__ float4 part[2 * 256 * T::VEC / 4];                 // partial rows of the groups: the first run's, the last one's
    __shared__ int state[256];
    const int group = threadIdx.x >> log_lanes, lane = threadIdx.x & ((1 << log_lanes) - 1);
    const uint32_t none = static_cast<uint32_t>(a.vocab), outside = 0xffffffffu;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.span;
    const int count = static_cast<int>(min(static_cast<int64_t>(a.span), a.n - first));
    for (int i = threadIdx.x; i < count + 2; i += 256) {
        const int64_t at = first + i - 1;
        keys[i] = at >= 0 && at < a.n ? a.keys[at] : outside;
        if (i < count) order[i] = a.order[first + i];
    }
    __syncthreads();
    const int lane_col = lane * T::VEC, col = (blockIdx.y << log_lanes) * T::VEC + lane_col, left = a.D - col;
    const int begin = group * a.chunk, end = min(count, begin + a.chunk);
    const bool has = begin < end;
    bool from_before = has && keys[begin] == keys[begin + 1];
    const bool goes_on = has && keys[end + 1] == keys[end];
    if (lane == 0) {
        // 1: the chunk begins inside a run, 2: it ends inside one, 4: that is one and the same
        int all = 0;
        if (has) {
            const uint32_t k0 = keys[begin + 1], k1 = keys[end];
            all = k0 == none && k1 == none ? 0 : (from_before && k0 != none ? 1 : 0) | (goes_on && k1 != none ? 2 : 0) | (k0 == k1 ? 4 : 0);
        }
        state[group] = all;
    }
    float sum[T::VEC];
#pragma unroll
    for (int j = 0; j < T::VEC; ++j) sum[j] = 0.f;
    constexpr int AHEAD = 8;
    ftc_u32x4 w[AHEAD], next[AHEAD];
    auto fetch = [&](int i, ftc_u32x4(&to)[AHEAD]) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const bool in = i + k < end && keys[i + k + 1] != none;
            to[k] = load_piece<T>(a.G, (in ? static_cast<int64_t>(order[i + k]) : 0) * a.ldg + col, in ? left : 0);
        }
    };
    if (has && left > 0) fetch(begin, w);
    for (int i = begin; i < end && left > 0; i += AHEAD) {
        if (i + AHEAD < end) fetch(i + AHEAD, next);
        uint32_t key[AHEAD + 1];
#pragma unroll
        for (int k = 0; k <= AHEAD; ++k) key[k] = i + k < end ? keys[i + k + 1] : outside;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i + k >= end || key[k] == none) break;  // padded positions are the last ones
            float f[T::VEC];
            piece_values<T>(w[k], f);
#pragma unroll
            for (int j = 0; j < T::VEC; ++j) sum[j] += f[j];
            if (key[k + 1] == key[k]) continue;
            if (from_before || (i + k + 1 == end && goes_on)) {
                float4 *to = &part[(group * 2 + (from_before ? 0 : 1)) * (T::VEC / 4 << log_lanes) + lane_col / 4];
#pragma unroll
                for (int j = 0; j < T::VEC; j += 4) to[j / 4] = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
            } else {
#pragma unroll
                for (int j = 0; j < T::VEC; ++j) sum[j] *= a.scale;
                store_left<T::VEC>(a.dE, key[k] * a.lde + col, a.de_dt, left, sum);
            }
            from_before = false;
#pragma unroll
            for (int j = 0; j < T::VEC; ++j) sum[j] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) w[k] = next[k];
    }
    __syncthreads();
    // a group adds up the run that begins in its chunk and goes on; the first also the one that comes from before the workgroup
    if (!has || left <= 0) return;
    const int chunks = (count + a.chunk - 1) / a.chunk;
    constexpr int QUADS = T::VEC / 4;
    const int quads = QUADS << log_lanes;
    const auto through = [&](int g) { return state[g] == 7; };  // in at one end and out at the other
    for (int lead = group == 0 && (state[0] & 1) ? 1 : 0; lead >= 0; --lead) {
        if (!lead && !((state[group] & 2) && !through(group))) continue;
        float4 run[QUADS];
        bool open = true;
        int g = group;
#pragma unroll
        for (int q = 0; q < QUADS; ++q) run[q] = part[(g * 2 + (lead ? 0 : 1)) * quads + lane * QUADS + q];
        if (lead) open = through(0);
        while (open && g + 1 < chunks) {
            ++g;
#pragma unroll
            for (int q = 0; q < QUADS; ++q) add4(run[q], part[g * 2 * quads + lane * QUADS + q]);
            open = through(g);
        }
#pragma unroll
        for (int q = 0; q < QUADS; ++q) {
            const int c4 = col + 4 * q;
            if (c4 >= a.D) break;
            if (lead || open) *reinterpret_cast<float4 *>((lead ? a.head : a.tail) + static_cast<int64_t>(blockIdx.x) * a.pad + c4) = run[q];
            else store_joined(a, keys[end], c4, run[q]);
        }
    }
}

// The first join_groups workgroups: runs that a span of positions (those of a workgroup of the kernel above) ends with, where they began there and go on: its tail and the heads of the
// spans after it.  A group has a span, and adds up what goes on for less than JOIN_FEW spans itself, eight at a time; longer runs the
// workgroup takes one by one, its groups a part of the heads each.  The other workgroups: zeros for the ids that no position has, ABSENT rows each.
constexpr int FINISH = 512, JOIN_FEW = 16, ABSENT = 128;
__global__ __launch_bounds__(FINISH) void embedding_finish_kernel(GradArgs a, int log_lanes, int join_groups)
{
    __shared__ float4 part[FINISH];
    __shared__ int others, list[FINISH];
    const int lanes = 1 << log_lanes, groups = FINISH >> log_lanes, group = threadIdx.x >> log_lanes, lane = threadIdx.x & (lanes - 1);
    if (threadIdx.x == 0) others = 0;
    __syncthreads();
    if (static_cast<int>(blockIdx.x) >= join_groups) {
        const int64_t v0 = (static_cast<int64_t>(blockIdx.x) - join_groups) * ABSENT, v = v0 + threadIdx.x;
        const bool looks = threadIdx.x < ABSENT && v < a.vocab;
        int lo = 0, hi = looks ? a.n : 0;
        while (lo < hi) {  // first place of the sorted keys that is not below v
            const int mid = lo + (hi - lo) / 2;
            if (a.keys[mid] < static_cast<uint32_t>(v)) lo = mid + 1; else hi = mid;
        }
        const bool absent = looks && (lo == a.n || a.keys[lo] != static_cast<uint32_t>(v));
        if (absent) list[atomicAdd(&others, 1)] = threadIdx.x;  // in any order
        __syncthreads();
        const int count = others, pieces = (a.D + 7) / 8;
        const float zeros[8] = {};
        for (int i = threadIdx.x; i < count * pieces; i += FINISH) {
            const int64_t row = v0 + list[i / pieces];
            const int col = i % pieces * 8;
            store_left<8>(a.dE, row * a.lde + col, a.de_dt, a.D - col, zeros);
        }
        return;
    }
    const int64_t span = static_cast<int64_t>(blockIdx.x) * groups + group, end = (span + 1) * a.span;
    uint32_t key = static_cast<uint32_t>(a.vocab);
    bool begins = false;
    if (end < a.n) {
        key = a.keys[end - 1];
        const int64_t begin = end - a.span;
        begins = key != static_cast<uint32_t>(a.vocab) && a.keys[end] == key && !(begin > 0 && a.keys[begin - 1] == key);
    }
    if (begins) {
        int reach = 0;  // spans after this one whose first position is the run's
        for (int more = 8; more == 8 && reach < JOIN_FEW; reach += more) {
            more = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t at = end + (reach + k) * a.span;
                more += at < a.n && a.keys[at] == key ? 1 : 0;
            }
        }
        if (reach < JOIN_FEW) {
            for (int col = lane * 4; col < a.D; col += lanes * 4) {
                float4 sum = *reinterpret_cast<const float4 *>(a.tail + span * a.pad + col);
#pragma unroll 8
                for (int k = 1; k <= reach; ++k) add4(sum, *reinterpret_cast<const float4 *>(a.head + (span + k) * a.pad + col));
                store_joined(a, key, col, sum);
            }
        } else if (lane == 0) {
            list[atomicAdd(&others, 1)] = group;
        }
    }
    __syncthreads();
    const int count = others;
    for (int i = 0; i < count; ++i) {  // in any order: every run is a sum of its own
        const int64_t c = static_cast<int64_t>(blockIdx.x) * groups + list[i];
        const uint32_t run = a.keys[(c + 1) * a.span - 1];
        int reach = JOIN_FEW;  // at least; the spans whose first position is the run's come first
        for (int step = (a.spans - static_cast<int>(c) + FINISH - 1) / FINISH; step > 0; step = step > 1 ? (step + FINISH - 1) / FINISH : 0) {
            const int64_t at = (c + reach + static_cast<int64_t>(threadIdx.x + 1) * step) * a.span;
            reach += step * __syncthreads_count(at < a.n && a.keys[at] == run);
        }
        const int each = (reach + groups - 1) / groups;
        const int64_t c0 = c + 1 + group * each, c1 = min(c + 1 + reach, c0 + each);
        for (int base = 0; base < a.D; base += lanes * 4) {
            const int col = base + lane * 4;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            if (col < a.D) {
#pragma unroll 8
                for (int64_t k = c0; k < c1; ++k) add4(sum, *reinterpret_cast<const float4 *>(a.head + k * a.pad + col));
            }
            part[threadIdx.x] = sum;
            __syncthreads();
            if (group == 0 && col < a.D) {
                sum = *reinterpret_cast<const float4 *>(a.tail + c * a.pad + col);
                for (int g = 0; g < min(groups, reach); ++g) add4(sum, part[g * lanes + lane]);
                store_joined(a, run, col, sum);
            }
            __syncthreads();
        }
    }
}

static int log_of(int x)
{
    int b = 0;
    while ((1 << b) < x) ++b;
    return b;
}

// Threads of the largest launch, along x, and workgroups along y; of the lookup, and of the gradient.
LaunchSize embedding_size(int n, int D)
{
    LaunchSize z;
    for (int vec = 4; vec <= 8; vec *= 2) {
        const int lanes = row_lanes(D, vec);
        z.add(256ll * ceil_div(n, 256 / lanes * LOOKUP_ROWS), ceil_div(D, lanes * vec));
    }
    return z;
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

// Sorted positions of a chunk: such that there are some 4096 waves, 8 to 64, and what a workgroup's groups have room for.
static int chunk_tokens(int n, int D, int vec)
{
    const int lanes = row_lanes(D, vec), room = RUN_TOKENS * lanes / 256;
    int c = 8;
    while (c < 64 && static_cast<int64_t>(n) * lanes > 64ll * 4096 * c) c *= 2;
    return c < room ? c : room;
}

static size_t partial_row_bytes(int n, int D, int vec)
{
    return align_up(static_cast<size_t>(ceil_div(n, chunk_tokens(n, D, vec) * (256 / row_lanes(D, vec)))) * align_up(D, 8) * sizeof(float), 256);
}

LaunchSize embedding_backward_size(int n, int vocab, int D)
{
    LaunchSize z;
    for (int vec = 4; vec <= 8; vec *= 2) {
        const int lanes = row_lanes(D, vec);
        const int64_t spans = ceil_div(n, chunk_tokens(n, D, vec) * (256 / lanes));
        z.add(256 * spans, ceil_div(D, lanes * vec));
        z.add(FINISH * (spans / (FINISH / row_lanes(D, 4)) + 1 + ceil_div(vocab, ABSENT)), 1);
    }
    return z;
}

size_t embedding_backward_ws(int n, int vocab, int D)
{
    (void)vocab;
    const size_t a = partial_row_bytes(n, D, 4), b = partial_row_bytes(n, D, 8);
    return id_sort_ws(n) + 2 * (a > b ? a : b);
}

int32_t launch_embedding_backward(int n, const int *ids, int vocab, const void *G, int ldg, int dt, int D, float scale, void *dE, int lde,
                                  int de_dt, void *ws, hipStream_t s)
{
    GradArgs a = {};
    const int32_t st = launch_sort_ids(n, ids, vocab, &a.keys, &a.order, ws, s);
    if (st != FTC_OK) return st;
    const int vec = dt == FTC_F32 ? 4 : 8, lanes = row_lanes(D, vec), lanes4 = row_lanes(D, 4);
    char *p = static_cast<char *>(ws) + id_sort_ws(n);
    a.head = reinterpret_cast<float *>(p);
    a.tail = reinterpret_cast<float *>(p + partial_row_bytes(n, D, vec));
    a.G = G; a.ldg = ldg; a.dE = dE; a.lde = lde;
    a.n = n; a.vocab = vocab; a.D = D; a.pad = static_cast<int>(align_up(D, 8)); a.de_dt = de_dt; a.scale = scale;
    a.chunk = chunk_tokens(n, D, vec);
    a.span = a.chunk * (256 / lanes);
    a.spans = ceil_div(n, a.span);
    if (n > 0) {
        const dim3 grid(a.spans, ceil_div(D, lanes * vec));
        if (dt == FTC_F32) hipLaunchKernelGGL(embedding_runs_kernel<F32>, grid, dim3(256), 0, s, a, log_of(lanes));
        else if (dt == FTC_F16) hipLaunchKernelGGL(embedding_runs_kernel<F16>, grid, dim3(256), 0, s, a, log_of(lanes));
        else hipLaunchKernelGGL(embedding_runs_kernel<BF16>, grid, dim3(256), 0, s, a, log_of(lanes));
    }
    const int joins = ceil_div(a.spans > 1 ? a.spans - 1 : 0, FINISH / lanes4);
    hipLaunchKernelGGL(embedding_finish_kernel, dim3(joins + ceil_div(vocab, ABSENT)), dim3(FINISH), 0, s, a, log_of(lanes4), joins);
    return launch_status("embedding backward");
}

}  // namespace ftc
