// The norm over many gradients, norm = |scale| sqrt(sum of all g^2), and their clipping, out = scale min(1, max_norm / norm) g.
//
// A launch has as many gradients as fit its arguments, so there is nothing to copy to the device, and all of them in chunks of up to GRAD_CHUNK numbers
// that its workgroups take in turn.  Squares are added in 64 bits: no gradient that is finite overflows, and a sum over 10^8 numbers is as exact as one over ten.
// Each workgroup leaves one sum; whoever needs the norm adds these up in order, the workgroups that clip for themselves, which saves a launch between.
//
// Bound by memory, which the gradients cross twice: 63 M in fp32, 133 tensors, squares 45 us (254 MB at 5.6 TB/s), clipping 78 (507 MB at 6.5, some of it from cache); small lists by
// two launches, 3 and 4 us.
#include "stream_piece.hpp"

namespace ftc {

constexpr int GRAD_THREADS = 256, GRAD_CHUNK = 8192;  // numbers of a chunk
// Up to FEW_NUMBERS of all gradients in shorter ones, for more workgroups: clipping of 100 000 in 20 tensors 5.9 us in a graph, 8.3 in chunks of GRAD_CHUNK, a million 8.4 and 9.2, level at
// 1.5 million, three 15.7 and 15.1.
constexpr int FEW_CHUNK = 2048, FEW_NUMBERS = 1 << 20;
constexpr int GRAD_GROUPS = 2048;                       // workgroups of a launch at most
// 16 bytes each: neighbouring lanes have neighbouring ones
constexpr int grad_vec(int dtype) { return dtype == FTC_F32 ? 4 : 8; }

// The gradients of a launch: where each begins, how many numbers it has (a row of it) with its type in the two highest bits, and its first chunk.  What is contiguous, almost
// everything, is one row; matrices of rows that are not have launches of their own.
template <int MOST, int NUMBERS = GRAD_CHUNK>
struct GradWhole {
    static constexpr int ENTRIES = MOST, CHUNK = NUMBERS;
    static constexpr bool ONE_ROW = true;
    const void *grad[MOST];
    void *out[MOST];
    uint64_t cols[MOST];
    uint32_t first[MOST];
    __device__ __forceinline__ void place(int, int64_t piece, int vec, int64_t &at, int64_t &to, int64_t &col) const { at = to = col = piece * vec; }
};
template <int MOST>
struct GradRows : GradWhole<MOST> {
    static constexpr bool ONE_ROW = false;
    int64_t ld[MOST], ldo[MOST];
    uint32_t rows[MOST], pieces[MOST];  // pieces of a row
    __device__ __forceinline__ void place(int e, int64_t piece, int vec, int64_t &at, int64_t &to, int64_t &col) const
    {
        const uint32_t row = static_cast<uint32_t>(piece) / pieces[e];
        col = row < rows[e] ? static_cast<int64_t>(static_cast<uint32_t>(piece) % pieces[e]) * vec : INT64_MAX / 2;
        at = row * ld[e] + col;
        to = row * ldo[e] + col;
    }
};
constexpr int GRAD_TYPE_SHIFT = 62;
template <class E>
struct GradArgs {
    E e;
    int entries;
    uint32_t chunks;
    double *sums;  // one a workgroup
};
typedef GradArgs<GradWhole<140>> GradArgsWhole;
typedef GradArgs<GradWhole<140, FEW_CHUNK>> GradArgsSmall;
typedef GradArgs<GradWhole<32, FEW_CHUNK>> GradArgsFew;  // a launch with 4 kB of arguments takes the host 0.4 us more
typedef GradArgs<GradRows<64>> GradArgsRows;
static_assert(sizeof(GradArgsWhole) <= 4000 && sizeof(GradArgsRows) <= 4000, "within the arguments of a launch");

// One row, however it is cut; clip: `out`, too.
bool grad_whole(const ftc_grad &g, bool clip) { return g.rows == 1 || (g.ld == g.cols && (!clip || g.ldo == g.cols)); }

#if defined(__HIPCC__)

// Which gradient a chunk is of, the last one that begins at or before it (uniform): 64 of them are looked at at once.
template <class E>
__device__ __forceinline__ int entry_of(const GradArgs<E> &a, uint32_t c)
{
    int count = 0;
#pragma unroll
    for (int b = 0; b < E::ENTRIES; b += 64) {
        const int i = b + (threadIdx.x & 63);
        count += __popcll(__builtin_amdgcn_ballot_w64(i < a.entries && a.e.first[i] <= c));
    }
    return count - 1;
}
template <class E>
__device__ __forceinline__ int type_of(const GradArgs<E> &a, int e) { return static_cast<int>(a.e.cols[e] >> GRAD_TYPE_SHIFT); }

// This thread's pieces of chunk c, all on their way at once; and where they go.
template <class T, int CHUNK>
struct GradPieces {
    static constexpr int COUNT = CHUNK / (GRAD_THREADS * T::VEC);
    ftc_u32x4 w[COUNT];
    int left[COUNT];
    int64_t to[COUNT];
    template <class E>
    __device__ __forceinline__ void load(const GradArgs<E> &a, int e, uint32_t c)
    {
        const int64_t cols = static_cast<int64_t>(a.e.cols[e] & ((1ull << GRAD_TYPE_SHIFT) - 1)), first = static_cast<int64_t>(c - a.e.first[e]) * (CHUNK / T::VEC) + threadIdx.x;
        if constexpr (E::ONE_ROW) {
            if (static_cast<int64_t>(c - a.e.first[e] + 1) * CHUNK <= cols) {  // uniform: all of the chunk is there
#pragma unroll
                for (int i = 0; i < COUNT; ++i) {
                    to[i] = (first + i * GRAD_THREADS) * T::VEC;
                    left[i] = T::VEC;
                    w[i] = load_piece<T>(a.e.grad[e], to[i], T::VEC);
                }
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            int64_t at, col;
            a.e.place(e, first + i * GRAD_THREADS, T::VEC, at, to[i], col);
            const int64_t rest = cols - col;
            left[i] = static_cast<int>(rest < T::VEC ? (rest > 0 ? rest : 0) : T::VEC);
            w[i] = load_piece<T>(a.e.grad[e], at, left[i]);
        }
    }
    __device__ __forceinline__ void numbers(int i, float (&x)[T::VEC]) const
    {
        RawVec<T, T::VEC> r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r.w[j] = w[i][j];
        unpack<T, T::VEC>(r, x);
    }
};
// f(type) for the one of a number, uniform
template <class F>
__device__ __forceinline__ void by_type(int dtype, const F &f)
{
    if (dtype == FTC_F32) f(F32());
    else if (dtype == FTC_F16) f(F16());
    else f(BF16());
}

// Sum over the workgroup, in each of its threads, in a fixed order.
__device__ __forceinline__ double group_total(double s, double *area)
{
#pragma unroll
    for (int m = 32; m > 0; m /= 2) s += __shfl_xor(s, m, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) area[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0;
#pragma unroll
    for (int w = 0; w < GRAD_THREADS / 64; ++w) s += area[w];
    return s;
}

template <class E>
__global__ __launch_bounds__(GRAD_THREADS) void grad_squares_kernel(GradArgs<E> a)
{
    __shared__ double area[GRAD_THREADS / 64];
    double s = 0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int e = entry_of(a, c);
        by_type(type_of(a, e), [&](auto type) {
            typedef decltype(type) T;
            GradPieces<T, E::CHUNK> p;
            p.load(a, e, c);
#pragma unroll
            for (int i = 0; i < p.COUNT; ++i) {
                float x[T::VEC];
                p.numbers(i, x);
#pragma unroll
                for (int j = 0; j < T::VEC; ++j) s = fma(static_cast<double>(x[j]), static_cast<double>(x[j]), s);
            }
        });
    }
    s = group_total(s, area);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
}

__device__ __forceinline__ double grad_norm_of(const double *sums, int count, double scale, double *area)
{
    double s = 0;
    for (int i = threadIdx.x; i < count; i += GRAD_THREADS) s += sums[i];
    return sqrt(group_total(s, area)) * scale;
}

__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_kernel(const double *sums, int count, double scale, float *norm)
{
    __shared__ double area[GRAD_THREADS / 64];
    const double v = grad_norm_of(sums, count, fabs(scale), area);
    if (threadIdx.x == 0) *norm = static_cast<float>(v);
}

// From the last chunk to the first: what was read last for the norm is in cache still.
template <class E>
__global__ __launch_bounds__(GRAD_THREADS) void grad_clip_kernel(GradArgs<E> a, const double *sums, int count, double scale, double max_norm, float *norm)
{
    __shared__ double area[GRAD_THREADS / 64];
    double factor = 0;
    bool known = false;  // the factor is computed while the first chunk is on its way
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const uint32_t chunk = a.chunks - 1 - c;
        const int e = entry_of(a, chunk);
        const bool in_place = a.e.out[e] == a.e.grad[e];
        if (known && factor == 1 && in_place) continue;
        by_type(type_of(a, e), [&](auto type) {
            typedef decltype(type) T;
            constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
            GradPieces<T, E::CHUNK> p;
            p.load(a, e, chunk);
            if (!known) {
                const double v = grad_norm_of(sums, count, fabs(scale), area);
                if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(v);
                factor = scale;
                if (!(v <= max_norm)) factor *= max_norm / v;  // NaN: NaN, for all to see
                known = true;
                if (factor == 1 && in_place) return;
            }
#pragma unroll
            for (int i = 0; i < p.COUNT; ++i) {
                float x[T::VEC];
                p.numbers(i, x);
#pragma unroll
                for (int j = 0; j < T::VEC; ++j) x[j] = static_cast<float>(x[j] * factor);
                if (p.left[i] == T::VEC) {
                    store_piece_nt<T>(a.e.out[e], p.to[i], x);
                } else {
#pragma unroll
                    for (int j = 0; j < T::VEC - 1; ++j)
                        if (j < p.left[i]) store_elem(a.e.out[e], p.to[i] + j, DT, x[j]);
                }
            }
        });
    }
}

#endif  // __HIPCC__

// ---- launches --------------------------------------------------------------------------------------------------
size_t grad_norm_ws(int count)
{
    // of either kind no launch but the last has fewer gradients than fit, and 64 of one kind, 140 of the other fit
    const int64_t launches = count / 64 + 2;
    return count > 0 ? align_up(static_cast<size_t>(launches) * GRAD_GROUPS * sizeof(double), 256) : 0;
}

// f(arguments, workgroups) for every launch's share of the gradients; sums: for the norm, NULL: to clip.  The workgroups of all launches.
template <class Args, class F>
static int each_launch_of(bool whole, const ftc_grad *grads, int count, double *sums, const F &f)
{
    constexpr int MOST = decltype(Args::e)::ENTRIES, CHUNK = decltype(Args::e)::CHUNK;
    const bool clip = !sums;
    int all = 0;
    for (int i = 0; i < count;) {
        Args a;
        a.entries = 0;
        a.chunks = 0;
        for (; i < count && a.entries < MOST; ++i) {
            const ftc_grad &g = grads[i];
            if (g.rows == 0 || g.cols == 0 || grad_whole(g, clip) != whole) continue;
            const int64_t rows = whole ? 1 : g.rows, cols = whole ? g.rows * g.cols : g.cols, vec = grad_vec(g.dtype), pieces = (cols + vec - 1) / vec, each = CHUNK / vec;
            const int e = a.entries++;
            a.e.grad[e] = g.grad;
            a.e.out[e] = g.out;
            a.e.cols[e] = static_cast<uint64_t>(cols) | static_cast<uint64_t>(g.dtype) << GRAD_TYPE_SHIFT;
            a.e.first[e] = a.chunks;
            if constexpr (std::is_same<Args, GradArgsRows>::value) {
                a.e.ld[e] = g.ld;
                a.e.ldo[e] = g.ldo;
                a.e.rows[e] = static_cast<uint32_t>(rows);
                a.e.pieces[e] = static_cast<uint32_t>(pieces);
            }
            a.chunks += static_cast<uint32_t>((rows * pieces + each - 1) / each);
        }
        if (a.entries == 0) break;
        const int groups = static_cast<int>(a.chunks < GRAD_GROUPS ? a.chunks : GRAD_GROUPS);
        a.sums = sums ? sums + all : nullptr;
        f(a, groups);
        all += groups;
    }
    return all;
}
template <class F>
static int each_launch(const ftc_grad *grads, int count, double *sums, const F &f)
{
    int64_t numbers = 0;
    for (int i = 0; i < count && numbers <= FEW_NUMBERS; ++i) numbers += grads[i].rows * grads[i].cols;
    const int whole = numbers > FEW_NUMBERS ? each_launch_of<GradArgsWhole>(true, grads, count, sums, f)
                      : count > decltype(GradArgsFew::e)::ENTRIES ? each_launch_of<GradArgsSmall>(true, grads, count, sums, f)
                                                                  : each_launch_of<GradArgsFew>(true, grads, count, sums, f);
    return whole + each_launch_of<GradArgsRows>(false, grads, count, sums ? sums + whole : nullptr, f);
}

static int launch_squares(const ftc_grad *grads, int count, void *ws, hipStream_t s)
{
    return each_launch(grads, count, static_cast<double *>(ws), [&](const auto &a, int groups) {
        hipLaunchKernelGGL((grad_squares_kernel<std::remove_const_t<decltype(a.e)>>), dim3(groups), dim3(GRAD_THREADS), 0, s, a);
    });
}

int32_t launch_grad_norm(const ftc_grad *grads, int count, double scale, float *norm, void *ws, hipStream_t s)
{
    const int parts = count > 0 ? launch_squares(grads, count, ws, s) : 0;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(GRAD_THREADS), 0, s, static_cast<const double *>(ws), parts, scale, norm);
    return launch_status("gradient norm");
}

int32_t launch_clip_grad_norm(const ftc_grad *grads, int count, double max_norm, double scale, float *norm, void *ws, hipStream_t s)
{
    const int parts = count > 0 ? launch_squares(grads, count, ws, s) : 0;
    if (parts == 0) {  // nothing to clip: the norm of nothing
        hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(GRAD_THREADS), 0, s, static_cast<const double *>(ws), 0, scale, norm);
        return launch_status("gradient clipping");
    }
    float *to = norm;  // the first launch writes it
    each_launch(grads, count, nullptr, [&](const auto &a, int groups) {
        hipLaunchKernelGGL((grad_clip_kernel<std::remove_const_t<decltype(a.e)>>), dim3(groups), dim3(GRAD_THREADS), 0, s, a, static_cast<const double *>(ws), parts, scale, max_norm, to);
        to = nullptr;
    });
    return launch_status("gradient clipping");
}

}  // namespace ftc
