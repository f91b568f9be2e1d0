// The norm over many gradients, norm = |scale| sqrt(sum of all g^2), and their clipping, out = scale min(1, max_norm / norm) g.
//
// A launch has up to GRAD_ENTRIES gradients in its arguments, so there is nothing to copy to the device, and all of them in chunks of GRAD_CHUNK numbers
// that its workgroups take in turn.  Squares are added in 64 bits: no gradient that is finite overflows, and a sum over 10^8 numbers is as exact as one over ten.
// Each workgroup leaves one sum; whoever needs the norm adds these up in order, the workgroups that clip for themselves, which saves a launch between.
#include "matrix_frag.hpp"

namespace ftc {

constexpr int GRAD_ENTRIES = 64, GRAD_THREADS = 256, GRAD_PIECES = 4, GRAD_CHUNK = GRAD_THREADS * GRAD_PIECES;  // a chunk in pieces of eight numbers
constexpr int GRAD_GROUPS = 1024;  // workgroups of a launch at most

struct GradEntry {
    const void *grad;
    void *out;
    int64_t cols, ld, ldo;
    uint32_t rows, pieces;  // pieces of a row (rows 1: not looked at)
    uint32_t first;         // the entry's first chunk
    int32_t dtype;
};
struct GradArgs {
    GradEntry e[GRAD_ENTRIES];
    int entries;
    uint32_t chunks;
    double *sums;  // one a workgroup
};
static_assert(sizeof(GradArgs) <= 4000, "within the arguments of a launch");

// One row, however it is cut; clip: `out`, too.
bool grad_whole(const ftc_grad &g, bool clip) { return g.rows == 1 || (g.ld == g.cols && (!clip || g.ldo == g.cols)); }

#if defined(__HIPCC__)

// This thread's pieces of chunk c: f(entry, which piece, its place in the gradient and in `out`, how many numbers from there on)
template <class F>
__device__ __forceinline__ void each_piece(const GradArgs &a, uint32_t c, const F &f)
{
    int lo = 0, hi = a.entries;  // the last entry that begins at or before it
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.e[mid].first <= c) lo = mid;
        else hi = mid;
    }
    const GradEntry &e = a.e[lo];
    const int64_t piece0 = static_cast<int64_t>(c - e.first) * GRAD_CHUNK + threadIdx.x;
    int64_t at[GRAD_PIECES], to[GRAD_PIECES];
    int left[GRAD_PIECES];
#pragma unroll
    for (int i = 0; i < GRAD_PIECES; ++i) {
        const int64_t piece = piece0 + i * GRAD_THREADS;
        int64_t row = 0, col = piece * 8;
        if (e.rows > 1) {  // uniform
            row = static_cast<uint32_t>(piece) / e.pieces;
            col = static_cast<int64_t>(static_cast<uint32_t>(piece) % e.pieces) * 8;
        }
        at[i] = row * e.ld + col;
        to[i] = row * e.ldo + col;
        const int64_t rest = row < e.rows ? e.cols - col : 0;
        left[i] = static_cast<int>(rest < 8 ? (rest > 0 ? rest : 0) : 8);
    }
    f(e, at, to, left);
}

template <class T>
__device__ __forceinline__ double squares(const GradEntry &e, const int64_t (&at)[GRAD_PIECES], const int (&left)[GRAD_PIECES])
{
    Frag<T> v[GRAD_PIECES];
#pragma unroll
    for (int i = 0; i < GRAD_PIECES; ++i) v[i] = load_frag<T>(e.grad, at[i], left[i]);
    double s = 0;
#pragma unroll
    for (int i = 0; i < GRAD_PIECES; ++i) {
        float x[8];
        frag_numbers<T>(v[i], x);
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fma(static_cast<double>(x[j]), static_cast<double>(x[j]), s);
    }
    return s;
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

__global__ __launch_bounds__(GRAD_THREADS) void grad_squares_kernel(GradArgs a)
{
    __shared__ double area[GRAD_THREADS / 64];
    double s = 0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x)
        each_piece(a, c, [&](const GradEntry &e, const int64_t (&at)[GRAD_PIECES], const int64_t (&)[GRAD_PIECES], const int (&left)[GRAD_PIECES]) {
            if (e.dtype == FTC_F32) s += squares<F32>(e, at, left);
            else if (e.dtype == FTC_F16) s += squares<F16>(e, at, left);
            else s += squares<BF16>(e, at, left);
        });
    s = group_total(s, area);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
}

__device__ __forceinline__ double grad_norm_of(const double *sums, int count, double scale, double *area)
{
    double s = 0;
    for (int i = threadIdx.x; i < count; i += GRAD_THREADS) s += sums[i];
    return sqrt(group_total(s, area)) * scale;
}

__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_kernel(const double *sums, int count, float scale, float *norm)
{
    __shared__ double area[GRAD_THREADS / 64];
    const double v = grad_norm_of(sums, count, fabsf(scale), area);
    if (threadIdx.x == 0) *norm = static_cast<float>(v);
}

template <class T>
__device__ __forceinline__ void scaled(const GradEntry &e, const int64_t (&at)[GRAD_PIECES], const int64_t (&to)[GRAD_PIECES], const int (&left)[GRAD_PIECES], double factor)
{
    Frag<T> v[GRAD_PIECES];
#pragma unroll
    for (int i = 0; i < GRAD_PIECES; ++i) v[i] = load_frag<T>(e.grad, at[i], left[i]);
#pragma unroll
    for (int i = 0; i < GRAD_PIECES; ++i) {
        float x[8];
        frag_numbers<T>(v[i], x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = static_cast<float>(x[j] * factor);
        if (left[i] > 0) store_eight_numbers(e.out, to[i], e.dtype, left[i], x);
    }
}

// From the last chunk to the first: what was read last for the norm is in cache still.
__global__ __launch_bounds__(GRAD_THREADS) void grad_clip_kernel(GradArgs a, const double *sums, int count, float scale, float max_norm, float *norm)
{
    __shared__ double area[GRAD_THREADS / 64];
    const double v = grad_norm_of(sums, count, fabsf(scale), area);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(v);
    double factor = scale;
    if (!(v <= max_norm)) factor *= max_norm / v;  // NaN: NaN, for all to see
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x)
        each_piece(a, a.chunks - 1 - c, [&](const GradEntry &e, const int64_t (&at)[GRAD_PIECES], const int64_t (&to)[GRAD_PIECES], const int (&left)[GRAD_PIECES]) {
            if (factor == 1 && e.out == e.grad) return;  // uniform
            if (e.dtype == FTC_F32) scaled<F32>(e, at, to, left, factor);
            else if (e.dtype == FTC_F16) scaled<F16>(e, at, to, left, factor);
            else scaled<BF16>(e, at, to, left, factor);
        });
}

#endif  // __HIPCC__

// ---- launches --------------------------------------------------------------------------------------------------
static int launches_of(int count) { return (count + GRAD_ENTRIES - 1) / GRAD_ENTRIES; }
size_t grad_norm_ws(int count) { return align_up(static_cast<size_t>(launches_of(count)) * GRAD_GROUPS * sizeof(double), 256); }

// f(arguments, workgroups) for every launch's share of the gradients; sums: for the norm, NULL: to clip
template <class F>
static void each_launch(const ftc_grad *grads, int count, double *sums, const F &f)
{
    for (int from = 0; from < count; from += GRAD_ENTRIES) {
        GradArgs a = {};
        uint32_t chunks = 0;
        for (int i = from; i < count && i < from + GRAD_ENTRIES; ++i) {
            const ftc_grad &g = grads[i];
            if (g.rows == 0 || g.cols == 0) continue;
            const bool whole = grad_whole(g, !sums);
            const int64_t rows = whole ? 1 : g.rows, cols = whole ? g.rows * g.cols : g.cols, pieces = (cols + 7) / 8;
            a.e[a.entries++] = {g.grad, g.out, cols, whole ? 0 : g.ld, whole ? 0 : g.ldo, static_cast<uint32_t>(rows), static_cast<uint32_t>(whole ? 1 : pieces), chunks, g.dtype};
            chunks += static_cast<uint32_t>((rows * pieces + GRAD_CHUNK - 1) / GRAD_CHUNK);
        }
        a.chunks = chunks;
        a.sums = sums;
        const int groups = static_cast<int>(chunks < GRAD_GROUPS ? chunks : GRAD_GROUPS);
        if (groups > 0) f(a, groups);
        if (sums) sums += groups;
    }
}

static int launch_squares(const ftc_grad *grads, int count, void *ws, hipStream_t s)
{
    int parts = 0;
    each_launch(grads, count, static_cast<double *>(ws), [&](const GradArgs &a, int groups) {
        hipLaunchKernelGGL(grad_squares_kernel, dim3(groups), dim3(GRAD_THREADS), 0, s, a);
        parts += groups;
    });
    return parts;
}

int32_t launch_grad_norm(const ftc_grad *grads, int count, float scale, float *norm, void *ws, hipStream_t s)
{
    const int parts = launch_squares(grads, count, ws, s);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(GRAD_THREADS), 0, s, static_cast<const double *>(ws), parts, scale, norm);
    return launch_status("gradient norm");
}

int32_t launch_clip_grad_norm(const ftc_grad *grads, int count, float max_norm, float scale, float *norm, void *ws, hipStream_t s)
{
    const int parts = launch_squares(grads, count, ws, s);
    if (parts == 0) {  // nothing to clip: the norm of nothing
        hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(GRAD_THREADS), 0, s, static_cast<const double *>(ws), 0, scale, norm);
        return launch_status("gradient clipping");
    }
    float *to = norm;  // the first launch writes it
    each_launch(grads, count, nullptr, [&](const GradArgs &a, int groups) {
        hipLaunchKernelGGL(grad_clip_kernel, dim3(groups), dim3(GRAD_THREADS), 0, s, a, static_cast<const double *>(ws), parts, scale, max_norm, to);
        to = nullptr;
    });
    return launch_status("gradient clipping");
}

}  // namespace ftc
