// Rows of the norms around a block (block_norm.hip, block_norm_backward.hip): which lanes have a row, its sums, its statistics.
//
// A row is in the registers of L lanes, C pieces of eight numbers each, lane l having the pieces l, l + L, ...; it is read once whatever is computed
// of it.  Up to 64 lanes are lanes of one wave and their sums stay in registers; more are waves of one workgroup, whose sums meet in LDS.
#pragma once
#include <initializer_list>

#include "stream_piece.hpp"

namespace ftc {

// Lanes of a row: as many as make it one piece each, up to 512, and two from there on, 1024 lanes above 8192 numbers.  Rows of a workgroup that are 2^31 bytes apart have 64 lanes at least.
constexpr int ROW_LANES[] = {4, 8, 16, 32, 64, 128, 192, 256, 384, 512};
inline int row_lanes(int d, int64_t widest_ld, int bytes)
{
    const int least = 64 * widest_ld * bytes < (1ll << 31) ? 4 : 64;
    for (int lanes : ROW_LANES)
        if (lanes >= least && d <= (lanes == 512 ? 16 : 8) * lanes) return lanes;
    return 1024;
}
constexpr int row_threads(int lanes) { return lanes > 64 ? lanes : 256; }  // of a workgroup

// Workgroups of a launch: at most as many as the compute units hold at once, and as many turns for each of them.
inline int row_groups(int n, int lanes, int threads_a_unit)
{
    const int threads = row_threads(lanes), groups = ceil_div(n, threads / lanes), most = 256 * (threads_a_unit / threads > 0 ? threads_a_unit / threads : 1);
    return groups <= most ? groups : ceil_div(groups, ceil_div(groups, most));
}
// Whether a pass over these matrices (NULL: not there) takes the non-temporal hint (stream_piece.hpp): more than a third of the last-level cache of 256 MB, of which the kernels
// before and behind have theirs.  us with / without, over three sets of inputs in turn: 74 MB (46 000 x 200 in fp32, normed) 16.6 / 13.5; 123 MB (20 000 x 768 in bf16, a block's join with two layer norms) 35.0 / 36.6, its gradients
// (184 MB) with their sums 52.4 / 53.3; 256 MB (200 000 x 128) 46 / 50; 410 MB (50 000 x 1024) 76 / 82.
inline bool row_stream(int n, int d, int bytes, std::initializer_list<const void *> matrices)
{
    int64_t all = 0;
    for (const void *p : matrices) all += p ? static_cast<int64_t>(n) * d * bytes : 0;
    return all > 85ll << 20;
}

struct BlockArgs {
    int n, d, post, pre;
    float eps, x_scale;
    const void *X, *F, *gate, *post_w, *post_b, *pre_w, *pre_b;
    int64_t ldx, ldf, ldg;  // ldg: 0 where all rows have one gate
};

#if defined(__HIPCC__)

// Totals of K sums, one or two, over the L lanes of a row, in each of them.  `area`: 2 x 32 floats of LDS, `turn`: which half, the other one at the next call, whatever its K
// (a wave that writes a half again has passed the barrier of the call between, and so have all that read it).
template <int L, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float *area, int &turn)
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if constexpr (L >= 64) v[k] += __shfl_xor(v[k], 32, 64);
        v[k] = group_sum_dpp<(L < 64 ? L : 32)>(v[k]);
    }
    if constexpr (L > 64) {
        constexpr int WAVES = L / 64;
        const int wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;  // of the row
        static_assert(K <= 2, "within a half");
        float *half = area + turn * 32;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) half[k * 16 + wave] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[k] += half[k * 16 + first + w];
        }
        turn ^= 1;
    }
}

// A lane's C pieces of rows of d numbers.  Loads and stores are of 16 bytes, those of neighbouring lanes beside each other: in fp32 a piece is two of
// them, 4 L numbers apart.  What a lane adds to the address of the workgroup's first row (of its own row, from 64 lanes on) is 32 bits and the same for every turn.
// WHOLE: rows are whole 16 bytes, which are there or not; else the last ones of a row are loaded as the row's last 16 bytes, and moved.
template <class T, int L, int C, bool WHOLE, bool NT>
struct RowPieces {
    static constexpr int V = T::VEC, UNITS = 8 / V;
    int d, lane, sub;  // sub: which of the workgroup's rows (uniform from 64 lanes on)
    __device__ __forceinline__ int col(int c, int u) const { return V * ((c * UNITS + u) * L + lane); }
    __device__ __forceinline__ bool has(int c, int j) const { return WHOLE ? col(c, j / V) < d : col(c, j / V) + j % V < d; }
    // of the number `col` of this lane's row
    __device__ __forceinline__ int64_t byte(int64_t row0, int64_t ld, int col) const
    {
        if constexpr (L >= 64) return (row0 + sub) * ld * T::BYTES + static_cast<uint32_t>(col * T::BYTES);
        else return row0 * ld * T::BYTES + (static_cast<uint32_t>(sub) * static_cast<uint32_t>(ld) + static_cast<uint32_t>(col)) * static_cast<uint32_t>(T::BYTES);
    }
    static __device__ __forceinline__ ftc_u32x4 whole_piece(const void *base, int64_t at) { return NT ? load_piece_nt<T>(base, at) : load_piece<T>(base, at, V); }
    static __device__ __forceinline__ void store_whole(void *base, int64_t at, const float (&y)[V])
    {
        if constexpr (NT) store_piece_nt<T>(base, at, y);
        else store_piece<T>(base, at, y);
    }
    static __device__ __forceinline__ void put(Frag<T> &f, int u, ftc_u32x4 w)
    {
        if constexpr (T::BYTES == 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f.f[4 * u + j] = __uint_as_float(w[j]);
        } else {
            f.w = w;
        }
    }
    static __device__ __forceinline__ void clear(Frag<T> (&f)[C])
    {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int u = 0; u < UNITS; ++u) put(f[c], u, ftc_u32x4{0u, 0u, 0u, 0u});
    }
    // What this lane has of a row of the workgroup's, row0 the first of them; there: whether there is this lane's.  What is not there keeps what it was.
    __device__ __forceinline__ void load(const void *base, int64_t ld, int64_t row0, bool there, Frag<T> (&f)[C]) const
    {
        const char *p = static_cast<const char *>(base);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int at = col(c, u);
                if (!there || at >= d) continue;
                ftc_u32x4 w;
                if (WHOLE || d >= V) w = whole_piece(p + byte(row0, ld, WHOLE ? at : min(at, d - V)), 0);
                else w = load_piece<T>(p + byte(row0, ld, at), 0, d);
                put(f[c], u, w);
            }
    }
    // The numbers of what load() brought; the last ones of a row go to their places here, not where the load would have to be waited for.
    __device__ __forceinline__ void numbers(const Frag<T> (&f)[C], float (&x)[C][8]) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            Frag<T> v = f[c];
            if constexpr (!WHOLE) {
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    const int at = col(c, u);
                    if (d < V || at >= d || at + V <= d) continue;
                    ftc_u32x4 w;
                    if constexpr (T::BYTES == 4) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(v.f[4 * u + j]);
                    } else {
                        w = v.w;
                    }
                    move_down<T>(w, at + V - d);
                    put(v, u, w);
                }
            }
            frag_numbers<T>(v, x[c]);
        }
    }
    __device__ __forceinline__ void store(void *base, int64_t ld, int64_t row0, bool there, const float (&x)[C][8]) const
    {
        char *p = static_cast<char *>(base);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int at = col(c, u), left = d - at;
                if (!there || left <= 0) continue;
                char *to = p + byte(row0, ld, at);
                float y[V];
#pragma unroll
                for (int j = 0; j < V; ++j) y[j] = x[c][u * V + j];
                if (WHOLE || left >= V) store_whole(to, 0, y);
                else store_first<T>(to, left, y);
            }
    }
    // A vector of d numbers; all vectors are loaded before the first is looked at.  NULL: `none` each
    __device__ __forceinline__ void fetch(const void *base, Frag<T> (&f)[C]) const
    {
        clear(f);
        if (!base) return;  // uniform
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int at = col(c, u);
                if (at >= d) continue;
                ftc_u32x4 w;
                if (WHOLE || d >= V) w = load_piece<T>(base, WHOLE ? at : min(at, d - V), V);
                else w = load_piece<T>(base, at, d);
                put(f[c], u, w);
            }
    }
    __device__ __forceinline__ void vector(const void *base, const Frag<T> (&f)[C], float none, float (&x)[C][8]) const
    {
        if (base) {
            numbers(f, x);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] = none;
        }
    }
};

// Mean (0 for FTC_NORM_RMS) of a row and what its distance from there is multiplied by.  A sum of d numbers is off by some roundings of the numbers
// themselves, which is much beside a small spread, so the mean is taken in two steps: the distances from the first one, m, are exact but for a rounding of their own,
// and their mean, which the sum of their squares brings along, is what m is off by.  sum (x - m)^2 / d is more than the variance by the square of that; where this is not
// little (equal numbers), the squares are summed again.  So are, times 2^-96, distances from 1e19 on, whose squares are infinite in fp32,
// also where only eps makes them so.
template <class T, int L, int C, bool WHOLE, bool NT>
__device__ __forceinline__ void row_statistics(const RowPieces<T, L, C, WHOLE, NT> &r, int kind, float eps, const float (&x)[C][8], float *area, int &turn, float &mean, float &rstd)
{
    const float each = 1.f / static_cast<float>(r.d);
    float s[1] = {0.f}, moved = 0.f;
    mean = 0.f;
    if (kind == FTC_NORM_LAYER) {  // uniform
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] = fmaf(x[c][j], each, s[0]);  // zeros behind the row; no sum beyond the largest number
        row_sums<L, 1>(s, area, turn);
        mean = s[0];
        float two[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = r.has(c, j) ? x[c][j] - mean : 0.f;
                two[0] = fmaf(v, v, two[0]);
                two[1] = fmaf(v, each, two[1]);
            }
        row_sums<L, 2>(two, area, turn);
        s[0] = two[0];
        mean += two[1];
        moved = two[1] * two[1];
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] = fmaf(x[c][j], x[c][j], s[0]);
        row_sums<L, 1>(s, area, turn);
    }
    const float square = fmaf(s[0], each, eps - moved);
    rstd = 1.f / sqrtf(square);
    // lanes that meet in row_sums go the same way: those of a wave, or of a workgroup, which has one row then
    const bool wide = !(square < INFINITY), again = wide || 64.f * moved > s[0] * each;
    if (L > 64 ? again : __builtin_amdgcn_ballot_w64(again) != 0) {
        const float scale = wide ? 0x1p-96f : 1.f;
        s[0] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = r.has(c, j) ? (x[c][j] - mean) * scale : 0.f;
                s[0] = fmaf(v, v, s[0]);
            }
        row_sums<L, 1>(s, area, turn);
        if (again) rstd = scale / sqrtf(fmaf(s[0], each, eps * scale * scale));
    }
}

#endif  // __HIPCC__
}  // namespace ftc
