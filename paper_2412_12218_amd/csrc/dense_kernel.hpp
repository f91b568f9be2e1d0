// The product kernel of the dense layer and its gradients (linear.hip): C = A B with an epilogue, in tiles of the result.
//
// A workgroup has a tile; its waves, RW x CW of them, WM x WN blocks of 32 x 32 each (matrix_frag.hpp).  An operand whose memory rows run along the
// contraction is a tile of rows read along rows, one whose memory rows run across it (AX, BX) is read along columns, so nothing is
// transposed in memory.  Steps of 128 bytes of the contraction go from memory to one of two LDS buffers while the other is
// multiplied.
//   whole pieces (FAST)  rows and widths of whole 16-byte pieces at 16-byte alignment: global_load_lds, no registers on the way.  An instruction
//                        fills 64 consecutive pieces of LDS, so the lanes fetch the pieces that the swizzle puts there.  Rows and columns behind the
//                        result's ends are those at the end once more: what they give is not stored.
//   else                 through registers, the last piece of a row as the row's last 16 bytes, moved to their place.
// The indices that a last step lacks are zeros in both operands.
//
// Results go through LDS once more, so that neighbouring lanes have neighbouring columns: bias, activation, residual and the store work on
// eight numbers of a row.
//
// Bound by the matrix instructions for wide layers: 8192^3 in bf16 902 us, 1219 TFLOP/s (a library product of that size 804 to 960); 65 536 x 1024 -> 4096 635 us, 866
// TFLOP/s, 681 with GELU, which the vector units compute for every result while no other workgroup multiplies.  20 000 x 768 -> 768: 31 us, 37 with GELU, 53
// with SiLU, its slope and a residual (124 MB at 2.3 TB/s; tiles of 64, 128 and 256 are level; the residual's rows are asked for before the activation).
// Unaligned: 30 001 x 333 -> 777 61 us, 255 TFLOP/s.  fp32 runs six products of bf16 pieces: 1032 x 3696 -> 2920 197 us, 113 TFLOP/s of fp32.
#pragma once
#include "bf16_split.hpp"
#include "dense_plan.hpp"
#include "matrix_frag.hpp"

namespace ftc {

struct DenseArgs {
    const void *A, *B;  // M x K, K x N
    int64_t lda, ldb;
    int M, N, K, splits, k_each;
    float *part;  // splits x M x N
    const void *bias, *residual;
    void *slope, *out;
    int64_t ldr, lds, ldo;
    int act, out_dtype;
};

// One launch for each place of the operands' rows: Z (A along, B across), dX (both along), dW (both across).
template <bool AX, bool BX>
void launch_dense(const DenseArgs &a, int dtype, int tile, hipStream_t s);

// linear_rows.hip: a few rows of A (dense_few_rows in dense_plan.hpp), B across the contraction or along it
void launch_dense_rows(const DenseArgs &a, int dtype, bool across, hipStream_t s);

// Rows of whole 16-byte pieces at 16-byte alignment, 256 of them within 2^32 bytes.
inline bool dense_whole_pieces(const void *p, int64_t ld, int width, int dtype)
{
    const int e = elem_size(dtype);
    return aligned16(p) && ld * e % 16 == 0 && static_cast<int64_t>(width) * e % 16 == 0 && ld * e < (1 << 24);
}

#if defined(__HIPCC__)
constexpr int SLOPE_BITS = 14;

// act(p) and, if asked for, act'(p), from one exponential and one reciprocal (a step of fp32 each).
//   GELU  p Phi(p) = max(p, 0) - |p| Phi(-|p|).  In 16 bits Phi(-a) = exp(-a^2 / 2) (a1 t + .. + a5 t^5) / 2 and t = 1 / (1 + 0.3275911 a / sqrt 2), off by at
//         most 0.75e-7 (Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26), far below a rounding of the results.  For fp32 inputs nine terms in
//         t = 1 / (1 + 0.35 a), fitted to exp(a^2 / 2) Phi(-a) by weighted least squares such that the largest relative error, 3.2e-8, is least: of normal p
//         the results are 2.1e-8 from 64 bits in the mean (five terms 5.4e-8, p (1 + erf) / 2 in fp32 2.5e-8), of p from -3 to -2 4e-9 (11e-8, 2.1e-8)
//   SiLU  p sigma(p), sigma(p) = 1 / (1 + exp(-p))
// Infinite p: the limits, as the factor that is infinite is cut off where the other is zero.  NaN: through the exponential, which takes p as it is.
template <int ACT, bool SLOPE, bool WIDE>
__device__ __forceinline__ float activation(float p, float &slope)
{
    if constexpr (ACT == FTC_ACT_RELU) {
        slope = p > 0.f ? 1.f : p != p ? p : 0.f;
        return p > 0.f ? p : p != p ? p : 0.f;
    } else if constexpr (ACT == FTC_ACT_GELU) {
        const float e = __builtin_amdgcn_exp2f(p * p * -0.72134752044448170f), t = __builtin_amdgcn_rcpf(fmaf(fabsf(p), WIDE ? 0.35f : 0.23164188f, 1.f));
        constexpr float FIT[2][9] = {{0.127414796f, -0.142248368f, 0.7107068705f, -0.7265760135f, 0.5307027145f},
                                     {0.139621570f, 0.139859083f, 0.119852434f, 0.105432949f, -0.022937165f, 0.158929327f, -0.255504595f, 0.143872250f, -0.029125868f}};
        constexpr int TERMS = WIDE ? 9 : 5;
        float tail = FIT[WIDE][TERMS - 1];
#pragma unroll
        for (int i = TERMS - 2; i >= 0; --i) tail = fmaf(t, tail, FIT[WIDE][i]);
        tail = e * (t * tail);
        if constexpr (SLOPE) slope = fmaf(__builtin_amdgcn_fmed3f(p, -40.f, 40.f) * 0.39894228040143268f, e, p > 0.f ? 1.f - tail : tail);
        return fmaf(-fminf(fabsf(p), 40.f), tail, fmaxf(p, 0.f));
    } else if constexpr (ACT == FTC_ACT_SILU) {
        const float g = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(p * -1.4426950408889634f));
        if constexpr (SLOPE) slope = g * fmaf(__builtin_amdgcn_fmed3f(p, -88.f, 88.f), 1.f - g, 1.f);
        return fmaxf(p, -88.f) * g;
    } else {
        slope = 1.f;
        return p;
    }
}
template <bool SLOPE, bool WIDE>
__device__ __forceinline__ void activations(int act, float (&x)[8], float (&slope)[8])  // act: uniform
{
    auto all = [&](auto code) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = activation<decltype(code)::value, SLOPE, WIDE>(x[j], slope[j]);
    };
    if (act == FTC_ACT_GELU) all(std::integral_constant<int, FTC_ACT_GELU>());
    else if (act == FTC_ACT_SILU) all(std::integral_constant<int, FTC_ACT_SILU>());
    else if (act == FTC_ACT_RELU) all(std::integral_constant<int, FTC_ACT_RELU>());
    else all(std::integral_constant<int, FTC_ACT_NONE>());
}

__device__ __forceinline__ int16_t slope_code(float s)
{
    return s != s ? INT16_MIN : static_cast<int16_t>(rintf(s * (1 << SLOPE_BITS)));
}
__device__ __forceinline__ float slope_value(int16_t c)
{
    return c == INT16_MIN ? __builtin_nanf("") : c * (1.f / (1 << SLOPE_BITS));
}

// Eight neighbouring numbers of a row of the result, `left` of them inside it; bias: theirs.  Bias, activation and its slope.
template <class T>
__device__ __forceinline__ void activate(const DenseArgs &a, int row, int col, int left, const float (&bias)[8], float (&x)[8])
{
    float slope[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += bias[j];
    if (!a.slope) {  // uniform
        if (a.act != FTC_ACT_NONE) activations<false, T::BYTES == 4>(a.act, x, slope);
        return;
    }
    activations<true, T::BYTES == 4>(a.act, x, slope);
    if constexpr (T::BYTES == 4) {
        store_eight_numbers(a.slope, row * a.lds + col, FTC_F32, left, slope);
    } else {
        int16_t *to = static_cast<int16_t *>(a.slope) + row * a.lds + col;
        typedef int16_t s8 __attribute__((ext_vector_type(8), aligned(2)));
        s8 code;
#pragma unroll
        for (int j = 0; j < 8; ++j) code[j] = slope_code(slope[j]);
        if (left >= 8) {
            *reinterpret_cast<s8 *>(to) = code;
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < left) to[j] = code[j];
        }
    }
}
template <class T>
__device__ __forceinline__ void epilogue(const DenseArgs &a, int row, int col, int left, const float (&bias)[8], float (&x)[8])
{
    activate<T>(a, row, col, left, bias, x);
    if (a.residual) {
        float add[8];
        load_eight_numbers<T>(a.residual, row * a.ldr + col, left, add);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += add[j];
    }
    store_eight_numbers(a.out, row * a.ldo + col, a.out_dtype, left, x);
}

// One operand's tile: SIDE rows of the result's side and STEP of the contraction, staged by WAVES waves.
template <class T, int SIDE, int STEP, bool ACROSS, int WAVES>
struct Operand {
    static constexpr int ROWS = ACROSS ? STEP : SIDE, COLS = ACROSS ? SIDE : STEP;
    typedef LdsTile<T, COLS> L;
    static constexpr int BYTES = ROWS * L::ROW, EACH = BYTES / (WAVES * 64 * 16);
    static_assert(BYTES % (WAVES * 64 * 16) == 0, "whole pieces a thread");

    // ---- straight to LDS: piece number e * threads + thread of the tile, as it lies there
    const char *base;    // the step's first number
    uint32_t off[EACH];  // this lane's pieces from there, in bytes (dense_whole_pieces: below 2^32)
    __device__ __forceinline__ void aim(const void *p, int64_t ld, int side0, int side, int k0)
    {
        base = static_cast<const char *>(p) + (ACROSS ? k0 * ld + side0 : side0 * ld + k0) * T::BYTES;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * WAVES * 64 + static_cast<int>(threadIdx.x), r = id / L::PIECES, c = ((id % L::PIECES) ^ L::swizzle(r)) * T::VEC;
            const uint32_t row = ACROSS ? r : min(r, side - 1 - side0), col = ACROSS ? min(c, side - T::VEC - side0) : c;
            off[e] = (row * static_cast<uint32_t>(ld) + col) * T::BYTES;
        }
    }
    // `step`: bytes to the next step
    __device__ __forceinline__ void fetch(char *tile, int64_t step)
    {
        typedef __attribute__((address_space(3))) void *lds_ptr;
        typedef const __attribute__((address_space(1))) void *global_ptr;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            __builtin_amdgcn_global_load_lds((global_ptr)(base + off[e]), (lds_ptr)(tile + (e * WAVES + wave) * 1024), 16, 0, 0);
        base += step;
    }
    // the same where indices from `left` on are to be zeros
    __device__ __forceinline__ void fetch_last(char *tile, int left) const
    {
        ftc_u32x4 w[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * WAVES * 64 + static_cast<int>(threadIdx.x), r = id / L::PIECES, c = ((id % L::PIECES) ^ L::swizzle(r)) * T::VEC;
            w[e] = ftc_u32x4{0u, 0u, 0u, 0u};
            if ((ACROSS ? r : c) < left) w[e] = *reinterpret_cast<const ftc_u32x4 *>(base + off[e]);
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) *reinterpret_cast<ftc_u32x4 *>(tile + (e * WAVES * 64 + static_cast<int>(threadIdx.x)) * 16) = w[e];
    }

    // ---- through registers; `side`, `k_end`: where zeros begin.  A piece that a row ends in is loaded as the last 16 bytes of the row, and
    // its numbers move to their places when it is stored, so that no lane waits for its loads one by one
    ftc_u32x4 v[EACH];
    __device__ __forceinline__ void load(const void *base, int64_t ld, int side0, int side, int k0, int k_end, int width)
    {
        const int row0 = ACROSS ? k0 : side0, rows = ACROSS ? k_end : side, col0 = ACROSS ? side0 : k0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * WAVES * 64 + static_cast<int>(threadIdx.x), r = row0 + id / L::PIECES, c = col0 + id % L::PIECES * T::VEC;
            v[e] = ftc_u32x4{0u, 0u, 0u, 0u};
            if (r < rows && c < width) {
                RawVec<T, T::VEC> w;
                load_raw_any<T>(base, r * ld + min(c, width - T::VEC), w);
                v[e] = ftc_u32x4{w.w[0], w.w[1], w.w[2], w.w[3]};
            }
        }
    }
    // the rows of an operand are shorter than a piece
    __device__ __forceinline__ void load_short(const void *base, int64_t ld, int side0, int side, int k0, int k_end, int width)
    {
        const int row0 = ACROSS ? k0 : side0, rows = ACROSS ? k_end : side, col0 = ACROSS ? side0 : k0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * WAVES * 64 + static_cast<int>(threadIdx.x), r = row0 + id / L::PIECES, c = col0 + id % L::PIECES * T::VEC;
            v[e] = load_piece<T>(base, r * ld + c, r < rows ? width - c : 0);
        }
    }
    // columns from `end` on (of the part of the contraction, where the rows run along it) are zeros; brief: after load_short()
    __device__ __forceinline__ void store(char *tile, int side0, int k0, int k_end, int width, bool brief)
    {
        const int col0 = ACROSS ? side0 : k0, end = ACROSS ? width : k_end;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int id = e * WAVES * 64 + static_cast<int>(threadIdx.x), c = col0 + id % L::PIECES * T::VEC;
            ftc_u32x4 w = v[e];
            if (!brief && c + T::VEC > width) move_down<T>(w, c + T::VEC - width);
            if (!ACROSS && c + T::VEC > end) keep_first<T>(w, end - c);
            L::store(tile, id / L::PIECES, id % L::PIECES, w);
        }
    }

    // the 32 from side0 on, indices 16 s .. of the step
    static __device__ __forceinline__ Frag<T> frag(const char *tile, int side0, int s, int lane)
    {
        const int half = lane >> 5;
        if constexpr (ACROSS) return L::along_column(tile + 16 * s * L::ROW, 8 * half, 8 * half + 4, side0);
        else return L::along_row(tile + side0 * L::ROW, lane & 31, 2 * s + half);
    }
};

// A wave's blocks of an fp32 product from memory and on the fp32 instruction: the sums that the pieces left not finite, or (all) every one.
template <bool AX, bool BX, int WM, int WN>
__device__ __forceinline__ void dense_again(const DenseArgs &a, int row0, int col0, int k_begin, int k_end, bool all, f32x16 (&c)[WM][WN])
{
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const float *A = static_cast<const float *>(a.A), *B = static_cast<const float *>(a.B);
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) {
            const int64_t row = min(row0 + 32 * i + (lane & 31), a.M - 1), col = min(col0 + 32 * j + (lane & 31), a.N - 1);
            f32x16 sum = zero16();
            for (int k0 = k_begin; k0 < k_end; k0 += 2) {
                const int64_t k = k0 + half;
                const bool in = k < k_end;
                const float x = in ? A[AX ? k * a.lda + row : row * a.lda + k] : 0.f, y = in ? B[BX ? k * a.ldb + col : col * a.ldb + k] : 0.f;
                sum = __builtin_amdgcn_mfma_f32_32x32x2f32(y, x, sum, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) c[i][j][e] = !all && fabsf(c[i][j][e]) < INFINITY ? c[i][j][e] : sum[e];
        }
}

// The tiles in the order of bands of eight tile rows, column by column inside a band.
__device__ __forceinline__ void dense_band(int id, int tiles_m, int tiles_n, int &m, int &n)
{
    constexpr int BAND = 8;
    const int band = id / (BAND * tiles_n), in = id % (BAND * tiles_n), rows = min(BAND, tiles_m - band * BAND);
    m = band * BAND + in % rows;
    n = in / rows;
}
// Which tile a workgroup has.  Workgroups go round the eight XCDs, each of which has an L2: every XCD gets a range of consecutive
// tiles (the rest keep their place), so that the tiles at work in an XCD share rows of A and columns of B.
__device__ __forceinline__ void dense_tile(int id, int tiles_m, int tiles_n, int &m, int &n)
{
    const int each = tiles_m * tiles_n / 8;
    if (id < each * 8) id = (id % 8) * each + id / 8;
    dense_band(id, tiles_m, tiles_n, m, n);
}

// The tile (tm, tn) of a product over the indices k_begin .. k_end - 1, with the epilogue, or without it to `part` (rows part_ld apart, the first that of the product).
template <class T, bool AX, bool BX, bool FAST, int RW, int CW, int WM, int WN>
__device__ __forceinline__ void dense_product(const DenseArgs &a, int tm, int tn, int k_begin, int k_end, float *part, int64_t part_ld)
{
    constexpr int WAVES = RW * CW, TM = 32 * WM * RW, TN = 32 * WN * CW, STEP = 128 / T::BYTES, KS = STEP / 16;
    typedef Operand<T, TM, STEP, AX, WAVES> OA;
    typedef Operand<T, TN, STEP, BX, WAVES> OB;
    // arrays of their own: the compiler sees that reads of one buffer need not wait for the loads into the other
    __shared__ __align__(16) char A0[OA::BYTES], B0[OB::BYTES], A1[OA::BYTES], B1[OB::BYTES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int m0 = tm * TM, n0 = tn * TN, wm = wave / CW * 32 * WM, wn = wave % CW * 32 * WN;
    f32x16 c[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) c[i][j] = zero16();
    // operands of the next 16 indices are read while these are multiplied, and not earlier: registers
    auto multiply = [&](const char *A, const char *B) {
        Frag<T> fa[2][WM], fb[2][WN];
        auto read = [&](int s) {
#pragma unroll
            for (int i = 0; i < WM; ++i) fa[s & 1][i] = OA::frag(A, wm + 32 * i, s, lane);
#pragma unroll
            for (int j = 0; j < WN; ++j) fb[s & 1][j] = OB::frag(B, wn + 32 * j, s, lane);
        };
        read(0);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (s + 1 < KS) read(s + 1);
            if constexpr (T::BYTES == 4) {
                Pieces pa[WM], pb[WN];
#pragma unroll
                for (int i = 0; i < WM; ++i) pa[i] = pieces_of(fa[s & 1][i]);
#pragma unroll
                for (int j = 0; j < WN; ++j) pb[j] = pieces_of(fb[s & 1][j]);
#pragma unroll
                for (int i = 0; i < WM; ++i)
#pragma unroll
                    for (int j = 0; j < WN; ++j) mma(c[i][j], pb[j], pa[i]);
            } else {
#pragma unroll
                for (int i = 0; i < WM; ++i)
#pragma unroll
                    for (int j = 0; j < WN; ++j) mma<T>(c[i][j], fb[s & 1][j], fa[s & 1][i]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    OA oa;
    OB ob;
    const bool few = T::BYTES == 4 && a.K <= SPLIT_FROM;  // uniform: sums that pieces would be further off in (bf16_split.hpp)
    if (few) {
    } else if constexpr (FAST) {
        const int64_t da = (AX ? STEP * a.lda : STEP) * T::BYTES, db = (BX ? STEP * a.ldb : STEP) * T::BYTES;
        const int whole = (k_end - k_begin) / STEP, left = (k_end - k_begin) % STEP;
        oa.aim(a.A, a.lda, m0, a.M, k_begin);
        ob.aim(a.B, a.ldb, n0, a.N, k_begin);
        if (whole > 0) {
            oa.fetch(A0, da);
            ob.fetch(B0, db);
        }
        __syncthreads();
        for (int k = 1; k < whole; k += 2) {
            oa.fetch(A1, da);
            ob.fetch(B1, db);
            multiply(A0, B0);
            __syncthreads();
            if (k + 1 < whole) {
                oa.fetch(A0, da);
                ob.fetch(B0, db);
            }
            multiply(A1, B1);
            __syncthreads();
        }
        if (left > 0) {
            oa.fetch_last(A1, left);
            ob.fetch_last(B1, left);
        }
        if (whole & 1) multiply(A0, B0);
        __syncthreads();
        if (left > 0) {
            multiply(A1, B1);
            __syncthreads();
        }
    } else {
        const int wa = AX ? a.M : a.K, wb = BX ? a.N : a.K;  // the operands' rows
        const bool brief = wa < T::VEC || wb < T::VEC;
        auto load = [&](int k) {
            if (brief) {
                oa.load_short(a.A, a.lda, m0, a.M, k, k_end, wa);
                ob.load_short(a.B, a.ldb, n0, a.N, k, k_end, wb);
            } else {
                oa.load(a.A, a.lda, m0, a.M, k, k_end, wa);
                ob.load(a.B, a.ldb, n0, a.N, k, k_end, wb);
            }
        };
        // one buffer is multiplied while the next step, loaded before, goes to the other
        auto turn = [&](int k, const char *__restrict__ A, const char *__restrict__ B, char *__restrict__ An, char *__restrict__ Bn) {
            if (k + STEP < k_end) load(k + STEP);
            multiply(A, B);
            if (k + STEP < k_end) {
                oa.store(An, m0, k + STEP, k_end, wa, brief);
                ob.store(Bn, n0, k + STEP, k_end, wb, brief);
            }
            __syncthreads();
        };
        if (k_begin < k_end) {
            load(k_begin);
            oa.store(A0, m0, k_begin, k_end, wa, brief);
            ob.store(B0, n0, k_begin, k_end, wb, brief);
        }
        __syncthreads();
        for (int k = k_begin, b = 0; k < k_end; k += STEP, b ^= 1) turn(k, b ? A1 : A0, b ? B1 : B0, b ? A0 : A1, b ? B0 : B1);
    }
    if constexpr (T::BYTES == 4) {
        bool finite = true;
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int j = 0; j < WN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) finite = finite && fabsf(c[i][j][e]) < INFINITY;
        if (few || __builtin_amdgcn_ballot_w64(!finite)) dense_again<AX, BX, WM, WN>(a, m0 + wm, n0 + wn, k_begin, k_end, few, c);
    }
    // A wave's 32 rows through LDS, where no other wave looks any more: neighbouring lanes then have neighbouring columns.
    constexpr int WIDTH = 32 * WN, PITCH = WIDTH * 4 + 16, EIGHTS = WIDTH / 8;
    constexpr bool EACH = (WAVES / 4) * 32 * PITCH <= OA::BYTES;  // all four have room for a fourth of the waves, else the two of B for half of them
    static_assert((WAVES / (EACH ? 4 : 2)) * 32 * PITCH <= OB::BYTES, "a place for every wave");
    char *area = EACH ? ((wave & 3) == 0 ? A0 : (wave & 3) == 1 ? B0 : (wave & 3) == 2 ? A1 : B1) + (wave >> 2) * 32 * PITCH
                      : ((wave & 1) == 0 ? B0 : B1) + (wave >> 1) * 32 * PITCH;
    const int q = lane % EIGHTS, col = n0 + wn + 8 * q, left = a.N - col;
    float bias[8];
    load_eight_numbers<T>(a.bias, col, a.bias && !part ? left : 0, bias);
#pragma unroll
    for (int i = 0; i < WM; ++i) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<ftc_f32x4 *>(area + (lane & 31) * PITCH + (32 * j + 8 * b + 4 * (lane >> 5)) * 4) =
                    ftc_f32x4{c[i][j][4 * b], c[i][j][4 * b + 1], c[i][j][4 * b + 2], c[i][j][4 * b + 3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        constexpr int ROWS = 64 / EIGHTS, TURNS = 32 / ROWS;  // rows at a time
        const int r0 = lane / EIGHTS, row0 = m0 + wm + 32 * i;
        const bool adds = a.residual && !part;
        Frag<T> add[TURNS];  // all on their way while the activation is computed
        if (adds) {
#pragma unroll
            for (int t = 0; t < TURNS; ++t) {
                const int row = row0 + r0 + t * ROWS;
                add[t] = load_frag<T>(a.residual, row * a.ldr + col, row < a.M ? left : 0);
            }
        }
#pragma unroll 1
        for (int r = r0; r < 32; r += ROWS) {
            const int row = row0 + r;
            if (row >= a.M || left <= 0) break;
            float *at = reinterpret_cast<float *>(area + r * PITCH + 32 * q);
            const ftc_f32x4 u = *reinterpret_cast<const ftc_f32x4 *>(at), v = *reinterpret_cast<const ftc_f32x4 *>(at + 4);
            float x[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
            if (part) {
                store_eight_numbers(part, row * part_ld + col, FTC_F32, left, x);
                continue;
            }
            activate<T>(a, row, col, left, bias, x);
            if (adds) {  // back to where this lane took them from
                *reinterpret_cast<ftc_f32x4 *>(at) = ftc_f32x4{x[0], x[1], x[2], x[3]};
                *reinterpret_cast<ftc_f32x4 *>(at + 4) = ftc_f32x4{x[4], x[5], x[6], x[7]};
            } else {
                store_eight_numbers(a.out, row * a.ldo + col, a.out_dtype, left, x);
            }
        }
        if (adds) {
#pragma unroll
            for (int t = 0; t < TURNS; ++t) {
                const int r = r0 + t * ROWS, row = row0 + r;
                if (row >= a.M || left <= 0) break;
                const float *at = reinterpret_cast<const float *>(area + r * PITCH + 32 * q);
                float x[8], y[8];
                frag_numbers<T>(add[t], y);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = at[j] + y[j];
                store_eight_numbers(a.out, row * a.ldo + col, a.out_dtype, left, x);
            }
        }
    }
}

template <class T, bool AX, bool BX, bool FAST, int RW, int CW, int WM, int WN>
__global__ __launch_bounds__(64 * RW * CW, 2) void dense_kernel(DenseArgs a)
{
    constexpr int TM = 32 * WM * RW, TN = 32 * WN * CW;
    int tm, tn;
    dense_tile(blockIdx.x, (a.M + TM - 1) / TM, (a.N + TN - 1) / TN, tm, tn);
    const int k_begin = static_cast<int>(blockIdx.y) * a.k_each, k_end = min(a.K, k_begin + a.k_each);
    float *part = a.splits > 1 ? a.part + static_cast<int64_t>(blockIdx.y) * a.M * a.N : nullptr;
    dense_product<T, AX, BX, FAST, RW, CW, WM, WN>(a, tm, tn, k_begin, k_end, part, a.N);
}

template <class T, bool AX, bool BX, bool FAST>
void launch_dense_t(const DenseArgs &a, int tile, hipStream_t s)
{
    const int side = dense_side(tile);
    const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(ceil_div(a.M, side)) * ceil_div(a.N, side)), a.splits);
    if (tile == DENSE_64) {
        hipLaunchKernelGGL((dense_kernel<T, AX, BX, FAST, 2, 2, 1, 1>), grid, dim3(256), 0, s, a);
    } else if (tile == DENSE_128) {
        hipLaunchKernelGGL((dense_kernel<T, AX, BX, FAST, 2, 2, 2, 2>), grid, dim3(256), 0, s, a);
    } else if constexpr (FAST && T::BYTES == 2) {
        hipLaunchKernelGGL((dense_kernel<T, AX, BX, FAST, 2, 4, 4, 2>), grid, dim3(512), 0, s, a);
    }
}

template <bool AX, bool BX>
void launch_dense(const DenseArgs &a, int dtype, int tile, hipStream_t s)
{
    const bool fast = dense_whole_pieces(a.A, a.lda, AX ? a.M : a.K, dtype) && dense_whole_pieces(a.B, a.ldb, BX ? a.N : a.K, dtype);
#define FTC_DENSE(T)                                                  \
    do {                                                             \
        if (fast) launch_dense_t<T, AX, BX, true>(a, tile, s);        \
        else launch_dense_t<T, AX, BX, false>(a, tile, s);            \
    } while (0)
    if (dtype == FTC_F32) FTC_DENSE(F32);
    else if (dtype == FTC_F16) FTC_DENSE(F16);
    else FTC_DENSE(BF16);
#undef FTC_DENSE
}

#endif  // __HIPCC__
}  // namespace ftc
