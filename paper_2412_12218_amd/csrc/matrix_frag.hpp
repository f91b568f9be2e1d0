// Operands of 32 x 32 matrix-core products, as the attention and linear kernels hold them: in registers, and as swizzled
// tiles in LDS that can be read along their rows or along their columns.
//
// A step of a product contracts 16 indices: lane l holds, of row (column) l % 32 of its operand, the eight indices of half
// l / 32.  In 16 bits that is one v_mfma_f32_32x32x16; in fp32 eight v_mfma_f32_32x32x2 with one index of each half (attention), or six
// v_mfma_f32_32x32x16 of bf16 pieces (dense layer), so kernels are written once for the three types.  Which eight indices a half has is free as long as both operands agree; the result
// of a product (lane l: column l % 32, rows 8 b + 4 (l / 32) + i in element 4 b + i) is itself an operand of a next product
// over its rows with the order {4 h + i, 8 + 4 h + i} of each 16, which the reads along columns can give.
#pragma once
#include "ftc_common.hpp"

namespace ftc {
#if defined(__HIPCC__)

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float frag_f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 frag_half8 __attribute__((ext_vector_type(8)));
typedef __bf16 frag_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 frag_half2 __attribute__((ext_vector_type(2)));
typedef __bf16 frag_bf16x2 __attribute__((ext_vector_type(2)));
typedef short frag_s16x4 __attribute__((ext_vector_type(4)));

// Eight numbers of one row (column) of an operand.
template <class T>
struct Frag {
    ftc_u32x4 w;
};
template <>
struct Frag<F32> {
    float f[8];
};

// Eight fp32 numbers as an operand, rounded to nearest even where it has 16 bits.
template <class T>
__device__ __forceinline__ Frag<T> frag_of(const float (&x)[8])
{
    Frag<T> a;
    if constexpr (T::BYTES == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) a.f[j] = x[j];
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const frag_f32x2 v = {x[2 * j], x[2 * j + 1]};
            if constexpr (std::is_same<T, F16>::value) a.w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, frag_half2));
            else a.w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, frag_bf16x2));
        }
    }
    return a;
}

template <class T>
__device__ __forceinline__ void mma(f32x16 &c, const Frag<T> &a, const Frag<T> &b)
{
    if constexpr (T::BYTES == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.f[j], b.f[j], c, 0, 0, 0);
    } else if constexpr (std::is_same<T, F16>::value) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(frag_half8, a.w), __builtin_bit_cast(frag_half8, b.w), c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(frag_bf16x8, a.w), __builtin_bit_cast(frag_bf16x8, b.w), c, 0, 0, 0);
    }
}

// An fp32 operand in three bf16 pieces, a = a1 + a2 + a3 (bf16_split.hpp: six of the nine products are exact in fp32 and what is left out is below an
// fp32 rounding), for products at six sixteenths of the time of v_mfma_f32_32x32x2.  Infinities, numbers that round to one, and sums of pieces that overflow
// show as results that are not finite.  Numbers below 2^-110 are held to 2^-134, half a step of the smallest bf16 numbers, and that does not show: bf16_split.hpp
// looks at every last piece, which here, where each wave takes its operands apart by itself, costs 6 to 17 % of the time of every fp32 product (16 384 x 2048
// x 2048 736 / 781 us, a training step of 20 000 x 768 -> 768 519 / 605; with the packed first pieces, each looked at by one wave of a workgroup, 1 to 11 %).
struct Pieces {
    Frag<BF16> p[3];
};
__device__ __forceinline__ Pieces pieces_of(const Frag<F32> &a)
{
    Pieces s;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x = a.f[2 * j], y = a.f[2 * j + 1];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector((frag_f32x2{x, y}), frag_bf16x2));
            s.p[q].w[j] = w;
            if (q < 2) {
                x -= __uint_as_float(w << 16);
                y -= __uint_as_float(w & 0xffff0000u);
            }
        }
    }
    return s;
}
__device__ __forceinline__ void mma(f32x16 &c, const Pieces &a, const Pieces &b)  // the smallest first
{
    mma<BF16>(c, a.p[1], b.p[1]);
    mma<BF16>(c, a.p[2], b.p[0]);
    mma<BF16>(c, a.p[0], b.p[2]);
    mma<BF16>(c, a.p[1], b.p[0]);
    mma<BF16>(c, a.p[0], b.p[1]);
    mma<BF16>(c, a.p[0], b.p[0]);
}

// ---- global memory ----------------------------------------------------------------------------------------
// 16 bytes (T::VEC elements) at element `idx`, aligned to an element; elements from `left` on are zero and not read.
template <class T>
__device__ __forceinline__ ftc_u32x4 load_piece(const void *base, int64_t idx, int left)
{
    ftc_u32x4 v = {0u, 0u, 0u, 0u};
    if (left >= T::VEC) {
        RawVec<T, T::VEC> r;
        load_raw_any<T>(base, idx, r);
        v = ftc_u32x4{r.w[0], r.w[1], r.w[2], r.w[3]};
    } else if (left > 0) {
        if constexpr (T::BYTES == 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = j < left ? static_cast<const uint32_t *>(base)[idx + j] : 0u;
        } else {
            const uint16_t *p = static_cast<const uint16_t *>(base) + idx;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (2 * j < left ? p[2 * j] : 0u) | ((2 * j + 1 < left ? static_cast<uint32_t>(p[2 * j + 1]) : 0u) << 16);
        }
    }
    return v;
}

template <class T>
__device__ __forceinline__ Frag<T> load_frag(const void *base, int64_t idx, int left)
{
    Frag<T> a;
    if constexpr (T::BYTES == 4) {
        const ftc_u32x4 x = load_piece<T>(base, idx, left), y = load_piece<T>(base, idx + 4, left - 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) { a.f[j] = __uint_as_float(x[j]); a.f[4 + j] = __uint_as_float(y[j]); }
    } else {
        a.w = load_piece<T>(base, idx, left);
    }
    return a;
}

// Elements moved to places s lower (0 < s < VEC, or all of it), zeros behind; and those from n on zeros.
template <class T>
__device__ __forceinline__ void move_down(ftc_u32x4 &w, int s)
{
    if constexpr (T::BYTES == 2) {
        if (s & 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (w[j] >> 16) | (j < 3 ? w[j + 1] << 16 : 0u);
        }
        s >>= 1;
    }
#pragma unroll
    for (int b = 1; b <= 2; b *= 2)
        if (s & b) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = j + b < 4 ? w[j + b] : 0u;
        }
    if (s >= 4) w = ftc_u32x4{0u, 0u, 0u, 0u};
}
template <class T>
__device__ __forceinline__ void keep_first(ftc_u32x4 &w, int n)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (T::BYTES == 4) w[j] = j < n ? w[j] : 0u;
        else w[j] = 2 * j + 1 < n ? w[j] : 2 * j < n ? w[j] & 0xffffu : 0u;
    }
}

// The piece from element c on of a row of `width` elements that is readable from `row` on, zeros behind it, without a branch for the row's last piece:
// the last 16 bytes of the row, moved.
template <class T>
__device__ __forceinline__ ftc_u32x4 load_piece_of_row(const void *row, int c, int width)
{
    if (width < T::VEC) return load_piece<T>(row, c, width - c);  // uniform
    RawVec<T, T::VEC> r;
    load_raw_any<T>(row, min(c, width - T::VEC), r);
    ftc_u32x4 v = {r.w[0], r.w[1], r.w[2], r.w[3]};
    if (c + T::VEC > width) move_down<T>(v, c + T::VEC - width);
    return v;
}

// The eight numbers of an operand in fp32.
template <class T>
__device__ __forceinline__ void frag_numbers(const Frag<T> &a, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (T::BYTES == 4) x[j] = a.f[j];
        else if constexpr (std::is_same<T, F16>::value) x[j] = f16_bits_to_f32((a.w[j / 2] >> (16 * (j & 1))) & 0xffffu);
        else x[j] = bf16_bits_to_f32((a.w[j / 2] >> (16 * (j & 1))) & 0xffffu);
    }
}
// Eight consecutive numbers at element `idx`, aligned to an element; those from `left` on are zero and not read.
template <class T>
__device__ __forceinline__ void load_eight_numbers(const void *base, int64_t idx, int left, float (&x)[8])
{
    frag_numbers<T>(load_frag<T>(base, idx, left), x);
}
// ... in a run-time type; those from `left` on are not written
__device__ __forceinline__ void store_eight_numbers(void *base, int64_t idx, int dtype, int left, const float (&x)[8])
{
    if (left >= 8) {
        if (dtype == FTC_F32) {
            store_vec_any<8>(base, idx, dtype, x);
        } else {
            typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
            const ftc_u32x4 w = dtype == FTC_F16 ? frag_of<F16>(x).w : frag_of<BF16>(x).w;
            *reinterpret_cast<u4 *>(static_cast<uint16_t *>(base) + idx) = u4{w[0], w[1], w[2], w[3]};
        }
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) store_elem(base, idx + j, dtype, x[j]);
    }
}

// Four consecutive numbers at element `idx`, aligned to an element; those from `left` on are not written.
template <class T>
__device__ __forceinline__ void store_four(void *base, int64_t idx, int left, const float (&x)[4])
{
    constexpr int DT = T::BYTES == 4 ? FTC_F32 : std::is_same<T, F16>::value ? FTC_F16 : FTC_BF16;
    if (left >= 4) {
        store_vec_any<4>(base, idx, DT, x);
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < left) store_elem(base, idx + j, DT, x[j]);
    }
}

// ---- tiles in LDS -------------------------------------------------------------------------------------------
// Rows of COLS elements, 16-byte pieces permuted inside a row by its number: the 16 rows that a read along rows touches at
// once, and the four rows by 64 bytes of a read along columns, each fall on the 64 banks without conflict.  The permutation repeats
// every 16 rows, so reads take the place of such a row as `tile` and rows from there: what remains of an address is the lane's, and the
// same for all of them.
template <class T, int COLS>
struct LdsTile {
    static constexpr int ROW = COLS * T::BYTES, PIECES = ROW / 16;
    static_assert(ROW == 64 || ROW == 128 || ROW % 256 == 0, "pieces are permuted inside 4, 8 or 16 pieces");
    static __device__ __forceinline__ int swizzle(int r)
    {
        if constexpr (ROW == 64) return (r >> 2) & 3;
        else if constexpr (ROW == 128) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
        else return ((r & 3) << 2) | ((r >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int r, int piece) { return r * ROW + ((piece ^ swizzle(r)) << 4); }

    static __device__ __forceinline__ void store(char *tile, int r, int piece, ftc_u32x4 v)
    {
        *reinterpret_cast<ftc_u32x4 *>(tile + at(r, piece)) = v;
    }
    // elements 8 e .. 8 e + 7 of row r (r, e: this lane's)
    static __device__ __forceinline__ Frag<T> along_row(const char *tile, int r, int e)
    {
        Frag<T> a;
        if constexpr (T::BYTES == 4) {
            const ftc_f32x4 x = *reinterpret_cast<const ftc_f32x4 *>(tile + at(r, 2 * e));
            const ftc_f32x4 y = *reinterpret_cast<const ftc_f32x4 *>(tile + at(r, 2 * e + 1));
#pragma unroll
            for (int j = 0; j < 4; ++j) { a.f[j] = x[j]; a.f[4 + j] = y[j]; }
        } else {
            a.w = *reinterpret_cast<const ftc_u32x4 *>(tile + at(r, e));
        }
        return a;
    }
    // rows r0 .. r0 + 3, r1 .. r1 + 3 of column col0 + lane % 32 (r0, r1: the same in a half of the wave, multiples of 4).  In 16 bits
    // ds_read_b64_tr_b16: 16 lanes read four rows of 16 elements, lane 4 i + j the four elements from 4 j of row i, and lane k gets
    // element k of the four rows.
    static __device__ __forceinline__ Frag<T> along_column(const char *tile, int r0, int r1, int col0)
    {
        const int lane = threadIdx.x & 63;
        Frag<T> a;
        if constexpr (T::BYTES == 4) {
            const int col = col0 + (lane & 31), piece = col >> 2, in = (col & 3) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a.f[j] = *reinterpret_cast<const float *>(tile + at(r0 + j, piece) + in);
                a.f[4 + j] = *reinterpret_cast<const float *>(tile + at(r1 + j, piece) + in);
            }
        } else {
            typedef __attribute__((address_space(3))) frag_s16x4 *lds_ptr;
            const int row = (lane & 15) >> 2, col = col0 + (lane & 16) + (lane & 3) * 4, piece = col >> 3, in = (col & 4) * 2;
            const frag_s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + at(r0 + row, piece) + in));
            const frag_s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + at(r1 + row, piece) + in));
            const ftc_u32x2 u = __builtin_bit_cast(ftc_u32x2, x), v = __builtin_bit_cast(ftc_u32x2, y);
            a.w = ftc_u32x4{u[0], u[1], v[0], v[1]};
        }
        return a;
    }
};

__device__ __forceinline__ f32x16 zero16()
{
    f32x16 z;
#pragma unroll
    for (int j = 0; j < 16; ++j) z[j] = 0.f;
    return z;
}

#endif  // __HIPCC__
}  // namespace ftc
