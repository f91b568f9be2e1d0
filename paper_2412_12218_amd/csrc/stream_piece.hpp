// 16-byte pieces, aligned to their elements, of data that a kernel touches once and nobody soon after: with the non-temporal hint such stores do not stay in the
// last-level cache, where what they push out, and their own way to memory later, costs the kernels behind.  Copies of 256 MB on one MI355X: 5.6 TB/s, with the hint on both sides
// 6.3 TB/s; reads 6.3 and 6.8.  A pass that reads 253 MB behind one that wrote as much: 70 us, 47 with the hint on those stores.
#pragma once
#include "matrix_frag.hpp"

namespace ftc {
#if defined(__HIPCC__)

template <class T>
__device__ __forceinline__ ftc_u32x4 load_piece_nt(const void *base, int64_t idx)
{
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
    const u4 v = __builtin_nontemporal_load(reinterpret_cast<const u4 *>(static_cast<const char *>(base) + idx * T::BYTES));
    return ftc_u32x4{v.x, v.y, v.z, v.w};
}
template <class T>  // without the hint
__device__ __forceinline__ void store_piece(void *base, int64_t idx, const float (&x)[T::VEC])
{
    if constexpr (T::BYTES == 4) {
        typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
        *reinterpret_cast<f4 *>(static_cast<float *>(base) + idx) = f4{x[0], x[1], x[2], x[3]};
    } else {
        typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
        const ftc_u32x4 w = frag_of<T>(x).w;
        *reinterpret_cast<u4 *>(static_cast<uint16_t *>(base) + idx) = u4{w[0], w[1], w[2], w[3]};
    }
}
template <class T>
__device__ __forceinline__ void store_piece_nt(void *base, int64_t idx, const float (&x)[T::VEC])
{
    if constexpr (T::BYTES == 4) {
        typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
        const f4 v = {x[0], x[1], x[2], x[3]};
        __builtin_nontemporal_store(v, reinterpret_cast<f4 *>(static_cast<float *>(base) + idx));
    } else {
        typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
        const ftc_u32x4 w = frag_of<T>(x).w;
        const u4 v = {w[0], w[1], w[2], w[3]};
        __builtin_nontemporal_store(v, reinterpret_cast<u4 *>(static_cast<uint16_t *>(base) + idx));
    }
}

// The first `left` numbers of a piece, fewer than it has, in at most three stores.
template <class T>
__device__ __forceinline__ void store_first(void *base, int left, const float (&x)[T::VEC])
{
    if constexpr (T::BYTES == 4) {
        float *p = static_cast<float *>(base);
        typedef float f2 __attribute__((ext_vector_type(2), aligned(4)));
        float last = x[0];
        if (left & 2) {
            *reinterpret_cast<f2 *>(p) = f2{x[0], x[1]};
            last = x[2];
            p += 2;
        }
        if (left & 1) *p = last;
    } else {
        typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
        typedef uint32_t u1 __attribute__((aligned(2)));
        uint16_t *p = static_cast<uint16_t *>(base);
        ftc_u32x4 w = frag_of<T>(x).w;
        if (left & 4) {
            *reinterpret_cast<u2 *>(p) = u2{w[0], w[1]};
            w[0] = w[2];
            w[1] = w[3];
            p += 4;
        }
        if (left & 2) {
            *reinterpret_cast<u1 *>(p) = w[0];
            w[0] = w[1];
            p += 2;
        }
        if (left & 1) *p = static_cast<uint16_t>(w[0]);
    }
}

#endif  // __HIPCC__
}  // namespace ftc
