// Tensors of the three element types (qgx_dtype) in the kernels beside the exchange: 16 bytes at a time, as binary32.
#pragma once

#include "qgx_device.h"

namespace qgx {

// A piece: 16 bytes of elements, at any multiple of an element's size (global accesses of 16 bytes need no more on this
// target: the type's alignment says so to the compiler, which then keeps them whole), so that rows of odd widths and tensors at odd
// places take the same path as aligned ones.
template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);

template <typename T> struct PieceOf { typedef T type __attribute__((ext_vector_type(kPiece<T>), aligned(sizeof(T)))); };

template <typename T> using Piece = typename PieceOf<T>::type;

template <typename T>
__device__ __forceinline__ nt_u32x4 load_bits(const T* p)
{
    return __builtin_bit_cast(nt_u32x4, *reinterpret_cast<const Piece<T>*>(p));
}

// The elements of a piece out of its four words.  (Word by word: taken from a vector of 16-bit elements, the compiler keeps each in a
// register of its own from the load on.)
template <typename T>
__device__ __forceinline__ void values_of(nt_u32x4 x, float (&v)[kPiece<T>])
{
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            v[i] = __uint_as_float(x[i]);
        } else if constexpr (__is_same(T, _Float16)) {
            const pair h = __builtin_bit_cast(pair, (uint32_t)x[i]);
            v[2 * i] = (float)h.x;
            v[2 * i + 1] = (float)h.y;
        } else {
            v[2 * i] = __uint_as_float(x[i] << 16);
            v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
        }
    }
}

template <typename T>
__device__ __forceinline__ void load_piece(const T* p, float (&v)[kPiece<T>])
{
    values_of<T>(load_bits(p), v);
}

template <typename T>
__device__ __forceinline__ void store_piece(T* p, const float (&v)[kPiece<T>])
{
    Piece<T> x;
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) x[i] = (T)v[i];
    *reinterpret_cast<Piece<T>*>(p) = x;
}

// A store of what is not read again soon: marked non-temporal (see nt_load4).
template <typename T>
__device__ __forceinline__ void stream_piece(T* p, const float (&v)[kPiece<T>])
{
    Piece<T> x;
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) x[i] = (T)v[i];
    __builtin_nontemporal_store(x, reinterpret_cast<Piece<T>*>(p));
}

// The same for the first n elements of a piece (any n; zeros beyond), where the rest may be no memory at all.
template <typename T>
__device__ __forceinline__ Piece<T> load_raw(const T* p, int n)
{
    if (n >= kPiece<T>) return *reinterpret_cast<const Piece<T>*>(p);
    Piece<T> x;
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) x[i] = i < n ? p[i] : (T)0.0f;
    return x;
}

template <typename T>
__device__ __forceinline__ void load_piece(const T* p, int n, float (&v)[kPiece<T>])
{
    if (n >= kPiece<T>) return load_piece(p, v);
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
}

template <typename T>
__device__ __forceinline__ void store_piece(T* p, int n, const float (&v)[kPiece<T>])
{
    if (n >= kPiece<T>) return store_piece(p, v);
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i)
        if (i < n) p[i] = (T)v[i];
}

// The sum of LANES neighbouring lanes (4, 16 or 64) in each of them, lanes i and i xor LANES / 2 .. 1 joined in turn.
template <int LANES, int D = LANES / 2>
__device__ __forceinline__ float lanes_sum(float x)
{
    static_assert(LANES == 4 || LANES == 16 || LANES == 64, "see xor_lane");
    const LanePair p = lane_pair<D>(__float_as_uint(x));
    x = __uint_as_float(p.a) + __uint_as_float(p.b);
    if constexpr (D > 1) return lanes_sum<LANES, D / 2>(x);
    else return x;
}

}  // namespace qgx
