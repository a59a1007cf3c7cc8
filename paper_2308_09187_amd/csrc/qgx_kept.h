// Activations kept in 8 bits: a block of 32 elements of a row has one power of two 2^e, an element is a whole number of at most 127 of
// it.  The numbers are powers of two apart so that a kept element is exact in bfloat16 (8 bits of significand): products with it on the matrix cores are
// exact, and so is a decoding by one multiplication.  Against a scale of its own (the block's maximum / 127) the step is up to twice as wide,
// 1.4 times on average.
#pragma once

#include "qgx_types.h"

namespace qgx {

// A block's stored power: the smallest 2^e with the largest magnitude at most 127 * 2^e (127 = 1.984375 * 2^6), biased by 127; 0 for zeros.  From
// the magnitude's bits: a significand beyond 1.984375 carries into the exponent.
constexpr uint32_t kKeptSpoilt = 255u;                     // of a block with an infinity or a NaN
__device__ __forceinline__ uint32_t kept_power(uint32_t bits) { return (uint32_t)max((int)((bits + 0x1FFFFu) >> 23) - 6, 0); }

// What that leaves to be put right: infinities and NaNs, magnitudes beyond the type's largest power `top` or below those whose inverse powers, times 2^16,
// are numbers.
__device__ __forceinline__ bool kept_is_rare(uint32_t bits, uint32_t power, uint32_t top)
{
    return power >= top || (bits != 0u && power < 16u);
}

// 2^e; 0 for zeros, infinity (and so 0 * infinity = NaN) for a spoilt block.
__device__ __forceinline__ float kept_scale(uint32_t power) { return __uint_as_float(power << 23); }

// An element out of its byte: both steps exact.
__device__ __forceinline__ float kept_value(uint32_t code, float scale) { return ((float)code - 128.0f) * scale; }

__device__ __forceinline__ uint32_t kept_call(const KeptDraws& d, const Scalars* sc)
{
    return d.call_mode ? 2u * (scalar_load(&sc->t) - 1u) + (d.call_mode - 1u) : d.call_id;
}

// A code rounded to the nearest whole number, into byte `at` of a word: u = the element over the block's power of two.
__device__ __forceinline__ uint32_t kept_code(float u, uint32_t at, uint32_t word)
{
    return __builtin_amdgcn_cvt_pk_u8_f32(rintf(u) + 128.0f, at, word);
}

// Four codes rounded away from zero where the draw d, 16 bits, is below 2^16 times the remainder of |u|, u16 = 2^16 u.  With T = ceil(2^16 |u|), a whole
// number of 23 bits, the magnitude's negative is (d - T) >> 16: its byte 2 is b = 256 - magnitude, or 0.  Of a negative element the code is b ^ 0x80, of
// another (b ^ 0x7F) + 1, which never carries into the next byte, so that four are put right in their word.  (One element after the other took 8 operations
// each for these 5: 8 x 4096 x 2048 bfloat16 51 us, with these and addresses of 32 bits 45.)
__device__ __forceinline__ uint32_t kept_less(float u16, uint32_t draw)
{
    int minus_T;
    asm("v_cvt_flr_i32_f32_e64 %0, -|%1|" : "=v"(minus_T) : "v"(u16));
    return draw + (uint32_t)minus_T;
}

__device__ __forceinline__ uint32_t kept_word(const float (&u16)[4], uint32_t draws01, uint32_t draws23)
{
    const uint32_t b0 = kept_less(u16[0], draws01 & 0xFFFFu), b1 = kept_less(u16[1], draws01 >> 16), b2 = kept_less(u16[2], draws23 & 0xFFFFu),
                   b3 = kept_less(u16[3], draws23 >> 16);
    const uint32_t lo = __builtin_amdgcn_perm(b1, b0, 0x0C0C0602u), hi = __builtin_amdgcn_perm(b3, b2, 0x06020C0Cu);
    // (a selector of 9 or 11: the sign of the first or second word, all over a byte)
    const uint32_t sign_lo = __builtin_amdgcn_perm(__float_as_uint(u16[1]), __float_as_uint(u16[0]), 0x0C0C0B09u);
    const uint32_t sign_hi = __builtin_amdgcn_perm(__float_as_uint(u16[3]), __float_as_uint(u16[2]), 0x0B090C0Cu);
    const uint32_t turn = (sign_lo | sign_hi) ^ 0x7F7F7F7Fu;
    return ((lo | hi) ^ turn) + (turn & 0x01010101u);
}

// The codes of W neighbouring columns, as the words that are stored, and the block's power, from the bits of its largest magnitude.  W = 8: the columns of one
// Philox block; W = 4: its half `half`.
template <int W>
__device__ __forceinline__ uint32_t kept_codes(float (&v)[W], uint32_t bits, uint32_t top, bool draws, uint32_t group, uint32_t half, uint32_t row, uint32_t domain,
                                               uint32_t call, const PhiloxKeys& keys, uint32_t (&word)[W / 4])
{
    uint32_t power = kept_power(bits);
    uint32_t over = (254u - power) << 23;                  // 2^-e (of zeros it may be anything)
    float wide = 65536.0f;
    if (__builtin_amdgcn_ballot_w64(kept_is_rare(bits, power, top)) != 0ull) {
        // (no branches within: their results would be copied on the way past them too)
        const bool spoilt = bits >= 0x7F800000u;
        power = bits ? min(max(power, 1u), top) : 0u;
        const bool small = draws && power < 16u;           // the elements by 2^16
        const float most = __uint_as_float(power << 23) * 127.0f, by = small ? 65536.0f : 1.0f;
        wide = small ? 1.0f : 65536.0f;
        over = spoilt ? 0u : (254u - power) << 23;
        power = spoilt ? kKeptSpoilt : power;
#pragma unroll
        for (int c = 0; c < W; ++c) v[c] = spoilt ? 0.0f : __builtin_amdgcn_fmed3f(v[c], -most, most) * by;      // (0 * infinity is no zero)
    }
    if (draws) {
        uint32_t w[4];
        philox4x32_10(group, domain, row, call, keys, w);
        if (W == 4 && half) { w[0] = w[2]; w[1] = w[3]; }
        const float over16 = __uint_as_float(over) * wide;
#pragma unroll
        for (int h = 0; h < W / 4; ++h) {
            float u16[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) u16[c] = v[4 * h + c] * over16;
            word[h] = kept_word(u16, w[2 * h], w[2 * h + 1]);
        }
    } else {
#pragma unroll
        for (int h = 0; h < W / 4; ++h) {
            word[h] = 0u;
#pragma unroll
            for (int c = 0; c < 4; ++c) word[h] = kept_code(v[4 * h + c] * __uint_as_float(over), (uint32_t)c, word[h]);
        }
    }
    return power;
}

// The bits of the largest magnitude of a piece's elements, as binary32's: of 16-bit elements two at a time.
template <typename T>
__device__ __forceinline__ uint32_t largest_bits(nt_u32x4 x)
{
    if constexpr (sizeof(T) == 4) {
        const nt_u32x4 m = x & 0x7FFFFFFFu;
        return max(max(m[0], m[1]), max(m[2], m[3]));
    } else {
        typedef uint16_t pair __attribute__((ext_vector_type(2)));
        pair m = __builtin_bit_cast(pair, (uint32_t)x[0] & 0x7FFF7FFFu);
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(pair, (uint32_t)x[i] & 0x7FFF7FFFu));
        const uint16_t most = m.x > m.y ? m.x : m.y;
        if constexpr (__is_same(T, _Float16)) return __float_as_uint((float)__builtin_bit_cast(_Float16, most));
        else return (uint32_t)most << 16;
    }
}

// The largest over the four lanes of a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));      // quad_perm [1,0,3,2]
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));   // quad_perm [2,3,0,1]
}

}  // namespace qgx
