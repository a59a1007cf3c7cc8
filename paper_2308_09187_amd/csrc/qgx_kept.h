// Activations kept in 8 bits: a block of 32 elements of a row has one power of two 2^e, an element is a whole number of at most 127 of
// it.  The numbers are powers of two apart so that a kept element is exact in bfloat16 (8 bits of significand): products with it on the matrix cores are
// exact, and so is a decoding by one multiplication.  Against a scale of its own (the block's maximum / 127) the step is up to twice as wide,
// 1.4 times on average.
#pragma once

#include "qgx_types.h"

namespace qgx {

// A block's stored power, from the bits of its largest magnitude: the smallest 2^e with the magnitude at most 127 * 2^e (127 = 1.984375 * 2^6),
// biased by 127; `top`: the type's largest.  0 for zeros, 255 where the magnitude is an infinity or a NaN.
constexpr uint32_t kKeptSpoilt = 255u;
__device__ __forceinline__ uint32_t kept_power(uint32_t bits, uint32_t top)
{
    const int p = (int)(bits >> 23) - 6 + (int)((bits & 0x7FFFFFu) > 0x7E0000u);
    if (bits == 0u) return 0u;
    return bits >= 0x7F800000u ? kKeptSpoilt : (uint32_t)min(max(p, 1), (int)top);
}

// 2^-e of a stored power (zeros and spoilt blocks: 0, so that their codes are those of zeros).
__device__ __forceinline__ float kept_over(uint32_t power)
{
    return power == 0u || power == kKeptSpoilt ? 0.0f : __uint_as_float((254u - power) << 23);
}

// 2^e; 0 for zeros, infinity (and so 0 * infinity = NaN) for a spoilt block.
__device__ __forceinline__ float kept_scale(uint32_t power) { return __uint_as_float(power << 23); }

// Rounded to the nearest whole number.
__device__ __forceinline__ uint32_t kept_code(float u)
{
    return (uint32_t)(int)(fminf(fmaxf(rintf(u), -127.0f), 127.0f) + 128.0f);
}

// Rounded away from zero where the draw, 16 bits, is below 2^16 times the remainder (|u| less its whole part: exact).
__device__ __forceinline__ uint32_t kept_code(float u, uint32_t draw)
{
    const float m = fabsf(u), down = floorf(m);
    const float up = (float)draw < (m - down) * 65536.0f ? down + 1.0f : down;
    const float code = fminf(up, 127.0f);
    return (uint32_t)(int)(128.0f + (u < 0.0f ? -code : code));
}

// An element out of its byte: both steps exact.
__device__ __forceinline__ float kept_value(uint32_t code, float scale) { return ((float)code - 128.0f) * scale; }

__device__ __forceinline__ uint32_t kept_call(const KeptDraws& d, const Scalars* sc)
{
    return d.call_mode ? 2u * (scalar_load(&sc->t) - 1u) + (d.call_mode - 1u) : d.call_id;
}

// The codes of eight columns' elements, with the bits of the block's largest magnitude known: the two words that are stored.
// group: the column / 8.
__device__ __forceinline__ void kept_codes(const float (&v)[8], float over, bool draws, uint32_t group, uint32_t row, uint32_t call,
                                           const PhiloxKeys& keys, uint32_t (&word)[2])
{
    uint32_t code[8];
    if (draws) {
        uint32_t w[4];
        philox4x32_10(group, 2u, row, call, keys, w);
#pragma unroll
        for (int c = 0; c < 8; ++c) code[c] = kept_code(v[c] * over, (c & 1) ? w[c / 2] >> 16 : w[c / 2] & 0xFFFFu);
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) code[c] = kept_code(v[c] * over);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) word[h] = code[4 * h] | code[4 * h + 1] << 8 | code[4 * h + 2] << 16 | code[4 * h + 3] << 24;
}

// The largest over the four lanes of a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));      // quad_perm [1,0,3,2]
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));   // quad_perm [2,3,0,1]
}

}  // namespace qgx
