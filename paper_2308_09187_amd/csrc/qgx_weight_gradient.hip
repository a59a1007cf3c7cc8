// The weight gradient of a linear layer from its kept input: dW = X^T dY, X [rows][cols] in codes and powers, dY [rows][out].
// On the matrix cores, 32 x 32 x 16 in bfloat16 with sums in binary32.  A kept element is exact in bfloat16 (its step is a power of two),
// an element of dY is the exact sum of P bfloat16 numbers, each the next eight bits of what is left: 1 of bfloat16, 2 of binary16, 3 of
// binary32; so all products are exact, and P times the products are made.
// Both operands lie with the summed index (the rows) outermost, the matrix cores take eight consecutive rows of a column from a lane: a thread
// loads eight rows of four columns, brings them into that order in its registers (codes are decoded on the way) and leaves each
// column's eight rows, 16 bytes, in LDS, from where a wave's operands are single loads of 16 bytes.
#include "qgx_kept.h"
#include "qgx_plan.h"

namespace qgx {

constexpr int kGradThreads = 256;
constexpr int kGradRows = 64;                              // rows of a step
constexpr int kGradTile = 128;                             // columns of X, and of dY, of a workgroup

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T> constexpr int kGradParts = sizeof(T) == 4 ? 3 : __is_same(T, _Float16) ? 2 : 1;

// The slot of a column among its tile's: the low bits turned so that neither eight threads that write columns four apart nor eight that read
// neighbouring ones meet in a bank.
__device__ __forceinline__ uint32_t grad_slot(uint32_t i) { return i ^ ((i >> 3) & 7u); }

// The upper halves of two words (a binary32's is its bfloat16, rounded to zero), the first in the low half.
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

template <typename T> struct FourAs { typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T)))); };
template <typename T> using FourOf = typename FourAs<T>::type;

template <typename T>
__device__ __forceinline__ FourOf<T> load_four(const T* p, int left)
{
    if (left >= 4) return *reinterpret_cast<const FourOf<T>*>(p);
    FourOf<T> v;
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = c < left ? p[c] : (T)0.0f;
    return v;
}

template <typename T>
__global__ __launch_bounds__(kGradThreads, 2) void k_weight_gradient(WeightGradArgs a)
{
    constexpr int P = kGradParts<T>, kOcts = kGradRows / 8;
    __shared__ __align__(16) uint4 s_x[2][kOcts][kGradTile];
    __shared__ __align__(16) uint4 s_dy[2][P][kOcts][kGradTile];
    __shared__ __align__(16) uint8_t s_power[2][kGradTile / 32][kGradRows];
    const uint32_t k = blockIdx.y, tiles = a.tiles_i * a.tiles_o;
    const uint32_t part = blockIdx.x / tiles, tile = blockIdx.x % tiles, tile_i = tile % a.tiles_i, tile_o = tile / a.tiles_i;
    const uint32_t row0 = part * a.part_rows, row1 = min(row0 + a.part_rows, a.rows);
    const uint32_t quad = threadIdx.x % 32u, oct = threadIdx.x / 32u;
    // loads: four columns of eight rows (those past the kept blocks again the last; their results are not stored)
    const uint32_t i0 = min(tile_i * kGradTile + quad * 4u, a.blocks * 32u - 4u), o0 = tile_o * kGradTile + quad * 4u;
    const uint8_t* codes = a.codes + ((uint64_t)k * a.rows * a.blocks) * 32u + i0;
    const T* dy = (const T*)a.dy + k * a.dy_worker + o0;
    const int left = (int)min((int64_t)a.out - (int64_t)o0, (int64_t)4);
    // a byte of the powers: thread t has block t / 64, row t % 64
    const uint32_t p_block = min(tile_i * (kGradTile / 32u) + threadIdx.x / kGradRows, a.blocks - 1u), p_row = threadIdx.x % kGradRows;
    const uint8_t* powers = a.powers + (uint64_t)k * a.rows * a.blocks + p_block;
    uint32_t x[8], power;
    FourOf<T> d[8];
    auto load = [&](uint32_t row) {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const uint32_t at = row + oct * 8u + (uint32_t)r, ok = min(at, row1 - 1u);
            x[r] = *reinterpret_cast<const uint32_t*>(codes + (uint64_t)ok * a.blocks * 32u);
            d[r] = load_four(dy + ok * a.dy_row, at < row1 ? left : 0);
        }
    };
    auto load_power = [&](uint32_t row) {
        const uint32_t at = row + p_row;
        power = powers[(uint64_t)min(at, row1 - 1u) * a.blocks];
        if (at >= row1) power = 0u;                        // (rows past the last: zeros)
    };
    float db[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const bool sums = a.db && tile_i == 0;
    auto store = [&](int to) {
        // X: decoded, column by column eight rows
        float scale[8];
        const uint2 pw = *reinterpret_cast<const uint2*>(&s_power[to][quad / 8u][oct * 8u]);
#pragma unroll
        for (int r = 0; r < 8; ++r) scale[r] = kept_scale(((r < 4 ? pw.x : pw.y) >> (8 * (r & 3))) & 0xFFu);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            uint32_t v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = __float_as_uint(kept_value((x[r] >> (8 * c)) & 0xFFu, scale[r]));
            s_x[to][oct][grad_slot(quad * 4u + c)] = make_uint4(upper_halves(v[0], v[1]), upper_halves(v[2], v[3]), upper_halves(v[4], v[5]), upper_halves(v[6], v[7]));
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = (float)d[r][c];
            if (sums)
#pragma unroll
                for (int r = 0; r < 8; ++r) db[c] += v[r];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                uint32_t u[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    u[r] = __float_as_uint(v[r]);
                    // what the upper half leaves (of an infinity nothing)
                    if (p + 1 < P) v[r] = (u[r] & 0x7F800000u) == 0x7F800000u ? 0.0f : v[r] - __uint_as_float(u[r] & 0xFFFF0000u);
                }
                s_dy[to][p][oct][grad_slot(quad * 4u + c)] = make_uint4(upper_halves(u[0], u[1]), upper_halves(u[2], u[3]), upper_halves(u[4], u[5]), upper_halves(u[6], u[7]));
            }
        }
    };
    const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, wi = wave % 2u * 64u, wo = wave / 2u * 64u;
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    const uint32_t steps = (row1 - row0 + kGradRows - 1u) / kGradRows;
    load_power(row0);
    load(row0);
    s_power[0][threadIdx.x / kGradRows][p_row] = (uint8_t)power;
    load_power(row0 + kGradRows);
    __syncthreads();
    store(0);
    s_power[1][threadIdx.x / kGradRows][p_row] = (uint8_t)power;
    __syncthreads();
    for (uint32_t s = 0; s < steps; ++s) {
        const int now = (int)(s & 1u);
        const uint32_t next = row0 + (s + 1u) * kGradRows;
        const bool more = s + 1u < steps, after = s + 2u < steps;
        if (more) load(next);
        if (after) load_power(next + kGradRows);
#pragma unroll
        for (int t = 0; t < kGradRows / 16; ++t) {
            const uint32_t o = 2u * t + lane / 32u, c = lane % 32u;
            bf16x8 u[2], v[P][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) u[i] = __builtin_bit_cast(bf16x8, s_x[now][o][grad_slot(wi + 32u * i + c)]);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int j = 0; j < 2; ++j) v[p][j] = __builtin_bit_cast(bf16x8, s_dy[now][p][o][grad_slot(wo + 32u * j + c)]);
#pragma unroll
            for (int p = P - 1; p >= 0; --p)               // (the smallest first)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u[i], v[p][j], acc[i][j], 0, 0, 0);
        }
        if (more) store(now ^ 1);                          // (s_power[now ^ 1] holds the next step's since the last barrier)
        if (after) s_power[now][threadIdx.x / kGradRows][p_row] = (uint8_t)power;   // (read for this step before the last barrier)
        __syncthreads();
    }
    float* dw = a.parts == 1u ? a.dw + k * a.dw_worker : a.scratch + ((uint64_t)k * a.parts + part) * ((uint64_t)a.cols * a.out + a.out);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t o = tile_o * kGradTile + wo + 32u * j + lane % 32u;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t row = tile_i * kGradTile + wi + 32u * i + 8u * (e / 4) + 4u * (lane / 32u) + (e % 4);
                if (row < a.cols && o < a.out) dw[(uint64_t)row * a.out + o] = acc[i][j][e];
            }
        }
    if (!sums) return;
    float* s_db = reinterpret_cast<float*>(s_x);           // (free since the last barrier) [octs][tile]
#pragma unroll
    for (int c = 0; c < 4; ++c) s_db[oct * kGradTile + quad * 4u + c] = db[c];
    __syncthreads();
    const uint32_t o = tile_o * kGradTile + threadIdx.x;
    if (threadIdx.x < kGradTile && o < a.out) {
        float x = s_db[threadIdx.x];
#pragma unroll
        for (int i = 1; i < kOcts; ++i) x += s_db[i * kGradTile + threadIdx.x];
        float* to = a.parts == 1u ? a.db + k * a.db_worker : dw + (uint64_t)a.cols * a.out;
        to[o] = x;
    }
}

// ---- large layers ---------------------------------------------------------------------------------------------------------
// A wave has 128 columns of X by 64 of dY, so that a byte of an operand meets many products: the matrix cores then need less of LDS and of the
// vector units than those have.  X is decoded once for its WN waves and passes through LDS; dY goes from memory into the operand's place in
// registers: lane c has columns 2 c and 2 c + 1, which are the columns c of two tiles, and eight rows of them, transposed in pairs.  What a
// group of 16 rows is worked on from is loaded again for the next step as soon as it is used.
template <typename T> struct PairAs { typedef T type __attribute__((ext_vector_type(2), aligned(sizeof(T)))); };
template <typename T> using PairOf = typename PairAs<T>::type;

template <typename T, int WM, int WN>
__global__ __launch_bounds__(WM * WN * kWave, 2) void k_weight_gradient_wide(WeightGradArgs a)
{
    constexpr int P = kGradParts<T>, kThreads = WM * WN * kWave, TM = 128 * WM, TN = 64 * WN, kOcts = kGradRows / 8;
    constexpr int kUnits = kOcts * (TM / 4) / kThreads;    // eight rows of four columns of X, of a thread
    constexpr int kGroups = kGradRows / 16, kAhead = sizeof(T) == 4 ? 2 : 4;     // groups of 16 rows of a step; those that are loaded ahead
    constexpr int kPowers = TM / 32 * kGradRows / kThreads;
    static_assert(kUnits >= 1 && kPowers >= 1, "");
    __shared__ __align__(16) uint4 s_x[2][kOcts][TM];
    __shared__ __align__(16) uint8_t s_power[2][TM / 32][kGradRows];
    __shared__ float s_db[2][TN];
    const uint32_t tiles = a.tiles_i * a.tiles_o, k = blockIdx.y;
    const uint32_t part = blockIdx.x / tiles, tile = blockIdx.x % tiles, tile_i = tile % a.tiles_i, tile_o = tile / a.tiles_i;
    const uint32_t row0 = part * a.part_rows, row1 = min(row0 + a.part_rows, a.rows), steps = (row1 - row0 + kGradRows - 1u) / kGradRows;
    const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, wm = wave % WM, wn = wave / WM, c = lane % 32u, half = lane / 32u;
    const uint64_t code_row = (uint64_t)a.blocks * 32u;
    const uint8_t* codes0 = a.codes + (uint64_t)k * a.rows * code_row;
    const uint8_t* powers0 = a.powers + (uint64_t)k * a.rows * a.blocks;
    const uint32_t o = tile_o * TN + wn * 64u + 2u * c;
    const bool edge = tile_o * TN + TN > a.out;
    const T* dy = (const T*)a.dy + k * a.dy_worker + o;

    uint32_t x[kUnits][8], next_x[kUnits][8], power[kPowers];
    PairOf<T> d[kAhead][8];
    auto load_codes = [&](uint32_t row) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const uint32_t unit = threadIdx.x + u * kThreads, quad = unit % (TM / 4), oct = unit / (TM / 4);
            const uint32_t i0 = min(tile_i * TM + quad * 4u, a.blocks * 32u - 4u);
            const uint8_t* p = codes0 + i0;
#pragma unroll
            for (int r = 0; r < 8; ++r) next_x[u][r] = *reinterpret_cast<const uint32_t*>(p + min(row + oct * 8u + (uint32_t)r, row1 - 1u) * code_row);
        }
    };
    auto load_powers = [&](uint32_t row) {
#pragma unroll
        for (int u = 0; u < kPowers; ++u) {
            const uint32_t unit = threadIdx.x + u * kThreads, block = unit / kGradRows, at = row + unit % kGradRows;
            power[u] = powers0[(uint64_t)min(at, row1 - 1u) * a.blocks + min(tile_i * (TM / 32) + block, a.blocks - 1u)];
            if (at >= row1) power[u] = 0u;                 // (rows past the last: zeros)
        }
    };
    auto store_powers = [&](int to) {
#pragma unroll
        for (int u = 0; u < kPowers; ++u) {
            const uint32_t unit = threadIdx.x + u * kThreads;
            s_power[to][unit / kGradRows][unit % kGradRows] = (uint8_t)power[u];
        }
    };
    // rows row .. row + 15 of dY, this half's eight
    auto load_dy = [&](uint32_t row, PairOf<T> (&v)[8]) {
        const uint32_t first = row + half * 8u;
        if (!edge && row + 16u <= row1) {
            const T* p = dy + (uint64_t)first * a.dy_row;
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = *reinterpret_cast<const PairOf<T>*>(p + r * a.dy_row);
        } else {
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const T* p = dy + (uint64_t)(first + r) * a.dy_row;
                v[r].x = first + r < row1 && o < a.out ? p[0] : (T)0.0f;
                v[r].y = first + r < row1 && o + 1u < a.out ? p[1] : (T)0.0f;
            }
        }
    };
    // a column of the thread's units of X, decoded, into LDS
    auto store_column = [&](int to, int col) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const uint32_t unit = threadIdx.x + u * kThreads, quad = unit % (TM / 4), oct = unit / (TM / 4);
            const uint2 pw = *reinterpret_cast<const uint2*>(&s_power[to][quad / 8u][oct * 8u]);
            uint32_t v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r)
                v[r] = __float_as_uint(kept_value((x[u][r] >> (8 * col)) & 0xFFu, kept_scale(((r < 4 ? pw.x : pw.y) >> (8 * (r & 3))) & 0xFFu)));
            s_x[to][oct][grad_slot(quad * 4u + col)] = make_uint4(upper_halves(v[0], v[1]), upper_halves(v[2], v[3]), upper_halves(v[4], v[5]), upper_halves(v[6], v[7]));
        }
    };
    auto take_codes = [&]() {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int r = 0; r < 8; ++r) x[u][r] = next_x[u][r];
    };

    f32x16 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    const bool sums = a.db && tile_i == 0 && wm == 0;
    float db[2] = {0.0f, 0.0f};

    load_powers(row0);
    store_powers(0);
    load_powers(row0 + kGradRows);
    store_powers(1);
    load_codes(row0);
#pragma unroll
    for (int g = 0; g < kAhead; ++g) load_dy(row0 + 16u * g, d[g]);
    take_codes();
    load_codes(row0 + kGradRows);
    __syncthreads();
#pragma unroll
    for (int col = 0; col < 4; ++col) store_column(0, col);
    __syncthreads();
    for (uint32_t s = 0; s < steps; ++s) {
        const int now = (int)(s & 1u);
        const uint32_t row = row0 + s * kGradRows;
        const bool more = s + 1u < steps;
        take_codes();
        load_codes(row + 2u * kGradRows);                  // (past the end: the last row again)
        load_powers(row + 2u * kGradRows);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            bf16x8 v[P][2], u[4];
            PairOf<T> (&raw)[8] = d[g % kAhead];
            float left[2][8];
            if constexpr (P == 1) {
                uint32_t w[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) w[r] = __builtin_bit_cast(uint32_t, raw[r]);
                v[0][0] = __builtin_bit_cast(bf16x8, make_uint4(__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u),
                                                                __builtin_amdgcn_perm(w[5], w[4], 0x05040100u), __builtin_amdgcn_perm(w[7], w[6], 0x05040100u)));
                v[0][1] = __builtin_bit_cast(bf16x8, make_uint4(upper_halves(w[0], w[1]), upper_halves(w[2], w[3]), upper_halves(w[4], w[5]), upper_halves(w[6], w[7])));
                if (sums)
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        db[0] += __uint_as_float(w[r] << 16);
                        db[1] += __uint_as_float(w[r] & 0xFFFF0000u);
                    }
            } else {
                float most = 0.0f;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    left[0][r] = (float)raw[r].x;
                    left[1][r] = (float)raw[r].y;
                    most = fmaxf(fmaxf(most, fabsf(left[0][r])), fabsf(left[1][r]));
                    if (sums) { db[0] += left[0][r]; db[1] += left[1][r]; }
                }
                const bool finite = most <= 3.402823466e38f;       // (a NaN may hide here, and is a NaN in every part)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t w[8];
#pragma unroll
                        for (int r = 0; r < 8; ++r) w[r] = __float_as_uint(left[j][r]);
                        v[p][j] = __builtin_bit_cast(bf16x8, make_uint4(upper_halves(w[0], w[1]), upper_halves(w[2], w[3]), upper_halves(w[4], w[5]), upper_halves(w[6], w[7])));
                        if (p + 1 < P)
#pragma unroll
                            for (int r = 0; r < 8; ++r) {
                                left[j][r] = left[j][r] - __uint_as_float(w[r] & 0xFFFF0000u);
                                if (!finite && (w[r] & 0x7FFFFFFFu) == 0x7F800000u) left[j][r] = 0.0f;    // (of an infinity nothing is left)
                            }
                    }
            }
            {
                // the group's next rows
                const uint32_t next = row + 16u * (g + kAhead);
                if (next < row1) load_dy(next, raw);
                else
#pragma unroll
                    for (int r = 0; r < 8; ++r) raw[r] = PairOf<T>{(T)0.0f, (T)0.0f};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = __builtin_bit_cast(bf16x8, s_x[now][2u * g + half][grad_slot(wm * 128u + 32u * i + c)]);
            if (more) store_column(now ^ 1, g);            // (of the next step, whose powers are there since the last barrier)
#pragma unroll
            for (int p = P - 1; p >= 0; --p)               // (the smallest first)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u[i], v[p][j], acc[i][j], 0, 0, 0);
        }
        store_powers(now);                                 // (of step s + 2; this step's were read before the last barrier)
        __syncthreads();
    }
    float* dw = a.parts == 1u ? a.dw + k * a.dw_worker : a.scratch + ((uint64_t)k * a.parts + part) * ((uint64_t)a.cols * a.out + a.out);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t row = tile_i * TM + wm * 128u + 32u * i + 8u * (e / 4) + 4u * half + (e % 4);
            if (row >= a.cols) continue;
            float* to = dw + (uint64_t)row * a.out + o;
            if (o + 1u < a.out) *reinterpret_cast<PairOf<float>*>(to) = PairOf<float>{acc[i][0][e], acc[i][1][e]};
            else if (o < a.out) to[0] = acc[i][0][e];
        }
    if (!a.db || tile_i != 0) return;
    if (wm == 0) {
        s_db[half][wn * 64u + 2u * c] = db[0];
        s_db[half][wn * 64u + 2u * c + 1u] = db[1];
    }
    __syncthreads();
    float* to = a.parts == 1u ? a.db + k * a.db_worker : dw + (uint64_t)a.cols * a.out;
    for (uint32_t i = threadIdx.x; i < TN; i += kThreads)
        if (tile_o * TN + i < a.out) to[tile_o * TN + i] = s_db[0][i] + s_db[1][i];
}

// The parts' sums, joined in order.
__global__ __launch_bounds__(256) void k_weight_gradient_join(WeightGradArgs a)
{
    const uint64_t n = (uint64_t)a.cols * a.out, all = n + a.out, k = blockIdx.y;
    const float* from = a.scratch + k * a.parts * all;
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < (a.db ? all : n); i += (uint64_t)gridDim.x * 256u) {
        float x = from[i];
#pragma unroll 4
        for (uint32_t p = 1; p < a.parts; ++p) x += from[p * all + i];
        if (i < n) a.dw[k * a.dw_worker + i] = x;
        else a.db[k * a.db_worker + i - n] = x;
    }
}

__global__ __launch_bounds__(256) void k_weight_gradient_zero(WeightGradArgs a)
{
    const uint64_t n = (uint64_t)a.cols * a.out, k = blockIdx.y;
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < n + (a.db ? a.out : 0u); i += (uint64_t)gridDim.x * 256u) {
        if (i < n) a.dw[k * a.dw_worker + i] = 0.0f;
        else a.db[k * a.db_worker + i - n] = 0.0f;
    }
}

// Rows are split where there are fewer tiles than compute units, in parts of 256 rows at least.
WeightGradPlan weight_grad_plan(int dtype, uint32_t workers, uint32_t rows, uint32_t cols, uint32_t out, uint32_t n_cu)
{
    (void)dtype;
    WeightGradPlan p{};
    p.wide = cols > 128u && out > 128u;
    p.tiles_i = p.wide ? (cols + 255u) / 256u : (cols + kGradTile - 1u) / kGradTile;
    p.tiles_o = p.wide ? (out + 255u) / 256u : (out + kGradTile - 1u) / kGradTile;
    p.parts = 1;
    p.part_rows = rows;
    if (workers == 0 || rows == 0) return p;
    const uint64_t tiles = (uint64_t)workers * p.tiles_i * p.tiles_o;
    const uint32_t most = (rows + 255u) / 256u;
    const uint32_t want = (uint32_t)min((uint64_t)most, max((uint64_t)1u, (p.wide ? 1u : 2u) * n_cu / tiles));
    p.part_rows = ((rows + want - 1u) / want + kGradRows - 1u) / kGradRows * kGradRows;
    p.parts = (rows + p.part_rows - 1u) / p.part_rows;
    if (p.parts > 1u) p.scratch = (uint64_t)workers * p.parts * ((uint64_t)cols * out + out) * sizeof(float);
    return p;
}

hipError_t launch_weight_grad(int dtype, const WeightGradArgs& args, uint32_t workers, const WeightGradPlan& plan, hipStream_t st)
{
    WeightGradArgs a = args;
    a.tiles_i = plan.tiles_i; a.tiles_o = plan.tiles_o; a.parts = plan.parts; a.part_rows = plan.part_rows;
    if (workers == 0) return hipSuccess;
    const uint64_t values = (uint64_t)a.cols * a.out + a.out;
    const dim3 each((uint32_t)((values + 255u) / 256u < 4096u ? (values + 255u) / 256u : 4096u), workers);
    if (a.rows == 0) {
        hipLaunchKernelGGL(k_weight_gradient_zero, each, dim3(256), 0, st, a);
        return hipGetLastError();
    }
    const dim3 grid(a.tiles_i * a.tiles_o * a.parts, workers);
    if (plan.wide) {
        const dim3 threads(512);
        if (dtype == QGX_F32) hipLaunchKernelGGL((k_weight_gradient_wide<float, 2, 4>), grid, threads, 0, st, a);
        else if (dtype == QGX_F16) hipLaunchKernelGGL((k_weight_gradient_wide<_Float16, 2, 4>), grid, threads, 0, st, a);
        else hipLaunchKernelGGL((k_weight_gradient_wide<__bf16, 2, 4>), grid, threads, 0, st, a);
    } else if (dtype == QGX_F32) hipLaunchKernelGGL(k_weight_gradient<float>, grid, dim3(kGradThreads), 0, st, a);
    else if (dtype == QGX_F16) hipLaunchKernelGGL(k_weight_gradient<_Float16>, grid, dim3(kGradThreads), 0, st, a);
    else hipLaunchKernelGGL(k_weight_gradient<__bf16>, grid, dim3(kGradThreads), 0, st, a);
    if (a.parts > 1u) hipLaunchKernelGGL(k_weight_gradient_join, each, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qgx
