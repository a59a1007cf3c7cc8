// The weight gradient of a linear layer from its kept input: dW = X^T dY, X [rows][cols] in codes and powers, dY [rows][out].
// On the matrix cores, 32 x 32 x 16 in bfloat16 with sums in binary32.  A kept element is exact in bfloat16 (its step is a power of two),
// an element of dY is the exact sum of P bfloat16 numbers, each the next eight bits of what is left: 1 of bfloat16, 2 of binary16, 3 of
// binary32; so all products are exact, and P times the products are made.
// Both operands lie with the summed index (the rows) outermost, the matrix cores take eight consecutive rows of a column from a lane: a thread
// loads eight rows of four columns, brings them into that order in its registers (codes are decoded on the way) and leaves each
// column's eight rows, 16 bytes, in LDS, from where a wave's operands are single loads of 16 bytes.
// Bound by how steadily the matrix cores are fed.  In calls one after the other 8 x 4096 x 1024 x 4096 bfloat16: 288 us, 955 TFLOP/s (223 for the library's product
// of operands laid out for it; 240 without decoding and loads); 4 x 65536 x 256 x 320 binary32, three times the products: 171 us with the join of its parts.
// (Under a kernel trace, median and least: 327 and 293; 190 and 158, the join 12.)
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
__global__ __launch_bounds__(kGradThreads) void k_weight_gradient(WeightGradArgs a)
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
                    // what the upper half leaves: of an infinity nothing, of a NaN a NaN (its upper half may be an infinity's)
                    if (p + 1 < P) v[r] = (u[r] & 0x7FFFFFFFu) == 0x7F800000u ? 0.0f : v[r] - __uint_as_float(u[r] & 0xFFFF0000u);
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
// group of 16 rows is worked on from is loaded again for a later one as soon as it is used.  No branch in a step: columns past the last are the
// last ones again (and equal numbers are stored twice), rows past the last full step are a step of their own at the end.
template <typename T> struct PairAs { typedef T type __attribute__((ext_vector_type(2), aligned(sizeof(T)))); };
template <typename T> using PairOf = typename PairAs<T>::type;

// A signed byte of a word as a number, in one instruction.
template <int BYTE>
__device__ __forceinline__ float byte_value(uint32_t x)
{
    float v;
    if constexpr (BYTE == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(v) : "v"(x));
    else if constexpr (BYTE == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(v) : "v"(x));
    else if constexpr (BYTE == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(v) : "v"(x));
    else asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(v) : "v"(x));
    return v;
}

// sum += the eight, here and now (left to later, they would all be kept until then).
__device__ __forceinline__ void add_eight(const float (&f)[8], float& sum)
{
    sum += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
    asm volatile("" : "+v"(sum));
}

template <int C> struct Column { static constexpr int value = C; };

template <typename T, int WM, int WN>
struct WideGradient {
    static constexpr int P = kGradParts<T>, kThreads = WM * WN * kWave, TM = 128 * WM, TN = 64 * WN, kOcts = kGradRows / 8;
    static constexpr int kUnits = kOcts * (TM / 4) / kThreads;                   // eight rows of four columns of X, of a thread
    static constexpr int kGroups = kGradRows / 16;                               // groups of 16 rows of a step
    static constexpr int kAhead = P == 1 ? 2 : 1;                   // groups that are loaded ahead (P products from each)
    static constexpr int kPowers = TM / 32 * kGradRows / kThreads;
    static_assert(kUnits >= 1 && kPowers >= 1 && kGroups % kAhead == 0, "");

    struct Shared {
        uint4 x[2][kOcts][TM];
        float scale[2][TM / 32][kGradRows + 4];            // (blocks a bank apart)
        float db[2][TN];
    };
};

template <typename T, int WM, int WN, bool SUMS>
__device__ __forceinline__ void weight_gradient_tile(const WeightGradArgs& a, typename WideGradient<T, WM, WN>::Shared& sh, uint32_t k, uint32_t part, uint32_t tile_i, uint32_t tile_o)
{
    typedef WideGradient<T, WM, WN> G;
    constexpr int P = G::P, kThreads = G::kThreads, TM = G::TM, TN = G::TN, kUnits = G::kUnits, kAhead = G::kAhead;
    const uint32_t row0 = part * a.part_rows, row1 = min(row0 + a.part_rows, a.rows), full = (row1 - row0) / kGradRows;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = threadIdx.x % kWave;
    const uint32_t wm = wave % WM, wn = wave / WM, c = lane % 32u, half = lane / 32u;
    const uint64_t code_row = (uint64_t)a.blocks * 32u;
    const uint8_t* codes0 = a.codes + (uint64_t)k * a.rows * code_row;
    const uint8_t* powers0 = a.powers + (uint64_t)k * a.rows * a.blocks;
    const uint32_t o = tile_o * TN + wn * 64u + 2u * c, oc = min(o, a.out - 2u);
    const T* dy0 = (const T*)a.dy + k * a.dy_worker;
    const uint64_t dy_row = a.dy_row;

    // a thread's offsets from a step's first row (32 bits: the caller has seen to that)
    uint32_t x_at[kUnits], p_at[G::kPowers];
    uint32_t to_at[kUnits], scale_at[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const uint32_t unit = threadIdx.x + u * kThreads, quad = unit % (TM / 4), oct = unit / (TM / 4);
        x_at[u] = oct * 8u * (uint32_t)code_row + min(tile_i * TM + quad * 4u, a.blocks * 32u - 4u);
        to_at[u] = oct * TM;
        scale_at[u] = quad / 8u * (kGradRows + 4u) + oct * 8u;
    }
#pragma unroll
    for (int u = 0; u < G::kPowers; ++u) {
        const uint32_t unit = threadIdx.x + u * kThreads;
        p_at[u] = unit / (TM / 32) * a.blocks + min(tile_i * (TM / 32) + unit % (TM / 32), a.blocks - 1u);
    }
    // codes as loaded, and as signed bytes; in the same place where registers are few (of split operands, whose steps are long, or of two
    // units)
    constexpr bool kApart = P == 1 && kUnits == 1;
    uint32_t x[kUnits][8], loaded[kApart ? kUnits : 1][8];
    uint32_t (&next_x)[kUnits][8] = [&]() -> uint32_t (&)[kUnits][8] { if constexpr (kApart) return loaded; else return x; }();
    float scale[G::kPowers];
    PairOf<T> d[kAhead][8];
    // of the step at `row`, all of whose rows are there: rows' addresses are the wave's, a thread's own part is 32 bits beside them
    struct Rows { const uint8_t* p[8]; };
    auto code_rows = [&](uint32_t row) {
        Rows b;
#pragma unroll
        for (int r = 0; r < 8; ++r) b.p[r] = codes0 + (uint64_t)(row + (uint32_t)r) * code_row;
        return b;
    };
    auto dy_rows = [&](uint32_t row) {
        Rows b;
#pragma unroll
        for (int r = 0; r < 8; ++r) b.p[r] = reinterpret_cast<const uint8_t*>(dy0 + (uint64_t)(row + (uint32_t)r) * dy_row);
        return b;
    };
    auto advance = [&](Rows& b, uint64_t bytes) {
#pragma unroll
        for (int r = 0; r < 8; ++r) b.p[r] += bytes;
    };
    auto load_codes = [&](const Rows& b) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            uint32_t at = x_at[u];
            asm volatile("" : "+v"(at));                   // (else the lane's part is added to the rows' in 64 bits beforehand)
#pragma unroll
            for (int r = 0; r < 8; ++r) next_x[u][r] = *reinterpret_cast<const uint32_t*>(b.p[r] + at);
        }
    };
    auto load_powers = [&](uint32_t row) {
        const uint8_t* p = powers0 + (uint64_t)row * a.blocks;
#pragma unroll
        for (int u = 0; u < G::kPowers; ++u) scale[u] = kept_scale(p[p_at[u]]);
    };
    // its rows 16 g .. 16 g + 15 of dY
    const uint32_t dy_at = (uint32_t)(half * 8u * dy_row * sizeof(T)) + oc * (uint32_t)sizeof(T);
    auto load_dy = [&](const Rows& b, int g, PairOf<T> (&v)[8]) {
        uint32_t at = dy_at + (uint32_t)(16u * g * dy_row * sizeof(T));
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = *reinterpret_cast<const PairOf<T>*>(b.p[r] + at);
    };
    auto store_scales = [&](int to) {
#pragma unroll
        for (int u = 0; u < G::kPowers; ++u) {
            const uint32_t unit = threadIdx.x + u * kThreads;
            sh.scale[to][unit % (TM / 32)][unit / (TM / 32)] = scale[u];
        }
    };
    // a column of the thread's units of X, decoded, into LDS
    auto store_column = [&](int to, auto column) {
        constexpr int col = decltype(column)::value;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const float* sc = &sh.scale[to][0][0] + scale_at[u];
            const float4 lo = *reinterpret_cast<const float4*>(sc), hi = *reinterpret_cast<const float4*>(sc + 4);
            const float f[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            uint32_t v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = __float_as_uint(byte_value<col>(x[u][r]) * f[r]);
            const uint32_t quad = (threadIdx.x + u * kThreads) % (TM / 4);
            (&sh.x[to][0][0])[to_at[u] + grad_slot(quad * 4u + col)] = make_uint4(upper_halves(v[0], v[1]), upper_halves(v[2], v[3]), upper_halves(v[4], v[5]), upper_halves(v[6], v[7]));
        }
    };
    auto take_codes = [&]() {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int r = 0; r < 8; ++r) x[u][r] = next_x[u][r] ^ 0x80808080u;          // (code - 128 as signed bytes)
    };

    f32x16 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    float db[2] = {0.0f, 0.0f};

    // the operand of 16 rows of dY for the thread's j-th column, in P parts
    auto operand = [&](const PairOf<T> (&raw)[8], int j, bf16x8 (&v)[P]) {
        if constexpr (P == 1) {
            uint32_t w[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) w[r] = __builtin_bit_cast(uint32_t, raw[r]);
            const uint32_t pick = j ? 0x07060302u : 0x05040100u;
            v[0] = __builtin_bit_cast(bf16x8, make_uint4(__builtin_amdgcn_perm(w[1], w[0], pick), __builtin_amdgcn_perm(w[3], w[2], pick),
                                                         __builtin_amdgcn_perm(w[5], w[4], pick), __builtin_amdgcn_perm(w[7], w[6], pick)));
            if constexpr (SUMS) {
                float f[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) f[r] = __uint_as_float(j ? w[r] & 0xFFFF0000u : w[r] << 16);
                add_eight(f, db[j]);
            }
        } else {
            float left[8], most = 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                left[r] = (float)(j ? raw[r].y : raw[r].x);
                most = __builtin_elementwise_maximum(most, fabsf(left[r]));
            }
            if constexpr (SUMS) add_eight(left, db[j]);
            // of an infinity the parts after the first are zeros; of a NaN they are NaNs, and so they may be of an infinity beside it (`most` is a NaN then): the
            // column is one
            const bool infinite = most > 3.402823466e38f;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                uint32_t w[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) w[r] = __float_as_uint(left[r]);
                v[p] = __builtin_bit_cast(bf16x8, make_uint4(upper_halves(w[0], w[1]), upper_halves(w[2], w[3]), upper_halves(w[4], w[5]), upper_halves(w[6], w[7])));
                if (p + 1 < P)
#pragma unroll
                    for (int r = 0; r < 8; ++r) left[r] = left[r] - __uint_as_float(w[r] & 0xFFFF0000u);
            }
            if (__builtin_expect(infinite, 0)) {
#pragma unroll
                for (int p = 1; p < P; ++p)
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        if (fabsf((float)v[0][r]) > 3.402823466e38f) v[p][r] = (__bf16)0.0f;
            }
        }
    };
    auto columns = [&](int now, uint32_t g, bf16x8 (&u)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __builtin_bit_cast(bf16x8, sh.x[now][2u * g + half][grad_slot(wm * 128u + 32u * i + c)]);
    };
    auto multiply = [&](const bf16x8 (&u)[4], int j, const bf16x8 (&v)[P]) {
#pragma unroll
        for (int p = P - 1; p >= 0; --p)                   // (the smallest first)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u[i], v[p], acc[i][j], 0, 0, 0);
    };

    if (full) {
        const uint32_t last = row0 + (full - 1u) * kGradRows;          // (what is loaded ahead of it is its rows again)
        const uint32_t second = min(row0 + kGradRows, last);
        load_powers(row0);
        store_scales(0);
        load_powers(second);
        store_scales(1);
        Rows codes = code_rows(row0), rows = dy_rows(row0);
        load_codes(codes);
        take_codes();
        advance(codes, (second - row0) * code_row);
        if (kApart) load_codes(codes);                     // (before dY's, as in the steps: what is waited for goes by the loads' order)
#pragma unroll
        for (int g = 0; g < kAhead; ++g) load_dy(rows, g, d[g]);
        __syncthreads();
        store_column(0, Column<0>{});
        store_column(0, Column<1>{});
        store_column(0, Column<2>{});
        store_column(0, Column<3>{});
        __syncthreads();
        constexpr int kSets = P == 1 ? 2 : 1;              // of X's operands: the next group's beside this one's, where registers are left
        bf16x8 u[kSets][4];
        if (!kApart) load_codes(codes);
        columns(0, 0, u[0]);
        for (uint32_t s = 0; s < full; ++s) {
            const int now = (int)(s & 1u);
            const uint32_t row = row0 + s * kGradRows, next = min(row + kGradRows, last), after = min(row + 2u * kGradRows, last);
            take_codes();
            if (kApart) {
                advance(codes, (after - next) * code_row);
                load_codes(codes);
            }
            load_powers(after);
            Rows ahead = rows;
            advance(ahead, (next - row) * dy_row * sizeof(T));
            // The next step's X is in LDS before the last group, which has its operands by then and covers the barrier.
#pragma unroll
            for (int g = 0; g < G::kGroups; ++g) {
                bf16x8 v[2][P];
                if (kSets == 1 && g) columns(now, g, u[0]);
                if (kSets == 2 && g + 1 < G::kGroups) columns(now, g + 1, u[(g + 1) % kSets]);
                operand(d[g % kAhead], 0, v[0]);
                if (P > 1 && g + 1 < G::kGroups) {
                    multiply(u[g % kSets], 0, v[0]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                operand(d[g % kAhead], 1, v[1]);
                load_dy(g + kAhead < G::kGroups ? rows : ahead, (g + kAhead) % G::kGroups, d[g % kAhead]);
                if (g == 0) {
                    store_column(now ^ 1, Column<0>{});    // (whose scales are there since the last barrier)
                    store_column(now ^ 1, Column<1>{});
                } else if (g == 1) {
                    store_column(now ^ 1, Column<2>{});
                } else if (g == 2) {
                    store_column(now ^ 1, Column<3>{});
                    store_scales(now);                     // (of step s + 2; this step's were read before the last barrier)
                    if (!kApart) {
                        advance(codes, (after - next) * code_row);
                        load_codes(codes);
                    }
                } else {
                    __syncthreads();
                    if (kSets == 2) columns(now ^ 1, 0, u[0]);
                    if (P > 1) multiply(u[g % kSets], 0, v[0]);
                }
                if (P == 1) multiply(u[g % kSets], 0, v[0]);
                multiply(u[g % kSets], 1, v[1]);
                if (kSets == 1 && g + 1 == G::kGroups) columns(now ^ 1, 0, u[0]);
                __builtin_amdgcn_sched_barrier(0);
            }
            rows = ahead;
        }
        __syncthreads();
    }
    const uint32_t rest = row0 + full * kGradRows;
    if (rest < row1) {                                     // rows past the last full step: zeros beyond the last
#pragma unroll
        for (int u = 0; u < G::kPowers; ++u) {
            const uint32_t at = rest + (threadIdx.x + u * kThreads) / (TM / 32), ok = min(at, row1 - 1u) - rest;
            scale[u] = kept_scale((powers0 + (uint64_t)rest * a.blocks)[ok * a.blocks + p_at[u] - (at - rest) * a.blocks]);
            if (at >= row1) scale[u] = 0.0f;
        }
        store_scales(0);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const uint32_t unit = threadIdx.x + u * kThreads, quad = unit % (TM / 4), oct = unit / (TM / 4);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                next_x[u][r] = *reinterpret_cast<const uint32_t*>(codes0 + min(rest + oct * 8u + (uint32_t)r, row1 - 1u) * code_row + min(tile_i * TM + quad * 4u, a.blocks * 32u - 4u));
        }
        take_codes();
        __syncthreads();
        store_column(0, Column<0>{});
        store_column(0, Column<1>{});
        store_column(0, Column<2>{});
        store_column(0, Column<3>{});
        __syncthreads();
#pragma unroll 1
        for (uint32_t g = 0; g < (uint32_t)G::kGroups && rest + 16u * g < row1; ++g) {
            bf16x8 v[P];
            PairOf<T> raw[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const uint32_t at = rest + 16u * g + half * 8u + (uint32_t)r;
                raw[r] = *reinterpret_cast<const PairOf<T>*>(dy0 + min(at, row1 - 1u) * dy_row + oc);
                if (at >= row1) raw[r] = PairOf<T>{(T)0.0f, (T)0.0f};
            }
            bf16x8 u[4];
            columns(0, g, u);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                operand(raw, j, v);
                multiply(u, j, v);
            }
        }
    }
    float* dw = a.parts == 1u ? a.dw + k * a.dw_worker : a.scratch + ((uint64_t)k * a.parts + part) * ((uint64_t)a.cols * a.out + a.out);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t row = tile_i * TM + wm * 128u + 32u * i + 8u * (e / 4) + 4u * half + (e % 4);
            if (row < a.cols && o < a.out) *reinterpret_cast<PairOf<float>*>(dw + (uint64_t)row * a.out + oc) = PairOf<float>{acc[i][0][e], acc[i][1][e]};
        }
    if constexpr (!SUMS) return;
    if (wm == 0) {
        sh.db[half][wn * 64u + 2u * c] = db[0];
        sh.db[half][wn * 64u + 2u * c + 1u] = db[1];
    }
    __syncthreads();
    float* to = a.parts == 1u ? a.db + k * a.db_worker : dw + (uint64_t)a.cols * a.out;
    for (uint32_t i = threadIdx.x; i < TN; i += kThreads) {
        const uint32_t at = min(tile_o * TN + (i & ~1u), a.out - 2u) + (i & 1u);
        if (tile_o * TN + (i & ~1u) < a.out) to[at] = sh.db[0][i] + sh.db[1][i];
    }
}

template <typename T, int WM, int WN>
__global__ __launch_bounds__(WM * WN * kWave, 2) void k_weight_gradient_wide(WeightGradArgs a)
{
    __shared__ __align__(16) typename WideGradient<T, WM, WN>::Shared sh;
    // the tiles of a part of a worker's rows one after the other on one XCD: they share its operands
    const uint32_t unit = unit_of_block(blockIdx.x, gridDim.x), tiles = a.tiles_i * a.tiles_o, run = unit / tiles;
    const uint32_t k = run / a.parts, part = run % a.parts, tile_i = unit % a.tiles_i, tile_o = unit % tiles / a.tiles_i;
    if (a.db && tile_i == 0u) weight_gradient_tile<T, WM, WN, true>(a, sh, k, part, tile_i, tile_o);
    else weight_gradient_tile<T, WM, WN, false>(a, sh, k, part, tile_i, tile_o);
}

// The parts' sums joined: four neighbouring ones to a thread, the parts dealt to RUNS threads of a workgroup, whose sums are then added in order.
template <int RUNS>
__global__ __launch_bounds__(256) void k_weight_gradient_join(WeightGradArgs a)
{
    constexpr uint32_t kFours = 256 / RUNS;
    __shared__ float4 s_run[RUNS][kFours];
    const uint64_t n = (uint64_t)a.cols * a.out, all = n + a.out, k = blockIdx.y;
    const float* from = a.scratch + k * a.parts * all;
    const uint32_t four = threadIdx.x % kFours, run = threadIdx.x / kFours;
    // (first the fours of dW, then those of db)
    const uint64_t fours = (n + 3u) / 4u, end = fours + (a.db ? (a.out + 3u) / 4u : 0u);
    for (uint64_t first = (uint64_t)blockIdx.x * kFours; first < end; first += (uint64_t)gridDim.x * kFours) {
        const uint64_t i = first + four;
        const bool bias = i >= fours;
        const uint64_t at = bias ? 4u * (i - fours) : 4u * i;
        const int left = i < end ? (int)min((bias ? a.out : n) - at, (uint64_t)4u) : 0;
        const float* p = from + (bias ? n : 0u) + at;
        float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
        for (uint32_t j = run; j < a.parts; j += RUNS) {
            float y[4];
            load_piece(p + j * all, left, y);
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] += y[c];
        }
        if constexpr (RUNS > 1) {
            s_run[run][four] = make_float4(x[0], x[1], x[2], x[3]);
            __syncthreads();
            if (run == 0)
#pragma unroll
                for (int r = 1; r < RUNS; ++r) {
                    const float4 y = s_run[r][four];
                    x[0] += y.x; x[1] += y.y; x[2] += y.z; x[3] += y.w;
                }
            __syncthreads();
        }
        if (run == 0) store_piece((bias ? a.db + k * a.db_worker : a.dw + k * a.dw_worker) + at, left, x);
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

// Which kernel, its tile, and how the rows are split: by what a row of a tile and the join of the parts were measured to take (us, with all
// places of the GPU taken; 4 x 8192 x 1024 x 1024: 128 columns of X by 256 of dY 77, 132, 184 us of bfloat16, binary16, binary32, by 128
// 100, 145, 194).  A tile of 256 columns is left for one of 128 where it has more columns to spare than that costs.
WeightGradPlan weight_grad_plan(int dtype, uint32_t workers, uint32_t rows, uint32_t cols, uint32_t out, uint64_t dy_row, uint32_t n_cu)
{
    WeightGradPlan p{};
    const uint32_t parts_of = dtype == QGX_F32 ? 2u : dtype == QGX_F16 ? 1u : 0u;
    const double row_256[3] = {0.038, 0.065, 0.090}, row_128[3] = {0.049, 0.071, 0.095};
    p.tiles_i = (cols + 127u) / 128u;
    p.parts = 1;
    p.part_rows = rows;
    // (a thread's part of an address has 32 bits, and pairs of columns are loaded)
    const bool pairs = out >= 2u && dy_row <= (1u << 24);
    p.tile = pairs ? 128u : 0u;
    p.tiles_o = (out + 127u) / 128u;
    if (workers == 0 || rows == 0) return p;
    double best = 0.0;
    for (uint32_t tile = pairs ? 256u : 128u; tile >= 128u; tile -= 128u) {
        const uint32_t tiles_o = (out + tile - 1u) / tile, places = n_cu * (!pairs ? 1u : tile == 256u ? 2u : 4u);
        const uint64_t tiles = (uint64_t)workers * p.tiles_i * tiles_o;
        const double row = tile == 256u ? row_256[parts_of] : row_128[parts_of];
        for (uint32_t want = 1; want <= 256u && (want == 1u || (want - 1u) * 128u < rows); ++want) {
            const uint32_t part_rows = ((rows + want - 1u) / want + kGradRows - 1u) / kGradRows * kGradRows, parts = (rows + part_rows - 1u) / part_rows;
            const uint64_t groups = tiles * parts, rounds = (groups + places - 1u) / places;
            if (parts != want) continue;
            // (with half of the places empty a row takes some two thirds of its time; a workgroup's start and end some 96 rows')
            double us = (double)rounds * (part_rows + 96.0) * row * (2u * groups <= places ? 0.65 : 1.0);
            if (parts > 1u) us += 4.0 + (2.0 * parts + 1.0) * workers * ((double)cols * out) * 4.0 / 5.0e6;
            if (best == 0.0 || us < best) { best = us; p.parts = parts; p.part_rows = part_rows; p.tiles_o = tiles_o; p.tile = pairs ? tile : 0u; }
            if (groups > 4u * places) break;
        }
    }
    if (p.parts > 1u) p.scratch = (uint64_t)workers * p.parts * ((uint64_t)cols * out + out) * sizeof(float);
    return p;
}

template <typename T>
static hipError_t launch_tiles(const WeightGradArgs& a, uint32_t groups, uint32_t workers, uint32_t tile, hipStream_t st)
{
    if (tile == 256u) hipLaunchKernelGGL((k_weight_gradient_wide<T, 1, 4>), dim3(groups * workers), dim3(4 * kWave), 0, st, a);
    else if (tile == 128u) hipLaunchKernelGGL((k_weight_gradient_wide<T, 1, 2>), dim3(groups * workers), dim3(2 * kWave), 0, st, a);
    else hipLaunchKernelGGL(k_weight_gradient<T>, dim3(groups, workers), dim3(kGradThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_weight_grad(int dtype, const WeightGradArgs& args, uint32_t workers, const WeightGradPlan& plan, hipStream_t st)
{
    WeightGradArgs a = args;
    a.tiles_i = plan.tiles_i; a.tiles_o = plan.tiles_o; a.parts = plan.parts; a.part_rows = plan.part_rows;
    if (workers == 0) return hipSuccess;
    const uint64_t values = (uint64_t)a.cols * a.out + a.out;
    const dim3 each((uint32_t)((values + 63u) / 64u < 8192u ? (values + 63u) / 64u : 8192u), workers);
    if (a.rows == 0) {
        hipLaunchKernelGGL(k_weight_gradient_zero, each, dim3(256), 0, st, a);
        return hipGetLastError();
    }
    const uint32_t groups = a.tiles_i * a.tiles_o * a.parts;
    const hipError_t e = dtype == QGX_F32   ? launch_tiles<float>(a, groups, workers, plan.tile, st)
                         : dtype == QGX_F16 ? launch_tiles<_Float16>(a, groups, workers, plan.tile, st)
                                            : launch_tiles<__bf16>(a, groups, workers, plan.tile, st);
    if (e != hipSuccess) return e;
    // (by sixteen threads where parts are many: 256 parts of 128 x 128 sums took 65 us by one)
    if (a.parts > 16u) hipLaunchKernelGGL(k_weight_gradient_join<16>, each, dim3(256), 0, st, a);
    else if (a.parts > 1u) hipLaunchKernelGGL(k_weight_gradient_join<1>, each, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qgx
