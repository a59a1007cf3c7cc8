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
    p.tiles_i = (cols + kGradTile - 1u) / kGradTile;
    p.tiles_o = (out + kGradTile - 1u) / kGradTile;
    p.parts = 1;
    p.part_rows = rows;
    if (workers == 0 || rows == 0) return p;
    const uint64_t tiles = (uint64_t)workers * p.tiles_i * p.tiles_o;
    const uint32_t most = (rows + 255u) / 256u;
    const uint32_t want = (uint32_t)min((uint64_t)most, max((uint64_t)1u, 2u * n_cu / tiles));
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
    if (dtype == QGX_F32) hipLaunchKernelGGL(k_weight_gradient<float>, grid, dim3(kGradThreads), 0, st, a);
    else if (dtype == QGX_F16) hipLaunchKernelGGL(k_weight_gradient<_Float16>, grid, dim3(kGradThreads), 0, st, a);
    else hipLaunchKernelGGL(k_weight_gradient<__bf16>, grid, dim3(kGradThreads), 0, st, a);
    if (a.parts > 1u) hipLaunchKernelGGL(k_weight_gradient_join, each, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qgx
