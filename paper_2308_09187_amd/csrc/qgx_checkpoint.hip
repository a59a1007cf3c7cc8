// Rows kept in 8 bits, and restored (see qgx_kept.h).  A thread has eight columns, four neighbours a block; rows follow each other without
// a gap, each filled up to whole blocks.
#include "qgx_kept.h"

namespace qgx {

constexpr uint32_t kKeepThreads = 256;
constexpr int kKeepTurns = 4;                              // eights of columns to a thread, their loads under way together

// Eight columns of a row at p of which n are there.
template <typename T>
__device__ __forceinline__ void load_eight(const T* p, int n, float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        load_piece(p, n, v);
    } else {
        float a[4], b[4];
        load_piece(p, n, a);
        load_piece(p + 4, n - 4, b);
#pragma unroll
        for (int c = 0; c < 4; ++c) { v[c] = a[c]; v[4 + c] = b[c]; }
    }
}

// The row and eight of a thread's turn, from its workgroup's first: a division of 64 bits by the workgroup, of 32 by the thread.
struct EightAt { uint32_t row, group; bool any; };
__device__ __forceinline__ EightAt eight_at(uint64_t first_row, uint32_t first_group, uint32_t turn, uint32_t groups, uint32_t rows)
{
    const uint32_t at = first_group + turn * kKeepThreads + threadIdx.x;
    const uint64_t row = first_row + at / groups;
    return EightAt{(uint32_t)min(row, (uint64_t)rows - 1u), at % groups, row < rows};
}

template <typename T>
__global__ __launch_bounds__(kKeepThreads) void k_checkpoint(KeepArgs a, KeptDraws d, Scalars* sc)
{
    const uint32_t groups = a.blocks * 4u;
    const uint32_t call = d.on ? kept_call(d, sc) : 0u;
    const PhiloxKeys keys = philox_keys(d.seed_lo, d.seed_hi);
    for (uint64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const uint64_t first = tile * (kKeepThreads * kKeepTurns), first_row = first / groups;
        const uint32_t first_group = (uint32_t)(first - first_row * groups);
        float v[kKeepTurns][8];
        EightAt at[kKeepTurns];
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            at[i] = eight_at(first_row, first_group, (uint32_t)i, groups, a.n_rows);
            const uint32_t sample = at[i].row / a.rows, r = at[i].row % a.rows, k = sample / a.batch;
            const int n = at[i].any ? (int)a.cols - (int)at[i].group * 8 : 0;
            load_eight((const T*)a.x + k * a.x_worker + (sample - k * a.batch) * a.x_batch + r * a.x_row + (size_t)at[i].group * 8u, n, v[i]);
        }
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            uint32_t bits = 0u;
#pragma unroll
            for (int c = 0; c < 8; ++c) bits = max(bits, __float_as_uint(v[i][c]) & 0x7FFFFFFFu);
            const uint32_t power = kept_power(quad_max(bits), a.top);
            uint32_t word[2];
            if (power == kKeptSpoilt) {                    // (0 * infinity is no zero)
#pragma unroll
                for (int c = 0; c < 8; ++c) v[i][c] = 0.0f;
            }
            kept_codes(v[i], kept_over(power), d.on != 0u, at[i].group, at[i].row, call, keys, word);
            if (!at[i].any) continue;
            const size_t to = (size_t)at[i].row * groups + at[i].group;
            *reinterpret_cast<uint2*>(a.codes + to * 8u) = make_uint2(word[0], word[1]);
            if ((at[i].group & 3u) == 0u) {
                a.powers[to / 4u] = (uint8_t)power;
                if (power == kKeptSpoilt) raise_error(sc, QGX_EBIT_NONFINITE);
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kKeepThreads) void k_restore(KeepArgs a)
{
    const uint32_t groups = a.blocks * 4u;
    for (uint64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const uint64_t first = tile * (kKeepThreads * kKeepTurns), first_row = first / groups;
        const uint32_t first_group = (uint32_t)(first - first_row * groups);
        EightAt at[kKeepTurns];
        uint2 word[kKeepTurns];
        uint32_t power[kKeepTurns];
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            at[i] = eight_at(first_row, first_group, (uint32_t)i, groups, a.n_rows);
            const size_t from = (size_t)at[i].row * groups + at[i].group;
            word[i] = *reinterpret_cast<const uint2*>(a.codes + from * 8u);
            power[i] = a.powers[from / 4u];
        }
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            const float scale = kept_scale(power[i]);
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = kept_value(((c < 4 ? word[i].x : word[i].y) >> (8 * (c & 3))) & 0xFFu, scale);
            const int n = at[i].any ? (int)a.cols - (int)at[i].group * 8 : 0;
            T* y = (T*)a.y + at[i].row * a.y_row + (size_t)at[i].group * 8u;
            if constexpr (sizeof(T) == 2) {
                store_piece(y, n, v);
            } else {
                const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
                store_piece(y, n, lo);
                store_piece(y + 4, n - 4, hi);
            }
        }
    }
}

static KeepArgs tiles_of(const KeepArgs& args)
{
    KeepArgs a = args;
    const uint64_t eights = (uint64_t)a.n_rows * a.blocks * 4u, per = kKeepThreads * kKeepTurns;
    a.tiles = (eights + per - 1u) / per;
    return a;
}

hipError_t launch_checkpoint(int dtype, const KeepArgs& args, const KeptDraws& d, Scalars* sc, hipStream_t st)
{
    if (args.n_rows == 0) return hipSuccess;
    const KeepArgs a = tiles_of(args);
    const dim3 grid((uint32_t)(a.tiles < (1u << 20) ? a.tiles : 1u << 20)), block(kKeepThreads);
    if (dtype == QGX_F32) hipLaunchKernelGGL(k_checkpoint<float>, grid, block, 0, st, a, d, sc);
    else if (dtype == QGX_F16) hipLaunchKernelGGL(k_checkpoint<_Float16>, grid, block, 0, st, a, d, sc);
    else hipLaunchKernelGGL(k_checkpoint<__bf16>, grid, block, 0, st, a, d, sc);
    return hipGetLastError();
}

hipError_t launch_restore(int dtype, const KeepArgs& args, hipStream_t st)
{
    if (args.n_rows == 0) return hipSuccess;
    const KeepArgs a = tiles_of(args);
    const dim3 grid((uint32_t)(a.tiles < (1u << 20) ? a.tiles : 1u << 20)), block(kKeepThreads);
    if (dtype == QGX_F32) hipLaunchKernelGGL(k_restore<float>, grid, block, 0, st, a);
    else if (dtype == QGX_F16) hipLaunchKernelGGL(k_restore<_Float16>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(k_restore<__bf16>, grid, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace qgx
