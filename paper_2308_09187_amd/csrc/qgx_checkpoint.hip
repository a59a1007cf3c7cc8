// Rows kept in 8 bits, and restored (see qgx_kept.h).  A thread has eight columns, four neighbours a block; rows follow each other without
// a gap, each filled up to whole blocks.
#include "qgx_kept.h"

namespace qgx {

constexpr uint32_t kKeepThreads = 256;
constexpr int kKeepTurns = 4;                              // eights of columns to a thread, their loads under way together

// Eight columns of a row, as loaded: one piece of 16-bit elements, two of binary32.
template <typename T> struct Eight { nt_u32x4 bits[sizeof(T) / 2]; };

// Of a row at p of which n are there; WHOLE: all are.
template <typename T, bool WHOLE>
__device__ __forceinline__ Eight<T> load_eight(const T* p, int n)
{
    Eight<T> e;
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        const T* q = p + h * kPiece<T>;
        if constexpr (WHOLE) e.bits[h] = load_bits(q);
        else e.bits[h] = __builtin_bit_cast(nt_u32x4, load_raw(q, n - h * kPiece<T>));
    }
    return e;
}

// The row and eight of a thread's turn, from its workgroup's first: a division of 64 bits by the workgroup; by the thread one of a number of at most 22
// bits, in binary32 and put right by one (whole divisions, three to a turn, were half of the kernel's time).
struct EightAt { uint32_t row, group; bool any; };
__device__ __forceinline__ EightAt eight_at(uint64_t first_row, uint32_t first_group, uint32_t turn, uint32_t groups, float per_group, uint32_t rows)
{
    const uint32_t at = first_group + turn * kKeepThreads + threadIdx.x;
    uint32_t q = (uint32_t)((float)at * per_group);
    int rest = (int)(at - q * groups);
    if (rest < 0) { --q; rest += (int)groups; }
    else if (rest >= (int)groups) { ++q; rest -= (int)groups; }
    const uint64_t row = first_row + q;
    return EightAt{(uint32_t)min(row, (uint64_t)rows - 1u), (uint32_t)rest, row < rows};
}

// WHOLE: rows one step apart throughout, of whole blocks.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kKeepThreads) void k_checkpoint(KeepArgs a, KeptDraws d, Scalars* sc)
{
    constexpr int W = kPiece<T>;
    const uint32_t groups = a.blocks * 4u;
    const float per_group = 1.0f / (float)groups;
    const uint32_t call = d.on ? kept_call(d, sc) : 0u;
    const PhiloxKeys keys = philox_keys(d.seed_lo, d.seed_hi);
    for (uint64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const uint64_t first = tile * (kKeepThreads * kKeepTurns), first_row = first / groups;
        const uint32_t first_group = (uint32_t)(first - first_row * groups);
        Eight<T> raw[kKeepTurns];
        EightAt at[kKeepTurns];
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            at[i] = eight_at(first_row, first_group, (uint32_t)i, groups, per_group, a.n_rows);
            uint64_t row = at[i].row * a.x_row;
            if (!WHOLE && !a.even) {
                const uint32_t sample = at[i].row / a.rows, r = at[i].row % a.rows, k = sample / a.batch;
                row = k * a.x_worker + (sample - k * a.batch) * a.x_batch + r * a.x_row;
            }
            // (past the last row: of the last)
            raw[i] = load_eight<T, WHOLE>((const T*)a.x + row + (size_t)at[i].group * 8u, at[i].any ? (int)a.cols - (int)at[i].group * 8 : 0);
        }
        uint8_t* codes = a.codes + first * 8u;
        uint8_t* powers = a.powers + first / 4u;
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            float v[8];
            uint32_t bits = largest_bits<T>(raw[i].bits[0]);
#pragma unroll
            for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
                float x[W];
                values_of<T>(raw[i].bits[h], x);
                if (h) bits = max(bits, largest_bits<T>(raw[i].bits[h]));
#pragma unroll
                for (int c = 0; c < W; ++c) v[h * W + c] = x[c];
            }
            uint32_t word[2];
            const uint32_t power = kept_codes<8>(v, quad_max(bits), a.top, d.on != 0u, at[i].group, 0u, at[i].row, call, keys, word);
            if (!at[i].any) continue;
            const uint32_t to = i * kKeepThreads + threadIdx.x;
            *reinterpret_cast<uint2*>(codes + to * 8u) = make_uint2(word[0], word[1]);
            if ((to & 3u) == 0u) {
                powers[to / 4u] = (uint8_t)power;
                if (power == kKeptSpoilt) raise_error(sc, QGX_EBIT_NONFINITE);
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kKeepThreads) void k_restore(KeepArgs a)
{
    const uint32_t groups = a.blocks * 4u;
    const float per_group = 1.0f / (float)groups;
    for (uint64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const uint64_t first = tile * (kKeepThreads * kKeepTurns), first_row = first / groups;
        const uint32_t first_group = (uint32_t)(first - first_row * groups);
        EightAt at[kKeepTurns];
        uint2 word[kKeepTurns];
        uint32_t power[kKeepTurns];
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            at[i] = eight_at(first_row, first_group, (uint32_t)i, groups, per_group, a.n_rows);
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
    const uint32_t workers = a.batch ? a.n_rows / a.rows / a.batch : 1u;
    a.even = (a.batch <= 1u || a.x_batch == a.rows * a.x_row) && (workers <= 1u || a.x_worker == (uint64_t)a.batch * a.rows * a.x_row);
    return a;
}

template <typename T>
static void launch_checkpoint_of(const KeepArgs& a, const KeptDraws& d, Scalars* sc, dim3 grid, hipStream_t st)
{
    if (a.even && a.cols % QGX_KEPT_BLOCK == 0u) hipLaunchKernelGGL((k_checkpoint<T, true>), grid, dim3(kKeepThreads), 0, st, a, d, sc);
    else hipLaunchKernelGGL((k_checkpoint<T, false>), grid, dim3(kKeepThreads), 0, st, a, d, sc);
}

hipError_t launch_checkpoint(int dtype, const KeepArgs& args, const KeptDraws& d, Scalars* sc, hipStream_t st)
{
    if (args.n_rows == 0) return hipSuccess;
    const KeepArgs a = tiles_of(args);
    const dim3 grid((uint32_t)(a.tiles < (1u << 20) ? a.tiles : 1u << 20));
    if (dtype == QGX_F32) launch_checkpoint_of<float>(a, d, sc, grid, st);
    else if (dtype == QGX_F16) launch_checkpoint_of<_Float16>(a, d, sc, grid, st);
    else launch_checkpoint_of<__bf16>(a, d, sc, grid, st);
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
