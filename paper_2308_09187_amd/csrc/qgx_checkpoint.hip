// Rows kept in 8 bits, and restored (see qgx_kept.h).  A thread has eight columns, which is what one Philox block rounds, four neighbours a block: its largest
// magnitude is two exchanges between lanes, and no element leaves its thread.  Rows follow each other without a gap, each filled up to whole blocks.
// Keeping without bias is bound by vector arithmetic: of some 190 issue slots for eight elements Philox takes 104, rounding 46; restoring by memory.
// (8 x 4096 x 2048 bfloat16: kept 46 us, the bytes alone 31 at 6.5 TB/s; restored 30, 6.7 TB/s.)
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

// A thread's eights, turn by turn, from its workgroup's first: the row after the first, and the eight of it.  A division of 64 bits by the workgroup; by the
// thread one of numbers of at most 22 bits, in binary32 and put right by one, and from one turn to the next an addition (whole divisions, three to a turn, were
// half of the kernel's time; one of these to a turn, with 64-bit addresses, a sixth).
struct EightAt {
    uint32_t row, group;
    bool carried;                                          // in the last step: into a row more than the step's own

    __device__ __forceinline__ EightAt(uint32_t first_group, uint32_t groups)
    {
        const uint32_t at = first_group + threadIdx.x;
        row = (uint32_t)((float)at * (1.0f / (float)groups));
        const int rest = (int)(at - row * groups), below = rest >> 31;
        row += (uint32_t)below;
        group = (uint32_t)(rest + (below & (int)groups));
        carry(groups);
    }
    __device__ __forceinline__ void next(uint32_t step_rows, uint32_t step_groups, uint32_t groups)
    {
        row += step_rows;
        group += step_groups;
        carry(groups);
    }
    __device__ __forceinline__ void carry(uint32_t groups)
    {
        carried = group >= groups;
        group -= carried ? groups : 0u;
        row += carried ? 1u : 0u;
    }
};

// WHOLE: rows one step apart throughout, of whole blocks, a workgroup's rows less than 2^31 bytes apart.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kKeepThreads) void k_checkpoint(KeepArgs a, KeptDraws d, Scalars* sc)
{
    constexpr int W = kPiece<T>;
    const uint32_t groups = a.blocks * 4u, step_rows = kKeepThreads / groups, step_groups = kKeepThreads % groups;
    const uint32_t call = d.on ? kept_call(d, sc) : 0u;
    const PhiloxKeys keys = philox_keys(d.seed_lo, d.seed_hi);
    const uint32_t gap = (uint32_t)a.x_row - a.cols, step = 8u * kKeepThreads + step_rows * gap;
    for (uint64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const uint64_t first = tile * (kKeepThreads * kKeepTurns), first_row = first / groups;
        const uint32_t rows = a.n_rows - (uint32_t)first_row;
        EightAt at((uint32_t)(first - first_row * groups), groups);
        Eight<T> raw[kKeepTurns];
        uint32_t row[kKeepTurns], group[kKeepTurns], offset = at.row * (uint32_t)a.x_row + at.group * 8u;
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            row[i] = at.row;
            group[i] = at.group;
            const bool any = at.row < rows;                // (past the last row: the workgroup's first)
            if constexpr (WHOLE) {
                raw[i] = load_eight<T, true>((const T*)a.x + first_row * a.x_row + (any ? offset : 0u), 8);
            } else {
                const uint32_t whole = (uint32_t)first_row + (any ? at.row : 0u), sample = whole / a.rows, r = whole % a.rows, k = sample / a.batch;
                const uint64_t from = k * a.x_worker + (sample - k * a.batch) * a.x_batch + r * a.x_row;
                raw[i] = load_eight<T, false>((const T*)a.x + from + (size_t)at.group * 8u, any ? (int)a.cols - (int)at.group * 8 : 0);
            }
            at.next(step_rows, step_groups, groups);
            offset += step + (at.carried ? gap : 0u);
        }
        uint8_t* codes = a.codes + first * 8u;
        uint8_t* powers = a.powers + first / 4u;
        uint32_t to = threadIdx.x;
        asm volatile("" : "+v"(to));                       // (else every thread's address is kept in 64 bits)
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
            const uint32_t power = kept_codes<8>(v, quad_max(bits), a.top, d.on != 0u, group[i], 0u, (uint32_t)first_row + row[i], d.domain, call, keys, word);
            if (row[i] >= rows) continue;
            *reinterpret_cast<uint2*>(codes + i * kKeepThreads * 8u + to * 8u) = make_uint2(word[0], word[1]);
            if ((to & 3u) == 0u) {
                powers[i * kKeepThreads / 4u + to / 4u] = (uint8_t)power;
                if (power == kKeptSpoilt) raise_error(sc, QGX_EBIT_NONFINITE);
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kKeepThreads) void k_restore(KeepArgs a)
{
    const uint32_t groups = a.blocks * 4u, step_rows = kKeepThreads / groups, step_groups = kKeepThreads % groups;
    for (uint64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const uint64_t first = tile * (kKeepThreads * kKeepTurns), first_row = first / groups;
        const uint32_t rows = a.n_rows - (uint32_t)first_row;
        EightAt at((uint32_t)(first - first_row * groups), groups);
        uint32_t row[kKeepTurns], group[kKeepTurns], power[kKeepTurns];
        uint2 word[kKeepTurns];
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            row[i] = at.row;
            group[i] = at.group;
            const uint32_t from = at.row < rows ? i * kKeepThreads + threadIdx.x : 0u;           // (rows follow each other without a gap)
            word[i] = *reinterpret_cast<const uint2*>(a.codes + first * 8u + from * 8u);
            power[i] = (a.powers + first / 4u)[from / 4u];
            at.next(step_rows, step_groups, groups);
        }
#pragma unroll
        for (int i = 0; i < kKeepTurns; ++i) {
            const float scale = kept_scale(power[i]);
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = kept_value(((c < 4 ? word[i].x : word[i].y) >> (8 * (c & 3))) & 0xFFu, scale);
            const int n = row[i] < rows ? (int)a.cols - (int)group[i] * 8 : 0;
            T* y = (T*)a.y + first_row * a.y_row + row[i] * a.y_row + (size_t)group[i] * 8u;
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
    const uint64_t apart = (kKeepThreads * kKeepTurns / (a.blocks * 4u) + 2u) * a.x_row;         // (x_row < 2^60 / rows: of one row it may be anything)
    if (a.even && a.cols % QGX_KEPT_BLOCK == 0u && a.x_row < (1u << 28) && apart * sizeof(T) < (1ull << 31)) hipLaunchKernelGGL((k_checkpoint<T, true>), grid, dim3(kKeepThreads), 0, st, a, d, sc);
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
