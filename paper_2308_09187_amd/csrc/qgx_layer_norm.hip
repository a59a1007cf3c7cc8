// Layer norm, forward and backward.
//   h = (x - mean) rstd,  y = h w + b;   g = dy w,  dx = rstd (g - mean(g) - h mean(g h)),  dw = sum_rows dy h,  db = sum_rows dy
// A row stays in registers between its sums, so that it crosses memory once; LANES threads share it, N pieces of 16 bytes each.
// Sums are in binary32.  A row's: a thread's columns one by one, at most 32 of them (of rows too long for registers cols / 1024), then the
// threads' in a tree.  A column's: the rows of a workgroup's group one by one (a worker's rows over its workgroups and their groups), then the
// groups', and the workgroups' by 64 runs and a tree.
// Both passes are bound by memory.  8 x 4096 x 4096 bfloat16 forward, 537 MB: 91 us, 5.9 TB/s, with its memory out of the cache, 79 where the last
// pass's is used again; backward, 805 MB and the workgroups' sums: 158 us, 5.1 TB/s, either way.  8 x 4096 x 2048 backward, 403 MB: 86 to 90 us,
// 4.5 to 4.7 TB/s, and 75.
#include "qgx_types.h"

namespace qgx {

// Shapes with a form for small tensors; larger ones have columns enough for their sums' launch.
template <int LANES> constexpr bool kSmall = LANES <= 256;
template <int LANES> constexpr int kNormThreads = LANES > 256 ? LANES : 256;
template <int LANES> constexpr int kNormGroups = kNormThreads<LANES> / LANES;     // groups of LANES threads in a workgroup
// A thread's group: the same in all lanes of a wave, and known to be, where a group has whole waves.
template <int LANES>
__device__ __forceinline__ uint32_t norm_group()
{
    if constexpr (kNormGroups<LANES> == 1) return 0u;
    else if constexpr (LANES == kWave) return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / LANES));
    else return threadIdx.x / LANES;
}
constexpr uint32_t kNormBlocksMax = 1u << 20;             // workgroups of a launch (a grid's threads stay below 2^32); they go on from there

// The sums over the LANES threads of a row, of M values at once, in each of the threads.  slot: LDS of these sums' own,
// [M][kNormSlots], where a row has several waves; one barrier for all.
constexpr int kNormSlots = 16;
template <int LANES, int M>
__device__ __forceinline__ void row_sums(float (&x)[M], float (*slot)[kNormSlots])
{
    if constexpr (LANES <= kWave) {
#pragma unroll
        for (int m = 0; m < M; ++m) x[m] = lanes_sum<LANES>(x[m]);
    } else {
#pragma unroll
        for (int m = 0; m < M; ++m) x[m] = lanes_sum<kWave>(x[m]);
        if (lane_id() == 0)
#pragma unroll
            for (int m = 0; m < M; ++m) slot[m][wave_id()] = x[m];
        __syncthreads();
#pragma unroll
        for (int m = 0; m < M; ++m) {
            x[m] = slot[m][0];
#pragma unroll
            for (int w = 1; w < LANES / kWave; ++w) x[m] += slot[m][w];
        }
    }
}

// The place of thread `lane`'s j-th piece in a row of cols >= W columns.  A piece that would pass the row's end is moved back to
// end there (and one that starts past it lies there too), so that every access is whole and inside the row: its first `shift`
// columns belong to another piece.  They are left out of the row's sums; what is written for them is the same bits twice.
struct PieceAt {
    int c, shift;
    bool any;                                              // some of its columns are its own
    __device__ __forceinline__ bool owns(int i) const { return i >= shift; }
};

template <int W, int LANES>
__device__ __forceinline__ PieceAt piece_at(int lane, int j, int cols)
{
    const int c0 = (lane + j * LANES) * W, c = min(c0, cols - W);
    return PieceAt{c, c0 - c, c0 < cols};
}

// The parameters of a piece's columns, `none` where there is no such vector.
template <int W>
__device__ __forceinline__ void load_parameters(const float* p, int c0, float none, float (&v)[W])
{
#pragma unroll
    for (int h = 0; h < W / 4; ++h) {
        float q[4] = {none, none, none, none};
        if (p) load_piece(p + c0 + 4 * h, q);
#pragma unroll
        for (int c = 0; c < 4; ++c) v[4 * h + c] = q[c];
    }
}

// The same past whose last column there may be no memory.
template <int W>
__device__ __forceinline__ void load_parameters(const float* p, int c0, int cols, float none, float (&v)[W])
{
#pragma unroll
    for (int c = 0; c < W; ++c) v[c] = p && c0 + c < cols ? p[c0 + c] : none;
}

// R rows to a group, one after the other in memory: the parameters are read once for them (they are 32 bytes to a piece of 16),
// their loads are under way together, and their sums share the barriers.
template <typename T, int LANES, int N, int R>
__global__ __launch_bounds__(kNormThreads<LANES>) void k_layer_norm(NormArgs a)
{
    constexpr int W = kPiece<T>, kGroups = kNormGroups<LANES>;
    __shared__ float s_sum[2][R][kNormSlots];
    const int lane = (int)(threadIdx.x % LANES), cols = (int)a.cols;
    PieceAt at[N];
#pragma unroll
    for (int j = 0; j < N; ++j) at[j] = piece_at<W, LANES>(lane, j, cols);
    for (uint64_t first = ((uint64_t)blockIdx.x * kGroups + norm_group<LANES>()) * R; first < a.n_rows; first += (uint64_t)gridDim.x * kGroups * R) {
        float v[R][N][W], sum[R], sq[R];
        uint32_t k[R], r[R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const uint32_t row = (uint32_t)min(first + q, (uint64_t)a.n_rows - 1u);      // (past the last: it again, and not written)
            k[q] = row / a.rows;
            r[q] = row % a.rows;
            const T* x = (const T*)a.x + k[q] * a.x_worker + r[q] * a.x_row;
#pragma unroll
            for (int j = 0; j < N; ++j) load_piece(x + at[j].c, v[q][j]);
        }
#pragma unroll
        for (int q = 0; q < R; ++q) {
            sum[q] = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int c = 0; c < W; ++c) sum[q] += at[j].owns(c) ? v[q][j][c] : 0.0f;
        }
        row_sums<LANES>(sum, s_sum[0]);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float mean = sum[q] = sum[q] / (float)cols;
            sq[q] = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int c = 0; c < W; ++c) {
                    v[q][j][c] -= mean;
                    const float own = at[j].owns(c) ? v[q][j][c] : 0.0f;
                    sq[q] = fmaf(own, own, sq[q]);
                }
        }
        row_sums<LANES>(sq, s_sum[1]);
#pragma unroll
        for (int q = 0; q < R; ++q) sq[q] = 1.0f / sqrtf(sq[q] / (float)cols + a.eps);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float w[W], b[W];
            load_parameters<W>(a.w, at[j].c, 1.0f, w);
            load_parameters<W>(a.b, at[j].c, 0.0f, b);
#pragma unroll
            for (int q = 0; q < R; ++q) {
#pragma unroll
                for (int c = 0; c < W; ++c) v[q][j][c] = fmaf(v[q][j][c] * sq[q], w[c], b[c]);
                if (at[j].any && first + q < a.n_rows) stream_piece((T*)a.y + k[q] * a.y_worker + r[q] * a.y_row + at[j].c, v[q][j]);
            }
        }
        if (lane == 0)
#pragma unroll
            for (int q = 0; q < R; ++q)
                if (first + q < a.n_rows) {
                    if (a.mean) a.mean[first + q] = sum[q];
                    if (a.rstd) a.rstd[first + q] = sq[q];
                }
    }
}

// Rows too long for registers, or (SHORT) shorter than a piece: read three times, twice from the cache.  All threads take as many turns, four
// turns' loads under way at once (300 x 50001 bfloat16 106 us where every turn asked for its columns first, 36; 2 x 3000 x 33000 binary32
// 579 and 404).
template <typename T, int THREADS, bool SHORT>
__device__ __forceinline__ void long_piece(const T* row, PieceAt at, int cols, float (&v)[kPiece<T>])
{
    if constexpr (SHORT) load_piece(row + at.c, at.any ? cols - at.c : 0, v);
    else load_piece(row + at.c, v);
}

template <int W, int THREADS, bool SHORT>
__device__ __forceinline__ PieceAt long_piece_at(int turn, int cols)
{
    if constexpr (SHORT) return PieceAt{(int)threadIdx.x * W, 0, (int)threadIdx.x * W < cols};
    else return piece_at<W, THREADS>((int)threadIdx.x, turn, cols);
}

// A thread's own columns of a piece; where it has been moved back the others may have been written already, from what was there.
template <typename T, bool SHORT>
__device__ __forceinline__ void store_own(T* row, PieceAt at, int cols, const float (&v)[kPiece<T>])
{
    if (!at.any) return;
    if constexpr (SHORT) {
        store_piece(row + at.c, cols - at.c, v);
    } else if (at.shift == 0) {
        store_piece(row + at.c, v);
    } else {
#pragma unroll
        for (int c = 0; c < kPiece<T>; ++c)
            if (at.owns(c)) row[at.c + c] = (T)v[c];
    }
}

template <int W, bool SHORT>
__device__ __forceinline__ void long_parameters(const float* p, PieceAt at, int cols, float none, float (&v)[W])
{
    if constexpr (SHORT) load_parameters<W>(p, at.c, cols, none, v);
    else load_parameters<W>(p, at.c, none, v);
}

template <typename T, int THREADS, bool SHORT>
__global__ __launch_bounds__(THREADS) void k_layer_norm_long(NormArgs a)
{
    constexpr int W = kPiece<T>;
    __shared__ float s_sum[2][1][kNormSlots];
    const int cols = (int)a.cols, turns = (cols + THREADS * W - 1) / (THREADS * W);
    for (uint32_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
        const uint32_t k = row / a.rows, r = row % a.rows;
        const T* x = (const T*)a.x + k * a.x_worker + r * a.x_row;
        T* y = (T*)a.y + k * a.y_worker + r * a.y_row;
        float sum[1] = {0.0f}, sq[1] = {0.0f};
#pragma unroll 4
        for (int j = 0; j < turns; ++j) {
            const PieceAt at = long_piece_at<W, THREADS, SHORT>(j, cols);
            float v[W];
            long_piece<T, THREADS, SHORT>(x, at, cols, v);
#pragma unroll
            for (int c = 0; c < W; ++c) sum[0] += at.owns(c) ? v[c] : 0.0f;
        }
        row_sums<THREADS>(sum, s_sum[0]);
        const float mean = sum[0] / (float)cols;
#pragma unroll 4
        for (int j = 0; j < turns; ++j) {
            const PieceAt at = long_piece_at<W, THREADS, SHORT>(j, cols);
            float v[W];
            long_piece<T, THREADS, SHORT>(x, at, cols, v);
#pragma unroll
            for (int c = 0; c < W; ++c) {
                const float t = at.owns(c) && (!SHORT || at.c + c < cols) ? v[c] - mean : 0.0f;
                sq[0] = fmaf(t, t, sq[0]);
            }
        }
        row_sums<THREADS>(sq, s_sum[1]);
        const float rstd = 1.0f / sqrtf(sq[0] / (float)cols + a.eps);
#pragma unroll 4
        for (int j = 0; j < turns; ++j) {
            const PieceAt at = long_piece_at<W, THREADS, SHORT>(j, cols);
            float v[W], w[W], b[W];
            long_piece<T, THREADS, SHORT>(x, at, cols, v);
            long_parameters<W, SHORT>(a.w, at, cols, 1.0f, w);
            long_parameters<W, SHORT>(a.b, at, cols, 0.0f, b);
#pragma unroll
            for (int c = 0; c < W; ++c) v[c] = fmaf((v[c] - mean) * rstd, w[c], b[c]);
            store_own<T, SHORT>(y, at, cols, v);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// ---- backward ---------------------------------------------------------------------------------------------------------
// One pass over dy and x for all three gradients: a workgroup takes every parts-th set of rows of a worker, writes their dx and
// keeps the columns' sums in registers (a thread has the same columns in every row).  At its end it leaves them in scratch, one row
// of sums for each of dw and db, for k_layer_norm_join, or, where a worker has one workgroup, where they belong.

// Where a workgroup's sums go: dw's and db's row of it.
struct NormSums { float* w; float* b; };
__device__ __forceinline__ NormSums norm_sums(const NormBackArgs& a, uint32_t k, uint32_t part)
{
    if (a.parts == 1u) return NormSums{a.dw ? a.dw + k * a.param_stride : nullptr, a.db ? a.db + k * a.param_stride : nullptr};
    float* s = a.scratch + ((size_t)k * a.parts + part) * 2u * a.sum_stride;
    return NormSums{a.dw ? s : nullptr, a.db ? s + a.sum_stride : nullptr};
}

// Small tensors: the sums of sixteen pieces' columns by a workgroup of their own, from dy and x once more (from the cache): no scratch and
// no second launch, which would take longer.  The rows are dealt to THREADS / 16 threads for each piece.
template <typename T, int THREADS>
__device__ __forceinline__ void columns_apart(const NormBackArgs& a, uint32_t k, uint32_t block, float (*s_part)[16 * kPiece<T>])
{
    constexpr int W = kPiece<T>, kRuns = THREADS / 16;
    const int quad = (int)threadIdx.x % 16, run = (int)threadIdx.x / 16, cols = (int)a.cols;
    const PieceAt at = piece_at<W, 16>(quad, (int)block, cols);
    float dw[W], db[W];
#pragma unroll
    for (int c = 0; c < W; ++c) dw[c] = db[c] = 0.0f;
#pragma unroll 4
    for (uint32_t r = (uint32_t)run; r < a.rows; r += kRuns) {
        float u[W], v[W];
        load_piece((const T*)a.x + k * a.x_worker + r * a.x_row + at.c, u);
        load_piece((const T*)a.dy + k * a.dy_worker + r * a.dy_row + at.c, v);
        const float mean = a.mean[(size_t)k * a.rows + r], rstd = a.rstd[(size_t)k * a.rows + r];
#pragma unroll
        for (int c = 0; c < W; ++c) {
            dw[c] = fmaf(v[c], (u[c] - mean) * rstd, dw[c]);
            db[c] += v[c];
        }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* to = which ? a.db : a.dw;
        if (which) __syncthreads();
#pragma unroll
        for (int c = 0; c < W; ++c) s_part[run][quad * W + c] = which ? db[c] : dw[c];
        __syncthreads();
        if (!to || run != 0 || !at.any) continue;
#pragma unroll
        for (int c = 0; c < W; ++c) {
            float x = s_part[0][quad * W + c];
#pragma unroll
            for (int i = 1; i < kRuns; ++i) x += s_part[i][quad * W + c];
            if (at.owns(c)) to[k * a.param_stride + at.c + c] = x;
        }
    }
}

template <typename T, int LANES, int N, int R>
__global__ __launch_bounds__(kNormThreads<LANES>) void k_layer_norm_back(NormBackArgs a)
{
    constexpr int W = kPiece<T>, kGroups = kNormGroups<LANES>;
    __shared__ float s_sum[2][2 * R][kNormSlots];
    __shared__ float s_cols[kGroups > 1 ? kGroups : 1][kGroups > 1 ? LANES * N * W : 1];
    if constexpr (kSmall<LANES>) {
        __shared__ float s_part[kNormThreads<LANES> / 16][16 * W];
        if (a.apart && blockIdx.x >= a.parts) return columns_apart<T, kNormThreads<LANES>>(a, blockIdx.y, blockIdx.x - a.parts, s_part);
    }
    const int lane = (int)(threadIdx.x % LANES), cols = (int)a.cols;
    const uint32_t group = norm_group<LANES>();
    const uint32_t k = blockIdx.y;
    // (No registers are left for the next rows of binary32 of more than 8192 columns: the 128 that 1024 threads leave each are 6 too few even so,
    // which lie in scratch memory.  2 x 1024 x 16384: 97 us, 4.2 TB/s.)
    constexpr bool kAhead = LANES * N < 4096;
    float w[N][W], dw[N][W], db[N][W];
    PieceAt at[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        at[j] = piece_at<W, LANES>(lane, j, cols);
        load_parameters<W>(a.w, at[j].c, 1.0f, w[j]);
#pragma unroll
        for (int c = 0; c < W; ++c) dw[j][c] = db[j][c] = 0.0f;
    }
    // Of a set of rows, as loaded: half the registers of the values in binary32.  The next set's loads are under way before this one's dx is
    // stored: a wave's loads and stores are waited for in their order.
    nt_u32x4 x[R][N], dy[R][N], next_x[R][N], next_dy[R][N];
    float mean[R], rstd[R], next_mean[R], next_rstd[R], sum[2 * R];
    const uint32_t sets = (a.rows + (kGroups * R - 1u)) / (kGroups * R);
    auto load = [&](uint32_t set) {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            // (in place of a row past the last: zeros)
            const uint32_t at_row = (set * kGroups + group) * R + q, r = min(at_row, a.rows - 1u);
            const bool ok = at_row < a.rows;
            const T* px = (const T*)a.x + k * a.x_worker + r * a.x_row;
            const T* pg = (const T*)a.dy + k * a.dy_worker + r * a.dy_row;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                next_x[q][j] = load_bits(px + at[j].c);
                next_dy[q][j] = load_bits(pg + at[j].c);
                if (!ok) next_x[q][j] = next_dy[q][j] = nt_u32x4{0u, 0u, 0u, 0u};
            }
            next_mean[q] = a.mean[(size_t)k * a.rows + r];
            next_rstd[q] = a.rstd[(size_t)k * a.rows + r];
            if (!ok) next_mean[q] = next_rstd[q] = 0.0f;
        }
    };
    if (kAhead && blockIdx.x < sets) load(blockIdx.x);
    int turn = 0;
    for (uint32_t set = blockIdx.x; set < sets; set += a.parts, turn ^= 1) {
        const uint32_t first = (set * kGroups + group) * R;
        if (!kAhead) load(set);
#pragma unroll
        for (int q = 0; q < R; ++q) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                x[q][j] = next_x[q][j];
                dy[q][j] = next_dy[q][j];
            }
            mean[q] = next_mean[q];
            rstd[q] = next_rstd[q];
        }
        if (kAhead && set + a.parts < sets) load(set + a.parts);     // (the same for the whole workgroup)
        // With h = (x - mean) rstd: sums of g and g h, dw += dy h, db += dy.  (rstd stands beside x - mean wherever it is multiplied: of a row
        // with hardly any spread rstd^2, and of others g (x - mean), lie outside binary32 where the gradients do not.)
#pragma unroll
        for (int q = 0; q < R; ++q) {
            sum[q] = sum[R + q] = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float u[W], v[W];
                values_of<T>(x[q][j], u);
                values_of<T>(dy[q][j], v);
#pragma unroll
                for (int c = 0; c < W; ++c) {
                    const float d = v[c], h = (u[c] - mean[q]) * rstd[q], g = at[j].owns(c) ? d * w[j][c] : 0.0f;
                    sum[q] += g;
                    sum[R + q] = fmaf(g, h, sum[R + q]);
                    dw[j][c] = fmaf(d, h, dw[j][c]);
                    db[j][c] += d;
                }
                // (added here and now: left to the end of the round, the terms would be kept across the sums)
#pragma unroll
                for (int c = 0; c < W; ++c) asm volatile("" : "+v"(dw[j][c]), "+v"(db[j][c]));
            }
        }
        if (!a.dx) continue;
        row_sums<LANES>(sum, s_sum[turn]);                 // (two sets of slots in turn: one barrier a round)
        // dx = rstd (g - mean g - h mean(g h))
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float minus_m1 = -(sum[q] / (float)cols), minus_m2 = -(sum[R + q] / (float)cols);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                // (worked out again from what was loaded: kept across the sums, the values would take twice its registers)
                asm volatile("" : "+v"(x[q][j]), "+v"(dy[q][j]));
                float u[W], out[W];
                values_of<T>(x[q][j], u);
                values_of<T>(dy[q][j], out);
#pragma unroll
                for (int c = 0; c < W; ++c) out[c] = rstd[q] * fmaf((u[c] - mean[q]) * rstd[q], minus_m2, fmaf(out[c], w[j][c], minus_m1));
                if (at[j].any && first + q < a.rows) stream_piece((T*)a.dx + k * a.dx_worker + (first + q) * a.dx_row + at[j].c, out);
            }
        }
    }
    if (kSmall<LANES> && a.apart) return;
    const NormSums out = norm_sums(a, k, blockIdx.x);
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int h = 0; h < W / 4; ++h) {              // (columns that another piece has too: the same bits)
                const float pw[4] = {dw[j][4 * h], dw[j][4 * h + 1], dw[j][4 * h + 2], dw[j][4 * h + 3]};
                const float pb[4] = {db[j][4 * h], db[j][4 * h + 1], db[j][4 * h + 2], db[j][4 * h + 3]};
                if (out.w && at[j].any) store_piece(out.w + at[j].c + 4 * h, pw);
                if (out.b && at[j].any) store_piece(out.b + at[j].c + 4 * h, pb);
            }
    } else {
        // the groups' sums joined, those of dw first, then db's in the same memory
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float* to = which ? out.b : out.w;
            if (which) __syncthreads();
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int c = 0; c < W; ++c)
                    if (at[j].any) s_cols[group][at[j].c + c] = which ? db[j][c] : dw[j][c];
            __syncthreads();
            if (to)
                for (int c = (int)threadIdx.x; c < cols; c += kNormThreads<LANES>) {
                    float x = s_cols[0][c];
#pragma unroll
                    for (int g = 1; g < kGroups; ++g) x += s_cols[g][c];
                    to[c] = x;
                }
        }
    }
}

// Rows too long for registers, or (SHORT) shorter than a piece: dx by itself, dy and x read a second time from the cache (all three
// gradients of 2 x 1024 x 32768 bfloat16, 402 MB: 310 us where every turn asked for its columns first, 159).
template <typename T, int THREADS, bool SHORT>
__global__ __launch_bounds__(THREADS) void k_layer_norm_dx_long(NormBackArgs a)
{
    constexpr int W = kPiece<T>;
    __shared__ float s_sum[2][2][kNormSlots];
    const int cols = (int)a.cols, turns = (cols + THREADS * W - 1) / (THREADS * W);
    int turn = 0;
    for (uint32_t row = blockIdx.x; row < a.n_rows; row += gridDim.x, turn ^= 1) {
        const uint32_t k = row / a.rows, r = row % a.rows;
        const T* x = (const T*)a.x + k * a.x_worker + r * a.x_row;
        const T* dy = (const T*)a.dy + k * a.dy_worker + r * a.dy_row;
        T* dx = (T*)a.dx + k * a.dx_worker + r * a.dx_row;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sum[2] = {0.0f, 0.0f};
#pragma unroll 2
        for (int j = 0; j < turns; ++j) {
            const PieceAt at = long_piece_at<W, THREADS, SHORT>(j, cols);
            float u[W], v[W], w[W];
            long_piece<T, THREADS, SHORT>(x, at, cols, u);
            long_piece<T, THREADS, SHORT>(dy, at, cols, v);
            long_parameters<W, SHORT>(a.w, at, cols, 1.0f, w);
#pragma unroll
            for (int c = 0; c < W; ++c) {
                const float g = at.owns(c) ? v[c] * w[c] : 0.0f;       // (past the end of a short row: v is 0)
                sum[0] += g;
                sum[1] = fmaf(g, (u[c] - mean) * rstd, sum[1]);
            }
        }
        row_sums<THREADS>(sum, s_sum[turn]);
        const float m1 = sum[0] / (float)cols, m2 = sum[1] / (float)cols;
#pragma unroll 2
        for (int j = 0; j < turns; ++j) {
            const PieceAt at = long_piece_at<W, THREADS, SHORT>(j, cols);
            float u[W], v[W], w[W];
            long_piece<T, THREADS, SHORT>(x, at, cols, u);
            long_piece<T, THREADS, SHORT>(dy, at, cols, v);
            long_parameters<W, SHORT>(a.w, at, cols, 1.0f, w);
#pragma unroll
            for (int c = 0; c < W; ++c) v[c] = rstd * (v[c] * w[c] - m1 - (u[c] - mean) * rstd * m2);
            store_own<T, SHORT>(dx, at, cols, v);
        }
    }
}

// And their columns' sums: a thread has a piece's columns in every parts-th row of a worker.
template <typename T>
__global__ __launch_bounds__(256) void k_layer_norm_columns(NormBackArgs a)
{
    constexpr int W = kPiece<T>;
    const uint32_t k = blockIdx.z, part = blockIdx.y;
    const int c0 = (int)(blockIdx.x * 256u + threadIdx.x) * W, n = (int)a.cols - c0;
    float dw[W], db[W];
#pragma unroll
    for (int c = 0; c < W; ++c) dw[c] = db[c] = 0.0f;
    for (uint32_t r = part; r < a.rows; r += a.parts) {
        float u[W], v[W];
        load_piece((const T*)a.x + k * a.x_worker + r * a.x_row + c0, n, u);
        load_piece((const T*)a.dy + k * a.dy_worker + r * a.dy_row + c0, n, v);
        const float mean = a.mean[(size_t)k * a.rows + r], rstd = a.rstd[(size_t)k * a.rows + r];
#pragma unroll
        for (int c = 0; c < W; ++c) {
            dw[c] = fmaf(v[c], (u[c] - mean) * rstd, dw[c]);
            db[c] += v[c];
        }
    }
    const NormSums out = norm_sums(a, k, part);
#pragma unroll
    for (int h = 0; h < W / 4; ++h) {
        const float pw[4] = {dw[4 * h], dw[4 * h + 1], dw[4 * h + 2], dw[4 * h + 3]}, pb[4] = {db[4 * h], db[4 * h + 1], db[4 * h + 2], db[4 * h + 3]};
        if (out.w) store_piece(out.w + c0 + 4 * h, n - 4 * h, pw);
        if (out.b) store_piece(out.b + c0 + 4 * h, n - 4 * h, pb);
    }
}

// x over the sixteen lanes that differ in all but the lowest two bits.
__device__ __forceinline__ float join_runs(float x)
{
    LanePair p = lane_pair<32>(__float_as_uint(x));
    p = lane_pair<16>(__float_as_uint(__uint_as_float(p.a) + __uint_as_float(p.b)));
    p = lane_pair<8>(__float_as_uint(__uint_as_float(p.a) + __uint_as_float(p.b)));
    p = lane_pair<4>(__float_as_uint(__uint_as_float(p.a) + __uint_as_float(p.b)));
    return __uint_as_float(p.a) + __uint_as_float(p.b);
}

// The workgroups' sums of sixteen columns joined: four to a thread, 64 runs of the parts side by side.
__global__ __launch_bounds__(256) void k_layer_norm_join(NormBackArgs a)
{
    __shared__ float4 s_run[4][4];
    const uint32_t k = blockIdx.y / 2u, which = blockIdx.y % 2u, quad = threadIdx.x % 4u, run = threadIdx.x / 4u;
    float* out = which ? a.db : a.dw;
    if (!out) return;
    const uint32_t c0 = (blockIdx.x * 4u + quad) * 4u;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c0 < a.cols) {                                     // (a row of sums is whole fours of columns)
        const float* p = a.scratch + ((size_t)k * a.parts * 2u + which) * a.sum_stride + c0;
#pragma unroll 4
        for (uint32_t i = run; i < a.parts; i += 64u) {
            const float4 x = *reinterpret_cast<const float4*>(p + (size_t)i * 2u * a.sum_stride);
            sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
        }
    }
    sum = make_float4(join_runs(sum.x), join_runs(sum.y), join_runs(sum.z), join_runs(sum.w));
    if (lane_id() < 4) s_run[wave_id()][quad] = sum;
    __syncthreads();
    if (run != 0 || c0 >= a.cols) return;
    for (int i = 1; i < 4; ++i) {
        const float4 x = s_run[i][quad];
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
    store_piece(out + k * a.param_stride + c0, (int)(a.cols - c0), v);
}

// ---- which kernel -------------------------------------------------------------------------------------------------------

template <typename T, int LANES, int N, int R>
static hipError_t launch_norm_as(const NormArgs& a, hipStream_t st)
{
    constexpr uint32_t per = kNormGroups<LANES> * R;
    hipLaunchKernelGGL((k_layer_norm<T, LANES, N, R>), dim3(min((a.n_rows - 1u) / per + 1u, kNormBlocksMax)), dim3(kNormThreads<LANES>), 0, st, a);
    return hipGetLastError();
}

// Two rows at a time once that leaves eight workgroups for every compute unit (8 x 4096 x 4096 bfloat16: 83 us with four rows, 88 with
// one, 81 with two).
template <typename T, int LANES, int N>
static hipError_t launch_norm_by_rows(const NormArgs& a, uint32_t n_cu, hipStream_t st)
{
    if (a.n_rows / ((uint32_t)kNormGroups<LANES> * 2u) >= 8u * n_cu) return launch_norm_as<T, LANES, N, 2>(a, st);
    return launch_norm_as<T, LANES, N, 1>(a, st);
}

// The fewest threads that hold a row in a piece or two each, where steps are wide in three (8 x 8192 x 1100 bfloat16: 62 us in three pieces of 64
// threads, 84 in one of 256 of which half are idle), and in up to four of a workgroup's 256 or more (four pieces to each of four
// threads took 32 us for 8 x 65536 x 64, two 24).
template <typename T>
static hipError_t launch_norm_of(const NormArgs& a, uint32_t n_cu, hipStream_t st)
{
    const uint32_t pieces = (a.cols + kPiece<T> - 1u) / kPiece<T>;
    if (a.cols < (uint32_t)kPiece<T>) {
        hipLaunchKernelGGL((k_layer_norm_long<T, 64, true>), dim3(min(a.n_rows, kNormBlocksMax)), dim3(64), 0, st, a);
        return hipGetLastError();
    }
    if (pieces <= 4u) return launch_norm_by_rows<T, 4, 1>(a, n_cu, st);
    if (pieces <= 8u) return launch_norm_by_rows<T, 4, 2>(a, n_cu, st);
    if (pieces <= 16u) return launch_norm_by_rows<T, 16, 1>(a, n_cu, st);
    if (pieces <= 32u) return launch_norm_by_rows<T, 16, 2>(a, n_cu, st);
    if (pieces <= 64u) return launch_norm_by_rows<T, 64, 1>(a, n_cu, st);
    if (pieces <= 128u) return launch_norm_by_rows<T, 64, 2>(a, n_cu, st);
    if (pieces <= 192u) return launch_norm_by_rows<T, 64, 3>(a, n_cu, st);
    if (pieces <= 256u) return launch_norm_by_rows<T, 256, 1>(a, n_cu, st);
    if (pieces <= 512u) return launch_norm_by_rows<T, 256, 2>(a, n_cu, st);
    if (pieces <= 768u) return launch_norm_as<T, 256, 3, 1>(a, st);
    if (pieces <= 1024u) return launch_norm_as<T, 256, 4, 1>(a, st);
    if (pieces <= 1536u) return launch_norm_as<T, 512, 3, 1>(a, st);
    if (pieces <= 2048u) return launch_norm_as<T, 512, 4, 1>(a, st);
    if (pieces <= 4096u) return launch_norm_as<T, 1024, 4, 1>(a, st);
    hipLaunchKernelGGL((k_layer_norm_long<T, 1024, false>), dim3(min(a.n_rows, kNormBlocksMax)), dim3(1024), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_layer_norm(int dtype, const NormArgs& a, uint32_t n_cu, hipStream_t st)
{
    if (a.n_rows == 0) return hipSuccess;
    return dtype == QGX_F32   ? launch_norm_of<float>(a, n_cu, st)
           : dtype == QGX_F16 ? launch_norm_of<_Float16>(a, n_cu, st)
                              : launch_norm_of<__bf16>(a, n_cu, st);
}

// The backward kernel's shape for a row: threads that share one, pieces and rows of each thread; no threads: rows too long or too
// short for it.  (The longest by 1024 threads, one workgroup to a compute unit: 2 x 1024 x 16384 binary32 112 us by 512 threads of eight
// pieces, 95; 8 x 128 x 16384 bfloat16 54 by 512 of four, 37.)
struct BackShape { uint32_t lanes, pieces, rows; };
static BackShape back_shape(uint32_t cols, uint32_t W)
{
    const uint32_t pieces = (cols + W - 1u) / W;
    if (cols < W || cols > 16384u) return BackShape{0, 0, 0};          // (32 columns to a thread: their sums alone take 64 registers)
    if (pieces <= 4u) return BackShape{4, 1, 2};
    if (pieces <= 16u) return pieces <= 8u ? BackShape{4, 2, 1} : BackShape{16, 1, 2};
    if (pieces <= 64u) return pieces <= 32u ? BackShape{16, 2, 1} : BackShape{64, 1, 2};
    if (pieces <= 128u) return BackShape{64, 2, 1};
    if (pieces <= 256u) return BackShape{256, 1, 2};
    if (pieces <= 512u) return BackShape{256, 2, 1};
    if (pieces <= 1024u) return BackShape{256, 4, 1};
    return pieces <= 2048u ? BackShape{1024, 2, 1} : BackShape{1024, 4, 1};
}

NormBackPlan norm_back_plan(int dtype, uint32_t workers, uint32_t rows, uint32_t cols, uint32_t n_cu)
{
    const uint32_t W = dtype == QGX_F32 ? 4u : 8u, pieces = (cols + W - 1u) / W;
    const BackShape shape = back_shape(cols, W);
    NormBackPlan p{};
    p.sum_stride = (cols + 3u) / 4u * 4u;
    const uint32_t at_once = shape.lanes ? max(256u, shape.lanes) / shape.lanes * shape.rows : 4u;
    const uint32_t sets = rows / at_once + (rows % at_once != 0u);
    // a few workgroups for every compute unit, over all workers (and, where rows are long, over the columns)
    // (the more columns, the more a workgroup's sums weigh: 8 x 4096 x 4096 bfloat16 167 us with three for each, 159 with two, 162 with
    // one; 8 x 2048 x 8192 173 with two, 156 with one; up to 64 threads to a row three are as good as two or better)
    const uint32_t each = shape.pieces == 4u || shape.lanes == 1024u ? 1u : shape.lanes == 256u ? 2u : shape.lanes ? 3u : 4u;
    const uint32_t want = max(1u, each * n_cu / (workers * (shape.lanes ? 1u : (pieces + 255u) / 256u)));
    p.parts = max(1u, min(sets, want));
    // Few rows and little in all: a workgroup for every set, the columns' sums apart.  (4 x 512 x 500 binary32 18 us a call with the sums joined by a
    // launch, 14; of its kernels 8.6 and 7.7.  1000 x 1000 bfloat16: 9.7 and 13.8.)
    p.apart = p.parts > 1u && shape.lanes && shape.lanes <= 256u && rows <= 512u && (uint64_t)workers * rows * cols <= (1u << 20);
    if (p.apart) p.parts = sets;
    p.scratch = p.parts == 1u || p.apart ? 0 : (uint64_t)workers * p.parts * 2u * p.sum_stride * sizeof(float);
    return p;
}

template <typename T, int LANES, int N, int R>
static hipError_t launch_back_as(const NormBackArgs& a, uint32_t workers, hipStream_t st)
{
    const uint32_t apart = a.apart ? (a.cols + 16u * kPiece<T> - 1u) / (16u * kPiece<T>) : 0u;
    hipLaunchKernelGGL((k_layer_norm_back<T, LANES, N, R>), dim3(a.parts + apart, workers), dim3(kNormThreads<LANES>), 0, st, a);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_back_of(const NormBackArgs& a, uint32_t workers, hipStream_t st)
{
    const uint32_t pieces = (a.cols + kPiece<T> - 1u) / kPiece<T>;
    const BackShape s = back_shape(a.cols, kPiece<T>);
    if (s.lanes == 4u) return s.pieces == 1u ? launch_back_as<T, 4, 1, 2>(a, workers, st) : launch_back_as<T, 4, 2, 1>(a, workers, st);
    if (s.lanes == 16u) return s.pieces == 1u ? launch_back_as<T, 16, 1, 2>(a, workers, st) : launch_back_as<T, 16, 2, 1>(a, workers, st);
    if (s.lanes == 64u) return s.pieces == 1u ? launch_back_as<T, 64, 1, 2>(a, workers, st) : launch_back_as<T, 64, 2, 1>(a, workers, st);
    if (s.lanes == 256u)
        return s.pieces == 1u   ? launch_back_as<T, 256, 1, 2>(a, workers, st)
               : s.pieces == 2u ? launch_back_as<T, 256, 2, 1>(a, workers, st)
                                : launch_back_as<T, 256, 4, 1>(a, workers, st);
    if constexpr (sizeof(T) == 4)
        if (s.pieces == 4u) return launch_back_as<T, 1024, 4, 1>(a, workers, st);
    if (s.lanes == 1024u) return launch_back_as<T, 1024, 2, 1>(a, workers, st);
    if (a.dx && a.n_rows) {
        const dim3 grid(min(a.n_rows, kNormBlocksMax));
        if (a.cols < (uint32_t)kPiece<T>) hipLaunchKernelGGL((k_layer_norm_dx_long<T, 64, true>), grid, dim3(64), 0, st, a);
        else hipLaunchKernelGGL((k_layer_norm_dx_long<T, 1024, false>), grid, dim3(1024), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!a.dw && !a.db) return hipSuccess;
    hipLaunchKernelGGL(k_layer_norm_columns<T>, dim3((pieces + 255u) / 256u, a.parts, workers), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_layer_norm_back(int dtype, const NormBackArgs& args, uint32_t workers, const NormBackPlan& plan, hipStream_t st)
{
    NormBackArgs a = args;
    a.parts = plan.parts;
    a.sum_stride = plan.sum_stride;
    a.apart = plan.apart && (a.dw || a.db);
    if (a.apart && !a.dx) a.parts = 0u;                    // no rows' workgroups
    if (!a.dx && !a.dw && !a.db) return hipSuccess;
    const hipError_t e = dtype == QGX_F32   ? launch_back_of<float>(a, workers, st)
                         : dtype == QGX_F16 ? launch_back_of<_Float16>(a, workers, st)
                                            : launch_back_of<__bf16>(a, workers, st);
    if (e != hipSuccess || a.parts == 1u || a.apart || (!a.dw && !a.db)) return e;
    hipLaunchKernelGGL(k_layer_norm_join, dim3((a.cols + 15u) / 16u, 2u * workers), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qgx
