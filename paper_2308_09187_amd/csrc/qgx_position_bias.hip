// Learned relative position bias by buckets, out = scores + table[row(j - i - p)][head], and the table's gradient.
// Both go by squares of W queries x W keys (W: the elements of 16 bytes): a thread has 2 W - 1 diagonals in registers at places
// that the compiler knows (key - query within the square), and the squares on one block diagonal all have the same ones.
//   forward: a square's 2 W - 1 biases come from a list of the tile's diagonals in LDS, then serve W pieces of 16 bytes;
//   gradient: a thread walks down a block diagonal, its sums of 2 W - 1 diagonals in registers over all queries and sequences, and only at its
//     end are they sorted into the buckets, which are runs of diagonals.  No element meets a bucket, an atomic or a search.
#include "qgx_types.h"

namespace qgx {

constexpr int kBiasThreads = 256;

// p of a sequence, kept within +-2^30 so that a delta fits 32 bits.
__device__ __forceinline__ int position_of(const BiasArgs& a, uint32_t seq)
{
    const int64_t p = a.q_offset + (a.positions ? (int64_t)a.positions[seq] : 0);
    return (int)max((int64_t)-(1 << 30), min(p, (int64_t)(1 << 30)));
}

// ---- forward --------------------------------------------------------------------------------------------------------------
// Squares have ROWS queries (W, or one where there are fewer than W queries).  A workgroup's tile: up to 256 neighbouring squares of
// one band of ROWS queries, or, where a band has no more than 256, 256 squares of several bands that follow each other.
struct Tiling {
    uint32_t per_band;                                     // squares
    uint32_t tiles, tiles_per_band, chunk;                 // tiles_per_band 0: a tile goes on in the next band; else squares of a tile
};

template <int W, int ROWS>
__host__ __device__ inline Tiling tiling(uint32_t q, uint32_t k)
{
    Tiling t{};
    t.per_band = (k + W - 1u) / W;
    const uint32_t bands = (q + ROWS - 1u) / ROWS;
    if (t.per_band > (uint32_t)kBiasThreads) {
        t.tiles_per_band = (t.per_band + kBiasThreads - 1u) / kBiasThreads;
        t.chunk = (t.per_band + t.tiles_per_band - 1u) / t.tiles_per_band;
    }
    // (below 2^32: q k is at most 2^42)
    t.tiles = t.tiles_per_band ? bands * t.tiles_per_band : (uint32_t)(((uint64_t)bands * t.per_band + kBiasThreads - 1u) / kBiasThreads);
    return t;
}

// The most diagonals a tile can have: its squares' keys (all of a band's where it has several) and its queries.
template <int W, int ROWS>
static uint32_t tile_diagonals(const Tiling& t)
{
    if (t.tiles_per_band) return t.chunk * W + ROWS;
    return t.per_band * W + ((kBiasThreads - 2u) / t.per_band + 2u) * ROWS;
}

// A list entry's place: one word is left out after every W, so that lanes W entries apart do not meet in a bank.
template <int W>
__device__ __forceinline__ uint32_t diagonal_slot(uint32_t x) { return x + x / W; }

template <typename T, int ROWS>
__global__ __launch_bounds__(kBiasThreads) void k_position_bias(BiasArgs a, BucketArgs b)
{
    constexpr int W = kPiece<T>;
    extern __shared__ float s_value[];
    const Tiling t = tiling<W, ROWS>(a.q, a.k);
    const uint32_t bands = (a.q + ROWS - 1u) / ROWS;
    const int lo = b.bounds[0], hi = b.bounds[b.n];
    for (uint32_t plane = blockIdx.y; plane < a.planes; plane += gridDim.y) {       // (worker, sequence, head)
        const uint32_t head = plane % a.heads, seq = plane / a.heads, worker = seq / a.batch, n = seq % a.batch;
        const int p = position_of(a, seq);
        const T* in = a.in ? (const T*)a.in + worker * a.i_worker + n * a.i_batch + head * a.i_head : nullptr;
        T* out = (T*)a.out + worker * a.o_worker + n * a.o_batch + head * a.o_head;
        for (uint32_t tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
            uint32_t band0, band1, square, first = 0, end = t.per_band;    // this thread's square of `band`; the tile's squares of a band
            uint32_t band;
            if (t.tiles_per_band) {
                band0 = band1 = band = tile / t.tiles_per_band;
                first = tile % t.tiles_per_band * t.chunk;
                end = min(first + t.chunk, t.per_band);
                square = first + threadIdx.x;
            } else {
                const uint64_t at = (uint64_t)tile * kBiasThreads;
                band0 = (uint32_t)(at / t.per_band);
                band1 = min((uint32_t)((at + kBiasThreads - 1u) / t.per_band), bands - 1u);
                band = (uint32_t)((at + threadIdx.x) / t.per_band);
                square = (uint32_t)((at + threadIdx.x) % t.per_band);
            }
            // deltas of the tile: first, and how many
            const int d0 = (int)(first * W) - (int)((band1 + 1u) * ROWS - 1u) - p;
            const int count = (int)(end * W) - (int)(band0 * ROWS) - p - d0;

            const int j0 = (int)square * W, i0 = (int)band * ROWS, left = (int)a.k - j0;
            const int rows = square < end && band < bands ? min(ROWS, (int)a.q - i0) : 0;
            const int delta0 = j0 - i0 - p;                // of the first query and key
            float v[ROWS][W];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
#pragma unroll
                for (int c = 0; c < W; ++c) v[r][c] = 0.0f;
                // (a piece that is masked as a whole is not read)
                if (in && r < rows && delta0 - r + W > lo && delta0 - r < hi) load_piece(in + (uint32_t)(i0 + r) * a.i_row + j0, left, v[r]);
            }
            __syncthreads();                               // the tile before has been dealt with
            for (uint32_t s = threadIdx.x / kWave; s < b.n; s += kBiasThreads / kWave) {
                const int x0 = max(b.bounds[s], d0), x1 = (int)min((int64_t)b.bounds[s + 1], (int64_t)d0 + count);
                if (x0 >= x1) continue;
                const float value = a.table[(size_t)b.rows[s] * a.heads + head];
                for (int x = x0 + lane_id(); x < x1; x += kWave) s_value[diagonal_slot<W>((uint32_t)(x - d0))] = value;
            }
            __syncthreads();
            if (rows > 0) {
                float bias[ROWS + W - 1];                  // of delta0 - (ROWS - 1) on
#pragma unroll
                for (int e = 0; e < ROWS + W - 1; ++e) bias[e] = s_value[diagonal_slot<W>((uint32_t)(delta0 - (ROWS - 1) - d0 + e))];
                const bool all = delta0 - (ROWS - 1) >= lo && delta0 + W <= hi;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
#pragma unroll
                    for (int c = 0; c < W; ++c) {
                        v[r][c] += bias[ROWS - 1 - r + c];
                        if (!all && (delta0 - r + c < lo || delta0 - r + c >= hi)) v[r][c] = -__builtin_inff();
                    }
                    if (r < rows) store_piece(out + (uint32_t)(i0 + r) * a.o_row + j0, left, v[r]);
                }
            }
        }
    }
}

template <typename T, int ROWS>
static hipError_t launch_bias_rows(const BiasArgs& a, const BucketArgs& b, hipStream_t st)
{
    constexpr int W = kPiece<T>;
    const Tiling t = tiling<W, ROWS>(a.q, a.k);
    const dim3 grid(min(t.tiles, 1u << 20), min(a.planes, 65535u));
    const uint32_t slots = tile_diagonals<W, ROWS>(t);
    hipLaunchKernelGGL((k_position_bias<T, ROWS>), grid, dim3(kBiasThreads), (slots + slots / W + 1u) * sizeof(float), st, a, b);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_bias_of(const BiasArgs& a, const BucketArgs& b, hipStream_t st)
{
    return a.q < (uint32_t)kPiece<T> ? launch_bias_rows<T, 1>(a, b, st) : launch_bias_rows<T, kPiece<T>>(a, b, st);
}

hipError_t launch_position_bias(int dtype, const BiasArgs& a, const BucketArgs& b, hipStream_t st)
{
    return dtype == QGX_F32 ? launch_bias_of<float>(a, b, st) : dtype == QGX_F16 ? launch_bias_of<_Float16>(a, b, st) : launch_bias_of<__bf16>(a, b, st);
}

// ---- gradient -------------------------------------------------------------------------------------------------------------
// Block diagonal D holds the squares of queries s W .. and keys (s + D) W .., s = 0, 1, ..  A wave has 64 neighbouring ones, a lane
// each; at a step it reads W queries' runs of 64 W neighbouring keys.  (sequence, step) pairs are dealt to the waves of a band's
// workgroups in turn.
constexpr int kBackWaves = kBiasThreads / kWave;

// First block diagonal that holds a place that is not masked, and their number, of queries q and keys k (in squares).
__host__ __device__ inline void visible_diagonals(const BiasArgs& a, const BucketArgs& b, int W, int64_t* first, int64_t* count)
{
    const int64_t q = (a.q + W - 1) / W, k = (a.k + W - 1) / W;
    const int64_t lo = (int64_t)b.bounds[0] + a.q_offset, hi = (int64_t)b.bounds[b.n] - 1 + a.q_offset;       // visible j - i: lo .. hi
    // square D has j - i in D W - (W - 1) .. D W + W - 1
    auto floor_div = [](int64_t x, int64_t y) { return x >= 0 ? x / y : -((-x + y - 1) / y); };
    int64_t d0 = floor_div(lo, W), d1 = floor_div(hi + W - 1, W);
    d0 = d0 < -(q - 1) ? -(q - 1) : d0;
    d1 = d1 > k - 1 ? k - 1 : d1;
    *first = d0;
    *count = d1 >= d0 ? d1 - d0 + 1 : 0;
}

template <typename T>
__global__ __launch_bounds__(kBiasThreads) void k_position_bias_back(BiasArgs a, BucketArgs b, BiasBackPlan plan, float* __restrict__ partial)
{
    constexpr int W = kPiece<T>, E = 2 * W - 1, kSpan = kWave * W + W;
    __shared__ float s_low[kBackWaves][kWave + 1][W + 1];  // sums of the diagonals below a square's main one, and from it on
    __shared__ float s_high[kBackWaves][kWave + 1][W + 1];
    __shared__ float s_diag[kSpan];
    const uint32_t band = blockIdx.x / plan.splits, split = blockIdx.x % plan.splits;
    const int lane = lane_id(), wave = wave_id();
    const int64_t D0 = plan.first + (int64_t)band * kWave, D1 = min(D0 + kWave, plan.first + plan.count) - 1;     // of the band
    const int q_steps = (int)((a.q + W - 1u) / W), k_steps = (int)((a.k + W - 1u) / W);
    // steps at which any lane has a square
    const int s0 = (int)max((int64_t)0, -D1), s1 = (int)min((int64_t)q_steps, (int64_t)k_steps - D0), steps = max(0, s1 - s0);
    const uint64_t work = (uint64_t)steps * a.batch;
    const int64_t D = D0 + lane;
    for (uint32_t kh = blockIdx.y; kh < plan.pairs; kh += gridDim.y) {
        const uint32_t worker = kh / a.heads, head = kh % a.heads;
        const T* base = (const T*)a.in + worker * a.i_worker + head * a.i_head;
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0f;
        for (uint64_t x = (uint64_t)split * kBackWaves + wave; x < work; x += (uint64_t)plan.splits * kBackWaves) {
            const uint32_t n = (uint32_t)(x / (uint32_t)steps);
            const int s = s0 + (int)(x % (uint32_t)steps);
            const int64_t jb = s + D;                      // the square's keys
            if (D > D1 || jb < 0 || jb >= k_steps) continue;
            const int i0 = s * W, left = (int)((int64_t)a.k - jb * W), rows = min(W, (int)a.q - i0);
            const T* in = base + n * a.i_batch + (uint32_t)i0 * a.i_row + jb * W;
            float v[W][W];
#pragma unroll
            for (int r = 0; r < W; ++r) {
#pragma unroll
                for (int c = 0; c < W; ++c) v[r][c] = 0.0f;
                if (r < rows) load_piece(in + (uint32_t)r * a.i_row, left, v[r]);
            }
#pragma unroll
            for (int r = 0; r < W; ++r)
#pragma unroll
                for (int c = 0; c < W; ++c) sum[c - r + W - 1] += v[r][c];
        }
        // A diagonal of the band is that of one lane's square from its main one on and of the next lane's below it.
        __syncthreads();                                   // the pair before has been dealt with
#pragma unroll
        for (int e = 0; e < W; ++e) {
            s_high[wave][lane][e] = sum[e + W - 1];
            s_low[wave][lane][e] = e < W - 1 ? sum[e] : 0.0f;        // diagonal D W - (W - 1) + e
        }
        if (lane == 0)
#pragma unroll
            for (int e = 0; e < W; ++e) s_high[wave][kWave][e] = s_low[wave][kWave][e] = 0.0f;
        __syncthreads();
        // s_diag[x]: diagonal D0 W - W + x, x = 0 .. 64 W + W - 1
        for (int x = (int)threadIdx.x; x < kSpan; x += kBiasThreads) {
            const int l = x / W - 1, e = x % W;            // from the main diagonal of lane l's square on, below that of lane l + 1's
            float t = 0.0f;
#pragma unroll
            for (int w = 0; w < kBackWaves; ++w) {
                if (l >= 0) t += s_high[w][l][e];
                if (e > 0) t += s_low[w][l + 1][e - 1];
            }
            s_diag[x] = t;
        }
        __syncthreads();
        const int64_t first = D0 * W - W - a.q_offset;     // delta of s_diag[0]
        for (uint32_t i = (uint32_t)wave; i < b.n; i += kBackWaves) {
            const int x0 = (int)max((int64_t)0, b.bounds[i] - first), x1 = (int)min((int64_t)kSpan, b.bounds[i + 1] - first);
            float t = 0.0f;
            for (int x = x0 + lane; x < x1; x += kWave) t += s_diag[x];
            t = lanes_sum<kWave>(t);
            if (lane == 0) partial[((size_t)kh * gridDim.x + blockIdx.x) * b.n + i] = t;
        }
    }
}

// The workgroups' sums of a worker's and a head's table row joined, in binary64, a wave for each.
__global__ __launch_bounds__(kBiasThreads) void k_position_bias_join(BucketArgs b, BiasBackPlan plan, uint32_t heads, uint32_t table_rows,
                                                                     uint32_t parts, const float* __restrict__ partial, float* dtable,
                                                                     uint64_t param_stride)
{
    const uint64_t each = (uint64_t)table_rows * heads, all = plan.pairs / heads * each;
    for (uint64_t x = (uint64_t)blockIdx.x * kBackWaves + wave_id(); x < all; x += (uint64_t)gridDim.x * kBackWaves) {
        const uint32_t worker = (uint32_t)(x / each), r = (uint32_t)(x % each / heads), head = (uint32_t)(x % heads);
        const float* p = partial + ((size_t)worker * heads + head) * parts * b.n;
        double sum = 0.0;
        for (uint32_t i = 0; i < b.n; ++i) {
            if (b.rows[i] != r) continue;
            for (uint32_t u = (uint32_t)lane_id(); u < parts; u += kWave) sum += (double)p[(size_t)u * b.n + i];
        }
        sum = wave_sum(sum);
        if (lane_id() == 0) dtable[worker * param_stride + (size_t)r * heads + head] = (float)sum;
    }
}

BiasBackPlan bias_back_plan(int dtype, const BiasArgs& a, const BucketArgs& b, uint32_t workers, uint32_t n_cu)
{
    const uint32_t W = dtype == QGX_F32 ? 4u : 8u;
    BiasBackPlan p{};
    p.pairs = workers * a.heads;
    int64_t first = 0, count = 0;
    if (a.batch && a.q && a.k) visible_diagonals(a, b, (int)W, &first, &count);
    p.first = first;
    p.count = count;
    p.bands = (uint32_t)((count + kWave - 1) / kWave);
    if (!p.bands) return p;
    // four workgroups for every compute unit over pairs and bands, of at least one step to a wave
    const uint64_t work = (uint64_t)((a.q + W - 1u) / W) * a.batch, most = (work + kBackWaves - 1u) / kBackWaves;
    const uint64_t have = (uint64_t)p.pairs * p.bands, want = (4u * n_cu + have - 1u) / have;
    p.splits = (uint32_t)max((uint64_t)1u, min(want, most));
    p.scratch = (uint64_t)p.pairs * p.bands * p.splits * b.n * sizeof(float);
    return p;
}

template <typename T>
static hipError_t launch_bias_back_of(const BiasArgs& a, const BucketArgs& b, const BiasBackPlan& p, float* partial, hipStream_t st)
{
    hipLaunchKernelGGL(k_position_bias_back<T>, dim3(p.bands * p.splits, min(p.pairs, 65535u)), dim3(kBiasThreads), 0, st, a, b, p, partial);
    return hipGetLastError();
}

hipError_t launch_position_bias_back(int dtype, const BiasArgs& a, const BucketArgs& b, const BiasBackPlan& p, float* dtable, uint32_t table_rows,
                                     uint64_t param_stride, void* scratch, hipStream_t st)
{
    float* partial = (float*)scratch;
    if (p.bands) {
        const hipError_t e = dtype == QGX_F32   ? launch_bias_back_of<float>(a, b, p, partial, st)
                             : dtype == QGX_F16 ? launch_bias_back_of<_Float16>(a, b, p, partial, st)
                                                : launch_bias_back_of<__bf16>(a, b, p, partial, st);
        if (e != hipSuccess) return e;
    }
    const uint64_t outputs = (uint64_t)(p.pairs / a.heads) * table_rows * a.heads;
    hipLaunchKernelGGL(k_position_bias_join, dim3((uint32_t)min((outputs + kBackWaves - 1u) / kBackWaves, (uint64_t)1u << 20)), dim3(kBiasThreads), 0, st,
                       b, p, a.heads, table_rows, p.bands * p.splits, partial, dtable, param_stride);
    return hipGetLastError();
}

}  // namespace qgx
