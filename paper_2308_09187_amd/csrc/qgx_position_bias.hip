// Learned relative position bias by buckets, out = scores + table[row(j - i - p)][head], and the table's gradient.
// Both go by squares of W queries x W keys (W: the elements of 16 bytes): a thread has 2 W - 1 diagonals in registers at places
// that the compiler knows (key - query within the square), and the squares on one block diagonal all have the same ones.
//   forward: a square's 2 W - 1 biases come from a list of the tile's diagonals in LDS, then serve W pieces of 16 bytes;
//   gradient: a thread walks down a block diagonal, its sums of 2 W - 1 diagonals in registers over all queries and sequences, and only at its
//     end are they sorted into the buckets, which are runs of diagonals.  No element meets a bucket, an atomic or a search.
// Both are bound by memory.  8 x 16 x 1024 x 1024 bfloat16: forward, 537 MB, 82 us, 6.5 TB/s (95 with its memory out of the cache);
// gradient, 268 MB, 53 us, 5.1 TB/s; 64 x 16 x 197 x 197 28 us, 2.8 TB/s.
#include "qgx_types.h"
#include "qgx_plan.h"

namespace qgx {

constexpr int kBiasThreads = 256, kBiasWaves = kBiasThreads / kWave;

// p of a sequence, kept within +-2^30 so that a delta fits 32 bits.
__device__ __forceinline__ int position_of(const BiasArgs& a, uint32_t seq)
{
    const int64_t p = a.q_offset + (a.positions ? (int64_t)a.positions[seq] : 0);
    return (int)max((int64_t)-(1 << 30), min(p, (int64_t)(1 << 30)));
}

// The intervals in a wave's registers, i and i + 64 in lane i (past the last: it again).
struct Intervals {
    int bound0, bound1, end0, end1;
    uint32_t row0, row1;
    bool is0, is1, more;                                   // there is one; more than 64 in all
    __device__ __forceinline__ explicit Intervals(const BucketArgs& b)
    {
        const uint32_t i = (uint32_t)lane_id(), i0 = min(i, b.n - 1u);
        bound0 = b.bounds[i0]; end0 = b.bounds[i0 + 1u]; row0 = b.rows[i0]; is0 = i < b.n;
        bound1 = bound0; end1 = end0; row1 = row0; is1 = i + kWave < b.n; more = b.n > (uint32_t)kWave;
        if (more) {
            const uint32_t i1 = min(i + kWave, b.n - 1u);
            bound1 = b.bounds[i1]; end1 = b.bounds[i1 + 1u]; row1 = b.rows[i1];
        }
    }
    // x0 of lane i, or x1 of lane i - 64.  (Every lane has to be here, as for any exchange between lanes.)
    template <typename X>
    __device__ __forceinline__ X lookup(int i, X x0, X x1) const
    {
        const int y0 = __builtin_amdgcn_ds_bpermute(i * 4, __builtin_bit_cast(int, x0));
        if (!more) return __builtin_bit_cast(X, y0);
        const int y1 = __builtin_amdgcn_ds_bpermute(i * 4, __builtin_bit_cast(int, x1));      // (the lane's number counts modulo 64)
        return __builtin_bit_cast(X, i < kWave ? y0 : y1);
    }
    // The last interval that starts at delta or before, 0 where none does: a binary search through the lanes.
    __device__ __forceinline__ int at(int delta) const
    {
        int i = more && __builtin_amdgcn_readfirstlane(bound1) <= delta ? kWave : 0;
#pragma unroll
        for (int step = kWave / 2; step > 0; step /= 2)
            if (lookup(i + step, bound0, bound1) <= delta) i += step;
        return i;
    }
    __device__ __forceinline__ int number(int first, int end) const
    {
        return __popcll(__ballot(is0 && bound0 < end && end0 > first)) + __popcll(__ballot(is1 && bound1 < end && end1 > first));
    }
    // f(i, j, x0, x1) for every interval that meets first .. end: i its number, j its lane's, x0 .. x1 what it has of that run
    template <typename F>
    __device__ __forceinline__ void meeting(int first, int end, F f) const
    {
        for (uint64_t which = __ballot(is0 && bound0 < end && end0 > first); which; which &= which - 1u) {
            const int j = __ffsll((unsigned long long)which) - 1;
            f(j, j, max(__builtin_amdgcn_readlane(bound0, j), first), min(__builtin_amdgcn_readlane(end0, j), end));
        }
        for (uint64_t which = __ballot(is1 && bound1 < end && end1 > first); which; which &= which - 1u) {
            const int j = __ffsll((unsigned long long)which) - 1;
            f(j + kWave, j, max(__builtin_amdgcn_readlane(bound1, j), first), min(__builtin_amdgcn_readlane(end1, j), end));
        }
    }
};

// ---- forward --------------------------------------------------------------------------------------------------------------
// Squares have ROWS queries (W, or one where there are fewer than W), a band is ROWS queries' squares.  A wave takes up to 64
// neighbouring squares of a band, or whole bands where they have few squares, a lane each.  It lists its diagonals' biases in LDS of its own
// (one or two intervals in most places): no barrier, and the scores' loads are under way meanwhile.  The last squares of a band and the last
// band are moved back to end with the keys and queries, so that every access is whole: what two squares have in common they
// write twice, the same bits.
struct Tiling {
    uint32_t per_band, bands;                              // squares of a band; bands
    uint32_t chunks, chunk;                                // waves that share a band, squares of each; or
    uint32_t bands_each;                                   // bands of a wave (chunks is 1)
    uint32_t inverse;                                      // 65536 / chunk and one, for the lanes' division: lane and chunk are at most 64
    uint32_t tasks;                                        // (below 2^26: q k is at most 2^34)
};

template <int W, int ROWS>
static Tiling tiling(uint32_t q, uint32_t k)
{
    Tiling t{};
    t.per_band = (k + W - 1u) / W;
    t.bands = (q + ROWS - 1u) / ROWS;
    t.chunks = (t.per_band + kWave - 1u) / kWave;
    t.chunk = (t.per_band + t.chunks - 1u) / t.chunks;
    t.bands_each = t.chunks == 1u ? kWave / t.per_band : 1u;
    t.inverse = 65536u / t.chunk + 1u;
    t.tasks = (t.bands + t.bands_each - 1u) / t.bands_each * t.chunks;
    return t;
}

// The most diagonals of a wave: chunk W + bands_each ROWS - 1, and chunk bands_each is at most 64.
constexpr int wave_diagonals(int W) { return 65 * W; }
// One word is left out after every W, so that lanes W entries apart do not meet in a bank.
template <int W> __device__ __forceinline__ uint32_t diagonal_slot(uint32_t x) { return x + x / W; }

constexpr int kFewIntervals = 6;

// GUARDED: squares with something in common write it once.  In place a square's scores may otherwise have been overwritten by the
// one it overlaps before they are read.
template <typename T, int ROWS, bool GUARDED>
__global__ __launch_bounds__(kBiasThreads) void k_position_bias(BiasArgs a, BucketArgs b, Tiling t)
{
    constexpr int W = kPiece<T>;
    __shared__ float s_list[kBiasWaves][wave_diagonals(W) / W * (W + 1)];
    float* list = s_list[wave_id()];
    const uint32_t task = blockIdx.x * kBiasWaves + (uint32_t)__builtin_amdgcn_readfirstlane(wave_id()), plane = blockIdx.z * gridDim.y + blockIdx.y;
    if (task >= t.tasks || plane >= a.planes) return;
    const int lane = lane_id(), q = (int)a.q, k = (int)a.k, lo = b.bounds[0], hi = b.bounds[b.n];
    const uint32_t head = plane % a.heads, seq = plane / a.heads, worker = seq / a.batch, n = seq % a.batch;
    // All intervals' biases at once and first: one after the other, or after the scores, they would be the longest wait there is.
    const Intervals interval(b);
    const float value0 = a.table[(size_t)interval.row0 * a.heads + head], value1 = a.table[(size_t)interval.row1 * a.heads + head];
    const uint32_t group = task / t.chunks, band0 = group * t.bands_each, first = (task - group * t.chunks) * t.chunk;
    const uint32_t end = min(first + t.chunk, t.per_band), band1 = min(band0 + t.bands_each, t.bands);
    const uint32_t mine = ((uint32_t)lane * t.inverse) >> 16, band = band0 + mine, square = first + (uint32_t)lane - mine * t.chunk;
    const bool any = band < band1 && square < end;
    const int i_at = (int)band * ROWS, j_at = (int)square * W;         // before they are moved back
    const int i0 = min(i_at, q - ROWS), j0 = min(j_at, k - W);
    const int p = position_of(a, seq), delta0 = j0 - i0 - p;           // of the first query and key

    float v[ROWS][W];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < W; ++c) v[r][c] = 0.0f;
    // (a square that is masked as a whole is not read)
    if (a.in && any && delta0 + W > lo && delta0 - (ROWS - 1) < hi) {
        const T* in = (const T*)a.in + worker * a.i_worker + n * a.i_batch + head * a.i_head + (uint32_t)i0 * a.i_row + j0;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) load_piece(in + (uint32_t)r * a.i_row, v[r]);
    }

    // deltas of the wave: d0 .. d1
    const int d0 = min((int)(first * W), k - W) - (min((int)(band1 * ROWS), q) - 1) - p;
    const int d1 = min((int)(end * W), k) - min((int)(band0 * ROWS), q - ROWS) - p;
    // Three in four waves of long rows meet one interval or two; where there are many (they take 0.1 us each), every diagonal is searched for.
    if (interval.number(d0, d1) <= kFewIntervals) {
        interval.meeting(d0, d1, [&](int i, int j, int x0, int x1) {
            const float value = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(i < kWave ? value0 : value1), j));
            for (int x = x0 + lane; x < x1; x += kWave) list[diagonal_slot<W>((uint32_t)(x - d0))] = value;
        });
    } else {
        for (int x0 = 0; x0 < d1 - d0; x0 += kWave) {
            const float value = interval.lookup(interval.at(d0 + x0 + lane), value0, value1);
            if (x0 + lane < d1 - d0) list[diagonal_slot<W>((uint32_t)(x0 + lane))] = value;
        }
    }
    wave_lds_fence();
    if (!any) return;
    float bias[ROWS + W - 1];                              // of delta0 - (ROWS - 1) on
    bool seen[ROWS + W - 1];
#pragma unroll
    for (int e = 0; e < ROWS + W - 1; ++e) {
        const int delta = delta0 - (ROWS - 1) + e;
        bias[e] = list[diagonal_slot<W>((uint32_t)(delta - d0))];      // (of a masked one: anything, and not used)
        seen[e] = delta >= lo && delta < hi;
    }
    T* out = (T*)a.out + worker * a.o_worker + n * a.o_batch + head * a.o_head + (uint32_t)i0 * a.o_row + j0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int c = 0; c < W; ++c) v[r][c] = seen[ROWS - 1 - r + c] ? v[r][c] + bias[ROWS - 1 - r + c] : -__builtin_inff();
        if constexpr (!GUARDED) {
            stream_piece(out + (uint32_t)r * a.o_row, v[r]);       // (8 x 16 x 1024 x 1024 bfloat16: 99 us with plain stores, 82; loads so marked lose on odd rows)
        } else if (i0 + r >= i_at) {
            if (j0 == j_at) store_piece(out + (uint32_t)r * a.o_row, v[r]);
            else
#pragma unroll
                for (int c = 0; c < W; ++c)
                    if (j0 + c >= j_at) out[(uint32_t)r * a.o_row + c] = (T)v[r][c];
        }
    }
}

// Fewer queries than a square has, and a row of 64 pieces or more: the form for single tokens.  A wave takes up to kTokenRuns runs of 64
// neighbouring pieces of a query's row, all its loads under way at once.  Most runs lie in one interval, whose bias every lane then has; in
// the others a lane looks up its piece's, and only where a piece crosses a bound every element's.  64 x 16 x 1 x 32768 bfloat16, 134 MB:
// 24 us, 5.6 TB/s (39 as squares of one query, through the list); 32 x 16 x 1 x 4099 8 us by either way, most of it the first loads' wait.
constexpr int kTokenRuns = 4;

template <typename T, bool GUARDED>
__global__ __launch_bounds__(kBiasThreads) void k_position_bias_token(BiasArgs a, BucketArgs b, uint32_t runs, uint32_t each)
{
    constexpr int W = kPiece<T>;
    const uint32_t chunks = (runs + each - 1u) / each, task = blockIdx.x * kBiasWaves + (uint32_t)__builtin_amdgcn_readfirstlane(wave_id());
    const uint32_t plane = blockIdx.z * gridDim.y + blockIdx.y;
    if (task >= chunks * a.q || plane >= a.planes) return;
    const int lane = lane_id(), k = (int)a.k, lo = b.bounds[0], hi = b.bounds[b.n];
    const uint32_t head = plane % a.heads, seq = plane / a.heads, worker = seq / a.batch, n = seq % a.batch;
    const Intervals interval(b);
    const float value0 = a.table[(size_t)interval.row0 * a.heads + head], value1 = a.table[(size_t)interval.row1 * a.heads + head];
    const uint32_t i = task / chunks, run0 = (task - i * chunks) * each;
    const int at_query = (int)i + position_of(a, seq), n_runs = (int)min(each, runs - run0);
    const T* in = a.in ? (const T*)a.in + worker * a.i_worker + n * a.i_batch + head * a.i_head + i * a.i_row : nullptr;
    T* out = (T*)a.out + worker * a.o_worker + n * a.o_batch + head * a.o_head + i * a.o_row;
    nt_u32x4 raw[kTokenRuns];
    int j_at[kTokenRuns], j0[kTokenRuns];                  // a lane's piece, and moved back to end with the keys
#pragma unroll
    for (int m = 0; m < kTokenRuns; ++m) {
        j_at[m] = (int)((run0 + m) * kWave + lane) * W;
        j0[m] = min(j_at[m], k - W);
        const int delta = j0[m] - at_query;
        raw[m] = nt_u32x4{0u, 0u, 0u, 0u};
        // (a piece that is masked as a whole is not read)
        if (in && m < n_runs && j_at[m] < k && delta + W > lo && delta < hi) raw[m] = load_bits(in + j0[m]);
    }
#pragma unroll
    for (int m = 0; m < kTokenRuns; ++m) {
        if (m >= n_runs) break;
        const int delta = j0[m] - at_query;
        const int d0 = min((int)((run0 + m) * kWave) * W, k - W) - at_query, d1 = min((int)((run0 + m + 1) * kWave) * W, k) - at_query;
        float v[W], bias[W];
        values_of<T>(raw[m], v);
        const uint64_t in0 = __ballot(interval.is0 && interval.bound0 < d1 && interval.end0 > d0), in1 = __ballot(interval.is1 && interval.bound1 < d1 && interval.end1 > d0);
        if (__popcll(in0) + __popcll(in1) <= 1) {
            const float one = __int_as_float(in0 ? __builtin_amdgcn_readlane(__float_as_int(value0), __ffsll((unsigned long long)in0) - 1)
                                             : in1 ? __builtin_amdgcn_readlane(__float_as_int(value1), __ffsll((unsigned long long)in1) - 1) : 0);
#pragma unroll
            for (int c = 0; c < W; ++c) bias[c] = one;
        } else {
            const int mine = interval.at(delta), stop = interval.lookup(mine, interval.end0, interval.end1);
            const float own = interval.lookup(mine, value0, value1);
            // (a piece before the first bound has its first elements masked, and the others belong to the first interval or later ones)
            if (__ballot(delta + W > stop || delta < lo) == 0) {
#pragma unroll
                for (int c = 0; c < W; ++c) bias[c] = own;
            } else {
#pragma unroll
                for (int c = 0; c < W; ++c) bias[c] = interval.lookup(interval.at(delta + c), value0, value1);
            }
        }
#pragma unroll
        for (int c = 0; c < W; ++c) v[c] = delta + c >= lo && delta + c < hi ? v[c] + bias[c] : -__builtin_inff();
        if (j_at[m] >= k) continue;
        if (!GUARDED || j0[m] == j_at[m]) {
            if constexpr (GUARDED) store_piece(out + j0[m], v);
            else stream_piece(out + j0[m], v);
        } else {
#pragma unroll
            for (int c = 0; c < W; ++c)
                if (j0[m] + c >= j_at[m]) out[j0[m] + c] = (T)v[c];
        }
    }
}

// Fewer keys than a piece has elements: a thread for each query.
template <typename T>
__global__ __launch_bounds__(kBiasThreads) void k_position_bias_narrow(BiasArgs a, BucketArgs b)
{
    const uint32_t i = blockIdx.x * kBiasThreads + threadIdx.x, plane = blockIdx.z * gridDim.y + blockIdx.y;
    if (i >= a.q || plane >= a.planes) return;
    const uint32_t head = plane % a.heads, seq = plane / a.heads, worker = seq / a.batch, n = seq % a.batch;
    const int p = position_of(a, seq);
    for (uint32_t j = 0; j < a.k; ++j) {
        const int delta = (int)j - (int)i - p;
        float x = -__builtin_inff();
        for (uint32_t s = 0; s < b.n; ++s)
            if (delta >= b.bounds[s] && delta < b.bounds[s + 1]) {
                x = a.table[(size_t)b.rows[s] * a.heads + head];
                if (a.in) x += (float)((const T*)a.in + worker * a.i_worker + n * a.i_batch + head * a.i_head + i * a.i_row)[j];
            }
        ((T*)a.out + worker * a.o_worker + n * a.o_batch + head * a.o_head + i * a.o_row)[j] = (T)x;
    }
}

// Planes over two dimensions of a grid.
static dim3 plane_grid(uint32_t blocks, uint32_t planes)
{
    const uint32_t y = min(planes, 65535u);
    return dim3(blocks, y, (planes + y - 1u) / y);
}

template <typename T, int ROWS>
static hipError_t launch_bias_rows(const BiasArgs& a, const BucketArgs& b, hipStream_t st)
{
    const Tiling t = tiling<kPiece<T>, ROWS>(a.q, a.k);
    const dim3 grid = plane_grid((t.tasks + kBiasWaves - 1u) / kBiasWaves, a.planes);
    const bool overlap = a.q % ROWS != 0u || a.k % kPiece<T> != 0u;
    if (a.in == a.out && overlap) hipLaunchKernelGGL((k_position_bias<T, ROWS, true>), grid, dim3(kBiasThreads), 0, st, a, b, t);
    else hipLaunchKernelGGL((k_position_bias<T, ROWS, false>), grid, dim3(kBiasThreads), 0, st, a, b, t);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_bias_token(const BiasArgs& a, const BucketArgs& b, uint32_t n_cu, hipStream_t st)
{
    constexpr uint32_t W = kPiece<T>;
    const uint32_t pieces = (a.k + W - 1u) / W, runs = (pieces + kWave - 1u) / kWave;
    // as many runs to a wave as leave sixteen waves for every compute unit
    const uint64_t waves = (uint64_t)runs * a.q * a.planes;
    const uint32_t most = (uint32_t)max((uint64_t)1u, min((uint64_t)kTokenRuns, waves / (16u * n_cu)));
    const uint32_t chunks = (runs + most - 1u) / most, each = (runs + chunks - 1u) / chunks, used = (runs + each - 1u) / each;
    const dim3 grid = plane_grid((used * a.q + kBiasWaves - 1u) / kBiasWaves, a.planes);
    if (a.in == a.out && a.k % W != 0u) hipLaunchKernelGGL((k_position_bias_token<T, true>), grid, dim3(kBiasThreads), 0, st, a, b, runs, each);
    else hipLaunchKernelGGL((k_position_bias_token<T, false>), grid, dim3(kBiasThreads), 0, st, a, b, runs, each);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_bias_of(const BiasArgs& a, const BucketArgs& b, uint32_t n_cu, hipStream_t st)
{
    if (a.k < (uint32_t)kPiece<T>) {
        hipLaunchKernelGGL(k_position_bias_narrow<T>, plane_grid((a.q + kBiasThreads - 1u) / kBiasThreads, a.planes), dim3(kBiasThreads), 0, st, a, b);
        return hipGetLastError();
    }
    if (a.q >= (uint32_t)kPiece<T>) return launch_bias_rows<T, kPiece<T>>(a, b, st);
    return a.k >= (uint32_t)kWave * kPiece<T> ? launch_bias_token<T>(a, b, n_cu, st) : launch_bias_rows<T, 1>(a, b, st);
}

hipError_t launch_position_bias(int dtype, const BiasArgs& a, const BucketArgs& b, uint32_t n_cu, hipStream_t st)
{
    return dtype == QGX_F32   ? launch_bias_of<float>(a, b, n_cu, st)
           : dtype == QGX_F16 ? launch_bias_of<_Float16>(a, b, n_cu, st)
                              : launch_bias_of<__bf16>(a, b, n_cu, st);
}

// ---- gradient -------------------------------------------------------------------------------------------------------------
// Block diagonal D holds the squares of queries s W .. and keys (s + D) W .., s = 0, 1, ..  A band is BAND neighbouring ones, a lane each;
// at a step the lanes of a band read W queries' runs of BAND W neighbouring keys.  A band's items are its steps in all sequences,
// dealt in turn to the groups of BAND lanes of its workgroups; bands get workgroups by their items, for the corner
// bands of a square of queries and keys have few.

// The first and the number of the block diagonals that hold a place that is not masked.
static void visible_diagonals(const BiasArgs& a, const BucketArgs& b, int W, int64_t* first, int64_t* count)
{
    const int64_t q = ((int64_t)a.q + W - 1) / W, k = ((int64_t)a.k + W - 1) / W;
    const int64_t lo = (int64_t)b.bounds[0] + a.q_offset, hi = (int64_t)b.bounds[b.n] - 1 + a.q_offset;       // visible j - i: lo .. hi
    // square D has j - i in D W - (W - 1) .. D W + W - 1
    auto floor_div = [](int64_t x, int64_t y) { return x >= 0 ? x / y : -((-x + y - 1) / y); };
    const int64_t d0 = max(floor_div(lo, W), -(q - 1)), d1 = min(floor_div(hi + W - 1, W), k - 1);
    *first = d0;
    *count = d1 >= d0 ? d1 - d0 + 1 : 0;
}

// Steps at which a band has a square: s0 .. s1.
struct BandSteps { int s0, s1; };
__host__ __device__ inline BandSteps band_steps(int64_t D0, int64_t D1, int q_steps, int k_steps)
{
    const int64_t s0 = D1 < 0 ? -D1 : 0, s1 = k_steps - D0 < q_steps ? k_steps - D0 : q_steps;
    return BandSteps{(int)s0, (int)(s1 > s0 ? s1 : s0)};
}

// The last n elements of a piece, moved to its front, and zeros after them.
template <typename T>
__device__ __forceinline__ nt_u32x4 last_elements(nt_u32x4 x, int n)
{
    uint64_t lo = x.x | (uint64_t)x.y << 32, hi = x.z | (uint64_t)x.w << 32;
    const int bits = (kPiece<T> - n) * 8 * (int)sizeof(T);     // 0, 16 or 32 .. 112
    if (bits >= 64) {
        lo = hi >> (bits - 64);
        hi = 0;
    } else if (bits) {
        lo = lo >> bits | hi << (64 - bits);
        hi >>= bits;
    }
    return nt_u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// A square as loaded: the rows that it has (none where there is no square), and its keys' number.
template <int ROWS> struct Square {
    nt_u32x4 row[ROWS];
    int rows, keys;
};

constexpr int kShort = 16;                                 // diagonals of an interval that a lane adds up

// ROWS: W, or 1 where there is one query (64 x 16 x 1 x 32768 bfloat16 51 us with W, 23).  NARROW: fewer keys than a piece has elements.
template <typename T, int BAND, int ROWS, bool NARROW>
__global__ __launch_bounds__(kBiasThreads) void k_position_bias_back(BiasArgs a, BucketArgs b, BiasBackPlan plan, float* __restrict__ partial)
{
    constexpr int W = kPiece<T>, E = 2 * W - 1, kSpan = BAND * W + W, kGroups = kBiasThreads / BAND;
    __shared__ float s_low[kBiasWaves][BAND + 1][W + 1];  // sums of the diagonals below a square's main one, and from it on
    __shared__ float s_high[kBiasWaves][BAND + 1][W + 1];
    __shared__ float s_diag[kSpan];
    __shared__ float s_out[QGX_MAX_INTERVALS];
    const int lane = lane_id(), wave = wave_id();
    // this workgroup's band, its place among the band's and their number
    uint32_t band, split, splits;
    if (plan.even) {
        band = blockIdx.x / plan.even;
        split = blockIdx.x % plan.even;
        splits = plan.even;
    } else {
        // first_block ascends, and every band has a workgroup
        const uint32_t i0 = (uint32_t)lane < plan.bands ? plan.first_block[lane] : 0xFFFFFFFFu;
        const uint32_t i1 = (uint32_t)lane + kWave < plan.bands ? plan.first_block[lane + kWave] : 0xFFFFFFFFu;
        band = (uint32_t)(__popcll(__ballot(i0 <= blockIdx.x)) + __popcll(__ballot(i1 <= blockIdx.x))) - 1u;
        split = blockIdx.x - plan.first_block[band];
        splits = plan.first_block[band + 1u] - plan.first_block[band];
    }
    const int64_t D0 = plan.first + (int64_t)band * BAND, D1 = min(D0 + BAND, plan.first + plan.count) - 1, D = D0 + lane % BAND;
    const int q_steps = (int)((a.q + W - 1u) / W), k_steps = (int)((a.k + W - 1u) / W);
    const BandSteps at = band_steps(D0, D1, q_steps, k_steps);
    const uint32_t steps = (uint32_t)(at.s1 - at.s0);
    const uint64_t items = (uint64_t)steps * a.batch;
    const Intervals interval(b);
    for (uint32_t kh = blockIdx.y; kh < plan.pairs; kh += gridDim.y) {
        const uint32_t worker = kh / a.heads, head = kh % a.heads;
        const T* base = (const T*)a.in + worker * a.i_worker + head * a.i_head;
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0f;
        // this group's first item: sequence n, step s; and from one item to its next
        const uint32_t x0 = split * kGroups + threadIdx.x / BAND, hop = splits * kGroups;
        uint32_t n = steps ? x0 / steps : a.batch, s = steps ? x0 % steps : 0u;
        const uint32_t hop_n = steps ? hop / steps : 0u, hop_s = steps ? hop % steps : 0u;
        // Two squares' loads are under way at a time (64 x 16 x 197 x 197 bfloat16 39 us with one, 28; 8 x 16 x 1024 x 1024 53 either way).
        // Every lane loads W pieces whether it has a square or not (a neighbour's then), for a wait for the square before has to know how
        // many loads came after it.
        auto load = [&](Square<ROWS>& x) {
            const int64_t jb = (int64_t)at.s0 + s + D;     // the square's keys
            const bool any = n < a.batch && D <= D1 && jb >= 0 && jb < k_steps;
            const uint32_t i0 = ((uint32_t)at.s0 + s) * W, j0 = (uint32_t)max((int64_t)0, min(jb - max(D - D1, (int64_t)0), (int64_t)k_steps - 1)) * W;
            const T* in = base + min(n, a.batch - 1u) * a.i_batch + i0 * a.i_row;
            x.rows = any ? (int)min((uint32_t)ROWS, a.q - i0) : 0;
            x.keys = (int)min((uint32_t)W, a.k - j0);
            if constexpr (NARROW) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
                    x.row[r] = __builtin_bit_cast(nt_u32x4, load_raw(in + min((uint32_t)r, a.q - 1u - i0) * a.i_row, x.keys));
            } else {
                in += j0 - (uint32_t)(W - x.keys);         // (moved back to end with its row)
                if (__ballot(i0 + ROWS > a.q) == 0) {
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) x.row[r] = load_bits(in + (uint32_t)r * a.i_row);
                } else {
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) x.row[r] = load_bits(in + min((uint32_t)r, a.q - 1u - i0) * a.i_row);
                }
            }
            n += hop_n;
            s += hop_s;
            if (s >= steps) { s -= steps; ++n; }
        };
        auto add = [&](Square<ROWS>& x) {
            if (__ballot(x.rows < ROWS || x.keys < W) != 0)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    if (!NARROW) x.row[r] = last_elements<T>(x.row[r], x.keys);
                    if (r >= x.rows) x.row[r] = nt_u32x4{0u, 0u, 0u, 0u};
                }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float v[W];
                values_of<T>(x.row[r], v);
#pragma unroll
                for (int c = 0; c < W; ++c) sum[c - r + W - 1] += v[c];
            }
        };
        // (the same number of turns for the whole workgroup: a group without an item any more has squares of no rows)
        const uint64_t before = (uint64_t)split * kGroups;
        uint64_t turns = items > before ? (items - before + hop - 1u) / hop : 0u;
        if (turns) {
            Square<ROWS> even, odd;
            load(even);
            for (;; turns -= 2u) {
                if (turns == 1u) { add(even); break; }
                load(odd);
                add(even);
                if (turns == 2u) { add(odd); break; }
                load(even);
                add(odd);
            }
        }
        // the wave's groups joined, then a diagonal of the band is that of one lane's square from its main one on and of the next
        // lane's below it
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (BAND <= 32) {
                const LanePair o = lane_pair<32>(__float_as_uint(sum[e]));
                sum[e] = __uint_as_float(o.a) + __uint_as_float(o.b);
            }
            if constexpr (BAND <= 16) {
                const LanePair o = lane_pair<16>(__float_as_uint(sum[e]));
                sum[e] = __uint_as_float(o.a) + __uint_as_float(o.b);
            }
        }
        __syncthreads();                                   // the pair before has been dealt with
        if (lane < BAND) {
#pragma unroll
            for (int e = 0; e < W; ++e) {
                s_high[wave][lane][e] = sum[e + W - 1];
                s_low[wave][lane][e] = e < W - 1 ? sum[e] : 0.0f;          // diagonal D W - (W - 1) + e
            }
        }
        if (lane < W) s_high[wave][BAND][lane] = s_low[wave][BAND][lane] = 0.0f;
        __syncthreads();
        // s_diag[x]: diagonal D0 W - W + x
        for (int y = (int)threadIdx.x; y < kSpan; y += kBiasThreads) {
            const int l = y / W - 1, e = y % W;            // from the main diagonal of lane l's square on, below that of lane l + 1's
            float z = 0.0f;
#pragma unroll
            for (int w = 0; w < kBiasWaves; ++w) {
                if (l >= 0) z += s_high[w][l][e];
                if (e > 0) z += s_low[w][l + 1][e - 1];
            }
            s_diag[y] = z;
        }
        __syncthreads();
        const int first = (int)(D0 * W - W - a.q_offset);  // delta of s_diag[0]
        // Short intervals, most near the diagonal, by a lane each (the first 64 in wave 0, the others in wave 1); the long ones by a
        // wave each in turn.  (All of them by waves, one after the other, take 0.1 us each.)
        int turn = 0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int bound = half ? interval.bound1 : interval.bound0, stop = half ? interval.end1 : interval.end0;
            const BandPart part = band_part(bound, stop, first, kSpan);
            const int y0 = part.at, n = (half ? interval.is1 : interval.is0) ? part.n : 0;
            if (wave == half && n <= kShort) {
                float z = 0.0f;
#pragma unroll
                for (int y = 0; y < kShort; ++y)
                    if (y < n) z += s_diag[y0 + y];
                s_out[half * kWave + lane] = z;
            }
            for (uint64_t which = __ballot(n > kShort); which; which &= which - 1u, ++turn) {
                if (turn % kBiasWaves != wave) continue;
                const int j = __ffsll((unsigned long long)which) - 1, from = __builtin_amdgcn_readlane(y0, j), to = from + __builtin_amdgcn_readlane(n, j);
                float z = 0.0f;
                for (int y = from + lane; y < to; y += kWave) z += s_diag[y];
                z = lanes_sum<kWave>(z);
                if (lane == 0) s_out[half * kWave + j] = z;
            }
        }
        __syncthreads();
        if (threadIdx.x < b.n) partial[((size_t)kh * gridDim.x + blockIdx.x) * b.n + threadIdx.x] = s_out[threadIdx.x];
    }
}

// The workgroups' sums of a worker's and a head's table row joined, in binary64, a wave for each.
__global__ __launch_bounds__(kBiasThreads) void k_position_bias_join(BucketArgs b, uint32_t heads, uint32_t table_rows,
                                                                     uint32_t parts, const float* __restrict__ partial, float* dtable,
                                                                     uint64_t param_stride)
{
    const Intervals interval(b);
    const uint32_t worker = blockIdx.y, outputs = table_rows * heads;
    for (uint32_t x = blockIdx.x * kBiasWaves + (uint32_t)__builtin_amdgcn_readfirstlane(wave_id()); x < outputs; x += gridDim.x * kBiasWaves) {
        const uint32_t r = x / heads, head = x - r * heads;
        const float* p = partial + ((size_t)worker * heads + head) * parts * b.n;
        double sum = 0.0;
        for (int half = 0; half < 2; ++half)
            for (uint64_t which = __ballot(half ? interval.is1 && interval.row1 == r : interval.is0 && interval.row0 == r); which; which &= which - 1u) {
                const uint32_t i = (uint32_t)(half * kWave + __ffsll((unsigned long long)which) - 1);
                for (uint32_t u = (uint32_t)lane_id(); u < parts; u += kWave) sum += (double)p[(size_t)u * b.n + i];
            }
        sum = wave_sum(sum);
        if (lane_id() == 0) dtable[worker * param_stride + (size_t)r * heads + head] = (float)sum;
    }
}

// The lanes of a band.
static uint32_t back_band(uint32_t k, int W) { return (k + W - 1u) / W >= 64u ? 64u : 16u; }

BiasBackPlan bias_back_plan(int dtype, const BiasArgs& a, const BucketArgs& b, uint32_t workers, uint32_t n_cu)
{
    const int W = dtype == QGX_F32 ? 4 : 8;
    BiasBackPlan p{};
    p.pairs = workers * a.heads;
    if (a.batch && a.q && a.k) visible_diagonals(a, b, W, &p.first, &p.count);
    p.band = back_band(a.k, W);
    const int64_t band = p.band;
    const uint32_t groups = kBiasThreads / p.band;
    p.bands = (uint32_t)((p.count + band - 1) / band);
    if (!p.bands) return p;
    const int q_steps = (int)((a.q + W - 1u) / W), k_steps = (int)((a.k + W - 1u) / W);
    // Workgroups of a pair: six for every compute unit over all pairs and bands while a group of lanes has four items then, and not below three,
    // which is what a compute unit holds at once (4 x 3 x 4 x 1019 x 1019 bfloat16 27 us with six, 25 with three; 8 x 16 x 1024 x 1024 53 and 55).
    const uint64_t want = max((uint64_t)1u, (6u * (uint64_t)n_cu + p.pairs - 1u) / p.pairs), least = max((uint64_t)1u, (3u * (uint64_t)n_cu + p.pairs - 1u) / p.pairs);
    if (p.bands > kMaxBands) {
        const uint64_t most = ((uint64_t)q_steps * a.batch + groups - 1u) / groups;
        p.even = (uint32_t)min((want + p.bands - 1u) / p.bands, most);
        p.blocks = p.bands * p.even;
    } else {
        uint64_t items[kMaxBands], all = 0;
        for (uint32_t i = 0; i < p.bands; ++i) {
            const int64_t D0 = p.first + (int64_t)i * band, D1 = min(D0 + band, p.first + p.count) - 1;
            const BandSteps s = band_steps(D0, D1, q_steps, k_steps);
            all += items[i] = (uint64_t)(s.s1 - s.s0) * a.batch;
        }
        // items of a workgroup
        const uint64_t each = max((uint64_t)groups, max((all + want - 1u) / want, min((uint64_t)groups * 4u, (all + least - 1u) / least)));
        for (uint32_t i = 0; i < p.bands; ++i) {
            p.first_block[i] = p.blocks;
            p.blocks += (uint32_t)max((uint64_t)1u, (items[i] + each - 1u) / each);
        }
        p.first_block[p.bands] = p.blocks;
    }
    p.scratch = (uint64_t)p.pairs * p.blocks * b.n * sizeof(float);
    return p;
}

template <typename T>
static hipError_t launch_bias_back_of(const BiasArgs& a, const BucketArgs& b, const BiasBackPlan& p, float* partial, hipStream_t st)
{
    const dim3 grid(p.blocks, min(p.pairs, 65535u));
    constexpr int W = kPiece<T>;
    if (a.k < (uint32_t)W) hipLaunchKernelGGL((k_position_bias_back<T, 16, W, true>), grid, dim3(kBiasThreads), 0, st, a, b, p, partial);
    else if (a.q == 1u && p.band == 64u) hipLaunchKernelGGL((k_position_bias_back<T, 64, 1, false>), grid, dim3(kBiasThreads), 0, st, a, b, p, partial);
    else if (a.q == 1u) hipLaunchKernelGGL((k_position_bias_back<T, 16, 1, false>), grid, dim3(kBiasThreads), 0, st, a, b, p, partial);
    else if (p.band == 64u) hipLaunchKernelGGL((k_position_bias_back<T, 64, W, false>), grid, dim3(kBiasThreads), 0, st, a, b, p, partial);
    else hipLaunchKernelGGL((k_position_bias_back<T, 16, W, false>), grid, dim3(kBiasThreads), 0, st, a, b, p, partial);
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
    const uint32_t outputs = table_rows * a.heads;         // (below 2^24)
    hipLaunchKernelGGL(k_position_bias_join, dim3((outputs + kBiasWaves - 1u) / kBiasWaves, p.pairs / a.heads), dim3(kBiasThreads), 0, st, b, a.heads,
                       table_rows, p.blocks, partial, dtable, param_stride);
    return hipGetLastError();
}

}  // namespace qgx
