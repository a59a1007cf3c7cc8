// Each worker's global gradient norm over its many tensors, and clipping, gathered into the dual vectors or in place.
//   N_k = (sum over tensors and elements x^2)^(1/2), or max |x|;   c_k = N_k > M ? M / N_k : 1;   V[k][offset + i] = c_k x_i
// A launch that reads everything once and leaves a sum per workgroup, one workgroup per worker that adds those up and leaves the
// factor, and a launch that scales; where a worker's sums are few every scaling wave adds them up itself, and where its pieces are few one
// launch does it all, each workgroup for itself.  Which it is, and with it the order of all sums, follows from the sizes, the types, the device
// and whether what is written is memory of the tensors; not from where they lie otherwise.
// (The last workgroup to arrive could do it, counting: but an agent-wide release and acquire in every workgroup costs 28 ns, one after
// the other: 2048 workgroups over 33 MB took 56 us.)  The scaling launch consists of tiny workgroups, a thread moves four elements: reading
// and writing runs at 6.5 TB/s that way and at 4.5 to 5 with workgroups that go on from tile to tile, where reads wait behind
// the writes before them; reading alone runs at 7.2 either way (1 GiB and more).  Squares are summed in binary64: no gradient of
// binary32 overflows there, and the sum's rounding does not show in the norm's 24 bits.  Elements are scaled in binary64 too: a
// factor of a few denormal bits, or none, would lose gradients that are huge but finite.
// Bound by memory: 16 x 2^26 binary32 into V 0.61 ms for the norms, 7.0 TB/s, and 1.35 ms for the scaling, 6.4 TB/s.
#include <type_traits>

#include "qgx_types.h"

namespace qgx {

// The pieces of a batch's tensors, a thread for each.
__global__ __launch_bounds__(256) void k_tensor_list(TensorBatch batch, TensorPiece* __restrict__ table)
{
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < batch.pieces; i += (uint64_t)gridDim.x * 256u) {
        const uint64_t p = batch.first_piece + i;
        uint32_t lo = 0, hi = batch.count;                 // the last tensor whose first piece is at most p (one without elements has none)
        while (hi - lo > 1u) {
            const uint32_t mid = (lo + hi) / 2u;
            if (batch.entry[mid].first_piece <= p) lo = mid;
            else hi = mid;
        }
        const TensorBatch::Entry& e = batch.entry[lo];
        const uint64_t at = (p - e.first_piece) * kClipPiece, size = e.dtype == QGX_F32 ? 4u : 2u;
        const uint32_t n = (uint32_t)min((uint64_t)kClipPiece, e.n - at);
        table[p] = TensorPiece{e.data + at * size, e.stride * size, e.offset + (uint32_t)at, n | e.dtype << 16};
    }
}

hipError_t launch_tensor_list(const TensorBatch& batch, TensorPiece* table, hipStream_t st)
{
    hipLaunchKernelGGL(k_tensor_list, dim3((uint32_t)min((batch.pieces + 255u) / 256u, (uint64_t)4096u)), dim3(256), 0, st, batch, table);
    return hipGetLastError();
}

// f with a value of the piece's type (the same in the whole workgroup).
template <typename F>
__device__ __forceinline__ void with_type(const TensorPiece& e, F f)
{
    const uint32_t type = e.n_type >> 16;
    if (type == QGX_F32) f(float());
    else if (type == QGX_F16) f(_Float16());
    else f(__bf16());
}

template <bool MAX> struct ClipSum { double x = 0.0; };
template <> struct ClipSum<true> { float x = 0.0f; };

// A NaN among two is the result.
template <bool MAX, typename X>
__device__ __forceinline__ X clip_join(X a, X b)
{
    if constexpr (MAX) return __builtin_elementwise_maximum(a, b);
    else return a + b;
}

template <typename T, bool MAX>
__device__ __forceinline__ void sum_piece(const T* x, int n, ClipSum<MAX>& s)
{
    constexpr int W = kPiece<T>, N = (int)kClipPiece / (kClipThreads * W);
    nt_u32x4 x4[N];
    const int i0 = (int)threadIdx.x * W;
    if (n == (int)kClipPiece) {                            // (the same for the whole workgroup: all loads are under way at once)
#pragma unroll
        for (int j = 0; j < N; ++j) x4[j] = __builtin_bit_cast(nt_u32x4, __builtin_nontemporal_load(reinterpret_cast<const Piece<T>*>(x + i0 + j * kClipThreads * W)));
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x4[j] = __builtin_bit_cast(nt_u32x4, load_raw(x + i0 + j * kClipThreads * W, n - i0 - j * kClipThreads * W));
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float v[W];
        values_of<T>(x4[j], v);
#pragma unroll
        for (int c = 0; c < W; ++c) {
            if constexpr (MAX) s.x = __builtin_elementwise_maximum(s.x, fabsf(v[c]));
            else s.x = fma((double)v[c], (double)v[c], s.x);
        }
    }
}

// The largest of a wave's binary32 values, a NaN among them the result.
__device__ __forceinline__ double wave_largest(double x)
{
    return (double)__uint_as_float(wave_join_u32<32>(__float_as_uint((float)x), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__builtin_elementwise_maximum(__uint_as_float(a), __uint_as_float(b)));
    }));
}

// The sum over a workgroup, in its first thread.
template <bool MAX>
__device__ __forceinline__ double clip_group_sum(double x, double* slot)
{
    if constexpr (MAX) x = wave_largest(x);
    else x = wave_sum(x);
    if (lane_id() == 0) slot[wave_id()] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kClipThreads / kWave; ++w) x = clip_join<MAX>(x, slot[w]);
    return x;
}

template <bool MAX>
__global__ __launch_bounds__(kClipThreads) void k_clip_norm(ClipArgs a)
{
    __shared__ double s_sum[kClipThreads / kWave];
    const uint32_t k = blockIdx.y;
    ClipSum<MAX> sum;
    TensorPiece next = a.table[blockIdx.x];                // (the grid has no more workgroups than pieces)
    for (uint64_t p = blockIdx.x; p < a.n_pieces; p += a.parts) {
        const TensorPiece e = next;
        next = a.table[min(p + a.parts, a.n_pieces - 1u)];
        const void* x = reinterpret_cast<const void*>(e.data + (uint64_t)k * e.stride);
        const int n = (int)(e.n_type & 0xFFFFu);
        with_type(e, [&](auto t) { sum_piece<decltype(t), MAX>((const decltype(t)*)x, n, sum); });
    }
    const double x = clip_group_sum<MAX>((double)sum.x, s_sum);
    if (threadIdx.x == 0) a.partial[(size_t)k * kClipParts + blockIdx.x] = x;
}

// A worker's norm out of its sum, and its factor.  A norm that is no finite number: the sum of squares is beyond binary64 only if an
// element is infinite or no number.
struct ClipFactor { double norm, scale; };
template <bool MAX>
__device__ __forceinline__ ClipFactor clip_factor(double sum, float max_norm)
{
    const double norm = MAX ? sum : sqrt(sum);
    return ClipFactor{norm, norm < __builtin_inf() && norm > (double)max_norm ? (double)max_norm / norm : 1.0};
}

__device__ __forceinline__ void report_norm(const ClipArgs& a, uint32_t k, double norm, Scalars* sc)
{
    if (a.norms) a.norms[k] = (float)norm;
    if (!(norm < __builtin_inf())) raise_error(sc, QGX_EBIT_NONFINITE);
}

// Up to kWave partial sums, in every lane of a wave.
template <bool MAX>
__device__ __forceinline__ double join_few(const double* __restrict__ partial, uint32_t parts)
{
    const double x = (uint32_t)lane_id() < parts ? partial[lane_id()] : 0.0;
    if constexpr (MAX) return wave_largest(x);
    else return wave_sum(x);
}

template <bool MAX>
__global__ __launch_bounds__(kClipThreads) void k_clip_join(ClipArgs a, Scalars* sc)
{
    __shared__ double s_sum[kClipThreads / kWave];
    const uint32_t k = blockIdx.x;
    double x = 0.0;
    for (uint32_t i = threadIdx.x; i < a.parts; i += kClipThreads) x = clip_join<MAX>(x, a.partial[(size_t)k * kClipParts + i]);
    x = clip_group_sum<MAX>(x, s_sum);
    if (threadIdx.x != 0) return;
    const ClipFactor f = clip_factor<MAX>(x, a.max_norm);
    a.scale[k] = f.scale;
    report_norm(a, k, f.norm, sc);
}

constexpr int kScaleEach = 4;                              // elements that a thread moves at once
constexpr uint32_t kScaleTile = kClipThreads * kScaleEach;
constexpr uint32_t kScaleTiles = kClipPiece / kScaleTile;  // tiles of a piece

// Four elements of a piece from element i on as they lie there (two words of 16-bit ones), zeros past its end.
template <typename T, bool AGAIN = false>
__device__ __forceinline__ nt_u32x4 load_four(const TensorPiece& e, uint32_t k, int i)
{
    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const T* x = reinterpret_cast<const T*>(e.data + (uint64_t)k * e.stride) + i;
    const int n = (int)(e.n_type & 0xFFFFu) - i;
    four y;
    if (n >= 4) {
        // (AGAIN: others read it as well)
        if constexpr (AGAIN) y = *reinterpret_cast<const four*>(x);
        else y = __builtin_nontemporal_load(reinterpret_cast<const four*>(x));
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = q < n ? x[q] : (T)0.0f;
    }
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(nt_u32x4, y);
    } else {
        const uint64_t z = __builtin_bit_cast(uint64_t, y);
        return nt_u32x4{(uint32_t)z, (uint32_t)(z >> 32), 0u, 0u};
    }
}

template <typename T>
__device__ __forceinline__ void values_of_four(nt_u32x4 x, float (&v)[4])
{
    if constexpr (sizeof(T) == 4) {
        values_of<T>(x, v);
    } else {
        float w[kPiece<T>];
        values_of<T>(x, w);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = w[q];
    }
}

// They scaled, to V (row: the piece's first coordinate there) or to where they were.  The product is rounded to binary32 and, in place, from there to
// a type of 16 bits: one result in some 2^14 (binary16) or 2^17 (bfloat16) becomes the other neighbour of a middle that binary32 cannot tell from
// it.  (From binary64 at once: 8 x 2^24 binary16 172 us, 124 so; 8 x 2^20 bfloat16 20.3 and 18.8.)
template <typename T, bool GATHER>
__device__ __forceinline__ void store_four(const TensorPiece& e, uint32_t k, int i, double c, const float (&v)[4], float* row)
{
    using To = std::conditional_t<GATHER, float, T>;
    typedef To four __attribute__((ext_vector_type(4), aligned(sizeof(To))));
    To* to;
    if constexpr (GATHER) to = row + i;
    else to = reinterpret_cast<T*>(e.data + (uint64_t)k * e.stride) + i;
    const int n = (int)(e.n_type & 0xFFFFu) - i;
    four y;
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = (To)(float)((double)v[q] * c);
    if (n >= 4) {
        if constexpr (GATHER) __builtin_nontemporal_store(y, reinterpret_cast<four*>(to));
        else *reinterpret_cast<four*>(to) = y;
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < n) to[q] = y[q];
    }
}

constexpr uint32_t kInPlaceTiles = 4;                      // tiles of a workgroup in place

enum class ClipJoin { Done, Sum, Max };                     // the factor is there, or comes from the few partial sums

// EACH tiles to a workgroup.  In place four, for a worker that is not clipped then has a quarter of the workgroups that come for nothing
// (16 x 2^26 binary32 without clipping 835 us with one, 680 with four; with clipping 2.15 ms either way).
template <bool GATHER, ClipJoin JOIN, int EACH>
__global__ __launch_bounds__(kClipThreads) void k_clip_scale(ClipArgs a, uint32_t sets, Scalars* sc)
{
    // from the last tile of the last worker back: part of what was read last is still in the cache
    const uint32_t k = gridDim.y - 1u - blockIdx.y, x = sets - 1u - blockIdx.x;
    const TensorPiece e = a.table[x / (kScaleTiles / EACH)];
    double c;
    if constexpr (JOIN == ClipJoin::Done) {
        c = a.scale[k];
    } else {
        const ClipFactor f = clip_factor<JOIN == ClipJoin::Max>(join_few<JOIN == ClipJoin::Max>(a.partial + (size_t)k * kClipParts, a.parts), a.max_norm);
        c = f.scale;
        if (x == 0u && threadIdx.x == 0) report_norm(a, k, f.norm, sc);
    }
    if (!GATHER && c == 1.0) return;
    const int i0 = (int)(x % (kScaleTiles / EACH) * (EACH * kScaleTile) + threadIdx.x * kScaleEach);
    if (i0 >= (int)(e.n_type & 0xFFFFu)) return;
    float* to = GATHER ? a.V + (uint64_t)k * a.d + e.offset : nullptr;
    with_type(e, [&](auto t) {
        using T = decltype(t);
        nt_u32x4 raw[EACH];
#pragma unroll
        for (int j = 0; j < EACH; ++j) raw[j] = load_four<T>(e, k, i0 + j * (int)kScaleTile);
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            float v[4];
            values_of_four<T>(raw[j], v);
            store_four<T, GATHER>(e, k, i0 + j * (int)kScaleTile, c, v, to);
        }
    });
}

// A few pieces: a workgroup for each worker holds them in registers between its sum and its stores, in one launch (4 x 16384 binary32
// 5.8 us a call, in two launches 8.5; sixteen pieces take one compute unit 16 us, two launches over the GPU 5.5).
constexpr int kSmallThreads = 1024, kSmallPieces = 4;
static_assert(kSmallThreads * kScaleEach == (int)kClipPiece, "a thread has four elements of a piece");

template <bool MAX, bool GATHER>
__global__ __launch_bounds__(kSmallThreads) void k_clip_small(ClipArgs a, Scalars* sc)
{
    __shared__ double s_sum[kSmallThreads / kWave];
    const uint32_t k = blockIdx.x, n_pieces = (uint32_t)a.n_pieces;
    const int i = (int)threadIdx.x * kScaleEach;
    // (no way out of the loops: the pieces' places, then all elements, are under way at once)
    TensorPiece e[kSmallPieces];
#pragma unroll
    for (int p = 0; p < kSmallPieces; ++p) {
        e[p] = a.table[min((uint32_t)p, n_pieces - 1u)];
        if (p >= (int)n_pieces) e[p].n_type &= ~0xFFFFu;   // no elements
    }
    nt_u32x4 raw[kSmallPieces];
#pragma unroll
    for (int p = 0; p < kSmallPieces; ++p) with_type(e[p], [&](auto t) { raw[p] = load_four<decltype(t)>(e[p], k, i); });
    ClipSum<MAX> sum;
#pragma unroll
    for (int p = 0; p < kSmallPieces; ++p) {
        float v[4];
        with_type(e[p], [&](auto t) { values_of_four<decltype(t)>(raw[p], v); });
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (MAX) sum.x = __builtin_elementwise_maximum(sum.x, fabsf(v[q]));
            else sum.x = fma((double)v[q], (double)v[q], sum.x);
        }
    }
    double x = (double)sum.x;
    if constexpr (MAX) x = wave_largest(x);
    else x = wave_sum(x);
    if (lane_id() == 0) s_sum[wave_id()] = x;
    __syncthreads();
    x = s_sum[0];
#pragma unroll
    for (int w = 1; w < kSmallThreads / kWave; ++w) x = clip_join<MAX>(x, s_sum[w]);
    const ClipFactor f = clip_factor<MAX>(x, a.max_norm);
    if (threadIdx.x == 0) report_norm(a, k, f.norm, sc);
    if (!GATHER && f.scale == 1.0) return;
#pragma unroll
    for (int p = 0; p < kSmallPieces; ++p)
        with_type(e[p], [&](auto t) {
            float v[4];
            values_of_four<decltype(t)>(raw[p], v);
            store_four<decltype(t), GATHER>(e[p], k, i, f.scale, v, GATHER ? a.V + (uint64_t)k * a.d + e[p].offset : nullptr);
        });
}

// Some pieces more, all of one type, into V: a workgroup for each piece of each worker, which sums up all of the worker's pieces, as every other
// one of that worker's does, and scales its own: no second launch has to wait for the sums.  (Not in place, where a piece might have been
// scaled before another workgroup has read it.)  For 4 workers, a call this way and in two launches: 8 pieces of binary32 5.8 us and 8.1, 16 6.2 and
// 8.0; from 18 to 24 8.2 to 8.5 and 8.7, of bfloat16 8.9 to 9.3 and 8.6; 32 18.9 and 8.7, 11.1 and 8.6.  1 and 8 workers are within 0.3 us.  Of
// several types, the dispatch for every piece costs more than it gains.
constexpr int kAgainPieces = 16;
static_assert(kAgainPieces <= QGX_FEW_TENSORS, "their places are known");

template <typename T, bool MAX, int PIECES>
__global__ __launch_bounds__(kSmallThreads) void k_clip_again(ClipArgs a, Scalars* sc)
{
    __shared__ double s_sum[kSmallThreads / kWave];
    const uint32_t k = blockIdx.x, mine = blockIdx.y, n_pieces = (uint32_t)a.n_pieces;      // (a worker's workgroups on as few XCDs as can be)
    const int i = (int)threadIdx.x * kScaleEach;
    nt_u32x4 raw[PIECES], own = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        TensorPiece e = a.table[min((uint32_t)p, n_pieces - 1u)];
        if (p >= (int)n_pieces) e.n_type &= ~0xFFFFu;      // no elements
        raw[p] = load_four<T, true>(e, k, i);
    }
    ClipSum<MAX> sum;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        float v[4];
        values_of_four<T>(raw[p], v);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (MAX) sum.x = __builtin_elementwise_maximum(sum.x, fabsf(v[q]));
            else sum.x = fma((double)v[q], (double)v[q], sum.x);
        }
        if (p == (int)mine) own = raw[p];
    }
    double x = (double)sum.x;
    if constexpr (MAX) x = wave_largest(x);
    else x = wave_sum(x);
    if (lane_id() == 0) s_sum[wave_id()] = x;
    __syncthreads();
    x = s_sum[0];
#pragma unroll
    for (int w = 1; w < kSmallThreads / kWave; ++w) x = clip_join<MAX>(x, s_sum[w]);
    const ClipFactor f = clip_factor<MAX>(x, a.max_norm);
    if (mine == 0u && threadIdx.x == 0) report_norm(a, k, f.norm, sc);
    const TensorPiece e = a.table[mine];
    float v[4];
    values_of_four<T>(own, v);
    store_four<T, true>(e, k, i, f.scale, v, a.V + (uint64_t)k * a.d + e.offset);
}

template <typename T, int PIECES>
static hipError_t launch_again(const ClipArgs& a, uint32_t K, bool max_kind, Scalars* sc, hipStream_t st)
{
    const dim3 grid(K, (uint32_t)a.n_pieces);
    if (max_kind) hipLaunchKernelGGL((k_clip_again<T, true, PIECES>), grid, dim3(kSmallThreads), 0, st, a, sc);
    else hipLaunchKernelGGL((k_clip_again<T, false, PIECES>), grid, dim3(kSmallThreads), 0, st, a, sc);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_again_of(const ClipArgs& a, uint32_t K, bool max_kind, Scalars* sc, hipStream_t st)
{
    return a.n_pieces <= (uint64_t)kAgainPieces / 2u ? launch_again<T, kAgainPieces / 2>(a, K, max_kind, sc, st)
                                                     : launch_again<T, kAgainPieces>(a, K, max_kind, sc, st);
}

static hipError_t launch_small(const ClipArgs& a, uint32_t K, bool max_kind, Scalars* sc, hipStream_t st)
{
    if (max_kind && a.V) hipLaunchKernelGGL((k_clip_small<true, true>), dim3(K), dim3(kSmallThreads), 0, st, a, sc);
    else if (max_kind) hipLaunchKernelGGL((k_clip_small<true, false>), dim3(K), dim3(kSmallThreads), 0, st, a, sc);
    else if (a.V) hipLaunchKernelGGL((k_clip_small<false, true>), dim3(K), dim3(kSmallThreads), 0, st, a, sc);
    else hipLaunchKernelGGL((k_clip_small<false, false>), dim3(K), dim3(kSmallThreads), 0, st, a, sc);
    return hipGetLastError();
}

template <ClipJoin JOIN>
static hipError_t launch_scale(ClipArgs a, uint32_t K, Scalars* sc, hipStream_t st)
{
    // (a grid's threads stay below 2^32: more tiles than that, of more than two million tensors, take another launch)
    constexpr uint64_t most = 1u << 21;
    const TensorPiece* table = a.table;
    for (uint64_t left = a.n_pieces; left;) {
        const uint32_t now = (uint32_t)min(left, most);
        const uint32_t each = a.V ? 1u : kInPlaceTiles, sets = now * (kScaleTiles / each);
        const dim3 grid(sets, K);
        a.table = table + (left - now);
        if (a.V) hipLaunchKernelGGL((k_clip_scale<true, JOIN, 1>), grid, dim3(kClipThreads), 0, st, a, sets, sc);
        else hipLaunchKernelGGL((k_clip_scale<false, JOIN, kInPlaceTiles>), grid, dim3(kClipThreads), 0, st, a, sets, sc);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        left -= now;
    }
    return hipSuccess;
}

hipError_t launch_clip(const ClipArgs& args, uint32_t K, bool max_kind, uint32_t n_cu, Scalars* sc, hipStream_t st)
{
    ClipArgs a = args;
    if (a.n_pieces && a.n_pieces <= (uint32_t)kSmallPieces) return launch_small(a, K, max_kind, sc, st);
    if (a.apart && a.n_pieces && a.n_pieces <= (uint64_t)kAgainPieces && K * a.n_pieces <= n_cu) {
        if (a.dtype == QGX_F32) return launch_again_of<float>(a, K, max_kind, sc, st);
        if (a.dtype == QGX_F16) return launch_again_of<_Float16>(a, K, max_kind, sc, st);
        if (a.dtype == QGX_BF16) return launch_again_of<__bf16>(a, K, max_kind, sc, st);
    }
    // eight workgroups for every compute unit over all workers
    const uint64_t each = max(1u, min(kClipParts, 8u * n_cu / K));
    a.parts = (uint32_t)min(a.n_pieces, each);
    const dim3 grid(a.parts, K);
    if (a.parts) {
        if (max_kind) hipLaunchKernelGGL(k_clip_norm<true>, grid, dim3(kClipThreads), 0, st, a);
        else hipLaunchKernelGGL(k_clip_norm<false>, grid, dim3(kClipThreads), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // Few sums: a launch less.  Many: the waves' additions would outweigh it.
    if (a.n_pieces && a.parts <= (uint32_t)kWave && a.n_pieces * kScaleTiles * K <= 16u * n_cu)
        return max_kind ? launch_scale<ClipJoin::Max>(a, K, sc, st) : launch_scale<ClipJoin::Sum>(a, K, sc, st);
    if (max_kind) hipLaunchKernelGGL(k_clip_join<true>, dim3(K), dim3(kClipThreads), 0, st, a, sc);
    else hipLaunchKernelGGL(k_clip_join<false>, dim3(K), dim3(kClipThreads), 0, st, a, sc);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_scale<ClipJoin::Done>(a, K, sc, st);
}

}  // namespace qgx
