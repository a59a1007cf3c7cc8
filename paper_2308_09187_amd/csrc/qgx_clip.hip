// Each worker's global gradient norm over its many tensors, and clipping, gathered into the dual vectors or in place.
//   N_k = (sum over tensors and elements x^2)^(1/2), or max |x|;   c_k = N_k > M ? M / N_k : 1;   V[k][offset + i] = c_k x_i
// Two launches: the sums of every workgroup's run of pieces, then, in every workgroup that scales, the sum of the worker's partial
// sums again (at most kClipParts doubles from the cache) in place of a launch or a wait between the two.  Squares are summed in
// binary64: no gradient of binary32 overflows there, and the sum's rounding does not show in the norm's 24 bits.
// Elements are scaled in binary64 too: a factor of a few denormal bits, or none, would lose gradients that are huge but finite.
#include "qgx_types.h"

namespace qgx {

__global__ __launch_bounds__(64) void k_tensor_list(TensorBatch batch, TensorEntry* __restrict__ table)
{
    if (threadIdx.x < batch.count) table[batch.first + threadIdx.x] = batch.entry[threadIdx.x];
}

hipError_t launch_tensor_list(const TensorBatch& batch, TensorEntry* table, hipStream_t st)
{
    hipLaunchKernelGGL(k_tensor_list, dim3(1), dim3(kTensorBatch), 0, st, batch, table);
    return hipGetLastError();
}

// The tensor that piece p of the list lies in: the last entry whose first piece is at most p (tensors without elements
// have no piece, and their successor's first piece is theirs).
__device__ __forceinline__ uint32_t tensor_of_piece(const TensorEntry* __restrict__ table, uint32_t n_tensors, uint64_t p)
{
    uint32_t lo = 0, hi = n_tensors;
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) / 2u;
        if (table[mid].first_piece <= p) lo = mid;
        else hi = mid;
    }
    return lo;
}

// f(entry, i, n): 16 bytes of the entry's elements from element i on, n of them still in the tensor; for every such run of
// pieces [p0, p1).
template <typename F>
__device__ __forceinline__ void for_pieces(const TensorEntry* __restrict__ table, uint32_t n_tensors, uint64_t p0, uint64_t p1, F f)
{
    if (p0 >= p1) return;
    uint32_t t = tensor_of_piece(table, n_tensors, p0);
    for (uint64_t p = p0; p < p1;) {
        while (t + 1u < n_tensors && table[t + 1u].first_piece <= p) ++t;
        const TensorEntry e = table[t];
        const uint64_t next = t + 1u < n_tensors ? table[t + 1u].first_piece : p1;
        const uint64_t stop = next < p1 ? next : p1;
        const uint64_t i0 = (p - e.first_piece) * kClipPiece, cut = (stop - e.first_piece) * kClipPiece, i1 = cut < e.n ? cut : e.n;
        f(e, i0, i1);
        p = stop;
    }
}

template <typename T, bool MAX>
__device__ __forceinline__ void sum_run(const TensorEntry& e, uint32_t k, uint64_t i0, uint64_t i1, double& sum, float& big)
{
    constexpr int W = kPiece<T>;
    const T* x = reinterpret_cast<const T*>(e.data) + (uint64_t)k * e.stride;
    for (uint64_t i = i0 + threadIdx.x * W; i < i1; i += kClipThreads * W) {
        float v[W];
        load_piece(x + i, (int)min((uint64_t)W, i1 - i), v);
#pragma unroll
        for (int c = 0; c < W; ++c) {
            if constexpr (MAX) big = __builtin_elementwise_maximum(big, fabsf(v[c]));      // (a NaN among them is the result)
            else sum = fma((double)v[c], (double)v[c], sum);
        }
    }
}

template <bool MAX>
__global__ __launch_bounds__(kClipThreads) void k_clip_norm(ClipArgs a)
{
    __shared__ double s_sum[kClipThreads / kWave];
    __shared__ float s_big[kClipThreads / kWave];
    const uint32_t k = blockIdx.y;
    const uint64_t p0 = blockIdx.x * a.per_part, p1 = min(p0 + a.per_part, a.n_pieces);
    double sum = 0.0;
    float big = 0.0f;
    for_pieces(a.table, a.n_tensors, p0, p1, [&](const TensorEntry& e, uint64_t i0, uint64_t i1) {
        if (e.dtype == QGX_F32) sum_run<float, MAX>(e, k, i0, i1, sum, big);
        else if (e.dtype == QGX_F16) sum_run<_Float16, MAX>(e, k, i0, i1, sum, big);
        else sum_run<__bf16, MAX>(e, k, i0, i1, sum, big);
    });
    if constexpr (MAX) {
        big = __uint_as_float(wave_join_u32<32>(__float_as_uint(big), [](uint32_t x, uint32_t y) {
            return __float_as_uint(__builtin_elementwise_maximum(__uint_as_float(x), __uint_as_float(y)));
        }));
        if (lane_id() == 0) s_big[wave_id()] = big;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kClipThreads / kWave; ++w) big = __builtin_elementwise_maximum(big, s_big[w]);
            a.partial[(size_t)k * kClipParts + blockIdx.x] = (double)big;
        }
    } else {
        sum = wave_sum(sum);
        if (lane_id() == 0) s_sum[wave_id()] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kClipThreads / kWave; ++w) sum += s_sum[w];
            a.partial[(size_t)k * kClipParts + blockIdx.x] = sum;
        }
    }
}

template <typename T, bool GATHER>
__device__ __forceinline__ void scale_run(const TensorEntry& e, uint32_t k, uint64_t i0, uint64_t i1, double c, float* row)
{
    constexpr int W = kPiece<T>;
    T* x = reinterpret_cast<T*>(e.data) + (uint64_t)k * e.stride;
    for (uint64_t i = i0 + threadIdx.x * W; i < i1; i += kClipThreads * W) {
        float v[W];
        const int n = (int)min((uint64_t)W, i1 - i);
        load_piece(x + i, n, v);
#pragma unroll
        for (int q = 0; q < W; ++q) v[q] = (float)((double)v[q] * c);
        if constexpr (GATHER) {
            float* out = row + e.offset + i;
#pragma unroll
            for (int h = 0; h < W / 4; ++h) {
                const float part[4] = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                store_piece(out + 4 * h, n - 4 * h, part);
            }
        } else {
            store_piece(x + i, n, v);
        }
    }
}

// The worker's norm from its partial sums, in every thread of the workgroup.
template <bool MAX>
__device__ __forceinline__ double join_parts(const double* __restrict__ partial, uint32_t parts)
{
    __shared__ double s_part[kClipThreads];
    double x = 0.0;
    for (uint32_t i = threadIdx.x; i < parts; i += kClipThreads) {
        if constexpr (MAX) x = __builtin_elementwise_maximum(x, partial[i]);
        else x += partial[i];
    }
    s_part[threadIdx.x] = x;
    __syncthreads();
    for (int off = kClipThreads / 2; off > 0; off >>= 1) {
        if ((int)threadIdx.x < off) {
            const double y = s_part[threadIdx.x + off];
            if constexpr (MAX) s_part[threadIdx.x] = __builtin_elementwise_maximum(s_part[threadIdx.x], y);
            else s_part[threadIdx.x] += y;
        }
        __syncthreads();
    }
    return MAX ? s_part[0] : sqrt(s_part[0]);
}

template <bool MAX, bool GATHER>
__global__ __launch_bounds__(kClipThreads) void k_clip_scale(ClipArgs a, Scalars* sc)
{
    const uint32_t k = blockIdx.y;
    const double norm = join_parts<MAX>(a.partial + (size_t)k * kClipParts, a.parts);
    // A norm that is no finite number: the sum of squares is beyond binary64 only if an element is infinite or no number.
    const bool finite = norm < __builtin_inf();
    const double c = finite && norm > (double)a.max_norm ? (double)a.max_norm / norm : 1.0;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (a.norms) a.norms[k] = (float)norm;
        if (!finite) raise_error(sc, QGX_EBIT_NONFINITE);
    }
    if (!GATHER && c == 1.0) return;
    const uint64_t p0 = blockIdx.x * a.per_scale, p1 = min(p0 + a.per_scale, a.n_pieces);
    float* row = GATHER ? a.V + (uint64_t)k * a.d : nullptr;
    for_pieces(a.table, a.n_tensors, p0, p1, [&](const TensorEntry& e, uint64_t i0, uint64_t i1) {
        if (e.dtype == QGX_F32) scale_run<float, GATHER>(e, k, i0, i1, c, row);
        else if (e.dtype == QGX_F16) scale_run<_Float16, GATHER>(e, k, i0, i1, c, row);
        else scale_run<__bf16, GATHER>(e, k, i0, i1, c, row);
    });
}

hipError_t launch_clip(const ClipArgs& args, uint32_t K, bool max_kind, Scalars* sc, hipStream_t st)
{
    ClipArgs a = args;
    // enough workgroups to fill the GPU (eight of 256 threads per compute unit)
    const uint64_t each = max(1u, min((uint32_t)kClipParts, (2048u + K - 1u) / K));
    const uint64_t want = min(max(a.n_pieces, (uint64_t)1), each);
    a.per_part = (a.n_pieces + want - 1u) / want;
    a.parts = a.per_part ? (uint32_t)((a.n_pieces + a.per_part - 1u) / a.per_part) : 0u;
    a.per_scale = a.per_part;
    const dim3 grid(max(a.parts, 1u), K);
    if (a.parts) {
        if (max_kind) hipLaunchKernelGGL(k_clip_norm<true>, grid, dim3(kClipThreads), 0, st, a);
        else hipLaunchKernelGGL(k_clip_norm<false>, grid, dim3(kClipThreads), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.V) {
        if (max_kind) hipLaunchKernelGGL((k_clip_scale<true, true>), grid, dim3(kClipThreads), 0, st, a, sc);
        else hipLaunchKernelGGL((k_clip_scale<false, true>), grid, dim3(kClipThreads), 0, st, a, sc);
    } else {
        if (max_kind) hipLaunchKernelGGL((k_clip_scale<true, false>), grid, dim3(kClipThreads), 0, st, a, sc);
        else hipLaunchKernelGGL((k_clip_scale<false, false>), grid, dim3(kClipThreads), 0, st, a, sc);
    }
    return hipGetLastError();
}

}  // namespace qgx
