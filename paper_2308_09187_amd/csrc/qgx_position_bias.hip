// Learned relative position bias by buckets: out = scores + table[row(j - i - p)][head], and the table's gradient.
#include "qgx_types.h"

namespace qgx {

// p of a (worker, sequence), kept within +-2^30 so that a delta fits 32 bits.
__device__ __forceinline__ int position_of(const BiasArgs& a, uint32_t n)
{
    const int64_t p = a.q_offset + (a.positions ? (int64_t)a.positions[n] : 0);
    return (int)max((int64_t)-(1 << 30), min(p, (int64_t)(1 << 30)));
}

// Index of the interval of delta: -1 before the first bound, n from the last on.
__device__ __forceinline__ int interval_of(const int* bounds, int n, int delta)
{
    int lo = -1, hi = n;                                   // bounds[lo] <= delta < bounds[hi + 1], outer ones taken as infinite
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (bounds[mid] <= delta) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <typename T>
__global__ __launch_bounds__(256) void k_position_bias(BiasArgs a, BucketArgs b)
{
    constexpr int W = kPiece<T>;
    __shared__ int s_bound[QGX_MAX_INTERVALS + 1];
    __shared__ float s_value[QGX_MAX_INTERVALS];
    const uint32_t per_row = (a.k + W - 1u) / W;
    const uint64_t pieces = (uint64_t)per_row * a.q;
    for (uint32_t i = threadIdx.x; i <= b.n; i += 256u) s_bound[i] = b.bounds[i];
    for (uint32_t plane = blockIdx.y; plane < a.planes; plane += gridDim.y) {       // (worker, sequence, head)
        const uint32_t head = plane % a.heads, seq = plane / a.heads, worker = seq / a.batch, n = seq % a.batch;
        const int p = position_of(a, seq);
        __syncthreads();                                   // the plane before has been dealt with
        for (uint32_t i = threadIdx.x; i < b.n; i += 256u) s_value[i] = a.table[(size_t)b.rows[i] * a.heads + head];
        __syncthreads();
        for (uint64_t piece = (uint64_t)blockIdx.x * 256u + threadIdx.x; piece < pieces; piece += (uint64_t)gridDim.x * 256u) {
            const uint32_t i = (uint32_t)(piece / per_row), j0 = (uint32_t)(piece % per_row) * W;
            const int left = (int)(a.k - j0), delta0 = (int)j0 - (int)i - p;
            T* out = (T*)a.out + worker * a.o_worker + n * a.o_batch + head * a.o_head + i * a.o_row + j0;
            float v[W];
#pragma unroll
            for (int c = 0; c < W; ++c) v[c] = 0.0f;
            if (a.in) load_piece((const T*)a.in + worker * a.i_worker + n * a.i_batch + head * a.i_head + i * a.i_row + j0, left, v);
            int at = interval_of(s_bound, (int)b.n, delta0);
#pragma unroll
            for (int c = 0; c < W; ++c) {
                while (at < (int)b.n && s_bound[at + 1] <= delta0 + c) ++at;
                v[c] = at < 0 || at >= (int)b.n ? -__builtin_inff() : v[c] + s_value[at];
            }
            store_piece(out, left, v);
        }
    }
}

// A workgroup adds up all of a worker's and a head's scores that take one row of the table.
template <typename T>
__global__ __launch_bounds__(256) void k_position_bias_back(BiasArgs a, BucketArgs b, float* __restrict__ dtable, uint64_t param_stride)
{
    __shared__ double s_sum[4];
    const uint32_t head = blockIdx.x % a.heads, r = blockIdx.x / a.heads, worker = blockIdx.y;
    const int p = position_of(a, 0);
    double sum = 0.0;
    for (uint32_t v = 0; v < b.n; ++v) {
        if (b.rows[v] != r) continue;
        for (uint32_t n = 0; n < a.batch; ++n)
            for (uint32_t i = 0; i < a.q; ++i) {
                const int64_t j0 = max((int64_t)0, (int64_t)b.bounds[v] + (int)i + p), j1 = min((int64_t)a.k, (int64_t)b.bounds[v + 1] + (int)i + p);
                const T* in = (const T*)a.in + worker * a.i_worker + n * a.i_batch + head * a.i_head + i * a.i_row;
                for (int64_t j = j0 + threadIdx.x; j < j1; j += 256) sum += (double)(float)in[j];
            }
    }
    sum = wave_sum(sum);
    if (lane_id() == 0) s_sum[wave_id()] = sum;
    __syncthreads();
    if (threadIdx.x == 0) dtable[worker * param_stride + (size_t)r * a.heads + head] = (float)(((sum + s_sum[1]) + s_sum[2]) + s_sum[3]);
}

hipError_t launch_position_bias(int dtype, const BiasArgs& a, const BucketArgs& b, hipStream_t st)
{
    const uint32_t W = dtype == QGX_F32 ? 4u : 8u;
    const uint64_t pieces = (uint64_t)((a.k + W - 1u) / W) * a.q;
    const dim3 grid((uint32_t)min((pieces + 255u) / 256u, (uint64_t)65536u), min(a.planes, 65535u));
    if (dtype == QGX_F32) hipLaunchKernelGGL(k_position_bias<float>, grid, dim3(256), 0, st, a, b);
    else if (dtype == QGX_F16) hipLaunchKernelGGL(k_position_bias<_Float16>, grid, dim3(256), 0, st, a, b);
    else hipLaunchKernelGGL(k_position_bias<__bf16>, grid, dim3(256), 0, st, a, b);
    return hipGetLastError();
}

uint64_t bias_back_scratch(int, const BiasArgs&, const BucketArgs&, uint32_t) { return 0; }

hipError_t launch_position_bias_back(int dtype, const BiasArgs& a, const BucketArgs& b, uint32_t workers, float* dtable, uint32_t table_rows,
                                     uint64_t param_stride, void*, hipStream_t st)
{
    const dim3 grid(table_rows * a.heads, workers);
    if (dtype == QGX_F32) hipLaunchKernelGGL(k_position_bias_back<float>, grid, dim3(256), 0, st, a, b, dtable, param_stride);
    else if (dtype == QGX_F16) hipLaunchKernelGGL(k_position_bias_back<_Float16>, grid, dim3(256), 0, st, a, b, dtable, param_stride);
    else hipLaunchKernelGGL(k_position_bias_back<__bf16>, grid, dim3(256), 0, st, a, b, dtable, param_stride);
    return hipGetLastError();
}

}  // namespace qgx
