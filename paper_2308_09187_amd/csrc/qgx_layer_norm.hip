// Layer norm, forward and backward.
//   h = (x - mean) rstd,  y = h w + b;   g = dy w,  dx = rstd (g - mean(g) - h mean(g h)),  dw = sum_rows dy h,  db = sum_rows dy
// A row stays in registers between its sums, so that it crosses memory once; LANES threads share it.
#include "qgx_types.h"

namespace qgx {

// The sum over the LANES threads of a row, in each of them; slot: LDS of this sum's own where a row has several waves.
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float* slot)
{
    if constexpr (LANES <= kWave) {
        return lanes_sum<LANES>(x);
    } else {
        x = lanes_sum<kWave>(x);
        if (lane_id() == 0) slot[wave_id()] = x;
        __syncthreads();
        x = slot[0];
#pragma unroll
        for (int w = 1; w < LANES / kWave; ++w) x += slot[w];
        return x;
    }
}

template <int LANES> constexpr int kNormThreads = LANES > 256 ? LANES : 256;

constexpr uint32_t kNormBlocksMax = 1u << 20;             // workgroups of a launch (a grid's threads stay below 2^32); they go on from there

// The rows of a group of LANES threads: f(worker, row).
template <int LANES, typename F>
__device__ __forceinline__ void for_rows(uint32_t rows, uint32_t n_rows, F f)
{
    constexpr uint32_t per = kNormThreads<LANES> / LANES;
    for (uint64_t i = (uint64_t)blockIdx.x * per + threadIdx.x / LANES; i < n_rows; i += (uint64_t)gridDim.x * per)
        f((uint32_t)i / rows, (uint32_t)i % rows);
}

template <int LANES>
static dim3 row_grid(uint32_t n_rows)
{
    constexpr uint32_t per = kNormThreads<LANES> / LANES;
    return dim3(min((n_rows - 1u) / per + 1u, kNormBlocksMax));
}

template <typename T, int LANES, int N>
__global__ __launch_bounds__(kNormThreads<LANES>) void k_layer_norm(NormArgs a)
{
    constexpr int W = kPiece<T>;
    __shared__ float s_sum[2][16];
    for_rows<LANES>(a.rows, a.n_rows, [&](uint32_t k, uint32_t r) {
        const int lane = (int)(threadIdx.x % LANES), cols = (int)a.cols;
        const T* x = (const T*)a.x + k * a.x_worker + r * a.x_row;
        float v[N][W], sum = 0.0f, sq = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int c0 = (lane + j * LANES) * W;
            load_piece(x + c0, cols - c0, v[j]);
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int c = 0; c < W; ++c) sum += v[j][c];
        const float mean = row_sum<LANES>(sum, s_sum[0]) / (float)cols;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int n = cols - (lane + j * LANES) * W;
#pragma unroll
            for (int c = 0; c < W; ++c) {
                v[j][c] -= mean;
                sq += c < n ? v[j][c] * v[j][c] : 0.0f;
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<LANES>(sq, s_sum[1]) / (float)cols + a.eps);
        T* y = (T*)a.y + k * a.y_worker + r * a.y_row;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int c0 = (lane + j * LANES) * W;
            float w[W], b[W];
#pragma unroll
            for (int c = 0; c < W; ++c) {
                w[c] = a.w && c0 + c < cols ? a.w[c0 + c] : 1.0f;
                b[c] = a.b && c0 + c < cols ? a.b[c0 + c] : 0.0f;
            }
#pragma unroll
            for (int c = 0; c < W; ++c) v[j][c] = v[j][c] * rstd * w[c] + b[c];
            store_piece(y + c0, cols - c0, v[j]);
        }
        if (lane == 0) {
            const size_t row = (size_t)k * a.rows + r;
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    });
}

// Rows too long for registers: read three times, twice from the cache.
template <typename T>
__global__ __launch_bounds__(1024) void k_layer_norm_long(NormArgs a)
{
    constexpr int W = kPiece<T>, LANES = 1024;
    __shared__ float s_sum[2][16];
    for_rows<LANES>(a.rows, a.n_rows, [&](uint32_t k, uint32_t r) {
        const int cols = (int)a.cols;
        const T* x = (const T*)a.x + k * a.x_worker + r * a.x_row;
        T* y = (T*)a.y + k * a.y_worker + r * a.y_row;
        float sum = 0.0f, sq = 0.0f;
        for (int c0 = (int)threadIdx.x * W; c0 < cols; c0 += LANES * W) {
            float v[W];
            load_piece(x + c0, cols - c0, v);
            for (int c = 0; c < W; ++c) sum += v[c];
        }
        const float mean = row_sum<LANES>(sum, s_sum[0]) / (float)cols;
        for (int c0 = (int)threadIdx.x * W; c0 < cols; c0 += LANES * W) {
            float v[W];
            load_piece(x + c0, cols - c0, v);
            for (int c = 0; c < W; ++c) sq += c0 + c < cols ? (v[c] - mean) * (v[c] - mean) : 0.0f;
        }
        const float rstd = 1.0f / sqrtf(row_sum<LANES>(sq, s_sum[1]) / (float)cols + a.eps);
        for (int c0 = (int)threadIdx.x * W; c0 < cols; c0 += LANES * W) {
            float v[W];
            load_piece(x + c0, cols - c0, v);
            for (int c = 0; c < W; ++c) {
                const float w = a.w && c0 + c < cols ? a.w[c0 + c] : 1.0f, b = a.b && c0 + c < cols ? a.b[c0 + c] : 0.0f;
                v[c] = (v[c] - mean) * rstd * w + b;
            }
            store_piece(y + c0, cols - c0, v);
        }
        if (threadIdx.x == 0) {
            const size_t row = (size_t)k * a.rows + r;
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    });
}

// dx, a row per workgroup, read twice (the second time from the cache).
template <typename T, int LANES>
__global__ __launch_bounds__(kNormThreads<LANES>) void k_layer_norm_dx(NormBackArgs a)
{
    constexpr int W = kPiece<T>;
    __shared__ float s_sum[2][16];
    for_rows<LANES>(a.rows, a.n_rows, [&](uint32_t k, uint32_t r) {
        const int lane = (int)(threadIdx.x % LANES), cols = (int)a.cols;
        const T* x = (const T*)a.x + k * a.x_worker + r * a.x_row;
        const T* dy = (const T*)a.dy + k * a.dy_worker + r * a.dy_row;
        T* dx = (T*)a.dx + k * a.dx_worker + r * a.dx_row;
        const size_t row = (size_t)k * a.rows + r;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c0 = lane * W; c0 < cols; c0 += LANES * W) {
            float u[W], v[W];
            load_piece(x + c0, cols - c0, u);
            load_piece(dy + c0, cols - c0, v);
            for (int c = 0; c < W; ++c)
                if (c0 + c < cols) {
                    const float g = v[c] * (a.w ? a.w[c0 + c] : 1.0f);
                    s1 += g;
                    s2 += g * ((u[c] - mean) * rstd);
                }
        }
        s1 = row_sum<LANES>(s1, s_sum[0]) / (float)cols;
        s2 = row_sum<LANES>(s2, s_sum[1]) / (float)cols;
        for (int c0 = lane * W; c0 < cols; c0 += LANES * W) {
            float u[W], v[W];
            load_piece(x + c0, cols - c0, u);
            load_piece(dy + c0, cols - c0, v);
            for (int c = 0; c < W; ++c) {
                const float g = v[c] * (a.w && c0 + c < cols ? a.w[c0 + c] : 1.0f);
                v[c] = rstd * (g - s1 - (u[c] - mean) * rstd * s2);
            }
            store_piece(dx + c0, cols - c0, v);
        }
    });
}

// dw and db of 64 columns of a worker, four runs of its rows side by side.
template <typename T>
__global__ __launch_bounds__(256) void k_layer_norm_columns(NormBackArgs a)
{
    __shared__ float s_w[4][64], s_b[4][64];
    const uint32_t k = blockIdx.y, c = blockIdx.x * 64u + threadIdx.x % 64u, run = threadIdx.x / 64u;
    float dw = 0.0f, db = 0.0f;
    if (c < a.cols)
        for (uint32_t r = run; r < a.rows; r += 4u) {
            const size_t row = (size_t)k * a.rows + r;
            const float dy = (float)((const T*)a.dy + k * a.dy_worker + r * a.dy_row)[c];
            const float x = (float)((const T*)a.x + k * a.x_worker + r * a.x_row)[c];
            dw += dy * ((x - a.mean[row]) * a.rstd[row]);
            db += dy;
        }
    s_w[run][threadIdx.x % 64u] = dw;
    s_b[run][threadIdx.x % 64u] = db;
    __syncthreads();
    if (run == 0 && c < a.cols) {
        for (int i = 1; i < 4; ++i) { dw += s_w[i][threadIdx.x]; db += s_b[i][threadIdx.x]; }
        if (a.dw) a.dw[k * a.param_stride + c] = dw;
        if (a.db) a.db[k * a.param_stride + c] = db;
    }
}

template <typename T, int LANES, int N>
static hipError_t launch_norm_as(const NormArgs& a, hipStream_t st)
{
    hipLaunchKernelGGL((k_layer_norm<T, LANES, N>), row_grid<LANES>(a.n_rows), dim3(kNormThreads<LANES>), 0, st, a);
    return hipGetLastError();
}

// The fewest threads that hold a row in four pieces each.
template <typename T>
static hipError_t launch_norm_of(const NormArgs& a, hipStream_t st)
{
    const uint32_t pieces = (a.cols + kPiece<T> - 1u) / kPiece<T>;
    if (pieces <= 4u) return launch_norm_as<T, 4, 1>(a, st);
    if (pieces <= 16u) return launch_norm_as<T, 4, 4>(a, st);
    if (pieces <= 32u) return launch_norm_as<T, 16, 2>(a, st);
    if (pieces <= 64u) return launch_norm_as<T, 16, 4>(a, st);
    if (pieces <= 128u) return launch_norm_as<T, 64, 2>(a, st);
    if (pieces <= 256u) return launch_norm_as<T, 64, 4>(a, st);
    if (pieces <= 512u) return launch_norm_as<T, 256, 2>(a, st);
    if (pieces <= 1024u) return launch_norm_as<T, 256, 4>(a, st);
    if (pieces <= 2048u) return launch_norm_as<T, 1024, 2>(a, st);
    if (pieces <= 4096u) return launch_norm_as<T, 1024, 4>(a, st);
    hipLaunchKernelGGL(k_layer_norm_long<T>, row_grid<1024>(a.n_rows), dim3(1024), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_layer_norm(int dtype, const NormArgs& a, hipStream_t st)
{
    if (a.n_rows == 0) return hipSuccess;
    return dtype == QGX_F32 ? launch_norm_of<float>(a, st) : dtype == QGX_F16 ? launch_norm_of<_Float16>(a, st) : launch_norm_of<__bf16>(a, st);
}

template <typename T>
static hipError_t launch_norm_back_of(const NormBackArgs& a, uint32_t workers, hipStream_t st)
{
    if (a.dx && a.n_rows) {
        if (a.cols <= 64u * kPiece<T>) hipLaunchKernelGGL((k_layer_norm_dx<T, 64>), row_grid<64>(a.n_rows), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_layer_norm_dx<T, 256>), row_grid<256>(a.n_rows), dim3(256), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.dw || a.db) hipLaunchKernelGGL(k_layer_norm_columns<T>, dim3((a.cols + 63u) / 64u, workers), dim3(256), 0, st, a);
    return hipGetLastError();
}

uint64_t norm_back_scratch(int, uint32_t, uint32_t, uint32_t) { return 0; }

hipError_t launch_layer_norm_back(int dtype, const NormBackArgs& a, uint32_t workers, hipStream_t st)
{
    return dtype == QGX_F32 ? launch_norm_back_of<float>(a, workers, st) : dtype == QGX_F16 ? launch_norm_back_of<_Float16>(a, workers, st)
                                                                                    : launch_norm_back_of<__bf16>(a, workers, st);
}

}  // namespace qgx
