// Rotary positions with several axes: pair p of a head turns by the token's position along the pair's axis times frequency p.
// Bound by memory, one read and one write.  The angles are the same for all heads of a token: a workgroup works out the sines and cosines of
// its tokens once, in LDS, and then streams their heads, 16 bytes of pairs to a thread at a time.
#include "qgx_types.h"

namespace qgx {

constexpr uint32_t kTurnThreads = 256;
constexpr uint32_t kTurnAngles = 2048;                     // most sines of a workgroup's tokens

// Sine and cosine of an angle in turns, reduced in binary64 before it becomes binary32.
__device__ __forceinline__ float2 cos_sin_of(double turns)
{
    const float r = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.0f * r, &s, &c);
    return make_float2(c, s);
}

// The frequencies come with the launch; PAIRS: as many as there is room for (the fewer, the sooner a launch is made).
template <int PAIRS> struct Frequencies { double turns[PAIRS]; };

template <typename T, bool NEIGHBOURS, int PAIRS>
__global__ __launch_bounds__(kTurnThreads) void k_rotary(RotaryArgs a, Frequencies<PAIRS> f, uint32_t tile_tokens, uint32_t turned, uint32_t items)
{
    constexpr int W = kPiece<T>;
    __shared__ float s_cos[kTurnAngles], s_sin[kTurnAngles];
    const uint32_t P = a.pairs;
    for (uint32_t first = blockIdx.x * tile_tokens; first < a.n_tokens; first += gridDim.x * tile_tokens) {
        const uint32_t count = min(tile_tokens, a.n_tokens - first);
        for (uint32_t i = threadIdx.x; i < count * P; i += kTurnThreads) {
            const uint32_t token = first + i / P, p = i % P, sequence = token / a.tokens, t = token % a.tokens;
            uint32_t axis = 0;
#pragma unroll
            for (uint32_t x = 0; x + 1 < QGX_MAX_AXES; ++x) axis += p >= a.axis_end[x];
            const int32_t at = a.positions[axis * a.p_axis + sequence / a.batch * a.p_worker + sequence % a.batch * a.p_batch + t];
            const float2 cs = cos_sin_of((double)at * f.turns[p]);
            s_cos[i] = cs.x;
            s_sin[i] = a.back ? -cs.y : cs.y;
        }
        __syncthreads();
        // an item: a piece of pairs (the first `turned` of a head's), or a piece of what stays as it is
        for (uint32_t i = threadIdx.x; i < count * a.heads * items; i += kTurnThreads) {
            const uint32_t row = i / items, item = i % items, local = row / a.heads, head = row % a.heads;
            const uint32_t token = first + local, sequence = token / a.tokens, t = token % a.tokens, k = sequence / a.batch, n = sequence % a.batch;
            const T* in = (const T*)a.in + k * a.i_worker + n * a.i_batch + t * a.i_token + head * a.i_head;
            T* out = (T*)a.out + k * a.o_worker + n * a.o_batch + t * a.o_token + head * a.o_head;
            if (item >= turned) {
                const uint32_t c = 2u * P + (item - turned) * W;
                float v[W];
                load_piece(in + c, (int)(a.dim - c), v);
                store_piece(out + c, (int)(a.dim - c), v);
            } else if constexpr (NEIGHBOURS) {
                const uint32_t c = item * W, p = local * P + c / 2u;
                const int left = (int)(2u * P - c);
                float v[W], w[W];
                load_piece(in + c, left, v);
#pragma unroll
                for (int j = 0; j < W / 2; ++j) {
                    const uint32_t q = p + (2 * j < left ? j : 0);
                    const float cs = s_cos[q], sn = s_sin[q];
                    w[2 * j] = fmaf(v[2 * j], cs, -(v[2 * j + 1] * sn));
                    w[2 * j + 1] = fmaf(v[2 * j], sn, v[2 * j + 1] * cs);
                }
                store_piece(out + c, left, w);
            } else {
                const uint32_t c = item * W, p = local * P + c;
                const int left = (int)(P - c);
                float v[W], u[W], w[W], z[W];
                load_piece(in + c, left, v);
                load_piece(in + P + c, left, u);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const uint32_t q = p + (j < left ? j : 0);
                    const float cs = s_cos[q], sn = s_sin[q];
                    w[j] = fmaf(v[j], cs, -(u[j] * sn));
                    z[j] = fmaf(v[j], sn, u[j] * cs);
                }
                store_piece(out + c, left, w);
                store_piece(out + P + c, left, z);
            }
        }
        __syncthreads();
    }
}

template <typename T, int PAIRS>
static hipError_t launch_rotary_as(const RotaryArgs& a, const double* turns, uint32_t n_cu, hipStream_t st)
{
    constexpr uint32_t W = kPiece<T>;
    const uint32_t turned = a.neighbours ? (2u * a.pairs + W - 1u) / W : (a.pairs + W - 1u) / W;
    const uint32_t rest = a.dim - 2u * a.pairs, items = turned + (a.in == a.out ? 0u : (rest + W - 1u) / W);
    const uint32_t most = max(1u, min(kTurnAngles / a.pairs, (1u << 30) / (a.heads * items)));
    const uint32_t tile = min(most, max(1u, a.n_tokens / (8u * n_cu)));
    const dim3 grid(min((a.n_tokens + tile - 1u) / tile, 1u << 20));
    Frequencies<PAIRS> f;
    for (uint32_t p = 0; p < (uint32_t)PAIRS; ++p) f.turns[p] = p < a.pairs ? turns[p] : 0.0;
    if (a.neighbours) hipLaunchKernelGGL((k_rotary<T, true, PAIRS>), grid, dim3(kTurnThreads), 0, st, a, f, tile, turned, items);
    else hipLaunchKernelGGL((k_rotary<T, false, PAIRS>), grid, dim3(kTurnThreads), 0, st, a, f, tile, turned, items);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_rotary_of(const RotaryArgs& a, const double* turns, uint32_t n_cu, hipStream_t st)
{
    return a.pairs <= 64u ? launch_rotary_as<T, 64>(a, turns, n_cu, st) : launch_rotary_as<T, (int)QGX_MAX_PAIRS>(a, turns, n_cu, st);
}

hipError_t launch_rotary(int dtype, const RotaryArgs& a, const double* turns, uint32_t n_cu, hipStream_t st)
{
    if (a.n_tokens == 0) return hipSuccess;
    return dtype == QGX_F32   ? launch_rotary_of<float>(a, turns, n_cu, st)
           : dtype == QGX_F16 ? launch_rotary_of<_Float16>(a, turns, n_cu, st)
                              : launch_rotary_of<__bf16>(a, turns, n_cu, st);
}

}  // namespace qgx
