// Group norm with an activation, channels last, forward and backward.
//   h = (x - mean) rstd,  z = h w + b,  y = act(z);   dz = dy act'(z),  g = dz w,  dx = rstd (g - mean(g) - h mean(g h)),
//   dw = sum dz h,  db = sum dz over a worker's samples and places
// Bound by memory.  A thread has W neighbouring channels (16 bytes) of every so manieth place, so that whatever belongs to a channel stays in
// its registers; sums are made channel by channel (a thread's places one by one, then the threads' of a channel) and only then
// joined to groups, whose borders may lie anywhere in a piece.  (8 x 16 x 1024 x 256 bfloat16 in 32 groups: forward with the input kept 51 us, backward from
// that 56, the bytes alone 26 each at 6.5 TB/s; 4 x 65536 x 128 forward, in parts, 47 of 21.)  Where all places of some groups fit a workgroup's registers it has them whole: one
// launch, x (and dy) cross memory once.  Else the places are dealt to workgroups that leave their channels' sums in scratch, a launch joins
// them, and a second pass over x makes y or dx.
#include "qgx_kept.h"
#include "qgx_plan.h"

namespace qgx {

// ---- pieces ---------------------------------------------------------------------------------------------------------------

// Where a thread's piece lies: channels c .. c + W - 1 of the sample, of which those before `shift` belong to the piece before (the last piece
// of a span is moved back to end there).  SHORT: fewer than W channels in all, `n` of them there.
struct ChannelsAt {
    int c, shift, n;
    __device__ __forceinline__ bool owns(int i) const { return i >= shift && i < n; }
};

template <int W, bool SHORT>
__device__ __forceinline__ ChannelsAt channels_at(uint32_t j, uint32_t first, uint32_t span)
{
    if constexpr (SHORT) return ChannelsAt{(int)first, 0, (int)span};
    const int c0 = (int)j * W, c = min(c0, (int)span - W);  // (of a last span shorter than a piece: before its first channel)
    return ChannelsAt{(int)first + c, c0 - c, W};
}

// A piece as loaded: sixteen bytes, or W codes and the powers of the one or two blocks they lie in.
template <typename T, bool KEPT> struct RawPiece { nt_u32x4 bits; };
template <typename T> struct RawPiece<T, true> { uint32_t code[kPiece<T> / 4]; uint32_t powers; };

// A sample's places: base addresses of worker k's sample n.
template <typename T, bool KEPT>
struct Places {
    const T* x;
    const uint8_t* codes;
    const uint8_t* powers;
    uint64_t place, power_place;
    int cut;                                               // of a kept piece: its first channel in the second block
};

template <typename T, bool KEPT>
__device__ __forceinline__ Places<T, KEPT> places_of(const GroupArgs& a, uint32_t sample, uint32_t batch, ChannelsAt at)
{
    Places<T, KEPT> p{};
    const uint32_t k = sample / batch, n = sample % batch;
    if constexpr (KEPT) {
        const uint64_t row = (uint64_t)sample * a.places;
        const int block = at.c / (int)QGX_KEPT_BLOCK;
        p.codes = a.codes + row * a.code_place + at.c;
        p.powers = a.powers + row * a.power_place + block;
        p.place = a.code_place;
        p.power_place = a.power_place;
        p.cut = (block + 1) * (int)QGX_KEPT_BLOCK - at.c;
    } else {
        p.x = (const T*)a.x + k * a.x_worker + n * a.x_batch + at.c;
        p.place = a.x_place;
    }
    return p;
}

template <typename T>
__device__ __forceinline__ Places<T, false> gradients_of(const GroupArgs& a, uint32_t sample, uint32_t batch, ChannelsAt at)
{
    Places<T, false> p{};
    p.x = (const T*)a.dy + sample / batch * a.dy_worker + sample % batch * a.dy_batch + at.c;
    p.place = a.dy_place;
    return p;
}

template <typename T, bool KEPT, bool SHORT>
__device__ __forceinline__ RawPiece<T, KEPT> load_place(const Places<T, KEPT>& p, uint32_t place, int n)
{
    constexpr int W = kPiece<T>;
    RawPiece<T, KEPT> raw;
    if constexpr (KEPT) {
        typedef uint32_t Words __attribute__((ext_vector_type(W / 4), aligned(1)));
        const Words w = *reinterpret_cast<const Words*>(p.codes + place * p.place);      // (a row is filled up to 32 codes)
#pragma unroll
        for (int i = 0; i < W / 4; ++i) raw.code[i] = w[i];
        const uint8_t* q = p.powers + place * p.power_place;
        raw.powers = q[0];
        if (p.cut < W && p.cut < n) raw.powers |= (uint32_t)q[1] << 8;
    } else if constexpr (SHORT) {
        raw.bits = __builtin_bit_cast(nt_u32x4, load_raw(p.x + place * p.place, n));
    } else {
        raw.bits = load_bits(p.x + place * p.place);
    }
    return raw;
}

template <typename T, bool KEPT>
__device__ __forceinline__ RawPiece<T, KEPT> no_place()
{
    RawPiece<T, KEPT> raw;
    if constexpr (KEPT) {
#pragma unroll
        for (int i = 0; i < kPiece<T> / 4; ++i) raw.code[i] = 0u;
        raw.powers = 0u;
    } else {
        raw.bits = nt_u32x4{0u, 0u, 0u, 0u};
    }
    return raw;
}

template <typename T, bool KEPT>
__device__ __forceinline__ void values_at(const RawPiece<T, KEPT>& raw, const Places<T, KEPT>& p, float (&v)[kPiece<T>])
{
    if constexpr (KEPT) {
        const float lo = kept_scale(raw.powers & 0xFFu), hi = kept_scale(raw.powers >> 8);
#pragma unroll
        for (int c = 0; c < kPiece<T>; ++c) v[c] = kept_value((raw.code[c / 4] >> (8 * (c & 3))) & 0xFFu, c < p.cut ? lo : hi);
    } else {
        values_of<T>(raw.bits, v);
    }
}

// Keeps the compiler from holding what it has made of a piece across a barrier: it is made again from what was loaded.
template <typename T, bool KEPT>
__device__ __forceinline__ void forget(RawPiece<T, KEPT>& raw)
{
    if constexpr (KEPT) {
#pragma unroll
        for (int i = 0; i < kPiece<T> / 4; ++i) asm volatile("" : "+v"(raw.code[i]));
        asm volatile("" : "+v"(raw.powers));
    } else {
        asm volatile("" : "+v"(raw.bits));
    }
}

template <typename T>
__device__ __forceinline__ void store_place(T* p, ChannelsAt at, const float (&v)[kPiece<T>])
{
    if (at.shift == 0 && at.n >= kPiece<T>) return stream_piece(p, v);
#pragma unroll
    for (int c = 0; c < kPiece<T>; ++c)
        if (at.owns(c)) p[c] = (T)v[c];
}

// A channel's parameter, `none` where there is no such vector.
template <int W>
__device__ __forceinline__ void channel_parameters(const float* p, ChannelsAt at, float none, float (&v)[W])
{
#pragma unroll
    for (int c = 0; c < W; ++c) v[c] = p && c < at.n ? p[at.c + c] : none;
}

// ---- activations ----------------------------------------------------------------------------------------------------------

// 1 / (1 + e^-z).  Binary32 results take the library's exponential, those rounded to 16 bits the hardware's, whose argument z log2 e is
// off by up to 2^-24 of itself (5e-7 of the result at |z| = 5) and whose reciprocal is off by one step.
template <typename T>
__device__ __forceinline__ float sigmoid(float z)
{
    if constexpr (sizeof(T) == 4) return 1.0f / (1.0f + expf(-z));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

template <typename T, int W>
__device__ __forceinline__ void activate(float (&z)[W], int activation, float slope)
{
    if (activation == QGX_ACT_SILU) {
#pragma unroll
        for (int c = 0; c < W; ++c) z[c] = z[c] * sigmoid<T>(z[c]);
    } else if (activation == QGX_ACT_LEAKY) {
#pragma unroll
        for (int c = 0; c < W; ++c) z[c] = z[c] > 0.0f ? z[c] : slope * z[c];
    }
}

// dy -> dz = dy act'(z)
template <typename T, int W>
__device__ __forceinline__ void activate_back(float (&dy)[W], const float (&h)[W], const float (&w)[W], const float (&b)[W], int activation, float slope)
{
    if (activation == QGX_ACT_SILU) {
#pragma unroll
        for (int c = 0; c < W; ++c) {
            const float z = fmaf(h[c], w[c], b[c]), s = sigmoid<T>(z);
            dy[c] *= s * fmaf(z, 1.0f - s, 1.0f);
        }
    } else if (activation == QGX_ACT_LEAKY) {
#pragma unroll
        for (int c = 0; c < W; ++c) {
            const float z = h[c] * w[c] + b[c];
            if (!(z > 0.0f)) dy[c] *= slope;
        }
    }
}

constexpr int kGroupsMost = 256;                           // groups of a workgroup

// ---- sums over a workgroup ------------------------------------------------------------------------------------------------

// The threads' sums of their channels in LDS, M numbers of each, joined over the places: afterwards [M][THREADS * W] with [runs][slots] in each, slot
// j W + c the piece j's channel c.
struct Runs { uint32_t runs, slots; };
template <int THREADS, int W, int M>
__device__ __forceinline__ Runs column_sums(const float (&x)[M][W], uint32_t pieces, float* s)
{
    const uint32_t slots = pieces * W, steps = THREADS / pieces;
    __syncthreads();                                       // (the memory may have been read for the sums before)
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < W / 4; ++h)
            *reinterpret_cast<float4*>(s + (m * THREADS + threadIdx.x) * W + 4 * h) = make_float4(x[m][4 * h], x[m][4 * h + 1], x[m][4 * h + 2], x[m][4 * h + 3]);
    __syncthreads();
    if (slots > THREADS) return Runs{steps, slots};
    const uint32_t runs = THREADS / slots, run = threadIdx.x / slots, col = threadIdx.x % slots;
    float sum[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
        sum[m] = 0.0f;
        if (run < runs)
            for (uint32_t i = run; i < steps; i += runs) sum[m] += s[m * THREADS * W + i * slots + col];
    }
    __syncthreads();
    if (run < runs)
#pragma unroll
        for (int m = 0; m < M; ++m) s[m * THREADS * W + threadIdx.x] = sum[m];          // run * slots + col
    __syncthreads();
    return Runs{runs, slots};
}

template <int W, bool SHORT>
__device__ __forceinline__ uint32_t slot_of(uint32_t channel, uint32_t pieces, uint32_t span)
{
    return SHORT || channel < (pieces - 1u) * W ? channel : channel + pieces * W - span;
}

// Every group's sums of what column_sums left, each times its channel's weight: out[m][group].  A wave takes a group.
template <int THREADS, int W, bool SHORT, int M>
__device__ __forceinline__ void group_sums(Runs r, uint32_t pieces, uint32_t span, uint32_t per, const float* weight, const float* s, float (*out)[kGroupsMost])
{
    const uint32_t groups = span / per, n = r.runs * per;
    for (uint32_t g = wave_id(); g < groups; g += THREADS / kWave) {
        float sum[M];
#pragma unroll
        for (int m = 0; m < M; ++m) sum[m] = 0.0f;
        for (uint32_t i = lane_id(); i < n; i += kWave) {
            const uint32_t c = g * per + i % per, at = i / per * r.slots + slot_of<W, SHORT>(c, pieces, span);
            const float w = weight ? weight[c] : 1.0f;
#pragma unroll
            for (int m = 0; m < M; ++m) sum[m] = fmaf(s[m * THREADS * W + at], w, sum[m]);
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            sum[m] = lanes_sum<kWave>(sum[m]);
            if (lane_id() == 0) out[m][g] = sum[m];
        }
    }
    __syncthreads();
}

// ---- forward, whole groups ------------------------------------------------------------------------------------------------

template <typename T, int THREADS, int N, bool SHORT>
__global__ __launch_bounds__(THREADS) void k_group_norm(GroupArgs a, uint32_t batch)
{
    constexpr int W = kPiece<T>;
    __shared__ __align__(16) float s_sums[THREADS * W];
    __shared__ float s_mean[1][kGroupsMost], s_rstd[1][kGroupsMost];
    const uint32_t unit = unit_of_block(blockIdx.x, a.units), sample = unit / a.spans, first = unit % a.spans * a.span;
    const uint32_t span = min(a.span, a.channels - first), pieces = SHORT ? 1u : (span + W - 1u) / W, steps = THREADS / pieces;
    const uint32_t j = threadIdx.x % pieces, step = threadIdx.x / pieces;
    const bool any = step < steps;
    const ChannelsAt at = channels_at<W, SHORT>(j, first, span);
    const Places<T, false> places = places_of<T, false>(a, sample, batch, at);
    const float n = (float)a.places * (float)a.per;
    RawPiece<T, false> raw[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t p = i * steps + step;
        raw[i] = any && p < a.places ? load_place<T, false, SHORT>(places, p, at.n) : no_place<T, false>();
    }
    float sum[1][W];
#pragma unroll
    for (int c = 0; c < W; ++c) sum[0][c] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[W];
        values_at(raw[i], places, v);
#pragma unroll
        for (int c = 0; c < W; ++c) sum[0][c] += v[c];
    }
#pragma unroll
    for (int c = 0; c < W; ++c) sum[0][c] = at.owns(c) ? sum[0][c] : 0.0f;
    Runs r = column_sums<THREADS, W, 1>(sum, pieces, s_sums);
    group_sums<THREADS, W, SHORT, 1>(r, pieces, span, a.per, nullptr, s_sums, s_mean);
    float mean[W], rstd[W];
#pragma unroll
    for (int c = 0; c < W; ++c) {
        mean[c] = s_mean[0][min((uint32_t)(at.c + c) - first, span - 1u) / a.per] / n;
        sum[0][c] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool ok = any && i * steps + step < a.places;
        float v[W];
        forget(raw[i]);
        values_at(raw[i], places, v);
#pragma unroll
        for (int c = 0; c < W; ++c) {
            const float t = ok ? v[c] - mean[c] : 0.0f;
            sum[0][c] = fmaf(t, t, sum[0][c]);
        }
    }
#pragma unroll
    for (int c = 0; c < W; ++c) sum[0][c] = at.owns(c) ? sum[0][c] : 0.0f;
    r = column_sums<THREADS, W, 1>(sum, pieces, s_sums);
    group_sums<THREADS, W, SHORT, 1>(r, pieces, span, a.per, nullptr, s_sums, s_rstd);
    const uint32_t own_groups = span / a.per;
    for (uint32_t g = threadIdx.x; g < own_groups; g += THREADS) {
        const size_t to = (size_t)sample * a.groups + first / a.per + g;
        if (a.mean) a.mean[to] = s_mean[0][g] / n;
        if (a.rstd) a.rstd[to] = 1.0f / sqrtf(s_rstd[0][g] / n + a.eps);
    }
    float w[W], b[W];
    channel_parameters<W>(a.w, at, 1.0f, w);
    channel_parameters<W>(a.b, at, 0.0f, b);
#pragma unroll
    for (int c = 0; c < W; ++c) rstd[c] = 1.0f / sqrtf(s_rstd[0][min((uint32_t)(at.c + c) - first, span - 1u) / a.per] / n + a.eps);
    T* y = (T*)a.y + sample / batch * a.y_worker + sample % batch * a.y_batch + at.c;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t p = i * steps + step;
        if (!any || p >= a.places) continue;
        float v[W];
        forget(raw[i]);
        values_at(raw[i], places, v);
#pragma unroll
        for (int c = 0; c < W; ++c) v[c] = fmaf((v[c] - mean[c]) * rstd[c], w[c], b[c]);
        activate<T>(v, a.activation, a.slope);
        store_place(y + p * a.y_place, at, v);
    }
}

// ---- backward, whole groups -----------------------------------------------------------------------------------------------

// h and dz of a piece.
template <typename T, bool KEPT>
__device__ __forceinline__ void back_values(const GroupArgs& a, const RawPiece<T, KEPT>& x, const Places<T, KEPT>& places, const RawPiece<T, false>& dy,
                                            const Places<T, false>& grads, const float (&mean)[kPiece<T>], const float (&rstd)[kPiece<T>],
                                            const float (&w)[kPiece<T>], const float (&b)[kPiece<T>], float (&h)[kPiece<T>], float (&dz)[kPiece<T>])
{
    values_at(x, places, h);
    values_at(dy, grads, dz);
#pragma unroll
    for (int c = 0; c < kPiece<T>; ++c) h[c] = (h[c] - mean[c]) * rstd[c];
    activate_back<T>(dz, h, w, b, a.activation, a.slope);
}

template <int W>
__device__ __forceinline__ void statistics_of(const GroupArgs& a, uint32_t sample, ChannelsAt at, float (&mean)[W], float (&rstd)[W])
{
#pragma unroll
    for (int c = 0; c < W; ++c) {
        const size_t g = (size_t)sample * a.groups + min((uint32_t)(at.c + c), a.channels - 1u) / a.per;
        mean[c] = a.mean_in[g];
        rstd[c] = a.rstd_in[g];
    }
}

// Where a workgroup's channels' sums go: in scratch [samples][parts][2][channels], or, where it has all of a worker's places, where they belong.
__device__ __forceinline__ float* channel_sums_at(const GroupArgs& a, uint32_t sample, uint32_t batch, uint32_t part, int which)
{
    if (a.apart) return nullptr;
    if (batch * a.parts == 1u) {
        float* to = which ? a.db : a.dw;
        return to ? to + sample * a.param_stride : nullptr;
    }
    return (which ? a.db : a.dw) ? a.scratch + (((size_t)sample * a.parts + part) * 2u + which) * a.channels : nullptr;
}

// Small tensors: the parameters' gradients of four pieces' channels by a workgroup of their own, from dy and x once more (from the cache): no scratch and
// no second launch, which would take longer.  A worker's samples and places are dealt to THREADS / 4 threads for each piece.  s: [2][THREADS][W].
template <typename T, int THREADS, bool KEPT>
__device__ __forceinline__ void parameters_apart(const GroupArgs& a, uint32_t batch, uint32_t block, float* s)
{
    constexpr int W = kPiece<T>;
    constexpr uint32_t kRuns = THREADS / 4;
    const uint32_t columns = (a.channels + 4u * W - 1u) / (4u * W), k = block / columns, first = block % columns * 4u * W;
    const uint32_t piece = threadIdx.x % 4u, run = threadIdx.x / 4u, span = min(4u * W, a.channels - first), pieces = (span + W - 1u) / W;
    const ChannelsAt at = channels_at<W, false>(min(piece, pieces - 1u), first, span);
    float w[W], b[W], sum[2][W];
    channel_parameters<W>(a.w, at, 1.0f, w);
    channel_parameters<W>(a.b, at, 0.0f, b);
#pragma unroll
    for (int c = 0; c < W; ++c) sum[0][c] = sum[1][c] = 0.0f;
    const uint32_t rows = batch * a.places;
#pragma unroll 4
    for (uint32_t r = run; r < rows; r += kRuns) {
        const uint32_t sample = k * batch + r / a.places, p = r % a.places;
        const Places<T, KEPT> places = places_of<T, KEPT>(a, sample, batch, at);
        const Places<T, false> grads = gradients_of<T>(a, sample, batch, at);
        const RawPiece<T, KEPT> x = load_place<T, KEPT, false>(places, p, W);
        const RawPiece<T, false> dy = load_place<T, false, false>(grads, p, W);
        float mean[W], rstd[W], h[W], dz[W];
        statistics_of<W>(a, sample, at, mean, rstd);
        back_values<T, KEPT>(a, x, places, dy, grads, mean, rstd, w, b, h, dz);
#pragma unroll
        for (int c = 0; c < W; ++c) {
            sum[0][c] = fmaf(dz[c], h[c], sum[0][c]);
            sum[1][c] += dz[c];
        }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int c = 0; c < W; ++c) s[(m * THREADS + threadIdx.x) * W + c] = sum[m][c];
    __syncthreads();
    // eight threads to a sum: a run of the threads' each, then those in a tree
    const uint32_t which = threadIdx.x / (THREADS / 2), each = threadIdx.x % (THREADS / 2), share = each % 8u;
    float* to = which ? a.db : a.dw;
    for (uint32_t c = each / 8u; c < 4u * W; c += THREADS / 16) {
        const uint32_t j = c / W, lane = c % W;
        float t = 0.0f;
        for (uint32_t i = share; i < kRuns; i += 8u) t += s[(which * THREADS + i * 4u + j) * W + lane];
        t = __uint_as_float(xor_lane<1>(__float_as_uint(t))) + t;
        t = __uint_as_float(xor_lane<2>(__float_as_uint(t))) + t;
        t += __shfl_xor(t, 4, 64);
        const int channel = min((int)(j * W), (int)span - W) + (int)lane;              // of the span, where the piece lies
        if (to && share == 0u && j < pieces && (int)lane >= (int)(j * W) - min((int)(j * W), (int)span - W)) to[k * a.param_stride + first + channel] = t;
    }
}

template <typename T, int THREADS, int N, bool KEPT, bool SHORT>
__global__ __launch_bounds__(THREADS) void k_group_norm_back(GroupArgs a, uint32_t batch)
{
    constexpr int W = kPiece<T>;
    __shared__ __align__(16) float s_sums[2 * THREADS * W];
    __shared__ float s_group[2][kGroupsMost];
    if constexpr (THREADS == 256)
        if (a.apart && blockIdx.x >= a.units) return parameters_apart<T, THREADS, KEPT>(a, batch, blockIdx.x - a.units, s_sums);
    const uint32_t unit = unit_of_block(blockIdx.x, a.units), sample = unit / a.spans, first = unit % a.spans * a.span;
    const uint32_t span = min(a.span, a.channels - first), pieces = SHORT ? 1u : (span + W - 1u) / W, steps = THREADS / pieces;
    const uint32_t j = threadIdx.x % pieces, step = threadIdx.x / pieces;
    const bool any = step < steps;
    const ChannelsAt at = channels_at<W, SHORT>(j, first, span);
    const Places<T, KEPT> places = places_of<T, KEPT>(a, sample, batch, at);
    const Places<T, false> grads = gradients_of<T>(a, sample, batch, at);
    RawPiece<T, KEPT> x[N];
    RawPiece<T, false> dy[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t p = i * steps + step;
        const bool ok = any && p < a.places;
        x[i] = ok ? load_place<T, KEPT, SHORT>(places, p, at.n) : no_place<T, KEPT>();
        dy[i] = ok ? load_place<T, false, SHORT>(grads, p, at.n) : no_place<T, false>();
    }
    float mean[W], rstd[W], w[W], b[W], dw[W], db[W];
    statistics_of<W>(a, sample, at, mean, rstd);
    channel_parameters<W>(a.w, at, 1.0f, w);
    channel_parameters<W>(a.b, at, 0.0f, b);
#pragma unroll
    for (int c = 0; c < W; ++c) dw[c] = db[c] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float h[W], dz[W];
        back_values<T, KEPT>(a, x[i], places, dy[i], grads, mean, rstd, w, b, h, dz);
        const bool ok = any && i * steps + step < a.places;        // (a place that is none: dz is 0, h may be anything)
#pragma unroll
        for (int c = 0; c < W; ++c) {
            dw[c] = ok ? fmaf(dz[c], h[c], dw[c]) : dw[c];
            db[c] = ok ? db[c] + dz[c] : db[c];
            asm volatile("" : "+v"(dw[c]), "+v"(db[c]));
        }
    }
    const float* weight = a.w ? a.w + first : nullptr;
    float sum[2][W];
#pragma unroll
    for (int c = 0; c < W; ++c) {
        sum[0][c] = at.owns(c) ? dw[c] : 0.0f;
        sum[1][c] = at.owns(c) ? db[c] : 0.0f;
    }
    const Runs r = column_sums<THREADS, W, 2>(sum, pieces, s_sums);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* to = channel_sums_at(a, sample, batch, 0u, which);
        if (to)
            for (uint32_t c = threadIdx.x; c < span; c += THREADS) {
                float t = 0.0f;
                for (uint32_t i = 0; i < r.runs; ++i) t += s_sums[which * THREADS * W + i * r.slots + slot_of<W, SHORT>(c, pieces, span)];
                to[first + c] = t;
            }
    }
    if (a.y) group_sums<THREADS, W, SHORT, 2>(r, pieces, span, a.per, weight, s_sums, s_group);
    if (!a.y) return;
    const float n = (float)a.places * (float)a.per;
    float minus_m1[W], minus_m2[W];
#pragma unroll
    for (int c = 0; c < W; ++c) {
        const uint32_t g = min((uint32_t)(at.c + c) - first, span - 1u) / a.per;
        minus_m2[c] = -(s_group[0][g] / n);
        minus_m1[c] = -(s_group[1][g] / n);
    }
    T* dx = (T*)a.y + sample / batch * a.y_worker + sample % batch * a.y_batch + at.c;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t p = i * steps + step;
        if (!any || p >= a.places) continue;
        float h[W], dz[W];
        forget(x[i]);
        forget(dy[i]);
        back_values<T, KEPT>(a, x[i], places, dy[i], grads, mean, rstd, w, b, h, dz);
#pragma unroll
        for (int c = 0; c < W; ++c) dz[c] = rstd[c] * fmaf(h[c], minus_m2[c], fmaf(dz[c], w[c], minus_m1[c]));
        store_place(dx + p * a.y_place, at, dz);
    }
}

// ---- whole groups, whose pieces lie in one group each ---------------------------------------------------------------------
// Where a group's channels are whole pieces and a span has 1, 2, 4 .. 64 of them, a thread has one group: its sum is one number, joined
// with the lanes of its piece in registers and with the waves through LDS, one barrier a sum.

template <int D, int M>
__device__ __forceinline__ void join_lanes(float (&x)[M])
{
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const LanePair p = lane_pair<D>(__float_as_uint(x[m]));
        x[m] = __uint_as_float(p.a) + __uint_as_float(p.b);
    }
}

// The sums over the lanes of one piece (lanes that agree in their number mod pieces), in each of them.
template <int M>
__device__ __forceinline__ void piece_sums(float (&x)[M], uint32_t pieces)
{
    if (pieces <= 32u) join_lanes<32>(x);
    if (pieces <= 16u) join_lanes<16>(x);
    if (pieces <= 8u) join_lanes<8>(x);
    if (pieces <= 4u) join_lanes<4>(x);
    if (pieces <= 2u) join_lanes<2>(x);
    if (pieces <= 1u) join_lanes<1>(x);
}

// The sums over the threads of a group, of M numbers.  s: LDS of these sums' own, [M][64][THREADS / 64].
template <int THREADS, int M>
__device__ __forceinline__ void one_group_sums(float (&x)[M], uint32_t pieces, uint32_t group_pieces, float* s)
{
    constexpr uint32_t kWaves = THREADS / kWave;
    piece_sums(x, pieces);
    if (lane_id() < (int)pieces)
#pragma unroll
        for (int m = 0; m < M; ++m) s[(m * kWave + lane_id()) * kWaves + wave_id()] = x[m];
    __syncthreads();
    const uint32_t first = threadIdx.x % pieces / group_pieces * group_pieces;
#pragma unroll
    for (int m = 0; m < M; ++m) {
        x[m] = 0.0f;
        for (uint32_t p = 0; p < group_pieces; ++p)
#pragma unroll
            for (uint32_t w = 0; w < kWaves; w += 4u) {
                const float4 y = *reinterpret_cast<const float4*>(s + (m * kWave + first + p) * kWaves + w);
                x[m] += (y.x + y.y) + (y.z + y.w);
            }
    }
}

// A piece's codes and, where its first column is a block's, the power; the lanes of a block are neighbours.
template <typename T, int W>
__device__ __forceinline__ void keep_piece(const GroupArgs& a, const RawPiece<T, false>& raw, float (&v)[W], uint32_t channel, uint32_t row, uint32_t call,
                                           const PhiloxKeys& keys, bool ok, Scalars* sc)
{
    uint32_t bits = quad_max(largest_bits<T>(raw.bits));
    if constexpr (W == 4) bits = max(bits, (uint32_t)__builtin_amdgcn_mov_dpp((int)bits, 0x141, 0xf, 0xf, true));       // row_half_mirror: the other four lanes
    uint32_t word[W / 4];
    const uint32_t power = kept_codes<W>(v, bits, a.keep_top, a.draws.on != 0u, channel / 8u, channel / 4u & 1u, row, a.draws.domain, call, keys, word);
    asm volatile("" : : "v"(word[0]));                     // (made before the next piece's is begun)
    if (!ok) return;
    uint8_t* to = a.keep_codes + (size_t)row * a.channels + channel;                    // (whole blocks: rows without a gap)
    if constexpr (W == 8) *reinterpret_cast<uint2*>(to) = make_uint2(word[0], word[1]);
    else *reinterpret_cast<uint32_t*>(to) = word[0];
    if (channel % QGX_KEPT_BLOCK == 0u) {
        a.keep_powers[((size_t)row * a.channels + channel) / QGX_KEPT_BLOCK] = (uint8_t)power;
        if (power == kKeptSpoilt) raise_error(sc, QGX_EBIT_NONFINITE);
    }
}

template <typename T, int THREADS, int N, bool KEEP>
__global__ __launch_bounds__(THREADS, 4) void k_group_norm_one(GroupArgs a, uint32_t batch, Scalars* sc)
{
    constexpr int W = kPiece<T>;
    __shared__ __align__(16) float s_sum[2][kWave * THREADS / kWave];
    const uint32_t unit = unit_of_block(blockIdx.x, a.units), sample = unit / a.spans, first = unit % a.spans * a.span;
    const uint32_t pieces = a.span / W, group_pieces = a.per / W, steps = THREADS / pieces;
    const uint32_t j = threadIdx.x % pieces, step = threadIdx.x / pieces;
    const ChannelsAt at{(int)(first + j * W), 0, W};
    const Places<T, false> places = places_of<T, false>(a, sample, batch, at);
    RawPiece<T, false> raw[N];
#pragma unroll
    for (int i = 0; i < N; ++i) raw[i] = load_place<T, false, false>(places, min(i * steps + step, a.places - 1u), W);
    const float n = (float)a.places * (float)a.per;
    const uint32_t call = KEEP && a.draws.on ? kept_call(a.draws, sc) : 0u;
    const PhiloxKeys keys = philox_keys(a.draws.seed_lo, a.draws.seed_hi);
    float sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t p = i * steps + step;
        forget(raw[i]);
        if constexpr (KEEP) asm volatile("" : "+v"(p));    // (else the draws of all pieces are made side by side, in registers of their own)
        float v[W], t = 0.0f;
        values_at(raw[i], places, v);
#pragma unroll
        for (int c = 0; c < W; ++c) t += v[c];
        sum[0] += p < a.places ? t : 0.0f;
        if constexpr (KEEP) keep_piece<T, W>(a, raw[i], v, (uint32_t)at.c, sample * a.places + p, call, keys, p < a.places, sc);
    }
    one_group_sums<THREADS>(sum, pieces, group_pieces, s_sum[0]);
    const float mean = sum[0] / n;
    sum[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[W], t = 0.0f;
        forget(raw[i]);
        values_at(raw[i], places, v);
#pragma unroll
        for (int c = 0; c < W; ++c) t = fmaf(v[c] - mean, v[c] - mean, t);
        sum[0] += i * steps + step < a.places ? t : 0.0f;
    }
    one_group_sums<THREADS>(sum, pieces, group_pieces, s_sum[1]);
    const float rstd = 1.0f / sqrtf(sum[0] / n + a.eps);
    if (threadIdx.x < pieces && j % group_pieces == 0u) {
        const size_t to = (size_t)sample * a.groups + (first + j * W) / a.per;
        if (a.mean) a.mean[to] = mean;
        if (a.rstd) a.rstd[to] = rstd;
    }
    float w[W], b[W];
    channel_parameters<W>(a.w, at, 1.0f, w);
    channel_parameters<W>(a.b, at, 0.0f, b);
    T* y = (T*)a.y + sample / batch * a.y_worker + sample % batch * a.y_batch + at.c;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t p = i * steps + step;
        float v[W];
        forget(raw[i]);
        values_at(raw[i], places, v);
#pragma unroll
        for (int c = 0; c < W; ++c) v[c] = fmaf((v[c] - mean) * rstd, w[c], b[c]);
        activate<T>(v, a.activation, a.slope);
        if (p < a.places) stream_piece(y + p * a.y_place, v);
    }
}

// h and dz of a piece of one group.  A kept element over its group's spread is one product and one sum of its code, with A = scale rstd and B = (-128 scale - mean)
// rstd (off by 2^-23 of A's 255 steps); `plain`, where the side of 0 decides, and where B (and 128 A with it) may be beyond binary32, as of a nearly constant group
// far from 0 or of a block that holds another group's far larger values too: by the operations the header names.  (Thread by thread: what a group gets is no matter of
// its neighbours.)
template <typename T, bool KEPT>
__device__ __forceinline__ void back_values_one(const GroupArgs& a, const RawPiece<T, KEPT>& x, const Places<T, KEPT>& places, const RawPiece<T, false>& dy,
                                                const Places<T, false>& grads, float mean, float rstd, bool plain, const float (&w)[kPiece<T>],
                                                const float (&b)[kPiece<T>], float (&h)[kPiece<T>], float (&dz)[kPiece<T>])
{
    values_at(dy, grads, dz);
    if constexpr (KEPT) {
        // (one block to a piece: pieces start at multiples of W)
        const float scale = kept_scale(x.powers & 0xFFu);
        const float A = scale * rstd, B = fmaf(-128.0f, scale, -mean) * rstd;
        if (!plain && fabsf(B) < 1e30f) {
#pragma unroll
            for (int c = 0; c < kPiece<T>; ++c) h[c] = fmaf((float)((x.code[c / 4] >> (8 * (c & 3))) & 0xFFu), A, B);
        } else {
#pragma unroll
            for (int c = 0; c < kPiece<T>; ++c) h[c] = (kept_value((x.code[c / 4] >> (8 * (c & 3))) & 0xFFu, scale) - mean) * rstd;
        }
    } else {
        values_at(x, places, h);
#pragma unroll
        for (int c = 0; c < kPiece<T>; ++c) h[c] = (h[c] - mean) * rstd;
    }
    activate_back<T>(dz, h, w, b, a.activation, a.slope);
}

template <typename T, int THREADS, int N, bool KEPT>
__global__ __launch_bounds__(THREADS, 4) void k_group_norm_back_one(GroupArgs a, uint32_t batch)
{
    constexpr int W = kPiece<T>, kWaves = THREADS / kWave;
    __shared__ __align__(16) float s_sum[2 * kWave * kWaves];
    __shared__ float s_channel[2][kWaves][kWave * W];
    if constexpr (THREADS == 256)
        if (a.apart && blockIdx.x >= a.units) return parameters_apart<T, THREADS, KEPT>(a, batch, blockIdx.x - a.units, &s_channel[0][0][0]);
    const uint32_t unit = unit_of_block(blockIdx.x, a.units), sample = unit / a.spans, first = unit % a.spans * a.span;
    const uint32_t pieces = a.span / W, group_pieces = a.per / W, steps = THREADS / pieces;
    const uint32_t j = threadIdx.x % pieces, step = threadIdx.x / pieces;
    const ChannelsAt at{(int)(first + j * W), 0, W};
    const Places<T, KEPT> places = places_of<T, KEPT>(a, sample, batch, at);
    const Places<T, false> grads = gradients_of<T>(a, sample, batch, at);
    RawPiece<T, KEPT> x[N];
    RawPiece<T, false> dy[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t p = min(i * steps + step, a.places - 1u);
        x[i] = load_place<T, KEPT, false>(places, p, W);
        dy[i] = load_place<T, false, false>(grads, p, W);
    }
    // past the last place: the last one's x (another's h might be no number, and so dz) and a dy of zeros, so that nothing is added
    if (a.places != steps * N)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * steps + step >= a.places) dy[i] = no_place<T, false>();
    const size_t g = (size_t)sample * a.groups + (first + j * W) / a.per;
    float w[W], b[W], dw[W], db[W];
    const float one_mean = a.mean_in[g], one_rstd = a.rstd_in[g];
    const bool plain = a.activation == QGX_ACT_LEAKY;
    channel_parameters<W>(a.w, at, 1.0f, w);
    channel_parameters<W>(a.b, at, 0.0f, b);
#pragma unroll
    for (int c = 0; c < W; ++c) dw[c] = db[c] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float h[W], dz[W];
        forget(x[i]);
        forget(dy[i]);
        back_values_one<T, KEPT>(a, x[i], places, dy[i], grads, one_mean, one_rstd, plain, w, b, h, dz);
#pragma unroll
        for (int c = 0; c < W; ++c) {
            dw[c] = fmaf(dz[c], h[c], dw[c]);
            db[c] += dz[c];
            asm volatile("" : "+v"(dw[c]), "+v"(db[c]));
        }
    }
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < W; ++c) {
        sum[0] = fmaf(dw[c], w[c], sum[0]);
        sum[1] = fmaf(db[c], w[c], sum[1]);
    }
    if ((a.dw || a.db) && !a.apart) {
        piece_sums(dw, pieces);
        piece_sums(db, pieces);
        if (lane_id() < (int)pieces)
#pragma unroll
            for (int c = 0; c < W; ++c) {
                s_channel[0][wave_id()][lane_id() * W + c] = dw[c];
                s_channel[1][wave_id()][lane_id() * W + c] = db[c];
            }
    }
    one_group_sums<THREADS>(sum, pieces, group_pieces, s_sum);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* to = channel_sums_at(a, sample, batch, 0u, which);
        if (to)
            for (uint32_t c = threadIdx.x; c < a.span; c += THREADS) {
                float t = s_channel[which][0][c];
#pragma unroll
                for (int i = 1; i < kWaves; ++i) t += s_channel[which][i][c];
                to[first + c] = t;
            }
    }
    if (!a.y) return;
    const float n = (float)a.places * (float)a.per, minus_m2 = -(sum[0] / n), minus_m1 = -(sum[1] / n);
    T* dx = (T*)a.y + sample / batch * a.y_worker + sample % batch * a.y_batch + at.c;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t p = i * steps + step;
        float h[W], dz[W];
        forget(x[i]);
        forget(dy[i]);
        back_values_one<T, KEPT>(a, x[i], places, dy[i], grads, one_mean, one_rstd, plain, w, b, h, dz);
#pragma unroll
        for (int c = 0; c < W; ++c) dz[c] = one_rstd * fmaf(h[c], minus_m2, fmaf(dz[c], w[c], minus_m1));
        if (p < a.places) stream_piece(dx + p * a.y_place, dz);
    }
}

// ---- places dealt to workgroups -------------------------------------------------------------------------------------------
// Workgroup (part, column, sample) has `part` places from part * a.part on of `span` channels.

constexpr int kPartThreads = 256;
constexpr int kPartTurns = 8, kBackTurns = 4;              // places of a thread whose loads are under way together

// Mean and sum of squares about it of every channel over the part's places, [samples][parts][2][channels].
template <typename T, bool SHORT>
__global__ __launch_bounds__(kPartThreads) void k_group_channels(GroupArgs a, uint32_t batch)
{
    constexpr int W = kPiece<T>;
    __shared__ __align__(16) float s_sums[kPartThreads * W];
    const uint32_t sample = blockIdx.z, part = blockIdx.x, first = blockIdx.y * a.span;
    const uint32_t span = min(a.span, a.channels - first), pieces = SHORT ? 1u : (span + W - 1u) / W, steps = kPartThreads / pieces;
    const uint32_t j = threadIdx.x % pieces, step = threadIdx.x / pieces;
    const ChannelsAt at = channels_at<W, SHORT>(j, first, span);
    const Places<T, false> places = places_of<T, false>(a, sample, batch, at);
    const uint32_t p0 = part * a.part, p1 = min(p0 + a.part, a.places);
    float mean[W], m2[W], n = 0.0f;
#pragma unroll
    for (int c = 0; c < W; ++c) mean[c] = m2[c] = 0.0f;
    if (step < steps)
        for (uint32_t p = p0 + step; p < p1; p += steps * kPartTurns) {
            // the turn's own mean and squares first, then joined with those before (Chan, Golub, LeVeque 1979)
            RawPiece<T, false> raw[kPartTurns];
            uint32_t here = 0;
#pragma unroll
            for (int i = 0; i < kPartTurns; ++i) {
                raw[i] = p + i * steps < p1 ? load_place<T, false, SHORT>(places, p + i * steps, at.n) : no_place<T, false>();
                here += p + i * steps < p1;
            }
            float v[kPartTurns][W];
#pragma unroll
            for (int i = 0; i < kPartTurns; ++i) values_at(raw[i], places, v[i]);
            const float one = 1.0f / (float)here, share = (float)here / (n + (float)here);
#pragma unroll
            for (int c = 0; c < W; ++c) {
                float sum = 0.0f, sq = 0.0f;
#pragma unroll
                for (int i = 0; i < kPartTurns; ++i) sum += v[i][c];
                const float mu = sum * one;
#pragma unroll
                for (int i = 0; i < kPartTurns; ++i) {
                    const float t = (uint32_t)i < here ? v[i][c] - mu : 0.0f;
                    sq = fmaf(t, t, sq);
                }
                const float apart = mu - mean[c];
                mean[c] = fmaf(apart, share, mean[c]);
                m2[c] += fmaf(apart * apart, n * share, sq);
            }
            n += (float)here;
        }
    // the threads' joined: sum of n mean, then of the squares about the whole's mean
    float* to = a.scratch + ((size_t)sample * a.parts + part) * 2u * a.channels + first;
    const float total = (float)(p1 - p0);
    float x[1][W];
#pragma unroll
    for (int c = 0; c < W; ++c) x[0][c] = at.owns(c) ? n * mean[c] : 0.0f;
    Runs r = column_sums<kPartThreads, W, 1>(x, pieces, s_sums);
    float all[W];
#pragma unroll
    for (int c = 0; c < W; ++c) {
        all[c] = 0.0f;
        if (at.owns(c))
            for (uint32_t i = 0; i < r.runs; ++i) all[c] += s_sums[i * r.slots + j * W + c];
        all[c] /= total;
        if (step == 0 && at.owns(c)) to[at.c + c - (int)first] = all[c];
    }
#pragma unroll
    for (int c = 0; c < W; ++c) x[0][c] = at.owns(c) ? fmaf((mean[c] - all[c]) * (mean[c] - all[c]), n, m2[c]) : 0.0f;
    r = column_sums<kPartThreads, W, 1>(x, pieces, s_sums);
    if (step == 0)
#pragma unroll
        for (int c = 0; c < W; ++c)
            if (at.owns(c)) {
                float sum = 0.0f;
                for (uint32_t i = 0; i < r.runs; ++i) sum += s_sums[i * r.slots + j * W + c];
                to[a.channels + at.c + c - (int)first] = sum;
            }
}

// The sum over a workgroup of 256 threads, in each.
__device__ __forceinline__ float block_sum(float x, float* s)
{
    x = lanes_sum<kWave>(x);
    if (lane_id() == 0) s[wave_id()] = x;
    __syncthreads();
    x = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    return x;
}

// A group's mean and rstd from its channels' over the parts.
__global__ __launch_bounds__(256) void k_group_join(GroupArgs a)
{
    __shared__ float s[4];
    const uint32_t sample = blockIdx.y, g = blockIdx.x;
    const float* from = a.scratch + (size_t)sample * a.parts * 2u * a.channels + g * a.per;
    const float all = (float)a.places * (float)a.per;
    const uint32_t entries = a.parts * a.per;
    float sum = 0.0f;
    for (uint32_t i = threadIdx.x; i < entries; i += 256u) {
        const uint32_t part = i / a.per, c = i % a.per;
        const float n = (float)min(a.part, a.places - part * a.part);
        sum = fmaf(n, from[(size_t)part * 2u * a.channels + c], sum);
    }
    const float mean = block_sum(sum, s) / all;
    sum = 0.0f;
    for (uint32_t i = threadIdx.x; i < entries; i += 256u) {
        const uint32_t part = i / a.per, c = i % a.per;
        const float* p = from + (size_t)part * 2u * a.channels + c;
        const float n = (float)min(a.part, a.places - part * a.part), apart = p[0] - mean;
        sum += fmaf(apart * apart, n, p[a.channels]);
    }
    const float rstd = 1.0f / sqrtf(block_sum(sum, s) / all + a.eps);
    if (threadIdx.x == 0) {
        const size_t to = (size_t)sample * a.groups + g, groups = (size_t)a.samples * a.groups;
        a.sums[to] = mean;
        a.sums[groups + to] = rstd;
        if (a.mean) a.mean[to] = mean;
        if (a.rstd) a.rstd[to] = rstd;
    }
}

// Samples without places: 0 / 0 each.
__global__ __launch_bounds__(256) void k_group_no_places(GroupArgs a)
{
    const uint64_t n = (uint64_t)a.samples * a.groups;
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256u) {
        if (a.mean) a.mean[i] = __builtin_nanf("");
        if (a.rstd) a.rstd[i] = __builtin_nanf("");
    }
}

template <typename T, bool SHORT>
__global__ __launch_bounds__(kPartThreads) void k_group_apply(GroupArgs a, uint32_t batch)
{
    constexpr int W = kPiece<T>;
    // the last places first: the pass before left them in the cache
    const uint32_t sample = gridDim.z - 1u - blockIdx.z, part = gridDim.x - 1u - blockIdx.x, first = blockIdx.y * a.span;
    const uint32_t span = min(a.span, a.channels - first), pieces = SHORT ? 1u : (span + W - 1u) / W, steps = kPartThreads / pieces;
    const uint32_t j = threadIdx.x % pieces, step = threadIdx.x / pieces;
    if (step >= steps) return;
    const ChannelsAt at = channels_at<W, SHORT>(j, first, span);
    const Places<T, false> places = places_of<T, false>(a, sample, batch, at);
    const uint32_t p0 = part * a.part, p1 = min(p0 + a.part, a.places);
    float mean[W], rstd[W], w[W], b[W];
    statistics_of<W>(a, sample, at, mean, rstd);
    channel_parameters<W>(a.w, at, 1.0f, w);
    channel_parameters<W>(a.b, at, 0.0f, b);
    T* y = (T*)a.y + sample / batch * a.y_worker + sample % batch * a.y_batch + at.c;
    for (uint32_t p = p0 + step; p < p1; p += steps * kPartTurns) {
        RawPiece<T, false> raw[kPartTurns];
#pragma unroll
        for (int i = 0; i < kPartTurns; ++i)
            raw[i] = p + i * steps < p1 ? load_place<T, false, SHORT>(places, p + i * steps, at.n) : no_place<T, false>();
#pragma unroll
        for (int i = 0; i < kPartTurns; ++i) {
            if (p + i * steps >= p1) break;
            float v[W];
            values_at(raw[i], places, v);
#pragma unroll
            for (int c = 0; c < W; ++c) v[c] = fmaf((v[c] - mean[c]) * rstd[c], w[c], b[c]);
            activate<T>(v, a.activation, a.slope);
            store_place(y + (p + i * steps) * a.y_place, at, v);
        }
    }
}

// Sums of dz h and dz of every channel over the part's places.
template <typename T, bool KEPT, bool SHORT>
__global__ __launch_bounds__(kPartThreads) void k_group_back_channels(GroupArgs a, uint32_t batch)
{
    constexpr int W = kPiece<T>;
    __shared__ __align__(16) float s_sums[2 * kPartThreads * W];
    const uint32_t sample = blockIdx.z, part = blockIdx.x, first = blockIdx.y * a.span;
    const uint32_t span = min(a.span, a.channels - first), pieces = SHORT ? 1u : (span + W - 1u) / W, steps = kPartThreads / pieces;
    const uint32_t j = threadIdx.x % pieces, step = threadIdx.x / pieces;
    const ChannelsAt at = channels_at<W, SHORT>(j, first, span);
    const Places<T, KEPT> places = places_of<T, KEPT>(a, sample, batch, at);
    const Places<T, false> grads = gradients_of<T>(a, sample, batch, at);
    const uint32_t p0 = part * a.part, p1 = min(p0 + a.part, a.places);
    float mean[W], rstd[W], w[W], b[W], dw[W], db[W];
    statistics_of<W>(a, sample, at, mean, rstd);
    channel_parameters<W>(a.w, at, 1.0f, w);
    channel_parameters<W>(a.b, at, 0.0f, b);
#pragma unroll
    for (int c = 0; c < W; ++c) dw[c] = db[c] = 0.0f;
    if (step < steps)
        for (uint32_t p = p0 + step; p < p1; p += steps * kBackTurns) {
            RawPiece<T, KEPT> x[kBackTurns];
            RawPiece<T, false> dy[kBackTurns];
#pragma unroll
            for (int i = 0; i < kBackTurns; ++i) {
                const bool ok = p + i * steps < p1;
                x[i] = ok ? load_place<T, KEPT, SHORT>(places, p + i * steps, at.n) : no_place<T, KEPT>();
                dy[i] = ok ? load_place<T, false, SHORT>(grads, p + i * steps, at.n) : no_place<T, false>();
            }
#pragma unroll
            for (int i = 0; i < kBackTurns; ++i) {
                if (p + i * steps >= p1) break;
                float h[W], dz[W];
                back_values<T, KEPT>(a, x[i], places, dy[i], grads, mean, rstd, w, b, h, dz);
#pragma unroll
                for (int c = 0; c < W; ++c) {
                    dw[c] = fmaf(dz[c], h[c], dw[c]);
                    db[c] += dz[c];
                }
            }
        }
    float* to = a.scratch + ((size_t)sample * a.parts + part) * 2u * a.channels;
    float sum[2][W];
#pragma unroll
    for (int c = 0; c < W; ++c) {
        sum[0][c] = at.owns(c) ? dw[c] : 0.0f;
        sum[1][c] = at.owns(c) ? db[c] : 0.0f;
    }
    const Runs r = column_sums<kPartThreads, W, 2>(sum, pieces, s_sums);
#pragma unroll
    for (int which = 0; which < 2; ++which)
        for (uint32_t c = threadIdx.x; c < span; c += kPartThreads) {
            float x = 0.0f;
            for (uint32_t i = 0; i < r.runs; ++i) x += s_sums[which * kPartThreads * W + i * r.slots + slot_of<W, SHORT>(c, pieces, span)];
            to[which * a.channels + first + c] = x;
        }
}

// A group's means of g h and g from its channels' sums.  s: four numbers of LDS.
__device__ __forceinline__ void join_group(const GroupArgs& a, uint32_t sample, uint32_t g, float* s)
{
    const uint32_t entries = a.parts * a.per;
    const float* from = a.scratch + (size_t)sample * a.parts * 2u * a.channels + g * a.per;
    float gh = 0.0f, gs = 0.0f;
    for (uint32_t i = threadIdx.x; i < entries; i += 256u) {
        const uint32_t part = i / a.per, c = i % a.per;
        const float* p = from + (size_t)part * 2u * a.channels + c;
        const float w = a.w ? a.w[g * a.per + c] : 1.0f;
        gh = fmaf(p[0], w, gh);
        gs = fmaf(p[a.channels], w, gs);
    }
    const float all = (float)a.places * (float)a.per;
    gh = block_sum(gh, s);
    gs = block_sum(gs, s);
    if (threadIdx.x == 0) {
        const size_t to = (size_t)sample * a.groups + g, groups = (size_t)a.samples * a.groups;
        a.sums[to] = gh / all;
        a.sums[groups + to] = gs / all;
    }
}

// A worker's parameters' gradients: its samples' and parts' sums, of sixteen channels by sixteen runs side by side.  (Of 64 channels by four, 770 of them took
// 18 us.)  s: [runs][channels].
constexpr uint32_t kJoinChannels = 16, kJoinRuns = 16;
__device__ __forceinline__ void join_parameters(const GroupArgs& a, uint32_t batch, uint32_t k, uint32_t which, uint32_t first, float* s)
{
    const uint32_t i = threadIdx.x % kJoinChannels, run = threadIdx.x / kJoinChannels, c = first + i, entries = batch * a.parts;
    float* to = which ? a.db : a.dw;
    if (!to) return;
    float sum = 0.0f;
    if (c < a.channels) {
        const float* from = a.scratch + ((size_t)k * entries * 2u + which) * a.channels + c;
#pragma unroll 8
        for (uint32_t e = run; e < entries; e += kJoinRuns) sum += from[(size_t)e * 2u * a.channels];
    }
    s[threadIdx.x] = sum;
    __syncthreads();
    if (run == 0 && c < a.channels) {
#pragma unroll
        for (uint32_t r = 1; r < kJoinRuns; ++r) sum += s[r * kJoinChannels + i];
        to[k * a.param_stride + c] = sum;
    }
    __syncthreads();
}

// Both, in one launch: the first `group_blocks` workgroups take the `joins` groups of all samples, the others the parameters of all workers.
__global__ __launch_bounds__(kJoinChannels * kJoinRuns) void k_group_back_join(GroupArgs a, uint32_t batch, uint64_t joins, uint32_t group_blocks, uint64_t columns)
{
    __shared__ float s[kJoinChannels * kJoinRuns];
    if (blockIdx.x < group_blocks) {
        for (uint64_t u = blockIdx.x; u < joins; u += group_blocks) join_group(a, (uint32_t)(u / a.groups), (uint32_t)(u % a.groups), s);
        return;
    }
    const uint32_t each = (a.channels + kJoinChannels - 1u) / kJoinChannels;
    for (uint64_t u = blockIdx.x - group_blocks; u < columns; u += gridDim.x - group_blocks)
        join_parameters(a, batch, (uint32_t)(u / 2u / each), (uint32_t)(u % 2u), (uint32_t)(u / 2u % each) * kJoinChannels, s);
}

template <typename T, bool KEPT, bool SHORT>
__global__ __launch_bounds__(kPartThreads) void k_group_back_apply(GroupArgs a, uint32_t batch)
{
    constexpr int W = kPiece<T>;
    const uint32_t sample = gridDim.z - 1u - blockIdx.z, part = gridDim.x - 1u - blockIdx.x, first = blockIdx.y * a.span;
    const uint32_t span = min(a.span, a.channels - first), pieces = SHORT ? 1u : (span + W - 1u) / W, steps = kPartThreads / pieces;
    const uint32_t j = threadIdx.x % pieces, step = threadIdx.x / pieces;
    if (step >= steps) return;
    const ChannelsAt at = channels_at<W, SHORT>(j, first, span);
    const Places<T, KEPT> places = places_of<T, KEPT>(a, sample, batch, at);
    const Places<T, false> grads = gradients_of<T>(a, sample, batch, at);
    const uint32_t p0 = part * a.part, p1 = min(p0 + a.part, a.places);
    float mean[W], rstd[W], w[W], b[W], minus_m1[W], minus_m2[W];
    statistics_of<W>(a, sample, at, mean, rstd);
    channel_parameters<W>(a.w, at, 1.0f, w);
    channel_parameters<W>(a.b, at, 0.0f, b);
#pragma unroll
    for (int c = 0; c < W; ++c) {
        const size_t g = (size_t)sample * a.groups + min((uint32_t)(at.c + c), a.channels - 1u) / a.per;
        minus_m2[c] = -a.sums[g];
        minus_m1[c] = -a.sums[(size_t)a.samples * a.groups + g];
    }
    T* dx = (T*)a.y + sample / batch * a.y_worker + sample % batch * a.y_batch + at.c;
    for (uint32_t p = p0 + step; p < p1; p += steps * kBackTurns) {
        RawPiece<T, KEPT> x[kBackTurns];
        RawPiece<T, false> dy[kBackTurns];
#pragma unroll
        for (int i = 0; i < kBackTurns; ++i) {
            const bool ok = p + i * steps < p1;
            x[i] = ok ? load_place<T, KEPT, SHORT>(places, p + i * steps, at.n) : no_place<T, KEPT>();
            dy[i] = ok ? load_place<T, false, SHORT>(grads, p + i * steps, at.n) : no_place<T, false>();
        }
#pragma unroll
        for (int i = 0; i < kBackTurns; ++i) {
            if (p + i * steps >= p1) break;
            float h[W], dz[W];
            back_values<T, KEPT>(a, x[i], places, dy[i], grads, mean, rstd, w, b, h, dz);
#pragma unroll
            for (int c = 0; c < W; ++c) dz[c] = rstd[c] * fmaf(h[c], minus_m2[c], fmaf(dz[c], w[c], minus_m1[c]));
            store_place(dx + (p + i * steps) * a.y_place, at, dz);
        }
    }
}

// ---- which kernel ---------------------------------------------------------------------------------------------------------

static uint32_t ceil_div(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1u) / b); }

// Whole groups where a span of at least 64 bytes (or of all channels) has its places in a workgroup's registers: 1024 threads with up to 16 pieces of
// 16 bytes forward, 8 backward (of each of two streams).
GroupPlan group_plan(int dtype, uint32_t workers, uint32_t samples, uint32_t places, uint32_t channels, uint32_t groups, bool backward, uint32_t n_cu)
{
    const uint32_t W = dtype == QGX_F32 ? 4u : 8u, per = channels / groups, most = backward ? 8u : 16u;
    GroupPlan p{};
    p.parts = 1;
    p.part = places;
    if (samples == 0 || places == 0) return p;
    // groups of a workgroup: those of 128 bytes where that leaves two workgroups for every compute unit, else of 64, and of more while there are enough
    // (8 x 16 x 1024 x 256 bfloat16, forward and kept / backward: spans of 64 bytes 63 / 62 us, of 128 56 / 58)
    auto pieces_of = [&](uint32_t n) { return ceil_div((uint64_t)n * per, W); };
    auto fits = [&](uint32_t n) {
        const uint32_t pieces = pieces_of(n);
        return n <= (uint32_t)kGroupsMost && pieces <= 1024u && ceil_div(places, 1024u / pieces) <= most;
    };
    // a piece in one group each, and 1, 2, 4 .. 64 pieces in a span (of all of which there are whole ones)
    auto one = [&](uint32_t n) {
        const uint32_t pieces = pieces_of(n);
        return per % W == 0u && groups % n == 0u && pieces <= 64u && (pieces & (pieces - 1u)) == 0u && per / W <= 8u;
    };
    const uint32_t wide = min(groups, ceil_div(8u * W, per));
    uint32_t of = fits(wide) && (uint64_t)samples * groups >= 2u * n_cu * (uint64_t)wide ? wide : min(groups, ceil_div(4u * W, per));
    if (!one(of) && 2u * of <= groups && one(2u * of) && fits(2u * of)) of *= 2u;
    while (of < groups && 2u * of <= groups && fits(2u * of) && (one(2u * of) || !one(of)) && (uint64_t)samples * (groups / (2u * of)) >= 4u * n_cu) of *= 2u;
    const uint32_t pieces = pieces_of(of);
    uint32_t threads = 1024u;
    for (uint32_t t = 256u; t < 1024u; t *= 2u)
        if (pieces <= t && ceil_div(places, t / pieces) <= most) { threads = t; break; }
    // (few workgroups, each with much to do in threads of several groups: 8 x 2120 x 112 in 16 groups forward 27 us whole, 17 in parts, 7 x 1000 x 144 in 8
    // groups backward 40 and 21; but 32 x 1024 x 320 in 32 groups forward 24 and 29)
    const bool few = !one(of) && threads > 256u && (uint64_t)samples * ceil_div(groups, of) < n_cu;
    if (channels >= W && fits(of) && !few) {
        p.whole = true;
        p.one = one(of);
        p.span = of * per;
        p.spans = ceil_div(groups, of);
        p.threads = threads;
        p.pieces = ceil_div(places, threads / pieces);
    } else {
        p.span = min(channels, 256u * W);                  // (any channels: borders of groups do not matter here)
        p.spans = ceil_div(channels, p.span);
        const uint32_t steps = 256u / ceil_div(p.span, W);
        // two or three workgroups for every compute unit, but a turn for each of them (4 x 65536 x 128 bfloat16 forward, 1, 2, 3, 4 of them: 55, 49, 50,
        // 51 us; 6 x 17332 x 184 binary32 backward 120, 98, 85, 88, 77 since; 20 x 4301 x 30 forward 19, with four turns at least 30)
        const uint32_t want = max(1u, ceil_div((backward ? 3u : 2u) * n_cu, (uint64_t)samples * p.spans));
        p.part = max(ceil_div(places, want), steps * (uint32_t)(backward ? kBackTurns : kPartTurns));
        p.parts = ceil_div(places, p.part);
    }
    // Little in all: the parameters' gradients apart.  (4 x 3 x 221 x 90 binary32 8.9 us, with the sums joined by a launch 11.2; 2 x 11 x 154 x 192 19.9 and
    // 11.8)
    p.apart = p.whole && backward && samples > workers && p.threads == 256u && (uint64_t)samples * places * channels <= (1u << 20) &&
              (uint64_t)(samples / workers) * places <= 1024u;
    const bool sums = !p.whole || (backward && samples > workers && !p.apart);
    p.at_sums = sums ? ((uint64_t)samples * p.parts * 2u * channels + 3u) / 4u * 4u : 0u;
    const uint64_t floats = p.at_sums + (p.whole ? 0u : 2u * (uint64_t)samples * groups);
    p.scratch = floats * sizeof(float);
    return p;
}

static void deal(GroupArgs& a, const GroupPlan& p)
{
    a.span = p.span; a.spans = p.spans; a.parts = p.parts; a.part = p.part;
    a.units = a.samples * p.spans;
    a.apart = p.apart && (a.dw || a.db);
    a.sums = a.scratch ? a.scratch + p.at_sums : nullptr;
}

template <typename T, int THREADS, int N>
static hipError_t launch_whole_as(const GroupArgs& a, uint32_t batch, const GroupPlan& p, Scalars* sc, hipStream_t st)
{
    const dim3 grid(a.samples * a.spans), block(THREADS);
    if (!p.one) hipLaunchKernelGGL((k_group_norm<T, THREADS, N, false>), grid, block, 0, st, a, batch);
    else if (a.keep_codes) hipLaunchKernelGGL((k_group_norm_one<T, THREADS, N, true>), grid, block, 0, st, a, batch, sc);
    else hipLaunchKernelGGL((k_group_norm_one<T, THREADS, N, false>), grid, block, 0, st, a, batch, sc);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_whole(const GroupArgs& a, uint32_t batch, const GroupPlan& p, Scalars* sc, hipStream_t st)
{
    if (p.threads == 256u) {
        if (p.pieces <= 4u) return launch_whole_as<T, 256, 4>(a, batch, p, sc, st);
        return p.pieces <= 8u ? launch_whole_as<T, 256, 8>(a, batch, p, sc, st) : launch_whole_as<T, 256, 16>(a, batch, p, sc, st);
    }
    return p.threads == 512u ? launch_whole_as<T, 512, 16>(a, batch, p, sc, st) : launch_whole_as<T, 1024, 16>(a, batch, p, sc, st);
}

template <typename T, bool SHORT>
static hipError_t launch_forward(GroupArgs& a, uint32_t batch, const GroupPlan& p, Scalars* sc, hipStream_t st)
{
    if constexpr (!SHORT)
        if (p.whole) return launch_whole<T>(a, batch, p, sc, st);
    const dim3 grid(a.parts, a.spans, a.samples);
    hipLaunchKernelGGL((k_group_channels<T, SHORT>), grid, dim3(kPartThreads), 0, st, a, batch);
    hipLaunchKernelGGL(k_group_join, dim3(a.groups, a.samples), dim3(256), 0, st, a);
    a.mean_in = a.sums;
    a.rstd_in = a.sums + (size_t)a.samples * a.groups;
    hipLaunchKernelGGL((k_group_apply<T, SHORT>), grid, dim3(kPartThreads), 0, st, a, batch);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_forward_of(GroupArgs& a, uint32_t batch, const GroupPlan& p, Scalars* sc, hipStream_t st)
{
    return a.channels < (uint32_t)kPiece<T> ? launch_forward<T, true>(a, batch, p, sc, st) : launch_forward<T, false>(a, batch, p, sc, st);
}

bool group_keeps(const GroupPlan& plan, uint32_t channels) { return plan.one && plan.span % QGX_KEPT_BLOCK == 0u && channels % QGX_KEPT_BLOCK == 0u; }

hipError_t launch_group_no_places(const GroupArgs& a, hipStream_t st)
{
    const uint64_t n = (uint64_t)a.samples * a.groups;
    if (n == 0u || (!a.mean && !a.rstd)) return hipSuccess;
    hipLaunchKernelGGL(k_group_no_places, dim3(ceil_div(n < (1ull << 24) ? n : 1ull << 24, 256u)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_group_norm(int dtype, const GroupArgs& args, uint32_t workers, const GroupPlan& plan, Scalars* sc, hipStream_t st)
{
    GroupArgs a = args;
    if (a.samples == 0 || a.places == 0) return hipSuccess;
    deal(a, plan);
    const uint32_t batch = a.samples / workers;
    return dtype == QGX_F32   ? launch_forward_of<float>(a, batch, plan, sc, st)
           : dtype == QGX_F16 ? launch_forward_of<_Float16>(a, batch, plan, sc, st)
                              : launch_forward_of<__bf16>(a, batch, plan, sc, st);
}

template <typename T, int THREADS, int N, bool KEPT>
static hipError_t launch_back_whole_as(const GroupArgs& a, uint32_t batch, const GroupPlan& p, hipStream_t st)
{
    const uint32_t apart = a.apart ? a.samples / batch * ((a.channels + 4u * kPiece<T> - 1u) / (4u * kPiece<T>)) : 0u;
    const dim3 grid(a.units + apart), block(THREADS);
    if (p.one) hipLaunchKernelGGL((k_group_norm_back_one<T, THREADS, N, KEPT>), grid, block, 0, st, a, batch);
    else hipLaunchKernelGGL((k_group_norm_back<T, THREADS, N, KEPT, false>), grid, block, 0, st, a, batch);
    return hipGetLastError();
}

template <typename T, bool KEPT>
static hipError_t launch_back_whole(const GroupArgs& a, uint32_t batch, const GroupPlan& p, hipStream_t st)
{
    if (p.threads == 256u) return p.pieces <= 4u ? launch_back_whole_as<T, 256, 4, KEPT>(a, batch, p, st) : launch_back_whole_as<T, 256, 8, KEPT>(a, batch, p, st);
    return p.threads == 512u ? launch_back_whole_as<T, 512, 8, KEPT>(a, batch, p, st) : launch_back_whole_as<T, 1024, 8, KEPT>(a, batch, p, st);
}

// The groups' sums (of parts) and the parameters'.
static void launch_join(const GroupArgs& a, uint32_t batch, bool parts, hipStream_t st)
{
    const uint64_t joins = parts && a.y ? (uint64_t)a.samples * a.groups : 0u;
    const uint64_t columns = a.dw || a.db ? 2u * (uint64_t)a.workers * ((a.channels + kJoinChannels - 1u) / kJoinChannels) : 0u;
    const uint32_t most = 1u << 22, group_blocks = (uint32_t)(joins < most ? joins : most), blocks = group_blocks + (uint32_t)(columns < most ? columns : most);
    if (blocks) hipLaunchKernelGGL(k_group_back_join, dim3(blocks), dim3(kJoinChannels * kJoinRuns), 0, st, a, batch, joins, group_blocks, columns);
}

template <typename T, bool KEPT, bool SHORT>
static hipError_t launch_back(const GroupArgs& a, uint32_t batch, const GroupPlan& p, hipStream_t st)
{
    if constexpr (!SHORT)
        if (p.whole) return launch_back_whole<T, KEPT>(a, batch, p, st);
    const dim3 grid(a.parts, a.spans, a.samples);
    hipLaunchKernelGGL((k_group_back_channels<T, KEPT, SHORT>), grid, dim3(kPartThreads), 0, st, a, batch);
    launch_join(a, batch, true, st);
    if (a.y) hipLaunchKernelGGL((k_group_back_apply<T, KEPT, SHORT>), grid, dim3(kPartThreads), 0, st, a, batch);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_back_of(const GroupArgs& a, uint32_t batch, const GroupPlan& p, hipStream_t st)
{
    const bool few = a.channels < (uint32_t)kPiece<T>;
    if (a.x) return few ? launch_back<T, false, true>(a, batch, p, st) : launch_back<T, false, false>(a, batch, p, st);
    return few ? launch_back<T, true, true>(a, batch, p, st) : launch_back<T, true, false>(a, batch, p, st);
}

hipError_t launch_group_norm_back(int dtype, const GroupArgs& args, uint32_t workers, const GroupPlan& plan, hipStream_t st)
{
    GroupArgs a = args;
    if (!a.y && !a.dw && !a.db) return hipSuccess;
    deal(a, plan);
    a.workers = workers;
    if (a.apart && !a.y) a.units = 0u;                     // no groups' workgroups
    const uint32_t batch = a.samples / workers;
    if (batch && a.places) {
        const hipError_t e = dtype == QGX_F32   ? launch_back_of<float>(a, batch, plan, st)
                             : dtype == QGX_F16 ? launch_back_of<_Float16>(a, batch, plan, st)
                                                : launch_back_of<__bf16>(a, batch, plan, st);
        if (e != hipSuccess) return e;
    }
    // (parts: made in the launch that joins them; no samples or places: sums of nothing)
    if (!plan.whole && batch && a.places) return hipSuccess;
    if (plan.whole && (batch == 1u || plan.apart)) return hipSuccess;
    launch_join(a, a.places ? batch : 0u, false, st);
    return hipGetLastError();
}

}  // namespace qgx
