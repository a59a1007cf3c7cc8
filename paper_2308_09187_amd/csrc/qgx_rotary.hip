// Rotary positions with several axes: pair p of a head turns by the token's position along the pair's axis times frequency p.
// Bound by memory, one read and one write.  The angles are the same for all heads of a token: a workgroup works out the sines and cosines of
// its tokens once, in LDS, and then streams their heads, 16 bytes of pairs to a thread at a time.  (4 x 16384 tokens of 16 x 128 bfloat16: 94 us, 5.7 TB/s.)
#include "qgx_types.h"

namespace qgx {

constexpr uint32_t kTurnThreads = 256;
constexpr uint32_t kTurnAngles = 2048, kTurnTokens = 64;   // most sines, and tokens, of a workgroup

// Cosine and sine of position * frequency radians.  The product and its turns are sums of two binary64 numbers each, the second what the rounding of the first left
// (by fma, exactly), 1 / (2 pi) too; whole turns go before anything becomes binary32.  So the angle's own size costs 2^-103 of it, 1e-10 of a turn at 1e21 turns.  (In one
// binary64 number it was 5e-8 of a turn at the farthest position of frequency 1.)
__device__ __forceinline__ float2 cos_sin_of(int32_t position, double frequency)
{
    constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;          // 1 / (2 pi)
    const double at = (double)position, angle = at * frequency, angle_rest = fma(at, frequency, -angle);
    const double turns = angle * kTurn, rest = fma(angle, kTurn, -turns) + fma(angle, kTurnRest, angle_rest * kTurn);
    const double left = (turns - rint(turns)) + rest;
    const float r = (float)(left - rint(left));
    float s, c;
    sincospif(2.0f * r, &s, &c);
    return make_float2(c, s);
}

// The frequencies come with the launch; PAIRS: as many as there is room for (the fewer, the sooner a launch is made).
template <int PAIRS> struct Frequencies { double radians[PAIRS]; };

template <int BYTES> struct Bytes { static constexpr int value = BYTES; };
typedef uint32_t Word __attribute__((aligned(2)));         // at any element

// A thread's piece of a head: pairs from the item's first on, or elements that stay as they are.
// REST: of 16-bit elements, where there are some behind the pairs, which are copied as they are (through binary32 a signalling NaN would become a quiet one).
template <typename T, bool NEIGHBOURS, bool REST>
struct HeadPiece {
    static constexpr int W = kPiece<T>;
    uint32_t c;                                            // its first element, in the first half where pairs are apart
    int left;                                              // elements of it that are there
    bool turned;
    float v[W], u[W];
    uint32_t word[4];                                      // of elements that stay: a piece, or runs of 8, 4 and 2 bytes

    // Bit by bit of their number, instead of element by element.  (12 x 3890 tokens of 11 x 78 binary16, neighbours, six elements behind the pairs 61 us, so 41; of
    // binary32, at most three, this is no gain.)
    template <typename F> __device__ __forceinline__ void runs(F&& copy)
    {
        const uint32_t n = (uint32_t)max(left, 0);
        if (n & 4u) {
            copy(c, &word[0], Bytes<4>{});
            copy(c + 2u, &word[1], Bytes<4>{});
        }
        if (n & 2u) copy(c + (n & 4u), &word[2], Bytes<4>{});
        if (n & 1u) copy(c + (n & 6u), &word[3], Bytes<2>{});
    }

    __device__ __forceinline__ void load(const T* in, uint32_t P)
    {
        if (REST && !turned) {
            if (left >= W) {
                const nt_u32x4 x = load_bits(in + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) word[i] = x[i];
                return;
            }
            runs([&](uint32_t at, uint32_t* to, auto bytes) {
                if constexpr (decltype(bytes)::value == 4) *to = *reinterpret_cast<const Word*>(in + at);
                else *to = *reinterpret_cast<const uint16_t*>(in + at);
            });
            return;
        }
        load_piece(in + c, left, v);
        if (!NEIGHBOURS && turned) load_piece(in + P + c, left, u);
    }
    // cs, sn: of the piece's first pair on, 16-byte aligned (what lies past the last pair may be anything)
    __device__ __forceinline__ void turn(const float* cs, const float* sn)
    {
        if (!turned) return;
        constexpr int n = NEIGHBOURS ? W / 2 : W;
        float co[n], si[n];
        if constexpr (n == 2) {
            const float2 x = *reinterpret_cast<const float2*>(cs), y = *reinterpret_cast<const float2*>(sn);
            co[0] = x.x; co[1] = x.y; si[0] = y.x; si[1] = y.y;
        } else {
#pragma unroll
            for (int h = 0; h < n / 4; ++h) {
                const float4 x = *reinterpret_cast<const float4*>(cs + 4 * h), y = *reinterpret_cast<const float4*>(sn + 4 * h);
                co[4 * h] = x.x; co[4 * h + 1] = x.y; co[4 * h + 2] = x.z; co[4 * h + 3] = x.w;
                si[4 * h] = y.x; si[4 * h + 1] = y.y; si[4 * h + 2] = y.z; si[4 * h + 3] = y.w;
            }
        }
#pragma unroll
        for (int j = 0; j < n; ++j) {
            float& x = NEIGHBOURS ? v[2 * j] : v[j];
            float& y = NEIGHBOURS ? v[2 * j + 1] : u[j];
            const float t = fmaf(x, co[j], -(y * si[j]));
            y = fmaf(x, si[j], y * co[j]);
            x = t;
        }
    }
    __device__ __forceinline__ void store(T* out, uint32_t P)
    {
        auto put = [&](T* p, const float (&x)[W]) {
            if (left >= W) stream_piece(p, x);
            else store_piece(p, left, x);
        };
        if (REST && !turned) {
            if (left >= W) {
                *reinterpret_cast<Piece<T>*>(out + c) = __builtin_bit_cast(Piece<T>, nt_u32x4{word[0], word[1], word[2], word[3]});
                return;
            }
            runs([&](uint32_t at, uint32_t* from, auto bytes) {
                if constexpr (decltype(bytes)::value == 4) *reinterpret_cast<Word*>(out + at) = *from;
                else *reinterpret_cast<uint16_t*>(out + at) = (uint16_t)*from;
            });
            return;
        }
        put(out + c, v);
        if (!NEIGHBOURS && turned) put(out + P + c, u);
    }
};

template <typename T, bool NEIGHBOURS, int PAIRS, bool REST>
__global__ __launch_bounds__(kTurnThreads) void k_rotary(RotaryArgs a, Frequencies<PAIRS> f, uint32_t tile_tokens, uint32_t turned, uint32_t items, uint32_t moved)
{
    constexpr int W = kPiece<T>;
    constexpr uint32_t kPairs = NEIGHBOURS ? W / 2 : W;    // of a piece
    __shared__ __align__(16) float s_cos[kTurnAngles], s_sin[kTurnAngles];
    __shared__ uint64_t s_in[kTurnTokens], s_out[kTurnTokens];
    const uint32_t P = a.pairs, stride = (P + 7u) & ~7u;
    for (uint32_t first = blockIdx.x * tile_tokens; first < a.n_tokens; first += gridDim.x * tile_tokens) {
        const uint32_t count = min(tile_tokens, a.n_tokens - first);
        // (piece by piece: the last one's pairs where it has been moved to)
        const uint32_t slots = turned * kPairs;
        for (uint32_t i = threadIdx.x; i < count * slots; i += kTurnThreads) {
            const uint32_t local = i / slots, token = first + local, slot = i % slots, sequence = token / a.tokens, t = token % a.tokens;
            const uint32_t p = min(slot < slots - kPairs ? slot : slot - moved, P - 1u);
            uint32_t axis = 0;
#pragma unroll
            for (uint32_t x = 0; x + 1 < QGX_MAX_AXES; ++x) axis += p >= a.axis_end[x];
            const uint32_t k = sequence / a.batch, n = sequence % a.batch;
            const int32_t at = a.positions[axis * a.p_axis + k * a.p_worker + n * a.p_batch + t];
            const float2 cs = cos_sin_of(at, f.radians[p]);
            s_cos[local * stride + slot] = cs.x;
            s_sin[local * stride + slot] = a.back ? -cs.y : cs.y;
            if (slot == 0u) {
                s_in[local] = k * a.i_worker + n * a.i_batch + t * a.i_token;
                s_out[local] = k * a.o_worker + n * a.o_batch + t * a.o_token;
            }
        }
        __syncthreads();
        // The items of a head (pieces of pairs, the first `turned`, then pieces of what stays) to as many threads, heads and tokens in turn, two at
        // a time: their loads are under way together.
        const uint32_t heads_at_once = items <= kTurnThreads ? kTurnThreads / items : 1u, rows = count * a.heads;
        const uint32_t row0 = threadIdx.x / items, next_token = heads_at_once / a.heads, next_head = heads_at_once % a.heads;
        for (uint32_t item = threadIdx.x % items; item < items && row0 < heads_at_once; item += items <= kTurnThreads ? items : kTurnThreads) {
            HeadPiece<T, NEIGHBOURS, REST> x[2];
            const bool turns = item < turned;
            const uint32_t c = turns ? item * W - (item + 1u == turned ? moved * (W / kPairs) : 0u) : 2u * P + (item - turned) * W, pair = item * kPairs;
            const int left = turns ? (NEIGHBOURS ? (int)(2u * P - c) : (int)(P - c)) : (int)(a.dim - c);
            uint32_t local = row0 / a.heads, head = row0 % a.heads;
            for (uint32_t row = row0; row < rows; row += 2u * heads_at_once) {
                uint32_t where[2];
                T* to[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bool ok = row + j * heads_at_once < rows;
                    where[j] = local * stride + pair;
                    x[j].c = c;
                    x[j].turned = turns;
                    x[j].left = ok ? left : 0;
                    const uint32_t token = min(local, count - 1u);
                    to[j] = (T*)a.out + s_out[token] + head * a.o_head;
                    x[j].load((const T*)a.in + s_in[token] + head * a.i_head, P);
                    if (!ok) where[j] = 0u;
                    local += next_token;
                    head += next_head;
                    if (head >= a.heads) { head -= a.heads; ++local; }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    x[j].turn(s_cos + where[j], s_sin + where[j]);
                    x[j].store(to[j], P);
                }
            }
        }
        __syncthreads();
    }
}

template <typename T, int PAIRS>
static hipError_t launch_rotary_as(const RotaryArgs& a, const double* frequencies, uint32_t n_cu, hipStream_t st)
{
    constexpr uint32_t W = kPiece<T>;
    const uint32_t turned = a.neighbours ? (2u * a.pairs + W - 1u) / W : (a.pairs + W - 1u) / W;
    const uint32_t rest = a.dim - 2u * a.pairs, items = turned + (a.in == a.out ? 0u : (rest + W - 1u) / W);
    const uint32_t most = min(kTurnTokens, kTurnAngles / ((a.pairs + 7u) & ~7u));
    // (more workgroups than find room at once, so that the last ones are short: 4 x 16384 tokens of 16 x 128 bfloat16 117 us with 8 to a compute
    // unit, 107 with 16, 94 with 32, 95 with 64)
    const uint32_t tile = min(most, max(1u, a.n_tokens / (32u * n_cu)));
    const dim3 grid(min((a.n_tokens + tile - 1u) / tile, 1u << 20));
    // The last piece of pairs moved back by so many, to end where they do: some are turned twice, with equal results, and no piece is in part.  Not in
    // place, where the second would turn the first's.  (8 x 4481 tokens of 13 x 102 bfloat16 64 us with the last piece element by element, so 50; 12 x 3890 of 11 x 90
    // neighbours in binary32 75 and 60)
    const uint32_t pairs_of = a.neighbours ? W / 2u : W, moved = a.in != a.out && a.pairs >= pairs_of ? turned * pairs_of - a.pairs : 0u;
    Frequencies<PAIRS> f;
    for (uint32_t p = 0; p < (uint32_t)PAIRS; ++p) f.radians[p] = p < a.pairs ? frequencies[p] : 0.0;
    const dim3 block(kTurnThreads);
    if constexpr (sizeof(T) == 2)
        if (items > turned) {
            if (a.neighbours) hipLaunchKernelGGL((k_rotary<T, true, PAIRS, true>), grid, block, 0, st, a, f, tile, turned, items, moved);
            else hipLaunchKernelGGL((k_rotary<T, false, PAIRS, true>), grid, block, 0, st, a, f, tile, turned, items, moved);
            return hipGetLastError();
        }
    if (a.neighbours) hipLaunchKernelGGL((k_rotary<T, true, PAIRS, false>), grid, block, 0, st, a, f, tile, turned, items, moved);
    else hipLaunchKernelGGL((k_rotary<T, false, PAIRS, false>), grid, block, 0, st, a, f, tile, turned, items, moved);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_rotary_of(const RotaryArgs& a, const double* frequencies, uint32_t n_cu, hipStream_t st)
{
    return a.pairs <= 64u ? launch_rotary_as<T, 64>(a, frequencies, n_cu, st) : launch_rotary_as<T, (int)QGX_MAX_PAIRS>(a, frequencies, n_cu, st);
}

hipError_t launch_rotary(int dtype, const RotaryArgs& a, const double* frequencies, uint32_t n_cu, hipStream_t st)
{
    if (a.n_tokens == 0) return hipSuccess;
    return dtype == QGX_F32   ? launch_rotary_of<float>(a, frequencies, n_cu, st)
           : dtype == QGX_F16 ? launch_rotary_of<_Float16>(a, frequencies, n_cu, st)
                              : launch_rotary_of<__bf16>(a, frequencies, n_cu, st);
}

}  // namespace qgx
