// Rotation of queries and keys by their positions:  of each head the first `rot` values are rot / 2 pairs, pair i of token t
// turns by the angle 2 pi position_t turns_i / 2^64 and is multiplied with the amplitude; values behind them stay.  The
// gradient is the turn back (inverse), with the same amplitude.
//
// turns_i is a position's share of a whole turn as 64 binary places behind the point: the product wraps at whole turns by
// itself, so the angle at position 2^31 is as exact as at position 1, where a binary32 angle would be off by whole turns.  The
// angle is then brought to an eighth of a turn round the nearest quarter, rounded to binary32, and enters two Taylor sums
// (sine to the ninth power, cosine to the tenth: 2e-9 and 2e-10 at pi/4).
//
// Bound by memory.  A workgroup has a few tokens; each thread fetches a piece of 2 x 8 values, the sines of all pairs are formed
// meanwhile, once for all heads, in LDS, and the pieces turn.  16384 tokens of 24 heads of 64 in bfloat16 take 23 us, 4.4 TB/s
// (131072 of 8 heads 45.5, 5.9 TB/s); with the sines formed by every thread 27, with four pieces a thread and fewer waves 25.5.
#include <algorithm>

#include "agc_operators.h"
#include "agc_vector.h"

namespace agc {

namespace {

constexpr int kBlock = 256;

constexpr int kTable = kMostRotary / 2;   // pairs whose sines fit LDS

struct Rotary {
    int64_t ldx, ldo, n;
    const void* positions;
    const uint64_t* turns;
    int wide, heads, dim, rot;
    int units, rot_units;       // pieces of a head; those of them that turn
    int tokens;                 // of a workgroup
    int pairs;                  // whose sines are in LDS: all of a token's
    float amplitude;
    int inverse;
};

__device__ __forceinline__ void turn(uint64_t phase, float amplitude, float& c, float& s)
{
    const uint32_t quarter = (uint32_t)((phase + ((uint64_t)1 << 61)) >> 62);
    const int64_t rest = (int64_t)(phase - ((uint64_t)quarter << 62));
    // rest = 2^32 top + low with signs of their own, times 2 pi / 2^64: small angles keep their 24 bits too
    const int32_t low = (int32_t)rest, top = (int32_t)(rest >> 32) + (low < 0);
    const float x = fmaf((float)top, 1.4629180793e-9f, (float)low * 3.4061215801e-19f);
    const float y = x * x;
    float sine = fmaf(y, 2.7557319224e-6f, -1.9841269841e-4f);
    sine = fmaf(y, sine, 8.3333333333e-3f);
    sine = fmaf(y, sine, -1.6666666667e-1f);
    sine = fmaf(x * y, sine, x);
    float cosine = fmaf(y, -2.7557319224e-7f, 2.4801587302e-5f);
    cosine = fmaf(y, cosine, -1.3888888889e-3f);
    cosine = fmaf(y, cosine, 4.1666666667e-2f);
    cosine = fmaf(y, cosine, -0.5f);
    cosine = fmaf(y, cosine, 1.0f);
    const float a = quarter & 1 ? sine : cosine, b = quarter & 1 ? cosine : sine;
    c = amplitude * ((quarter + 1) & 2 ? -a : a);
    s = amplitude * (quarter & 2 ? -b : b);
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kBlock) void k_rotary(Rotary a, const T* x, T* out)
{
    extern __shared__ __attribute__((aligned(16))) float cosines[];
    float* const sines = cosines + a.tokens * a.pairs;
    const int64_t token0 = (int64_t)blockIdx.x * a.tokens;
    const int tokens = (int)min((int64_t)a.tokens, a.n - token0), half = a.rot >> 1;

    // pieces are numbered by token, head and place in the head
    const int per = a.heads * a.units, n = blockIdx.y * blockDim.x + threadIdx.x, t = n / per, in = n - t * per, h = in / a.units, unit = in - h * a.units;
    const bool turns = unit < a.rot_units;
    int at, at1, count0 = 0, count1;   // two runs: where they begin and their lengths
    float v[16];
    if (t < tokens) {
        if (turns && !INTERLEAVED) {
            at = unit * 8, at1 = at + half;
            count0 = count1 = min(8, half - at);
        } else {
            at = turns ? unit * 16 : a.rot + (unit - a.rot_units) * 16, at1 = at + 8;
            const int end = turns ? a.rot : a.dim;
            count0 = min(8, end - at), count1 = max(0, min(8, end - at1));
        }
        const T* from = x + (token0 + t) * a.ldx + h * a.dim;
        load8(from + at, count0, v);
        load8(from + at1, count1, v + 8);
    }
    for (int i = threadIdx.x; i < tokens * a.pairs; i += blockDim.x) {
        const int token = i / a.pairs, pair = min(i - token * a.pairs, half - 1);   // places behind the last pair are read, not used
        const int64_t position =
            a.wide ? static_cast<const int64_t*>(a.positions)[token0 + token] : static_cast<const int32_t*>(a.positions)[token0 + token];
        const uint64_t phase = (uint64_t)position * a.turns[pair];
        turn(a.inverse ? 0 - phase : phase, a.amplitude, cosines[i], sines[i]);
    }
    __syncthreads();
    if (count0 == 0) return;
    if (turns) {
        float c[8], s[8];
        load8(cosines + t * a.pairs + unit * 8, 8, c);
        load8(sines + t * a.pairs + unit * 8, 8, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float& p0 = INTERLEAVED ? v[2 * e] : v[e];
            float& p1 = INTERLEAVED ? v[2 * e + 1] : v[8 + e];
            const float was = p0;
            p0 = fmaf(was, c[e], -(p1 * s[e]));
            p1 = fmaf(was, s[e], p1 * c[e]);
        }
    }
    T* to = out + (token0 + t) * a.ldo + h * a.dim;
    store8(to + at, count0, v);
    store8(to + at1, count1, v + 8);
}

template <typename T>
void launch(const Rotary& a, const RotaryCall& c, int64_t token, dim3 grid, int threads, hipStream_t stream)
{
    const size_t lds = (size_t)a.tokens * a.pairs * 2 * sizeof(float);
    const T* x = static_cast<const T*>(c.x) + token * c.ldx;
    T* out = static_cast<T*>(c.out) + token * c.ldo;
    if (c.interleaved)
        k_rotary<T, true><<<grid, threads, lds, stream>>>(a, x, out);
    else
        k_rotary<T, false><<<grid, threads, lds, stream>>>(a, x, out);
}

}  // namespace

hipError_t launch_rotary(const RotaryCall& c, hipStream_t stream)
{
    Rotary a{};
    a.ldx = c.ldx, a.ldo = c.ldo, a.turns = c.turns, a.wide = c.wide_ids;
    a.heads = c.heads, a.dim = c.dim, a.rot = c.rot, a.amplitude = c.amplitude, a.inverse = c.inverse;
    a.rot_units = (c.rot / 2 + 7) / 8;
    a.units = a.rot_units + (c.dim - c.rot + 15) / 16;
    a.pairs = a.rot_units * 8;
    // as many tokens as have a piece a thread and whose sines fit, and no more waves than they need
    const int per = a.heads * a.units;
    a.tokens = std::max(1, std::min(kBlock / per, kTable / a.pairs));
    const int threads = std::min(kBlock, (a.tokens * per + 63) / 64 * 64);
    // 2^23 workgroups a launch: a grid has fewer than 2^32 threads
    for (int64_t token = 0; token < c.n; token += (int64_t)a.tokens << 23) {
        a.n = std::min(c.n - token, (int64_t)a.tokens << 23);
        a.positions = static_cast<const char*>(c.positions) + token * (c.wide_ids ? 8 : 4);
        const dim3 grid((uint32_t)((a.n + a.tokens - 1) / a.tokens), (uint32_t)((a.tokens * per + threads - 1) / threads));
        c.bf16 ? launch<uint16_t>(a, c, token, grid, threads, stream) : launch<float>(a, c, token, grid, threads, stream);
    }
    return hipGetLastError();
}

}  // namespace agc
