// Rotation of queries and keys by their positions:  of each head the first `rot` values are rot / 2 pairs, pair i of token t
// turns by the angle 2 pi position_t turns_i / 2^64 and is multiplied with the amplitude; values behind them stay.  The
// gradient is the turn back (inverse), with the same amplitude.
//
// turns_i is a position's share of a whole turn as 64 binary places behind the point: the product wraps at whole turns by
// itself, so the angle at position 2^31 is as exact as at position 1 (2^-34 of a turn), where a binary32 angle would be off
// by whole turns.  The angle is then brought to an eighth of a turn round the nearest quarter and enters two Taylor sums
// (sine to the ninth power, cosine to the tenth: 2e-9 and 2e-10 at pi/4).
//
// Bound by memory.  A thread owns the same pairs of several heads of a token and forms their sines once.
#include "agc_operators.h"
#include "agc_vector.h"

namespace agc {

namespace {

constexpr int kBlock = 256;

struct Rotary {
    int64_t ldx, ldo, n;
    const void* positions;
    const uint64_t* turns;
    int wide, heads, dim, rot;
    int units, rot_units;       // pieces of 2 x 8 values of a head; those of them that turn
    int lanes_u, lanes_h;       // units and heads that a token's threads work on at once
    int tokens;                 // of a workgroup
    float amplitude;
    int inverse;
};

__device__ __forceinline__ void turn(uint64_t phase, float amplitude, float& c, float& s)
{
    const uint32_t quarter = (uint32_t)((phase + ((uint64_t)1 << 61)) >> 62);
    const int64_t rest = (int64_t)(phase - ((uint64_t)quarter << 62));
    const float x = (float)(int32_t)(rest >> 30) * 3.6572951981e-10f;   // 2 pi / 2^34
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
    const int per = a.lanes_u * a.lanes_h;
    const int sub = threadIdx.x / per, in = threadIdx.x - sub * per;
    const int head0 = in / a.lanes_u, unit = blockIdx.y * a.lanes_u + in - head0 * a.lanes_u;
    const int64_t token = (int64_t)blockIdx.x * a.tokens + sub;
    if (sub >= a.tokens || token >= a.n || unit >= a.units) return;

    const bool turns = unit < a.rot_units;
    const int half = a.rot >> 1;
    // two runs of up to eight values
    int at0, at1, count0, count1;
    if (turns && !INTERLEAVED) {
        at0 = unit * 8, at1 = at0 + half;
        count0 = count1 = min(8, half - at0);
    } else {
        at0 = turns ? unit * 16 : a.rot + (unit - a.rot_units) * 16, at1 = at0 + 8;
        const int end = turns ? a.rot : a.dim;
        count0 = min(8, end - at0), count1 = max(0, min(8, end - at1));
    }
    float c[8], s[8];
    if (turns) {
        const int64_t position = a.wide ? static_cast<const int64_t*>(a.positions)[token] : static_cast<const int32_t*>(a.positions)[token];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint64_t phase = (uint64_t)position * a.turns[min(unit * 8 + i, half - 1)];
            turn(a.inverse ? 0 - phase : phase, a.amplitude, c[i], s[i]);
        }
    }
    const T* from = x + token * a.ldx;
    T* to = out + token * a.ldo;
    for (int h = head0; h < a.heads; h += a.lanes_h) {
        float v[16];
        load8(from + h * a.dim + at0, count0, v);
        load8(from + h * a.dim + at1, count1, v + 8);
        if (turns) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float& p = INTERLEAVED ? v[2 * i] : v[i];
                float& q = INTERLEAVED ? v[2 * i + 1] : v[8 + i];
                const float p0 = p;
                p = fmaf(p0, c[i], -(q * s[i]));
                q = fmaf(p0, s[i], q * c[i]);
            }
        }
        store8(to + h * a.dim + at0, count0, v);
        store8(to + h * a.dim + at1, count1, v + 8);
    }
}

template <typename T>
void launch(const Rotary& a, const RotaryCall& c, dim3 grid, hipStream_t stream)
{
    const T* x = static_cast<const T*>(c.x);
    T* out = static_cast<T*>(c.out);
    if (c.interleaved)
        k_rotary<T, true><<<grid, kBlock, 0, stream>>>(a, x, out);
    else
        k_rotary<T, false><<<grid, kBlock, 0, stream>>>(a, x, out);
}

}  // namespace

hipError_t launch_rotary(const RotaryCall& c, hipStream_t stream)
{
    Rotary a{};
    a.ldx = c.ldx, a.ldo = c.ldo, a.n = c.n, a.positions = c.positions, a.turns = c.turns, a.wide = c.wide_ids;
    a.heads = c.heads, a.dim = c.dim, a.rot = c.rot, a.amplitude = c.amplitude, a.inverse = c.inverse;
    a.rot_units = (c.rot / 2 + 7) / 8;
    a.units = a.rot_units + (c.dim - c.rot + 15) / 16;
    a.lanes_u = a.units < kBlock ? a.units : kBlock;
    const int most = kBlock / a.lanes_u;
    const int rounds = (c.heads + most - 1) / most;
    a.lanes_h = (c.heads + rounds - 1) / rounds;
    a.tokens = kBlock / (a.lanes_u * a.lanes_h);
    const dim3 grid((uint32_t)((c.n + a.tokens - 1) / a.tokens), (uint32_t)((a.units + a.lanes_u - 1) / a.lanes_u));
    c.bf16 ? launch<uint16_t>(a, c, grid, stream) : launch<float>(a, c, grid, stream);
    return hipGetLastError();
}

}  // namespace agc
