// Rotation of queries and keys by their positions:  of each head the first `rot` values are rot / 2 pairs, pair i of token t
// turns by the angle 2 pi position_t turns_i / 2^64 and is multiplied with the amplitude; values behind them stay.  The
// gradient is the turn back (inverse), with the same amplitude.
//
// turns_i is a position's share of a whole turn as 64 binary places behind the point: the product wraps at whole turns by
// itself, so the angle at position 2^31 is as exact as at position 1 (2^-34 of a turn), where a binary32 angle would be off
// by whole turns.  The angle is then brought to an eighth of a turn round the nearest quarter and enters two Taylor sums
// (sine to the ninth power, cosine to the tenth: 2e-9 and 2e-10 at pi/4).
//
// Bound by memory.  A workgroup has a few tokens, forms the sines of their pairs once, in LDS, and has each thread turn up to
// four pieces of 2 x 8 values, all of them fetched before the first is stored.  16384 tokens of 24 heads of 64 in bfloat16 take
// 25.5 us, 20 of them in the kernel (5.0 TB/s); with the sines formed by every thread 27, of which the sines were most.
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

template <typename T, bool INTERLEAVED, int PIECES>
__global__ __launch_bounds__(kBlock) void k_rotary(Rotary a, const T* x, T* out)
{
    __shared__ __attribute__((aligned(16))) float table[2][kTable];   // cosines, sines
    const int64_t token0 = (int64_t)blockIdx.x * a.tokens;
    const int tokens = (int)min((int64_t)a.tokens, a.n - token0), half = a.rot >> 1;

    // pieces are numbered by token, head and place in the head
    struct Piece {
        const T* from;
        T* to;
        int at1, count0, count1, pair;   // second run behind the first; lengths of both; place in the table, -1 of what stays
    } piece[PIECES];
    float v[PIECES][16];
    const int per = a.heads * a.units;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int n = (blockIdx.y * PIECES + i) * kBlock + threadIdx.x, t = n / per, in = n - t * per, h = in / a.units, unit = in - h * a.units;
        Piece& p = piece[i];
        p.count0 = 0;
        if (t >= tokens) continue;
        const bool turns = unit < a.rot_units;
        int at;
        if (turns && !INTERLEAVED) {
            at = unit * 8, p.at1 = half;
            p.count0 = p.count1 = min(8, half - at);
        } else {
            at = turns ? unit * 16 : a.rot + (unit - a.rot_units) * 16, p.at1 = 8;
            const int end = turns ? a.rot : a.dim;
            p.count0 = min(8, end - at), p.count1 = max(0, min(8, end - at - 8));
        }
        p.pair = turns ? t * a.pairs + unit * 8 : -1;
        p.from = x + (token0 + t) * a.ldx + h * a.dim + at;
        p.to = out + (token0 + t) * a.ldo + h * a.dim + at;
        load8(p.from, p.count0, v[i]);
        load8(p.from + p.at1, p.count1, v[i] + 8);
    }
    for (int n = threadIdx.x; n < tokens * a.pairs; n += kBlock) {
        const int t = n / a.pairs, pair = min(n - t * a.pairs, half - 1);   // places behind the last pair are read, not used
        const int64_t position = a.wide ? static_cast<const int64_t*>(a.positions)[token0 + t] : static_cast<const int32_t*>(a.positions)[token0 + t];
        const uint64_t phase = (uint64_t)position * a.turns[pair];
        turn(a.inverse ? 0 - phase : phase, a.amplitude, table[0][n], table[1][n]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const Piece& p = piece[i];
        if (p.count0 == 0) continue;
        if (p.pair >= 0) {
            float c[8], s[8];
            load8(&table[0][p.pair], 8, c);
            load8(&table[1][p.pair], 8, s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float& p0 = INTERLEAVED ? v[i][2 * e] : v[i][e];
                float& p1 = INTERLEAVED ? v[i][2 * e + 1] : v[i][8 + e];
                const float was = p0;
                p0 = fmaf(was, c[e], -(p1 * s[e]));
                p1 = fmaf(was, s[e], p1 * c[e]);
            }
        }
        store8(p.to, p.count0, v[i]);
        store8(p.to + p.at1, p.count1, v[i] + 8);
    }
}

template <typename T, int PIECES>
void launch(const Rotary& a, const RotaryCall& c, int64_t token, dim3 grid, hipStream_t stream)
{
    const T* x = static_cast<const T*>(c.x) + token * c.ldx;
    T* out = static_cast<T*>(c.out) + token * c.ldo;
    if (c.interleaved)
        k_rotary<T, true, PIECES><<<grid, kBlock, 0, stream>>>(a, x, out);
    else
        k_rotary<T, false, PIECES><<<grid, kBlock, 0, stream>>>(a, x, out);
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
    // Many tokens: as many a workgroup as have four pieces a thread and whose sines fit.  Few: a piece a thread, more workgroups.
    const int per = a.heads * a.units, pieces = c.n * per >= 524288 ? 4 : 1;
    a.tokens = std::max(1, std::min(kBlock * pieces / per, kTable / a.pairs));
    // 2^23 workgroups a launch: a grid has fewer than 2^32 threads
    for (int64_t token = 0; token < c.n; token += (int64_t)a.tokens << 23) {
        a.n = std::min(c.n - token, (int64_t)a.tokens << 23);
        a.positions = static_cast<const char*>(c.positions) + token * (c.wide_ids ? 8 : 4);
        const dim3 grid((uint32_t)((a.n + a.tokens - 1) / a.tokens), (uint32_t)((a.tokens * per + kBlock * pieces - 1) / (kBlock * pieces)));
        if (pieces == 4)
            c.bf16 ? launch<uint16_t, 4>(a, c, token, grid, stream) : launch<float, 4>(a, c, token, grid, stream);
        else
            c.bf16 ? launch<uint16_t, 1>(a, c, token, grid, stream) : launch<float, 1>(a, c, token, grid, stream);
    }
    return hipGetLastError();
}

}  // namespace agc
