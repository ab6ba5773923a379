// Dropout into a residual:  out = residual + keep * x / (1 - p), keep[r,c] = U[r,c] >= p.  The mask is never stored: U is a
// function of (seed, step, site, r, c), and the gradient is the same call on dout without a residual.
//
// U has 48 bits, as the quantizer's uniforms have: sixteen from a Philox block that eight columns share, and 32 more from a
// second block that is looked at only where the sixteen equal those of p, once in 65536 places.  p is held to 2^-48 that way
// at the cost of sixteen bits a place.  Counter word 1 has bit 30 set, which none of the quantizer's has.
//
// Bound by memory: a thread fetches its eight columns first and forms their block meanwhile.  65536 x 2048 bfloat16 into a
// residual take 135 us, 6.0 TB/s; 16383 x 1501 binary32 values without one 39 us, 5.0 TB/s (a copy of 1 GiB: 5.2).
#include "agc_device.h"
#include "agc_operators.h"
#include "agc_vector.h"

namespace agc {

namespace {

constexpr int kBlock = 256;

struct Dropout {
    int64_t ldx, ldr, ldo;
    Divider groups;            // of eight columns, in a row
    uint32_t items, row0;      // groups of this launch; its first row
    int cols;
    uint32_t site, step_lo, step_hi, key0, key1;
    uint32_t drop16, drop32;   // p in units of 2^-16, and what remains in units of 2^-48
    float scale;
};

template <typename X, typename O, bool RESIDUAL>
__global__ __launch_bounds__(kBlock) void k_dropout(Dropout a, const X* x, const O* residual, O* out)
{
    const uint32_t n = blockIdx.x * kBlock + threadIdx.x;
    if (n >= a.items) return;
    const uint32_t q = a.groups(n);
    const int64_t row = (int64_t)a.row0 + q;
    const int col = (int)(n - q * a.groups.d) * 8, count = min(8, a.cols - col);
    float v[8], r[8];
    load8(x + row * a.ldx + col, count, v);
    if constexpr (RESIDUAL) load8(residual + row * a.ldr + col, count, r);
    uint32_t word[4];
    philox4x32_10(a.site << 16 | (uint32_t)(col >> 3), 1u << 30 | (uint32_t)row, a.step_lo, a.step_hi, a.key0, a.key1, word);
    uint32_t keep = 0, tie = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = e & 1 ? word[e >> 1] >> 16 : word[e >> 1] & 0xFFFFu;
        keep |= u > a.drop16 ? 1u << e : 0u;
        tie |= u == a.drop16 ? 1u << e : 0u;
    }
    if (tie) {
        uint32_t low[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            philox4x32_10(a.site << 16 | (uint32_t)(col >> 2 | h), 3u << 30 | (uint32_t)row, a.step_lo, a.step_hi, a.key0, a.key1, low[h]);
#pragma unroll
        for (int e = 0; e < 8; ++e) keep |= low[e >> 2][e & 3] >= a.drop32 ? tie & 1u << e : 0u;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = keep >> e & 1 ? v[e] * a.scale : 0.0f;   // what is dropped counts for nothing, NaN among it
        if constexpr (RESIDUAL) v[e] += r[e];
    }
    store8(out + row * a.ldo + col, count, v);
}

template <typename X, typename O>
void launch(const Dropout& a, const DropoutCall& c, uint32_t blocks, hipStream_t stream)
{
    const X* x = static_cast<const X*>(c.x);
    const O* residual = static_cast<const O*>(c.residual);
    O* out = static_cast<O*>(c.out);
    if (residual)
        k_dropout<X, O, true><<<blocks, kBlock, 0, stream>>>(a, x, residual, out);
    else
        k_dropout<X, O, false><<<blocks, kBlock, 0, stream>>>(a, x, residual, out);
}

}  // namespace

hipError_t launch_dropout(const DropoutCall& c, hipStream_t stream)
{
    Dropout a{.groups = Divider((uint32_t)(c.cols + 7) / 8)};
    a.ldx = c.ldx, a.ldr = c.ldr, a.ldo = c.ldo, a.cols = c.cols;
    a.site = c.site, a.step_lo = (uint32_t)c.step, a.step_hi = (uint32_t)(c.step >> 32);
    a.key0 = (uint32_t)c.seed, a.key1 = (uint32_t)(c.seed >> 32);
    a.drop16 = (uint32_t)(c.drop48 >> 32), a.drop32 = (uint32_t)c.drop48, a.scale = c.scale;
    const int64_t rows_a_launch = (((int64_t)1 << 31) - 1) / a.groups.d;
    for (int64_t row = 0; row < c.rows; row += rows_a_launch) {
        const int64_t rows = c.rows - row < rows_a_launch ? c.rows - row : rows_a_launch;
        a.row0 = (uint32_t)row, a.items = (uint32_t)(rows * a.groups.d);
        const uint32_t blocks = (uint32_t)(((int64_t)a.items + kBlock - 1) / kBlock);
        if (c.x_bf16)
            c.out_bf16 ? launch<uint16_t, uint16_t>(a, c, blocks, stream) : launch<uint16_t, float>(a, c, blocks, stream);
        else
            c.out_bf16 ? launch<float, uint16_t>(a, c, blocks, stream) : launch<float, float>(a, c, blocks, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace agc
