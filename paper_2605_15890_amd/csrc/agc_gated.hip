// Gate of a gated feed-forward block, bfloat16:  a = x Wg^T, u = x Wu^T, h = act(a) * u, and its gradients by data
// partition (rows of G).  x is tokens x d_in, Wg and Wu are d_ff x d_in, all row-major.  The block's output projection, a
// product of h with a third matrix, is not part of it.
//
// Forward: one product whose columns take 16 rows of Wg and 16 rows of Wu in turn, so that a wave ends with a and u of
// the same places; activation and product follow from the binary32 sums, h is rounded once.
//
// Gradients: a and u are formed again (4 T D F operations, less than storing them in binary32 would save), and
//   da = dh u act'(a), du = dh act(a)          in the same pass
//   dx = da Wg + du Wu                          one product over 2 F
//   dWg_p = da_p^T x_p, dWu_p = du_p^T x_p      one product of 2 F rows a partition, written into row p of G
// da and du enter dx as two bfloat16 parts: 2^-16 of a term at most, so that the rounding of dx itself, 2^-8, is the one that
// counts (one part would add as much again: 2.35e-3 against 1.66e-3 in the 2-norm for random operands).  They enter G, which
// is binary32, with all their bits: as three bfloat16 parts, three products with x, which is bfloat16 as it is.  Any form
// with fewer bits of exponent (pairs of binary16 scaled by a power of two, two products) loses what lies far below the
// largest operands that its scale was made for: one token's large x, masked or not, would cost its whole partition's
// gradient its bits.  bfloat16 has binary32's exponents; the lowest part alone could fall below them, so values are lifted
// by 2^23 (kLift), which makes the smallest binary32 the smallest normal bfloat16.  da, du and G of 2^105 and more leave
// binary32 that way and become infinite.
// 8192 x 2048 x 5632 in 16 partitions: da, du 565 us, dx 587 us (1.29 PFLOP/s with its two products), G 1127 us (1.01, with
// 1.5 GB of G to write), where pairs for G and one part for dx took 524, 317 and 957 us and 44 us for the scales.
// The tile loop wants both operands contiguous along the sum: x and the weights are turned by passes of their own, da
// and du are written both ways.  A partition starts at a multiple of 32 in the turned order, the places between are
// zeros; `map` gives each place its token, or -1.
#include "agc_operators.h"
#include "agc_tile.h"

namespace agc {

namespace {

constexpr int kBlock = 256;
constexpr int kFewTokens = 64;   // up to here the forward pass is k_gated_few
constexpr float kLift = 8388608.0f;   // 2^23, of da and du as they enter G

struct Rows {
    const uint16_t* p;
    int64_t ld;
};

// what the kernels know of the partitions: first place and first token of each
struct GatedParts {
    int place[kMostParts + 1];
    int token[kMostParts + 1];
    int k;
};

struct Activation {
    int gelu;
    // 1 / (1 + exp(-a)) by the chip's 2^x and reciprocal (an ulp each).  -a log2(e) is formed with what its rounding leaves,
    // which would otherwise be off by up to |a| 2^-24 of the exponential.  An eighth of the time of expf and a division,
    // which were a fifth of the forward pass.
    static __device__ __forceinline__ float sigmoid(float a)
    {
        constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596303e-8f, kLn2 = 0.69314718f;
        const float t = -a * kLog2e;
        const float rest = fmaf(-a, kLog2e, -t) - a * kLog2eRest;
        const float e = __builtin_amdgcn_exp2f(t);
        // an infinite power times a rest of 0, or a power of 0 times an infinite rest, is no number
        const float p = e > 0.0f && e < 1e30f ? fmaf(e, rest * kLn2, e) : e;
        return __builtin_amdgcn_rcpf(1.0f + p);
    }
    // Phi(a) from the complement's side: 1 + erf would cancel below zero, down to nothing at a = -5.6.  8192 x 2048 x 8192
    // forward: 503 us where SiLU takes 460 (485 and 452 with erf, on another card).
    static __device__ __forceinline__ float normal_cdf(float a) { return 0.5f * erfcf(-0.70710678118654752f * a); }
    // activation and its derivative
    __device__ __forceinline__ void at(float a, float& value, float& slope) const
    {
        if (gelu) {
            const float cdf = normal_cdf(a);
            value = a * cdf;
            slope = fmaf(a * 0.39894228040143268f, expf(-0.5f * a * a), cdf);
        } else {
            const float sig = sigmoid(a);
            value = a * sig;
            slope = sig * fmaf(a, 1.0f - sig, 1.0f);
        }
    }
    __device__ __forceinline__ float operator()(float a) const
    {
        return a * (gelu ? normal_cdf(a) : sigmoid(a));
    }
};

__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// `count` of eight consecutive bfloat16 values, rounded
__device__ __forceinline__ void store_bf16(uint16_t* o, int count, const float v[8])
{
    if (count >= 8 && aligned16(o)) {
        *reinterpret_cast<tile_u32x4*>(o) = bf16_pack8(v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < count) o[e] = (uint16_t)bf16_bits(v[e]);
    }
}

__device__ __forceinline__ void load_bf16(const uint16_t* o, int count, float v[8])
{
    if (count >= 8 && aligned16(o)) {
        bf16_unpack8(*reinterpret_cast<const tile_u32x4*>(o), v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < count ? __uint_as_float((uint32_t)o[e] << 16) : 0.0f;
    }
}

// The 16 bytes of a bfloat16 row from element k on; elements from `end` on are zeros.
__device__ __forceinline__ tile_u32x4 load_bits8(const uint16_t* row, int k, int end)
{
    const uint16_t* p = row + k;
    if (k + 8 <= end && aligned16(p)) return *reinterpret_cast<const tile_u32x4*>(p);
    tile_u32x4 o = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (k + e < end) o[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
    return o;
}

// ------------------------------------------------------------------ laying operands out
// Rows whose width or alignment the tile loop's loads do not take, copied to rows of a whole number of k-steps; eight
// rows a workgroup.
struct PackRows {
    const uint16_t* src;
    int64_t ld;
    int rows, width, up;
    uint16_t* dst;
    __device__ __forceinline__ void run(int block) const
    {
        const int per = up / 8;
        for (int i = threadIdx.x; i < 8 * per; i += kBlock) {
            const int sub = i / per, c = (i - sub * per) * 8;
            const int64_t r = (int64_t)block * 8 + sub;
            if (r < rows) *reinterpret_cast<tile_u32x4*>(dst + r * up + c) = load_bits8(src + r * ld, c, width);
        }
    }
};

struct PlaceMap {
    int* map;
    int places;
    GatedParts parts;
    __device__ __forceinline__ void run(int block) const
    {
        const int i = block * kBlock + threadIdx.x;
        if (i >= places) return;
        int lo = 0, hi = parts.k - 1;   // the last partition that starts at or before i
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (parts.place[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        const int t = parts.token[lo] + (i - parts.place[lo]);
        map[i] = t < parts.token[lo + 1] ? t : -1;
    }
};

// dst row c = column c of src, along the rows of src (through `map`, if given; -1 and rows past the end are zeros),
// `up` of them.
struct Turn {
    const uint16_t* src;
    int64_t ld;
    int rows, cols, up;
    const int* map;
    char* dst;
    int64_t pitch;
    __device__ __forceinline__ void run(int r0, int c0) const
    {
        __shared__ uint16_t tile[64][66];
        const int tid = threadIdx.x;
        for (int i = tid; i < 512; i += kBlock) {
            const int r = i >> 3, c = (i & 7) * 8;
            int from = r0 + r < rows ? r0 + r : -1;
            if (map && from >= 0) from = map[from];
            tile_u32x4 v = {0u, 0u, 0u, 0u};
            if (from >= 0 && c0 + c < cols) v = load_bits8(src + (int64_t)from * ld, c0 + c, cols);
#pragma unroll
            for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(&tile[r][c + 2 * e]) = v[e];
        }
        __syncthreads();
        for (int i = tid; i < 512; i += kBlock) {
            const int c = i >> 3, r = (i & 7) * 8;
            if (c0 + c >= cols || r0 + r >= up) continue;
            tile_u32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (uint32_t)tile[r + 2 * e][c] | ((uint32_t)tile[r + 2 * e + 1][c] << 16);
            *reinterpret_cast<tile_u32x4*>(dst + (int64_t)(c0 + c) * pitch + (int64_t)(r0 + r) * 2) = v;
        }
    }
};

// All that needs nothing but the call's operands, in one launch: the copies of x, Wg, Wu that are needed, the map, and
// the weights turned.
struct Prepare {
    PackRows pack[3];
    int pack_blocks[3];
    PlaceMap map;
    int map_blocks;
    Turn turn[2];
    int turn_down, turn_blocks;   // of one
    int total() const { return pack_blocks[0] + pack_blocks[1] + pack_blocks[2] + map_blocks + 2 * turn_blocks; }
};

__global__ __launch_bounds__(kBlock) void k_gated_prepare(const Prepare a)
{
    int block = blockIdx.x;
    for (int i = 0; i < 3; ++i) {
        if (block < a.pack_blocks[i]) return a.pack[i].run(block);
        block -= a.pack_blocks[i];
    }
    if (block < a.map_blocks) return a.map.run(block);
    block -= a.map_blocks;
    const int which = block >= a.turn_blocks ? 1 : 0, at = block - which * a.turn_blocks, across = at / a.turn_down;
    a.turn[which].run((at - across * a.turn_down) * 64, across * 64);
}

__global__ __launch_bounds__(kBlock) void k_turn_tokens(const Turn a) { a.run(blockIdx.x * 64, blockIdx.y * 64); }

// ------------------------------------------------------------------ few tokens
// Up to NT * 16 tokens: bound by the one read of the weights.  A workgroup takes 16 rows of Wg and of Wu, its four
// waves take turns along the sum, 128 bytes of every row at a time, straight from memory into the matrix units'
// layout (weights as the 16 rows, tokens as the 16 columns); the waves' sums meet in LDS.  5 tokens of 1024 x 4096: 4.9 us
// for 16.8 MB.
// WHOLE: every 16 bytes of every row may be loaded as they are (d_in a multiple of 64, rows aligned).
template <int NT, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_gated_few(const uint16_t* x, int64_t ldx, const uint16_t* wg, const uint16_t* wu,
                                                      int64_t ldw, int tokens, int d_in, int d_ff, Activation act,
                                                      uint16_t* h, int64_t ldh)
{
    __shared__ float part[4][2][NT][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int f0 = blockIdx.x * 16, q = lane >> 4;
    const int f = f0 + (lane & 15) < d_ff ? f0 + (lane & 15) : d_ff - 1;
    const uint16_t *rg = wg + f * ldw, *ru = wu + f * ldw;
    const uint16_t* rx[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int tok = t * 16 + (lane & 15);
        rx[t] = x + (int64_t)(tok < tokens ? tok : tokens - 1) * ldx;
    }
    tile_f32x4 acc[2][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[0][t] = acc[1][t] = tile_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (WHOLE) {
        // four turns' loads at once; turns past the end load the last one again and count as zeros
        const tile_u32x4 zero = {0u, 0u, 0u, 0u};
        for (int k0 = wave * 64; k0 < d_in; k0 += 1024) {
            tile_u32x4 a[8], b[8], v[8][NT];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int k1 = k0 + (i >> 1) * 256, k = (k1 < d_in ? k1 : d_in - 64) + q * 16 + (i & 1) * 8;
                a[i] = *reinterpret_cast<const tile_u32x4*>(rg + k);
                b[i] = *reinterpret_cast<const tile_u32x4*>(ru + k);
#pragma unroll
                for (int t = 0; t < NT; ++t) v[i][t] = *reinterpret_cast<const tile_u32x4*>(rx[t] + k);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool on = k0 + (i >> 1) * 256 < d_in;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const tile_u32x4 w = on ? v[i][t] : zero;
                    acc[0][t] = tile_mfma<kPlain>(on ? a[i] : zero, w, acc[0][t]);
                    acc[1][t] = tile_mfma<kPlain>(on ? b[i] : zero, w, acc[1][t]);
                }
            }
        }
    } else {
        for (int k0 = wave * 64; k0 < d_in; k0 += 256) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int k = k0 + q * 16 + s * 8;
                const tile_u32x4 a = load_bits8(rg, k, d_in), b = load_bits8(ru, k, d_in);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const tile_u32x4 v = load_bits8(rx[t], k, d_in);
                    acc[0][t] = tile_mfma<kPlain>(a, v, acc[0][t]);
                    acc[1][t] = tile_mfma<kPlain>(b, v, acc[1][t]);
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            part[wave][0][t][(lane & 15) * 16 + q * 4 + e] = acc[0][t][e];
            part[wave][1][t][(lane & 15) * 16 + q * 4 + e] = acc[1][t][e];
        }
    __syncthreads();
    const int tok = tid >> 4, ff = f0 + (tid & 15);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t * 16 + tok >= tokens || ff >= d_ff) continue;
        const float a = (part[0][0][t][tid] + part[1][0][t][tid]) + (part[2][0][t][tid] + part[3][0][t][tid]);
        const float u = (part[0][1][t][tid] + part[1][1][t][tid]) + (part[2][1][t][tid] + part[3][1][t][tid]);
        h[(int64_t)(t * 16 + tok) * ldh + ff] = (uint16_t)bf16_bits(act(a) * u);
    }
}

// ------------------------------------------------------------------ products
// x against both weights.  GRAD: da and du, both ways; otherwise h.
template <bool GRAD>
struct GateJob {
    static constexpr TilePair kPair = kPlain;
    static constexpr int kRowParts = 4;
    static constexpr bool kTurned = GRAD;
    const uint16_t *x, *wg, *wu;      // rows of whole k-steps
    int64_t ldx, ldg, ldu;
    int n_rows, d_ff, steps;          // rows: tokens, or places of `map`
    Activation act;
    const int* map;
    // forward
    uint16_t* h;
    int64_t ldh;
    // gradient
    const uint16_t* dh;
    int64_t lddh;
    char* by_token;                   // places x 2 fp, two parts: da | du
    int fp;
    char* by_feature;                 // 2 d_ff rows of three parts along the places, lifted
    int64_t pitch;
    int mt, nt, side, total;

    __device__ __forceinline__ void place(int id, TilePos& p) const
    {
        int mi, ni;
        tile_order(xcd_order(id, total), mt, nt, mi, ni);
        p.batch = 0, p.m0 = mi * side, p.n0 = ni * side, p.steps = steps;
    }
    __device__ __forceinline__ const char* a_row(const TilePos& p, int r) const
    {
        int at = p.m0 + r < n_rows ? p.m0 + r : n_rows - 1;
        if (GRAD) at = map[at] < 0 ? 0 : map[at];
        return reinterpret_cast<const char*>(x + at * ldx);
    }
    __device__ __forceinline__ const char* b_row(const TilePos& p, int r) const
    {
        const int i = p.n0 + r, at = (i >> 5) * 16 + (i & 15);
        const int64_t f = at < d_ff ? at : d_ff - 1;
        return reinterpret_cast<const char*>((i & 16) ? wu + f * ldu : wg + f * ldg);
    }
    __device__ __forceinline__ bool turned(const TilePos&) const { return true; }
    __device__ __forceinline__ void rows(const TilePos&, int mb, int nb, float* s, int it, int lane) const
    {
        const int j = lane & 3, ca = (j >> 1) * 32 + (j & 1) * 8, f = nb / 2 + j * 8;
        const int r = it * 16 + (lane >> 2), row = mb + r;
        float a[8], u[8];
        piece_row8(s, r, ca, a);
        piece_row8(s, r, ca + 16, u);
        if (!GRAD) {
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = act(a[e]) * u[e];
            if (row < n_rows && f < d_ff) store_bf16(h + row * ldh + f, d_ff - f, a);
            return;
        }
        float da[8], du[8], g[8];
        const int t = row < n_rows ? map[row] : -1;
#pragma unroll
        for (int e = 0; e < 8; ++e) da[e] = du[e] = 0.0f;
        if (t >= 0 && f < d_ff) {
            load_bf16(dh + t * lddh + f, d_ff - f, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float value, slope;
                act.at(a[e], value, slope);
                if (f + e < d_ff) da[e] = g[e] * u[e] * slope, du[e] = g[e] * value;
            }
        }
        if (row < n_rows && f < fp) {
            char* o = by_token + (int64_t)row * fp * 8;
            parts2_store8(o, f, da);
            parts2_store8(o, fp + f, du);
        }
        piece_put_row8(s, r, ca, da);
        piece_put_row8(s, r, ca + 16, du);
    }
    __device__ __forceinline__ void cols(const TilePos&, int mb, int nb, const float* s, int it, int lane) const
    {
        const int run = (lane & 7) * 8, at = mb + run;
        const int c = it * 8 + (lane >> 3), ff = nb / 2 + (c >> 5) * 16 + (c & 15);
        if (ff >= d_ff || at >= n_rows) return;   // n_rows is a multiple of 32
        float v[8];
        piece_col8(s, run, c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= kLift;
        parts3_store8(by_feature + (int64_t)(((c & 16) ? d_ff : 0) + ff) * pitch, at, v);
    }
};

// dx = [da | du] [Wg | Wu]^T
struct InputJob {
    static constexpr TilePair kPair = kParts2;
    static constexpr int kRowParts = 8;
    static constexpr bool kTurned = false;
    const char *a, *b;
    int64_t pitch_a, pitch_b;
    int n_rows, d_in, steps;
    const int* map;
    uint16_t* dx;
    int64_t lddx;
    int mt, nt, side, total;

    __device__ __forceinline__ void place(int id, TilePos& p) const
    {
        int mi, ni;
        tile_order(xcd_order(id, total), mt, nt, mi, ni);
        p.batch = 0, p.m0 = mi * side, p.n0 = ni * side, p.steps = steps;
    }
    __device__ __forceinline__ const char* a_row(const TilePos& p, int r) const
    {
        return a + (p.m0 + r < n_rows ? p.m0 + r : n_rows - 1) * pitch_a;
    }
    __device__ __forceinline__ const char* b_row(const TilePos& p, int r) const
    {
        return b + (p.n0 + r < d_in ? p.n0 + r : d_in - 1) * pitch_b;
    }
    __device__ __forceinline__ void rows(const TilePos&, int mb, int nb, const float* s, int it, int lane) const
    {
        const int run = (lane & 7) * 8, c = nb + run, r = it * 8 + (lane >> 3), row = mb + r;
        const int t = row < n_rows ? map[row] : -1;
        if (t < 0 || c >= d_in) return;
        float v[8];
        piece_row8(s, r, run, v);
        store_bf16(dx + t * lddx + c, d_in - c, v);
    }
};

// Row p of G: [da | du]_p^T x_p
struct WeightJob {
    static constexpr TilePair kPair = kParts3;
    static constexpr int kRowParts = 8;
    static constexpr bool kTurned = false;
    const char *a, *b;        // 2 d_ff and d_in rows along the places
    int64_t places;
    int d_ff, d_in;
    bool whole;               // rows of G in units of four values, 16-byte aligned
    float *gate, *up;
    int64_t ldg;
    int mt, nt, side, total;
    GatedParts parts;

    __device__ __forceinline__ void place(int id, TilePos& p) const
    {
        const int t = xcd_order(id, total);
        p.batch = t / (mt * nt);
        int mi, ni;
        tile_order(t - p.batch * mt * nt, mt, nt, mi, ni);
        p.m0 = mi * side, p.n0 = ni * side;
        p.steps = (parts.place[p.batch + 1] - parts.place[p.batch]) >> 5;
    }
    __device__ __forceinline__ const char* a_row(const TilePos& p, int r) const
    {
        return a + ((p.m0 + r < 2 * d_ff ? p.m0 + r : 2 * d_ff - 1) * places + parts.place[p.batch]) * 6;
    }
    __device__ __forceinline__ const char* b_row(const TilePos& p, int r) const
    {
        return b + ((p.n0 + r < d_in ? p.n0 + r : d_in - 1) * places + parts.place[p.batch]) * 2;
    }
    __device__ __forceinline__ void rows(const TilePos& p, int mb, int nb, const float* s, int it, int lane) const
    {
        auto at = [&](int row) {
            return (row < d_ff ? gate + (int64_t)row * d_in : up + (int64_t)(row - d_ff) * d_in) + p.batch * ldg;
        };
        // rows of G that start anywhere: the lanes side by side, a value each (1999 x 519 x 1101 in five equal partitions:
        // 36 us with eight values a lane, 28 us so)
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = it * 8 + e;
                if (mb + r < 2 * d_ff && nb + lane < d_in) at(mb + r)[nb + lane] = s[piece_at(r, lane)] * (1.0f / kLift);
            }
            return;
        }
        const int run = (lane & 7) * 8, c = nb + run, r = it * 8 + (lane >> 3), row = mb + r;
        if (row >= 2 * d_ff || c >= d_in) return;
        float v[8];
        piece_row8(s, r, run, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= 1.0f / kLift;
        float* o = at(row) + c;
        *reinterpret_cast<tile_f32x4*>(o) = tile_f32x4{v[0], v[1], v[2], v[3]};
        if (c + 4 < d_in) *reinterpret_cast<tile_f32x4*>(o + 4) = tile_f32x4{v[4], v[5], v[6], v[7]};
    }
};

template <class JOB>
hipError_t launch_product(JOB j, int batch, int64_t m, int64_t n, int64_t steps, hipStream_t stream)
{
    const TileChoice c = choose_tile(batch, m, n, steps, false);
    j.side = c.side;
    j.mt = (int)c.mt;
    j.nt = (int)c.nt;
    j.total = (int)c.total;
    return launch_tiles(j, c, stream);
}

bool takes_whole_loads(const void* p, int64_t ld) { return (ld & 7) == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Rows that the tile loop's loads take as they are, or a copy of them in `room`, made by copy `i` of `prepare`.
Rows whole_steps(const void* src, int64_t ld, int64_t rows, int width, char*& room, Prepare& prepare, int i)
{
    const int up = (int)round_up(width, 64);
    uint16_t* mine = reinterpret_cast<uint16_t*>(room);
    room += round_up(rows * up * 2, 256);
    const uint16_t* p = static_cast<const uint16_t*>(src);
    if (up == width && takes_whole_loads(src, ld)) return Rows{p, ld};
    prepare.pack[i] = PackRows{p, ld, (int)rows, width, up, mine};
    prepare.pack_blocks[i] = (int)((rows + 7) / 8);
    return Rows{mine, up};
}

hipError_t launch_prepare(const Prepare& prepare, hipStream_t stream)
{
    if (prepare.total() == 0) return hipSuccess;
    hipLaunchKernelGGL(k_gated_prepare, dim3(prepare.total()), dim3(kBlock), 0, stream, prepare);
    return hipGetLastError();
}

int64_t packed_bytes(int64_t tokens, int d_in, int d_ff)
{
    const int64_t up = round_up(d_in, 64) * 2;
    return round_up(tokens * up, 256) + 2 * round_up(d_ff * up, 256);
}

template <int NT, bool WHOLE>
hipError_t launch_few(const GatedCall& c, hipStream_t stream)
{
    hipLaunchKernelGGL((k_gated_few<NT, WHOLE>), dim3((c.d_ff + 15) / 16), dim3(kBlock), 0, stream,
                       static_cast<const uint16_t*>(c.x), c.ldx, static_cast<const uint16_t*>(c.wg),
                       static_cast<const uint16_t*>(c.wu), c.ldw, (int)c.tokens, c.d_in, c.d_ff, Activation{c.gelu},
                       static_cast<uint16_t*>(c.h), c.ldh);
    return hipGetLastError();
}

}  // namespace

// packed x, Wg, Wu | map | da, du by token | by feature | x turned | weights turned
int64_t gated_workspace_bytes(int64_t tokens, int d_in, int d_ff, int k_parts)
{
    if (k_parts == 0 && tokens <= kFewTokens) return 256;   // nothing is laid out
    int64_t bytes = packed_bytes(tokens, d_in, d_ff);
    if (k_parts > 0) {
        const int64_t held = k_parts < tokens ? k_parts : tokens;   // partitions that are not empty, at most
        const int64_t places = round_up(tokens + 31 * held, 32), fp = round_up(d_ff, 64);
        bytes += round_up(places * 4, 256) + round_up(places * fp * 8, 256) + round_up(2 * d_ff * places * 6, 256) +
                 round_up(d_in * places * 2, 256) + round_up(d_in * fp * 4, 256);
    }
    return bytes > 256 ? bytes : 256;
}

hipError_t launch_gated_forward(const GatedCall& c, hipStream_t stream)
{
    if (c.tokens <= kFewTokens) {
        const bool whole = (c.d_in & 63) == 0 && takes_whole_loads(c.x, c.ldx) && takes_whole_loads(c.wg, c.ldw) &&
                           takes_whole_loads(c.wu, c.ldw);
        if (c.tokens <= 16) return whole ? launch_few<1, true>(c, stream) : launch_few<1, false>(c, stream);
        if (c.tokens <= 32) return whole ? launch_few<2, true>(c, stream) : launch_few<2, false>(c, stream);
        return whole ? launch_few<4, true>(c, stream) : launch_few<4, false>(c, stream);
    }
    const Activation act{c.gelu};
    char* room = c.workspace;
    Prepare prepare{};
    const Rows x = whole_steps(c.x, c.ldx, c.tokens, c.d_in, room, prepare, 0);
    const Rows wg = whole_steps(c.wg, c.ldw, c.d_ff, c.d_in, room, prepare, 1);
    const Rows wu = whole_steps(c.wu, c.ldw, c.d_ff, c.d_in, room, prepare, 2);
    const hipError_t e = launch_prepare(prepare, stream);
    if (e != hipSuccess) return e;
    GateJob<false> j{};
    j.x = x.p, j.ldx = x.ld, j.wg = wg.p, j.ldg = wg.ld, j.wu = wu.p, j.ldu = wu.ld;
    j.n_rows = (int)c.tokens, j.d_ff = c.d_ff, j.steps = (int)(round_up(c.d_in, 64) / 64), j.act = act;
    j.h = static_cast<uint16_t*>(c.h), j.ldh = c.ldh;
    return launch_product(j, 1, c.tokens, round_up(c.d_ff, 16) * 2, j.steps, stream);
}

hipError_t launch_gated_gradients(const GatedCall& c, hipStream_t stream)
{
    const Activation act{c.gelu};
    GatedParts parts{};
    parts.k = c.k_parts;
    for (int p = 0; p < c.k_parts; ++p) {
        parts.token[p + 1] = (int)c.part_end[p];
        parts.place[p + 1] = parts.place[p] + (int)round_up(parts.token[p + 1] - parts.token[p], 32);
    }
    const int places = parts.place[c.k_parts];
    const int64_t fp = round_up(c.d_ff, 64);
    char* room = c.workspace;
    auto take = [&](int64_t bytes) {
        char* p = room;
        room += round_up(bytes, 256);
        return p;
    };
    char *by_feature = nullptr, *x_turned = nullptr;
    hipError_t e = hipSuccess;
    if (places > 0) {
        Prepare prepare{};
        const Rows x = whole_steps(c.x, c.ldx, c.tokens, c.d_in, room, prepare, 0);
        const Rows wg = whole_steps(c.wg, c.ldw, c.d_ff, c.d_in, room, prepare, 1);
        const Rows wu = whole_steps(c.wu, c.ldw, c.d_ff, c.d_in, room, prepare, 2);
        int* map = reinterpret_cast<int*>(take((int64_t)places * 4));
        char* by_token = take(places * fp * 8);
        by_feature = take((int64_t)places * 2 * c.d_ff * 6);
        x_turned = take((int64_t)places * c.d_in * 2);
        char* w_turned = take(c.d_in * fp * 4);
        const int across = (c.d_in + 63) / 64;
        prepare.map = PlaceMap{map, places, parts};
        prepare.map_blocks = (places + kBlock - 1) / kBlock;
        if (c.dx) {
            prepare.turn[0] = Turn{static_cast<const uint16_t*>(c.wg), c.ldw, c.d_ff, c.d_in, (int)fp, nullptr, w_turned, fp * 4};
            prepare.turn[1] = prepare.turn[0];
            prepare.turn[1].src = static_cast<const uint16_t*>(c.wu), prepare.turn[1].dst = w_turned + fp * 2;
            prepare.turn_down = (int)(fp / 64);
            prepare.turn_blocks = prepare.turn_down * across;
        }
        e = launch_prepare(prepare, stream);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(k_turn_tokens, dim3((places + 63) / 64, across), dim3(kBlock), 0, stream,
                           Turn{static_cast<const uint16_t*>(c.x), c.ldx, places, c.d_in, places, map, x_turned,
                                (int64_t)places * 2});
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        GateJob<true> j{};
        j.x = x.p, j.ldx = x.ld, j.wg = wg.p, j.ldg = wg.ld, j.wu = wu.p, j.ldu = wu.ld;
        j.n_rows = places, j.d_ff = c.d_ff, j.steps = (int)(round_up(c.d_in, 64) / 64), j.act = act, j.map = map;
        j.dh = static_cast<const uint16_t*>(c.dh), j.lddh = c.lddh;
        j.by_token = by_token, j.fp = (int)fp, j.by_feature = by_feature, j.pitch = (int64_t)places * 6;
        e = launch_product(j, 1, places, fp * 2, j.steps, stream);
        if (e != hipSuccess) return e;
        if (c.dx) {
            InputJob d{by_token, w_turned, fp * 8, fp * 4, places, c.d_in, (int)(fp / 16), map,
                       static_cast<uint16_t*>(c.dx), c.lddx};
            e = launch_product(d, 1, places, c.d_in, d.steps, stream);
            if (e != hipSuccess) return e;
        }
    }
    WeightJob w{};
    w.a = by_feature, w.b = x_turned, w.places = places, w.d_ff = c.d_ff, w.d_in = c.d_in;
    w.whole = c.d_in % 4 == 0 && c.ldg % 4 == 0 && reinterpret_cast<uintptr_t>(c.g_gate) % 16 == 0 &&
              reinterpret_cast<uintptr_t>(c.g_up) % 16 == 0;
    w.gate = c.g_gate, w.up = c.g_up, w.ldg = c.ldg, w.parts = parts;
    return launch_product(w, c.k_parts, 2 * (int64_t)c.d_ff, c.d_in, places / 32 / c.k_parts, stream);
}

}  // namespace agc
