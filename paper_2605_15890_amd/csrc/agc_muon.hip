// Orthogonalised update of the matrices inside the parameter vector (the optimizer that consumes g_hat):
//   M <- mu M + g;   U = g + mu M  or  M;   X = U / (|U| + eps)
//   S times   A = X X^T,  B = a I + b A + c A A,  X <- B X       (p(x) = a x + b x^3 + c x^5 on the singular values)
//   beta <- keep * beta - rate * X
// with X taken as m x n, m <= n (the transpose of a tall matrix).
//
// Range and rounding.  With a, b, c = 3.4445, -4.7750, 2.0315, p maps [0, 1.21] into itself and the first X has
// singular values of at most 1, so |X| < 1.21, |A| < 1.47 and |B| <= a: every entry of each has a bound that is known
// before, and each is kept as a pair of binary16 values (hi + lo, 22 bits) scaled by a fixed power of two that fills
// the range.  Entries far below the bound lose relative but not absolute accuracy, 2^-25 of the unit 2^-14, which is
// below the rounding of binary32 sums of the products that they enter.  Three matrix products on the 16-bit units
// (hi hi + hi lo + lo hi) then stand for one in binary32: 1/3 of 2.5 PFLOP/s, where binary32 operands reach 0.157.
// X itself goes through this, not a rounded copy of it: single 16-bit values would leave errors that the products
// amplify by up to a^S = 485 in the directions of small singular values.
//
// Two steps at once.  All factors are polynomials of the first A, so with B0 and Q the step's own
//   A' = B0 A B0,  B1 = a I + b A' + c A' A',  Q = B1 B0,  X <- Q X
// is two steps with one product along n each way in place of two: 3 m^2 n + 5 m^3 multiplications against 6 m^2 n + 2 m^3
// (symmetric products counted half).  12 x 1024 x 4096: 2758 us in single steps, 2194 us so.
// It is taken where n >= 2 m.  Q reaches a^2 = 11.9 where X is small and is rounded against that; longer chains would lose
// more.  Pairs of steps stay with five single steps whose products are binary32, error of X against 64 bits in the 2-norm:
// 512 x 2048 1.5e-6 here, 3.2e-6 there, of rank four 4.3e-5 and 6.1e-5, singular values from 1 to 1e-6 5.9e-6 and 6.7e-6;
// 64 x 900 2.9e-6 and 1.9e-6, of rank four 2.7e-5 and 2.4e-5.
//
// Each product writes its result for the next one in the order in which that one reads it: X along n (for X X^T) and
// along m (for B X); A and B are symmetric, so half the tiles are formed and written twice.  The last product
// updates beta from its sums; X is not written.
#include "agc_operators.h"
#include "agc_tile.h"

namespace agc {

namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr double kMuonEps = 1e-7;
constexpr float kUnitX = 16384.0f;   // 2^14 * 1.21 < 65504
constexpr float kUnitA = 16384.0f;   // 2^14 * 1.47
constexpr float kUnitB = 8192.0f;    // 2^13 * 3.45
constexpr float kUnitQ = 4096.0f;    // 2^12 * 3.45^2
constexpr int kSumBlock = 256;       // threads of the elementwise passes
constexpr int kMostSums = 1024;      // partial sums of squares of a matrix

struct MuonGeom {
    int m, n;            // short and long side
    int tall;            // the matrix has more rows than columns: X is its transpose
    int mats;
    int64_t pitch_n;     // bytes of a split row of n values
    int64_t pitch_m;     // of m values
    int64_t size_x, size_t, size_a;   // bytes of a matrix stored along n, along m, and of A
};

MuonGeom muon_geom(int rows, int cols, int n_mats)
{
    MuonGeom g{};
    g.tall = rows > cols;
    g.m = g.tall ? cols : rows;
    g.n = g.tall ? rows : cols;
    g.mats = n_mats;
    g.pitch_n = round_up(g.n, 32) * 4;
    g.pitch_m = round_up(g.m, 32) * 4;
    g.size_x = g.m * g.pitch_n;
    g.size_t = g.n * g.pitch_m;
    g.size_a = g.m * g.pitch_m;
    return g;
}

int muon_sums(int64_t count)
{
    const int64_t blocks = (count + 16383) / 16384;
    return (int)(blocks < kMostSums ? blocks : kMostSums);
}

__device__ __forceinline__ double block_sum(double v, double* lds)
{
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// M <- mu M + g and the sum of the squares of U in binary64, one partial sum a workgroup (added in a fixed order
// by k_muon_start).  Bound by memory: 12 bytes a value; 12 x 1024 x 4096 in 114 us, 5.3 TB/s.
__global__ __launch_bounds__(kSumBlock) void k_muon_momentum(const MuonCall c, int64_t count, double* sums)
{
    __shared__ double lds[4];
    const int64_t off = c.offset[blockIdx.y];
    const float* g = c.ghat + off;
    float* m = c.m1 + off;
    const float mu = c.momentum;
    double sum = 0.0;
    auto one = [&](float gv, float mv) {
        mv = fmaf(mu, mv, gv);
        const float u = c.nesterov ? fmaf(mu, mv, gv) : mv;
        sum = fma((double)u, (double)u, sum);
        return mv;
    };
    const int64_t step = (int64_t)gridDim.x * kSumBlock, at = (int64_t)blockIdx.x * kSumBlock + threadIdx.x;
    int64_t done = 0;
    if (((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(m)) & 15) == 0) {
        const int64_t quads = count / 4;
        for (int64_t i = at; i < quads; i += step) {
            const float4 gv = reinterpret_cast<const float4*>(g)[i];
            float4 mv = reinterpret_cast<const float4*>(m)[i];
            mv.x = one(gv.x, mv.x), mv.y = one(gv.y, mv.y), mv.z = one(gv.z, mv.z), mv.w = one(gv.w, mv.w);
            reinterpret_cast<float4*>(m)[i] = mv;
        }
        done = quads * 4;
    }
    for (int64_t i = done + at; i < count; i += step) m[i] = one(g[i], m[i]);
    const double s = block_sum(sum, lds);
    if (threadIdx.x == 0) sums[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

// X = U / (|U| + eps) as binary16 pairs, stored along both sides.  A workgroup turns one 64 x 64 tile of U in LDS.  Bound
// by memory: 16 bytes a value; 12 x 1024 x 4096 in 171 us, 4.7 TB/s, the rate of a copy.
__global__ __launch_bounds__(kSumBlock) void k_muon_start(const MuonCall c, MuonGeom geo, const double* sums, int n_sums,
                                                          char* along_cols, char* along_rows)
{
    __shared__ double lds_sum[4];
    __shared__ float tile[64][65];
    const int mat = blockIdx.z, tid = threadIdx.x;
    double s = 0.0;
    for (int i = tid; i < n_sums; i += kSumBlock) s += sums[(int64_t)mat * n_sums + i];
    s = block_sum(s, lds_sum);
    const float unit = (float)((double)kUnitX / (sqrt(s) + kMuonEps));

    const float* g = c.ghat + c.offset[mat];
    const float* m = c.m1 + c.offset[mat];
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    for (int i = tid; i < 4096; i += kSumBlock) {
        const int r = r0 + (i >> 6), col = c0 + (i & 63);
        float u = 0.0f;
        if (r < c.rows && col < c.cols) {
            const int64_t at = (int64_t)r * c.cols + col;
            u = (c.nesterov ? fmaf(c.momentum, m[at], g[at]) : m[at]) * unit;
        }
        tile[i >> 6][i & 63] = u;
    }
    __syncthreads();
    const int64_t pitch_cols = geo.tall ? geo.pitch_m : geo.pitch_n, pitch_rows = geo.tall ? geo.pitch_n : geo.pitch_m;
    const int64_t cols_up = pitch_cols / 4, rows_up = pitch_rows / 4;
    char* by_row = along_cols + (int64_t)mat * c.rows * pitch_cols;
    char* by_col = along_rows + (int64_t)mat * c.cols * pitch_rows;
    for (int i = tid; i < 512; i += kSumBlock) {
        const int a = i >> 3, b = (i & 7) * 8;
        float v[8];
        if (r0 + a < c.rows && c0 + b < cols_up) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = tile[a][b + e];
            split_store8(by_row + (int64_t)(r0 + a) * pitch_cols, c0 + b, v);
        }
        if (c0 + a < c.cols && r0 + b < rows_up) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = tile[b + e][a];
            split_store8(by_col + (int64_t)(c0 + a) * pitch_rows, r0 + b, v);
        }
    }
}

// ------------------------------------------------------------------ the three products of a step
// A symmetric product of rows of two matrices (X and X, or two polynomials of one A, which commute), or a I + b A + c A A:
// tiles of the lower triangle.
struct SymJob {
    static constexpr TilePair kPair = kSplit;
    static constexpr int kRowParts = 8;
    static constexpr bool kTurned = true;
    const char *src, *other;
    char* dst;
    int64_t pitch, size;      // of src
    int64_t pitch_dst, size_dst;
    int m, steps, tiles, side, total;   // tiles of one matrix, tile edge, of all
    int poly;
    float unit;               // of what is stored over the unit of the sums

    __device__ __forceinline__ void place(int id, TilePos& p) const
    {
        const int t = xcd_order(id, total);
        p.batch = t / tiles;
        int mi, ni;
        triangle_order(t - p.batch * tiles, mi, ni);
        p.m0 = mi * side, p.n0 = ni * side, p.steps = steps;
    }
    __device__ __forceinline__ int64_t row(const TilePos& p, int r) const
    {
        return p.batch * size + (int64_t)(r < m ? r : m - 1) * pitch;
    }
    __device__ __forceinline__ const char* a_row(const TilePos& p, int r) const { return src + row(p, p.m0 + r); }
    __device__ __forceinline__ const char* b_row(const TilePos& p, int r) const { return other + row(p, p.n0 + r); }
    // a tile on the diagonal holds both halves
    __device__ __forceinline__ bool turned(const TilePos& p) const { return p.m0 != p.n0; }
    __device__ __forceinline__ void rows(const TilePos& p, int mb, int nb, float* s, int it, int lane) const
    {
        const int up = (int)(pitch_dst / 4), run = (lane & 7) * 8;
        const int r = it * 8 + (lane >> 3), gr = mb + r, gc = nb + run;
        float v[8];
        piece_row8(s, r, run, v);
        if (poly) {
            float a[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = 0.0f;
            if (gr < m && gc < up) split_load8(src + p.batch * size + (int64_t)gr * pitch, gc, a);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // units: sums 2^28, A 2^14, B 2^13
                float b = fmaf(kNsC * (kUnitB / (kUnitA * kUnitA)), v[e], kNsB * (kUnitB / kUnitA) * a[e]);
                if (gr == gc + e) b += kNsA * kUnitB;
                v[e] = b;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= unit;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (gr >= m || gc + e >= m) v[e] = 0.0f;
        if (gr < m && gc < up) split_store8(dst + p.batch * size_dst + (int64_t)gr * pitch_dst, gc, v);
        piece_put_row8(s, r, run, v);
    }
    __device__ __forceinline__ void cols(const TilePos& p, int mb, int nb, const float* s, int it, int lane) const
    {
        const int run = (lane & 7) * 8, cc = it * 8 + (lane >> 3), gc = nb + cc, gr = mb + run;
        float v[8];
        piece_col8(s, run, cc, v);
        if (gc < m && gr < (int)(pitch_dst / 4)) split_store8(dst + p.batch * size_dst + (int64_t)gc * pitch_dst, gr, v);
    }
};

// X <- B X (or Q X, with a unit of its own), or, at the end, beta <- keep * beta - rate * that.
template <bool LAST>
struct ApplyJob {
    static constexpr TilePair kPair = kSplit;
    static constexpr int kRowParts = 8;
    static constexpr bool kTurned = true;
    const char* b;           // m x m
    const char* xt;          // X along m: n rows
    char* out_x;             // along n
    char* out_t;             // along m
    MuonGeom g;
    int mt, nt, side, total;
    float per_unit_b;        // 1 over the unit of b, a power of two
    MuonCall call;           // at the end

    __device__ __forceinline__ void place(int id, TilePos& p) const
    {
        const int t = xcd_order(id, total);
        p.batch = t / (mt * nt);
        int mi, ni;
        tile_order(t - p.batch * mt * nt, mt, nt, mi, ni);
        p.m0 = mi * side, p.n0 = ni * side, p.steps = (int)(g.pitch_m / 128);
    }
    __device__ __forceinline__ const char* a_row(const TilePos& p, int r) const
    {
        const int at = p.m0 + r < g.m ? p.m0 + r : g.m - 1;
        return b + p.batch * g.size_a + (int64_t)at * g.pitch_m;
    }
    __device__ __forceinline__ const char* b_row(const TilePos& p, int r) const
    {
        const int at = p.n0 + r < g.n ? p.n0 + r : g.n - 1;
        return xt + p.batch * g.size_t + (int64_t)at * g.pitch_m;
    }
    // `count` of eight consecutive parameters from index at on
    __device__ __forceinline__ void update(int64_t at, int count, const float v[8]) const
    {
        float* beta = call.beta + at;
        const float rate = call.rate * (per_unit_b * (1.0f / kUnitX));
        float w[8];
        if (count == 8 && (reinterpret_cast<uintptr_t>(beta) & 15) == 0) {
            tile_f32x4* q = reinterpret_cast<tile_f32x4*>(beta);
            const tile_f32x4 x = q[0], y = q[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = fmaf(-rate, v[e], call.keep * x[e]);
                w[4 + e] = fmaf(-rate, v[4 + e], call.keep * y[e]);
            }
            q[0] = tile_f32x4{w[0], w[1], w[2], w[3]};
            q[1] = tile_f32x4{w[4], w[5], w[6], w[7]};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < count) beta[e] = w[e] = fmaf(-rate, v[e], call.keep * beta[e]);
        }
        if (call.beta_bf16) {
            uint16_t* o = call.beta_bf16 + at;
            if (count == 8 && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
                *reinterpret_cast<tile_u32x4*>(o) = bf16_pack8(w);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < count) o[e] = (uint16_t)bf16_bits(w[e]);
            }
        }
    }
    // the last step goes along the rows of the matrix as it lies
    __device__ __forceinline__ bool turned(const TilePos&) const { return !LAST || g.tall; }
    __device__ __forceinline__ void rows(const TilePos& p, int mb, int nb, float* s, int it, int lane) const
    {
        const int run = (lane & 7) * 8, gr = mb + it * 8 + (lane >> 3), gc = nb + run;
        float v[8];
        if (LAST) {
            if (g.tall || gr >= g.m || gc >= g.n) return;
            piece_row8(s, it * 8 + (lane >> 3), run, v);
            update(call.offset[p.batch] + (int64_t)gr * g.n + gc, g.n - gc < 8 ? g.n - gc : 8, v);
            return;
        }
        piece_row8(s, it * 8 + (lane >> 3), run, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = gc + e < g.n ? v[e] * per_unit_b : 0.0f;
        if (gr < g.m && gc < (int)(g.pitch_n / 4)) split_store8(out_x + p.batch * g.size_x + (int64_t)gr * g.pitch_n, gc, v);
    }
    __device__ __forceinline__ void cols(const TilePos& p, int mb, int nb, const float* s, int it, int lane) const
    {
        const int run = (lane & 7) * 8, gc = nb + it * 8 + (lane >> 3), gr = mb + run;
        float v[8];
        piece_col8(s, run, it * 8 + (lane >> 3), v);
        if (LAST) {
            if (gc < g.n && gr < g.m)
                update(call.offset[p.batch] + (int64_t)gc * g.m + gr, g.m - gr < 8 ? g.m - gr : 8, v);
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = gr + e < g.m ? v[e] * per_unit_b : 0.0f;
        if (gc < g.n && gr < (int)(g.pitch_m / 4)) split_store8(out_t + p.batch * g.size_t + (int64_t)gc * g.pitch_m, gr, v);
    }
};

// ------------------------------------------------------------------ small matrices
// A matrix whose X, its transpose and A fit into one workgroup's LDS (up to 64 x 256, 96 x 128): the whole update in one
// launch, one workgroup a matrix.  Bound by the latency of its 3 * steps products, one after another: the separate
// kernels take some 6 us for each, this one 1.3 (96 x 64: 106 us in 17 launches, 26 us in this one).
// Both sides are padded to 32 with zeros.  A split row lies in LDS as in memory, its 16-byte chunks permuted by the
// row's low bits within each 128 bytes.
// Two forms: 16 waves and one or two 16 x 16 blocks of each product a wave, or 8 waves with up to 5 of A and 9 of X.
struct SmallNarrow {
    static constexpr int kThreads = 1024, kPer = 8, kGram = 1, kBlocks = 2, kLds = 80 * 1024;
    static bool takes(int64_t m, int64_t n) { return m <= 64 && m * n <= 8192; }   // 8 m n + 4 m m <= 80 KB
};
struct SmallWide {
    static constexpr int kThreads = 512, kPer = 36, kGram = 5, kBlocks = 9, kLds = 152 * 1024;
    static bool takes(int64_t m, int64_t n) { return 8 * m * n + 4 * m * m <= kLds; }   // m <= 96, m n <= 18432
};

__device__ __forceinline__ int small_at(int row, int k, int pitch)   // byte of the high part; the low part: ^ 64
{
    return row * pitch + (k >> 5) * 128 + (((((k & 31) >> 3)) ^ (row & 7)) << 4) + (k & 7) * 2;
}

__device__ __forceinline__ void small_put(char* base, int row, int k, int pitch, float v)
{
    const int at = small_at(row, k, pitch);
    const _Float16 hi = (_Float16)v;
    *reinterpret_cast<_Float16*>(base + at) = hi;
    *reinterpret_cast<_Float16*>(base + (at ^ 64)) = (_Float16)(v - (float)hi);
}

// Four values of consecutive k (a multiple of 4)
__device__ __forceinline__ void small_put4(char* base, int row, int k, int pitch, const tile_f32x4& v)
{
    const int at = small_at(row, k, pitch);
    f16x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        hi[e] = (_Float16)v[e];
        lo[e] = (_Float16)(v[e] - (float)hi[e]);
    }
    *reinterpret_cast<f16x4*>(base + at) = hi;
    *reinterpret_cast<f16x4*>(base + (at ^ 64)) = lo;
}

// 16 x 16 block (rows ra.. of a, rows rb.. of b) of a product of split rows: `c` with a lane's four values along a's
// rows, and, if TWO, `t` with four values along b's rows (the same block, its operands exchanged), so that either can
// be stored four values at a time.
template <bool TWO>
__device__ __forceinline__ void small_block(const char* a, const char* b, int ra, int rb, int pitch, int steps, int lane,
                                            tile_f32x4& c, tile_f32x4& t)
{
    const tile_f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    tile_f32x4 c1 = zero, t1 = zero;
    c = t = zero;
    const int sub = lane & 15, chunk = ((lane >> 4) ^ (lane & 7)) << 4;   // rows start at multiples of 16
    const char *pa = a + (ra + sub) * pitch, *pb = b + (rb + sub) * pitch;
    for (int s = 0; s < steps; ++s, pa += 128, pb += 128) {
        const tile_u32x4 a0 = *reinterpret_cast<const tile_u32x4*>(pa + chunk);
        const tile_u32x4 a1 = *reinterpret_cast<const tile_u32x4*>(pa + (chunk ^ 64));
        const tile_u32x4 b0 = *reinterpret_cast<const tile_u32x4*>(pb + chunk);
        const tile_u32x4 b1 = *reinterpret_cast<const tile_u32x4*>(pb + (chunk ^ 64));
        c = tile_mfma<kSplit>(a0, b0, c);
        if (TWO) t = tile_mfma<kSplit>(b0, a0, t);
        c1 = tile_mfma<kSplit>(a0, b1, c1);
        if (TWO) t1 = tile_mfma<kSplit>(b0, a1, t1);
        c1 = tile_mfma<kSplit>(a1, b0, c1);
        if (TWO) t1 = tile_mfma<kSplit>(b1, a0, t1);
    }
    c += c1;
    t += t1;
}

template <class FORM>
__global__ __launch_bounds__(FORM::kThreads) void k_muon_small(const MuonCall c, MuonGeom g)
{
    constexpr int kSmallThreads = FORM::kThreads, kSmallWaves = kSmallThreads / 64, kSmallPer = FORM::kPer;
    constexpr int kSmallGram = FORM::kGram, kSmallBlocks = FORM::kBlocks, kSmallLds = FORM::kLds;
    __shared__ __attribute__((aligned(1024))) char lds[kSmallLds];
    __shared__ double part[kSmallWaves];
    const int tid = threadIdx.x, lane = tid & 63, q4 = (lane >> 4) * 4, col = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = g.m, n = g.n, mr = (int)(g.pitch_m / 4), nr = (int)(g.pitch_n / 4);
    const int pitch_m = (int)g.pitch_m, pitch_n = (int)g.pitch_n;
    char* x = lds;                       // mr rows along n
    char* xt = x + mr * pitch_n;         // nr rows along m
    char* a = xt + nr * pitch_m;         // mr rows along m: A, then B
    const int64_t off = c.offset[blockIdx.x];

    // M and U, a value of every kSmallThreads a register
    const int count = m * n;
    float u[kSmallPer], old[kSmallPer];
#pragma unroll
    for (int i = 0; i < kSmallPer; ++i) {
        const int at = tid + i * kSmallThreads;
        u[i] = old[i] = 0.0f;
        if (at < count) u[i] = c.ghat[off + at], old[i] = c.m1[off + at];
    }
    for (int i = tid * 16; i < mr * pitch_n + nr * pitch_m; i += kSmallThreads * 16)
        *reinterpret_cast<tile_u32x4*>(lds + i) = tile_u32x4{0u, 0u, 0u, 0u};
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kSmallPer; ++i) {
        const int at = tid + i * kSmallThreads;
        const float mv = fmaf(c.momentum, old[i], u[i]);
        if (at < count) c.m1[off + at] = mv;
        u[i] = c.nesterov ? fmaf(c.momentum, mv, u[i]) : mv;
        sum = fma((double)u[i], (double)u[i], sum);
    }
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < kSmallWaves; ++i) sum += part[i];
    const float unit = (float)((double)kUnitX / (sqrt(sum) + kMuonEps));
#pragma unroll
    for (int i = 0; i < kSmallPer; ++i) {
        const int at = tid + i * kSmallThreads;
        if (at >= count) continue;
        const int major = at / c.cols, minor = at - major * c.cols;
        const int r = g.tall ? minor : major, k = g.tall ? major : minor;
        small_put(x, r, k, pitch_n, u[i] * unit);
        small_put(xt, k, r, pitch_m, u[i] * unit);
    }
    __syncthreads();

    const int across_m = mr / 16, across_n = nr / 16;
    tile_f32x4 unused;
    for (int step = 0; step < c.steps; ++step) {
        for (int i = wave; i < across_m * across_m; i += kSmallWaves) {
            const int bi = i / across_m * 16, bj = (i - i / across_m * across_m) * 16;
            tile_f32x4 v;
            small_block<false>(x, x, bi, bj, pitch_n, nr / 32, lane, v, unused);
            small_put4(a, bj + col, bi + q4, pitch_m, v * (kUnitA / (kUnitX * kUnitX)));   // symmetric
        }
        __syncthreads();
        tile_f32x4 poly[kSmallGram];
#pragma unroll
        for (int b = 0; b < kSmallGram; ++b) {
            const int i = wave + b * kSmallWaves;
            if (i >= across_m * across_m) continue;
            const int bi = i / across_m * 16, bj = (i - i / across_m * across_m) * 16;
            small_block<false>(a, a, bi, bj, pitch_m, mr / 32, lane, poly[b], unused);
            const int at = small_at(bj + col, bi + q4, pitch_m);
            const f16x4 hi = *reinterpret_cast<const f16x4*>(a + at), lo = *reinterpret_cast<const f16x4*>(a + (at ^ 64));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v = fmaf(kNsC * (kUnitB / (kUnitA * kUnitA)), poly[b][e],
                               kNsB * (kUnitB / kUnitA) * ((float)hi[e] + (float)lo[e]));
                if (bj + col == bi + q4 + e) v += kNsA * kUnitB;
                poly[b][e] = v;
            }
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < kSmallGram; ++b) {
            const int i = wave + b * kSmallWaves;
            if (i >= across_m * across_m) continue;
            const int bi = i / across_m * 16, bj = (i - i / across_m * across_m) * 16;
            small_put4(a, bj + col, bi + q4, pitch_m, poly[b]);
        }
        __syncthreads();
        tile_f32x4 next[kSmallBlocks], turned[kSmallBlocks];
#pragma unroll
        for (int b = 0; b < kSmallBlocks; ++b) {
            const int i = wave + b * kSmallWaves;
            if (i >= across_m * across_n) continue;
            const int bi = i / across_n * 16, bj = (i - i / across_n * across_n) * 16;
            small_block<true>(a, xt, bi, bj, pitch_m, mr / 32, lane, next[b], turned[b]);
        }
        __syncthreads();
        const bool last = step + 1 == c.steps;
#pragma unroll
        for (int b = 0; b < kSmallBlocks; ++b) {
            const int i = wave + b * kSmallWaves;
            if (i >= across_m * across_n) continue;
            const int bi = i / across_n * 16, bj = (i - i / across_n * across_n) * 16;
            if (!last) {
                small_put4(x, bi + col, bj + q4, pitch_n, turned[b] * (1.0f / kUnitB));
                small_put4(xt, bj + col, bi + q4, pitch_m, next[b] * (1.0f / kUnitB));
                continue;
            }
            // along the rows of the matrix as it lies: four values of consecutive columns
            const int major = (g.tall ? bj : bi) + col, minor = (g.tall ? bi : bj) + q4;
            const tile_f32x4 v = g.tall ? next[b] : turned[b];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (major >= c.rows || minor + e >= c.cols) continue;
                const int64_t at = off + major * c.cols + minor + e;
                const float w = fmaf(-c.rate * (1.0f / (kUnitB * kUnitX)), v[e], c.keep * c.beta[at]);
                c.beta[at] = w;
                if (c.beta_bf16) c.beta_bf16[at] = (uint16_t)bf16_bits(w);
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ short sides of up to 96
// A = X X^T of a short side has one to three tiles, each of them a sum along the whole long side: the sum is cut into
// pieces for workgroups of their own, whose 64 x 64 sums k_muon_chain adds in order (2 x 44 x 7095: 37 us, cut 9 us).
struct GramPieceJob {
    static constexpr TilePair kPair = kSplit;
    static constexpr int kRowParts = 8;
    static constexpr bool kTurned = false;
    const char* x;
    float* sums;             // [matrix][tile][piece][64 * 64]
    int64_t pitch, size;
    int m, steps, pieces, tiles;

    __device__ __forceinline__ void place(int id, TilePos& p) const
    {
        const int tile = id / pieces, piece = id - tile * pieces;
        p.batch = tile / tiles;
        int mi, ni;
        triangle_order(tile - p.batch * tiles, mi, ni);
        p.m0 = mi * 64, p.n0 = ni * 64;
        const int first = (int)((int64_t)steps * piece / pieces);
        p.steps = (int)((int64_t)steps * (piece + 1) / pieces) - first;
        p.extra = first, p.id = id;
    }
    __device__ __forceinline__ const char* row(const TilePos& p, int r) const
    {
        return x + p.batch * size + (int64_t)(r < m ? r : m - 1) * pitch + (int64_t)p.extra * 128;
    }
    __device__ __forceinline__ const char* a_row(const TilePos& p, int r) const { return row(p, p.m0 + r); }
    __device__ __forceinline__ const char* b_row(const TilePos& p, int r) const { return row(p, p.n0 + r); }
    __device__ __forceinline__ void rows(const TilePos& p, int, int, const float* s, int it, int lane) const
    {
        const int run = (lane & 7) * 8, r = it * 8 + (lane >> 3);
        float v[8];
        piece_row8(s, r, run, v);
        tile_f32x4* o = reinterpret_cast<tile_f32x4*>(sums + (int64_t)p.id * 4096 + r * 64 + run);
        o[0] = tile_f32x4{v[0], v[1], v[2], v[3]};
        o[1] = tile_f32x4{v[4], v[5], v[6], v[7]};
    }
};

// What lies between the two products along the long side, B of one step or Q of two, in one launch: A and the
// polynomials stay in one workgroup's LDS, where the separate launches of each pair of steps take five times 5 us:
// 9 x 67 x 768 with 16-bit copy 120 us, then 101; 9 x 1 x 1856 116 us, then 81.
constexpr int kChainSide = 96, kChainBlocks = 5;   // 36 blocks of 16 x 16 over 8 waves

constexpr int kMostPieces = 16;

__host__ __device__ inline int chain_pieces(const MuonGeom& g)   // of eight k-steps or more, two a wave
{
    const int64_t pieces = g.pitch_n / 128 / 8;
    return pieces < 1 ? 1 : pieces < kMostPieces ? (int)pieces : kMostPieces;
}

__global__ __launch_bounds__(512) void k_muon_chain(const float* sums, char* out, MuonGeom g, int two)
{
    __shared__ __attribute__((aligned(1024))) char lds[3 * kChainSide * kChainSide * 4];
    const int tid = threadIdx.x, lane = tid & 63, q4 = (lane >> 4) * 4, col = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int mr = (int)(g.pitch_m / 4), pitch = (int)g.pitch_m, across = mr / 16;
    char *a = lds, *b = a + mr * pitch, *c = b + mr * pitch;
    out += blockIdx.x * g.size_a;
    const int side = (g.m + 63) / 64, tiles = side * (side + 1) / 2, pieces = chain_pieces(g);
    sums += (int64_t)blockIdx.x * tiles * pieces * 4096;
    for (int i = tid; i < tiles * 1024; i += 512) {
        const int t = i >> 10, mi = t > 0 ? 1 : 0, ni = t == 2 ? 1 : 0;   // (0, 0), (1, 0), (1, 1)
        const int r = mi * 64 + ((i & 1023) >> 4), k = ni * 64 + (i & 15) * 4;
        const float* from = sums + (int64_t)t * pieces * 4096 + (i & 1023) * 4;
        tile_f32x4 v = *reinterpret_cast<const tile_f32x4*>(from);
        for (int p = 1; p < pieces; ++p) v += *reinterpret_cast<const tile_f32x4*>(from + p * 4096);
        if (r >= mr || k >= mr) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = r < g.m && k + e < g.m ? v[e] * (kUnitA / (kUnitX * kUnitX)) : 0.0f;
        small_put4(a, r, k, pitch, v);
        if (mi != ni) {   // the half above the diagonal
#pragma unroll
            for (int e = 0; e < 4; ++e) small_put(a, k + e, r, pitch, v[e]);
        }
    }
    __syncthreads();
    tile_f32x4 unused;
    // blocks of left * right, four values of consecutive rows in a column each; symmetric
    auto product = [&](const char* left, const char* right, auto&& sink) {
#pragma unroll
        for (int t = 0; t < kChainBlocks; ++t) {
            const int i = wave + t * 8;
            if (i >= across * across) continue;
            const int bi = i / across * 16, bj = (i - i / across * across) * 16;
            tile_f32x4 v;
            small_block<false>(left, right, bi, bj, pitch, mr / 32, lane, v, unused);
            sink(bj + col, bi + q4, v);
        }
    };
    auto keep = [&](const char* left, const char* right, char* to, float unit) {
        product(left, right, [&](int r, int k, const tile_f32x4& v) { small_put4(to, r, k, pitch, v * unit); });
        __syncthreads();
    };
    auto step_factor = [&](const char* from, char* to) {   // a I + b A + c A A
        product(from, from, [&](int r, int k, tile_f32x4 v) {
            const int at = small_at(r, k, pitch);
            const f16x4 hi = *reinterpret_cast<const f16x4*>(from + at), lo = *reinterpret_cast<const f16x4*>(from + (at ^ 64));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = fmaf(kNsC * (kUnitB / (kUnitA * kUnitA)), v[e], kNsB * (kUnitB / kUnitA) * ((float)hi[e] + (float)lo[e]));
                if (r == k + e) v[e] += kNsA * kUnitB;
            }
            small_put4(to, r, k, pitch, v);
        });
        __syncthreads();
    };
    auto write = [&](int r, int k, const tile_f32x4& v) {
        if (r >= g.m) return;
        f16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            hi[e] = (_Float16)v[e];
            lo[e] = (_Float16)(v[e] - (float)hi[e]);
        }
        char* p = out + (int64_t)r * pitch + (k >> 5) * 128 + (k & 31) * 2;
        *reinterpret_cast<f16x4*>(p) = hi;
        *reinterpret_cast<f16x4*>(p + 64) = lo;
    };
    step_factor(a, b);
    if (two) {
        keep(b, a, c, 1.0f / kUnitB);   // B0 A
        keep(c, b, a, 1.0f / kUnitB);   // A'
        step_factor(a, c);              // B1
        product(c, b, [&](int r, int k, const tile_f32x4& v) { write(r, k, v * (kUnitQ / (kUnitB * kUnitB))); });
    } else {
        for (int i = tid; i < g.m * pitch / 16; i += 512) {
            const int r = i / (pitch / 16), at = i - r * (pitch / 16);
            *reinterpret_cast<tile_u32x4*>(out + (int64_t)r * pitch + at * 16) =
                *reinterpret_cast<const tile_u32x4*>(b + r * pitch + ((at ^ (r & 7)) << 4));
        }
    }
}

hipError_t launch_sym(SymJob j, int mats, hipStream_t stream)
{
    const TileChoice c = choose_tile(mats, j.m, j.m, j.steps, true);
    j.side = c.side;
    j.tiles = (int)(c.total / mats);
    j.total = (int)c.total;
    return launch_tiles(j, c, stream);
}

template <bool LAST>
hipError_t launch_apply(ApplyJob<LAST> j, hipStream_t stream)
{
    const TileChoice c = choose_tile(j.g.mats, j.g.m, j.g.n, j.g.pitch_m / 128, false);
    j.side = c.side;
    j.mt = (int)c.mt;
    j.nt = (int)c.nt;
    j.total = (int)c.total;
    return launch_tiles(j, c, stream);
}

}  // namespace

// Whether two steps are taken at once.  The multiplications are fewer from n = m on; at n = 2.9 m, with few tiles, both
// take the same (3 x 1501 x 515: 240 us and 239), at n = 4 m two at once take 0.8 of the time.
bool muon_pairs(const MuonGeom& g) { return g.n >= 2 * (int64_t)g.m; }

// the pieces' sums of A of one matrix with a short side of up to 96
int64_t chain_bytes(const MuonGeom& g)
{
    const int64_t side = (g.m + 63) / 64;
    return side * (side + 1) / 2 * chain_pieces(g) * 4096 * 4;
}

// sums | X along n, twice | X along m, twice | A | B | pieces of A | A', Q
int64_t muon_workspace_bytes(int rows, int cols, int n_mats)
{
    const MuonGeom g = muon_geom(rows, cols, n_mats);
    const int64_t sums = round_up((int64_t)n_mats * muon_sums((int64_t)rows * cols) * 8, 256);
    return sums + 2 * (round_up(n_mats * g.size_x, 256) + round_up(n_mats * g.size_t, 256)) +
           (muon_pairs(g) ? 4 : 2) * round_up(n_mats * g.size_a, 256) +
           (g.m <= kChainSide ? round_up(n_mats * chain_bytes(g), 256) : 0);
}

hipError_t launch_muon_update(const MuonCall& c, hipStream_t stream)
{
    const MuonGeom g = muon_geom(c.rows, c.cols, c.n_mats);
    const int64_t mr = round_up(g.m, 32), nr = round_up(g.n, 32);
    if (SmallNarrow::takes(mr, nr)) {
        hipLaunchKernelGGL(k_muon_small<SmallNarrow>, dim3(c.n_mats), dim3(SmallNarrow::kThreads), 0, stream, c, g);
        return hipGetLastError();
    }
    if (SmallWide::takes(mr, nr)) {
        hipLaunchKernelGGL(k_muon_small<SmallWide>, dim3(c.n_mats), dim3(SmallWide::kThreads), 0, stream, c, g);
        return hipGetLastError();
    }
    const int64_t count = (int64_t)c.rows * c.cols;
    const int n_sums = muon_sums(count);
    double* sums = reinterpret_cast<double*>(c.workspace);
    char* at = c.workspace + round_up((int64_t)c.n_mats * n_sums * 8, 256);
    auto take = [&](int64_t bytes) {
        char* p = at;
        at += round_up(bytes, 256);
        return p;
    };
    char* x[2] = {take(c.n_mats * g.size_x), take(c.n_mats * g.size_x)};
    char* t[2] = {take(c.n_mats * g.size_t), take(c.n_mats * g.size_t)};
    char *a = take(c.n_mats * g.size_a), *b = take(c.n_mats * g.size_a), *a2 = nullptr, *q = nullptr;
    const bool pairs = muon_pairs(g);
    float* pieces_sums = nullptr;
    if (mr <= kChainSide) pieces_sums = reinterpret_cast<float*>(take(c.n_mats * chain_bytes(g)));
    if (pairs) a2 = take(c.n_mats * g.size_a), q = take(c.n_mats * g.size_a);

    hipLaunchKernelGGL(k_muon_momentum, dim3(n_sums, c.n_mats), dim3(kSumBlock), 0, stream, c, count, sums);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_muon_start, dim3((c.cols + 63) / 64, (c.rows + 63) / 64, c.n_mats), dim3(kSumBlock), 0, stream, c, g,
                       sums, n_sums, g.tall ? t[0] : x[0], g.tall ? x[0] : t[0]);
    e = hipGetLastError();
    if (e != hipSuccess) return e;

    const int steps_m = (int)(g.pitch_m / 128), steps_n = (int)(g.pitch_n / 128);
    auto gram = [&](const char* from, char* to) {
        return launch_sym(SymJob{from, from, to, g.pitch_n, g.size_x, g.pitch_m, g.size_a, g.m, steps_n, 0, 0, 0, 0,
                                 kUnitA / (kUnitX * kUnitX)}, c.n_mats, stream);
    };
    // the product of two symmetric matrices that commute, or a I + b A + c A A
    auto square = [&](const char* one, const char* two, char* to, int poly, float unit) {
        return launch_sym(SymJob{one, two, to, g.pitch_m, g.size_a, g.pitch_m, g.size_a, g.m, steps_m, 0, 0, 0, poly, unit},
                          c.n_mats, stream);
    };
    int in = 0;
    for (int s = 0; s < c.steps;) {
        const bool two = pairs && s + 2 <= c.steps;
        const bool last = s + (two ? 2 : 1) == c.steps;
        if (mr <= kChainSide) {
            const int side = (g.m + 63) / 64, tiles = side * (side + 1) / 2, pieces = chain_pieces(g);
            hipLaunchKernelGGL(k_tile_cut<GramPieceJob>, dim3(c.n_mats * tiles * pieces), dim3(256), 0, stream,
                               GramPieceJob{x[in], pieces_sums, g.pitch_n, g.size_x, g.m, steps_n, pieces, tiles});
            hipLaunchKernelGGL(k_muon_chain, dim3(c.n_mats), dim3(512), 0, stream, pieces_sums, two ? q : b, g, (int)two);
            e = hipGetLastError();
        } else {
            e = gram(x[in], a);
            if (e == hipSuccess) e = square(a, a, b, 1, 1.0f);
        }
        if (two && mr > kChainSide) {
            if (e == hipSuccess) e = square(b, a, q, 0, kUnitA / (kUnitA * kUnitB));    // B0 A
            if (e == hipSuccess) e = square(q, b, a2, 0, kUnitA / (kUnitA * kUnitB));   // A'
            if (e == hipSuccess) e = square(a2, a2, a, 1, 1.0f);                        // B1
            if (e == hipSuccess) e = square(a, b, q, 0, kUnitQ / (kUnitB * kUnitB));
        }
        if (e != hipSuccess) return e;
        const char* factor = two ? q : b;
        const float per_unit = two ? 1.0f / kUnitQ : 1.0f / kUnitB;
        if (last) return launch_apply(ApplyJob<true>{factor, t[in], nullptr, nullptr, g, 0, 0, 0, 0, per_unit, c}, stream);
        e = launch_apply(ApplyJob<false>{factor, t[in], x[in ^ 1], t[in ^ 1], g, 0, 0, 0, 0, per_unit, c}, stream);
        if (e != hipSuccess) return e;
        in ^= 1;
        s += two ? 2 : 1;
    }
    return hipSuccess;
}

}  // namespace agc
