// Matrix products of the gated block and of the Newton-Schulz products: one tile loop for all of them.
//
// Every product here is C[m,n] = sum_k A[m,k] * B[n,k] with 16-bit operands whose rows are contiguous in k,
// held in groups ("k-steps") of parts of 64 bytes, 32 values each; operands that come in another order or with another
// end are laid out by a pass of their own before.  A k-step is either
//   plain   64 bfloat16 values of both operands:       C += A0 B0 + A1 B1     (its two halves of 32)
//   split   32 values as binary16 pairs, 32 high parts and 32 low parts (x = hi + lo to 22 bits):
//                                                      C += A0 B0 + A0 B1 + A1 B0   (lo * lo is below 2^-22)
//   parts3  32 binary32 values of A as three bfloat16 parts (v = A0 + A1 + A2, all 24 bits), 32 bfloat16 values of B:
//                                                      C += A0 B0 + A1 B0 + A2 B0
//   parts2  the same without the third part, 16 bits:  C += A0 B0 + A1 B0
// Products are v_mfma_f32_16x16x32, sums binary32.
//
// A workgroup of WM x WN waves owns a TM x TN tile of C and holds two k-steps of both operands in LDS, filled by
// loads that go from memory to LDS directly while the other k-step is multiplied.  Row r of a k-step of two parts lies at
// r * 128 bytes with its eight 16-byte chunks permuted by r & 7, which the loads do by choosing whose chunk a lane
// fetches: the sixteen rows that a wave reads at once then fall on all banks.  Where A and B differ in parts, both lie part
// by part, two rows of 64 bytes in 128, these eight chunks permuted in the same way.
// After the loop every wave stages its part of C, 64 x 64 values at a time, in its own 16 KB of the same LDS and
// hands it to the job, which reads it along rows or along columns, eight values a lane, and writes what it needs.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace agc {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 tile_bf16x8 __attribute__((ext_vector_type(8)));
typedef float tile_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t tile_u32x4 __attribute__((ext_vector_type(4)));

enum TilePair { kPlain, kSplit, kParts2, kParts3 };

// 64-byte parts of a row's k-step
template <TilePair PAIR>
struct TileStep {
    static constexpr bool kByPart = PAIR == kParts2 || PAIR == kParts3;
    static constexpr int kA = PAIR == kParts3 ? 3 : 2, kB = kByPart ? 1 : 2;
};

struct TilePos {
    int m0, n0;    // first row and column of the tile
    int batch;     // matrix or partition
    int steps;     // k-steps
    int extra, id; // what a job keeps of it
};

// Workgroup id -> place in the order of the tiles.  Workgroups go to the eight XCDs in turn; each XCD gets a
// contiguous run of tiles, so that the rows its tiles share stay in its own L2.
__device__ __forceinline__ int xcd_order(int id, int total)
{
    const int x = id & 7, per = total >> 3, rem = total & 7;
    return x * per + (x < rem ? x : rem) + (id >> 3);
}

// Place in the order -> (row tile, column tile) of mt x nt tiles: columns of up to kGroup row tiles, so that the 32
// tiles that an XCD works on at once form a block and not a line.
__device__ __forceinline__ void tile_order(int t, int mt, int nt, int& mi, int& ni)
{
    constexpr int kGroup = 8;
    const int block = t / (kGroup * nt), in = t - block * kGroup * nt;
    const int rows = mt - block * kGroup < kGroup ? mt - block * kGroup : kGroup;
    ni = in / rows;
    mi = block * kGroup + in - ni * rows;
}

// Place in the order -> (row tile, column tile <= row tile) of the lower triangle of a square of tiles.
__device__ __forceinline__ void triangle_order(int t, int& mi, int& ni)
{
    int r = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while ((r + 1) * (r + 2) / 2 <= t) ++r;      // the root is near, not exact
    while (r * (r + 1) / 2 > t) --r;
    mi = r;
    ni = t - r * (r + 1) / 2;
}

// ------------------------------------------------------------------ the staged part of C
// Value (r, c) of a 64 x 64 piece: the column is permuted by what the row's bits say, so that the writes from the
// matrix units' layout (4 x 16 rows and columns a wave), reads along rows and reads along columns (8 x 8 of them)
// each fall on all 64 banks.
__device__ __forceinline__ int piece_at(int r, int c)
{
    return r * 64 + (c ^ ((((r >> 2) & 3) << 4) ^ (((r >> 4) & 1) << 3) ^ (((r >> 5) & 1) << 4)));
}

__device__ __forceinline__ void piece_row8(const float* s, int r, int c, float v[8])
{
    const tile_f32x4* p = reinterpret_cast<const tile_f32x4*>(s + piece_at(r, c));
    const tile_f32x4 a = p[0], b = p[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}

__device__ __forceinline__ void piece_put_row8(float* s, int r, int c, const float v[8])
{
    tile_f32x4* p = reinterpret_cast<tile_f32x4*>(s + piece_at(r, c));
    p[0] = tile_f32x4{v[0], v[1], v[2], v[3]};
    p[1] = tile_f32x4{v[4], v[5], v[6], v[7]};
}

__device__ __forceinline__ void piece_col8(const float* s, int r, int c, float v[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = s[piece_at(r + i, c)];
}

// Lanes of one wave hand values to each other through LDS: nothing may move across.
__device__ __forceinline__ void wave_lds_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// ------------------------------------------------------------------ 16-bit stores
__device__ __forceinline__ uint32_t bf16_bits(float v)
{
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v);   // to nearest even
}

__device__ __forceinline__ tile_u32x4 bf16_pack8(const float v[8])
{
    typedef float pair_f32 __attribute__((ext_vector_type(2)));
    typedef __bf16 pair_bf16 __attribute__((ext_vector_type(2)));
    tile_u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i)   // both at once
        o[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pair_f32{v[2 * i], v[2 * i + 1]}, pair_bf16));
    return o;
}

__device__ __forceinline__ void bf16_unpack8(const tile_u32x4& u, float v[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}

// Eight values as binary16 pairs at element k (a multiple of 8) of a split row.
__device__ __forceinline__ void split_store8(char* row, int k, const float v[8])
{
    f16x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi[i] = (_Float16)v[i];
        lo[i] = (_Float16)(v[i] - (float)hi[i]);
    }
    char* p = row + (int64_t)(k >> 5) * 128 + (k & 31) * 2;
    *reinterpret_cast<f16x8*>(p) = hi;
    *reinterpret_cast<f16x8*>(p + 64) = lo;
}

__device__ __forceinline__ void split_load8(const char* row, int k, float v[8])
{
    const char* p = row + (int64_t)(k >> 5) * 128 + (k & 31) * 2;
    const f16x8 hi = *reinterpret_cast<const f16x8*>(p), lo = *reinterpret_cast<const f16x8*>(p + 64);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)hi[i] + (float)lo[i];
}

// Eight binary32 values as three bfloat16 parts at element k (a multiple of 8) of a row of A of parts3.  The first part is cut
// off, so that it cannot overflow, and leaves 16 bits; the second, rounded, leaves 8, which the third holds.  Infinity has no rest.
__device__ __forceinline__ void parts3_store8(char* row, int k, const float v[8])
{
    tile_u32x4 first;
    float rest[8], second[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = __float_as_uint(v[i]);
        rest[i] = (bits & 0x7FFFFFFFu) == 0x7F800000u ? 0.0f : v[i] - __uint_as_float(bits & 0xFFFF0000u);
        if (i & 1) first[i >> 1] = (__float_as_uint(v[i - 1]) >> 16) | (bits & 0xFFFF0000u);
    }
    const tile_u32x4 mid = bf16_pack8(rest);
    bf16_unpack8(mid, second);
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] -= second[i];
    char* p = row + (int64_t)(k >> 5) * 192 + (k & 31) * 2;
    *reinterpret_cast<tile_u32x4*>(p) = first;
    *reinterpret_cast<tile_u32x4*>(p + 64) = mid;
    *reinterpret_cast<tile_u32x4*>(p + 128) = bf16_pack8(rest);
}

// Eight binary32 values as two bfloat16 parts, both rounded, at element k of a row of A of parts2.
__device__ __forceinline__ void parts2_store8(char* row, int k, const float v[8])
{
    float first[8], rest[8];
    const tile_u32x4 top = bf16_pack8(v);
    bf16_unpack8(top, first);
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = fabsf(first[i]) == INFINITY ? 0.0f : v[i] - first[i];
    char* p = row + (int64_t)(k >> 5) * 128 + (k & 31) * 2;
    *reinterpret_cast<tile_u32x4*>(p) = top;
    *reinterpret_cast<tile_u32x4*>(p + 64) = bf16_pack8(rest);
}

// ------------------------------------------------------------------ the loop
template <TilePair PAIR>
__device__ __forceinline__ tile_f32x4 tile_mfma(const tile_u32x4& a, const tile_u32x4& b, const tile_f32x4& c)
{
    if constexpr (PAIR != kSplit)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(tile_bf16x8, a),
                                                       __builtin_bit_cast(tile_bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
}

__device__ __forceinline__ void load16_to_lds(const char* src, char* dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                     (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// Where the 16 rows of a fragment lie in LDS: the chunk of this lane (row lane & 15, values (lane >> 4) * 8 on) of the first part;
// the second part of rows of two: ^ 64.
template <bool BY_PART>
__device__ __forceinline__ int tile_chunk(int lane)
{
    const int row = lane & 15, q = lane >> 4;
    if (BY_PART) return (row >> 1) * 128 + ((((row & 1) * 4 + q) ^ (row >> 1)) << 4);
    return row * 128 + ((q ^ (row & 7)) << 4);
}

// One k-step of FM x FN blocks of 16 x 16, operands in LDS; parts of A that lie by part are `plane` bytes apart.
template <TilePair PAIR, int FM, int FN>
__device__ __forceinline__ void tile_multiply(const char* a, const char* b, int plane, int at0, int at1, tile_f32x4 (&acc)[FM][FN])
{
    if constexpr (TileStep<PAIR>::kByPart) {
        constexpr int kA = TileStep<PAIR>::kA;
        tile_u32x4 b0[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) b0[j] = *reinterpret_cast<const tile_u32x4*>(b + j * 1024 + at0);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            tile_u32x4 part[kA];
#pragma unroll
            for (int p = 0; p < kA; ++p) part[p] = *reinterpret_cast<const tile_u32x4*>(a + p * plane + i * 1024 + at0);
#pragma unroll
            for (int p = 0; p < kA; ++p)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = tile_mfma<PAIR>(part[p], b0[j], acc[i][j]);
        }
        return;
    }
    tile_u32x4 b0[FN], b1[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        b0[j] = *reinterpret_cast<const tile_u32x4*>(b + j * 2048 + at0);
        b1[j] = *reinterpret_cast<const tile_u32x4*>(b + j * 2048 + at1);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const tile_u32x4 a0 = *reinterpret_cast<const tile_u32x4*>(a + i * 2048 + at0);
        const tile_u32x4 a1 = *reinterpret_cast<const tile_u32x4*>(a + i * 2048 + at1);
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = tile_mfma<PAIR>(a0, b0[j], acc[i][j]);
        if constexpr (PAIR != kSplit) {
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = tile_mfma<PAIR>(a1, b1[j], acc[i][j]);
        } else {
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = tile_mfma<PAIR>(a0, b1[j], acc[i][j]);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = tile_mfma<PAIR>(a1, b0[j], acc[i][j]);
        }
    }
}

// JOB: kPair; void place(int id, TilePos&); const char* a_row(pos, r), b_row(pos, r): where row r of the tile starts
// (rows past the matrix name a row inside it; their results are not used); rows(pos, m, n, float* s, it, lane): what
// becomes of part `it` of kRowParts, along rows, of the 64 x 64 values staged at s, the first of them C[m, n]; and,
// where kTurned and turned(pos), cols(...): the same of eight parts along columns, after all rows().
//
// Bound by the matrix units at the power that they are given: B X of 2 x 4096 x 4096 (three products of pairs) 628 us,
// 1.31 PFLOP/s, and h of 8192 x 2048 x 8192 474 us, 1.16, where a library's product of 8192 x 8192 x 8192 reaches 1.45.
// 256 x 256 leaves room for one workgroup a compute unit, whose end (staging and stores, 9 to 20 us a tile) nothing
// overlaps; two workgroups of 128 x 128 overlap theirs but read LDS twice as much a product and are 7 to 20 % slower
// there.  They are taken where 256 x 256 would fill the units badly (choose_tile).
template <class JOB, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_tile(const JOB job)
{
    using Step = TileStep<JOB::kPair>;
    constexpr int kThreads = WM * WN * 64;
    constexpr int kWaveM = TM / WM, kWaveN = TN / WN, kFm = kWaveM / 16, kFn = kWaveN / 16;
    constexpr int kStep = (TM * Step::kA + TN * Step::kB) * 64;
    constexpr int kLds = 2 * kStep > WM * WN * 16384 ? 2 * kStep : WM * WN * 16384;
    // a load fills 128 bytes: a row of two parts, or two rows of one part
    constexpr int kRowsOf128 = Step::kByPart ? 2 : 1, kIssueLines = kThreads / 8;
    constexpr int kIssueA = TM / kRowsOf128 / kIssueLines, kIssueB = TN / kRowsOf128 / kIssueLines;
    constexpr int kLoadsA = Step::kByPart ? Step::kA : 1;   // of a lane for each of kIssueA
    static_assert(kWaveM % 64 == 0 && kWaveN == 64, "a wave stages pieces of 64 x 64");
    __shared__ __attribute__((aligned(1024))) char lds[kLds];

    TilePos pos;
    job.place((int)blockIdx.x, pos);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave - wm * WN;

    const char *src_a[kIssueA], *src_b[kIssueB];
    const int slot = (tid & 7) ^ ((tid >> 3) & 7);
    const int sub = Step::kByPart ? slot >> 2 : 0, chunk = (Step::kByPart ? slot & 3 : slot) * 16;
#pragma unroll
    for (int i = 0; i < kIssueA; ++i) src_a[i] = job.a_row(pos, (i * kIssueLines + (tid >> 3)) * kRowsOf128 + sub) + chunk;
#pragma unroll
    for (int i = 0; i < kIssueB; ++i) src_b[i] = job.b_row(pos, (i * kIssueLines + (tid >> 3)) * kRowsOf128 + sub) + chunk;

    auto issue = [&](int half) {
        char* base = lds + half * kStep + wave * 1024;
#pragma unroll
        for (int i = 0; i < kIssueA; ++i) {
#pragma unroll
            for (int p = 0; p < kLoadsA; ++p) load16_to_lds(src_a[i] + p * 64, base + p * TM * 64 + i * kIssueLines * 128);
            src_a[i] += Step::kA * 64;
        }
#pragma unroll
        for (int i = 0; i < kIssueB; ++i) {
            load16_to_lds(src_b[i], base + TM * Step::kA * 64 + i * kIssueLines * 128);
            src_b[i] += Step::kB * 64;
        }
    };

    tile_f32x4 acc[kFm][kFn];
#pragma unroll
    for (int i = 0; i < kFm; ++i)
#pragma unroll
        for (int j = 0; j < kFn; ++j) acc[i][j] = tile_f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int q = lane >> 4;
    const int at0 = tile_chunk<Step::kByPart>(lane), at1 = at0 ^ 64;
    auto multiply = [&](int half) {
        const char* a = lds + half * kStep + wm * kWaveM * (128 / kRowsOf128);
        const char* b = lds + half * kStep + TM * Step::kA * 64 + wn * kWaveN * (128 / kRowsOf128);
        tile_multiply<JOB::kPair, kFm, kFn>(a, b, TM * 64, at0, at1, acc);
    };

    if (pos.steps > 0) issue(0);
    for (int k = 0; k < pos.steps; ++k) {
        __syncthreads();   // this k-step has arrived, and nobody reads the other half any more
        if (k + 1 < pos.steps) issue((k + 1) & 1);
        multiply(k & 1);
    }

    __syncthreads();
    float* mine = reinterpret_cast<float*>(lds) + wave * 4096;
#pragma unroll
    for (int p = 0; p < kWaveM / 64; ++p) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    mine[piece_at(i * 16 + q * 4 + e, j * 16 + (lane & 15))] = acc[p * 4 + i][j][e];
        wave_lds_fence();
        const int m = pos.m0 + wm * kWaveM + p * 64, n = pos.n0 + wn * 64;
#pragma unroll
        for (int it = 0; it < JOB::kRowParts; ++it) job.rows(pos, m, n, mine, it, lane);
        if constexpr (JOB::kTurned) {
            wave_lds_fence();
            if (job.turned(pos)) {
#pragma unroll
                for (int it = 0; it < 8; ++it) job.cols(pos, m, n, mine, it, lane);
            }
        }
        wave_lds_fence();
    }
}

// The same product where there are few tiles: 64 x 64 tiles whose sum is cut among the four waves of a workgroup, every
// fourth k-step each.  A wave fills and reads LDS of its own, so nothing waits for anybody before the end, where the
// four parts are added in order.  Bound by the latency of a wave's own loads, 1.2 us for four k-steps: X X^T of
// 3 x 1501 x 515, 135 tiles of 47 k-steps, 14 us where 45 tiles of 128 x 128 take 35.
template <class JOB>
__global__ __launch_bounds__(256, 1) void k_tile_cut(const JOB job)
{
    using Step = TileStep<JOB::kPair>;
    constexpr int kStep = 64 * (Step::kA + Step::kB) * 64;
    constexpr int kRowsOf128 = Step::kByPart ? 2 : 1, kIssue = 8 / kRowsOf128, kLoadsA = Step::kByPart ? Step::kA : 1;
    __shared__ __attribute__((aligned(1024))) char lds[4 * 2 * kStep];
    TilePos pos;
    job.place((int)blockIdx.x, pos);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char* mine = lds + wave * 2 * kStep;

    const char *src_a[kIssue], *src_b[kIssue];
    const int slot = (lane & 7) ^ (lane >> 3);
    const int sub = Step::kByPart ? slot >> 2 : 0, chunk = (Step::kByPart ? slot & 3 : slot) * 16;
#pragma unroll
    for (int i = 0; i < kIssue; ++i) {
        const int r = (i * 8 + (lane >> 3)) * kRowsOf128 + sub;
        src_a[i] = job.a_row(pos, r) + chunk + wave * Step::kA * 64;
        src_b[i] = job.b_row(pos, r) + chunk + wave * Step::kB * 64;
    }
    auto issue = [&](char* base) {
#pragma unroll
        for (int i = 0; i < kIssue; ++i) {
#pragma unroll
            for (int p = 0; p < kLoadsA; ++p) load16_to_lds(src_a[i] + p * 64, base + p * 4096 + i * 1024);
            load16_to_lds(src_b[i], base + Step::kA * 4096 + i * 1024);
            src_a[i] += 4 * Step::kA * 64, src_b[i] += 4 * Step::kB * 64;
        }
    };
    constexpr int kLoads = kIssue * (kLoadsA + 1);   // of one k-step
    static_assert(kLoads == 16 || kLoads == 12, "the counted waits below");
    tile_f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = tile_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int q = lane >> 4;
    const int at0 = tile_chunk<Step::kByPart>(lane), at1 = at0 ^ 64;

    if (wave < pos.steps) issue(mine);
    for (int k = wave, half = 0; k < pos.steps; k += 4, half ^= 1) {
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the other half has been read
        if (k + 4 < pos.steps) {
            issue(mine + (half ^ 1) * kStep);
            if constexpr (kLoads == 16) __asm__ volatile("s_waitcnt vmcnt(16)" ::: "memory");   // all but the loads just issued
            else __asm__ volatile("s_waitcnt vmcnt(12)" ::: "memory");
        } else {
            __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const char* a = mine + half * kStep;
        tile_multiply<JOB::kPair, 4, 4>(a, a + Step::kA * 4096, 4096, at0, at1, acc);
    }
    __syncthreads();
    float* part = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                part[wave * 4096 + piece_at(i * 16 + q * 4 + e, j * 16 + (lane & 15))] = acc[i][j][e];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        tile_f32x4* p = reinterpret_cast<tile_f32x4*>(part) + i * 256 + tid;
        p[0] = (p[0] + p[1024]) + (p[2048] + p[3072]);
    }
    __syncthreads();
    for (int it = wave; it < JOB::kRowParts; it += 4) job.rows(pos, pos.m0, pos.n0, part, it, lane);
    if constexpr (JOB::kTurned) {
        __syncthreads();
        if (job.turned(pos)) {
            for (int it = wave; it < 8; it += 4) job.cols(pos, pos.m0, pos.n0, part, it, lane);
        }
    }
}

// Which of the three a product of `batch` matrices of m x n, `steps` k-steps each, takes, and how many tiles that are.
// The estimates are rounds of workgroups times microseconds of a k-step and of an end, as measured at 16 to 350 steps.
struct TileChoice {
    int side;        // 256, 128, or 64: the cut form
    int64_t mt, nt;  // tiles along m and n
    int64_t total;
};

inline TileChoice choose_tile(int64_t batch, int64_t m, int64_t n, int64_t steps, bool triangle)
{
    TileChoice best{};
    double least = 0.0;
    for (int side = 256; side >= 64; side /= 2) {
        TileChoice c{side, (m + side - 1) / side, (n + side - 1) / side, 0};
        c.total = batch * (triangle ? c.mt * (c.mt + 1) / 2 : c.mt * c.nt);
        const double s = (double)steps, t = (double)c.total;
        const double slots = side == 128 ? 512.0 : 256.0;
        const double rounds = (double)((c.total + (int64_t)slots - 1) / (int64_t)slots);
        double us;
        if (side == 256) us = rounds * (2.3 * s + 20.0);
        else if (side == 128) us = rounds * ((t > 256.0 ? 1.4 : 0.9) * s + 8.0);
        else us = rounds * (0.3 * s + 5.0);
        if (side == 256 || us < least) best = c, least = us;
    }
    return best;
}

template <class JOB>
hipError_t launch_tiles(JOB& j, const TileChoice& c, hipStream_t stream)
{
    if (c.total > INT32_MAX) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)c.total);
    if (c.side == 256) hipLaunchKernelGGL((k_tile<JOB, 256, 256, 2, 4>), grid, dim3(512), 0, stream, j);
    else if (c.side == 128) hipLaunchKernelGGL((k_tile<JOB, 128, 128, 2, 2>), grid, dim3(256), 0, stream, j);
    else hipLaunchKernelGGL(k_tile_cut<JOB>, grid, dim3(256), 0, stream, j);
    return hipGetLastError();
}

}  // namespace agc
