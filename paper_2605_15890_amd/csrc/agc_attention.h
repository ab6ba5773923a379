// Pieces of differential attention that its kernels share.
//
//   S_m = scale q_m k_m^T,  P_m = softmax of S_m over the keys in sight,  m = 1, 2;  out = (P_1 - lambda P_2) v
// Query head h holds its two maps' queries side by side, and shares keys and values with the other heads of its group.  A
// "row" is a (token, head of the group) pair: the rows of a sequence and key head are one matrix, whatever the group.
//
// All products are v_mfma_f32_32x32x16_bf16.  A wave owns 32 rows (or keys) as the columns of its products, so what
// belongs to a row stays in lane & 31 and the operands of its own side stay in registers; the other side passes through LDS
// in tiles that the whole workgroup shares.  A row of such a tile, both maps of a key or a value, has 4 D bytes; its 16-byte
// chunks are permuted by the row's low bits so that both kinds of reads fall on all banks: 32 rows at one chunk (an operand
// as it lies) and, by the transposing read, four rows at four neighbouring chunks (an operand turned).  Tiles come by loads
// that go from memory to LDS directly; the permutation is made by choosing whose chunk a lane fetches.
//
// The score product takes its keys in an order with bits 2 and 3 of the place swapped: a lane then ends with the scores of
// eight neighbouring keys twice, which is what the next product's operand wants, and P never leaves the registers.
#pragma once

#include "agc_dispatch.h"
#include "agc_operators.h"
#include "agc_vector.h"

namespace agc {

typedef float attn_f32x16 __attribute__((ext_vector_type(16)));
typedef short attn_s16x4 __attribute__((ext_vector_type(4)));

// What the kernels know of a call; operands as they are read, with 16-byte aligned rows.
struct Attn {
    const uint16_t *q, *k, *v;
    int64_t ldq, ldk, ldv;
    const float* lambda;
    const int32_t *q_end, *k_begin, *k_end;
    int n_seqs, tokens_q, tokens_k;
    int heads, kv_heads, d, e;
    int whole;            // heads of D and 2 D values; else of d and e, multiples of 8, whose tiles are filled up with zeros
    Divider group;        // heads that share keys, and the division of row numbers by them
    int causal;
    float scale;          // of the scores
    float to_log2;        // scale * log2(e), above zero: the maps are formed with powers of two
};

// A sequence's place in a tile's coordinates.
struct AttnSeq {
    int q0, lq, k0, lk;
};

__device__ __forceinline__ AttnSeq attn_sequence(const Attn& a, int s)
{
    AttnSeq o;
    const auto within = [](int v, int lo, int hi) { return min(max(v, lo), hi); };
    o.q0 = s ? within(a.q_end[s - 1], 0, a.tokens_q) : 0;
    o.lq = within(a.q_end[s], o.q0, a.tokens_q) - o.q0;
    o.k0 = a.k_begin ? within(a.k_begin[s], 0, a.tokens_k) : s ? within(a.k_end[s - 1], 0, a.tokens_k) : 0;
    o.lk = within(a.k_end[s], o.k0, a.tokens_k) - o.k0;
    return o;
}

// Which sequence tile `slot` belongs to, where sequence s has the tiles from begin_s * unit / size + s on: room for its
// ceil(length * unit / size), found without a table of them.  `end` are the sequences' ends.
__device__ __forceinline__ int attn_first_slot(const int32_t* end, int s, int most, uint32_t unit, uint32_t size)
{
    const uint32_t begin = s ? (uint32_t)min(max(end[s - 1], 0), most) : 0;
    return (int)(begin * unit / size) + s;
}

// The last sequence whose first tile is not behind `slot`, each lane looking at one of 64 evenly spaced ones at a time.
__device__ __forceinline__ int attn_find(const int32_t* end, int n_seqs, int most, uint32_t unit, uint32_t size, int slot)
{
    const int lane = threadIdx.x & 63;
    int first = 0;
    for (int left = n_seqs; left > 1;) {
        const int step = (left + 63) >> 6, s = lane * step;
        const int before = __popcll(__ballot(s < left && attn_first_slot(end, first + min(s, left - 1), most, unit, size) <= slot));
        const int go = max(before - 1, 0) * step;
        first += go;
        left = min(step, left - go);
    }
    return first;
}

// Workgroup id -> tile, key head, split.  Workgroups go to the eight XCDs in turn.
//
// Without `columns` each XCD gets a contiguous run, so that tiles of the same keys meet in its L2 -- or every eighth workgroup,
// which gives all as much to do where sequences differ: with tiles enough that some of them meet all the same (8111 tokens in
// five sequences, 8 heads of 128: 256 instead of 288 us), and with one tile a sequence, none of which meet (8 sequences' queries of
// 131072 keys, 8 heads of 128: 54 instead of 62; but 64 queries each, 4 tiles of a sequence, 122 instead of 80).  The gradients'
// passes follow: both together 2210 instead of 2330 us for the 8111 tokens, 1439 instead of 1447 for one sequence of 8300 (6 heads
// of 64), else no difference (12000 tokens in six, 15000 in seven).
//
// Under the causal mask a sequence's first tiles have most to do, and such a run ends with some of them: with columns, an XCD
// has whole key heads (or a share of one's tiles), every sequence's first tiles come before all second ones, and the last ones
// fill the gaps.  Tiles count as n_seqs rows of `columns` each, which they are if the sequences are alike; if not, the order is
// any.  8 x 2048 tokens, 16 heads: forward 281 -> 258 us, rows' pass 605 -> 535, keys' pass 612 -> 552.
struct AttnPlace {
    int slot, head_k, split;   // slot -1: none
};

__device__ __forceinline__ AttnPlace attn_place(const Attn& a, int id, int slots, int splits, int columns)
{
    if (columns == 0) {
        if (id >= slots * a.kv_heads * splits) return {-1, 0, 0};
        const bool spread = slots <= 2 * a.n_seqs || (splits == 1 && slots >= 32 * a.n_seqs);
        if (!spread) id = xcd_order(id, slots * a.kv_heads * splits);
        const int rest = id / splits, head_k = rest / slots;
        return {rest - head_k * slots, head_k, id - rest * splits};
    }
    const int x = id & 7, i = id >> 3, share = max(8 / a.kv_heads, 1), rows = max(a.kv_heads / 8, 1) * a.n_seqs;
    const int step = i / rows, row = i - step * rows, head = row / a.n_seqs, column = step * share + x % share;
    const int slot = (row - head * a.n_seqs) * columns + column;
    return {column < columns && slot < slots ? slot : -1, a.kv_heads >= 8 ? x * (a.kv_heads / 8) + head : x / share, 0};
}

// Keys in sight of query t.
__device__ __forceinline__ int attn_seen(const Attn& a, const AttnSeq& q, int t)
{
    return a.causal ? min(max(t + q.lk - q.lq + 1, 0), q.lk) : q.lk;
}

// 0 .. 31 with bits 2 and 3 swapped.
__device__ __forceinline__ int attn_swapped(int i) { return (i & 0x13) | (i & 4) << 1 | (i & 8) >> 1; }

typedef __attribute__((address_space(3))) char* AttnLds;

__device__ __forceinline__ void attn_load16(const char* src, AttnLds dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

__device__ __forceinline__ void attn_load4(const float* src, AttnLds dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 4, 0, 0);
}

static __device__ __attribute__((aligned(16))) const uint32_t attn_zeros[4] = {};

// A head of an operand in memory: RUNS runs (two maps or one of values), 2 D values in a tile, WHOLE if here too, `width` a run if
// not.
template <int D, int RUNS, bool WHOLE>
struct AttnHead {
    static constexpr int kRun = 2 * D / RUNS;
    int width;
    __device__ __forceinline__ int run() const { return WHOLE ? kRun : width; }
    __device__ __forceinline__ int size() const { return RUNS * run(); }
    // where chunk c of 16 bytes of a row that begins `at` bytes behind base comes from
    __device__ __forceinline__ const char* chunk(const char* base, uint32_t at, int c) const
    {
        if constexpr (WHOLE) return base + (at + c * 16);
        const int r = c / (kRun / 8), in = c % (kRun / 8) * 8;
        return in < width ? base + (at + (r * width + in) * 2) : reinterpret_cast<const char*>(attn_zeros);
    }
    // values in .. in + 7 of run r
    __device__ __forceinline__ tile_bf16x8 values(const uint16_t* row, int r, int in) const
    {
        return *reinterpret_cast<const tile_bf16x8*>(chunk(reinterpret_cast<const char*>(row), 0, (r * kRun + in) / 8));
    }
};

template <int D>
struct AttnTile {
    static constexpr int kRow = 4 * D, kChunks = kRow / 16;
    // what the chunks of a row are permuted by
    static __device__ __forceinline__ int mix(int row)
    {
        if constexpr (D == 32) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);   // two rows span the banks
        return (row & 3) << 2 | ((row >> 2) & 3);
    }

    // Rows 0 .. ROWS - 1 of a matrix in memory, `base` the first one's address, the same for all lanes, to LDS; those from `rows` on
    // are the last one again.  Whole tiles cost an addition a load.
    template <int ROWS, int WAVES, typename Head>
    static __device__ __forceinline__ void load(AttnLds lds, int wave, int lane, const Head& head, const char* base, uint32_t stride, int rows)
    {
        constexpr int kPer = 64 / kChunks;   // rows a wave fetches at once
        constexpr int kTimes = ROWS / kPer / WAVES;
        static_assert(ROWS % (kPer * WAVES) == 0, "every wave fetches alike");
        if (rows >= ROWS) {
#pragma unroll
            for (int i = 0; i < kTimes; ++i) {
                const int c = i * WAVES + wave, row = c * kPer + lane / kChunks;
                attn_load16(head.chunk(base + (int64_t)(c * kPer) * stride, (uint32_t)(lane / kChunks) * stride, (lane % kChunks) ^ mix(row)),
                            lds + c * 1024);
            }
        } else {
#pragma unroll 1
            for (int c = wave; c < ROWS / kPer; c += WAVES) {
                // more than 128 rows, 2^25 bytes apart at most, lie further than 32 bits reach: those count from a fetch's first one
                const int row = c * kPer + lane / kChunks, first = ROWS > 128 ? min(c * kPer, rows - 1) : 0;
                attn_load16(head.chunk(base + (int64_t)first * stride, (uint32_t)(min(row, rows - 1) - first) * stride, (lane % kChunks) ^ mix(row)),
                            lds + c * 1024);
            }
        }
    }
};

// A lane's places in a tile for both kinds of reads.  A chunk's permutation is an exclusive or, so one place gives all of them.
template <int D>
struct AttnReads {
    using Tile = AttnTile<D>;
    static constexpr int kWide = Tile::kChunks < 16 ? Tile::kChunks : 16;   // chunks that are permuted among each other
    uint32_t as_it_lies, across;

    __device__ __forceinline__ explicit AttnReads(int lane, int map0 = 0)
    {
        const int row = attn_swapped(lane & 31);
        as_it_lies = row * Tile::kRow + (((lane >> 5) ^ Tile::mix(row)) << 4) + map0 * 2 * D;
        const int i = lane & 15, x = ((lane >> 4) & 1) * 2 + ((i & 3) >> 1), r = 8 * (lane >> 5) + (i >> 2);
        across = r * Tile::kRow + ((x ^ Tile::mix(r)) << 4) + (i & 1) * 8;
    }
    // Values 16 j + 8 (lane / 32) + 0 .. 7 of a row of the 32 rows `tile` bytes behind `lds`, the row being lane & 31 with bits 2 and 3 swapped:
    // the registers of a product of it are then eight neighbouring rows twice.  (From the second map's values on with map0 = 1.)
    __device__ __forceinline__ tile_bf16x8 straight(AttnLds lds, uint32_t tile, int j) const
    {
        typedef __attribute__((address_space(3))) const tile_bf16x8* At;
        constexpr int kMod = kWide / 2;
        return *(At)(lds + ((tile + as_it_lies) ^ (j % kMod * 32)) + j / kMod * (kWide * 16));
    }
    // Value 32 b + (lane & 31) of the rows row0 + 8 (lane / 32) + 0 .. 7 there, row0 a multiple of 16.
    __device__ __forceinline__ tile_bf16x8 turned(AttnLds lds, uint32_t tile, int row0, int b) const
    {
        typedef __attribute__((address_space(3))) attn_s16x4* At;
        constexpr int kMod = kWide / 4;
        const uint32_t at = tile + across, more = row0 * Tile::kRow + b / kMod * (kWide * 16), flip = b % kMod * 64;
        const attn_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(lds + (at ^ flip) + more));
        // four rows on the permutation differs in its lowest bit
        const attn_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(lds + (at ^ (flip | 16)) + more + 4 * Tile::kRow));
        return __builtin_bit_cast(tile_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Row that register r of a 32 x 32 product belongs to, with the operand's rows swapped (score products) and as they are.
__device__ __forceinline__ int attn_row_swapped(int r, int lane) { return 16 * (r >> 3) + 8 * (lane >> 5) + (r & 7); }
__device__ __forceinline__ int attn_row_plain(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

__device__ __forceinline__ attn_f32x16 attn_mfma(const tile_bf16x8& a, const tile_bf16x8& b, const attn_f32x16& c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// N products whose operands come from LDS, AHEAD of them read while the AHEAD before are multiplied: left to itself the compiler
// puts each read right before its product, which then waits for it.  `start` may be called long before `run`.
template <int N, int AHEAD, typename Read>
struct AttnStream {
    static_assert(N % AHEAD == 0, "whole groups");
    const Read& read;
    tile_bf16x8 part[2][AHEAD];
    __device__ __forceinline__ explicit AttnStream(const Read& r) : read(r) {}
    __device__ __forceinline__ void start()
    {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) part[0][i] = read(i);
    }
    template <typename Use>
    __device__ __forceinline__ void run(const Use& use)
    {
#pragma unroll
        for (int g = 0; g < N / AHEAD; ++g) {
            __builtin_amdgcn_sched_barrier(0);
            if (g + 1 < N / AHEAD) {
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) part[(g + 1) & 1][i] = read((g + 1) * AHEAD + i);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) use(g * AHEAD + i, part[g & 1][i]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
};

template <int N, int AHEAD, typename Read>
__device__ __forceinline__ AttnStream<N, AHEAD, Read> attn_stream(const Read& read)
{
    return AttnStream<N, AHEAD, Read>(read);
}

// The other half's value of the same column.
__device__ __forceinline__ float attn_other_half(float v) { return __shfl_xor(v, 32); }

// Eight values as two bfloat16 parts, sixteen bits of each together.
struct AttnTwo {
    tile_bf16x8 top, rest;
    __device__ __forceinline__ explicit AttnTwo(const float v[8])
    {
        float first[8], low[8];
        const tile_u32x4 bits = bf16_pack8(v);
        bf16_unpack8(bits, first);
#pragma unroll
        for (int i = 0; i < 8; ++i) low[i] = v[i] - first[i];
        top = __builtin_bit_cast(tile_bf16x8, bits);
        rest = __builtin_bit_cast(tile_bf16x8, bf16_pack8(low));
    }
};

__device__ __forceinline__ attn_f32x16 attn_mfma(const tile_bf16x8& a, const AttnTwo& b, const attn_f32x16& c)
{
    return attn_mfma(a, b.rest, attn_mfma(a, b.top, c));
}

// Registers 8 b .. 8 b + 7 as an operand.
__device__ __forceinline__ tile_bf16x8 attn_operand(const float v[16], int b)
{
    return __builtin_bit_cast(tile_bf16x8, bf16_pack8(v + 8 * b));
}

// Values of a column of C (32 rows of `acc`, times `factor`) to a row of an output, as far as `width` goes.
__device__ __forceinline__ void attn_store(uint16_t* row, int at, int width, int lane, const attn_f32x16& acc, float factor)
{
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
        const int c = at + attn_row_plain(r, lane);
        if (c + 4 <= width) {
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            const u32x2 v = {bf16_bits(acc[r] * factor) | bf16_bits(acc[r + 1] * factor) << 16,
                             bf16_bits(acc[r + 2] * factor) | bf16_bits(acc[r + 3] * factor) << 16};
            __builtin_memcpy(row + c, &v, 8);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < width) row[c + i] = (uint16_t)bf16_bits(acc[r + i] * factor);
        }
    }
}

// The same in binary32, to a part of a split.
__device__ __forceinline__ void attn_store_part(float* row, int lane, const attn_f32x16& acc, float factor)
{
#pragma unroll
    for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<tile_f32x4*>(row + attn_row_plain(r, lane)) =
            tile_f32x4{acc[r] * factor, acc[r + 1] * factor, acc[r + 2] * factor, acc[r + 3] * factor};
}

__device__ __forceinline__ void attn_wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }   // vmcnt(0)

// ------------------------------------------------------------------ laying operands out
struct AttnPack {
    const uint16_t* from;
    uint16_t* to;
    int64_t ld;
    int rows, parts, width, up;   // `parts` runs of `width` values a row become runs of `up`
};

// What the gradients take of the workspace beyond that.
int64_t attn_gradients_bytes(int64_t tokens_q, int64_t tokens_k, int n_seqs, int heads, int kv_heads, int D);
hipError_t attn_pack(const AttnPack* jobs, int n, hipStream_t stream);
// Fills `a` from the call, copying operands that are not read where they lie to the workspace; `place` moves on behind them.
hipError_t attn_lay_out(const AttnCall& c, Attn& a, const uint16_t*& dout, int64_t& lddout, char*& place, hipStream_t stream);

}  // namespace agc
