// Differential attention, forward:  out = (softmax(scale q1 k1^T) - lambda softmax(scale q2 k2^T)) v  over the keys of each
// sequence that are in sight.  Both maps are formed in one pass over the keys with their running maxima and sums.
//
// A workgroup has 32 rows a wave, both maps of them (wide heads: one map a wave), and tiles of 64 keys pass two buffers.  For 32
// rows, 32 keys, both maps 64 wide and values of 128, a SIMD's matrix unit is busy for 768 cycles (24 products), its vector
// unit for about 950 with powers, sums and maxima, and the compute unit's LDS for 128 times four waves.  4 x 4096 tokens, 16
// heads on 4 key heads, causal, take 390 us: 1.05 PFLOP/s of products, matrix units busy for 0.50 and vector units for 0.64 of
// the time at the 1.6 to 1.9 GHz that the card's power then allows, where a library product of 8192^3 reaches 1.28.
// Few rows leave memory as the bound: 8 sequences' queries over 131072 keys, 16 heads on 4, 50 us, 5.4 TB/s, and 5 to join.
#include <algorithm>
#include <limits>

#include "agc_attention.h"

namespace agc {

namespace {

struct AttnForward {
    Attn a;
    uint16_t* out;
    int64_t ldo;
    float* lse;            // may be null
    int slots, splits, columns;
    float* part;           // of splits: per (split, row) both maps' sums of 2 D values
    struct AttnStat* stat; // and their maxima and sums
};

struct AttnStat {
    float top, sum;
};

constexpr int kMostSplits = 256, kFewSplits = 8;   // from there on a row's splits are joined several at once

// Wide heads are worked on by a wave for each map: both maps' sums of 256 values would take all its registers.
constexpr int attn_maps_of_a_wave(int D) { return D == 128 ? 1 : 2; }

// Once a row's largest score has grown by more than this many powers of two, what is summed so far is scaled down to it.
constexpr float kGrowth = 8.0f;

// SHARE waves have the same rows, and every SHAREth 32 keys of them each: where rows are few, pairs halve the chain of tiles that a
// wave goes through and meet once at its end (2999 queries in six sequences, 6 heads on 2: 24 instead of 36 us).
template <int D, int WAVES, int KT, int SHARE, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES, WAVES * attn_maps_of_a_wave(D) == 2 ? 1 : 2) void k_attn_forward(AttnForward f)
{
    using Tile = AttnTile<D>;
    constexpr int E = 2 * D, kSteps = D / 16, kBlocks = E / 32;
    constexpr int kMaps = attn_maps_of_a_wave(D), kRows = 32 * WAVES * kMaps / 2 / SHARE;
    constexpr int kTile = KT * Tile::kRow;
    __shared__ __attribute__((aligned(1024))) char lds[2][2][kTile];   // buffer; keys, values
    const Attn& a = f.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int map0 = kMaps == 2 ? 0 : wave & 1, rows_of = (kMaps == 2 ? wave : wave >> 1) / SHARE;
    const int turn = SHARE == 1 ? 0 : wave % SHARE;
    static_assert(SHARE == 1 || (SHARE == 2 && kMaps == 2), "a pair of waves for both maps");
    const AttnPlace place = attn_place(a, blockIdx.x, f.slots, f.splits, f.columns);
    const int slot = place.slot, head_k = place.head_k, split = place.split;
    if (slot < 0) return;
    const uint32_t group = a.group.d;

    const int s = attn_find(a.q_end, a.n_seqs, a.tokens_q, group, kRows, slot);
    const AttnSeq seq = attn_sequence(a, s);
    const int first = attn_first_slot(a.q_end, s, a.tokens_q, group, kRows);
    const int rows = seq.lq * (int)group, tiles = (rows + kRows - 1) / kRows;
    // the last tiles see most keys and come first
    const int tile_id = tiles - 1 - (slot - first);
    if (tile_id < 0 || tile_id >= tiles) return;

    const int row_ = tile_id * kRows + rows_of * 32 + (lane & 31);
    const int row = min(row_, rows - 1), t = (int)a.group(row), g = row - t * (int)group, head = head_k * (int)group + g;
    const int seen = attn_seen(a, seq, t);
    const int last_row = min(tile_id * kRows + kRows, rows) - 1;
    const int keys = attn_seen(a, seq, (int)a.group(last_row));   // of the tile
    const int run = (keys + f.splits * KT - 1) / (f.splits * KT) * KT;
    const int begin = min(split * run, keys), end = min(begin + run, keys);
    // of the wave's rows: what the first and the last one see
    const int seen_least = min(__builtin_amdgcn_readfirstlane(seen), end), seen_most = min(__builtin_amdgcn_readlane(seen, 31), end);

    const AttnHead<D, 2, WHOLE> maps{a.d};
    const AttnHead<D, 1, WHOLE> ofv{a.e};
    tile_bf16x8 q[kMaps][kSteps];
    {
        const uint16_t* p = a.q + (int64_t)(seq.q0 + t) * a.ldq + (int64_t)head * maps.size();
#pragma unroll
        for (int m = 0; m < kMaps; ++m)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) q[m][i] = maps.values(p, map0 + m, (lane >> 5) * 8 + i * 16);
    }
    const char* const keys_at = reinterpret_cast<const char*>(a.k + (int64_t)seq.k0 * a.ldk + head_k * maps.size());
    const char* const values_at = reinterpret_cast<const char*>(a.v + (int64_t)seq.k0 * a.ldv + head_k * ofv.size());
    const auto fetch = [&](AttnLds to, int j0) {
        Tile::template load<KT, WAVES>(to, wave, lane, maps, keys_at + (int64_t)j0 * a.ldk * 2, (uint32_t)a.ldk * 2, seq.lk - j0);
        Tile::template load<KT, WAVES>(to + kTile, wave, lane, ofv, values_at + (int64_t)j0 * a.ldv * 2, (uint32_t)a.ldv * 2, seq.lk - j0);
    };

    attn_f32x16 acc[kMaps][kBlocks];
    // the largest scores that the sums are relative to, zero where there is none yet
    float top[kMaps], from[kMaps], sum[kMaps];
#pragma unroll
    for (int m = 0; m < kMaps; ++m) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) acc[m][b] = attn_f32x16{};
        top[m] = -INFINITY, from[m] = sum[m] = 0.0f;
    }
    const AttnReads<D> reads(lane, map0);

    // __restrict__: the tile that is filled is another than the one that is read, else the first read would wait for the loads
    const auto step = [&](AttnLds __restrict__ from_lds, AttnLds __restrict__ to_lds, int j0) {
        if (j0 + KT < end) fetch(to_lds, j0 + KT);
        uint32_t k_tile = turn * 32 * Tile::kRow;
#pragma unroll 1
        for (int j = j0 + turn * 32; j < min(j0 + KT, seen_most); j += 32 * SHARE, k_tile += 32 * SHARE * Tile::kRow) {
            const uint32_t v_tile = k_tile + kTile;
            attn_f32x16 score[kMaps] = {};
            const auto read_k = [&](int n) { return reads.straight(from_lds, k_tile, n % kMaps * kSteps + n / kMaps); };
            auto of_k = attn_stream<kMaps * kSteps, 4>(read_k);
            of_k.start();
            of_k.run([&](int n, const tile_bf16x8& k) { score[n % kMaps] = attn_mfma(k, q[n % kMaps][n / kMaps], score[n % kMaps]); });
            if (j + 32 > seen_least) {
                const int left = min(seen, end) - j;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool in = attn_row_swapped(r, lane) < left;
#pragma unroll
                    for (int m = 0; m < kMaps; ++m) score[m][r] = in ? score[m][r] : -INFINITY;
                }
            }
            bool grown = false;
            float most[kMaps];
#pragma unroll
            for (int m = 0; m < kMaps; ++m) {
                most[m] = score[m][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) most[m] = fmaxf(most[m], score[m][r]);
                most[m] *= a.to_log2;
                grown |= most[m] > top[m] + kGrowth;
            }
            if (__any(grown)) {
#pragma unroll
                for (int m = 0; m < kMaps; ++m) {
                    const float now = fmaxf(top[m], fmaxf(most[m], attn_other_half(most[m])));
                    const float shrink = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top[m] - now);
                    top[m] = now;
                    from[m] = now == -INFINITY ? 0.0f : now;
                    sum[m] *= shrink;
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[m][b][r] *= shrink;
                }
            }
            const auto read_v = [&](int n) { return reads.turned(from_lds, v_tile, n / kBlocks * 16, n % kBlocks); };
            auto of_v = attn_stream<2 * kBlocks, kBlocks % 4 ? 2 : 4>(read_v);
            of_v.start();
            // The maps are rounded to one bfloat16 part: out is off by 1.7e-3 to 2.1e-3 in the 2-norm where its own rounding
            // leaves 1.66e-3.  Two parts, as in the gradients, would take 617 instead of 415 us (4 x 4096 tokens, 16 heads on 4),
            // 353 instead of 248 (8 x 2048, 16 heads) and 309 instead of 221 (8111 tokens, 8 heads of 128 on 2).
            tile_bf16x8 p[kMaps][2];
#pragma unroll
            for (int m = 0; m < kMaps; ++m) {
                float v[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    v[r] = __builtin_amdgcn_exp2f(fmaf(score[m][r], a.to_log2, -from[m]));
                    sum[m] += v[r];
                }
                p[m][0] = attn_operand(v, 0);
                p[m][1] = attn_operand(v, 1);
            }
            of_v.run([&](int n, const tile_bf16x8& v) {
#pragma unroll
                for (int m = 0; m < kMaps; ++m) acc[m][n % kBlocks] = attn_mfma(v, p[m][n / kBlocks], acc[m][n % kBlocks]);
            });
        }
    };
    const AttnLds all = (AttnLds)&lds[0][0][0];
    if (begin < end) fetch(all, begin);
    int buffer = 0;
#pragma unroll 1
    for (int j0 = begin; j0 < end; j0 += KT, buffer ^= 1) {
        attn_wait_loads();
        __syncthreads();
        step(all + buffer * (2 * kTile), all + (buffer ^ 1) * (2 * kTile), j0);
    }

    if constexpr (SHARE == 2) {
        // the second wave hands its sums to the first, where the tiles were
        __shared__ float stats[WAVES / 2][2][2][64];
        static_assert(WAVES / 2 * 2 * kBlocks * 16 * 64 * 4 <= (int)sizeof(lds), "they fit");
        float* box = reinterpret_cast<float*>(lds) + rows_of * (2 * kBlocks * 16 * 64) + lane;
        __syncthreads();
        if (turn == 1) {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                stats[rows_of][m][0][lane] = top[m], stats[rows_of][m][1][lane] = sum[m];
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) box[((m * kBlocks + b) * 16 + r) * 64] = acc[m][b][r];
            }
        }
        __syncthreads();
        if (turn == 1) return;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const float top2 = stats[rows_of][m][0][lane], now = fmaxf(top[m], top2);
            const float own = top[m] == now ? 1.0f : __builtin_amdgcn_exp2f(top[m] - now), by = top2 == now ? 1.0f : __builtin_amdgcn_exp2f(top2 - now);
            top[m] = now;
            sum[m] = fmaf(stats[rows_of][m][1][lane], by, sum[m] * own);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][b][r] = fmaf(box[((m * kBlocks + b) * 16 + r) * 64], by, acc[m][b][r] * own);
        }
    }
#pragma unroll
    for (int m = 0; m < kMaps; ++m) sum[m] += attn_other_half(sum[m]);
    if (f.splits > 1) {
        if (row_ >= rows) return;
        const int64_t at = (int64_t)split * a.tokens_q * a.heads + (int64_t)head_k * a.tokens_q * group + (int64_t)seq.q0 * group + row;
#pragma unroll
        for (int m = 0; m < kMaps; ++m) {
            if (lane < 32) f.stat[2 * at + map0 + m] = AttnStat{top[m], sum[m]};
            if (begin >= end) continue;
            float* o = f.part + (2 * at + map0 + m) * E;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) attn_store_part(o + b * 32, lane, acc[m][b], 1.0f);
        }
        return;
    }
    float by[kMaps];
#pragma unroll
    for (int m = 0; m < kMaps; ++m) {
        by[m] = sum[m] == 0.0f ? 0.0f : 1.0f / sum[m];
        if (f.lse && lane < 32 && row_ < rows)
            f.lse[(int64_t)(2 * head + map0 + m) * a.tokens_q + seq.q0 + t] = sum[m] == 0.0f ? -INFINITY : top[m] + __builtin_amdgcn_logf(sum[m]);
    }
    const float lambda = a.lambda[head];
    // a row without keys in sight is zeros, whatever the values that others see
    const auto share = [&](int m, int b, int r) { return by[m] == 0.0f ? 0.0f : acc[m][b][r] * by[m]; };
    if constexpr (kMaps == 2) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[0][b][r] = share(0, b, r) - lambda * share(1, b, r);
    } else {
        // the second map's wave hands its sums to the first map's, which has the same rows
        static_assert(WAVES / 2 * 32 * E * 4 <= (int)sizeof(lds), "they fit where the tiles were");
        float* box = reinterpret_cast<float*>(lds) + rows_of * (32 * E) + lane;
        __syncthreads();
        if (map0 == 1) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) box[(b * 16 + r) * 64] = lambda * share(0, b, r);
        }
        __syncthreads();
        if (map0 == 1) return;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[0][b][r] = share(0, b, r) - box[(b * 16 + r) * 64];
    }
    if (row_ >= rows) return;
    uint16_t* o = f.out + (int64_t)(seq.q0 + t) * f.ldo + (int64_t)head * a.e;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) attn_store(o, b * 32, a.e, lane, acc[0][b], 1.0f);
}

// Joins the splits: a row's 4 D sums of both maps by D threads, four each, times ABREAST splits at once, whose sums meet in LDS.
template <int D, int ABREAST>
__global__ __launch_bounds__(256) void k_attn_join(AttnForward f)
{
    constexpr int kRows = 256 / (D * ABREAST);
    const Attn& a = f.a;
    const int lane = threadIdx.x & 63;
    const int64_t all = (int64_t)a.tokens_q * a.heads, row0 = (int64_t)blockIdx.x * kRows;
    const int group = (int)a.group.d;
    __shared__ float weights[kRows][2][ABREAST > 1 ? kMostSplits : kFewSplits];
    for (int r = threadIdx.x >> 6; r < kRows && row0 + r < all; r += 4) {
        const int64_t at = row0 + r, of_head = (int64_t)a.tokens_q * group;
        const int head_k = (int)(at / of_head), row = (int)(at - head_k * of_head), t = (int)a.group(row), head = head_k * group + row - t * group;
        float top[2], sum[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            // a lane a split: what its sums are multiplied with; one without keys left nothing in memory
            constexpr int kEach = ABREAST > 1 ? kMostSplits / 64 : 1;
            AttnStat x[kEach];
            top[m] = -INFINITY;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int s = i * 64 + lane;
                x[i] = s < f.splits ? f.stat[2 * (s * all + at) + m] : AttnStat{-INFINITY, 0.0f};
                if (x[i].sum != 0.0f) top[m] = fmaxf(top[m], x[i].top);
            }
            for (int d = 32; d > 0; d >>= 1) top[m] = fmaxf(top[m], __shfl_xor(top[m], d));
            sum[m] = 0.0f;
            float weight[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                weight[i] = x[i].sum == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(x[i].top - top[m]);
                sum[m] += x[i].sum * weight[i];
            }
            for (int d = 32; d > 0; d >>= 1) sum[m] += __shfl_xor(sum[m], d);
            const float by = sum[m] == 0.0f ? 0.0f : (m ? -a.lambda[head] : 1.0f) / sum[m];
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (i * 64 + lane < f.splits) weights[r][m][i * 64 + lane] = weight[i] * by;
        }
        if (f.lse && lane < 2 && t < min(max(a.q_end[a.n_seqs - 1], 0), a.tokens_q)) {
            const float s = lane ? sum[1] : sum[0], m = lane ? top[1] : top[0];
            f.lse[(int64_t)(2 * head + lane) * a.tokens_q + t] = s == 0.0f ? -INFINITY : m + __builtin_amdgcn_logf(s);
        }
    }
    __syncthreads();
    const int in = threadIdx.x % D, sub = threadIdx.x / D % ABREAST, r = threadIdx.x / (D * ABREAST), m = in / (D / 2);
    const int64_t at = row0 + r;
    tile_f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (at < all) {
        const tile_f32x4* part = reinterpret_cast<const tile_f32x4*>(f.part) + at * D + in;
#pragma unroll 4
        for (int s = sub; s < f.splits; s += ABREAST) {
            const float w = weights[r][m][s];
            const tile_f32x4 x = part[s * all * D];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = w == 0.0f ? v[i] : fmaf(x[i], w, v[i]);
        }
    }
    __shared__ tile_f32x4 meet[256];
    meet[threadIdx.x] = v;
    __syncthreads();
    if (at >= all || sub != 0 || m != 0) return;
    v = tile_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < ABREAST; ++s) v += meet[threadIdx.x + s * D] + meet[threadIdx.x + s * D + D / 2];
    const int64_t of_head = (int64_t)a.tokens_q * group;
    const int head_k = (int)(at / of_head), row = (int)(at - head_k * of_head), t = (int)a.group(row), head = head_k * group + row - t * group;
    if (t >= min(max(a.q_end[a.n_seqs - 1], 0), a.tokens_q)) return;   // behind the last sequence: left as it was
    uint16_t* o = f.out + t * f.ldo + (int64_t)head * a.e;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (in * 4 + i < a.e) o[in * 4 + i] = (uint16_t)bf16_bits(v[i]);
}

template <int D, int WAVES, int KT, int SHARE>
hipError_t launch(AttnForward f, hipStream_t stream)
{
    f.columns = attn_columns(f.a.causal, f.a.n_seqs, f.a.kv_heads, f.slots, f.splits);
    const int blocks = attn_blocks(f.columns, f.a.n_seqs, f.a.kv_heads, f.slots, f.splits);
    if (f.a.whole)
        k_attn_forward<D, WAVES, KT, SHARE, true><<<blocks, 64 * WAVES, 0, stream>>>(f);
    else
        k_attn_forward<D, WAVES, KT, SHARE, false><<<blocks, 64 * WAVES, 0, stream>>>(f);
    if (f.splits > 1) {
        const int64_t all = (int64_t)f.a.tokens_q * f.a.heads;
        if (f.splits > kFewSplits)
            k_attn_join<D, 256 / D><<<(uint32_t)all, 256, 0, stream>>>(f);
        else
            k_attn_join<D, 1><<<(uint32_t)((all * D + 255) / 256), 256, 0, stream>>>(f);
    }
    return hipGetLastError();
}

// Rows of a workgroup, and over how many workgroups the keys are split.
struct Shape {
    int waves, slots, splits;   // one wave for each map where D is 128
};

Shape shape_of(int64_t tokens_q, int64_t tokens_k, int n_seqs, int heads, int kv_heads, int D)
{
    Shape o;
    const int64_t rows = tokens_q * (heads / kv_heads);
    const int unit = 2 / attn_maps_of_a_wave(D);   // waves of 32 rows
    // Lengths lie on the device, the rules go by their mean: 32 queries, one of 100000 keys and 31 of 1000, take 528 us, of 4094 keys
    // each 57 (16 heads of 64 on 4).
    // Large workgroups read the keys least often; small ones of 64 rows where those would leave compute units without work, down
    // to one wave (of each map) that has a sequence's up to 32 rows; and where these are too few, the keys split among several.
    const int64_t large = 32 * 8 / unit;
    const bool enough = rows / n_seqs >= large && rows / large * kv_heads >= 192;
    o.waves = enough ? 8 : (rows <= (int64_t)32 * n_seqs ? 1 : 2) * unit;
    const int64_t own = 32 * o.waves / unit;
    o.slots = (int)(rows / own) + n_seqs;
    // as many as the card has places for: a few more would make a second round of them
    const int64_t blocks = std::max<int64_t>((rows + own - 1) / own, n_seqs) * kv_heads;
    o.splits = enough ? 1 : (int)std::max<int64_t>(1, std::min({(own == 32 ? 1024 : 512) / blocks, tokens_k / n_seqs / 128, (int64_t)kMostSplits}));
    return o;
}

int64_t splits_bytes(const Shape& s, int64_t tokens_q, int heads, int D)
{
    return s.splits > 1 ? round_up((int64_t)s.splits * tokens_q * heads * (4 * D * 4 + 16), 256) : 0;
}

}  // namespace

int attn_width(int d, int e) { return d <= 32 && e <= 64 ? 32 : d <= 64 && e <= 128 ? 64 : 128; }

namespace {

struct PackJobs {
    AttnPack job[4];
};

__global__ __launch_bounds__(256) void k_attn_pack(PackJobs jobs)
{
    const AttnPack& j = jobs.job[blockIdx.y];
    const int per = j.up / 8, chunks = j.parts * per, at_once = max(1, 256 / chunks);
    const int sub = threadIdx.x / chunks, c0 = threadIdx.x - sub * chunks;
    if (sub >= at_once) return;
    for (int64_t r = (int64_t)blockIdx.x * at_once + sub; r < j.rows; r += (int64_t)gridDim.x * at_once)
        for (int c = c0; c < chunks; c += 256) {
            const int part = c / per, in = (c - part * per) * 8;
            float v[8];
            load8(j.from + r * j.ld + part * j.width + min(in, j.width), max(0, min(8, j.width - in)), v);
            store16(j.to + r * j.parts * j.up + c * 8, bf16_pack8(v));
        }
}

}  // namespace

hipError_t attn_pack(const AttnPack* jobs, int n, hipStream_t stream)
{
    if (n == 0) return hipSuccess;
    PackJobs all{};
    int64_t blocks = 1;
    for (int i = 0; i < n; ++i) {
        all.job[i] = jobs[i];
        const int at_once = std::max(1, 256 / (jobs[i].parts * jobs[i].up / 8));
        blocks = std::max(blocks, ((int64_t)jobs[i].rows + at_once - 1) / at_once);
    }
    k_attn_pack<<<dim3((uint32_t)std::min<int64_t>(blocks, 8192), n), 256, 0, stream>>>(all);
    return hipGetLastError();
}

hipError_t attn_lay_out(const AttnCall& c, Attn& a, const uint16_t*& dout, int64_t& lddout, char*& place, hipStream_t stream)
{
    const int D = attn_width(c.d, c.e), E = 2 * D;
    a.q = static_cast<const uint16_t*>(c.q), a.k = static_cast<const uint16_t*>(c.k), a.v = static_cast<const uint16_t*>(c.v);
    a.ldq = c.ldq, a.ldk = c.ldk, a.ldv = c.ldv;
    a.lambda = c.lambda, a.q_end = c.q_end, a.k_begin = c.k_begin, a.k_end = c.k_end;
    a.n_seqs = c.n_seqs, a.tokens_q = (int)c.tokens_q, a.tokens_k = (int)c.tokens_k;
    a.heads = c.heads, a.kv_heads = c.kv_heads, a.d = c.d, a.e = c.e;
    // Keys out of sight have scores of -infinity, which a factor of zero would make NaN.  The smallest number above zero, 2^-149,
    // leaves them what they are, and the largest other score, 2^128, is 2^-21 with it: every key in sight weighs alike.
    a.causal = c.causal, a.scale = c.scale, a.to_log2 = std::max(c.scale * kLog2e, std::numeric_limits<float>::denorm_min());
    dout = static_cast<const uint16_t*>(c.dout), lddout = c.lddout;
    // Other widths than the tiles' are filled up on the way to LDS if their chunks of 16 bytes can be read, else in the workspace
    // (forward and gradients of 2999 queries, 6 heads of 40 and 72 on 2: 104 against 118 us; 8 x 2048, 8 heads of 80 and 160: 1575
    // against 1675).
    const auto chunks = [](const void* p, int64_t ld, int64_t rows) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows < 2 || ld % 8 == 0); };
    a.whole = (c.d == D && c.e == E) || c.d % 8 || c.e % 8 || !chunks(c.q, c.ldq, c.tokens_q) || !chunks(c.k, c.ldk, c.tokens_k) ||
              !chunks(c.v, c.ldv, c.tokens_k) || (dout && !chunks(dout, lddout, c.tokens_q));
    if (!a.whole) return hipSuccess;
    AttnPack jobs[4];
    int n = 0;
    const auto lay = [&](const uint16_t*& p, int64_t& ld, int64_t rows, int parts, int width, int up) {
        if (width == up) return;
        uint16_t* to = reinterpret_cast<uint16_t*>(place);
        if (rows > 0) jobs[n++] = {p, to, ld, (int)rows, parts, width, up};
        p = to, ld = (int64_t)parts * up;
        place += round_up(rows * parts * up * 2, 256);
    };
    lay(a.q, a.ldq, c.tokens_q, 2 * c.heads, c.d, D);
    lay(a.k, a.ldk, c.tokens_k, 2 * c.kv_heads, c.d, D);
    lay(a.v, a.ldv, c.tokens_k, c.kv_heads, c.e, E);
    if (dout) lay(dout, lddout, c.tokens_q, c.heads, c.e, E);
    return attn_pack(jobs, n, stream);
}

int64_t attn_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int n_seqs, int heads, int kv_heads, int d, int e, int gradients)
{
    const int D = attn_width(d, e);
    int64_t bytes = 256;
    if (d != D) bytes += round_up(tokens_q * heads * 4 * D, 256) + round_up(tokens_k * kv_heads * 4 * D, 256);
    if (e != 2 * D) bytes += round_up(tokens_k * kv_heads * 4 * D, 256) + (gradients ? round_up(tokens_q * heads * 4 * D, 256) : 0);
    int64_t more = splits_bytes(shape_of(tokens_q, tokens_k, n_seqs, heads, kv_heads, D), tokens_q, heads, D);
    if (gradients) more = std::max(more, attn_gradients_bytes(tokens_q, tokens_k, n_seqs, heads, kv_heads, D));
    return bytes + more;
}

hipError_t launch_attn_forward(const AttnCall& c, hipStream_t stream)
{
    AttnForward f{Attn{.group = Divider(c.heads / c.kv_heads)}};
    const uint16_t* none;
    int64_t none_ld;
    char* place = c.workspace;
    const hipError_t e = attn_lay_out(c, f.a, none, none_ld, place, stream);
    if (e != hipSuccess) return e;
    const int D = attn_width(c.d, c.e);
    const Shape s = shape_of(c.tokens_q, c.tokens_k, c.n_seqs, c.heads, c.kv_heads, D);
    f.out = static_cast<uint16_t*>(c.out), f.ldo = c.ldo, f.lse = c.lse, f.slots = s.slots, f.splits = s.splits;
    f.stat = reinterpret_cast<AttnStat*>(place);
    f.part = reinterpret_cast<float*>(place + (int64_t)s.splits * c.tokens_q * c.heads * 16);
    if (D == 32) return s.waves == 8 ? launch<32, 8, 64, 1>(f, stream) : s.waves == 2 ? launch<32, 4, 64, 2>(f, stream) : launch<32, 1, 64, 1>(f, stream);
    if (D == 64) return s.waves == 8 ? launch<64, 8, 64, 1>(f, stream) : s.waves == 2 ? launch<64, 4, 64, 2>(f, stream) : launch<64, 1, 32, 1>(f, stream);
    return s.waves == 8 ? launch<128, 8, 64, 1>(f, stream) : s.waves == 4 ? launch<128, 4, 32, 1>(f, stream) : launch<128, 2, 32, 1>(f, stream);
}

}  // namespace agc
