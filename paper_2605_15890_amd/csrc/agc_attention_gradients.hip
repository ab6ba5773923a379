// Partial gradients of differential attention.  With the rows' binary logarithms of the sums, which the forward pass leaves,
// P_m = 2^(S_m log2(e) - lse_m) is formed again, and
//   dP = dout v^T,  D_m = sum over keys of P_m dP,  dS_1 = P_1 (dP - D_1),  dS_2 = -lambda P_2 (dP - D_2)
//   dq_m = scale dS_m k_m,  dk_m = scale dS_m^T q_m,  dv = (P_1 - lambda P_2)^T dout,  G[p,h] = - sum over p's queries of D_2
// dP is one product for both maps, dv one of their difference.
//
// Two passes, one whose workgroups own rows (D, dq) and one whose workgroups own keys (dk, dv), and no sums in memory whose
// order could change.  The first goes over its keys twice: D comes from the same P and dP as dS, which makes the rows of dS
// add up to zero to the last bits of binary32 (from dout and the rounded out they would miss it by 2^-8, and a query that
// sees one key would get a gradient where there is none), and makes D_2, whose sums are rows of G, a binary32 sum of
// binary32 terms.
// dS and the difference of the maps enter their products as two bfloat16 parts, 2^-16 of a term at most: one part would add as
// much error to a result as its own rounding does, and more where keys have a part in common, which dS, whose rows add up to
// zero, only cancels as far as it is exact (2.5e-3 in the 2-norm where the rounding alone is 1.66e-3).  Sums are binary32.
//
// That makes 28 d + 10 e operations a pair of a query and a key, where a single pass of one part would do with 12 d + 4 e.
// 8 x 2048 tokens, 16 heads of 64, causal: the rows' pass 457 to 504 us, 0.82 to 0.9 PFLOP/s of products, the keys' pass 491 to
// 555, 0.74 to 0.84 (a library product of 8192^3: 1.28).  Counters have the matrix units busy for 0.39 to 0.45 of the time and
// the vector units for 0.49 to 0.63: of the two waves a SIMD, which is what the registers of dq or of dk and dv leave room
// for, neither hides the other's waits, and the clock falls to 2 GHz.
#include <algorithm>

#include "agc_attention.h"

namespace agc {

namespace {

struct AttnGradients {
    Attn a;
    const uint16_t* dout;
    int64_t lddout;
    const float* lse;
    float* facts;          // lse_m and D_m of every (head, map, token), lse as the keys' pass takes it
    int64_t of_facts;      // values of each
    uint16_t *dq, *dk, *dv;
    int64_t lddq, lddk, lddv;
    int slots, splits, columns, blocks;
    // of splits: sums of D of every (split, head, map, token), and of dq or of dk and dv of every (split, row)
    float *part_mean, *part, *part_v, *part_k;
};

// A workgroup has all keys of its rows, or the keys are split and the sums over them joined: D first, which dq needs.
enum AttnKeys { kAll, kSplitMeans, kSplitRest };

// ------------------------------------------------------------------ D and dq: a workgroup's rows, all keys in sight, twice
// SHARE waves have the same rows, and every SHAREth 32 keys of them each, as in the forward pass (37 instead of 50 us there).
template <int D, int WAVES, int KT, AttnKeys KEYS, int SHARE, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES, D == 128 ? 1 : 2) void k_attn_dq(AttnGradients f)
{
    using Tile = AttnTile<D>;
    constexpr int E = 2 * D, kSteps = D / 16, kBlocks = D / 32, kRows = 32 * WAVES / SHARE;
    constexpr int kTile = KT * Tile::kRow;
    __shared__ __attribute__((aligned(1024))) char lds[2][2][kTile];   // buffer; keys, values
    const Attn& a = f.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnPlace place = attn_place(a, blockIdx.x, f.slots, f.splits, f.columns);
    const int slot = place.slot, head_k = place.head_k, split = place.split;
    if (slot < 0) return;
    const uint32_t group = a.group.d;

    const int s = attn_find(a.q_end, a.n_seqs, a.tokens_q, group, kRows, slot);
    const AttnSeq seq = attn_sequence(a, s);
    const int first = attn_first_slot(a.q_end, s, a.tokens_q, group, kRows);
    const int rows = seq.lq * (int)group, tiles = (rows + kRows - 1) / (kRows);
    const int tile = tiles - 1 - (slot - first);
    if (tile < 0 || tile >= tiles) return;

    const int rows_of = wave / SHARE, turn = wave % SHARE;
    const int row_ = tile * kRows + rows_of * 32 + (lane & 31);
    const int row = min(row_, rows - 1), t = (int)a.group(row), g = row - t * (int)group, head = head_k * (int)group + g;
    const int seen = attn_seen(a, seq, t);
    const int last_row = min(tile * kRows + kRows, rows) - 1;
    const int keys = attn_seen(a, seq, (int)a.group(last_row));   // of the tile
    const int run = (keys + f.splits * KT - 1) / (f.splits * KT) * KT;
    const int begin = min(split * run, keys), end = min(begin + run, keys);
    const int seen_least = min(__builtin_amdgcn_readfirstlane(seen), end), seen_most = min(__builtin_amdgcn_readlane(seen, 31), end);

    const AttnHead<D, 2, WHOLE> maps{a.d};
    const AttnHead<D, 1, WHOLE> ofv{a.e};
    tile_bf16x8 q[2][kSteps], go[2 * kSteps];
    {
        const uint16_t* p = a.q + (int64_t)(seq.q0 + t) * a.ldq + (int64_t)head * maps.size();
        const uint16_t* o = f.dout + (int64_t)(seq.q0 + t) * f.lddout + (int64_t)head * ofv.size();
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) q[m][i] = maps.values(p, m, (lane >> 5) * 8 + i * 16);
#pragma unroll
        for (int i = 0; i < 2 * kSteps; ++i) go[i] = ofv.values(o, 0, (lane >> 5) * 8 + i * 16);
    }
    float lse[2], mean[2] = {0.0f, 0.0f};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        lse[m] = f.lse[(int64_t)(2 * head + m) * a.tokens_q + seq.q0 + t];
        lse[m] = seen <= 1 ? 0.0f : lse[m];   // without keys it is -infinity; a single key's map is 2^0
    }

    const char* const keys_at = reinterpret_cast<const char*>(a.k + (int64_t)seq.k0 * a.ldk + head_k * maps.size());
    const char* const values_at = reinterpret_cast<const char*>(a.v + (int64_t)seq.k0 * a.ldv + head_k * ofv.size());
    const auto fetch = [&](AttnLds to, int j0) {
        Tile::template load<KT, WAVES>(to, wave, lane, maps, keys_at + (int64_t)j0 * a.ldk * 2, (uint32_t)a.ldk * 2, seq.lk - j0);
        Tile::template load<KT, WAVES>(to + kTile, wave, lane, ofv, values_at + (int64_t)j0 * a.ldv * 2, (uint32_t)a.ldv * 2, seq.lk - j0);
    };

    const AttnReads<D> reads(lane);
    // All keys in sight, 32 at a time: both maps and dP.
    const auto over_keys = [&](const auto& use) {
        const auto step = [&](AttnLds from_lds, AttnLds to_lds, int j0) {
            if (j0 + KT < end) fetch(to_lds, j0 + KT);
            uint32_t k_tile = turn * 32 * Tile::kRow;
#pragma unroll 1
            for (int j = j0 + turn * 32; j < min(j0 + KT, seen_most); j += 32 * SHARE, k_tile += 32 * SHARE * Tile::kRow) {
                const uint32_t v_tile = k_tile + kTile;
                // two products of dP, one of each map, in turn
                attn_f32x16 dp{}, score[2] = {};
                const auto read = [&](int n) {
                    return n % 4 < 2 ? reads.straight(from_lds, v_tile, n / 4 * 2 + n % 4) : reads.straight(from_lds, k_tile, n % 4 % 2 * kSteps + n / 4);
                };
                auto stream = attn_stream<4 * kSteps, 4>(read);
                stream.start();
                stream.run([&](int n, const tile_bf16x8& x) {
                    if (n % 4 < 2)
                        dp = attn_mfma(x, go[n / 4 * 2 + n % 4], dp);
                    else
                        score[n % 2] = attn_mfma(x, q[n % 2][n / 4], score[n % 2]);
                });
                if (j + 32 > seen_least) {
                    const int left = min(seen, end) - j;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool in = attn_row_swapped(r, lane) < left;
                        dp[r] = in ? dp[r] : 0.0f;   // nothing but zero times a map's zero is zero
#pragma unroll
                        for (int m = 0; m < 2; ++m) score[m][r] = in ? (seen == 1 ? 0.0f : score[m][r]) : -INFINITY;
                    }
                }
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int r = 0; r < 16; ++r) score[m][r] = __builtin_amdgcn_exp2f(fmaf(score[m][r], a.to_log2, -lse[m]));
                use(from_lds, k_tile, score, dp);
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
    };

    const int64_t fact = (int64_t)2 * head * a.tokens_q + seq.q0 + t;
    if constexpr (KEYS != kSplitRest) {
        over_keys([&](AttnLds, uint32_t, const attn_f32x16* map, const attn_f32x16& dp) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) mean[m] = fmaf(map[m][r], dp[r], mean[m]);
        });
#pragma unroll
        for (int m = 0; m < 2; ++m) mean[m] += attn_other_half(mean[m]);
        if constexpr (SHARE == 2) {
            __shared__ float means[WAVES][2][64];
#pragma unroll
            for (int m = 0; m < 2; ++m) means[wave][m][lane] = mean[m];
            __syncthreads();
#pragma unroll
            for (int m = 0; m < 2; ++m) mean[m] += means[wave ^ 1][m][lane];
        }
        if constexpr (KEYS == kSplitMeans) {
            if (row_ < rows && lane < 32 && turn == 0) {
#pragma unroll
                for (int m = 0; m < 2; ++m) f.part_mean[split * f.of_facts + fact + m * (int64_t)a.tokens_q] = mean[m];
            }
            return;
        }
        __syncthreads();   // nobody reads tiles any more
    } else {
#pragma unroll 8
        for (int n = 0; n < f.splits; ++n) {
#pragma unroll
            for (int m = 0; m < 2; ++m) mean[m] += f.part_mean[n * f.of_facts + fact + m * (int64_t)a.tokens_q];
        }
    }

    attn_f32x16 acc[2][kBlocks];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) acc[m][b] = attn_f32x16{};
    over_keys([&](AttnLds from_lds, uint32_t k_tile, const attn_f32x16* map, const attn_f32x16& dp) {
        const auto read = [&](int n) { return reads.turned(from_lds, k_tile, n / (2 * kBlocks) * 16, n % (2 * kBlocks)); };
        auto stream = attn_stream<4 * kBlocks, 2>(read);
        stream.start();
        const auto ds = [&](int i, int m) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = map[m][i * 8 + e] * (dp[i * 8 + e] - mean[m]);
            return AttnTwo(v);
        };
        const AttnTwo d[2][2] = {{ds(0, 0), ds(0, 1)}, {ds(1, 0), ds(1, 1)}};
        stream.run([&](int n, const tile_bf16x8& k) {
            const int i = n / (2 * kBlocks), m = n / kBlocks % 2, b = n % kBlocks;
            acc[m][b] = attn_mfma(k, d[i][m], acc[m][b]);
        });
    });
    if constexpr (SHARE == 2) {
        // the second wave hands its sums to the first, where the tiles were
        static_assert(WAVES / 2 * 2 * kBlocks * 16 * 64 * 4 <= (int)sizeof(lds), "they fit");
        float* box = reinterpret_cast<float*>(lds) + rows_of * (2 * kBlocks * 16 * 64) + lane;
        __syncthreads();
        if (turn == 1) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) box[((m * kBlocks + b) * 16 + r) * 64] = acc[m][b][r];
        }
        __syncthreads();
        if (turn == 1) return;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][b][r] += box[((m * kBlocks + b) * 16 + r) * 64];
    }
    if (row_ >= rows) return;
    if (lane < 32 && split == 0) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            f.facts[fact + m * (int64_t)a.tokens_q] = lse[m];
            f.facts[f.of_facts + fact + m * (int64_t)a.tokens_q] = mean[m];
        }
    }
    const float factor[2] = {a.scale, -a.scale * a.lambda[head]};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        if constexpr (KEYS == kAll) {
            uint16_t* o = f.dq + (int64_t)(seq.q0 + t) * f.lddq + (int64_t)(2 * head + m) * a.d;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) attn_store(o, b * 32, a.d, lane, acc[m][b], factor[m]);
        } else {
            float* o = f.part + (((int64_t)split * a.tokens_q + seq.q0 + t) * a.heads + head) * E + m * D;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) attn_store_part(o + b * 32, lane, acc[m][b], factor[m]);
        }
    }
}

// ------------------------------------------------------------------ rows of G
struct AttnParts {
    int end[kMostParts];
    int k;
    float* G;
    int64_t ldg;
};

// A workgroup adds up one partition's D_2 of one head, in binary64 and a fixed order.
template <int THREADS>
__device__ __forceinline__ void attn_lambda(const AttnParts& parts, const Attn& a, const float* means, int at, double* meet)
{
    const int h = at % a.heads, p = at / a.heads, covered = min(max(a.q_end[a.n_seqs - 1], 0), a.tokens_q);
    const int begin = p ? parts.end[p - 1] : 0, end = min(parts.end[p], covered);
    const float* from = means + (int64_t)(2 * h + 1) * a.tokens_q;
    double sum = 0;
#pragma unroll 4
    for (int t = begin + (int)threadIdx.x; t < end; t += THREADS) sum += from[t];
    meet[threadIdx.x] = sum;
    for (int half = THREADS / 2; half > 0; half >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < half) meet[threadIdx.x] += meet[threadIdx.x + half];
    }
    if (threadIdx.x == 0) parts.G[p * parts.ldg + h] = (float)-meet[0];
}

// ------------------------------------------------------------------ dk, dv: a workgroup's keys, all rows that see them
// Rows are the queries of one head after the other here.  They bring along lse and D of both maps.
//
// Wide heads are worked on by two workgroups, since dk and dv of 32 keys would take a wave's registers twice over: each forms
// both maps and dP, and has dk of one map (its own) and half of dv.  A third more products than one workgroup would need, in a
// half of the time that it takes when registers leave for memory (8 x 2048 tokens, 8 heads of 128: 922 instead of 2544 us).
constexpr int attn_halves(int D) { return D == 128 ? 2 : 1; }
// A wave a SIMD, with all of its registers.
constexpr bool attn_room(int D, int waves) { return D == 128 || waves == 2; }

template <int D, int WAVES, int RT, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES, attn_room(D, WAVES) ? 1 : 2) void k_attn_dkv(AttnGradients f, AttnParts parts)
{
    using Tile = AttnTile<D>;
    constexpr int E = 2 * D, kSteps = D / 16, kBlocks = D / 32;
    // of a buffer: queries, dout, facts
    constexpr int kTile = RT * Tile::kRow, kBuffer = 2 * kTile + 4 * RT * 4;
    __shared__ __attribute__((aligned(1024))) char lds[2 * kBuffer + 32 * WAVES * Tile::kRow];   // two buffers, the keys' values
    const AttnLds all = (AttnLds)&lds[0], values = all + 2 * kBuffer;
    const Attn& a = f.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr bool kRoom = attn_room(D, WAVES);
    constexpr int kHalves = attn_halves(D), kValues = 2 * kBlocks / kHalves;
    const int tiles = f.blocks * kHalves;
    if ((int)blockIdx.x >= tiles) {   // behind the tiles: the rows of G
        attn_lambda<64 * WAVES>(parts, a, f.facts + f.of_facts, (int)blockIdx.x - tiles, reinterpret_cast<double*>(lds));
        return;
    }
    // both halves on one XCD
    const int half = kHalves == 1 ? 0 : ((int)blockIdx.x >> 3) % kHalves;
    const int id = kHalves == 1 ? (int)blockIdx.x : ((int)blockIdx.x >> 3) / kHalves * 8 + ((int)blockIdx.x & 7);
    const AttnPlace place = attn_place(a, id, f.slots, f.splits, f.columns);
    const int slot = place.slot, head_k = place.head_k, split = place.split;
    if (slot < 0) return;
    const uint32_t group = a.group.d;

    const int s = attn_find(a.k_end, a.n_seqs, a.tokens_k, 1, 32 * WAVES, slot);
    const AttnSeq seq = attn_sequence(a, s);
    const int tile = slot - attn_first_slot(a.k_end, s, a.tokens_k, 1, 32 * WAVES);
    if (tile * 32 * WAVES >= seq.lk) return;

    const int key0 = tile * 32 * WAVES + wave * 32, key_ = key0 + attn_swapped(lane & 31), key = min(key_, seq.lk - 1);
    // Tiles of the queries that see this tile's first key, head after head of the group; a split has a run of them.
    const int seeing = (a.causal ? min(max(tile * 32 * WAVES + seq.lq - seq.lk, 0), seq.lq) : 0) / RT * RT;
    const int of_head = (seq.lq - seeing + RT - 1) / RT, run = (of_head * (int)group + f.splits - 1) / f.splits;
    const int begin = min(split * run, of_head * (int)group), end = min(begin + run, of_head * (int)group);

    const AttnHead<D, 2, WHOLE> maps{a.d};
    const AttnHead<D, 1, WHOLE> ofv{a.e};
    // the keys stay in registers, the values in LDS, as far as the waves' registers go
    tile_bf16x8 k[2][kSteps];   // of the own map, of the other one
    {
        const uint16_t* p = a.k + (int64_t)(seq.k0 + key) * a.ldk + head_k * maps.size();
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) k[m][i] = maps.values(p, m ^ half, (lane >> 5) * 8 + i * 16);
        const char* const values_at = reinterpret_cast<const char*>(a.v + (int64_t)seq.k0 * a.ldv + head_k * ofv.size());
        Tile::template load<32 * WAVES, WAVES>(values, wave, lane, ofv, values_at + (int64_t)(tile * 32 * WAVES) * a.ldv * 2, (uint32_t)a.ldv * 2,
                                               seq.lk - tile * 32 * WAVES);
    }
    // a tile's head of the group and first query, which grow without a division
    struct Rows {
        int head, t0;
    };
    const auto after = [&](Rows r) {
        r.t0 += RT;
        return r.t0 < seq.lq ? r : Rows{r.head + 1, seeing};
    };
    const auto fetch = [&](AttnLds to, Rows r) {
        const int head = r.head, t0 = r.t0, rows = seq.lq - t0;
        Tile::template load<RT, WAVES>(to, wave, lane, maps, reinterpret_cast<const char*>(a.q + (int64_t)(seq.q0 + t0) * a.ldq + (int64_t)head * maps.size()),
                                       (uint32_t)a.ldq * 2, rows);
        Tile::template load<RT, WAVES>(to + kTile, wave, lane, ofv, reinterpret_cast<const char*>(f.dout + (int64_t)(seq.q0 + t0) * f.lddout + (int64_t)head * ofv.size()),
                                       (uint32_t)f.lddout * 2, rows);
        // a wave a fact, a lane a row
        for (int w = wave; w < 4; w += WAVES) {
            const float* at = f.facts + (w >> 1) * f.of_facts + (int64_t)(2 * head + (w & 1)) * a.tokens_q + seq.q0 + t0;
            if (lane < RT) attn_load4(at + min(lane, rows - 1), to + 2 * kTile + w * RT * 4);
        }
    };
    attn_f32x16 acc_k[2 / kHalves][kBlocks], acc_v[kValues];
#pragma unroll
    for (int m = 0; m < 2 / kHalves; ++m)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) acc_k[m][b] = acc_v[m * kBlocks + b] = attn_f32x16{};

    const AttnReads<D> reads(lane);
    const auto step = [&](AttnLds from_lds, AttnLds to_lds, AttnLds v_lds, Rows rows, bool more) {
        if (more) fetch(to_lds, after(rows));
        const int t0 = rows.t0;
        const float lambda = a.lambda[rows.head];
        uint32_t q_tile = 0;
#pragma unroll 1
        for (int t_first = t0; t_first < min(t0 + RT, seq.lq); t_first += 32, q_tile += 32 * Tile::kRow) {
            // halves of wide rows lie 256 bytes apart, whole turns of the permutation
            static_assert(kHalves == 1 || D == 128, "2 D bytes are 256");
            const uint32_t o_tile = q_tile + kTile, q_own = q_tile + half * 256;
            const int t_last = t_first + 31, sub = t_first - t0;
            // keys in sight grow with the query
            if (attn_seen(a, seq, min(t_last, seq.lq - 1)) <= key0) continue;
            const bool masked = attn_seen(a, seq, t_first) < max(key0 + 32, 2) || t_last >= seq.lq;
            // eight rows' facts: rows 16 i + 8 (lane / 32) + 0 .. 7
            typedef __attribute__((address_space(3))) const tile_f32x4* Facts;
            const AttnLds fact = from_lds + 2 * kTile + (sub + 8 * (lane >> 5)) * 4;
            const auto fact8 = [&](int which, int i, float o[8]) {
                const Facts p = (Facts)(fact + (which * RT + i * 16) * 4);
                const tile_f32x4 lo = p[0], hi = p[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = lo[e], o[4 + e] = hi[e];
            };
            attn_f32x16 dp{}, score[2] = {};
            const auto read_q = [&](int m, int i) {
                return kHalves == 2 ? reads.straight(from_lds, q_tile + (m ^ half) * 256, i) : reads.straight(from_lds, q_tile, m * kSteps + i);
            };
            if constexpr (kRoom) {
                // a product of dP and one of a map in turn (8 x 2048 tokens, 8 heads of 128: 922 instead of 980 us)
                const auto read = [&](int n) {
                    const int i = n / 3;
                    return n % 3 == 0 ? reads.straight(from_lds, o_tile, i) : n % 3 == 1 ? reads.straight(v_lds, 0, i) : read_q(i & 1, i / 2);
                };
                auto stream = attn_stream<6 * kSteps, 6>(read);
                stream.start();
                tile_bf16x8 o;
                stream.run([&](int n, const tile_bf16x8& x) {
                    const int i = n / 3;
                    if (n % 3 == 0)
                        o = x;
                    else if (n % 3 == 1)
                        dp = attn_mfma(o, x, dp);
                    else
                        score[i & 1] = attn_mfma(x, k[i & 1][i / 2], score[i & 1]);
                });
            } else {
#pragma unroll
                for (int i = 0; i < 2 * kSteps; ++i) dp = attn_mfma(reads.straight(from_lds, o_tile, i), reads.straight(v_lds, 0, i), dp);
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
#pragma unroll
                    for (int m = 0; m < 2; ++m) score[m] = attn_mfma(read_q(m, i), k[m][i], score[m]);
            }
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = t_first + attn_row_swapped(r, lane), seen = t < seq.lq ? attn_seen(a, seq, t) : 0;
                    const bool in = key_ < seen;
                    dp[r] = in ? dp[r] : 0.0f;
#pragma unroll
                    for (int m = 0; m < 2; ++m) score[m][r] = in ? (seen == 1 ? 0.0f : score[m][r]) : -INFINITY;
                }
            }
            // of 16 rows: dS of the own map, of the other one, the difference of the maps
            struct Half {
                AttnTwo own, mixed, second;
            };
            const auto of_half = [&](int i) {
                float p[8], ds[8], lse[8], mean[8], other[8];
                fact8(half, i, lse);
                fact8(2 + half, i, mean);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(fmaf(score[0][i * 8 + e], a.to_log2, -lse[e]));
                    if (half) p[e] *= lambda;
                    ds[e] = p[e] * (dp[i * 8 + e] - mean[e]);
                }
                const AttnTwo own(ds);
                fact8(1 - half, i, lse);
                if constexpr (kHalves == 1) fact8(3, i, mean);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    other[e] = __builtin_amdgcn_exp2f(fmaf(score[1][i * 8 + e], a.to_log2, -lse[e]));
                    if (!half) other[e] *= lambda;
                    if constexpr (kHalves == 1) ds[e] = other[e] * (mean[e] - dp[i * 8 + e]);
                    p[e] -= other[e];
                }
                return Half{own, AttnTwo(p), AttnTwo(ds)};
            };
            constexpr int kOfHalf = kValues + 2 / kHalves * kBlocks;
            const auto read = [&](int n) {
                const int i = n / kOfHalf, b = n % kOfHalf;
                return b < kValues ? reads.turned(from_lds, o_tile + half * 256, i * 16, b) : reads.turned(from_lds, q_own, i * 16, b - kValues);
            };
            // with four reads ahead, or started before the halves, registers leave for memory (581 and 610 us instead of 555)
            auto stream = attn_stream<2 * kOfHalf, 2>(read);
            const Half of[2] = {of_half(0), of_half(1)};
            stream.start();
            stream.run([&](int n, const tile_bf16x8& x) {
                const int b = n % kOfHalf;
                const Half& h = of[n / kOfHalf];
                if (b < kValues)
                    acc_v[b] = attn_mfma(x, h.mixed, acc_v[b]);
                else if (b < kValues + kBlocks)
                    acc_k[0][b - kValues] = attn_mfma(x, h.own, acc_k[0][b - kValues]);
                else
                    acc_k[kHalves == 1][b - kValues - kBlocks] = attn_mfma(x, h.second, acc_k[kHalves == 1][b - kValues - kBlocks]);
            });
        }
    };
    int buffer = 0;
    if (begin < end) {
        const int g = begin / of_head;
        Rows rows = {head_k * (int)group + g, seeing + (begin - g * of_head) * RT};
        fetch(all, rows);
#pragma unroll 1
        for (int n = begin; n < end; ++n, buffer ^= 1, rows = after(rows)) {
            attn_wait_loads();
            __syncthreads();
            step(all + buffer * kBuffer, all + (buffer ^ 1) * kBuffer, values + wave * 32 * Tile::kRow, rows, n + 1 < end);
        }
    }
    if (key_ >= seq.lk) return;
    const float sign = half ? -1.0f : 1.0f, factor = sign * a.scale;
    const int value0 = half * (E / kHalves);
    if (f.splits > 1) {
        const int64_t at = (((int64_t)split * a.tokens_k + seq.k0 + key) * a.kv_heads + head_k) * E;
#pragma unroll
        for (int b = 0; b < kValues; ++b) attn_store_part(f.part_v + at + value0 + b * 32, lane, acc_v[b], sign);
#pragma unroll
        for (int m = 0; m < 2 / kHalves; ++m)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) attn_store_part(f.part + at + (m + half) * D + b * 32, lane, acc_k[m][b], factor);
        return;
    }
    uint16_t* o = f.dv + (int64_t)(seq.k0 + key) * f.lddv + (int64_t)head_k * a.e;
#pragma unroll
    for (int b = 0; b < kValues; ++b) attn_store(o, value0 + b * 32, a.e, lane, acc_v[b], sign);
#pragma unroll
    for (int m = 0; m < 2 / kHalves; ++m) {
        o = f.dk + (int64_t)(seq.k0 + key) * f.lddk + (int64_t)(2 * head_k + m + half) * a.d;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) attn_store(o, b * 32, a.d, lane, acc_k[m][b], factor);
    }
}

// ------------------------------------------------------------------ joining splits
struct AttnSum {
    const float* part;    // (split, row, run of `up` values)
    uint16_t* to;         // (row, run of `width` values)
    int64_t ld;
    int rows, runs, width, up, splits;
    const int32_t* last;  // rows behind it are left as they were
};

struct AttnSums {
    AttnSum job[3];
};

__global__ __launch_bounds__(256) void k_attn_sum(AttnSums jobs)
{
    const AttnSum& j = jobs.job[blockIdx.y];
    const int per = j.runs * (j.up / 4);
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(n / per), in = (int)(n - (int64_t)row * per), run = in / (j.up / 4), c = (in - run * (j.up / 4)) * 4;
    if (row >= min(max(*j.last, 0), j.rows)) return;
    tile_f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int s = 0; s < j.splits; ++s) sum += reinterpret_cast<const tile_f32x4*>(j.part)[s * (int64_t)j.rows * per + n];
    uint16_t* to = j.to + row * j.ld + run * j.width + c;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < j.width) to[e] = (uint16_t)bf16_bits(sum[e]);
}

// Workgroups of both passes: their waves, tiles and splits.
struct Shape {
    int waves_q, slots_q, splits_q, waves_k, slots_k, splits_k;
};

constexpr int kFewWaves = 2;
// Of large ones.  Two workgroups of four waves a compute unit serve the rows' pass better than one of eight, whose first rows
// wait for its last ones under the causal mask (506 against 534 us at 8 x 2048 tokens of 16 heads); the keys' pass has LDS for one.
constexpr int kRowWaves = 4;
constexpr int key_waves(int D) { return D == 128 ? 4 : 8; }

Shape shape_of(int64_t tokens_q, int64_t tokens_k, int n_seqs, int heads, int kv_heads, int D, bool causal)
{
    const int64_t rows = tokens_q * (heads / kv_heads);
    // Large workgroups read the other side least often; where they would leave compute units without work, small ones, and
    // where those are too few, the other side split among several.
    const auto side = [&](int64_t own, int64_t other, int most, int& waves, int& slots, int& splits) {
        const int64_t large = 32 * most;
        const bool enough = own / n_seqs >= large && own / large * kv_heads >= 192;
        waves = enough ? most : kFewWaves;
        slots = (int)(own / (32 * waves)) + n_seqs;
        const int64_t blocks = std::max<int64_t>((own + 32 * waves - 1) / (32 * waves), n_seqs) * kv_heads;
        splits = enough ? 1 : (int)std::max<int64_t>(1, std::min({512 / blocks, other / n_seqs / 128, (int64_t)64}));
    };
    Shape o;
    side(rows, tokens_k, kRowWaves, o.waves_q, o.slots_q, o.splits_q);
    side(tokens_k, rows, key_waves(D), o.waves_k, o.slots_k, o.splits_k);
    // A large workgroup with a sequence's first keys has twice the mean to do under the causal mask: where there is about one a
    // compute unit, two halves each.  Both passes with the join, us in halves | whole: 8 x 2048 tokens, 4 heads that 16 share 1033 |
    // 1093, 2 x 8192, 4 heads 985 | 1209;  4 x 2048, 8 heads 333 | 321, 5 x 2048 386 | 366, 4 heads of 128 477 | 426, of 32 (8
    // of them) 238 | 239: what long sequences and shared heads gain is more than what short ones lose.
    if (causal && o.waves_k > kFewWaves && tokens_k / (32 * o.waves_k) * kv_heads < 400) o.splits_k = 2;
    return o;
}

template <int D, int WAVES, int KT, int SHARE, bool WHOLE>
void launch_dq(const AttnGradients& f, const Shape& s, hipStream_t stream)
{
    const int blocks = attn_blocks(f.columns, f.a.n_seqs, f.a.kv_heads, f.slots, f.splits);
    if (s.splits_q == 1) {
        k_attn_dq<D, WAVES, KT, kAll, SHARE, WHOLE><<<blocks, 64 * WAVES, 0, stream>>>(f);
        return;
    }
    if constexpr (SHARE > 1) {
        k_attn_dq<D, WAVES, KT, kSplitMeans, SHARE, WHOLE><<<blocks, 64 * WAVES, 0, stream>>>(f);
        k_attn_dq<D, WAVES, KT, kSplitRest, SHARE, WHOLE><<<blocks, 64 * WAVES, 0, stream>>>(f);
    }
}

template <int D, int WAVES, int RT, bool WHOLE>
void launch_dkv(const AttnGradients& f, const AttnParts& parts, const Shape& s, hipStream_t stream)
{
    const int blocks = f.blocks * attn_halves(D) + f.a.heads * parts.k;
    k_attn_dkv<D, WAVES, RT, WHOLE><<<blocks, 64 * WAVES, 0, stream>>>(f, parts);
}

void launch_sums(const AttnSum* job, int n, hipStream_t stream)
{
    if (n == 0) return;
    AttnSums all{};
    int64_t most = 0;
    for (int i = 0; i < n; ++i) {
        all.job[i] = job[i];
        most = std::max(most, (int64_t)job[i].rows * job[i].runs * (job[i].up / 4));
    }
    k_attn_sum<<<dim3((uint32_t)((most + 255) / 256), n), 256, 0, stream>>>(all);
}

template <int D, int KT, int RT, bool WHOLE>
hipError_t launch(AttnGradients f, const AttnParts& parts, const Shape& s, hipStream_t stream)
{
    const Attn& a = f.a;
    AttnSum sums[3];
    int n = 0;
    if (a.tokens_q > 0) {
        f.slots = s.slots_q, f.splits = s.splits_q, f.columns = attn_columns(a.causal, a.n_seqs, a.kv_heads, f.slots, f.splits);
        if (s.waves_q == kFewWaves)
            launch_dq<D, 2 * kFewWaves, 64, 2, WHOLE>(f, s, stream);
        else
            launch_dq<D, kRowWaves, KT, 1, WHOLE>(f, s, stream);
        if (s.splits_q > 1) sums[n++] = {f.part, f.dq, f.lddq, a.tokens_q, 2 * a.heads, a.d, D, s.splits_q, a.q_end + a.n_seqs - 1};
    }
    f.slots = s.slots_k, f.splits = s.splits_k, f.columns = attn_columns(a.causal, a.n_seqs, a.kv_heads, f.slots, f.splits), f.part = f.part_k;
    f.blocks = (int)round_up(attn_blocks(f.columns, a.n_seqs, a.kv_heads, f.slots, f.splits), 8);   // the halves of eight workgroups follow each other
    f.part_v = f.part + (int64_t)s.splits_k * a.tokens_k * a.kv_heads * 2 * D;
    if (s.waves_k == kFewWaves)
        launch_dkv<D, kFewWaves, 32, WHOLE>(f, parts, s, stream);
    else
        launch_dkv<D, key_waves(D), RT, WHOLE>(f, parts, s, stream);
    if (s.splits_k > 1 && a.tokens_k > 0) {
        sums[n++] = {f.part, f.dk, f.lddk, a.tokens_k, 2 * a.kv_heads, a.d, D, s.splits_k, a.k_end + a.n_seqs - 1};
        sums[n++] = {f.part_v, f.dv, f.lddv, a.tokens_k, a.kv_heads, a.e, 2 * D, s.splits_k, a.k_end + a.n_seqs - 1};
    }
    launch_sums(sums, n, stream);
    return hipGetLastError();
}

}  // namespace

// lse and D of every row, and what splits leave: of D and dq, then of dk and dv
int64_t attn_gradients_bytes(int64_t tokens_q, int64_t tokens_k, int n_seqs, int heads, int kv_heads, int D)
{
    const Shape s = shape_of(tokens_q, tokens_k, n_seqs, heads, kv_heads, D, true);   // which splits most
    const int64_t q = s.splits_q > 1 ? s.splits_q * tokens_q * heads * (2 * D + 2) * 4 : 0;
    const int64_t k = s.splits_k > 1 ? s.splits_k * tokens_k * kv_heads * 4 * D * 4 : 0;
    return round_up(tokens_q * heads * 16, 256) + round_up(q, 256) + round_up(k, 256);
}

hipError_t launch_attn_gradients(const AttnCall& c, hipStream_t stream)
{
    AttnGradients f{Attn{.group = Divider(c.heads / c.kv_heads)}};
    char* place = c.workspace;
    hipError_t e = attn_lay_out(c, f.a, f.dout, f.lddout, place, stream);
    if (e != hipSuccess) return e;
    const int D = attn_width(c.d, c.e);
    const Shape s = shape_of(c.tokens_q, c.tokens_k, c.n_seqs, c.heads, c.kv_heads, D, c.causal != 0);
    f.lse = c.lse, f.facts = reinterpret_cast<float*>(place), f.of_facts = (int64_t)2 * c.heads * c.tokens_q;
    f.part = reinterpret_cast<float*>(place + round_up(c.tokens_q * c.heads * 16, 256));
    const int64_t of_part = (int64_t)s.splits_q * c.tokens_q * c.heads;
    f.part_mean = f.part + of_part * 2 * D;
    f.part_k = s.splits_q > 1 ? f.part + round_up(of_part * (2 * D + 2) * 4, 256) / 4 : f.part;
    f.dq = static_cast<uint16_t*>(c.dq), f.dk = static_cast<uint16_t*>(c.dk), f.dv = static_cast<uint16_t*>(c.dv);
    f.lddq = c.lddq, f.lddk = c.lddk, f.lddv = c.lddv;
    AttnParts parts;
    for (int p = 0; p < c.k_parts; ++p) parts.end[p] = (int)c.part_end[p];
    parts.k = c.k_parts, parts.G = c.G, parts.ldg = c.ldg;
    const auto of_width = [&]<int WIDTH, int RT>() {
        return f.a.whole ? launch<WIDTH, 64, RT, true>(f, parts, s, stream) : launch<WIDTH, 64, RT, false>(f, parts, s, stream);
    };
    if (D == 32) return of_width.template operator()<32, 64>();
    return D == 64 ? of_width.template operator()<64, 64>() : of_width.template operator()<128, 32>();
}

}  // namespace agc
