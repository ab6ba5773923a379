// Partial gradients of differential attention.  With the rows' binary logarithms of the sums, which the forward pass leaves,
// P_m = 2^(S_m log2(e) - lse_m) is formed again, and
//   dP = dout v^T,  D_m = sum over keys of P_m dP,  dS_1 = P_1 (dP - D_1),  dS_2 = -lambda P_2 (dP - D_2)
//   dq_m = scale dS_m k_m,  dk_m = scale dS_m^T q_m,  dv = (P_1 - lambda P_2)^T dout,  G[p,h] = - sum over p's queries of D_2
// dP is one product for both maps, dv one of their difference.
//
// Two passes, one whose workgroups own rows (D, dq) and one whose workgroups own keys (dk, dv), and no sums in memory whose
// order could change: 20 d + 8 e operations a pair where a single pass would do with 12 d + 4 e.  The first goes over its
// keys twice: D comes from the same P and dP as dS, which makes the rows of dS add up to zero to the last bits of binary32
// (from dout and the rounded out they would miss it by 2^-8, and a query that sees one key would get a gradient where
// there is none), and makes D_2, whose sums are rows of G, a binary32 sum of binary32 terms.
// dS and P enter their products as bfloat16, 2^-8 of a term at most, as the products' other operands are; sums are binary32.
#include "agc_attention.h"

namespace agc {

namespace {

struct AttnGradients {
    Attn a;
    const uint16_t* dout;
    int64_t lddout;
    const float* lse;
    float* sums;           // D_m of every (head, map, token)
    uint16_t *dq, *dk, *dv;
    int64_t lddq, lddk, lddv;
    int slots;
};

// ------------------------------------------------------------------ D and dq: a workgroup's rows, all keys in sight, twice
template <int D, int WAVES, int KT>
__global__ __launch_bounds__(64 * WAVES) void k_attn_dq(AttnGradients f)
{
    using Tile = AttnTile<D>;
    constexpr int E = 2 * D, kSteps = D / 16, kBlocks = D / 32;
    __shared__ __attribute__((aligned(1024))) char lds[2][2][KT * Tile::kRow];   // buffer; keys, values
    const Attn& a = f.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int id = xcd_order(blockIdx.x, f.slots * a.kv_heads);
    const int head_k = id / f.slots, slot = id - head_k * f.slots;
    const uint32_t group = a.group.d;

    const int s = attn_find(a.q_end, a.n_seqs, a.tokens_q, group, 32 * WAVES, slot);
    const AttnSeq seq = attn_sequence(a, s);
    const int first = attn_first_slot(a.q_end, s, a.tokens_q, group, 32 * WAVES);
    const int rows = seq.lq * (int)group, tiles = (rows + 32 * WAVES - 1) / (32 * WAVES);
    const int tile = tiles - 1 - (slot - first);
    if (tile < 0 || tile >= tiles) return;

    const int row_ = tile * 32 * WAVES + wave * 32 + (lane & 31);
    const int row = min(row_, rows - 1), t = (int)a.group(row), g = row - t * (int)group, head = head_k * (int)group + g;
    const int seen = attn_seen(a, seq, t);
    const int seen_least = __builtin_amdgcn_readfirstlane(seen), seen_most = __builtin_amdgcn_readlane(seen, 31);
    const int last_row = min(tile * 32 * WAVES + 32 * WAVES, rows) - 1;
    const int keys = attn_seen(a, seq, (int)a.group(last_row));

    tile_bf16x8 q[2][kSteps], go[2 * kSteps];
    {
        const uint16_t* p = a.q + (int64_t)(seq.q0 + t) * a.ldq + (int64_t)head * E + (lane >> 5) * 8;
        const uint16_t* o = f.dout + (int64_t)(seq.q0 + t) * f.lddout + (int64_t)head * E + (lane >> 5) * 8;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) q[m][i] = *reinterpret_cast<const tile_bf16x8*>(p + m * D + i * 16);
#pragma unroll
        for (int i = 0; i < 2 * kSteps; ++i) go[i] = *reinterpret_cast<const tile_bf16x8*>(o + i * 16);
    }
    float* const stat = f.sums + (int64_t)2 * head * a.tokens_q + seq.q0 + t;
    float lse[2], mean[2] = {0.0f, 0.0f};
#pragma unroll
    for (int m = 0; m < 2; ++m) lse[m] = f.lse[(int64_t)(2 * head + m) * a.tokens_q + seq.q0 + t];

    const char* const keys_at = reinterpret_cast<const char*>(a.k + (int64_t)seq.k0 * a.ldk + head_k * E);
    const char* const values_at = reinterpret_cast<const char*>(a.v + (int64_t)seq.k0 * a.ldv + head_k * E);
    const auto fetch = [&](int j0, int buffer) {
        Tile::template load<KT, WAVES>(lds[buffer][0], wave, lane, [&](int r) { return keys_at + (int64_t)min(j0 + r, seq.lk - 1) * a.ldk * 2; });
        Tile::template load<KT, WAVES>(lds[buffer][1], wave, lane, [&](int r) { return values_at + (int64_t)min(j0 + r, seq.lk - 1) * a.ldv * 2; });
    };

    attn_f32x16 acc[2][kBlocks];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) acc[m][b] = attn_f32x16{};

    // the first turn forms D, the second dq
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
        __syncthreads();   // nobody reads the last turn's tiles any more
        if (keys > 0) fetch(0, 0);
        int buffer = 0;
#pragma unroll 1
        for (int j0 = 0; j0 < keys; j0 += KT, buffer ^= 1) {
            attn_wait_loads();
            __syncthreads();
            if (j0 + KT < keys) fetch(j0 + KT, buffer ^ 1);
            const char *const k_lds = lds[buffer][0], *const v_lds = lds[buffer][1];
#pragma unroll 1
            for (int sub = 0; sub < KT / 32; ++sub) {
                const int j = j0 + sub * 32;
                if (j >= seen_most) break;
                const bool masked = j + 32 > seen_least;
                const int at = sub * 32 + attn_swapped(lane & 31), left = seen - j;
                attn_f32x16 dp{};
#pragma unroll
                for (int i = 0; i < 2 * kSteps; ++i) dp = attn_mfma(Tile::straight(v_lds, at, i * 2 + (lane >> 5)), go[i], dp);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    attn_f32x16 score{};
#pragma unroll
                    for (int i = 0; i < kSteps; ++i)
                        score = attn_mfma(Tile::straight(k_lds, at, m * (D / 8) + i * 2 + (lane >> 5)), q[m][i], score);
                    float v[16];
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = __builtin_amdgcn_exp2f(score[r] * a.to_log2 - lse[m]);
                        v[r] = p * (turn == 0 ? dp[r] : dp[r] - mean[m]);
                    }
                    if (masked) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) v[r] = attn_row_swapped(r, lane) < left ? v[r] : 0.0f;
                    }
                    if (turn == 0) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) mean[m] += v[r];
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const tile_bf16x8 ds = attn_operand(v, i);
#pragma unroll
                            for (int b = 0; b < kBlocks; ++b)
                                acc[m][b] = attn_mfma(Tile::turned(k_lds, sub * 32 + i * 16, m * (D / 8) + b * 4, lane), ds, acc[m][b]);
                        }
                    }
                }
            }
        }
        if (turn == 0) {
#pragma unroll
            for (int m = 0; m < 2; ++m) mean[m] += attn_other_half(mean[m]);
        }
    }
    if (row_ >= rows) return;
    if (lane < 32) stat[0] = mean[0], stat[a.tokens_q] = mean[1];
    const float factor[2] = {a.scale, -a.scale * a.lambda[head]};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        uint16_t* o = f.dq + (int64_t)(seq.q0 + t) * f.lddq + (int64_t)(2 * head + m) * a.d;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) attn_store(o, b * 32, a.d, lane, acc[m][b], factor[m]);
    }
}

// ------------------------------------------------------------------ dk, dv: a workgroup's keys, all rows that see them
// What a tile's rows bring along: lse and D of both maps, lambda, keys in sight.
struct RowFacts {
    float lse[2], mean[2], lambda;
    int seen;
};

template <int D, int WAVES, int RT>
__global__ __launch_bounds__(64 * WAVES) void k_attn_dkv(AttnGradients f)
{
    using Tile = AttnTile<D>;
    constexpr int E = 2 * D, kSteps = D / 16, kBlocks = D / 32;
    __shared__ __attribute__((aligned(1024))) char lds[2][2][RT * Tile::kRow];   // buffer; queries, dout
    __shared__ float facts[2][6][RT];
    const Attn& a = f.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int id = xcd_order(blockIdx.x, f.slots * a.kv_heads);
    const int head_k = id / f.slots, slot = id - head_k * f.slots;
    const uint32_t group = a.group.d;

    const int s = attn_find(a.k_end, a.n_seqs, a.tokens_k, 1, 32 * WAVES, slot);
    const AttnSeq seq = attn_sequence(a, s);
    const int tile = slot - attn_first_slot(a.k_end, s, a.tokens_k, 1, 32 * WAVES);
    if (tile * 32 * WAVES >= seq.lk) return;

    const int key0 = tile * 32 * WAVES + wave * 32, key_ = key0 + (lane & 31), key = min(key_, seq.lk - 1);
    const int rows = seq.lq * (int)group;
    // under the causal mask the first query that sees this tile's first key
    const int begin = (a.causal ? min(max(tile * 32 * WAVES + seq.lq - seq.lk, 0), seq.lq) * (int)group : 0) / RT * RT;

    tile_bf16x8 k[2][kSteps], v[2 * kSteps];
    {
        const uint16_t* p = a.k + (int64_t)(seq.k0 + key) * a.ldk + head_k * E + (lane >> 5) * 8;
        const uint16_t* o = a.v + (int64_t)(seq.k0 + key) * a.ldv + head_k * E + (lane >> 5) * 8;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) k[m][i] = *reinterpret_cast<const tile_bf16x8*>(p + m * D + i * 16);
#pragma unroll
        for (int i = 0; i < 2 * kSteps; ++i) v[i] = *reinterpret_cast<const tile_bf16x8*>(o + i * 16);
    }
    const char* const queries_at = reinterpret_cast<const char*>(a.q + (int64_t)seq.q0 * a.ldq + (int64_t)head_k * group * E);
    const char* const douts_at = reinterpret_cast<const char*>(f.dout + (int64_t)seq.q0 * f.lddout + (int64_t)head_k * group * E);
    const auto fetch = [&](int r0, int buffer) {
        const auto place = [&](const char* at, int64_t ld, int r) {
            const int row = min(r0 + r, rows - 1), t = (int)a.group(row);
            return at + (t * ld + (int64_t)(row - t * (int)group) * E) * 2;
        };
        Tile::template load<RT, WAVES>(lds[buffer][0], wave, lane, [&](int r) { return place(queries_at, a.ldq, r); });
        Tile::template load<RT, WAVES>(lds[buffer][1], wave, lane, [&](int r) { return place(douts_at, f.lddout, r); });
    };
    // a row's facts, read a tile ahead by one thread a row and put into LDS when its buffer is free
    const auto read_facts = [&](int r0) {
        RowFacts o;
        const int row_ = r0 + (int)threadIdx.x, row = min(row_, rows - 1), t = (int)a.group(row), head = head_k * (int)group + row - t * (int)group;
        const int64_t at = (int64_t)2 * head * a.tokens_q + seq.q0 + t;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            o.lse[m] = f.lse[at + m * (int64_t)a.tokens_q];
            o.mean[m] = f.sums[at + m * (int64_t)a.tokens_q];
        }
        o.lambda = a.lambda[head];
        o.seen = row_ < rows ? attn_seen(a, seq, t) : 0;
        return o;
    };

    attn_f32x16 acc_k[2][kBlocks], acc_v[2 * kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) acc_k[0][b] = acc_k[1][b] = acc_v[b] = acc_v[kBlocks + b] = attn_f32x16{};

    RowFacts mine{};
    if (begin < rows) {
        fetch(begin, 0);
        if (threadIdx.x < RT) mine = read_facts(begin);
    }
    int buffer = 0;
#pragma unroll 1
    for (int r0 = begin; r0 < rows; r0 += RT, buffer ^= 1) {
        if (threadIdx.x < RT) {
            facts[buffer][0][threadIdx.x] = mine.lse[0];
            facts[buffer][1][threadIdx.x] = mine.lse[1];
            facts[buffer][2][threadIdx.x] = mine.mean[0];
            facts[buffer][3][threadIdx.x] = mine.mean[1];
            facts[buffer][4][threadIdx.x] = mine.lambda;
            facts[buffer][5][threadIdx.x] = __int_as_float(mine.seen);
        }
        attn_wait_loads();
        __syncthreads();
        if (r0 + RT < rows) {
            fetch(r0 + RT, buffer ^ 1);
            if (threadIdx.x < RT) mine = read_facts(r0 + RT);
        }
        const char *const q_lds = lds[buffer][0], *const o_lds = lds[buffer][1];
#pragma unroll 1
        for (int sub = 0; sub < RT / 32; ++sub) {
            const int r_first = r0 + sub * 32, r_last = r_first + 31;
            if (r_first >= rows) break;
            // keys in sight grow with the row
            const int seen_first = attn_seen(a, seq, (int)a.group(r_first)), seen_last = attn_seen(a, seq, (int)a.group(min(r_last, rows - 1)));
            if (seen_last <= key0) continue;
            const bool masked = seen_first < key0 + 32 || r_last >= rows;
            const int at = sub * 32 + attn_swapped(lane & 31);
            attn_f32x16 dp{}, s1{}, s2{};
#pragma unroll
            for (int i = 0; i < 2 * kSteps; ++i) dp = attn_mfma(Tile::straight(o_lds, at, i * 2 + (lane >> 5)), v[i], dp);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                s1 = attn_mfma(Tile::straight(q_lds, at, i * 2 + (lane >> 5)), k[0][i], s1);
                s2 = attn_mfma(Tile::straight(q_lds, at, D / 8 + i * 2 + (lane >> 5)), k[1][i], s2);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {   // sixteen rows at a time, eight of them this lane's
                float mixed[8], ds1[8], ds2[8];
                const int r8 = sub * 32 + i * 16 + 8 * (lane >> 5);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r = r8 + e;
                    float p1 = __builtin_amdgcn_exp2f(s1[i * 8 + e] * a.to_log2 - facts[buffer][0][r]);
                    float p2 = facts[buffer][4][r] * __builtin_amdgcn_exp2f(s2[i * 8 + e] * a.to_log2 - facts[buffer][1][r]);
                    mixed[e] = p1 - p2;
                    ds1[e] = p1 * (dp[i * 8 + e] - facts[buffer][2][r]);
                    ds2[e] = p2 * (facts[buffer][3][r] - dp[i * 8 + e]);
                    if (masked && key_ >= __float_as_int(facts[buffer][5][r])) mixed[e] = ds1[e] = ds2[e] = 0.0f;
                }
                const tile_bf16x8 pm = __builtin_bit_cast(tile_bf16x8, bf16_pack8(mixed));
                const tile_bf16x8 d1 = __builtin_bit_cast(tile_bf16x8, bf16_pack8(ds1)), d2 = __builtin_bit_cast(tile_bf16x8, bf16_pack8(ds2));
#pragma unroll
                for (int b = 0; b < 2 * kBlocks; ++b)
                    acc_v[b] = attn_mfma(Tile::turned(o_lds, sub * 32 + i * 16, b * 4, lane), pm, acc_v[b]);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    acc_k[0][b] = attn_mfma(Tile::turned(q_lds, sub * 32 + i * 16, b * 4, lane), d1, acc_k[0][b]);
                    acc_k[1][b] = attn_mfma(Tile::turned(q_lds, sub * 32 + i * 16, D / 8 + b * 4, lane), d2, acc_k[1][b]);
                }
            }
        }
    }
    if (key_ >= seq.lk) return;
    uint16_t* o = f.dv + (int64_t)(seq.k0 + key) * f.lddv + (int64_t)head_k * a.e;
#pragma unroll
    for (int b = 0; b < 2 * kBlocks; ++b) attn_store(o, b * 32, a.e, lane, acc_v[b], 1.0f);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        o = f.dk + (int64_t)(seq.k0 + key) * f.lddk + (int64_t)(2 * head_k + m) * a.d;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) attn_store(o, b * 32, a.d, lane, acc_k[m][b], a.scale);
    }
}

// ------------------------------------------------------------------ rows of G
struct AttnParts {
    int end[kMostParts];
};

// A workgroup adds up one partition's D_2 of one head, in binary64 and a fixed order.
__global__ __launch_bounds__(256) void k_attn_lambda(AttnParts parts, const float* sums, int tokens, const int32_t* q_end, int n_seqs, float* G, int64_t ldg)
{
    const int p = blockIdx.y, h = blockIdx.x, covered = min(max(q_end[n_seqs - 1], 0), tokens);
    const int begin = p ? parts.end[p - 1] : 0, end = min(parts.end[p], covered);
    const float* from = sums + (int64_t)(2 * h + 1) * tokens;
    double sum = 0;
    for (int t = begin + (int)threadIdx.x; t < end; t += 256) sum += from[t];
    __shared__ double all[256];
    all[threadIdx.x] = sum;
    for (int half = 128; half > 0; half >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < half) all[threadIdx.x] += all[threadIdx.x + half];
    }
    if (threadIdx.x == 0) G[p * ldg + h] = (float)-all[0];
}

template <int D, int WAVES, int KT, int RT>
hipError_t launch(AttnGradients f, hipStream_t stream)
{
    const int64_t rows = (int64_t)f.a.tokens_q * f.a.group.d;
    f.slots = (int)(rows / (32 * WAVES)) + f.a.n_seqs;
    k_attn_dq<D, WAVES, KT><<<f.slots * f.a.kv_heads, 64 * WAVES, 0, stream>>>(f);
    f.slots = f.a.tokens_k / (32 * WAVES) + f.a.n_seqs;
    k_attn_dkv<D, WAVES, RT><<<f.slots * f.a.kv_heads, 64 * WAVES, 0, stream>>>(f);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_gradients(const AttnCall& c, hipStream_t stream)
{
    AttnGradients f{Attn{.group = Divider(c.heads / c.kv_heads)}};
    char* place = c.workspace;
    hipError_t e = attn_lay_out(c, f.a, f.dout, f.lddout, place, stream);
    if (e != hipSuccess) return e;
    f.lse = c.lse, f.sums = reinterpret_cast<float*>(place);
    f.dq = static_cast<uint16_t*>(c.dq), f.dk = static_cast<uint16_t*>(c.dk), f.dv = static_cast<uint16_t*>(c.dv);
    f.lddq = c.lddq, f.lddk = c.lddk, f.lddv = c.lddv;
    const int D = attn_width(c.d, c.e);
    e = D == 32 ? launch<32, 8, 64, 64>(f, stream) : D == 64 ? launch<64, 8, 64, 64>(f, stream) : launch<128, 4, 64, 32>(f, stream);
    if (e != hipSuccess) return e;
    AttnParts parts;
    for (int p = 0; p < c.k_parts; ++p) parts.end[p] = (int)c.part_end[p];
    k_attn_lambda<<<dim3(c.heads, c.k_parts), 256, 0, stream>>>(parts, f.sums, f.a.tokens_q, c.q_end, c.n_seqs, c.G, c.ldg);
    return hipGetLastError();
}

}  // namespace agc
