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
    float* facts;          // lse_m and D_m of every (head, map, token), lse as the keys' pass takes it
    int64_t of_facts;      // values of each
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
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
    float lse[2], mean[2] = {0.0f, 0.0f};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        lse[m] = f.lse[(int64_t)(2 * head + m) * a.tokens_q + seq.q0 + t];
        lse[m] = seen <= 1 ? 0.0f : lse[m];   // without keys it is -infinity; a single key's map is 2^0
    }

    const char* const keys_at = reinterpret_cast<const char*>(a.k + (int64_t)seq.k0 * a.ldk + head_k * E);
    const char* const values_at = reinterpret_cast<const char*>(a.v + (int64_t)seq.k0 * a.ldv + head_k * E);
    const auto fetch = [&](int j0, int buffer) {
        Tile::template load<KT, WAVES>(lds[buffer][0], wave, lane, [&](int r) { return keys_at + (int64_t)min(j0 + r, seq.lk - 1) * a.ldk * 2; });
        Tile::template load<KT, WAVES>(lds[buffer][1], wave, lane, [&](int r) { return values_at + (int64_t)min(j0 + r, seq.lk - 1) * a.ldv * 2; });
    };

    const AttnReads<D> reads(lane);
    // All keys in sight, 32 at a time: both maps and dP.
    const auto over_keys = [&](const auto& use) {
        if (keys > 0) fetch(0, 0);
        int buffer = 0;
#pragma unroll 1
        for (int j0 = 0; j0 < keys; j0 += KT, buffer ^= 1) {
            attn_wait_loads();
            __syncthreads();
            if (j0 + KT < keys) fetch(j0 + KT, buffer ^ 1);
            AttnLds k_tile = attn_lds(lds[buffer][0]), v_tile = attn_lds(lds[buffer][1]);
#pragma unroll 1
            for (int j = j0; j < min(j0 + KT, seen_most); j += 32, k_tile += 32 * Tile::kRow, v_tile += 32 * Tile::kRow) {
                // two products of dP, one of each map, in turn
                attn_f32x16 dp{}, score[2] = {};
                const auto read = [&](int n) {
                    return n % 4 < 2 ? reads.straight(v_tile, n / 4 * 2 + n % 4) : reads.straight(k_tile, n % 4 % 2 * kSteps + n / 4);
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
                    const int left = seen - j;
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
                use(k_tile, score, dp);
            }
        }
    };

    over_keys([&](AttnLds, const attn_f32x16* map, const attn_f32x16& dp) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) mean[m] = fmaf(map[m][r], dp[r], mean[m]);
    });
#pragma unroll
    for (int m = 0; m < 2; ++m) mean[m] += attn_other_half(mean[m]);
    __syncthreads();   // nobody reads tiles any more

    attn_f32x16 acc[2][kBlocks];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) acc[m][b] = attn_f32x16{};
    over_keys([&](AttnLds k_tile, const attn_f32x16* map, const attn_f32x16& dp) {
        const auto read = [&](int n) { return reads.turned(k_tile, n / (2 * kBlocks) * 16, n % (2 * kBlocks)); };
        auto stream = attn_stream<4 * kBlocks, 2>(read);
        stream.start();
        tile_bf16x8 ds[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = map[m][i * 8 + e] * (dp[i * 8 + e] - mean[m]);
                ds[i][m] = __builtin_bit_cast(tile_bf16x8, bf16_pack8(v));
            }
        stream.run([&](int n, const tile_bf16x8& k) {
            const int i = n / (2 * kBlocks), m = n / kBlocks % 2, b = n % kBlocks;
            acc[m][b] = attn_mfma(k, ds[i][m], acc[m][b]);
        });
    });
    if (row_ >= rows) return;
    if (lane < 32) {
        float* fact = f.facts + (int64_t)2 * head * a.tokens_q + seq.q0 + t;
#pragma unroll
        for (int m = 0; m < 2; ++m, fact += a.tokens_q) fact[0] = lse[m], fact[f.of_facts] = mean[m];
    }
    const float factor[2] = {a.scale, -a.scale * a.lambda[head]};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        uint16_t* o = f.dq + (int64_t)(seq.q0 + t) * f.lddq + (int64_t)(2 * head + m) * a.d;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) attn_store(o, b * 32, a.d, lane, acc[m][b], factor[m]);
    }
}

// ------------------------------------------------------------------ dk, dv: a workgroup's keys, all rows that see them
// A tile's rows bring along lse and D of both maps and, where heads share keys, lambda.
template <int D, int WAVES, int RT, bool SHARED>
__global__ __launch_bounds__(64 * WAVES) void k_attn_dkv(AttnGradients f)
{
    using Tile = AttnTile<D>;
    constexpr int E = 2 * D, kSteps = D / 16, kBlocks = D / 32;
    __shared__ __attribute__((aligned(1024))) char lds[2][2][RT * Tile::kRow];   // buffer; queries, dout
    __shared__ __attribute__((aligned(1024))) char values[32 * WAVES * Tile::kRow];
    __shared__ __attribute__((aligned(256))) float facts[2][SHARED ? 5 : 4][RT];
    const Attn& a = f.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int id = xcd_order(blockIdx.x, f.slots * a.kv_heads);
    const int head_k = id / f.slots, slot = id - head_k * f.slots;
    const uint32_t group = a.group.d;

    const int s = attn_find(a.k_end, a.n_seqs, a.tokens_k, 1, 32 * WAVES, slot);
    const AttnSeq seq = attn_sequence(a, s);
    const int tile = slot - attn_first_slot(a.k_end, s, a.tokens_k, 1, 32 * WAVES);
    if (tile * 32 * WAVES >= seq.lk) return;

    const int key0 = tile * 32 * WAVES + wave * 32, key_ = key0 + attn_swapped(lane & 31), key = min(key_, seq.lk - 1);
    const int rows = seq.lq * (int)group;
    // under the causal mask the first query that sees this tile's first key
    const int begin = (a.causal ? min(max(tile * 32 * WAVES + seq.lq - seq.lk, 0), seq.lq) * (int)group : 0) / RT * RT;

    // the keys stay in registers, the values in LDS, as far as the waves' registers go
    tile_bf16x8 k[2][kSteps];
    {
        const uint16_t* p = a.k + (int64_t)(seq.k0 + key) * a.ldk + head_k * E + (lane >> 5) * 8;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) k[m][i] = *reinterpret_cast<const tile_bf16x8*>(p + m * D + i * 16);
        const char* const values_at = reinterpret_cast<const char*>(a.v + (int64_t)seq.k0 * a.ldv + head_k * E);
        Tile::template load<32 * WAVES, WAVES>(values, wave, lane, [&](int r) { return values_at + (int64_t)min(tile * 32 * WAVES + r, seq.lk - 1) * a.ldv * 2; });
    }
    const AttnLds v_tile = attn_lds(values) + wave * 32 * Tile::kRow;
    const char* const queries_at = reinterpret_cast<const char*>(a.q + (int64_t)seq.q0 * a.ldq + (int64_t)head_k * group * E);
    const char* const douts_at = reinterpret_cast<const char*>(f.dout + (int64_t)seq.q0 * f.lddout + (int64_t)head_k * group * E);
    const auto fetch = [&](int r0, int buffer) {
        const auto place = [&](const char* at, int64_t ld, int r) {
            const int row = min(r0 + r, rows - 1), t = (int)a.group(row);
            return at + (t * ld + (int64_t)(row - t * (int)group) * E) * 2;
        };
        Tile::template load<RT, WAVES>(lds[buffer][0], wave, lane, [&](int r) { return place(queries_at, a.ldq, r); });
        Tile::template load<RT, WAVES>(lds[buffer][1], wave, lane, [&](int r) { return place(douts_at, f.lddout, r); });
        // a wave a fact, a lane a row
        for (int n = wave; n < (SHARED ? 5 : 4); n += WAVES) {
            const int row = min(r0 + lane, rows - 1), t = (int)a.group(row), head = head_k * (int)group + row - t * (int)group;
            const float* at = n == 4 ? a.lambda + head : f.facts + (n >> 1) * f.of_facts + (int64_t)(2 * head + (n & 1)) * a.tokens_q + seq.q0 + t;
            if (lane < RT) load4_to_lds(at, facts[buffer][n]);
        }
    };
    attn_f32x16 acc_k[2][kBlocks], acc_v[2 * kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) acc_k[0][b] = acc_k[1][b] = acc_v[b] = acc_v[kBlocks + b] = attn_f32x16{};

    const AttnReads<D> reads(lane);
    const float lambda_of_all = a.lambda[head_k * group];   // where every key head has one query head
    if (begin < rows) fetch(begin, 0);
    int buffer = 0;
#pragma unroll 1
    for (int r0 = begin; r0 < rows; r0 += RT, buffer ^= 1) {
        attn_wait_loads();
        __syncthreads();
        if (r0 + RT < rows) fetch(r0 + RT, buffer ^ 1);
        AttnLds q_tile = attn_lds(lds[buffer][0]), o_tile = attn_lds(lds[buffer][1]);
#pragma unroll 1
        for (int r_first = r0; r_first < min(r0 + RT, rows); r_first += 32, q_tile += 32 * Tile::kRow, o_tile += 32 * Tile::kRow) {
            const int r_last = r_first + 31, sub = r_first - r0;
            // keys in sight grow with the row
            const int seen_first = attn_seen(a, seq, (int)a.group(r_first)), seen_last = attn_seen(a, seq, (int)a.group(min(r_last, rows - 1)));
            if (seen_last <= key0) continue;
            const bool masked = seen_first < max(key0 + 32, 2) || r_last >= rows;
            const float* const fact = &facts[buffer][0][sub + 8 * (lane >> 5)];
            // eight rows' facts: rows 16 i + 8 (lane / 32) + 0 .. 7
            const auto fact8 = [&](int which, int i, float o[8]) {
                const tile_f32x4* p = reinterpret_cast<const tile_f32x4*>(fact + which * RT + i * 16);
                const tile_f32x4 lo = p[0], hi = p[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = lo[e], o[4 + e] = hi[e];
            };
            attn_f32x16 dp{}, score[2] = {};
#pragma unroll
            for (int i = 0; i < 2 * kSteps; ++i) dp = attn_mfma(reads.straight(o_tile, i), reads.straight(v_tile, i), dp);
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int m = 0; m < 2; ++m) score[m] = attn_mfma(reads.straight(q_tile, m * kSteps + i), k[m][i], score[m]);
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = r_first + attn_row_swapped(r, lane), seen = row < rows ? attn_seen(a, seq, (int)a.group(row)) : 0;
                    const bool in = key_ < seen;
                    dp[r] = in ? dp[r] : 0.0f;
#pragma unroll
                    for (int m = 0; m < 2; ++m) score[m][r] = in ? (seen == 1 ? 0.0f : score[m][r]) : -INFINITY;
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float mixed[8], ds[8], lse[8], mean[8], lambda[8];
                fact8(0, i, lse);
                fact8(2, i, mean);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    mixed[e] = __builtin_amdgcn_exp2f(fmaf(score[0][i * 8 + e], a.to_log2, -lse[e]));
                    ds[e] = mixed[e] * (dp[i * 8 + e] - mean[e]);
                }
                const tile_bf16x8 ds1 = __builtin_bit_cast(tile_bf16x8, bf16_pack8(ds));
                fact8(1, i, lse);
                fact8(3, i, mean);
                if constexpr (SHARED) fact8(4, i, lambda);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = (SHARED ? lambda[e] : lambda_of_all) * __builtin_amdgcn_exp2f(fmaf(score[1][i * 8 + e], a.to_log2, -lse[e]));
                    ds[e] = p * (mean[e] - dp[i * 8 + e]);
                    mixed[e] -= p;
                }
                const tile_bf16x8 ds2 = __builtin_bit_cast(tile_bf16x8, bf16_pack8(ds)), p = __builtin_bit_cast(tile_bf16x8, bf16_pack8(mixed));
#pragma unroll
                for (int b = 0; b < 2 * kBlocks; ++b) acc_v[b] = attn_mfma(reads.turned(o_tile, i * 16, b), p, acc_v[b]);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    acc_k[0][b] = attn_mfma(reads.turned(q_tile, i * 16, b), ds1, acc_k[0][b]);
                    acc_k[1][b] = attn_mfma(reads.turned(q_tile, i * 16, kBlocks + b), ds2, acc_k[1][b]);
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
    if (f.a.group.d > 1)
        k_attn_dkv<D, WAVES, RT, true><<<f.slots * f.a.kv_heads, 64 * WAVES, 0, stream>>>(f);
    else
        k_attn_dkv<D, WAVES, RT, false><<<f.slots * f.a.kv_heads, 64 * WAVES, 0, stream>>>(f);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_gradients(const AttnCall& c, hipStream_t stream)
{
    AttnGradients f{Attn{.group = Divider(c.heads / c.kv_heads)}};
    char* place = c.workspace;
    hipError_t e = attn_lay_out(c, f.a, f.dout, f.lddout, place, stream);
    if (e != hipSuccess) return e;
    f.lse = c.lse, f.facts = reinterpret_cast<float*>(place), f.of_facts = (int64_t)2 * c.heads * c.tokens_q;
    f.dq = static_cast<uint16_t*>(c.dq), f.dk = static_cast<uint16_t*>(c.dk), f.dv = static_cast<uint16_t*>(c.dv);
    f.lddq = c.lddq, f.lddk = c.lddk, f.lddv = c.lddv;
    const int D = attn_width(c.d, c.e);
    e = D == 32 ? launch<32, 8, 64, 64>(f, stream) : D == 64 ? launch<64, 8, 64, 64>(f, stream) : launch<128, 4, 64, 32>(f, stream);
    if (e != hipSuccess) return e;
    AttnParts parts;
    for (int p = 0; p < c.k_parts; ++p) parts.end[p] = (int)c.part_end[p];
    k_attn_lambda<<<dim3(c.heads, c.k_parts), 256, 0, stream>>>(parts, f.facts + f.of_facts, f.a.tokens_q, c.q_end, c.n_seqs, c.G, c.ldg);
    return hipGetLastError();
}

}  // namespace agc
