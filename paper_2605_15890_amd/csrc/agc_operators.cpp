// C ABI of the operators round the coded step (include/agc.h): synchronous argument validation and launches on the
// caller's stream.  No context: messages go to agc_last_error(NULL).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "../../include/agc.h"
#include "agc_operators.h"

namespace {

agc_status refuse(agc_status st, const std::string& msg)
{
    return (agc_status)agc::note_failure(st, msg.c_str());
}

agc_status launched(hipError_t e, const char* what)
{
    return e == hipSuccess ? AGC_OK : refuse(AGC_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

bool misaligned(const void* p, uintptr_t unit) { return (reinterpret_cast<uintptr_t>(p) & (unit - 1)) != 0; }

constexpr int64_t kMostTokens = (int64_t)1 << 26;
constexpr int kMostWidth = 65536;

// Data partitions as the ends of consecutive runs of tokens, empty ones among them.
agc_status partitions(const char* name, const int64_t* end, int k, int64_t n_tokens)
{
    if (!end) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (k < 1 || k > agc::kMostParts) return refuse(AGC_ESHAPE, std::string(name) + ": k_parts must be 1..256");
    int64_t last = 0;
    for (int p = 0; p < k; ++p) {
        if (end[p] < last) return refuse(AGC_ESHAPE, std::string(name) + ": the partitions' ends must not descend");
        last = end[p];
    }
    return last == n_tokens ? AGC_OK : refuse(AGC_ESHAPE, std::string(name) + ": the last partition must end at n_tokens");
}

agc_status embed_arguments(const char* name, const agc::EmbedCall& c, int token_bytes, int type, int64_t ld)
{
    if (!c.tokens && c.n > 0) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if ((token_bytes != 4 && token_bytes != 8) || (type != AGC_TYPE_F32 && type != AGC_TYPE_BF16))
        return refuse(AGC_EINVAL, std::string(name) + ": tokens have 4 or 8 bytes, values are float or bfloat16");
    if (c.n < 0 || c.n > kMostTokens || c.vocab < 1 || c.vocab > INT32_MAX || c.dim < 1 || c.dim > kMostWidth || ld < c.dim)
        return refuse(AGC_ESHAPE, std::string(name) + ": n_tokens must be 0..2^26, vocab 1..2^31-1, dim 1..65536 and at most the row stride");
    if (misaligned(c.tokens, token_bytes)) return refuse(AGC_EALIGN, std::string(name) + ": tokens are not aligned to their bytes");
    return AGC_OK;
}

agc_status gated_arguments(const char* name, const agc::GatedCall& c, int act)
{
    if ((!c.x && c.tokens > 0) || !c.wg || !c.wu || !c.workspace) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (act != AGC_ACT_SILU && act != AGC_ACT_GELU) return refuse(AGC_EINVAL, std::string(name) + ": unknown activation");
    if (c.tokens < 0 || c.tokens > kMostTokens || c.d_in < 1 || c.d_in > kMostWidth || c.d_ff < 1 || c.d_ff > kMostWidth)
        return refuse(AGC_ESHAPE, std::string(name) + ": n_tokens must be 0..2^26, d_in and d_ff 1..65536");
    if (c.ldx < c.d_in || c.ldw < c.d_in) return refuse(AGC_ESHAPE, std::string(name) + ": a row stride is smaller than the row");
    if (misaligned(c.x, 2) || misaligned(c.wg, 2) || misaligned(c.wu, 2) || misaligned(c.workspace, 256))
        return refuse(AGC_EALIGN, std::string(name) + ": operands need 2-byte alignment, the workspace 256 bytes");
    return AGC_OK;
}

agc_status attn_arguments(const char* name, const agc::AttnCall& c, bool gradients)
{
    const std::string n = name;
    if (c.tokens_q < 0 || c.tokens_q > kMostTokens || c.tokens_k < 0 || c.tokens_k > kMostTokens || c.n_seqs < 1 || c.n_seqs > (1 << 20))
        return refuse(AGC_ESHAPE, n + ": tokens_q and tokens_k must be 0..2^26, n_seqs 1..2^20");
    if (c.heads < 1 || c.kv_heads < 1 || c.heads > kMostWidth || c.heads % c.kv_heads || c.d < 1 || c.d > 128 || c.e < 1 || c.e > 256)
        return refuse(AGC_ESHAPE, n + ": heads must be a multiple of kv_heads, head_dim 1..128, value_dim 1..256");
    // a grid has fewer than 2^32 threads: at most two a row of a head (four of wide ones), and five small workgroups of 256 a
    // sequence and key head
    const int D = agc::attn_width(c.d, c.e), most = D == 128 ? 1 << 29 : 1 << 30;
    if (c.tokens_q * c.heads > most || c.tokens_k * c.kv_heads > most || (int64_t)c.n_seqs * c.kv_heads > (1 << 21))
        return refuse(AGC_ESHAPE, n + ": tokens times heads must be up to 2^30 (2^29 of wide ones), n_seqs * kv_heads up to 2^21");
    if (!std::isfinite(c.scale * agc::kLog2e) || c.scale < 0)
        return refuse(AGC_EINVAL, n + ": scale must not be negative, and finite times log2(e)");
    if ((c.tokens_q > 0 && !c.q) || (c.tokens_k > 0 && (!c.k || !c.v)) || !c.lambda || !c.q_end || !c.k_end || !c.workspace)
        return refuse(AGC_EINVAL, n + ": null pointer");
    const int64_t row_q = (int64_t)2 * c.heads * c.d, row_k = (int64_t)2 * c.kv_heads * c.d;
    if (c.ldq < row_q || c.ldk < row_k || c.ldv < (int64_t)c.kv_heads * c.e) return refuse(AGC_ESHAPE, n + ": a row stride is smaller than the row");
    if (std::max({c.ldq, c.ldk, c.ldv, c.lddout}) > (1 << 24)) return refuse(AGC_ESHAPE, n + ": row strides must be up to 2^24");
    // heads of just the kernels' widths are read where they lie, 16 bytes at a time
    const uintptr_t unit_d = c.d == D ? 16 : 2, unit_e = c.e == 2 * D ? 16 : 2;
    const auto strided = [](int64_t ld, int64_t rows, uintptr_t unit) { return unit == 16 && rows > 1 && ld % 8; };
    if (misaligned(c.q, unit_d) || misaligned(c.k, unit_d) || misaligned(c.v, unit_e) || strided(c.ldq, c.tokens_q, unit_d) ||
        strided(c.ldk, c.tokens_k, unit_d) || strided(c.ldv, c.tokens_k, unit_e) ||
        (gradients && (misaligned(c.dout, unit_e) || strided(c.lddout, c.tokens_q, unit_e))))
        return refuse(AGC_EALIGN, n + ": rows of heads that are read where they lie need 16-byte alignment");
    if (misaligned(c.lambda, 4) || misaligned(c.q_end, 4) || misaligned(c.k_begin, 4) || misaligned(c.k_end, 4) || misaligned(c.lse, 4) ||
        misaligned(c.workspace, 256))
        return refuse(AGC_EALIGN, n + ": vectors need their elements' alignment, the workspace 256 bytes");
    return AGC_OK;
}

bool known_type(int type) { return type == AGC_TYPE_F32 || type == AGC_TYPE_BF16; }
uintptr_t bytes_of(int type) { return type == AGC_TYPE_F32 ? 4 : 2; }

}  // namespace

extern "C" {

int64_t agc_muon_workspace_bytes(int rows, int cols, int n_mats)
{
    if (rows < 1 || cols < 1 || rows > AGC_MAX_MATRIX || cols > AGC_MAX_MATRIX || n_mats < 1 || n_mats > AGC_MAX_LAYERS) return 0;
    return agc::muon_workspace_bytes(rows, cols, n_mats);
}

agc_status agc_muon_update(float* beta_dev, float* m1_dev, const float* ghat_dev, const int64_t* offset_host, int n_mats,
                           int rows, int cols, float lr, float momentum, int nesterov, float weight_decay, float scale,
                           int steps, void* beta_bf16_dev, void* workspace_dev, void* hip_stream)
{
    if (!beta_dev || !m1_dev || !ghat_dev || !offset_host || !workspace_dev) return refuse(AGC_EINVAL, "agc_muon_update: null pointer");
    if (steps < 1 || steps > 32) return refuse(AGC_EINVAL, "agc_muon_update: steps must be 1..32");
    if (rows < 1 || cols < 1 || rows > AGC_MAX_MATRIX || cols > AGC_MAX_MATRIX || n_mats < 1 || n_mats > AGC_MAX_LAYERS)
        return refuse(AGC_ESHAPE, "agc_muon_update: rows, cols must be 1..32768 and n_mats 1..256");
    if (misaligned(beta_dev, 4) || misaligned(m1_dev, 4) || misaligned(ghat_dev, 4) || misaligned(beta_bf16_dev, 2) ||
        misaligned(workspace_dev, 256))
        return refuse(AGC_EALIGN, "agc_muon_update: vectors need their elements' alignment, the workspace 256 bytes");
    agc::MuonCall c{};
    for (int i = 0; i < n_mats; ++i) {
        if (offset_host[i] < 0) return refuse(AGC_ESHAPE, "agc_muon_update: negative offset");
        c.offset[i] = offset_host[i];
    }
    int64_t sorted[AGC_MAX_LAYERS];
    std::copy(c.offset, c.offset + n_mats, sorted);
    std::sort(sorted, sorted + n_mats);
    for (int i = 1; i < n_mats; ++i)
        if (sorted[i] - sorted[i - 1] < (int64_t)rows * cols) return refuse(AGC_ESHAPE, "agc_muon_update: matrices overlap");
    c.beta = beta_dev, c.m1 = m1_dev, c.ghat = ghat_dev, c.beta_bf16 = static_cast<uint16_t*>(beta_bf16_dev);
    c.n_mats = n_mats, c.rows = rows, c.cols = cols, c.nesterov = nesterov != 0, c.steps = steps;
    c.momentum = momentum;
    c.keep = (float)(1.0 - (double)lr * weight_decay);
    c.rate = lr * scale;
    c.workspace = static_cast<char*>(workspace_dev);
    return launched(agc::launch_muon_update(c, reinterpret_cast<hipStream_t>(hip_stream)), "agc_muon_update");
}

agc_status agc_embed_forward(const void* table_dev, int table_type, int64_t vocab, int dim, const void* tokens_dev,
                             int token_bytes, int64_t n_tokens, float scale, void* out_dev, int out_type, int64_t ldo,
                             void* hip_stream)
{
    const char* const name = "agc_embed_forward";
    agc::EmbedCall c{};
    c.tokens = tokens_dev, c.wide_ids = token_bytes == 8, c.n = n_tokens, c.vocab = vocab, c.dim = dim, c.scale = scale;
    const agc_status st = embed_arguments(name, c, token_bytes, out_type, ldo);
    if (st != AGC_OK) return st;
    if (table_type != AGC_TYPE_F32 && table_type != AGC_TYPE_BF16) return refuse(AGC_EINVAL, std::string(name) + ": unknown type");
    if (!table_dev || (!out_dev && n_tokens > 0)) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (misaligned(table_dev, table_type == AGC_TYPE_F32 ? 4 : 2) || misaligned(out_dev, out_type == AGC_TYPE_F32 ? 4 : 2))
        return refuse(AGC_EALIGN, std::string(name) + ": a pointer is not aligned to its elements");
    if (n_tokens == 0) return AGC_OK;
    c.table = table_dev, c.table_bf16 = table_type == AGC_TYPE_BF16, c.out = out_dev;
    c.value_bf16 = out_type == AGC_TYPE_BF16, c.ld = ldo;
    return launched(agc::launch_embed_forward(c, reinterpret_cast<hipStream_t>(hip_stream)), name);
}

int64_t agc_embed_workspace_bytes(int64_t n_tokens, int64_t vocab, int dim, int k_parts)
{
    if (n_tokens < 0 || n_tokens > kMostTokens || vocab < 1 || dim < 1 || dim > kMostWidth || k_parts < 1 ||
        k_parts > agc::kMostParts || vocab > INT32_MAX / k_parts)
        return 0;
    return agc::embed_workspace_bytes(n_tokens, vocab, dim, k_parts);
}

agc_status agc_embed_partial_gradients(const void* dout_dev, int dout_type, int64_t lddout, const void* tokens_dev,
                                       int token_bytes, int64_t n_tokens, const int64_t* part_end_host, int k_parts,
                                       int64_t vocab, int dim, float scale, float* G_dev, int64_t ldg, void* workspace_dev,
                                       void* hip_stream)
{
    const char* const name = "agc_embed_partial_gradients";
    agc::EmbedCall c{};
    c.tokens = tokens_dev, c.wide_ids = token_bytes == 8, c.n = n_tokens, c.vocab = vocab, c.dim = dim, c.scale = scale;
    agc_status st = embed_arguments(name, c, token_bytes, dout_type, lddout);
    if (st != AGC_OK) return st;
    st = partitions(name, part_end_host, k_parts, n_tokens);
    if (st != AGC_OK) return st;
    if (vocab > INT32_MAX / k_parts) return refuse(AGC_ESHAPE, std::string(name) + ": k_parts * vocab must be below 2^31");
    if (ldg < vocab * dim) return refuse(AGC_ESHAPE, std::string(name) + ": ldg is smaller than the table");
    if ((!dout_dev && n_tokens > 0) || !G_dev || !workspace_dev) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (misaligned(dout_dev, dout_type == AGC_TYPE_F32 ? 4 : 2) || misaligned(G_dev, 4) || misaligned(workspace_dev, 256))
        return refuse(AGC_EALIGN, std::string(name) + ": tensors need their elements' alignment, the workspace 256 bytes");
    c.dout = dout_dev, c.value_bf16 = dout_type == AGC_TYPE_BF16, c.ld = lddout;
    c.part_end = part_end_host, c.k_parts = k_parts, c.G = G_dev, c.ldg = ldg;
    c.workspace = static_cast<char*>(workspace_dev);
    return launched(agc::launch_embed_gradients(c, reinterpret_cast<hipStream_t>(hip_stream)), name);
}

int64_t agc_gated_workspace_bytes(int64_t n_tokens, int d_in, int d_ff, int k_parts)
{
    if (n_tokens < 0 || n_tokens > kMostTokens || d_in < 1 || d_in > kMostWidth || d_ff < 1 || d_ff > kMostWidth || k_parts < 0 ||
        k_parts > agc::kMostParts)
        return 0;
    return agc::gated_workspace_bytes(n_tokens, d_in, d_ff, k_parts);
}

agc_status agc_gated_forward(const void* x_dev, int64_t ldx, const void* w_gate_dev, const void* w_up_dev, int64_t ldw,
                             int64_t n_tokens, int d_in, int d_ff, int act, void* h_dev, int64_t ldh, void* workspace_dev,
                             void* hip_stream)
{
    agc::GatedCall c{};
    c.x = x_dev, c.wg = w_gate_dev, c.wu = w_up_dev, c.ldx = ldx, c.ldw = ldw;
    c.tokens = n_tokens, c.d_in = d_in, c.d_ff = d_ff, c.gelu = act == AGC_ACT_GELU;
    c.workspace = static_cast<char*>(workspace_dev);
    const agc_status st = gated_arguments("agc_gated_forward", c, act);
    if (st != AGC_OK) return st;
    if (!h_dev && n_tokens > 0) return refuse(AGC_EINVAL, "agc_gated_forward: null pointer");
    if (ldh < d_ff) return refuse(AGC_ESHAPE, "agc_gated_forward: ldh is smaller than d_ff");
    if (misaligned(h_dev, 2)) return refuse(AGC_EALIGN, "agc_gated_forward: h needs 2-byte alignment");
    if (n_tokens == 0) return AGC_OK;
    c.h = h_dev, c.ldh = ldh;
    return launched(agc::launch_gated_forward(c, reinterpret_cast<hipStream_t>(hip_stream)), "agc_gated_forward");
}

agc_status agc_gated_partial_gradients(const void* x_dev, int64_t ldx, const void* w_gate_dev, const void* w_up_dev,
                                       int64_t ldw, const void* dh_dev, int64_t lddh, int64_t n_tokens,
                                       const int64_t* part_end_host, int k_parts, int d_in, int d_ff, int act, void* dx_dev,
                                       int64_t lddx, float* G_gate_dev, float* G_up_dev, int64_t ldg, void* workspace_dev,
                                       void* hip_stream)
{
    const char* const name = "agc_gated_partial_gradients";
    agc::GatedCall c{};
    c.x = x_dev, c.wg = w_gate_dev, c.wu = w_up_dev, c.ldx = ldx, c.ldw = ldw;
    c.tokens = n_tokens, c.d_in = d_in, c.d_ff = d_ff, c.gelu = act == AGC_ACT_GELU;
    c.workspace = static_cast<char*>(workspace_dev);
    agc_status st = gated_arguments(name, c, act);
    if (st != AGC_OK) return st;
    st = partitions(name, part_end_host, k_parts, n_tokens);
    if (st != AGC_OK) return st;
    if ((!dh_dev && n_tokens > 0) || !G_gate_dev || !G_up_dev) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (lddh < d_ff || (dx_dev && lddx < d_in)) return refuse(AGC_ESHAPE, std::string(name) + ": a row stride is smaller than the row");
    if (ldg < (int64_t)d_in * d_ff) return refuse(AGC_ESHAPE, std::string(name) + ": ldg is smaller than a weight matrix");
    if (misaligned(dh_dev, 2) || misaligned(dx_dev, 2) || misaligned(G_gate_dev, 4) || misaligned(G_up_dev, 4))
        return refuse(AGC_EALIGN, std::string(name) + ": a pointer is not aligned to its elements");
    c.dh = dh_dev, c.lddh = lddh, c.part_end = part_end_host, c.k_parts = k_parts, c.dx = dx_dev, c.lddx = lddx;
    c.g_gate = G_gate_dev, c.g_up = G_up_dev, c.ldg = ldg;
    return launched(agc::launch_gated_gradients(c, reinterpret_cast<hipStream_t>(hip_stream)), name);
}

agc_status agc_rotary_frequencies(int rot_dim, double base, int scaling, double factor, double original_len,
                                  uint64_t* turns_out, double* amplitude_out)
{
    const char* const name = "agc_rotary_frequencies";
    if (!turns_out || !amplitude_out) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (rot_dim < 2 || rot_dim > agc::kMostRotary || rot_dim % 2) return refuse(AGC_ESHAPE, std::string(name) + ": rot_dim must be even, 2..8192");
    if (scaling != AGC_ROTARY_PLAIN && scaling != AGC_ROTARY_LINEAR && scaling != AGC_ROTARY_BY_PARTS)
        return refuse(AGC_EINVAL, std::string(name) + ": unknown scaling");
    if (!(base > 1) || !std::isfinite(base) || (scaling != AGC_ROTARY_PLAIN && (!(factor >= 1) || !std::isfinite(factor))) ||
        (scaling == AGC_ROTARY_BY_PARTS && (!(original_len > 0) || !std::isfinite(original_len))))
        return refuse(AGC_EINVAL, std::string(name) + ": base must be above 1, factor 1 or more, the original length positive");
    const long double pi = 3.14159265358979323846264338327950288L, log_base = std::log((long double)base);
    // the pair that turns `times` times over the original length
    const auto pair_of = [&](long double times) { return rot_dim * std::log(original_len / (times * 2 * pi)) / (2 * log_base); };
    long double low = 0, high = 0;
    if (scaling == AGC_ROTARY_BY_PARTS) {
        low = std::max(0.0L, std::floor(pair_of(32)));
        high = std::min((long double)rot_dim - 1, std::ceil(pair_of(1)));
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        long double f = std::exp(-2.0L * i / rot_dim * log_base);
        if (scaling == AGC_ROTARY_LINEAR) f /= factor;
        if (scaling == AGC_ROTARY_BY_PARTS) {
            const long double ramp = std::min(1.0L, std::max(0.0L, (i - low) / std::max(high - low, 1e-3L)));
            f = f / factor * ramp + f * (1 - ramp);
        }
        turns_out[i] = (uint64_t)std::round(f / (2 * pi) * 18446744073709551616.0L);
    }
    *amplitude_out = scaling == AGC_ROTARY_BY_PARTS ? 0.1 * std::log(factor) + 1 : 1;
    return AGC_OK;
}

agc_status agc_rotary_apply(const void* x_dev, int type, int64_t ldx, int64_t n_tokens, int heads, int head_dim, int rot_dim,
                            const void* positions_dev, int position_bytes, const uint64_t* turns_dev, int layout,
                            float amplitude, int inverse, void* out_dev, int64_t ldo, void* hip_stream)
{
    const char* const name = "agc_rotary_apply";
    if (!known_type(type) || (position_bytes != 4 && position_bytes != 8) || (layout != AGC_ROTARY_HALF && layout != AGC_ROTARY_INTERLEAVED))
        return refuse(AGC_EINVAL, std::string(name) + ": values are float or bfloat16, positions have 4 or 8 bytes, pairs are halves or neighbours");
    if (n_tokens < 0 || n_tokens > kMostTokens || heads < 1 || head_dim < 2 || (int64_t)heads * head_dim > kMostWidth || rot_dim < 2 ||
        rot_dim > head_dim || rot_dim > agc::kMostRotary || rot_dim % 2)
        return refuse(AGC_ESHAPE, std::string(name) + ": n_tokens must be 0..2^26, heads * head_dim up to 65536, rot_dim even, 2..head_dim and 8192");
    if (ldx < (int64_t)heads * head_dim || ldo < (int64_t)heads * head_dim)
        return refuse(AGC_ESHAPE, std::string(name) + ": a row stride is smaller than the row");
    if (!turns_dev || (n_tokens > 0 && (!x_dev || !out_dev || !positions_dev))) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (misaligned(x_dev, bytes_of(type)) || misaligned(out_dev, bytes_of(type)) || misaligned(positions_dev, position_bytes) ||
        misaligned(turns_dev, 8))
        return refuse(AGC_EALIGN, std::string(name) + ": a pointer is not aligned to its elements");
    if (x_dev == out_dev && ldx != ldo && n_tokens > 1) return refuse(AGC_EINVAL, std::string(name) + ": in place the row strides must be equal");
    if (n_tokens == 0) return AGC_OK;
    agc::RotaryCall c{};
    c.x = x_dev, c.out = out_dev, c.bf16 = type == AGC_TYPE_BF16, c.ldx = ldx, c.ldo = ldo, c.n = n_tokens;
    c.heads = heads, c.dim = head_dim, c.rot = rot_dim, c.positions = positions_dev, c.wide_ids = position_bytes == 8;
    c.turns = turns_dev, c.interleaved = layout == AGC_ROTARY_INTERLEAVED, c.inverse = inverse != 0, c.amplitude = amplitude;
    return launched(agc::launch_rotary(c, reinterpret_cast<hipStream_t>(hip_stream)), name);
}

agc_status agc_dropout(const void* x_dev, int x_type, int64_t ldx, const void* residual_dev, int64_t ldr, int64_t rows, int cols,
                       double p, uint64_t seed, uint64_t step, uint32_t site, void* out_dev, int out_type, int64_t ldo,
                       void* hip_stream)
{
    const char* const name = "agc_dropout";
    if (!known_type(x_type) || !known_type(out_type)) return refuse(AGC_EINVAL, std::string(name) + ": values are float or bfloat16");
    if (!(p >= 0 && p <= 1)) return refuse(AGC_EINVAL, std::string(name) + ": p must be 0..1");
    if (rows < 0 || rows > kMostTokens || cols < 1 || cols > kMostWidth || site > 65535)
        return refuse(AGC_ESHAPE, std::string(name) + ": rows must be 0..2^26, cols 1..65536, site 0..65535");
    if (ldx < cols || ldo < cols || (residual_dev && ldr < cols)) return refuse(AGC_ESHAPE, std::string(name) + ": a row stride is smaller than the row");
    if (rows > 0 && (!x_dev || !out_dev)) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (misaligned(x_dev, bytes_of(x_type)) || misaligned(out_dev, bytes_of(out_type)) || misaligned(residual_dev, bytes_of(out_type)))
        return refuse(AGC_EALIGN, std::string(name) + ": a pointer is not aligned to its elements");
    // the stride of a single row says nothing
    if (rows > 0 && ((x_dev == out_dev && (x_type != out_type || (rows > 1 && ldx != ldo))) || (rows > 1 && residual_dev == out_dev && ldr != ldo)))
        return refuse(AGC_EINVAL, std::string(name) + ": in place the types and row strides must be equal");
    if (rows == 0) return AGC_OK;
    agc::DropoutCall c{};
    c.x = x_dev, c.residual = residual_dev, c.out = out_dev, c.x_bf16 = x_type == AGC_TYPE_BF16, c.out_bf16 = out_type == AGC_TYPE_BF16;
    c.ldx = ldx, c.ldr = ldr, c.ldo = ldo, c.rows = rows, c.cols = cols, c.seed = seed, c.step = step, c.site = site;
    c.drop48 = (uint64_t)std::llround(p * 281474976710656.0);
    c.scale = p < 1 ? (float)(1 / (1 - p)) : 0.0f;
    return launched(agc::launch_dropout(c, reinterpret_cast<hipStream_t>(hip_stream)), name);
}

int64_t agc_diff_attn_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int n_seqs, int heads, int kv_heads, int head_dim,
                                      int value_dim, int gradients)
{
    if (tokens_q < 0 || tokens_q > kMostTokens || tokens_k < 0 || tokens_k > kMostTokens || n_seqs < 1 || n_seqs > (1 << 20) || heads < 1 ||
        kv_heads < 1 || heads > kMostWidth || heads % kv_heads || head_dim < 1 || head_dim > 128 || value_dim < 1 || value_dim > 256)
        return 0;
    return agc::attn_workspace_bytes(tokens_q, tokens_k, n_seqs, heads, kv_heads, head_dim, value_dim, gradients != 0);
}

agc_status agc_diff_attn_forward(const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk, const void* v_dev, int64_t ldv,
                                 int64_t tokens_q, int64_t tokens_k, int heads, int kv_heads, int head_dim, int value_dim,
                                 const float* lambda_dev, const int32_t* q_end_dev, const int32_t* k_begin_dev,
                                 const int32_t* k_end_dev, int n_seqs, float scale, int causal, void* out_dev, int64_t ldo,
                                 float* lse_dev, void* workspace_dev, void* hip_stream)
{
    const char* const name = "agc_diff_attn_forward";
    agc::AttnCall c{};
    c.q = q_dev, c.k = k_dev, c.v = v_dev, c.ldq = ldq, c.ldk = ldk, c.ldv = ldv, c.tokens_q = tokens_q, c.tokens_k = tokens_k;
    c.heads = heads, c.kv_heads = kv_heads, c.d = head_dim, c.e = value_dim, c.lambda = lambda_dev;
    c.q_end = q_end_dev, c.k_begin = k_begin_dev, c.k_end = k_end_dev, c.n_seqs = n_seqs, c.causal = causal != 0, c.scale = scale;
    c.lse = lse_dev, c.workspace = static_cast<char*>(workspace_dev);
    const agc_status st = attn_arguments(name, c, false);
    if (st != AGC_OK) return st;
    if (!out_dev && tokens_q > 0) return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (ldo < (int64_t)heads * value_dim) return refuse(AGC_ESHAPE, std::string(name) + ": a row stride is smaller than the row");
    if (misaligned(out_dev, 2)) return refuse(AGC_EALIGN, std::string(name) + ": out needs 2-byte alignment");
    if (tokens_q == 0) return AGC_OK;
    c.out = out_dev, c.ldo = ldo;
    return launched(agc::launch_attn_forward(c, reinterpret_cast<hipStream_t>(hip_stream)), name);
}

agc_status agc_diff_attn_partial_gradients(const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk, const void* v_dev,
                                           int64_t ldv, int64_t tokens_q, int64_t tokens_k, int heads, int kv_heads,
                                           int head_dim, int value_dim, const float* lambda_dev, const int32_t* q_end_dev,
                                           const int32_t* k_end_dev, int n_seqs, float scale, int causal, const float* lse_dev,
                                           const void* dout_dev, int64_t lddout, const int64_t* part_end_host, int k_parts,
                                           void* dq_dev, int64_t lddq, void* dk_dev, int64_t lddk, void* dv_dev, int64_t lddv,
                                           float* G_lambda_dev, int64_t ldg, void* workspace_dev, void* hip_stream)
{
    const char* const name = "agc_diff_attn_partial_gradients";
    agc::AttnCall c{};
    c.q = q_dev, c.k = k_dev, c.v = v_dev, c.ldq = ldq, c.ldk = ldk, c.ldv = ldv, c.tokens_q = tokens_q, c.tokens_k = tokens_k;
    c.heads = heads, c.kv_heads = kv_heads, c.d = head_dim, c.e = value_dim, c.lambda = lambda_dev;
    c.q_end = q_end_dev, c.k_end = k_end_dev, c.n_seqs = n_seqs, c.causal = causal != 0, c.scale = scale;
    c.lse = const_cast<float*>(lse_dev), c.workspace = static_cast<char*>(workspace_dev);
    c.dout = dout_dev, c.lddout = lddout;
    agc_status st = attn_arguments(name, c, true);
    if (st != AGC_OK) return st;
    st = partitions(name, part_end_host, k_parts, tokens_q);
    if (st != AGC_OK) return st;
    if ((int64_t)heads * k_parts >= (1 << 21)) return refuse(AGC_ESHAPE, std::string(name) + ": heads * k_parts must be below 2^21");
    if (((!dout_dev || !lse_dev || !dq_dev) && tokens_q > 0) || ((!dk_dev || !dv_dev) && tokens_k > 0) || !G_lambda_dev)
        return refuse(AGC_EINVAL, std::string(name) + ": null pointer");
    if (lddout < (int64_t)heads * value_dim || lddq < (int64_t)2 * heads * head_dim || lddk < (int64_t)2 * kv_heads * head_dim ||
        lddv < (int64_t)kv_heads * value_dim || ldg < heads)
        return refuse(AGC_ESHAPE, std::string(name) + ": a row stride is smaller than the row");
    if (misaligned(dq_dev, 2) || misaligned(dk_dev, 2) || misaligned(dv_dev, 2) || misaligned(G_lambda_dev, 4))
        return refuse(AGC_EALIGN, std::string(name) + ": a pointer is not aligned to its elements");
    c.part_end = part_end_host, c.k_parts = k_parts, c.dq = dq_dev, c.dk = dk_dev, c.dv = dv_dev;
    c.lddq = lddq, c.lddk = lddk, c.lddv = lddv, c.G = G_lambda_dev, c.ldg = ldg;
    return launched(agc::launch_attn_gradients(c, reinterpret_cast<hipStream_t>(hip_stream)), name);
}

}  // extern "C"
