// C ABI of the operators round the coded step (include/agc.h): synchronous argument validation and launches on the
// caller's stream.  No context: messages go to agc_last_error(NULL).
#include <hip/hip_runtime.h>

#include <algorithm>
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

}  // extern "C"
