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

}  // extern "C"
