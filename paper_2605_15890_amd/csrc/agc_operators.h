// Launch interface between the C ABI (agc_operators.cpp) and the kernels of the operators round the coded step:
// orthogonalised update, gated block, embedding.  Every pointer is a device pointer unless it says host.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace agc {

// Leaves a message for agc_last_error(NULL) and returns the status (agc_api.cpp).
int note_failure(int status, const char* message);

constexpr int kMostMatrices = 256;   // of one update; their offsets travel as kernel arguments
constexpr int kMostParts = 256;      // partitions; their ends travel as kernel arguments

inline int64_t round_up(int64_t v, int64_t unit) { return (v + unit - 1) / unit * unit; }

// ------------------------------------------------------------------ orthogonalised update
struct MuonCall {
    float* beta;
    float* m1;
    const float* ghat;
    uint16_t* beta_bf16;               // may be null
    int64_t offset[kMostMatrices];     // of each matrix in the vectors, in elements
    int n_mats, rows, cols, nesterov, steps;
    float momentum, keep, rate;        // beta <- keep * beta - rate * X
    char* workspace;
};
int64_t muon_workspace_bytes(int rows, int cols, int n_mats);
hipError_t launch_muon_update(const MuonCall& c, hipStream_t stream);

// ------------------------------------------------------------------ gated block
struct GatedCall {
    const void *x, *wg, *wu;
    int64_t ldx, ldw;
    int64_t tokens;
    int d_in, d_ff, gelu;
    // forward
    void* h;
    int64_t ldh;
    // gradients
    const void* dh;
    int64_t lddh;
    const int64_t* part_end;   // host
    int k_parts;
    void* dx;                  // may be null
    int64_t lddx;
    float *g_gate, *g_up;
    int64_t ldg;
    char* workspace;
};
int64_t gated_workspace_bytes(int64_t tokens, int d_in, int d_ff, int k_parts);   // k_parts 0: forward alone
hipError_t launch_gated_forward(const GatedCall& c, hipStream_t stream);
hipError_t launch_gated_gradients(const GatedCall& c, hipStream_t stream);

// ------------------------------------------------------------------ embedding
struct EmbedCall {
    const void* tokens;
    int wide_ids;              // 64-bit ids
    int64_t n, vocab;
    int dim;
    float scale;
    int value_bf16;            // out, or dout
    int64_t ld;                // its row stride
    // forward
    const void* table;
    int table_bf16;
    void* out;
    // gradients
    const void* dout;
    const int64_t* part_end;   // host
    int k_parts;
    float* G;
    int64_t ldg;
    char* workspace;
};
int64_t embed_workspace_bytes(int64_t n, int64_t vocab, int dim, int k_parts);
hipError_t launch_embed_forward(const EmbedCall& c, hipStream_t stream);
hipError_t launch_embed_gradients(const EmbedCall& c, hipStream_t stream);

}  // namespace agc
