// Launch interface between the C ABI (agc_operators.cpp) and the kernels of the operators round the coded step:
// orthogonalised update, gated block, embedding, rotary positions, dropout, differential attention.  Every pointer is a device
// pointer unless it says host.
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

// ------------------------------------------------------------------ rotary positions
constexpr int kMostRotary = 8192;    // values of a head that turn
struct RotaryCall {
    const void* x;             // may be out
    void* out;
    int bf16;                  // both
    int64_t ldx, ldo, n;
    int heads, dim, rot;
    const void* positions;
    int wide_ids;              // 64-bit positions
    const uint64_t* turns;
    int interleaved, inverse;
    float amplitude;
};
hipError_t launch_rotary(const RotaryCall& c, hipStream_t stream);

// ------------------------------------------------------------------ dropout
struct DropoutCall {
    const void *x, *residual;  // residual may be null, either may be out
    void* out;
    int x_bf16, out_bf16;      // the residual is of out's type
    int64_t ldx, ldr, ldo, rows;
    int cols;
    uint64_t seed, step, drop48;   // p in units of 2^-48
    uint32_t site;
    float scale;               // 1 / (1 - p)
};
hipError_t launch_dropout(const DropoutCall& c, hipStream_t stream);

// ------------------------------------------------------------------ differential attention
constexpr float kLog2e = 1.44269504088896f;

struct AttnCall {
    const void *q, *k, *v;     // bfloat16
    int64_t ldq, ldk, ldv;
    int64_t tokens_q, tokens_k;
    int heads, kv_heads, d, e;
    const float* lambda;
    const int32_t *q_end, *k_begin, *k_end;   // k_begin may be null: a sequence's keys begin where the last one's end
    int n_seqs, causal;
    float scale;
    // forward
    void* out;
    int64_t ldo;
    float* lse;                // may be null; an input of the gradients
    // gradients
    const void* dout;
    int64_t lddout;
    const int64_t* part_end;   // host
    int k_parts;
    void *dq, *dk, *dv;
    int64_t lddq, lddk, lddv;
    float* G;
    int64_t ldg;
    char* workspace;
};
// D of the kernels that take heads of d and e values.  Operands of exactly D and 2 D are read where they lie, others if their
// chunks of 16 bytes can be; else they are copied to the workspace.
int attn_width(int d, int e);
int64_t attn_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int n_seqs, int heads, int kv_heads, int d, int e, int gradients);
hipError_t launch_attn_forward(const AttnCall& c, hipStream_t stream);
hipError_t launch_attn_gradients(const AttnCall& c, hipStream_t stream);

}  // namespace agc
