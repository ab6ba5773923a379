/*
 * agc.h -- C ABI of the MI355X (gfx950) hot path of communication-efficient approximate
 * gradient coding: encode -> stochastic quantize + bit-pack -> masked dequantize + decode.
 *
 * Symbols (the paper's own letters in brackets): n workers [k], k data partitions [n],
 * d gradient coordinates [l], code matrix B [A] of shape n x k, partial gradients G
 * (k x d, row j = g_j), bit-width b_i [z_i], magnitude levels L_i = 2^(b_i-1)-1 [s_i],
 * decode weights w_i, arrival indicators mask_i [I_i], straggling probabilities p_i.
 *
 * General conventions
 *   - every entry point returns agc_status (0 = ok, negative = error); nothing throws or
 *     aborts; agc_last_error() gives a message for the last failure on a context;
 *   - "host" pointers are ordinary process memory, "device" pointers are HIP device memory
 *     of the GPU that was current when the context was created;
 *   - the caller owns every buffer it passes; the library owns only the workspace and the tables it
 *     allocates in agc_create(), agc_set_code() and agc_set_layers() and allocates nothing in the
 *     per-step calls;
 *   - per-step calls validate their arguments synchronously, enqueue kernels on the given
 *     HIP stream (a hipStream_t passed as void*, NULL = the default stream) and return
 *     without waiting and without any host<->device copy: the small host arrays (bits, w,
 *     mask, code pointers) travel as kernel arguments; they enqueue nothing but kernel launches
 *     (no allocation, fill, copy or wait), so a caller may record them into a HIP graph: a
 *     replay repeats the recorded call, seed and step counter included (not while the event
 *     timing of agc_debug.h is switched on);
 *   - NaN or infinity in G is outside the contract (no check on the hot path);
 *   - a context's workspace and tables are shared by all its calls: calls on one context must be
 *     ordered (one stream, or events between streams); concurrent streams need one context each.
 *
 * Arithmetic fixed by this library (the paper leaves these open; the CPU oracle in
 * oracle/ takes the same readings):
 *   encode     binary32; first stored entry of a row: rounded product; each further entry:
 *              one fused multiply-add, in stored order;
 *   scale      AGC_SCALE_MAXABS: max_m |f_i[m]|;  AGC_SCALE_L2: (float)sqrt(S) with S the
 *              binary64 sum of squares in the fixed tree described at agc_encode_quantize;
 *   draws      Philox4x32-10, key = seed; 16-bit primary field, 32-bit secondary word
 *              (see agc_encode_quantize);
 *   payload    per worker a little-endian bit stream, code m in bits [m*b, (m+1)*b),
 *              zero-padded to whole groups of 128 codes (agc_code_bytes);
 *   decode     binary32, arrived workers in ascending order, one fused multiply-add each;
 *   bucket-wise scales (agc_opts.bucket = 256; Sec. II-B names the extension, the arithmetic is
 *              this library's): bucket u = coordinates [256u, 256u+256) below d; scale_iu = largest
 *              magnitude of f_i in the bucket, or (float)sqrt of the bucket's binary64 sum of squares
 *              (the two lowest levels of the tree); multiplier = L_i*2^16 / scale_iu (2^15 / scale_iu
 *              for one bit) as ONE correctly rounded binary32 division, 0 for an empty or overflowing
 *              bucket; rounding rule, draws, codes and payload as above; decode weight =
 *              (float)((double)w_i / L_i) * scale_iu, one binary32 product; scales_dev is n x
 *              ceil(d/256), row-major.
 */
#ifndef AGC_H
#define AGC_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define AGC_MAX_WORKERS 256   /* n <= 256: per-worker arguments travel in the kernel argument block */
#define AGC_MAX_BITS 16
#define AGC_MAX_LAYERS 256    /* layer-wise scales: at most this many layers; matrices of one agc_muon_update */
#define AGC_MAX_MATRIX 32768  /* sides of the matrices of agc_muon_update */

typedef struct agc_ctx agc_ctx; /* opaque; owns device workspace and a copy of B */

typedef enum {
    AGC_OK = 0,
    AGC_EINVAL = -1, /* null pointer, non-positive size, unknown option value */
    AGC_ESHAPE = -2, /* n, k, d out of range; CSR malformed; column index out of range */
    AGC_EBITS = -3,  /* bit-width outside [2,16] (or 1 without allow_1bit) */
    AGC_EALIGN = -4, /* G or g_hat not 16-byte aligned, ldg not a multiple of 4, stream not 16-byte aligned */
    AGC_ENOMEM = -5, /* workspace allocation failed */
    AGC_EHIP = -6,   /* a HIP call failed (message in agc_last_error) */
    AGC_ESTATE = -7  /* agc_set_code() has not been called */
} agc_status;

typedef enum {
    AGC_SCALE_L2 = 0,    /* Euclidean norm: the quantizer of Sec. II-B as printed */
    AGC_SCALE_MAXABS = 1 /* largest magnitude: finer grid, still unbiased (any scale >= max|f| is) */
} agc_scale_mode;

typedef struct {
    int scale_mode;    /* agc_scale_mode */
    int allow_1bit;    /* non-zero: accept b_i = 1 (two-point grid {-scale,+scale}; outside the paper, which needs b >= 2) */
    int force_generic; /* testing hook (see agc_debug.h): non-zero = every code takes the generic gather path */
    int bucket;        /* 0: one scale per coded vector (the paper's quantizer).  256: one scale per
                          256-coordinate bucket (Sec. II-B names the bucket-wise extension): the
                          scales array becomes n x ceil(d/256) and the worker side reads G once */
    int unfused_step;  /* non-zero: agc_step runs agc_encode_quantize then agc_decode as two passes;
                          zero: one fused pass (same results bit for bit, see agc_step) */
    int reserved[3];   /* must be zero */
} agc_opts;

/* --------------------------------------------------------------------------------------
 * Context
 * ------------------------------------------------------------------------------------ */
/* Creates a context for n workers, k partitions, d coordinates on the current device and
 * allocates its workspace (scale partials: 4 bytes * 256 * n for the max-abs scale, whatever d is;
 * 8 bytes * n * ceil(d/1024) for the Euclidean one; none with bucket-wise scales; a few n-entry
 * tables).  agc_set_code() takes more with the Euclidean scale of a long vector.
 * opts may be NULL (AGC_SCALE_MAXABS, no 1-bit).  Limits: 1 <= n <= AGC_MAX_WORKERS,
 * 1 <= k <= 65536, 1 <= d <= 2^33. */
agc_status agc_create(agc_ctx **out, int n_workers, int k_parts, int64_t d, const agc_opts *opts);
void agc_destroy(agc_ctx *ctx);

/* Sets the code matrix B (Sec. II-A: f_i = sum_j a_ij g_j) as CSR rows over host arrays
 * row_ptr[n+1], col[nnz], val[nnz]; the arrays are copied (one synchronous upload).  The
 * order of the stored entries inside a row IS the summation order of the encode.  When
 * n == k and every row i stores exactly s <= 8 entries with columns (i+u) mod k, u=0..s-1 in
 * that order (cyclic replication), the kernels take a register sliding-window path that
 * reads every element of G once per pass; when every row is a run of at most 8 consecutive
 * ascending columns whose two ends never decrease from one worker to the next (the shape
 * agc_build_code produces), they take the same kind of path without the wrap-around; any other B
 * takes the generic gather path, which re-reads shared rows through the caches.  All three give
 * identical bits (agc_code_path tells which one a context runs).
 * With one Euclidean scale per vector and sizes at which it is faster, the call also takes the workspace for reading G
 * once instead of twice: for every 256 coordinates 1 KB of signs per 32 workers and 8 bytes for each of up to 32 * n, at
 * most 1118, coded values (0.97 GB at 64 x 25.6 M).  It is taken beside a G of at most half the device's memory, within an
 * eighth of what hipMemGetInfo reports as free (what a caching allocator holds is not), and whatever the bit-widths of
 * the steps will be; layers give it back.  Without it two reads are made, with the same results
 * (agc_debug_sketch_last tells which).  Likewise with one largest-magnitude scale per vector, G of 4 GB and more and up to 128
 * workers, where 8 bytes are held for each of up to 32 * k coded values (1.9 GB at 64 x 25.6 M). */
agc_status agc_set_code(agc_ctx *ctx, const int32_t *row_ptr, const int32_t *col, const float *val);

/* Layer-wise scales (Sec. II-B: the quantizer "at layer-wise or bucket-wise granularity"): the d
 * coordinates are cut into n_layers consecutive layers, layer l = [layer_end[l-1], layer_end[l])
 * with layer_end[-1] = 0, and every worker gets one scale per layer, of the context's kind:
 * scale_il = max over the layer of |f_i[m]|, or the Euclidean norm of the layer with the AGC_SCALE_L2
 * tree started anew at the layer's first coordinate (blocks, segments, groups and supergroups are
 * counted from there).  Everything else is the per-vector arithmetic with
 * the layer's scale in place of the vector's: inv16_il = (float)(L_i * 2^16 / scale_il), decode
 * weight (float)(((double)w_i * scale_il) / L_i); draws and payload layout do not change.  With
 * layers set, scales_dev of the per-step calls holds n x n_layers floats, [worker][layer]
 * (agc_scales_per_worker), and agc_encode_quantize, agc_decode, agc_decode2 and agc_step (both
 * forms) work on them; the worker side reads G twice.
 *   layer_end  host, n_layers ends, strictly ascending, all but the last multiples of 256 (a
 *              256-coordinate block lies in one layer), the last equal to d
 * 1 <= n_layers <= AGC_MAX_LAYERS; n_layers == 0 returns to one scale per vector.  Needs a context
 * with bucket == 0 (AGC_EINVAL otherwise).  Synchronous (waits for the device,
 * replaces small tables); not available in agc_decode_noalloc, which has no context. */
agc_status agc_set_layers(agc_ctx *ctx, int n_layers, const int64_t *layer_end);

/* 0 = generic gather path; 1..8 = cyclic-band path with replication s; 102, 104, 108 = monotone-
 * interval path (every row a run of at most 2, 4, 8 consecutive ascending columns whose ends never
 * decrease from one worker to the next - the shape agc_build_code produces); < 0 = no code set.
 * All paths give identical bits; the last two read every element of G once per pass. */
int agc_code_path(const agc_ctx *ctx);

/* Bytes of one worker's packed stream: ceil(d/128) * 16 * bits (Sec. II-B: the payload is
 * the scale plus d codes of b bits; the padding is this library's). */
int64_t agc_code_bytes(int64_t d, int bits);

/* Scales per worker in scales_dev: 1, ceil(d/256) with bucket-wise scales, n_layers with layer-wise scales. */
int64_t agc_scales_per_worker(const agc_ctx *ctx);

const char *agc_last_error(const agc_ctx *ctx);

/* --------------------------------------------------------------------------------------
 * Hot path
 * ------------------------------------------------------------------------------------ */
/*
 * Worker side (Sec. II-A encoded message, Sec. II-B quantizer): for every worker i
 *   f_i      = sum_j B[i,j] G[j,:]                      (never written to memory)
 *   scale_i  per scale_mode over all d coordinates
 *   code     = sign << (b_i-1) | level,  level = min(floor(T/2^16) + up, L_i),
 *              T = |f| * inv16_i (binary32), inv16_i = (float)(L_i * 2^16 / scale_i) (0 when
 *              scale_i is 0 or the quotient overflows), up = U < frac(T/2^16) with the
 *              48-bit uniform U = (u16 + r2 / 2^32) / 2^16:
 *                u16 = 16-bit field (i&1)*4 + (m&3) of Philox4x32-10(key = seed,
 *                      counter = (m>>2, i>>1, step lo, step hi)), fields counted from the
 *                      low half of output word 0;
 *                r2  = word m&3 of Philox4x32-10(key = seed, counter = (m>>2, 2^31 | i,
 *                      step lo, step hi)), consulted only when u16 ties;
 *              b_i = 1 (allow_1bit): T = max(fma(f, 2^15/scale_i, 2^15), 0), code = level in {0,1};
 *   stream_i = little-endian bit stream of the d codes.
 * All n workers are encoded: a straggler still computes, its message is merely late; the
 * arrival mask is an argument of the decode only.
 *
 * AGC_SCALE_L2 tree (binary64): 256-coordinate blocks; slot l of a block owns coordinates
 * 4l..4l+3 and holds (x0^2+x1^2)+(x2^2+x3^2); exchange-add over slots at distances
 * 1,2,4,8,16,32; 4 blocks are summed in order into a segment, 64 segments in order into a
 * group, 64 groups in order into a supergroup, supergroups in order into S (every
 * sequential sum starts from 0.0).
 *
 *   G_dev      device, k x d binary32, row-major with row stride ldg elements (ldg >= d,
 *              ldg % 4 == 0, base 16-byte aligned); read-only.  The kernels load whole 16-byte
 *              groups of four coordinates: the allocation must hold (k-1)*ldg + 4*ceil(d/4)
 *              floats (always true when every row owns its full stride of ldg floats); the up to
 *              three floats past d in a row are read and ignored
 *   bits_host  host, n bytes
 *   codes_dev  host array of n device pointers; stream i has agc_code_bytes(d, b_i) bytes,
 *              16-byte aligned; fully overwritten, padding included
 *   scales_dev device, n floats; overwritten
 */
agc_status agc_encode_quantize(agc_ctx *ctx, const float *G_dev, int64_t ldg,
                               const uint8_t *bits_host, uint64_t seed, uint64_t step,
                               void *const *codes_dev, float *scales_dev, void *hip_stream);

/*
 * Master side (Sec. II-A aggregation): g_hat[m] = sum over arrived i, ascending, of
 * coef_i * v_i[m] folded with one binary32 fused multiply-add each from 0, where
 * coef_i = (float)(((double)w_i * scale_i) / L_i) and v = +-level (b_i >= 2) or +-1 (b_i = 1).
 *
 *   codes_dev, scales_dev, bits_host   as written by agc_encode_quantize (read-only)
 *   w_host     host, n floats: decode weights
 *   mask_host  host, n bytes: 1 = worker arrived, 0 = straggler (its stream is not read)
 *   ghat_dev   device, d floats, 16-byte aligned; overwritten
 */
agc_status agc_decode(agc_ctx *ctx, void *const *codes_dev, const float *scales_dev,
                      const uint8_t *bits_host, const float *w_host, const uint8_t *mask_host,
                      float *ghat_dev, void *hip_stream);

/*
 * Two-track decoding (Sec. V, extension to adaptive optimizers; Appendix F): the master applies
 * two decoding vectors to the same received codes.  g_hat is formed with w exactly as in
 * agc_decode; g_hat2 is formed in the same way with v in place of w (same order, same
 * rounding), from the same single read of the streams.
 *
 *   v_host     host, n floats: second-moment decoding vector (agc_second_moment_decoder)
 *   ghat2_dev  device, d floats, 16-byte aligned, distinct from ghat_dev; overwritten
 * Everything else as in agc_decode.
 */
agc_status agc_decode2(agc_ctx *ctx, void *const *codes_dev, const float *scales_dev,
                       const uint8_t *bits_host, const float *w_host, const float *v_host,
                       const uint8_t *mask_host, float *ghat_dev, float *ghat2_dev, void *hip_stream);

/*
 * agc_decode for callers that cannot allocate device memory and therefore cannot hold a context:
 * code under HIP graph capture, tight serving loops on the master, harnesses that forbid
 * hipMalloc.  No context: n_workers, d and bucket (0, or 256 for bucket-wise scales) are passed
 * directly; a one-bit stream is always accepted.  Same kernels, same arithmetic and the same bits
 * in g_hat as agc_decode.  The small tables the decode kernel reads (one record and some 24 stream
 * pieces per arrived worker) live in a fixed device array of 106 KB inside the library,
 * which every GPU the library runs on holds until the process ends; hence n_workers <= 256
 * (AGC_ESHAPE with a message otherwise).  The call itself and everything below it performs no
 * hipMalloc/hipFree; the first call on a device looks the array's address up once (make that
 * call before starting a graph capture).  All calls on one GPU share the array: calls that
 * overlap on one GPU (different streams without an event between them, or different threads)
 * race on it and must be serialised by the caller.  Errors are reported through
 * agc_last_error(NULL).
 */
agc_status agc_decode_noalloc(int n_workers, int64_t d, int bucket, void *const *codes_dev,
                              const float *scales_dev, const uint8_t *bits_host, const float *w_host,
                              const uint8_t *mask_host, float *ghat_dev, void *hip_stream);

/* One whole pass, with the outputs of agc_encode_quantize followed by agc_decode on the same
 * stream (codes, scales, g_hat; identical bits).  By default the quantize kernel also forms
 * g_hat from the codes it has just produced, in the order and arithmetic of agc_decode, so the
 * payload is written but not read back; agc_opts.unfused_step selects the two-pass form. */
agc_status agc_step(agc_ctx *ctx, const float *G_dev, int64_t ldg, const uint8_t *bits_host,
                    const float *w_host, const uint8_t *mask_host, uint64_t seed, uint64_t step,
                    void *const *codes_dev, float *scales_dev, float *ghat_dev, void *hip_stream);

/* --------------------------------------------------------------------------------------
 * End-to-end least-squares loop (the producer of G and the consumer of g_hat)
 * ------------------------------------------------------------------------------------ */
/* Partial gradients of the least-squares loss 0.5 * ||X_p beta - y_p||^2 of k equal, contiguous
 * data partitions (Sec. II-A: g_j = grad L(D_j, beta)):  G[p,:] = X_p^T (X_p beta - y_p).
 *   X_dev     device, n_rows x n_feat bfloat16 (upper halves of binary32), row-major, 16-byte aligned
 *   y_dev     device, n_rows floats;  beta_dev  device, n_feat floats
 *   G_dev     device, k_parts x n_feat floats with row stride ldg; overwritten
 *   resid_dev device, n_rows floats; receives X beta - y (its squared norm is twice the loss)
 *   workspace_dev device, agc_ls_workspace_floats(...) floats, 16-byte aligned; scratch
 * Products are exact (beta enters as an exact three-way bfloat16 split on the matrix cores),
 * accumulation is binary32 in a fixed order, so the result is reproducible run to run.
 * Shapes: n_feat a multiple of 128 and <= 8192; n_rows a multiple of 16 * k_parts (AGC_ESHAPE). */
int64_t agc_ls_workspace_floats(int64_t n_rows, int n_feat, int k_parts);
agc_status agc_ls_partial_gradients(const void *X_dev, int64_t n_rows, int n_feat, const float *y_dev,
                                    const float *beta_dev, int k_parts, float *G_dev, int64_t ldg,
                                    float *resid_dev, float *workspace_dev, void *hip_stream);
/* Gradient-descent update of Sec. II-A: beta <- beta - lr * g_hat (one fused multiply-add per
 * coordinate), device pointers, d floats each. */
agc_status agc_gd_update(float *beta_dev, const float *ghat_dev, float lr, int64_t d, void *hip_stream);
/* Adam step t (t >= 1) that consumes the two tracks of agc_decode2 (Sec. V; update ratio of
 * Appendix F): the first-moment average takes g_hat, the second-moment average takes the
 * square of g_hat2; binary32 throughout:
 *   m1 <- beta1*m1 + (1-beta1)*g_hat;  m2 <- beta2*m2 + (1-beta2)*g_hat2^2;
 *   beta <- beta - lr * (m1/(1-beta1^t)) / (sqrt(m2/(1-beta2^t)) + eps).
 * The bias corrections and eps are the customary ones of the optimizer; the paper prints only
 * the ratio.  All pointers device, d floats each; beta, m1, m2 updated in place. */
agc_status agc_adam_update(float *beta_dev, float *m1_dev, float *m2_dev, const float *ghat_dev,
                           const float *ghat2_dev, float lr, float beta1, float beta2, float eps,
                           int64_t t, int64_t d, void *hip_stream);

/* --------------------------------------------------------------------------------------
 * Token models: two producers of rows of G and a consumer of g_hat
 * ------------------------------------------------------------------------------------ */
typedef enum {
    AGC_TYPE_F32 = 0,
    AGC_TYPE_BF16 = 1 /* upper halves of binary32 */
} agc_type;

/* Embedding with scaling:  out[t,:] = scale * E[id_t,:], one binary32 product a value, rounded once to out's type.  An id
 * outside [0, vocab) is an empty place (padding): its row of out is zeros.
 *   table_dev  device, vocab x dim of table_type, row-major (its section of the parameter vector, for instance)
 *   tokens_dev device, n_tokens ids of token_bytes = 4 or 8 bytes (signed)
 *   out_dev    device, n_tokens x dim of out_type, row stride ldo elements; overwritten
 * 0 <= n_tokens <= 2^26, 1 <= dim <= 65536, 1 <= vocab < 2^31; any alignment of the rows. */
agc_status agc_embed_forward(const void *table_dev, int table_type, int64_t vocab, int dim, const void *tokens_dev,
                             int token_bytes, int64_t n_tokens, float scale, void *out_dev, int out_type, int64_t ldo,
                             void *hip_stream);
/* Its partial gradients (Sec. II-A): for every data partition p (a run of tokens) and every id v
 *   G[p, v * dim + c] = scale * sum of dout[t, c] over the tokens t of p with id_t = v,
 * binary32, in a fixed order (the result is reproducible run to run); rows of ids that do not occur are zeros, empty
 * places count for nothing, whatever their dout holds.
 *   dout_dev   device, n_tokens x dim of dout_type, row stride lddout
 *   part_end_host  host, k_parts ends of the partitions in tokens, not descending, the last n_tokens
 *   G_dev      device, where row 0 of G holds the gradient of the table; row p lies p * ldg floats on; overwritten
 *   workspace_dev  device, agc_embed_workspace_bytes(...) bytes, 256-byte aligned; scratch
 * 1 <= k_parts <= 256, k_parts * vocab < 2^31; ldg >= vocab * dim. */
int64_t agc_embed_workspace_bytes(int64_t n_tokens, int64_t vocab, int dim, int k_parts);
agc_status agc_embed_partial_gradients(const void *dout_dev, int dout_type, int64_t lddout, const void *tokens_dev,
                                       int token_bytes, int64_t n_tokens, const int64_t *part_end_host, int k_parts,
                                       int64_t vocab, int dim, float scale, float *G_dev, int64_t ldg, void *workspace_dev,
                                       void *hip_stream);

typedef enum {
    AGC_ACT_SILU = 0, /* a / (1 + exp(-a)) */
    AGC_ACT_GELU = 1  /* a * Phi(a), by erf */
} agc_activation;

/* Gate of a gated feed-forward block in bfloat16:  h = act(x Wg^T) * (x Wu^T), sums and activation in binary32, h rounded
 * once.  The block's output projection, a product of h with a third matrix, is the caller's.
 *   x_dev      device, n_tokens x d_in, row stride ldx elements
 *   w_gate_dev, w_up_dev  device, d_ff x d_in, row stride ldw (their sections of the parameter vector, rounded to
 *              bfloat16, for instance)
 *   h_dev      device, n_tokens x d_ff, row stride ldh; overwritten
 *   workspace_dev  device, agc_gated_workspace_bytes(n_tokens, d_in, d_ff, 0) bytes, 256-byte aligned; scratch
 * Any alignment of the operands and any sizes: 0 <= n_tokens <= 2^26, 1 <= d_in, d_ff <= 65536.  Up to 64 tokens take
 * a form that is bound by the one read of the weights and needs no workspace (256 bytes are asked for); rows that are
 * not whole multiples of 128 bytes, 16-byte aligned, are copied to the workspace first when there are more. */
int64_t agc_gated_workspace_bytes(int64_t n_tokens, int d_in, int d_ff, int k_parts);
agc_status agc_gated_forward(const void *x_dev, int64_t ldx, const void *w_gate_dev, const void *w_up_dev, int64_t ldw,
                             int64_t n_tokens, int d_in, int d_ff, int act, void *h_dev, int64_t ldh, void *workspace_dev,
                             void *hip_stream);
/* Its partial gradients (Sec. II-A: g_j = grad L(D_j, beta)): with a = x Wg^T, u = x Wu^T, which are formed again,
 *   da = dh u act'(a),  du = dh act(a),  dx = da Wg + du Wu,
 * and for every data partition p (a run of tokens)  G_gate[p] = da_p^T x_p,  G_up[p] = du_p^T x_p, binary32.
 *   dh_dev     device, n_tokens x d_ff bfloat16, row stride lddh
 *   part_end_host  host, k_parts ends of the partitions in tokens, not descending, the last n_tokens; partition p is
 *              [part_end[p-1], part_end[p]) and may be empty: its gradients are zeros
 *   dx_dev     device, n_tokens x d_in bfloat16, row stride lddx; overwritten.  NULL: not wanted
 *   G_gate_dev, G_up_dev  device, where row 0 of G holds the d_ff x d_in gradients of Wg and of Wu (row-major);
 *              row p lies p * ldg floats on; overwritten
 *   workspace_dev  device, agc_gated_workspace_bytes(n_tokens, d_in, d_ff, k_parts) bytes, 256-byte aligned
 * da and du enter dx with 16 bits, so that dx is rounded once, and G with all 24 bits of binary32, whatever the sizes of
 * the other operands; sums are binary32 in a fixed order.  da, du and G of 2^105 and more become infinite.  NaN or infinity
 * in a token reaches its own row of dx and its own partition's gradients alone.
 * 1 <= k_parts <= 256; ldg >= d_in * d_ff. */
agc_status agc_gated_partial_gradients(const void *x_dev, int64_t ldx, const void *w_gate_dev, const void *w_up_dev,
                                       int64_t ldw, const void *dh_dev, int64_t lddh, int64_t n_tokens,
                                       const int64_t *part_end_host, int k_parts, int d_in, int d_ff, int act, void *dx_dev,
                                       int64_t lddx, float *G_gate_dev, float *G_up_dev, int64_t ldg, void *workspace_dev,
                                       void *hip_stream);

/* Rotation of queries and keys by their positions.  The first rot_dim values of each head are rot_dim / 2 pairs, values i and
 * i + rot_dim / 2 (AGC_ROTARY_HALF) or 2 i and 2 i + 1 (AGC_ROTARY_INTERLEAVED); pair i of token t becomes
 *   amplitude * (a cos - b sin, a sin + b cos)  at the angle  2 pi position_t turns_i / 2^64
 * (-angle with inverse, which is the gradient: dx = agc_rotary_apply(dout, inverse)).  Values behind them are copied.  Angles,
 * sines and products are binary32 or better at any position, a result is rounded once.
 *   x_dev, out_dev  device, n_tokens x (heads * head_dim) of one type, row strides ldx and ldo elements, any alignment; queries
 *              and keys that lie side by side in a row are one call.  out may be x, with the same stride, and not overlap it otherwise
 *   positions_dev  device, n_tokens positions of position_bytes = 4 or 8 bytes (signed)
 *   turns_dev  device, rot_dim / 2 numbers: a position's share of a whole turn in units of 2^-64
 * 0 <= n_tokens <= 2^26, heads * head_dim <= 65536, 2 <= rot_dim <= head_dim and 8192, rot_dim even. */
typedef enum { AGC_ROTARY_HALF = 0, AGC_ROTARY_INTERLEAVED = 1 } agc_rotary_layout;
agc_status agc_rotary_apply(const void* x_dev, int type, int64_t ldx, int64_t n_tokens, int heads, int head_dim, int rot_dim,
                            const void* positions_dev, int position_bytes, const uint64_t* turns_dev, int layout,
                            float amplitude, int inverse, void* out_dev, int64_t ldo, void* hip_stream);
/* Its table (host): turns_out[i] = 2^64 f_i / (2 pi), rot_dim / 2 numbers, f_i = base^(-2 i / rot_dim), and for contexts `factor`
 * times as long as original_len, the one that a model was trained for,
 *   AGC_ROTARY_LINEAR    f_i / factor
 *   AGC_ROTARY_BY_PARTS  f_i / factor where the pair turns once or less over original_len, f_i where it turns 32 times or more,
 *                        a linear ramp over the pairs between, which begins with the first pair at the earliest and leaves f_i
 *                        where it begins;  *amplitude_out = 0.1 ln(factor) + 1 (else 1). */
typedef enum { AGC_ROTARY_PLAIN = 0, AGC_ROTARY_LINEAR = 1, AGC_ROTARY_BY_PARTS = 2 } agc_rotary_scaling;
agc_status agc_rotary_frequencies(int rot_dim, double base, int scaling, double factor, double original_len,
                                  uint64_t* turns_out, double* amplitude_out);

/* Differential attention in bfloat16: for every query head h and its key head h / (heads / kv_heads)
 *   out = (softmax(scale q1 k1^T) - lambda_h softmax(scale q2 k2^T)) v
 * over the keys of the query's own sequence, with `causal` over those that lie no later, the ends of both runs taken as the
 * same place: of Lq queries and Lk keys, query i sees the keys 0 .. i + Lk - Lq.  A query that sees none gets zeros.
 *   q_dev      device, tokens_q x (heads * 2 * head_dim): both maps' queries of a head lie side by side
 *   k_dev, v_dev  device, tokens_k x (kv_heads * 2 * head_dim) and tokens_k x (kv_heads * value_dim)
 *              row strides ldq, ldk, ldv elements.  Where head_dim and value_dim are D and 2 D, D = 32, 64 or 128, rows must begin at
 *              multiples of 16 bytes (AGC_EALIGN).  Other widths may begin anywhere, the next D holds both: multiples of 8
 *              whose rows all begin at multiples of 16 bytes are read where they lie too, the rest is copied to the workspace
 *   lambda_dev device, heads floats
 *   q_end_dev, k_end_dev  device, n_seqs ends of the sequences in queries and in keys, not descending; sequence s has the
 *              queries from q_end[s-1] (0 for the first) to q_end[s], and the keys alike.  Either may be empty.  Rows of out
 *              behind the last sequence are left as they were.  Ends beyond the tensors count as their ends
 *   k_begin_dev  device, n_seqs first keys, or NULL: the keys of sequence s are k_begin[s] .. k_end[s] - 1 instead, anywhere in
 *              k and v, which are then a cache with room behind each sequence, or share keys
 *   out_dev    device, tokens_q x (heads * value_dim), row stride ldo; overwritten
 *   lse_dev    device, (2 * heads) x tokens_q floats, or NULL: receives log2 of the sum over keys of 2^(scale q_m k_m log2 e) of
 *              map m of head h in row 2 h + m, -infinity without keys; what the gradients take
 *   workspace_dev  device, agc_diff_attn_workspace_bytes(..., 0) bytes, 256-byte aligned; scratch, which calls that may run at
 *              the same time, captured ones among them, do not share
 * scale is 0 or more, and scale * log2(e) finite in binary32; scores, scale q_m k_m, are up to 2^29.  Scores, maxima, sums and out
 * are held in binary32; the maps enter their product with v as bfloat16, out is rounded once.  The order of the sums is fixed.
 * NaN or infinity in a sequence reaches that sequence's results alone.  out and lse must not overlap what is read.
 * Few queries have their keys split among workgroups, into as many parts as keys of the sequences' mean length, tokens_k / n_seqs,
 * need: a call whose sequences differ many times over takes what its longest one takes with those parts.
 * Row strides of q, k, v up to 2^24, 0 <= tokens_q, tokens_k <= 2^26, tokens_q * heads and tokens_k * kv_heads up to 2^30 (2^29
 * where head_dim is above 64 or value_dim above 128), 1 <= n_seqs <= 2^20, n_seqs * kv_heads up to 2^21, heads a multiple of
 * kv_heads, 1 <= head_dim <= 128, 1 <= value_dim <= 256. */
int64_t agc_diff_attn_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int n_seqs, int heads, int kv_heads, int head_dim,
                                      int value_dim, int gradients);
agc_status agc_diff_attn_forward(const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk, const void* v_dev, int64_t ldv,
                                 int64_t tokens_q, int64_t tokens_k, int heads, int kv_heads, int head_dim, int value_dim,
                                 const float* lambda_dev, const int32_t* q_end_dev, const int32_t* k_begin_dev,
                                 const int32_t* k_end_dev, int n_seqs, float scale, int causal, void* out_dev, int64_t ldo,
                                 float* lse_dev, void* workspace_dev, void* hip_stream);
/* Its gradients, and the partial gradients of lambda (Sec. II-A): with lse as the forward pass left it,
 *   dP = dout v^T,  D_m = sum over keys of P_m dP,  dS_1 = P_1 (dP - D_1),  dS_2 = -lambda P_2 (dP - D_2),
 *   dq_m = scale dS_m k_m,  dk_m = scale dS_m^T q_m,  dv = (P_1 - lambda P_2)^T dout, summed over the heads that share them,
 * and for every data partition p (a run of queries)  G_lambda[p, h] = - sum over its queries of D_2, binary32.
 *   dout_dev   device, tokens_q x (heads * value_dim), row stride lddout up to 2^24, aligned as v
 *   part_end_host  host, k_parts ends of the partitions in queries, not descending, the last tokens_q
 *   dq_dev, dk_dev, dv_dev  device, as q, k and v, row strides lddq, lddk, lddv, any alignment; overwritten but for rows behind
 *              the last sequence, which are left as they were
 *   G_lambda_dev  device, where row 0 of G holds the gradients of lambda; row p lies p * ldg floats on; overwritten.  No result
 *              may overlap what is read
 *   workspace_dev  device, agc_diff_attn_workspace_bytes(..., 1) bytes, 256-byte aligned (enough for the forward pass too)
 * The maps and dS enter the products with 16 bits, so that results are rounded once; sums are binary32 in a fixed order.  Maps
 * formed again from lse are off by up to 2^-24 |lse| of themselves (2^-17 at 128).
 * 1 <= k_parts <= 256, heads * k_parts below 2^21. */
agc_status agc_diff_attn_partial_gradients(const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk, const void* v_dev,
                                           int64_t ldv, int64_t tokens_q, int64_t tokens_k, int heads, int kv_heads,
                                           int head_dim, int value_dim, const float* lambda_dev, const int32_t* q_end_dev,
                                           const int32_t* k_end_dev, int n_seqs, float scale, int causal, const float* lse_dev,
                                           const void* dout_dev, int64_t lddout, const int64_t* part_end_host, int k_parts,
                                           void* dq_dev, int64_t lddq, void* dk_dev, int64_t lddk, void* dv_dev, int64_t lddv,
                                           float* G_lambda_dev, int64_t ldg, void* workspace_dev, void* hip_stream);

/* Dropout into a residual:  out = residual + (U >= p ? x / (1 - p) : 0), one binary32 product and sum, rounded once to out's
 * type.  The mask is not stored: it follows from (seed, step, site, row, column), whatever the types and strides, so the
 * gradient is the same call on dout without a residual.  U = (u16 + r2 / 2^32) / 2^16 with
 *   u16 = 16-bit field c&7 of Philox4x32-10(key = seed, counter = (site << 16 | c>>3, 2^30 | row, step lo, step hi)), fields
 *         counted from the low half of output word 0;
 *   r2  = word c&3 of Philox4x32-10(key = seed, counter = (site << 16 | c>>2, 2^31 | 2^30 | row, step lo, step hi)),
 * counters that agc_encode_quantize does not use: one seed and step serve both, and 65536 sites of a model.  p counts in
 * units of 2^-48.  A dropped x leaves no trace, NaN included.
 *   x_dev      device, rows x cols of x_type, row stride ldx elements
 *   residual_dev  device, rows x cols of out_type, row stride ldr, or NULL: none
 *   out_dev    device, rows x cols of out_type, row stride ldo; may be x or the residual, with the same type and stride, and
 *              not overlap them otherwise
 * 0 <= rows <= 2^26, 1 <= cols <= 65536, 0 <= p <= 1; any alignment of the rows. */
agc_status agc_dropout(const void* x_dev, int x_type, int64_t ldx, const void* residual_dev, int64_t ldr, int64_t rows, int cols,
                       double p, uint64_t seed, uint64_t step, uint32_t site, void* out_dev, int out_type, int64_t ldo,
                       void* hip_stream);

/* Orthogonalised update of n_mats matrices of one shape that lie inside the parameter vector.  For each,
 *   M <- momentum * M + g_hat;   U = g_hat + momentum * M (nesterov) or M;   X = U / (|U|_F + 1e-7);
 *   `steps` times  A = X X^T,  X <- a X + (b A + c A A) X,  a, b, c = 3.4445, -4.7750, 2.0315;
 *   beta <- (1 - lr * weight_decay) * beta - lr * scale * X
 * (products on the matrix's short side; five steps bring the singular values near 1).  `scale` is the caller's rule for
 * the shape, for instance sqrt(max(1, rows / cols)).
 *   beta_dev, m1_dev, ghat_dev  device, the vectors; matrix i is the rows * cols floats from offset_host[i] on,
 *              row-major.  beta and the average m1 are updated in place; matrices must not overlap
 *   offset_host  host, n_mats offsets in elements, in any order
 *   beta_bf16_dev  device, a vector of the same layout in bfloat16 that receives the updated matrices rounded to
 *              nearest even (what agc_gated_forward reads), or NULL
 *   workspace_dev  device, agc_muon_workspace_bytes(...) bytes, 256-byte aligned; scratch
 * Products are taken on operands of 22 bits (pairs of binary16), sums are binary32 in a fixed order, the norm is
 * binary64: the result is reproducible run to run and as near to the exact one as binary32 products come.  A zero
 * gradient gives X = 0; NaN or infinity in g_hat makes its own matrix NaN and no other.
 * 1 <= rows, cols <= AGC_MAX_MATRIX, 1 <= n_mats <= AGC_MAX_LAYERS (AGC_ESHAPE; the workspace size is 0 then),
 * 1 <= steps <= 32 (AGC_EINVAL). */
int64_t agc_muon_workspace_bytes(int rows, int cols, int n_mats);
agc_status agc_muon_update(float *beta_dev, float *m1_dev, const float *ghat_dev, const int64_t *offset_host, int n_mats,
                           int rows, int cols, float lr, float momentum, int nesterov, float weight_decay, float scale,
                           int steps, void *beta_bf16_dev, void *workspace_dev, void *hip_stream);

/* --------------------------------------------------------------------------------------
 * Host-side design routines (no GPU work; run once per change of the system statistics)
 * ------------------------------------------------------------------------------------ */
/* phi(z) = phi_coef / (2^(z-1)-1)^2.  The paper's constant is phi_coef = d/4 (Sec. II-B);
 * the error-balance scaling of Sec. V-B gives phi_coef = mean(p) * (2^(z_total/n - 1) - 1)^2,
 * returned by this helper. */
double agc_phi_coef_balanced(int n, const double *p, int z_total);

/* Low-complexity bit allocation (Sec. III-B.2, Algorithm 1): maximises
 * F = sum_i (1-p_i)/(p_i + phi(z_i)) subject to sum z_i = z_total, z_min <= z_i <= z_max
 * (z_max is this library's cap; the paper has none).  Steps the paper leaves open are read
 * as: Lagrangian candidate by bisection on the multiplier with each active worker on the
 * concave branch of its utility, rounded by largest remainder; equal candidate
 * floor/ceil; best-improvement one-bit swaps inside the active set.  bits_out: n bytes. */
agc_status agc_alloc_bits(int n, const double *p, double phi_coef, int z_total, int z_min,
                          int z_max, uint8_t *bits_out);
/* Optimal allocation by the Bellman recurrence of Sec. III-B.1 (O(n * z_res^2)). */
agc_status agc_alloc_bits_dp(int n, const double *p, double phi_coef, int z_total, int z_min,
                             int z_max, uint8_t *bits_out);
/* F(z) of problem b-SP1 for a given allocation. */
double agc_alloc_objective(int n, const double *p, double phi_coef, const uint8_t *bits);

/* Optimally structured sparse code (Theorem 1 and the interval construction of Sec. III-A):
 * c_i = (p_i + phi(b_i))/(1-p_i), Y_i = c_i^-1 k / sum c^-1, R_i = prefix sums,
 * alpha_ij = [min(R_i, j) - max(R_{i-1}, j-1)]_+, then a_ij = alpha_ij, w_i = 1/(1-p_i)
 * (the free factor w~_i is taken as 1).  Outputs: CSR over caller arrays row_ptr[n+1],
 * col[cap], val[cap] with columns ascending, w_out[n]; *nnz receives the count
 * (<= n + k - 1); cap is the capacity of col/val (AGC_ESHAPE when too small). */
agc_status agc_build_code(int n, int k, const double *p, const uint8_t *bits, double phi_coef,
                          int32_t *row_ptr, int32_t *col, float *val, float *w_out, int cap,
                          int *nnz);
/* Code on the cyclic support {i, .., i+s-1 mod k} (n == k): alpha_ij = c_i^-1 / (sum of
 * c^-1 over the workers holding j); column sums are 1, so the estimator is unbiased; it is a
 * heuristic on a prescribed support, not Theorem 1's optimum.  col/val hold n*s entries in
 * the order u = 0..s-1. */
agc_status agc_build_cyclic_code(int n, int k, int s, const double *p, const uint8_t *bits,
                                 double phi_coef, int32_t *row_ptr, int32_t *col, float *val,
                                 float *w_out);
/* Optimum of the structure problem (Sec. III-A, problem c-SP2) restricted to the same cyclic
 * support: minimises sum_i c_i (sum_j alpha_i^j)^2 over alpha >= 0 with column sums 1, by exact
 * minimisation over one column at a time (convex, converges to the optimum).  When the support
 * admits the row sums of Theorem 1 the result has them and *objective equals k^2 / sum_i c_i^-1
 * (then *reaches_bound = 1); otherwise it is the best the support allows.  A worker may end with
 * zero weight on a partition it holds (the entry is kept, with value 0, so that the layout stays
 * cyclic).  Outputs as agc_build_cyclic_code; objective and reaches_bound may be NULL. */
agc_status agc_build_cyclic_code_opt(int n, int k, int s, const double *p, const uint8_t *bits,
                                     double phi_coef, int32_t *row_ptr, int32_t *col, float *val,
                                     float *w_out, double *objective, int *reaches_bound);
/* Unbiasedness condition of Sec. III: max_j | sum_i (1-p_i) w_i a_ij - 1 | <= tol (binary64
 * over the binary32 inputs).  AGC_OK when it holds, AGC_EINVAL when it does not;
 * *residual (may be NULL) receives the maximum. */
agc_status agc_check_unbiased(int n, int k, const int32_t *row_ptr, const int32_t *col,
                              const float *val, const float *w, const double *p, double tol,
                              double *residual);

/* Second-moment decoding vector of the two-track decode (Sec. V, closed form below the
 * bias-variance objective): with A_i the i-th row sum of the code and c_i = (p_i+phi(z_i))/(1-p_i),
 *   v_i = k * Lambda / ((p_i + phi(z_i)) * A_i * (1 + Lambda * sum_m 1/c_m)),
 * k being the number of columns of the code (the count the bias term sums over).  Lambda > 0
 * weighs squared bias against variance.  v_out: host, n floats. */
agc_status agc_second_moment_decoder(int n, int k, const int32_t *row_ptr, const int32_t *col,
                                     const float *val, const double *p, const uint8_t *bits,
                                     double phi_coef, double Lambda, float *v_out);

#ifdef __cplusplus
}
#endif
#endif /* AGC_H */
