/*
 * dendsn_block.h — C ABI of the operators of a block of token-sequence layers, and of its
 * training step, on AMD Instinct MI355X (gfx950).  Same library as dendsn.h and dendsn_seq.h.
 *
 *   delta rule   the gated scan's relative with a matrix for a state: head by head,
 *                  S[t] = a S[t-1] + k (b (v - a S[t-1]^T k))^T,   a = exp(g), b = beta
 *                  o[t] = scale S[t]^T q,                          S[0] given (or 0)
 *                forward, backward and one token at a time
 *   norm         root-mean-square norm of rows, or of their sum with a residual stream,
 *                  s = x + residual,  rstd = (mean s^2 + eps)^-1/2,  y = s rstd weight
 *                forward (in io, or as 8-bit rows with scales) and backward
 *   AdamW        one optimizer step over many tensors,
 *                  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
 *                  p = p - lr (wd p + (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
 *                with states in fp32 or in 8 bits
 *
 * The conventions are those of dendsn_seq.h: device pointers of the caller's, aligned to
 * their elements (workspaces and checkpoints: 16 bytes); no allocation, no state between
 * calls, no synchronisation; no overlap of outputs with inputs or each other (not checked)
 * but where a tensor is updated in place; outputs overwritten, bit-identical for the same
 * inputs; every check on the host before a launch, and dendsn_seq_last_error() describes
 * the first that failed.  Sums, states and statistics are fp32 whatever io is.
 */
#ifndef DENDSN_BLOCK_H
#define DENDSN_BLOCK_H

#include "dendsn_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------- */
/* Gated delta rule                                                           */
/* ------------------------------------------------------------------------- */
typedef struct dendsn_delta_cfg {
    int64_t T;          /* steps, 0 <= T <= 2^24                               */
    int64_t batch;      /* sequences, 0 <= batch <= 65535                      */
    int64_t H;          /* heads of v, g, beta, o and the state, 0 <= H <= 65535 */
    int64_t Hk;         /* heads of q and k; H is a multiple: head h goes with h / (H / Hk) */
    int64_t K;          /* values of q and k, 1 <= K <= 128                    */
    int64_t V;          /* values of v and o, 1 <= V <= 65536                  */
    /* Strides of step, sequence and head: element (t, b, h, d) of q lies at
     * t * q_t + b * q_b + h * q_h + d, and so on (g and beta: without d).  Those of
     * inputs may be 0 (broadcast); rows of outputs may not overlap.  Over whole sequences
     * 64 steps of a tensor, gradients among them, span less than 2^31 bytes (or T is 1), and
     * batch * H * V is at most 2^26 (V in 32s). */
    int64_t q_t, q_b, q_h, k_t, k_b, k_h, v_t, v_b, v_h, g_t, g_b, g_h, beta_t, beta_b, beta_h, o_t, o_b, o_h;
    int64_t grad_o_t, grad_o_b, grad_o_h;                    /* backward             */
    int32_t io;         /* dendsn_io of q, k, v, g, beta, o and their gradients */
    float scale;        /* of o; finite                                        */
} dendsn_delta_cfg;

/* Bytes of what the forward writes for the backward (states at the first of every 64 steps,
 * and the steps' values), and of the scratch of each direction. */
dendsn_status dendsn_delta_ckpt_bytes(const dendsn_delta_cfg* cfg, size_t* bytes);
dendsn_status dendsn_delta_workspace_bytes(const dendsn_delta_cfg* cfg, int32_t backward, size_t* bytes);

/*
 * Forward over all steps.
 *   q, k     [T,batch,Hk,K] io   required
 *   v        [T,batch,H,V] io    required
 *   g        [T,batch,H] io      required: logarithms of the decays.  Meant to be <= 0; what
 *                                is below -200 (minus infinity too) forgets all, as -200 does;
 *                                above 0 a chunk's 64 may add up to 80 at most
 *   beta     [T,batch,H] io      required
 *   s0       [batch,H,K,V] fp32  NULL means 0
 *   lengths  [batch] int32       NULL: every sequence has T steps.  Steps at and past
 *                                lengths[b] (clamped to [0, T]) are no part of sequence b:
 *                                what the inputs hold there has no effect, o is +0 there
 *   o        [T,batch,H,V] io    required output
 *   s_last   [batch,H,K,V] fp32  optional output: the state after the sequence's last step
 *   ckpt     dendsn_delta_ckpt_bytes bytes, optional output (needed by the backward)
 * Steps go in chunks of 64: an input that is not finite may leave its whole chunk's outputs,
 * the steps before it among them, and all later ones not finite.  In bf16 what is neither an
 * input nor an output enters the products as the sum of three bf16 values where s_last and
 * grad_s0 hang on it (fp32's own rounding), of two (to 2^-17) where only outputs in bf16 do.
 */
dendsn_status dendsn_delta_forward(const dendsn_delta_cfg* cfg, const void* q, const void* k, const void* v,
                                   const void* g, const void* beta, const float* s0, const int32_t* lengths, void* o,
                                   float* s_last, void* ckpt, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream);

/*
 * Gradients of sum(grad_o * o) + sum(grad_s_last * s_last).
 *   grad_o       [T,batch,H,V] io     required
 *   grad_s_last  [batch,H,K,V] fp32   NULL means 0
 *   grad_q, grad_k [T,batch,Hk,K], grad_v [T,batch,H,V], grad_g, grad_beta [T,batch,H] io
 *                contiguous, required outputs, +0 past a sequence's end; shared heads of q
 *                and k have the sum over the heads that share them
 *   grad_s0      [batch,H,K,V] fp32   optional output
 */
dendsn_status dendsn_delta_backward(const dendsn_delta_cfg* cfg, const void* q, const void* k, const void* v,
                                    const void* g, const void* beta, const int32_t* lengths, const void* ckpt,
                                    const void* grad_o, const float* grad_s_last, void* grad_q, void* grad_k,
                                    void* grad_v, void* grad_g, void* grad_beta, float* grad_s0, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream);

/*
 * One token of each of cfg->batch requests (cfg->T must be 1; the strides of step are not used).
 *   state  [n_slots,H,K,V] fp32, updated in place
 *   slots  [batch] int32: the state of each request; NULL: state b for request b (then
 *          n_slots >= batch).  A request whose slot is outside [0, n_slots) is idle: its o
 *          is +0 and no state changes.  No slot may be named twice in one call (not checked).
 *   o      [batch,H,V] io
 */
dendsn_status dendsn_delta_step(const dendsn_delta_cfg* cfg, const void* q, const void* k, const void* v,
                                const void* g, const void* beta, int64_t n_slots, const int32_t* slots, float* state,
                                void* o, hipStream_t stream);

/* ------------------------------------------------------------------------- */
/* Root-mean-square norm                                                      */
/* ------------------------------------------------------------------------- */
typedef struct dendsn_norm_cfg {
    int64_t N;          /* rows, 0 <= N <= 2^31 - 1; forward: x and y of 2^39 bytes at most
                         * together, which is more than a card's memory       */
    int64_t D;          /* values of a row, 1 <= D <= 2^22                     */
    int64_t ld_x, ld_residual, ld_y, ld_sum;                 /* forward              */
    int64_t ld_grad_y, ld_grad_sum, ld_grad_x;               /* backward             */
    int32_t io;         /* dendsn_io of rows, weight and their gradients       */
    float eps;          /* finite, >= 0                                        */
} dendsn_norm_cfg;      /* strides in elements; of outputs >= D, of inputs >= 0 */

/*
 *   x        [N,D] io
 *   residual [N,D] io   NULL: s = x
 *   weight   [D] io     NULL: 1
 *   y        [N,D] io
 *   sum      [N,D] io   optional output: s, as the backward and the next layer read it
 *   rstd     [N] fp32   optional output
 * The statistics and y are of s before its rounding to io.  Squares are summed in fp32 as they are: a row
 * with values past some 10^19 has rstd 0, and a y of 0.
 */
dendsn_status dendsn_norm_forward(const dendsn_norm_cfg* cfg, const void* x, const void* residual, const void* weight,
                                  void* y, void* sum, float* rstd, hipStream_t stream);

/* The same with rows in 8 bits: y [N,D] e4m3 (ld_y bytes apart) and scale [N] fp32, where
 * y * scale is the row and scale the 448th part of its largest magnitude (1 of a row of zeros). */
dendsn_status dendsn_norm_forward_e4m3(const dendsn_norm_cfg* cfg, const void* x, const void* residual,
                                       const void* weight, void* y, float* scale, void* sum, float* rstd,
                                       hipStream_t stream);

/* Scratch of dendsn_norm_backward with a weight. */
dendsn_status dendsn_norm_workspace_bytes(const dendsn_norm_cfg* cfg, size_t* bytes);

/*
 * Gradients of sum(grad_y * y) + sum(grad_sum * sum); that of x is also the residual's.
 *   x           [N,D] io    the forward's x, or its sum where it had a residual (ld_x): what is
 *                           differentiated is the norm of this row.  In bf16 the sum's rounding moves
 *                           grad_weight by as much as grad_weight's own
 *   rstd        [N] fp32    the forward's
 *   grad_y      [N,D] io    required
 *   grad_sum    [N,D] io    NULL means 0
 *   grad_x      [N,D] io    required output
 *   grad_weight [D] io      required output where weight is given
 */
dendsn_status dendsn_norm_backward(const dendsn_norm_cfg* cfg, const void* x, const void* weight, const float* rstd,
                                   const void* grad_y, const void* grad_sum, void* grad_x, void* grad_weight,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream);

/* The same from the forward's x and residual [N,D] io (ld_residual; NULL: as above), whose sum is formed
 * again in fp32: gradients of what y is the norm of, for one more array read. */
dendsn_status dendsn_norm_backward_residual(const dendsn_norm_cfg* cfg, const void* x, const void* residual,
                                            const void* weight, const float* rstd, const void* grad_y,
                                            const void* grad_sum, void* grad_x, void* grad_weight, void* workspace,
                                            size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------- */
/* AdamW                                                                      */
/* ------------------------------------------------------------------------- */
typedef enum dendsn_adamw_state { DENDSN_STATE_F32 = 0, DENDSN_STATE_E4M3 = 1 } dendsn_adamw_state;

typedef struct dendsn_adamw_cfg {
    double lr, beta1, beta2, eps, weight_decay;   /* finite; 0 <= betas < 1; eps, weight_decay >= 0 */
    int32_t state;      /* dendsn_adamw_state                                  */
} dendsn_adamw_cfg;

/* One tensor: a HOST struct of device pointers, read during the call. */
typedef struct dendsn_adamw_tensor {
    int64_t n;          /* values, 0 <= n <= 2^34; all arrays contiguous       */
    float* param;       /* [n] updated in place                                */
    const void* grad;   /* [n] grad_io                                         */
    void* m;            /* [n] fp32, or e4m3, updated in place                 */
    void* v;            /* [n] fp32, or e4m3 of the root of v, updated in place */
    float* m_scale;     /* [ceil(n / 256)] with 8-bit states: a block's scale  */
    float* v_scale;     /* likewise, of the root of v                          */
    void* copy;         /* [n] bf16, optional output: the new param rounded    */
    int32_t grad_io;    /* dendsn_io                                           */
} dendsn_adamw_tensor;

/*
 * One step over `count` tensors (a HOST array; 0 <= count <= 2^20).
 *   step       the step's number, >= 1; step_dev [1] int32 on the device, if not NULL, takes
 *              its place (a captured step is replayed with other numbers)
 *   grad_scale [1] fp32 on the device, optional: gradients are multiplied by it first
 *   seed       of the random bits of 8-bit states
 * 8-bit states hold m and the root of v in blocks of 256 values, each value an e4m3 number
 * times its block's scale (the block's largest magnitude times 1/448 rounded to fp32).  A value is
 * rounded to one of its two neighbours at random, so that its mean is kept: with rounding
 * to the nearest v could not fall by less than a sixteenth, and would not fall at all.  A v
 * that is not 0 is kept above 0.  The random bits are a hash of seed, the step, the tensor's
 * place in the list and the value's place in the tensor.
 * A gradient that is not finite makes its own states and parameter not finite; an infinite one
 * does so, in 8 bits, to the states of its block of 256.
 * Arrays that are written (param, m, v, scales, copy) may not overlap, within a tensor or between two
 * (not checked); grad is read alone and may be shared.
 */
dendsn_status dendsn_adamw_step(const dendsn_adamw_cfg* cfg, const dendsn_adamw_tensor* tensors, int64_t count,
                                int64_t step, const int32_t* step_dev, const float* grad_scale, uint64_t seed,
                                hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DENDSN_BLOCK_H */
