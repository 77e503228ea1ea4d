/*
 * dendsn_seq.h — C ABI of the token-sequence operators around the DendSN layer
 * on AMD Instinct MI355X (gfx950).  Same library as dendsn.h.
 *
 * Three operators carry a stream of tokens through a network of DendSN layers:
 *
 *   embedding    rows of a table as input currents, and the table's gradient
 *   gated scan   the layer's leaky compartment with a leak set by the data:
 *                  a[t] = sigmoid(g[t])  (DENDSN_GATE_SIGMOID)   or   g[t]  (DENDSN_GATE_DECAY)
 *                  w[t] = 1 - a[t]       (leaky = 1)             or   1     (leaky = 0)
 *                  h[t] = a[t] h[t-1] + w[t] x[t],   h[0] given (or 0)
 *                channel by channel, forward, backward and one token at a time
 *   linear CE    softmax cross entropy of a linear readout over a vocabulary,
 *                  z = scale * hidden weight^T,  lse = log sum_v exp(z_v),  loss = lse - z_target
 *                with the gradients of both operands; at most 4 GiB of logits are held
 *                at a time (all of them where they fit), without gradients none
 *
 * Conventions (those of dendsn.h):
 *   - Every tensor pointer is a DEVICE pointer owned by the caller, aligned to
 *     its element size (workspaces and checkpoints: 16 bytes).  Wider alignment
 *     is used where it is there, never required.
 *   - The library allocates nothing, keeps no state between calls and never
 *     synchronises: every call enqueues kernels on the given stream and returns.
 *   - An output, a checkpoint or a workspace may overlap neither an input nor
 *     another of them (not checked), but for the state of dendsn_scan_step.
 *   - Outputs are overwritten, never accumulated.  Results are deterministic: the
 *     same inputs, of the same alignment and strides (by which kernels are chosen,
 *     whose sums run in other orders), give bit-identical outputs.
 *   - Kernels run on the current device, whose memory and stream the arguments are.
 *   - Every argument check runs on the host before anything is launched; on
 *     failure the call writes nothing, returns a status, and
 *     dendsn_seq_last_error() on the calling thread describes the first failed
 *     check.  A failed launch returns DENDSN_E_HIP.
 *   - io is dendsn_io: the storage of the tensors marked "io"; fp32 or bf16.  Sums,
 *     states, softmax statistics and losses are fp32 either way.
 *   - index is dendsn_index: the storage of ids and targets.
 *   - Strides are in elements, between rows whose D values are adjacent.
 *   - A count of zero is valid; pointers to arrays of no elements may be NULL.
 */
#ifndef DENDSN_SEQ_H
#define DENDSN_SEQ_H

#include "dendsn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum dendsn_index { DENDSN_INDEX_I32 = 0, DENDSN_INDEX_I64 = 1 } dendsn_index;
typedef enum dendsn_gate { DENDSN_GATE_SIGMOID = 0, DENDSN_GATE_DECAY = 1 } dendsn_gate;

/* ------------------------------------------------------------------------- */
/* Embedding                                                                  */
/* ------------------------------------------------------------------------- */
typedef struct dendsn_embed_cfg {
    int64_t n;          /* tokens, 0 <= n <= 2^25                              */
    int64_t V;          /* rows of the table, 0 <= V <= 2^27                   */
    int64_t D;          /* values of a row, 0 <= D < 2^22                      */
    int64_t ld_table;   /* stride of table and grad_table, >= D                */
    int64_t ld_out;     /* stride of out and grad_out, >= D (grad_out: any >= 0) */
    int32_t io;         /* dendsn_io                                           */
    int32_t index;      /* dendsn_index                                        */
    float scale;        /* finite                                              */
} dendsn_embed_cfg;

/* out[i] = scale * table[ids[i]].  An id outside [0, V) names no row: its out
 * row is +0, and it has no part in the gradient. */
dendsn_status dendsn_embed_forward(const dendsn_embed_cfg* cfg, const void* ids, const void* table, void* out,
                                   hipStream_t stream);

/* Scratch of dendsn_embed_backward (always > 0).  Both refuse n * D above
 * 2^36 (n in runs of 32, D in 64s) with DENDSN_E_UNSUPPORTED. */
dendsn_status dendsn_embed_workspace_bytes(const dendsn_embed_cfg* cfg, size_t* bytes);

/* grad_table[v] = scale * sum of grad_out[i] over the i with ids[i] = v, every
 * one of the V rows written (+0 where no token names it).  Sums are fp32 in an
 * order fixed by the ids, rounded once to io. */
dendsn_status dendsn_embed_backward(const dendsn_embed_cfg* cfg, const void* ids, const void* grad_out,
                                    void* grad_table, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream);

/* ------------------------------------------------------------------------- */
/* Gated scan                                                                 */
/* ------------------------------------------------------------------------- */
typedef struct dendsn_scan_cfg {
    int64_t T;          /* steps, 0 <= T <= 2^30                               */
    int64_t batch;      /* sequences, 0 <= batch < 65536                       */
    int64_t D;          /* channels, 0 <= D <= 2^27                            */
    /* Strides of step and of sequence: element (t, b, d) of x lies at
     * t * x_t + b * x_b + d, and so on.  Those of inputs may be 0 (broadcast);
     * rows of outputs may not overlap. */
    int64_t x_t, x_b, g_t, g_b, h_t, h_b;                    /* x, g, h              */
    int64_t grad_h_t, grad_h_b, grad_x_t, grad_x_b, grad_g_t, grad_g_b;  /* backward */
    int32_t io;         /* dendsn_io of x, g, h and their gradients            */
    int32_t gate;       /* dendsn_gate                                         */
    int32_t leaky;      /* 1: inputs weighted by 1 - a; 0: by 1                */
} dendsn_scan_cfg;

/* Bytes of the checkpoints (states at the first of every 64 steps) that the
 * forward writes and the backward reads, and of the scratch of each direction
 * (backward != 0: of dendsn_scan_backward); the scratch may be 0. */
dendsn_status dendsn_scan_ckpt_bytes(const dendsn_scan_cfg* cfg, size_t* bytes);
dendsn_status dendsn_scan_workspace_bytes(const dendsn_scan_cfg* cfg, int32_t backward, size_t* bytes);

/*
 * Forward over all steps.  Decays that are given (DENDSN_GATE_DECAY) may have any value,
 * beyond 1 too: products of many steps' carry exponents of their own.  After an input that
 * is not finite its channel's states are not finite either, infinite or NaN.
 *   x, g     [T,batch,D] io    required
 *   h0       [batch,D] fp32    NULL means 0
 *   lengths  [batch] int32     NULL: every sequence has T steps.  Steps at and past
 *                              lengths[b] (clamped to [0, T]) are no part of sequence b:
 *                              what x and g hold there has no effect, h is +0 there
 *   h        [T,batch,D] io    required output
 *   h_last   [batch,D] fp32    optional output: the state after the sequence's last step
 *   ckpt     dendsn_scan_ckpt_bytes bytes, optional output (needed by the backward)
 */
dendsn_status dendsn_scan_forward(const dendsn_scan_cfg* cfg, const void* x, const void* g, const float* h0,
                                  const int32_t* lengths, void* h, float* h_last, float* ckpt, void* workspace,
                                  size_t workspace_bytes, hipStream_t stream);

/*
 * Gradients of sum(grad_h * h) + sum(grad_h_last * h_last).  States are computed
 * again from x, g and the checkpoints, in fp32.
 *   grad_h       [T,batch,D] io   required
 *   grad_h_last  [batch,D] fp32   NULL means 0
 *   grad_x, grad_g [T,batch,D] io required outputs, +0 past a sequence's end
 *   grad_h0      [batch,D] fp32   optional output
 */
dendsn_status dendsn_scan_backward(const dendsn_scan_cfg* cfg, const void* x, const void* g,
                                   const int32_t* lengths, const float* ckpt, const void* grad_h,
                                   const float* grad_h_last, void* grad_x, void* grad_g, float* grad_h0,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * One token of each of cfg->batch requests (cfg->T must be 1; x_b, g_b, h_b are
 * the strides): h = a state + w x, and the state becomes h.
 *   x, g   [batch,D] io
 *   state  [n_slots,D] fp32, updated in place
 *   slots  [batch] int32: the state row of each request; NULL: row b for request b
 *          (then n_slots >= batch).  A request whose slot is outside [0, n_slots)
 *          is idle: its h is +0 and no state changes.  No slot may be named twice
 *          in one call (not checked).
 *   h      [batch,D] io
 */
dendsn_status dendsn_scan_step(const dendsn_scan_cfg* cfg, const void* x, const void* g, int64_t n_slots,
                               const int32_t* slots, float* state, void* h, hipStream_t stream);

/* ------------------------------------------------------------------------- */
/* Linear cross entropy                                                       */
/* ------------------------------------------------------------------------- */
typedef struct dendsn_ce_cfg {
    int64_t N;          /* rows, 0 <= N <= 2^26                                */
    int64_t V;          /* classes, 1 <= V <= 2^24                             */
    int64_t D;          /* features, 1 <= D <= 2^20                            */
    int64_t ld_hidden, ld_weight;            /* strides, >= D                  */
    int64_t ld_grad_hidden, ld_grad_weight;  /* dendsn_ce_train, >= D          */
    int32_t io;         /* dendsn_io of hidden, weight and their gradients     */
    int32_t index;      /* dendsn_index of targets                             */
    float logit_scale;  /* finite                                              */
} dendsn_ce_cfg;

/* Scratch of the loss alone (train = 0) or of the loss with gradients (train != 0).
 * Rows go through in pieces: at most 4 GiB of logits (in fp32 with their gradient) and
 * 4 GiB of copies of hidden are held at a time, or 256 rows' where those are more; the
 * rest does not grow with N but for some bytes a tile of logits. */
dendsn_status dendsn_ce_workspace_bytes(const dendsn_ce_cfg* cfg, int32_t train, size_t* bytes);

/* The same for operands that lie at these addresses (only their alignment counts):
 * without the copies of operands that the kernels read in place, which the query
 * above has room for.  The calls below ask for this much. */
dendsn_status dendsn_ce_workspace_bytes_at(const dendsn_ce_cfg* cfg, int32_t train, const void* hidden,
                                           const void* weight, size_t* bytes);

/*
 * loss[n] = lse[n] - z[n, targets[n]], lse[n] = log sum_v exp(z[n, v]).  A row
 * whose target is outside [0, V) is ignored: its loss and lse are +0, and
 * whatever its hidden row holds has no effect.
 *   hidden [N,D] io, weight [V,D] io, targets [N], loss [N] fp32, lse [N] fp32 (optional)
 */
dendsn_status dendsn_ce_forward(const dendsn_ce_cfg* cfg, const void* hidden, const void* weight,
                                const void* targets, float* loss, float* lse, void* workspace,
                                size_t workspace_bytes, hipStream_t stream);

/*
 * The same losses, and the gradients of sum_n row_weight[n] * loss[n] in the same
 * call: products of the training step are done once.
 *   row_weight  [N] fp32          NULL means 1
 *   grad_hidden [N,D] io, grad_weight [V,D] io   required outputs; rows of ignored
 *                                 rows, and of classes with no part, are +0
 * In bf16 the gradient of the logits, in units of the largest row weight, is
 * rounded to bf16 before the two products that it enters; every sum is fp32.
 */
dendsn_status dendsn_ce_train(const dendsn_ce_cfg* cfg, const void* hidden, const void* weight,
                              const void* targets, const float* row_weight, float* loss, float* lse,
                              void* grad_hidden, void* grad_weight, void* workspace, size_t workspace_bytes,
                              hipStream_t stream);

/* Description of the last failed check of this header's calls on the calling
 * thread ("" if none). */
const char* dendsn_seq_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* DENDSN_SEQ_H */
