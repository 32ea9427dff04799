/*
 * rnnt_layers.h - C ABI of the layers beside the transducer loss of rnnt_joint_loss.h (same library, same conventions, statuses
 * and dtypes): what the encoders in front of the joint network are made of, and the other loss of its output layer.
 *
 *   rnnt_linear_*    y = residual + dropout(act(x W + b)) and its gradients.  The dropout mask is a function of a seed, an offset and an entry's
 *                    place, not an array of its own.
 *   rnnt_ce_loss_*   cross entropy of softmax(x W + b) with one label per row, and its gradients, without the [R, V] scores.
 *
 * Conventions beyond those of rnnt_joint_loss.h: every array is dense; device pointers are 16-byte aligned (RNNT_ERR_UNSUPPORTED otherwise),
 * workspaces 256-byte aligned.  Every call can be recorded into a HIP graph: all it needs is in its arguments and in device memory, it allocates
 * nothing and copies nothing from the host.  Workspaces hold nothing between calls; calls that share one must be ordered (two graphs that may run
 * side by side need two).  All sums have a fixed order: equal inputs give equal bits.
 */
#ifndef RNNT_LAYERS_H
#define RNNT_LAYERS_H

#include "rnnt_joint_loss.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RNNT_ACT_NONE = 0,
    RNNT_ACT_RELU = 1,
    RNNT_ACT_SILU = 2, /* z sigmoid(z)                              */
    RNNT_ACT_GELU = 3, /* z Phi(z), Phi the normal distribution's   */
    RNNT_ACT_TANH = 4
} rnnt_activation;

typedef struct {
    int64_t M;          /* rows, 0..2^30                                                                    */
    int32_t K;          /* inputs, 1..2^20                                                                  */
    int32_t N;          /* outputs, 1..2^20                                                                 */
    int32_t dtype;      /* rnnt_dtype of x, W, residual, y, their gradients                                 */
    int32_t activation; /* rnnt_activation                                                                  */
    float dropout;      /* probability p of an entry to be dropped, 0 <= p < 1; taken as cut / 65536 with the integer cut nearest to 65536 p (at most
                           65535)                                                                                                       */
    int32_t accumulate_params; /* backward: 0: dW, db are overwritten; 1: added to (they are float then)    */
    int32_t param_grads_bf16;  /* backward, RNNT_BF16 only: bit 0: dW is bfloat16, bit 1: db is bfloat16; else float.  */
    int32_t bias_bf16;         /* b is 0: float, 1: bfloat16                                                */
} rnnt_linear_desc;

/*
 * z = x W + b,  a = act(z),  y = residual + a m / (1 - p)
 *
 * m: entry (r, n) is kept where its 16 random bits are at least cut.  They come from Philox4x32-10 with the key {low, high word of the seed} on the
 * counter {n / 8, r, low, high word of the offset}: entry n takes half n % 2 (0: the low one) of word (n % 8) / 2.  The same seed and offset give the
 * same mask, whatever the sizes of the call; calls that shall have different ones (layers, steps) take different offsets or seeds.
 *
 * x        dev [M, K]   desc->dtype
 * W        dev [K, N]   desc->dtype (the transpose of a torch Linear's weight)
 * b        dev [N]      float or bfloat16 (desc->bias_bf16), or NULL
 * residual dev [M, N]   desc->dtype, or NULL
 * rng      dev [2]      {seed, offset}, read by the kernels when they run (a replayed graph takes what is there then); NULL allowed with p = 0
 * rng_used dev [2]      out, or NULL: the seed and offset this call took (for its backward pass, where the caller advances rng meanwhile)
 * y        dev [M, N]   desc->dtype, out
 * saved    dev [M, N]   out, or NULL: what the backward pass needs of z, two bytes per entry with RNNT_BF16 (z in fp16; RNNT_ACT_RELU: its sign), four with
 *                       RNNT_F32; -infinity in dropped entries.  The backward pass of RNNT_ACT_NONE does without.
 * RNNT_BF16: the product runs on bf16 MFMA with fp32 accumulation, everything behind it in fp32, one rounding at the end.  RNNT_F32: every value as three
 * bf16 parts, six products of them (as exact as fp32 ones); up to 64 rows on the fp32 MFMA.
 * workspace_bytes >= rnnt_linear_workspace_bytes(desc, 0); with 0 bytes workspace may be NULL.
 */
size_t rnnt_linear_workspace_bytes(const rnnt_linear_desc* desc, int32_t backward);
rnnt_status rnnt_linear_fwd(const rnnt_linear_desc* desc, const void* x, const void* W, const void* b, const void* residual,
                            const uint64_t* rng, uint64_t* rng_used, void* y, void* saved, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Gradients for an incoming dy = d/dy: with dz = dy act'(z) m / (1 - p)
 *   dx = dz W^T,  dW = x^T dz,  db = column sums of dz   (and dy itself is the residual's)
 * RNNT_BF16: dy act'(z) m is rounded to bfloat16 as the operand of both products, in two values of it up to 64 rows (db: before that rounding).
 *
 * x, W, rng as in the forward call, with the same values; saved: what it left (NULL allowed with RNNT_ACT_NONE)
 * dy dev [M, N] desc->dtype;  dx dev [M, K] desc->dtype, out;  dW dev [K, N], db dev [N], out.  Each of dx, dW, db may be NULL: not wanted.
 * workspace_bytes >= rnnt_linear_workspace_bytes(desc, 1).
 */
rnnt_status rnnt_linear_bwd(const rnnt_linear_desc* desc, const void* x, const void* W, const void* saved, const uint64_t* rng, const void* dy,
                            void* dx, void* dW, void* db, void* workspace, size_t workspace_bytes, void* hip_stream);

typedef struct {
    int64_t R;            /* rows, 0..2^30                                                                  */
    int32_t D;            /* width of x, 1..2^20                                                            */
    int32_t V;            /* vocabulary, 1..2^20                                                            */
    int32_t dtype;        /* rnnt_dtype of x, W and their gradients                                         */
    int32_t ignore_label; /* rows with this label are padding                                               */
    int32_t accumulate_params; /* 0: dW, db are overwritten; 1: added to (they are float then)              */
    int32_t param_grads_bf16;  /* RNNT_BF16 only: bit 0: dW is bfloat16, bit 1: db is bfloat16; else float  */
    int32_t bias_bf16;         /* b is 0: float, 1: bfloat16                                                */
} rnnt_ce_desc;

/*
 * h = x W + b,  loss[r] = ln sum_v e^{h[r, v]} - h[r, label[r]]      (natural log)
 * and, for L = sum_r row_weight[r] loss[r] (dh = row_weight (softmax(h) - onehot)),  dx = dh W^T,  dW = x^T dh,  db = column sums of dh.
 *
 * The rows that are no padding are put together and go through in chunks: a chunk's exponentials (RNNT_BF16: fp16 relative to
 * maxima over parts of the vocabulary; RNNT_F32: its scores) are kept in the workspace until its score gradients have replaced them.  Three
 * products per row, as many as the gradients need.
 *
 * x          dev [R, D]  desc->dtype; padding rows may hold anything and are never used
 * W          dev [D, V]  desc->dtype (W_out of rnnt_joint_loss_fwd_bwd)
 * b          dev [V]     float or bfloat16 (desc->bias_bf16), or NULL; -inf takes an entry out of the vocabulary
 * label      dev [R]     int32
 * row_weight dev [R]     float, any sign, or NULL (ones); read by the kernels
 * loss       dev [R]     float, out; 0 in padding rows; +inf where the label is outside [0, V) (its gradient then is row_weight softmax(h)) or no entry
 *                        of the vocabulary is possible (all scores -inf: its gradient is that of the label alone)
 * dx         dev [R, D]  desc->dtype, out; zeros in padding rows
 * dW dev [D, V], db dev [V] (NULL: not wanted), out
 * RNNT_BF16: the three products run on bf16 MFMA with fp32 accumulation, the softmax in fp32; dh is rounded to bfloat16 as their operand,
 * relative to the mantissa of the largest weight, in two values of it up to 64 rows.  The label's entry, row_weight (p - 1), comes from the loss and is as
 * good as that one: about row_weight 2^-20 where p is near 1 (RNNT_F32 likewise).
 *
 * workspace bytes: grads = 0 for rnnt_ce_loss_fwd, 1 for rnnt_ce_loss_fwd_bwd.  budget_bytes = 0: the library's default (chunk buffers of at most
 * 1 GiB); otherwise the size for as few chunks as the budget has room for, or, where it is too small for any number of them, the least size there is.  A
 * call takes every workspace of at least such a size; one larger than the default's is used for larger chunks.
 */
size_t rnnt_ce_loss_workspace_bytes(const rnnt_ce_desc* desc, int32_t grads, size_t budget_bytes);
rnnt_status rnnt_ce_loss_fwd(const rnnt_ce_desc* desc, const void* x, const void* W, const void* b, const int32_t* label, float* loss,
                             void* workspace, size_t workspace_bytes, void* hip_stream);
rnnt_status rnnt_ce_loss_fwd_bwd(const rnnt_ce_desc* desc, const void* x, const void* W, const void* b, const int32_t* label,
                                 const float* row_weight, float* loss, void* dx, void* dW, void* db, void* workspace, size_t workspace_bytes,
                                 void* hip_stream);

/*
 * total (dev, float, out) = sum over the rows of row_weight[r] loss[r], without the rows of weight 0 (whose loss may be infinite); row_weight NULL: ones.
 */
rnnt_status rnnt_ce_loss_total(const rnnt_ce_desc* desc, const float* loss, const float* row_weight, float* total, void* hip_stream);
/*
 * dx, dW, db (each may be NULL) of rnnt_ce_loss_fwd_bwd times *factor (dev, read by the kernel), in place; a factor of 1 moves no data.  Those in bfloat16 are
 * rounded a second time, where the factor is no power of two: weights that hold it already spare them that.
 */
rnnt_status rnnt_ce_loss_scale(const rnnt_ce_desc* desc, const float* factor, void* dx, void* dW, void* db, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RNNT_LAYERS_H */
