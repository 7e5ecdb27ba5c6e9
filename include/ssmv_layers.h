/*
 * ssmv_layers.h - what stands around and in place of a selective layer in a recurrent language model, in training and in decoding:
 * the norms before and after a block with its gate and residual scale, a gated linear recurrence, and the rules that a request puts on
 * logits ahead of the choice (ssmv_beam_select).  The same library, the same conventions as ssmv.h: device memory of the caller's,
 * asynchronous on `hip_stream`, arguments checked on the host, an ssmv_status returned, the text in ssmv_last_error().
 *
 * As in the decoding calls there, strides are in elements, between the rows of a tensor or the tokens of a sequence, 0 = packed, at most
 * SSMV_LAYER_STRIDE_MAX; sequences are L strides apart.  Tensors need only the alignment of their elements, workspaces 16 bytes; what is
 * aligned to 128 bytes is read fastest.  No output may overlap an input or another output, but where it is said.  A pointer that may be NULL says so.
 *
 * Sums, statistics, states and the gradients of vectors are fp32; what is stored in bf16 is rounded once, to the nearest.  No result
 * depends on the order in which workgroups run: the same call gives the same bits.  Gradients are written, not added to what is there.  One workspace
 * must not be used by two calls that may run at once.
 */
#ifndef SSMV_LAYERS_H
#define SSMV_LAYERS_H

#include "ssmv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SSMV_LAYER_STRIDE_MAX (1 << 24)

/* ---- between two blocks of a residual network ------------------------------------------------------------------------
 * Per row of `channels` values, x the output of a block, res the residual stream:
 *   a = x * z * sigmoid(z)                                  (a = x where z is NULL)
 *   p = a * rsqrt(mean(a^2) + eps) * post_wgt               (p = a where post_wgt is NULL)
 *   r = res + res_scale * ch_scale * p                      (res NULL: 0;  ch_scale NULL: 1)      -> r_out
 *   n = r * rsqrt(mean(r^2) + eps) * pre_wgt                (pre_wgt NULL: 1)                     -> n_out, the next block's input
 * n is that of r before it is rounded.  x NULL: r = res, the norm ahead of the first block; z, post_wgt, ch_scale and r_out must be NULL.
 * res_dtype: io_dtype or SSMV_F32.  r_out may be res (with one stride).  Squares are summed in fp32: values from about 1e18 on overflow them.
 * eps = 0 leaves a row of zeros without a norm (NaN).  rows * ceil(channels / 512) up to 6e7. */
#define SSMV_BLOCK_NORM_MAX 16384       /* largest `channels` */
typedef struct ssmv_block_norm_args {
    const void *x;           /* [rows][channels] io_dtype or NULL                                 */
    const void *z;           /* [rows][channels] io_dtype or NULL                                 */
    const void *res;         /* [rows][channels] res_dtype or NULL                                */
    const float *post_wgt;   /* [channels] or NULL                                                */
    const float *ch_scale;   /* [channels] or NULL                                                */
    const float *pre_wgt;    /* [channels] or NULL                                                */
    void *r_out;             /* [rows][channels] res_dtype, or NULL: not wanted                   */
    void *n_out;             /* [rows][channels] io_dtype, or NULL: not wanted                    */
    int64_t x_stride, z_stride, res_stride, r_stride, n_stride;
    int32_t rows, channels, io_dtype, res_dtype;
    float eps, res_scale;
} ssmv_block_norm_args;
int ssmv_block_norm(const ssmv_block_norm_args *args, void *hip_stream);

/* Its gradients, from the inputs of the forward call alone (what r_out overwrote must still be there): dr and dn are the gradients of r_out and
 * n_out, NULL = zeros, not both.  Every gradient may be NULL: not wanted; one of an input that was NULL must be.  dres may be dr, dx may be dn (with
 * one stride).  workspace: ssmv_block_norm_backward_workspace bytes; NULL where no gradient of a vector is wanted. */
typedef struct ssmv_block_norm_grad_args {
    const void *x, *z, *res;                        /* as in the forward call                            */
    const float *post_wgt, *ch_scale, *pre_wgt;
    const void *dr;          /* [rows][channels] res_dtype or NULL                                */
    const void *dn;          /* [rows][channels] io_dtype or NULL                                 */
    void *dx;                /* [rows][channels] io_dtype                                         */
    void *dz;                /* [rows][channels] io_dtype                                         */
    void *dres;              /* [rows][channels] res_dtype                                        */
    float *dpost_wgt;        /* [channels]                                                        */
    float *dch_scale;        /* [channels]                                                        */
    float *dpre_wgt;         /* [channels]                                                        */
    void *workspace;
    int64_t x_stride, z_stride, res_stride, dr_stride, dn_stride, dx_stride, dz_stride, dres_stride;
    int32_t rows, channels, io_dtype, res_dtype;
    float eps, res_scale;
} ssmv_block_norm_grad_args;
int ssmv_block_norm_backward(const ssmv_block_norm_grad_args *args, void *hip_stream);
int ssmv_block_norm_backward_workspace(int32_t rows, int32_t channels, size_t *out_bytes);

/* ---- the gated linear recurrence ---------------------------------------------------------------------------------------
 * One state a channel, whose decay is a gate of the token, over L tokens (L = 1: one new token of every row):
 *   SSMV_GATED_LRU:  decay = exp(A * sigmoid(f + f_bias)),  m = sqrt(1 - decay^2)      (A [channels], negative)
 *   SSMV_GATED_MIX:  decay = sigmoid(f + f_bias),           m = 1 - decay              (A must be NULL)
 *   h <- decay * h + m * sigmoid(i + i_bias) * x            (i NULL: without that sigmoid; i_bias must then be NULL)
 *   y = h * z * sigmoid(z)                                  (y = h where z is NULL)
 * in fp32, y rounded once to io_dtype; m keeps its accuracy where the decay is near 1.  batch up to 65535, channels to 2^22, L to 2^30.  src_row, rows_in, seq_len, h_in and h_out as in
 * ssm_selective_scan: rows continue from rows of h_in, an index outside [0, rows_in) from zeros; sequence b has clamp(seq_len[b], 0, L) tokens, what lies behind them is
 * neither read nor written, h_out is the state after them.  h_out may be h_in where src_row is NULL.  An A of 0 keeps its state and takes nothing in; one of -inf
 * forgets at every token (but where the sigmoid is 0 in fp32: it keeps its state there).
 * states, for the backward pass: states[b][j] receives the state ahead of token SSMV_GATED_TILE * j for every such token that sequence b has, j = 0
 * always.  workspace: ssm_gated_recurrence_workspace bytes (0 where a sequence is not cut into segments). */
enum { SSMV_GATED_LRU = 0, SSMV_GATED_MIX = 1 };
#define SSMV_GATED_TILE 64
typedef struct ssmv_gated_args {
    const void *x;           /* [batch][L][channels] io_dtype                                     */
    const void *f;           /* [batch][L][channels] io_dtype: raw gate of the decay              */
    const void *i;           /* [batch][L][channels] io_dtype or NULL: raw gate of the input      */
    const void *z;           /* [batch][L][channels] io_dtype or NULL: gate of the output         */
    const float *A;          /* [channels], negative; NULL in form MIX                            */
    const float *f_bias;     /* [channels] or NULL                                                */
    const float *i_bias;     /* [channels] or NULL                                                */
    const float *h_in;       /* [rows_in][channels] or NULL: zeros                                */
    const int32_t *src_row;  /* [batch] or NULL                                                   */
    const int32_t *seq_len;  /* [batch] or NULL                                                   */
    void *y_out;             /* [batch][L][channels] io_dtype                                     */
    float *h_out;            /* [batch][channels], or NULL: not wanted                            */
    float *states;           /* [batch][ceil(L / SSMV_GATED_TILE)][channels], or NULL: not wanted */
    void *workspace;
    int64_t x_stride, f_stride, i_stride, z_stride, y_stride;
    int32_t batch, rows_in, channels, L, io_dtype, form;
} ssmv_gated_args;
int ssm_gated_recurrence(const ssmv_gated_args *args, void *hip_stream);
int ssm_gated_recurrence_workspace(int32_t batch, int32_t channels, int32_t L, size_t *out_bytes);

/* Its gradients.  x, f, i, z, A, the biases and seq_len as in the forward call, states as that call left them (they hold the start states: h_in is not
 * asked for).  dy is the gradient of y_out, dh_out of h_out (NULL: zeros).  Every gradient may be NULL: not wanted; one of an input that was NULL must be.
 * dh_in is the gradient of the state that row b starts from: rows that start from one row of h_in have it to add up, by src_row.  The gradients of A
 * and the biases are sums over all sequences' tokens; where A is 0, that of A has no value and is written as 0.  They are finite for every finite input otherwise: what grows
 * as the decay nears 1 is taken times what falls.  workspace: ssm_gated_recurrence_backward_workspace bytes. */
typedef struct ssmv_gated_grad_args {
    const void *x, *f, *i, *z;
    const float *A, *f_bias, *i_bias, *states;
    const int32_t *seq_len;
    const void *dy;          /* [batch][L][channels] io_dtype                                     */
    const float *dh_out;     /* [batch][channels] or NULL                                         */
    void *dx;                /* [batch][L][channels] io_dtype                                     */
    void *df;                /* [batch][L][channels] io_dtype                                     */
    void *di;                /* [batch][L][channels] io_dtype                                     */
    void *dz;                /* [batch][L][channels] io_dtype                                     */
    float *dA;               /* [channels]                                                        */
    float *df_bias;          /* [channels]                                                        */
    float *di_bias;          /* [channels]                                                        */
    float *dh_in;            /* [batch][channels]                                                 */
    void *workspace;
    int64_t x_stride, f_stride, i_stride, z_stride, dy_stride, dx_stride, df_stride, di_stride, dz_stride;
    int32_t batch, channels, L, io_dtype, form;
} ssmv_gated_grad_args;
int ssm_gated_recurrence_backward(const ssmv_gated_grad_args *args, void *hip_stream);
int ssm_gated_recurrence_backward_workspace(int32_t batch, int32_t channels, int32_t L, size_t *out_bytes);

/* ---- rules on logits -----------------------------------------------------------------------------------------------------
 * Per row b and token v, in this order, in fp32, rounded once to io_dtype (rows up to 65535, vocab to 2^24):
 *   1. v occurs in the row's history:   l <- l > 0 ? l / repetition[b] : l * repetition[b]
 *   2. v occurs c > 0 times behind the history's first prompt_len[b] tokens:   l <- l - frequency[b] * c - presence[b]
 *   3. every place j of the row's list with bias_token[b][j] = v:   l <- l + bias[b][j]  (their sum, in the order of the list)
 *   4. bit v of the row's mask (bit v % 32 of word v / 32) is 0:   l <- -inf, whatever it was
 * The history of row b is that of row src_row[b] of hist (NULL: row b; an index outside [0, rows_in): an empty one), its first clamp(hist_len, 0, hist_stride)
 * tokens, and behind them token[b] (NULL: none is added): with src_row and token the parent and token of ssmv_beam_select, what the beam has said so far.
 * hist_out and hist_len_out receive it for the next call; a history that is full keeps its tokens and the new one counts in this call only.
 * hist_out may be hist where src_row is NULL; hist_len_out is another array than hist_len.  What lies behind a history in hist_out is left as it was.
 * Tokens outside [0, vocab) in histories and lists count for nothing (a history keeps them).  hist NULL: hist_len, src_row, token, prompt_len, the outputs and the three penalties must be NULL, too.
 * repetition (positive), frequency, presence [rows] or NULL: 1, 0, 0.  prompt_len NULL: 0.
 * mask_row[b] (NULL: b, of at least `rows` mask_rows) is a row of `mask`, a state of the request's grammar; outside [0, mask_rows): no mask.  A mask may leave a row nothing.
 * out may be logits (with one stride): then only eights of logits (8 j to 8 j + 7 of a row) of which one changes are read and written; the others of these keep their values (a bf16 NaN
 * may come back with another payload).  Strides: row_stride and out_stride of logits, 0 = vocab; hist_stride 0 is not allowed
 * where hist is given: it is the room of a row of hist and of hist_out; mask_stride in words, 0 = ceil(vocab / 32). */
#define SSMV_RULES_HISTORY_MAX ((1 << 19) - 2)      /* largest hist_stride */
#define SSMV_RULES_BIAS_MAX 4095                    /* largest bias_n      */
typedef struct ssmv_rules_args {
    const void *logits;          /* [rows][vocab] io_dtype                                        */
    const int32_t *hist;         /* [rows_in][hist_stride] or NULL                                */
    const int32_t *hist_len;     /* [rows_in]                                                     */
    const int32_t *src_row;      /* [rows] or NULL                                                */
    const int32_t *token;        /* [rows] or NULL                                                */
    const int32_t *prompt_len;   /* [rows] or NULL                                                */
    const float *repetition;     /* [rows] or NULL                                                */
    const float *frequency;      /* [rows] or NULL                                                */
    const float *presence;       /* [rows] or NULL                                                */
    const int32_t *bias_token;   /* [rows][bias_n] or NULL                                        */
    const float *bias;           /* [rows][bias_n]                                                */
    const uint32_t *mask;        /* [mask_rows][mask_stride] or NULL                              */
    const int32_t *mask_row;     /* [rows] or NULL                                                */
    void *out;                   /* [rows][vocab] io_dtype                                        */
    int32_t *hist_out;           /* [rows][hist_stride] or NULL                                   */
    int32_t *hist_len_out;       /* [rows]; with hist_out                                         */
    int64_t row_stride, out_stride, mask_stride;
    int32_t rows, rows_in, vocab, io_dtype, hist_stride, bias_n, mask_rows;
} ssmv_rules_args;
int ssmv_logit_rules(const ssmv_rules_args *args, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SSMV_LAYERS_H */
