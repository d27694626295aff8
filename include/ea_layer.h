/*
 * ea_layer.h -- the part of libea's C ABI for the layers of a sequence model,
 * beside the optimizers and the embedding of ea_train.h: layer norm, dropout
 * from the library's counter-based draws, the gated linear recurrence, and the
 * token loss, each with its gradient.
 *
 * The conventions of ea.h and ea_train.h hold: device memory is the caller's,
 * work is enqueued on `stream` and the call returns without waiting, arguments
 * are checked before anything is enqueued, EA_OK or a negative EA_ERR_* is
 * returned and ea_last_error() describes the last failure of the thread.  Every
 * result is the same, bit for bit, from run to run.  No call keeps anything
 * between calls, and all can be captured in a HIP graph.
 *
 * Element types: EA_F32, EA_BF16, EA_F16.  A device pointer is aligned to its
 * element's size (else EA_ERR_ALIGN); vectors need no alignment beyond that.
 * All arithmetic is binary32 or wider; a result in 16 bits is rounded to
 * nearest even once, at the end.
 *
 * Rows: `x_stride` and its like are the elements from one row to the next, at
 * least the row's width; elements between rows are not written, and what they
 * hold has no effect.
 * Arrays that a call writes do not overlap any other array of the call, but
 * where it says so.  A workspace's contents do not matter; calls that share one
 * are ordered by the caller.
 */
#ifndef EA_LAYER_H
#define EA_LAYER_H

#include <stdint.h>

#include "ea.h"
#include "ea_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- layer norm ------------------------------------------------------------ */

typedef struct ea_layer_norm {
    int64_t rows;            /* 0 <= rows < 2^31                                      */
    int64_t dim;             /* columns, 1 <= dim <= 2^20                             */
    int64_t x_stride;        /* of x, dx and add, in [dim, 2^32)                      */
    int64_t y_stride;        /* of y and dy, in [dim, 2^32)                           */
    float eps;               /* finite, > 0                                           */
    int32_t x_type;          /* type of x, dx and add                                 */
    int32_t y_type;          /* type of y and dy                                      */
    int32_t w_type;          /* type of weight, bias and their gradients              */
} ea_layer_norm_t;

/* For every row:
 *     mean <- sum(x) / dim
 *     rstd <- 1 / sqrt(sum((x - mean)^2) / dim + eps)
 *     y    <- (x - mean) rstd weight + bias
 *   x, weight (device, dim, or NULL: ones), bias (device, dim, or NULL: zeros),
 *   y (device, rows, write; may be x when types and strides are the same),
 *   mean, rstd (device, rows floats each, write; may be NULL, but the gradient
 *   needs them).
 * The mean is the sum's quotient to the nearest: a row of one value whose sum is
 * exact gives the bias.  A row that holds an infinity or NaN, or whose sum, or
 * difference from the mean, overflows binary32, gives NaN, in that row only; one
 * whose squares alone overflow has rstd = 0 and y = bias. */
int ea_layer_norm(const ea_layer_norm_t *c, const void *x, const void *weight, const void *bias, void *y, float *mean,
                  float *rstd, void *stream);

/* Device workspace (bytes) of ea_layer_norm_grad. */
int64_t ea_layer_norm_workspace_bytes(const ea_layer_norm_t *c);

/* Gradient of the norm, with xh = (x - mean) rstd and q = dy weight:
 *     dx      <- rstd (q - sum(q) / dim - xh sum(q xh) / dim)   (+ add when add is not NULL)
 *     dweight <- sum over rows of dy xh    (+ dweight when accumulate is 1)
 *     dbias   <- sum over rows of dy       (+ dbias when accumulate is 1)
 * `add` is another gradient of x, as of a residual branch around the norm.
 *   x, dy, mean, rstd (as ea_layer_norm left them), weight (or NULL: ones),
 *   add (device, rows, read, or NULL; may be dx), dx (device, rows, write; may
 *   be x; may be dy when types and strides are the same), dweight, dbias
 *   (device, dim each, write or read/write, each may be NULL), workspace (device,
 *   ea_layer_norm_workspace_bytes bytes, 16-byte aligned; NULL when that is 0
 *   or when both dweight and dbias are). */
int ea_layer_norm_grad(const ea_layer_norm_t *c, const void *x, const void *dy, const void *weight, const float *mean,
                       const float *rstd, const void *add, void *dx, void *dweight, void *dbias, int32_t accumulate,
                       void *workspace, void *stream);

/* ---- dropout ---------------------------------------------------------------- */

typedef struct ea_dropout {
    int64_t rows;            /* 0 <= rows < 2^31                                      */
    int64_t dim;             /* columns, 1 <= dim <= 2^30                             */
    int64_t x_stride;        /* of x and dx, in [dim, 2^32)                           */
    int64_t y_stride;        /* of y, residual and dy, in [dim, 2^32)                 */
    float p;                 /* share of elements that are dropped, in [0, 1]         */
    int32_t x_type;          /* type of x and dx                                      */
    int32_t y_type;          /* type of y, residual and dy                            */
    uint32_t site;           /* tells the dropouts of one step apart                  */
    uint64_t seed;           /* key of the draws                                      */
} ea_dropout_t;

/* Dropout, with a residual added:
 *     y <- (residual +) (u >= T ? x s : 0),   T = round(65536 p),  s = 65536 / (65536 - T)
 * for 16-bit draws u, so that p is taken to the nearest multiple of 2^-16 and the
 * average of y over the draws is x to binary32's rounding of s.  A dropped element adds 0
 * whatever it is (an infinity or NaN too); with T = 65536 all are dropped.
 * Element n = row * dim + column takes half n & 1 (0: the low one) of word
 * (n >> 1) & 3 of Philox4x32-10 (see ea.h) at counter {lo(n >> 3), hi(n >> 3), t,
 * site} with key {lo(seed), hi(seed)}: nothing is stored, and the gradient
 * draws the same again.  The round and the 8-bit states of AdamW draw from the
 * same generator: give each a seed of its own.
 *   t: the step, in [0, 2^32 - 1]; t_dev (device, one uint32, read, or NULL):
 *   the step is read on the device instead, so that a captured graph drops
 *   others at each replay.
 *   x, residual (device, rows, or NULL), y (device, rows, write; may be residual;
 *   may be x when types and strides are the same). */
int ea_dropout(const ea_dropout_t *c, int64_t t, const uint32_t *t_dev, const void *x, const void *residual, void *y,
               void *stream);

/* Gradient of the dropout in x (that of the residual is dy itself):
 *     dx <- u >= T ? dy s : 0
 * with the draws of ea_dropout for the same t, site, seed, rows and dim.
 *   dy, dx (device, rows, write; may be dy when types and strides are the same). */
int ea_dropout_grad(const ea_dropout_t *c, int64_t t, const uint32_t *t_dev, const void *dy, void *dx, void *stream);

/* ---- gated linear recurrence ------------------------------------------------- */

#define EA_GATE_PLAIN 0      /* a = g,          w = 1                                 */
#define EA_GATE_SIGMOID 1    /* a = sigmoid(g), w = 1 - a                             */

/* Steps between two saved states. */
#define EA_RECURRENCE_BLOCK 64

typedef struct ea_recurrence {
    int64_t batch;           /* sequences, 0 <= batch < 2^31                          */
    int64_t length;          /* steps of each, 0 <= length < 2^31                     */
    int64_t dim;             /* channels, 1 <= dim <= 2^20                            */
    int64_t x_stride;        /* of x and dx, in [dim, 2^32); sequence b's step t is
                                row b * length + t of every array                     */
    int64_t g_stride;        /* of g and dg, in [dim, 2^32)                           */
    int64_t y_stride;        /* of y and dy, in [dim, 2^32)                           */
    int32_t gate;            /* EA_GATE_*                                             */
    int32_t x_type;          /* type of x, y, dx and dy                               */
    int32_t g_type;          /* type of g and dg                                      */
    int32_t reserved;        /* 0                                                     */
} ea_recurrence_t;

/* Bytes of the saved states: batch * ceil(length / 64) * dim floats. */
int64_t ea_recurrence_states_bytes(const ea_recurrence_t *c);

/* Device workspace (bytes) of ea_recurrence and of ea_recurrence_grad: 0 up to
 * 128 steps. */
int64_t ea_recurrence_workspace_bytes(const ea_recurrence_t *c);

/* For every sequence and channel, h in binary32:
 *     h_t <- a_t h_{t-1} + w_t x_t,   y_t <- h_t      t = 0 .. n - 1, h_{-1} = h0
 * where n is the sequence's length: lengths[b] (taken into [0, length]), or
 * `length` without lengths.  Steps from n on are not read and y is 0 there.
 * Sequences are cut into pieces whose gates are multiplied: with plain gates
 * a product over some of the steps that leaves binary32's range gives
 * infinities or NaN, or 0, even where the steps one by one would not.  A product
 * that falls to 0, of any gates, leaves 0 of a finite state and NaN of an infinite
 * one; the states behind an infinity are infinite or NaN.
 * Pieces hand their states on through the workspace, within one launch, and wait
 * for each other: calls that may run at the same time need a workspace each.  (A
 * state that does not come for a good part of a second is taken as NaN.)
 *   g, x (device, batch * length rows), h0 (device, batch * dim floats, or NULL:
 *   zeros), lengths (device, batch int32, or NULL), y (device, batch * length
 *   rows, write), states (device, batch * ceil(length / 64) * dim floats, write;
 *   NULL when no gradient will be asked for): state k of a sequence is h after
 *   its first min(64 k, n) steps, h_last (device, batch * dim floats, write, or
 *   NULL; may be h0): h after n steps, workspace (device,
 *   ea_recurrence_workspace_bytes bytes, 16-byte aligned; NULL when that is 0).
 * Length 1 with h0 = h_last is the step of a sequence that grows a token at a
 * time. */
int ea_recurrence(const ea_recurrence_t *c, const void *g, const void *x, const float *h0, const int32_t *lengths,
                  void *y, float *states, float *h_last, void *workspace, void *stream);

/* Gradient of the recurrence, for dy of every y_t and dh_last of h after n steps:
 *     d_t  = dy_t + a_{t+1} d_{t+1}      (t = n - 1: dy_t + dh_last)
 *     dx_t <- w_t d_t
 *     dg_t <- d_t h_{t-1}                      (EA_GATE_PLAIN)
 *             d_t (h_{t-1} - x_t) a_t w_t      (EA_GATE_SIGMOID)
 *     dh0  <- a_0 d_0                          (n = 0: dh_last)
 * Steps from n on are not read, and dg and dx are 0 there.  h is formed again
 * from the states; y is not needed.
 *   g, x, lengths as in ea_recurrence, states as it left them, dy (device, batch
 *   * length rows), dh_last (device, batch * dim floats, or NULL: zeros), dg, dx
 *   (device, batch * length rows, write), dh0 (device, batch * dim floats,
 *   write, or NULL; may be dh_last), workspace as above. */
int ea_recurrence_grad(const ea_recurrence_t *c, const void *g, const void *x, const float *states,
                       const int32_t *lengths, const void *dy, const float *dh_last, void *dg, void *dx, float *dh0,
                       void *workspace, void *stream);

/* ---- token loss --------------------------------------------------------------- */

#define EA_REDUCE_MEAN 0     /* over the tokens that count                            */
#define EA_REDUCE_SUM 1

typedef struct ea_token_loss {
    int64_t rows;            /* tokens, 0 <= rows < 2^31                              */
    int64_t vocab;           /* logits of a token, 1 <= vocab <= 2^24                 */
    int64_t logits_stride;   /* in [vocab, 2^32)                                      */
    int64_t dlogits_stride;  /* in [vocab, 2^32)                                      */
    float scale;             /* finite factor on the gradient, as a loss scale        */
    int32_t type;            /* type of the logits and their gradient                 */
    int32_t index_bits;      /* 32 or 64: the targets are int32 or int64              */
    int32_t reduction;       /* EA_REDUCE_*                                           */
} ea_token_loss_t;

/* Device workspace (bytes) of ea_token_loss. */
int64_t ea_token_loss_workspace_bytes(const ea_token_loss_t *c);

/* Cross-entropy of every row's softmax with its target, and its gradient in the
 * same pass.  A row whose target lies outside [0, vocab) does not count.
 *     loss[i]    <- log(sum_k exp(logits[i][k])) - logits[i][target]      (0 where it does not count)
 *     count      <- rows that count
 *     total      <- sum of loss, divided by count for EA_REDUCE_MEAN      (0 when count is 0)
 *     dlogits[i] <- (softmax(logits[i]) - onehot(target)) scale, divided by count for EA_REDUCE_MEAN
 *                   (a row of zeros where it does not count)
 * Logits of -infinity have probability 0.  A row that counts and holds NaN or
 * +infinity, or nothing but -infinity, gives NaN in its loss and its whole
 * gradient; what a row holds that does not count has no effect.  Logits are read
 * in whole aligned 16 bytes, so that up to 15 bytes on either side of a row may be
 * read too, with no effect.
 *   logits (device, rows), targets (device, rows), loss (device, rows floats,
 *   write, or NULL), total (device, one float, write), count (device, one int32,
 *   write, or NULL), dlogits (device, rows, write, or NULL; may be logits when
 *   the strides are the same), workspace (device,
 *   ea_token_loss_workspace_bytes bytes, 16-byte aligned). */
int ea_token_loss(const ea_token_loss_t *c, const void *logits, const void *targets, float *loss, float *total,
                  int32_t *count, void *dlogits, void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EA_LAYER_H */
