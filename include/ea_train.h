/*
 * ea_train.h -- the part of libea's C ABI beside the round of ea.h: AdamW over
 * many tensors with states in 32 or 8 bits, the global gradient norm that
 * clips it, and the embedding lookup with its gradient.
 *
 * The conventions of ea.h hold: device memory is the caller's, work is
 * enqueued on `stream` and the call returns without waiting, arguments are
 * checked before anything is enqueued, EA_OK or a negative EA_ERR_* is
 * returned and ea_last_error() describes the last failure of the thread.
 * Every result is the same, bit for bit, from run to run.
 *
 * Element types: EA_F32, EA_BF16, EA_F16.  A device pointer is aligned to its
 * element's size (else EA_ERR_ALIGN); vectors need no alignment beyond that.
 * All arithmetic is binary32 or wider; a result in 16 bits is rounded to
 * nearest even once, at the end.
 */
#ifndef EA_TRAIN_H
#define EA_TRAIN_H

#include <stdint.h>

#include "ea.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EA_F32 0
#define EA_BF16 1
#define EA_F16 2

#define EA_ROUND_NEAREST 0       /* to nearest even                                */
#define EA_ROUND_STOCHASTIC 1    /* up with probability equal to the fraction      */

/* Elements that share one scale of the 8-bit states. */
#define EA_STATE_BLOCK 256

/* One tensor of n elements (dense, any order as long as all arrays share it).
 * Arrays of different tensors, or of one, may not overlap. */
typedef struct ea_tensor {
    const void *g;           /* (device, n, read) gradient                            */
    void *p;                 /* (device, n, read/write) parameter                     */
    void *m;                 /* (device, n, read/write) first moment                  */
    void *v;                 /* (device, n, read/write) second moment, or its root    */
    float *m_scale;          /* (device, ceil(n/256), read/write) 8-bit states only   */
    float *v_scale;          /* (device, ceil(n/256), read/write) 8-bit states only   */
    float *master;           /* (device, n, read/write) binary32 copy of a 16-bit p,
                                or NULL: p itself is then widened and updated         */
    int64_t n;               /* elements, 0 <= n < 2^40                               */
    float weight_decay;      /* finite, >= 0                                          */
    float lr_scale;          /* factor on the learning rate, finite, >= 0             */
} ea_tensor_t;

typedef struct ea_adamw {
    float lr;                /* finite, >= 0                                          */
    float beta1;             /* in [0, 1)                                             */
    float beta2;             /* in [0, 1)                                             */
    float eps;               /* finite, > 0                                           */
    int32_t param_type;      /* EA_F32, EA_BF16, EA_F16: type of every p              */
    int32_t grad_type;       /* type of every g                                       */
    int32_t state_bits;      /* 32 or 8                                               */
    int32_t rounding;        /* EA_ROUND_*, of 8-bit states (32: EA_ROUND_NEAREST)    */
    uint64_t seed;           /* key of the stochastic rounding's draws                */
} ea_adamw_t;

/* One AdamW step (Loshchilov and Hutter: decoupled weight decay, bias
 * correction) over ntensors tensors, t >= 1 the step.  With s = *gscale (1
 * when gscale is NULL), lr_i = lr * lr_scale, every operation rounded to
 * binary32 by itself (with 8-bit states but for the root and the quotient, see below):
 *     g <- g * s
 *     m <- beta1 m + (1 - beta1) g
 *     v <- beta2 v + (1 - beta2) (g g)
 *     p <- p (1 - lr_i wd) - (lr_i / (1 - beta1^t)) (m / (sqrt(v) (1 / sqrt(1 - beta2^t)) + eps))
 * where the factors in parentheses that hold no element are formed in
 * binary64 and rounded once.  With a master the update is the master's and p
 * its rounding (p is not read).  If *gscale is not finite the call changes
 * nothing: a step whose gradients overflowed is skipped without the host.
 *
 * The states start at zero: zeroed memory, whatever state_bits is.
 *
 * 8-bit states.  m holds E4M3 codes (OCP 8-bit floating point, 1-4-3) and v
 * those of the root r of the second moment; element k is code * scale[k/256].
 * Both are widened, stepped and used for p in binary32, and rounded only to be
 * kept: scale = max|x| * (1/448) over the block, code = x * (1/scale) rounded to E4M3.
 *   - The square root of v and the quotient in p may each be one unit in the
 *     last place off the rounded result (in practice one in a million is).
 *     They are the rounded ones for blocks past the last multiple of 512
 *     elements, and near values that are subnormal, infinite or NaN.
 *   - A block whose scale falls under 2^-126 is kept as zeros.
 *   - Second moments are binary32 between reading and keeping them: roots
 *     under 2^-63 square to subnormal numbers and lose digits, then vanish.
 *   - A positive root never gets the code 0 (it would leave m / eps): the
 *     smallest code, 2^-9 of the scale, takes its place.
 *   - An infinity or NaN in a block, or a NaN among its codes, makes the
 *     block's scale NaN: it shows.
 *   - EA_ROUND_STOCHASTIC: codes between two neighbours go up with the
 *     probability of the fraction, from 16 bits.  To nearest, a relative change
 *     of a state by less than half a code step (3 to 6%) is lost every time,
 *     and 1 - beta2 is less than that; with draws the states follow their
 *     averages.  Element n of tensor i at step t takes word n&3 of Philox4x32-10
 *     applied to counter {lo(n>>2), hi(n>>2), t, i} with key {lo(seed),
 *     hi(seed)} (see ea.h): the high 16 bits for m, the low ones for r.
 *
 * tensors (host, ntensors) is read during the call.  0 <= ntensors <=
 * 2^22, fewer than 2^40 elements in all.  gscale (device, one float, or NULL). */
int ea_adamw_step(const ea_adamw_t *c, int64_t t, int32_t ntensors, const ea_tensor_t *tensors, const float *gscale,
                  void *stream);

/* The same with the step read on the device, and lr, beta2 from the schedule
 * (EA_SCHED_CONSTANT: c's), as ea_step_scheduled: t_dev (device, one uint32,
 * read/write) holds t >= 1 and is left at t + 1, also when a step is skipped.
 * Nothing on the host depends on t: the call can be captured in a HIP graph. */
int ea_adamw_step_scheduled(const ea_adamw_t *c, const ea_schedule_t *s, uint32_t *t_dev, int32_t ntensors,
                            const ea_tensor_t *tensors, const float *gscale, void *stream);

/* Device workspace (bytes) of ea_grad_norm for these tensors. */
int64_t ea_grad_norm_workspace_bytes(int32_t ntensors, const ea_tensor_t *tensors);

/* Global norm of the gradients (`g` and `n` of each tensor; the other fields
 * are not looked at) of type grad_type, summed in binary64:
 *     norm   <- scale * sqrt(sum of squares)
 *     gscale <- scale * (max_norm < norm ? max_norm / norm : 1)
 * `scale` (finite, > 0) undoes a loss scale or averages accumulated gradients;
 * max_norm > 0, infinity for no clipping.  Where the norm is not finite,
 * gscale is NaN, and ea_adamw_step with it changes nothing.
 *   norm, gscale (device, one float each, write; gscale may be NULL),
 *   workspace (device, ea_grad_norm_workspace_bytes bytes, 8-byte aligned;
 *   NULL when that is 0). */
int ea_grad_norm(int32_t grad_type, int32_t ntensors, const ea_tensor_t *tensors, float scale, float max_norm,
                 float *norm, float *gscale, void *workspace, void *stream);

/* ---- embedding ------------------------------------------------------------ */

typedef struct ea_embed {
    int64_t tokens;          /* ids, 0 <= tokens < 2^30                               */
    int64_t vocab;           /* rows of the table, 1 <= vocab < 2^31 - 1              */
    int64_t dim;             /* columns, 1 <= dim <= 2^20                             */
    int64_t table_stride;    /* elements from one row of the table (gradient) to the
                                next, >= dim, < 2^32                                  */
    int64_t x_stride;        /* the same for the tokens' rows                         */
    int64_t padding;         /* id that gets no gradient, or any value outside
                                [0, vocab) for none                                   */
    float scale;             /* finite factor on the rows, and on their gradient      */
    int32_t table_type;      /* type of the table and of its gradient                 */
    int32_t x_type;          /* type of the tokens' rows and of their gradient        */
    int32_t index_bits;      /* 32 or 64: the ids are int32 or int64                  */
} ea_embed_t;

/* x[i] <- scale * table[ids[i]] for every token; a zero row for an id outside
 * [0, vocab).  table (device, vocab rows), ids (device, tokens), x (device,
 * tokens rows, write; elements between rows are left alone). */
int ea_embed_lookup(const ea_embed_t *c, const void *table, const void *ids, void *x, void *stream);

/* Device workspace (bytes) of ea_embed_grad. */
int64_t ea_embed_workspace_bytes(const ea_embed_t *c);

/* Gradient of the lookup:
 *     dtable[k] <- scale * (sum of dx[i] over the tokens i with ids[i] = k)   (+ dtable[k] when accumulate is 1)
 * The ids are sorted (stably), each row's terms added in binary32 in an order
 * that the ids alone fix, the existing row added last.  Tokens whose id is
 * `padding` or outside [0, vocab) contribute nothing and their dx rows are not
 * read.  Without accumulate every row of dtable is written, rows without
 * tokens with zeros; with it rows without tokens are not touched.
 *   ids (device, tokens), dx (device, tokens rows), dtable (device, vocab rows,
 *   write or read/write), workspace (device, ea_embed_workspace_bytes bytes,
 *   16-byte aligned; NULL when that is 0; its contents do not matter).  The
 *   arrays may not overlap, and calls that share a workspace are ordered by the
 *   caller. */
int ea_embed_grad(const ea_embed_t *c, const void *ids, const void *dx, void *dtable, int32_t accumulate,
                  void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EA_TRAIN_H */
