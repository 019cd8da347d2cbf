/*
 * lossy_local.h -- C ABI of the workers' local gradients on one MI355X
 * (gfx950): the operators of a language model that read a worker's replica
 * row, write its gradient row, or keep activations between the two.
 *
 * Section 3 step (1) of "Distributed Training under Packet Loss" has each
 * worker W_i take the gradient of its loss on its own, possibly stale,
 * replica.  lossy.h takes it from there (gradient rows in, replica rows
 * out); the entry points here stand on the other side of the same buffers:
 *
 *   ll_embed        embedding lookup in every worker's replica, with scaling
 *   ll_embed_grad   its gradient, by sorted tokens, into the gradient rows
 *   ll_act_pack     8-bit checkpoint of activations (forward pass)
 *   ll_act_unpack   the activations back (backward pass)
 *   ll_act_wgrad    a linear layer's weight gradient straight from the 8-bit
 *                   checkpoint of its input, into the gradient rows
 *
 * The conventions of lossy.h hold: device pointers, the caller owns all
 * memory, calls only enqueue kernels on `stream` (and can be captured into a
 * HIP graph), return codes and ll_last_error().  Beyond those:
 *   - `stream` belongs to the calling thread's current device, and so does all
 *     memory.
 *   - n workers (1 to 1024), t token places per worker (0 <= t, n * t < 2^31).
 *     Token data are [n][ld_t] integers of itype (LL_I32 or LL_I64);
 *     activations are [n][t][ld] rows, ld >= their width, worker i's token j
 *     at row i * t + j.  Activations need no more alignment than their
 *     element's; rows on 16-byte boundaries are moved fastest.
 *   - lengths: int32 [n] (device) or NULL.  Worker i's batch has lengths[i]
 *     tokens (below 0 taken as 0, above t as t); NULL stands for t each.  What
 *     lies behind a batch is neither read nor written, columns between the
 *     width and ld neither.
 *   - replicas, grads: the row buffers of lossy.h ([n][ld], 16-byte aligned
 *     rows).  A table or weight is [rows][h], contiguous, starting at element
 *     `offset` of every row, anywhere (offset + rows * h <= ld, no alignment
 *     asked); other elements of the rows are not touched.
 *   - dtypes are LL_F32 or LL_BF16, in any combination.  Sums are fp32, each
 *     result is rounded once, to nearest even, when it is stored.
 *   - outputs may not overlap inputs or the workspace.
 *   - results do not depend on scheduling: the same call gives the same bits.
 *   - workspaces hold nothing between calls and need no initial contents;
 *     calls that share one (two captured graphs as well) must be ordered.
 *     They are 16-byte aligned.
 */
#ifndef LOSSY_LOCAL_H
#define LOSSY_LOCAL_H

#include "lossy.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { LL_I32 = 0, LL_I64 = 1 };

/* Columns of a token that share one scale in an 8-bit checkpoint. */
enum { LL_ACT_GROUP = 32 };

/*
 * Embedding lookup: with id = tokens[i][j] - first,
 *   out[i][j][c] = scale * replicas[i][offset + id * h + c]   0 <= id < v
 *                = 0                                          otherwise
 * (a padding token, or a row that another owner's shard holds: the sum of the
 * lookups over all shards is the lookup in the whole table).
 *   tokens    [n][ld_t] of itype, ld_t >= t.
 *   first     id of the table row at `offset`.
 *   out       [n][t][ld_o] of odtype.
 */
LL_API int ll_embed(int32_t n, int64_t t, int64_t h, int64_t v, int64_t first, int32_t itype,
                    const void* tokens, int64_t ld_t, const int32_t* lengths, int32_t rdtype,
                    const void* replicas, int64_t ld_r, int64_t offset, float scale,
                    int32_t odtype, void* out, int64_t ld_o, void* stream);

/*
 * Gradient of ll_embed with respect to the table, for every row id < v:
 *   grads[i][offset + id * h + c] =
 *       [accumulate: its value +] scale * sum_{j : tokens[i][j] - first = id} dy[i][j][c]
 * Without accumulate every row of the table is written, 0 where no token names
 * it; with accumulate (a table that is also the output layer's weight, or
 * gradients summed over micro-batches) rows that no token names are left
 * alone.  Rows of dy whose token is not in the table are not read.  The
 * order of summation depends only on the tokens and the sizes.
 *   dy         [n][t][ld_y] of ydtype.
 *   workspace  ws_bytes >= ll_embed_grad_workspace_bytes(n, t, h, v).
 */
LL_API int ll_embed_grad(int32_t n, int64_t t, int64_t h, int64_t v, int64_t first,
                         int32_t itype, const void* tokens, int64_t ld_t,
                         const int32_t* lengths, int32_t ydtype, const void* dy, int64_t ld_y,
                         float scale, int32_t gdtype, void* grads, int64_t ld_g, int64_t offset,
                         int32_t accumulate, void* workspace, size_t ws_bytes, void* stream);
LL_API size_t ll_embed_grad_workspace_bytes(int32_t n, int64_t t, int64_t h, int64_t v);

/*
 * 8-bit checkpoint of activations.  Of each token, groups of LL_ACT_GROUP
 * consecutive columns (the last may be short) share a power of two: with a the
 * largest finite |x| of the group,
 *   k = the smallest integer >= -117 with a <= 448 * 2^k   (-117 where a = 0)
 *   s = k + 127                       one byte a group
 *   q = e4m3(x * 2^-k)                one byte an element
 * e4m3 is the 8-bit float with 4 exponent and 3 mantissa bits (largest value
 * 448, no infinity; 0x7F is NaN), rounded to nearest even; what would round to
 * 2^128 stays at 1.875 * 2^127, so a finite x is restored finite.  The restored
 * value differs from x by at most 2^-4 |x|, or 2^(k-10) where that is more
 * (below 2^(k-6)).  An infinite or NaN x becomes NaN and leaves its
 * neighbours' scale alone.
 * With s a power of two every restored value is exact in bf16, so the
 * backward pass multiplies it on the bf16 matrix units with no second
 * rounding; the lower bound on k keeps the values off bf16's subnormals.
 *   x  [n][t][ld_x] of xdtype.
 *   q  uint8 [n][t][ld_q], ld_q >= h;  s  uint8 [n][t][ld_s], ld_s >= ceil(h / 32).
 */
LL_API int ll_act_pack(int32_t n, int64_t t, int64_t h, const int32_t* lengths, int32_t xdtype,
                       const void* x, int64_t ld_x, uint8_t* q, int64_t ld_q, uint8_t* s,
                       int64_t ld_s, void* stream);

/*
 * The activations of an 8-bit checkpoint: out = e4m3 value of q times
 * 2^(s - 127), exact in both dtypes.  Takes what ll_act_pack writes (10 <= s);
 * q, s as there, out [n][t][ld_o] of odtype.
 */
LL_API int ll_act_unpack(int32_t n, int64_t t, int64_t h, const int32_t* lengths,
                         const uint8_t* q, int64_t ld_q, const uint8_t* s, int64_t ld_s,
                         int32_t odtype, void* out, int64_t ld_o, void* stream);

/*
 * Weight gradient of a linear layer y = x W^T (W is [o][h]) from the 8-bit
 * checkpoint (q, s) of its input x:
 *   grads[i][offset + r * h + c] =
 *       [accumulate: its value +] scale * sum_j dy[i][j][r] * x^[i][j][c]
 * with x^ the restored values; products are exact in fp32 (fp32 dy is taken
 * as a sum of three bf16 terms that hold all its bits, but for what lies
 * below 2^-126), sums are fp32.
 *   dy         [n][t][ld_y] of ydtype, ld_y >= o.
 *   q, s       as ll_act_pack writes them.  ld_y, ld_q and ld_s are below 2^24.
 *   workspace  ws_bytes >= ll_act_wgrad_workspace_bytes(n, t, o, h); may be
 *              NULL where that is 0.
 */
LL_API int ll_act_wgrad(int32_t n, int64_t t, int64_t o, int64_t h, const int32_t* lengths,
                        int32_t ydtype, const void* dy, int64_t ld_y, const uint8_t* q,
                        int64_t ld_q, const uint8_t* s, int64_t ld_s, float scale,
                        int32_t gdtype, void* grads, int64_t ld_g, int64_t offset,
                        int32_t accumulate, void* workspace, size_t ws_bytes, void* stream);
LL_API size_t ll_act_wgrad_workspace_bytes(int32_t n, int64_t t, int64_t o, int64_t h);

#ifdef __cplusplus
}
#endif

#endif /* LOSSY_LOCAL_H */
