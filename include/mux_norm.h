/*
 * mux_norm.h -- C ABI of the layer norm of a chunk-aligned batch, every task with its own weights.
 *
 * Between the projections of a decoder block the rows of the aligned batch are normalised; each task may train norm
 * weights of its own beside (or instead of) its adapters, or all of them point at the backbone's frozen ones:
 *     y_i = (x_i - mean_i) * rstd_i * gamma_t + beta_t ,   mean_i = sum_n x_i[n] / N ,
 *     rstd_i = 1 / sqrt(sum_n (x_i[n] - mean_i)^2 / N + eps)              (row i of task t)
 * Backward, with xh_i = (x_i - mean_i) rstd_i and h_i = dy_i * gamma_t:
 *     dx_i = rstd_i (h_i - sum_n h_i[n] / N - xh_i sum_n h_i[n] xh_i[n] / N)
 *     dgamma_t = sum_i dy_i * xh_i ,   dbeta_t = sum_i dy_i               (rows of task t only)
 *
 * Conventions as in mux.h (table, streams, workspaces, errors, bit-identical repeats).  X, dX are device [T, width] with
 * ldx elements between rows, Y, dY [T, width] with ldy, all of the storage type `dtype`, as are gamma_t and beta_t [width].
 * Statistics, sums and the gradients dgamma_t, dbeta_t are fp32 in both types.  Rows of padding: their content is ignored, Y
 * and dX are written as zero there.  Any width from 1 to MUX_NORM_MAX_WIDTH, any leading dimension >= width, any
 * pointers aligned to their element, fewer than 2^24 rows.  What lies between a row's width and its leading dimension is left as
 * it is.
 * Y may be X itself and dX may be X or dY itself (same pointer, same leading dimension); other overlaps of what is
 * written with what is read, and dgamma / dbeta buffers that overlap each other, are refused (MUX_ERR_INVALID_ARG).
 */
#ifndef MUX_NORM_H_
#define MUX_NORM_H_

#include <stddef.h>
#include <stdint.h>

#include "mux.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MUX_NORM_MAX_WIDTH 32768

typedef struct {
  int32_t width;            /* N                                                                */
  int32_t dtype;            /* mux_dtype                                                        */
  float eps;                /* > 0, finite                                                      */
  int64_t ldx, ldy;         /* elements between rows of X (and dX), Y (and dY), >= width        */
  int32_t n_tasks;          /* must equal the table's                                           */
  const void* const* gamma; /* host array of n_tasks device pointers; a NULL array or entry: 1  */
  const void* const* beta;  /* host array of n_tasks device pointers; a NULL array or entry: 0  */
} mux_norm_desc;

/* Bytes of `saved` (forward -> backward: mean and rstd of every row, fp32 [2][T]) and of the backward's workspace (partial
 * sums of the weights' gradients).  Host arithmetic; 0 for a null argument or a width out of range. */
size_t mux_norm_saved_bytes(const mux_norm_desc* desc, const mux_segtab* st);
size_t mux_norm_workspace_bytes(const mux_norm_desc* desc, const mux_segtab* st);

/* Forward.  `saved` may be NULL when no backward pass follows. */
mux_status mux_norm_forward(const mux_norm_desc* desc, const mux_segtab* st, const void* dev_segtab, const void* X, void* Y,
                            void* saved, void* hip_stream);

/* Backward.  dX may be NULL to skip it; dgamma, dbeta: host arrays of n_tasks device pointers to fp32 buffers [width], a
 * NULL array or entry skips that gradient (with nothing of the two wanted `ws` may be NULL).  accumulate = 0 overwrites
 * them (with zero for a task without tokens), 1 adds to what they hold.  `saved` is the forward's. */
mux_status mux_norm_backward(const mux_norm_desc* desc, const mux_segtab* st, const void* dev_segtab, const void* X,
                             const void* dY, const void* saved, void* dX, void* const* dgamma, void* const* dbeta,
                             int accumulate, void* ws, size_t ws_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MUX_NORM_H_ */
