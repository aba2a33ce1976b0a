/*
 * pdb layer operators: what stands between the token operators of a model that
 * reads more than one token back -- a gated recurrence over sequences with its
 * backward pass -- and the clipping of a step by the norm of all its gradients.
 * C ABI, same conventions as pdb_tokens.h: caller-owned device pointers, work on
 * the caller's stream, PDB_OK or a negative pdb_status, nothing kept past the
 * call; every entry point is asynchronous and can be recorded into a HIP graph;
 * matrices are row-major with unit column stride and any row stride >= their
 * columns, aligned to their element; binary32 arithmetic unless said so, rounded
 * once where a 16-bit result is stored; a repeated call gives the same bits.
 */
#ifndef PDB_LAYERS_H
#define PDB_LAYERS_H

#include "pdb_tokens.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows between two marks of pdb_gated_scan. */
#define PDB_SCAN_MARK 64

/* Device workspace (bytes) of pdb_gated_scan and pdb_gated_scan_grad for n rows
 * of d channels.  Host-only arithmetic. */
int pdb_gated_scan_workspace_bytes(int64_t n, int64_t d, size_t *bytes);

/* A gated linear recurrence along the rows of each sequence, channel by channel:
 *   h_t = f_t h_{t-1} + (1 - f_t) x_t,   f_t = 1 / (1 + exp(-gate_t)),   y_t = h_t,
 * h before a sequence's first row being its row of h0, or 0 where h0 is NULL.
 * x, gate, y: device, n x d, row strides ldx, ldg, ldy, all of `dtype`.
 * The rows hold b sequences one behind another: sequence i is the rows
 * [starts[i], starts[i + 1]) (starts: device, [b + 1] int32, ascending from >= 0
 * to <= n; an empty sequence has equal ones); with starts = NULL each has n / b
 * rows (n a multiple of b; with one row each this is the decoding step).  Rows
 * before the first and behind the last sequence are left as they were in y.
 * Offsets that descend or leave 0 .. n set *status (if status is not NULL; see
 * pdb_tokens.h) to PDB_ERR_INVALID_ARG; what is written then is unspecified, but
 * nothing outside the outputs.
 * h0: device, b x d float without gaps, or NULL.  state: device, b x d float
 * without gaps, or NULL: h after every sequence's last row (its row of h0, or
 * zeros, where the sequence is empty); it may be h0 itself.  marks: device,
 * ceil(n / PDB_SCAN_MARK) x d float without gaps, or NULL: row i is the h that
 * enters row i * PDB_SCAN_MARK, for pdb_gated_scan_grad (unspecified where that
 * row is of no sequence).
 * A NaN, or an infinite x or h0, makes its channel not finite from its row to its
 * sequence's end, and reaches no other sequence.  Infinite gates keep the state, or
 * take the input.
 * n, d, b < 2^31.  ws: at least pdb_gated_scan_workspace_bytes(n, d), aligned to 8,
 * for this call alone until it has run; NULL in the decoding step (n = b, no starts).
 * Tiles of rows pass their states through it.  Where something else writes there
 * meanwhile (another call with the same workspace), what is written is unspecified, but
 * nothing outside the outputs, and a wait ends after 20 s, with NaN and *status =
 * PDB_ERR_DEVICE. */
int pdb_gated_scan(const void *x, int64_t ldx, const void *gate, int64_t ldg, int dtype, int64_t n,
                   int64_t d, const int32_t *starts, int64_t b, const float *h0, void *y,
                   int64_t ldy, float *state, float *marks, int32_t *status, void *ws,
                   size_t ws_bytes, hipStream_t stream);

/* The backward pass: from dy, the gradient by y (device, n x d, row stride lddy),
 * and d_state, that by state (device, b x d float without gaps, or NULL for
 * zeros), the gradients by x and gate (dx, dgate: device, n x d, row strides lddx
 * and lddg) and by h0 (dh0: device, b x d float without gaps, or NULL).  With
 * e_t = dy_t + f_{t+1} e_{t+1} along a sequence, and at its last row e = dy + d_state:
 *   dx_t = (1 - f_t) e_t,   dgate_t = e_t (h_{t-1} - x_t) f_t (1 - f_t),   dh0 = f_1 e_1
 * (d_state for an empty sequence).  The h are computed again, in binary32, from x,
 * gate, h0 and the marks that pdb_gated_scan gave for the same x, gate, starts and
 * h0.  All matrices are of `dtype`.  Rows of no sequence are left as they were in
 * dx and dgate.  A NaN among the gates or dy makes dx, dgate and dh0 of its channel NaN
 * from its row to its sequence's beginning; status and ws as there. */
int pdb_gated_scan_grad(const void *dy, int64_t lddy, const void *x, int64_t ldx, const void *gate,
                        int64_t ldg, int dtype, int64_t n, int64_t d, const int32_t *starts,
                        int64_t b, const float *h0, const float *marks, const float *d_state,
                        void *dx, int64_t lddx, void *dgate, int64_t lddg, float *dh0,
                        int32_t *status, void *ws, size_t ws_bytes, hipStream_t stream);

/* One of many tensors, as a device matrix (a vector has one row). */
typedef struct pdb_tensor {
    void *data;
    int64_t rows, cols, ld;
    int32_t dtype; /* pdb_dtype */
    int32_t reserved;
} pdb_tensor;

/* Device workspace (bytes) of pdb_grad_norm and pdb_grad_clip, whatever the
 * tensors.  Host-only arithmetic. */
int pdb_grad_workspace_bytes(size_t *bytes);

/* The norm of many tensors together: norm[0] (device float) = |scale| times the
 * square root of the sum of the squares of all elements; squares and sums in
 * binary64.  grads: host array of `count` tensors (read during the call), each
 * below 2^40 elements, of any of the types; count < 2^20; 0 for none.  scale
 * (finite): what the gradients are to be multiplied by, 1 / S with a loss scaled by S.
 * ws: at least pdb_grad_workspace_bytes(). */
int pdb_grad_norm(const pdb_tensor *grads, int64_t count, float scale, float *norm, void *ws,
                  size_t ws_bytes, hipStream_t stream);

/* Clipping by the norm of all: with norm as pdb_grad_norm gives it and
 * c = min(1, max_norm / norm),
 *   out_i = step * c * scale * grad_i,
 * or, with accumulate = 1, that added to what out_i holds (clipped gradient
 * descent: out the parameters, step = -lr).  outs: host array of `count` tensors,
 * each with its gradient's rows and columns, of any of the types; an out may be
 * its gradient (same pointer, type and row stride), and shares memory with nothing
 * else that the call reads or writes: PDB_ERR_INVALID_ARG where a tensor without gaps,
 * or the first row of one with, meets another's.  The factor is rounded to binary32
 * once, and the result to out's type.  max_norm >= 0 or +inf; step
 * finite.  Where norm[0] is not finite nothing is written but norm[0]; where the
 * factor is 1 an out that is its gradient is not written.  ws: at least
 * pdb_grad_workspace_bytes(). */
int pdb_grad_clip(const pdb_tensor *grads, int64_t count, float scale, float max_norm, float step,
                  int accumulate, const pdb_tensor *outs, float *norm, void *ws, size_t ws_bytes,
                  hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PDB_LAYERS_H */
