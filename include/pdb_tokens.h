/*
 * pdb token operators: what a model over a vocabulary of tokens needs around
 * the layers between -- the rows of a table that tokens pick and that table's
 * gradient (or its SGD step in place), log probabilities of given tokens with
 * entropies and the best alternatives, their gradient, and distillation from a
 * teacher's top logits with its gradient.  C ABI, same conventions as pdb.h:
 * caller-owned device pointers, work on the caller's stream, PDB_OK or a
 * negative pdb_status, nothing kept past the call.  Every entry point here is
 * asynchronous and can be recorded into a HIP graph (no host wait, no
 * allocation, no memset node).
 *
 * Matrices are row-major with unit column stride and any row stride >= their
 * columns (in elements); data pointers are aligned to their element, no more.
 * Sizes: n, v, d, and n * k (or n * top) < 2^31; offsets inside a matrix are
 * 64-bit.  Matrices, vectors and workspaces do not overlap unless said so.
 *
 * Tokens (int32 or int64): 0 .. v - 1 are rows of the table, or entries of a
 * row of logits.  A negative token is padding.  A token >= v is treated as
 * padding too and, when `status` is not NULL, sets *status to
 * PDB_ERR_INVALID_ARG: status is a device int32 that the caller clears, no
 * call here does, so one word can watch many calls.
 *
 * Arithmetic: binary32 whatever the types, rounded once (to nearest even) where
 * a 16-bit result is stored; what passes its type's range is infinite.  That
 * holds of differences too: in a row whose finite logits lie more than binary32's
 * largest value apart, the lower ones may count as -inf.  The
 * order of every sum follows from the call's sizes and, in pdb_embed_grad, from
 * all of its tokens, so a repeated call gives the same bits.
 */
#ifndef PDB_TOKENS_H
#define PDB_TOKENS_H

#include <stddef.h>
#include <stdint.h>

#include "pdb.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum pdb_dtype { PDB_F32 = 0, PDB_F16 = 1, PDB_BF16 = 2 } pdb_dtype;
typedef enum pdb_index { PDB_I32 = 0, PDB_I64 = 1 } pdb_index;

/* Largest `top` of pdb_token_logprobs and largest `k` of pdb_distill. */
#define PDB_MAX_TOP 128
#define PDB_MAX_TEACHER 1024

/* Rows of a table: out[i][j] = scale * table[tokens[i]][j], zeros where
 * tokens[i] is padding.  table: device, v x d, row stride ld, of `dtype`;
 * tokens: device, [n], of `index`; out: device, n x d, row stride ldo, of
 * out_dtype. */
int pdb_embed_lookup(const void *table, int dtype, int64_t ld, int64_t v, int64_t d,
                     const void *tokens, int index, int64_t n, float scale, void *out,
                     int out_dtype, int64_t ldo, int32_t *status, hipStream_t stream);

/* Device workspace (bytes) of pdb_embed_grad for n tokens, v table rows and d
 * columns.  Host-only arithmetic. */
int pdb_embed_grad_workspace_bytes(int64_t n, int64_t v, int64_t d, size_t *bytes);

/* The gradient of pdb_embed_lookup by its table, from the gradient dy by its
 * output (device, n x d, row stride ldy, of `dtype`):
 *   grad[t] = scale * sum of dy[i] over the i with tokens[i] = t,
 * and zeros in the rows that no token picked; with accumulate = 1 the sum is
 * added to what grad holds and the other rows are left alone.  With grad the
 * table itself and scale = -lr times the lookup's scale that is the gradient
 * step of Sec. 2 on the rows that the batch used (Definition 3: every read of
 * the batch before its writes).  grad: device, v x d, row stride ldg, of
 * grad_dtype.  A token's rows are summed in ascending i, in runs, then the runs'
 * sums.  Where the runs end depends on how many rows the smaller tokens have: a
 * row's last bits may differ between batches that differ in other tokens only.
 * ws: at least pdb_embed_grad_workspace_bytes(n, v, d). */
int pdb_embed_grad(const void *dy, int dtype, int64_t ldy, const void *tokens, int index,
                   int64_t n, void *grad, int grad_dtype, int64_t ldg, int64_t v, int64_t d,
                   float scale, int accumulate, int32_t *status, void *ws, size_t ws_bytes,
                   hipStream_t stream);

/* Device workspace (bytes) of pdb_token_logprobs.  Host-only arithmetic. */
int pdb_token_logprobs_workspace_bytes(int64_t n, int64_t v, int32_t top, size_t *bytes);

/* Log probabilities under softmax(logits / temp) (temp > 0 and finite), row by
 * row of logits (device, n x v, row stride ldz, of `dtype`):
 *   logp[i]      of tokens[i] (device, [n], of `index`);
 *   entropy[i]   -sum_j p_ij log p_ij (0 log 0 = 0);
 *   stats[2 i]   m_i, the largest logit; stats[2 i + 1] log of the sum over j
 *                of exp((z_ij - m_i) / temp): what pdb_token_logprobs_grad takes;
 *   top_id[i][0 .. top), top_logp[i][0 .. top): the entries with the largest
 *                logits, largest first and ties to the lowest index, and their
 *                log probabilities (0 <= top <= min(v, PDB_MAX_TOP)).
 * All outputs are device float or int32 arrays; each of logp, entropy, stats,
 * top_id and top_logp may be NULL.  tokens may be NULL when logp is.  Where
 * tokens[i] is padding the row is not read: logp and entropy 0, stats (0, 0),
 * top_id -1, top_logp -inf.  Logits of -inf have probability 0.  A row of
 * nothing but -inf has no distribution: logp and top_logp -inf, entropy 0,
 * stats (0, -inf), top_id the lowest indices.  A NaN or +inf in a row makes
 * its numbers NaN (in top_id NaN ranks below -inf).
 * ws: at least pdb_token_logprobs_workspace_bytes(n, v, top). */
int pdb_token_logprobs(const void *logits, int dtype, int64_t ldz, int64_t n, int64_t v,
                       const void *tokens, int index, float temp, float *logp, float *entropy,
                       float *stats, int32_t top, int32_t *top_id, float *top_logp,
                       int32_t *status, void *ws, size_t ws_bytes, hipStream_t stream);

/* The gradient by the logits of  sum_i d_logp[i] logp[i] + d_entropy[i] entropy[i]
 * (device, [n] each; either may be NULL):  with q the probabilities,
 *   dlogits[i][j] = (d_logp[i] (1[j = tokens[i]] - q_ij)
 *                    - d_entropy[i] q_ij (log q_ij + entropy[i])) / temp.
 * stats and entropy as pdb_token_logprobs gave them for the same logits and
 * temp (entropy may be NULL when d_entropy is; tokens may be NULL when d_logp
 * is).  Zeros in rows whose token is padding or that hold nothing but -inf.
 * dlogits: device, n x v, row stride ldd, of the logits' type; it may be the
 * logits themselves (same pointer and row stride). */
int pdb_token_logprobs_grad(const void *logits, int dtype, int64_t ldz, int64_t n, int64_t v,
                            const void *tokens, int index, float temp, const float *stats,
                            const float *entropy, const float *d_logp, const float *d_entropy,
                            void *dlogits, int64_t ldd, int32_t *status, hipStream_t stream);

/* Device workspace (bytes) of pdb_distill.  Host-only arithmetic. */
int pdb_distill_workspace_bytes(int64_t n, int64_t v, size_t *bytes);

/* Distillation from a teacher's k best logits per row (1 <= k <=
 * PDB_MAX_TEACHER): with p = softmax(teacher[i] / temp) over the row's k
 * entries and q = softmax(logits[i] / temp) over the vocabulary,
 *   loss[i] = weight[i] * sum_j p_j (log p_j - log q_{ids[i][j]})   (0 log 0 = 0),
 * and, unless dlogits is NULL, the gradient of sum_i loss[i]:
 *   dlogits[i][u] = (weight[i] / temp) (q_u - sum_{j: ids[i][j] = u} p_j).
 * logits: device, n x v, row stride ldz, of `dtype`; ids: device, n x k int32
 * and teacher: device, n x k of teacher_dtype, both without gaps (pdb_token_logprobs'
 * top_id and top_logp are such: any logits that differ from the teacher's by a
 * constant per row serve); a negative id is no entry.  weight: device, [n], or
 * NULL for ones.  temp > 0 and finite.  A row without entries (or whose
 * entries' teacher logits are all -inf), or of weight 0, has loss 0 and
 * gradient 0 whatever its logits; the ids of a row of weight 0 may hold
 * anything.  A logit of -inf where p > 0 makes the loss +inf (the gradient stays
 * finite).  dlogits: device, n x v, row stride ldd, of the logits' type; it may
 * be the logits themselves (same pointer and row stride).  status as for
 * tokens, for ids >= v in rows of other weights.  ws: at least
 * pdb_distill_workspace_bytes(n, v). */
int pdb_distill(const void *logits, int dtype, int64_t ldz, int64_t n, int64_t v,
                const int32_t *ids, const void *teacher, int teacher_dtype, int32_t k, float temp,
                const float *weight, float *loss, void *dlogits, int64_t ldd, int32_t *status,
                void *ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PDB_TOKENS_H */
