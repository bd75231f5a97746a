/*
 * ps_tokens.h -- C ABI of the two ends of a network of dense layers (ps_dense.h) that works on tokens: rows of a table
 * for given tokens and their gradient, and log probabilities of given tokens and their gradient.
 *
 *   ps_embedding_*  out[r] = scale * table[token of r], for rows in one group or in many (workers), each group on the
 *                   version of the table that it last pulled; the gradient of every group's table, for instance in
 *                   its row of the server's gradient buffer.
 *   ps_logprob_*    logarithms of the probabilities that logits give to given tokens, the distributions' entropies and
 *                   the most probable alternatives; the gradient of the first two.
 *
 * Conventions are those of ps_dense.h: no call throws, allocates device memory or depends on what an earlier one left in
 * a workspace; work is enqueued on the given stream of the current device; every call can be captured into a graph;
 * nothing is summed by atomics, so the same bytes come out every time; two calls may overlap if their workspaces and outputs
 * differ.  ps_dense_last_error() gives a message for the calling thread's last failing call.
 */
#ifndef PS_TOKENS_H
#define PS_TOKENS_H

#include "ps_dense.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One signed number for each row, of `bytes` (4 or 8) bytes, at data_dev + r * stride * bytes; aligned to its size.
 * stride in elements, 0 .. PS_DENSE_MAX_STRIDE.  What is outside 0 .. vocab - 1 is no token (padding). */
typedef struct {
    const void* data_dev;
    int64_t stride;
    int32_t bytes;
} ps_tokens;

/* One float for each row, at data_dev[r * stride]; a stride of 0 gives all rows the same. */
typedef struct {
    const float* data_dev;
    int64_t stride;
} ps_vector;

/* Groups as in ps_linear: group g has rows offsets[g] .. offsets[g+1] - 1 and uses table table_of_group[g] (NULL: g);
 * offsets_dev NULL: one group of all rows.  Their contents are read by the kernels and cannot be refused: offsets are taken
 * into 0 .. rows, and a table's number to the nearest.  Where offsets do not ascend, a row is in one of the groups that have it or in
 * none, the same to every call: among up to 64 groups in the last one that begins at it or before, if that ends behind it. */
typedef struct {
    int32_t dtype; /* ps_dtype of table, rows and gradients */
    int32_t n_groups, n_tables;
    int64_t rows, vocab, dim; /* backward: n_groups * vocab < 2^31 */
    const int32_t* offsets_dev;
    const int32_t* table_of_group_dev;
    double scale; /* finite; taken to 32 bits */
} ps_embedding;

/* out[r] [dim] = scale * table[token of r] [dim], the product of 32 bits rounded once; a row without a token is 0.  Rows in no group
 * are left as they are.  table [n_tables][vocab][dim], out [rows][dim], which may not overlap. */
PS_API ps_status ps_embedding_forward(const ps_embedding* e, const ps_tokens* tokens, const ps_matrix* table, const ps_matrix* out,
                                      void* hip_stream);

/* dtable[g][v] = scale * sum of dy[r] over the rows r of group g with token v, [n_groups][vocab][dim], summed in 32 bits, 16
 * rows after each other and these sums after each other, more than eight of them in up to sixteen shares (so a group's gradient has the
 * same bits whatever else is in the call), times the scale in 32 bits, and rounded once; tokens that no row has get 0.  n_tables and
 * table_of_group_dev are not looked at.  dtable may not overlap dy or the tokens. */
PS_API ps_status ps_embedding_workspace_bytes(const ps_embedding* e, uint64_t* bytes_out);
PS_API ps_status ps_embedding_backward(const ps_embedding* e, const ps_tokens* tokens, const ps_matrix* dy, const ps_matrix* dtable,
                                       void* workspace_dev, uint64_t workspace_bytes, void* hip_stream);

#define PS_LOGPROB_MAX_TOP 32

typedef struct {
    int32_t dtype; /* ps_dtype of logits and their gradient */
    int32_t top;   /* alternatives: 0 .. PS_LOGPROB_MAX_TOP */
    int64_t rows, vocab;
    double scale; /* logits are multiplied by it (one over a temperature): above 0, at most 2e38 */
} ps_logprob;

/* For each row of logits z [rows][vocab], with u = scale z:
 *   norm [rows][3]            the largest z, L = log(sum exp(u - largest u)), and the entropy
 *   logp [rows]               u[token] - largest u - L; 0 for a row without a token
 *   top_logp, top_tokens      [rows][top]: the most probable tokens and their log probabilities, the lower token first
 *                             among equals; behind the last token with a probability, -infinity and -1.
 * A logit of -infinity has probability 0.  A row of nothing else has -infinity, -infinity and 0 in norm, -infinity as log
 * probability, and no alternatives.  A row with a NaN or +infinity has NaN in what is a number (the largest excepted; NaN is no
 * alternative).  z less the row's largest is formed in 32 bits before the scale.  The sums' order goes by the number of rows and by where
 * a row begins in its 16 bytes.  logp, top_logp and top_tokens may be NULL (the last two for top = 0 only), tokens without logp. */
PS_API ps_status ps_logprob_workspace_bytes(const ps_logprob* l, uint64_t* bytes_out);
PS_API ps_status ps_logprob_forward(const ps_logprob* l, const ps_tokens* tokens, const ps_matrix* logits, float* logp_dev, float* norm_dev,
                                    float* top_logp_dev, int32_t* top_tokens_dev, void* workspace_dev, uint64_t workspace_bytes,
                                    void* hip_stream);

/* dlogits [rows][vocab], rounded once, from the gradients of logp and of the entropy (either may be NULL: zeros), the logits
 * and what the forward pass wrote to norm.  dlogits may be the logits themselves, and no part of them else.  A row of nothing
 * but -infinity has gradient 0, as has a row without a token as far as logp goes. */
PS_API ps_status ps_logprob_backward(const ps_logprob* l, const ps_tokens* tokens, const ps_matrix* logits, const float* norm_dev,
                                     const ps_vector* dlogp, const ps_vector* dentropy, const ps_matrix* dlogits, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PS_TOKENS_H */
