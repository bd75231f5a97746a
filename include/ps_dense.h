/*
 * ps_dense.h -- C ABI of the dense-layer and optimizer operators: what the parameter-server scheme of
 * ps_hotpath.h needs for models made of large dense layers.
 *
 *   ps_linear_*   y = act(x W^T + b) + r and its gradients, for rows of any number, in one group or in
 *                 many (workers), each group on a weight matrix of its own or on the version it last
 *                 pulled; every group's gradients land where the caller wants them, for instance in its
 *                 row of the server's gradient buffer.
 *   ps_adamw_*    one AdamW step over many tensors in one launch, the gradient being the sum of the
 *                 buffered rows, states in 32 bits or in 8.
 *
 * Conventions are those of ps_hotpath.h: every function returns a ps_status and never throws;
 * *_dev pointers are device memory that the caller keeps until the enqueued work is done, *_host
 * pointers host memory; the library allocates no device memory; work is enqueued on the given stream
 * (a hipStream_t, NULL for the default stream) of the current device and is asynchronous, and the
 * caller orders it against work on other streams.  No call depends on what an earlier one left in a
 * workspace, and two calls may overlap if their workspaces and outputs differ.  Every call but
 * ps_adamw_create can be captured into a graph (a captured step repeats its number, rates and scale on every
 * replay, and needs its handle's workspace as long).  Results do not depend on timing: nothing is summed
 * by atomics.  ps_dense_last_error() gives a message for the calling thread's last failing call.
 */
#ifndef PS_DENSE_H
#define PS_DENSE_H

#include "ps_hotpath.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PS_F32 = 0, PS_BF16 = 1, PS_F16 = 2 } ps_dtype;

/* act(z): z; max(z, 0), NaN staying NaN; z Phi(z) with the normal distribution's Phi; z / (1 + exp(-z)).
 * The slope of relu at 0 is 0. */
typedef enum { PS_ACT_NONE = 0, PS_ACT_RELU = 1, PS_ACT_GELU = 2, PS_ACT_SILU = 3 } ps_activation;

/* Matrices in device memory whose rows are contiguous: element (r, c) of matrix g at
 * data_dev[g * matrix + r * row + c], strides in elements, row stride at least the row's length unless
 * there is one row, at most PS_DENSE_MAX_STRIDE.  Data aligned to the element's size. */
typedef struct {
    void* data_dev;
    int64_t row, matrix;
} ps_matrix;

#define PS_DENSE_MAX_STRIDE 4194304 /* elements */
#define PS_DENSE_MAX_ROWS 268435456
#define PS_DENSE_MAX_GROUPS 32768

/* One layer.  Rows are in n_groups consecutive groups: group g has rows offsets[g] .. offsets[g+1] - 1
 * and uses matrix weight_of_group[g] of w and of the bias.  offsets_dev NULL: one group of all rows.
 * weight_of_group_dev NULL: group g uses matrix g.  Both are read by the kernels, so their contents
 * cannot be refused: offsets are taken into 0 .. rows, an end before its beginning is an empty group,
 * and a matrix number outside 0 .. n_weights - 1 is taken to the nearest.  Groups may be empty; rows
 * in no group are left as they are in every output. */
typedef struct {
    int32_t dtype;      /* ps_dtype of every operand and result */
    int32_t activation; /* ps_activation */
    int64_t rows, in_features, out_features;
    int32_t n_groups, n_weights;
    const int32_t* offsets_dev;         /* [n_groups + 1] or NULL */
    const int32_t* weight_of_group_dev; /* [n_groups] or NULL     */
} ps_linear;

/* Device bytes that a forward (backward = 0) or backward call with this layer needs as its workspace: dz, partial sums,
 * and copies of operands whose features are no multiples of 16 bytes, where these make a large product faster. */
PS_API ps_status ps_linear_workspace_bytes(const ps_linear* layer, int32_t backward, uint64_t* bytes_out);

/* z = x W^T + b, y = act(z) + r.  x [rows][in], w [out][in] per matrix, bias [out] per matrix (row stride
 * not used), residual, y and pre [rows][out]; bias, residual and pre may be NULL.  pre receives z, which
 * the backward pass of an activation reads.  y may be the residual itself; no other output may overlap
 * an input or another output.  Sums are held in 32 bits, y and pre are rounded once.  (fp32 operands below
 * 2^-134, which hold 15 bits or fewer, may count as 0 in a sum that they change by less than 2^-80.) */
PS_API ps_status ps_linear_forward(const ps_linear* layer, const ps_matrix* x, const ps_matrix* w, const ps_matrix* bias,
                                   const ps_matrix* residual, const ps_matrix* y, const ps_matrix* pre,
                                   void* workspace_dev, uint64_t workspace_bytes, void* hip_stream);

/* dz = dy act'(z): dx = dz W [rows][in], dw = dz^T x [out][in] and db = sum of dz [out] per group (a group
 * without rows has zeros); each of dx, dw and db may be NULL.  pre (z, as the forward pass wrote it) is
 * not read, and may be NULL, without activation.  The residual's gradient is dy itself.  dz is rounded to
 * the operands' type before the products (matrix instructions take no more), for db it is not. */
PS_API ps_status ps_linear_backward(const ps_linear* layer, const ps_matrix* dy, const ps_matrix* x, const ps_matrix* w,
                                    const ps_matrix* pre, const ps_matrix* dx, const ps_matrix* dw, const ps_matrix* db,
                                    void* workspace_dev, uint64_t workspace_bytes, void* hip_stream);

/* One tensor of an AdamW step.  The gradient of element i is the sum over the buffered rows k, in order,
 * of grad[k * grad_row + i].  States: 32 bits: m and v are float [numel].  8 bits: m and v hold e4m3
 * codes [numel], one byte each, and m_scale and v_scale one float for every PS_ADAMW_BLOCK elements; what
 * is held is code * scale, in m the first moment and in v the ROOT of the second (its range fits 8 bits).
 * All-zero states are the start.  copy, where not NULL, receives the new weights rounded to copy_dtype
 * (the snapshot that workers read). */
typedef struct {
    void* param_dev;
    const void* grad_dev;
    void* copy_dev;
    void *m_dev, *v_dev;
    float *m_scale_dev, *v_scale_dev;
    int64_t numel, grad_row;
    int32_t grad_rows; /* rows that grad_dev has room for, >= 1 */
    int32_t param_dtype, grad_dtype, copy_dtype;
    int32_t state_bits; /* 8 or 32 */
    float weight_decay;
} ps_adamw_tensor;

#define PS_ADAMW_BLOCK 256

typedef struct {
    double lr, beta1, beta2, eps; /* lr >= 0, betas in [0, 1), eps > 0 */
    double grad_scale;            /* the summed gradient is multiplied by it */
    int64_t step;                 /* >= 1: number of this step, for the bias corrections */
    int32_t n_rows;               /* rows to add up: 1 .. every tensor's grad_rows */
} ps_adamw_options;

typedef struct ps_adamw ps_adamw; /* the table of tensors; the tensors stay the caller's */

/* A table of n tensors (n = 0 is allowed) kept in the caller's workspace (16-byte aligned), which must
 * outlive the handle.  Copies the table on the stream and waits for it. */
PS_API ps_status ps_adamw_workspace_bytes(const ps_adamw_tensor* tensors_host, int32_t n, uint64_t* bytes_out);
PS_API ps_status ps_adamw_create(ps_adamw** out, const ps_adamw_tensor* tensors_host, int32_t n, void* workspace_dev,
                                 uint64_t workspace_bytes, void* hip_stream);
PS_API ps_status ps_adamw_destroy(ps_adamw* handle);

/* g = grad_scale * (sum of the rows);  m := beta1 m + (1 - beta1) g;  v := beta2 v + (1 - beta2) g^2;
 * w := w - lr weight_decay w - lr m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps),
 * all in 32 bits, the weights rounded once to their type.  The step uses m and v as computed; an 8-bit
 * state is rounded afterwards: to the nearest code, the largest magnitude of a block to 448, but a root
 * that is not 0 to the least code above 0 at the lowest, so that a later step does not divide by 0.  A
 * block of an 8-bit state with a value that is not finite becomes NaN as a whole. */
PS_API ps_status ps_adamw_step(ps_adamw* handle, const ps_adamw_options* options, void* hip_stream);

/* Message of the calling thread's last failing call of this header ("" if none). */
PS_API const char* ps_dense_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* PS_DENSE_H */
