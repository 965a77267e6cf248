/*
 * pwlq_block.h - the operators around the integer inner product (pwlq_linear_i8)
 * in a transformer block: rows of activations in 8 bits with a step each, the
 * norms before and after a block with its gate and residual scale, and low-rank
 * adapters beside a projection with frozen, packed weights; with the backward
 * passes that training the adapters and the norms takes, which read the same
 * 8-bit rows as activation checkpoints.
 *
 * Conventions: those of pwlq.h (device pointers owned by the caller, work
 * enqueued on `stream`, nothing allocated, pwlq_last_error), and
 *   - T is the number of rows (tokens), at most 2^26.  T = 0 is an empty batch:
 *     nothing is read, and only the gradients of parameters are written (zeros).
 *   - Rows are given as a pwlq_rows: `stride` elements from one row to the next,
 *     the columns of a row next to each other, so a block of columns of a wider
 *     matrix can be passed as it stands.  Outputs must not overlap inputs or
 *     each other, where a call does not say otherwise.
 *   - A workspace-size query that answers 0 means that the call takes NULL.
 *   - Sums, norms and gradients of parameters are held in binary32; a value is
 *     rounded to a narrower type once, where it is stored.
 *   - 8-bit rows: value = code * step[row], symmetric, codes -127..127.
 *     pwlq_linear_i8 takes the codes with s_x = 1 and z_x = 0; the row's step is
 *     then a factor of its output (pwlq_adapter's base.step).
 */
#ifndef PWLQ_BLOCK_H
#define PWLQ_BLOCK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PWLQ_F32 = 0, PWLQ_BF16 = 1, PWLQ_F16 = 2, PWLQ_I8 = 3 } pwlq_type;

/* A matrix of T rows.  data NULL: the argument is left out, where a call allows
 * it.  step: T binary32 factors of the rows; needed with PWLQ_I8, else NULL
 * unless the call says otherwise. */
typedef struct {
    void *data;
    float *step;
    int64_t stride;
    int type;
} pwlq_rows;

/*
 * Rows to 8 bits: a = max|x| of the row, code = rne(x * (127/a)),
 * step = a/127 (the quotients rounded to binary32 first).  A row with
 * a < 2^-100 gets step 0 and codes 0; a row with a NaN or an infinity gets step
 * NaN and codes 0, so that it stays a row of NaN.  x: PWLQ_F32, PWLQ_BF16 or
 * PWLQ_F16, K columns, 1 <= K <= 65536; codes [T, K] and step [T].
 * pwlq_unpack_rows writes code * step to out (PWLQ_F32, PWLQ_BF16, PWLQ_F16).
 */
int pwlq_pack_rows(const pwlq_rows *x, int64_t T, int64_t K, int8_t *codes, float *step, void *stream);
int pwlq_unpack_rows(const int8_t *codes, const float *step, int64_t T, int64_t K, const pwlq_rows *out,
                     void *stream);

/*
 * Between two blocks: the norm after one, its gate and residual scale, the
 * residual sum and the norm before the next, for rows of D columns:
 *     v     = f * post_weight / sqrt(mean(f^2) + eps)      (f, if post_weight is NULL)
 *     x_out = x + alpha * gate * v
 *     u     = x_out * pre_weight / sqrt(mean(x_out^2) + eps)
 * The sums use x_out before it is rounded.  f (the block's output) may be left
 * out: then x_out is not written and u is the norm of x.
 *   gate       gate_rows x D values of f's type, NULL for 1; gate_rows divides T
 *              and row t uses gate row t / (T / gate_rows): one gate for all rows,
 *              one per sequence of T/gate_rows tokens, or one per token
 *   x, x_out   one type; f's type or PWLQ_F32.  x_out may be x itself
 *   f          PWLQ_F32, PWLQ_BF16 or PWLQ_F16
 *   u          f's type (x's type where f is left out), or PWLQ_I8 with u.step:
 *              codes and steps of u as pwlq_pack_rows defines them, from u
 *              before it is rounded
 * post_weight, pre_weight: D binary32 values.  1 <= D <= 16384.
 */
typedef struct {
    int64_t T, D;
    pwlq_rows x, f, x_out, u;
    const float *post_weight, *pre_weight;
    const void *gate;
    int64_t gate_rows;
    float alpha, eps;
} pwlq_norm_args;

int pwlq_norm_block(const pwlq_norm_args *args, void *stream);

/*
 * Its backward pass: from du and dx_out, the gradients with respect to u and
 * x_out (either may be left out: zero), the gradients
 *     dx      of x (and of x_out in all), type of dx_out or, without it, of x
 *     df      of f, type of du (without it of f, as the forward pass had it)
 *     d_pre   [D], d_post [D] (NULL where there is no post_weight), d_gate
 *             [gate_rows, D] (NULL where there is no gate): binary32
 * x_out and f are the forward pass's, either both as they were or both as 8-bit
 * rows (PWLQ_I8, with steps).  gate has df's type.  With f left out there is
 * only the norm: dx and d_pre.
 * Workspace: device, 256-byte aligned,
 * pwlq_norm_block_backward_workspace_bytes(T, D, gate_rows) bytes.
 */
typedef struct {
    int64_t T, D;
    pwlq_rows du, dx_out, x_out, f, dx, df;
    const float *post_weight, *pre_weight;
    const void *gate;
    int64_t gate_rows;
    float alpha, eps;
    float *d_pre, *d_post, *d_gate;
} pwlq_norm_backward_args;

size_t pwlq_norm_block_backward_workspace_bytes(int64_t T, int64_t D, int64_t gate_rows);
int pwlq_norm_block_backward(const pwlq_norm_backward_args *args, void *workspace, size_t workspace_bytes,
                             void *stream);

/*
 * Low-rank adapters of many requests beside a shared projection.  Row t uses
 * adapter a = ids[t]; an id outside [0, adapters) means none.
 *     h[t]   = scale[a] * x[t] down[a]^T      (R values; 0 without an adapter)
 *     out[t] = base.step[t] * base[t] + h[t] up[a]
 *   x      K columns: weight_type, or PWLQ_I8 with steps
 *   down   [adapters, R, K], up [adapters, R, N]: weight_type (PWLQ_F32,
 *          PWLQ_BF16 or PWLQ_F16), both with the rank before the columns
 *   base   N columns, any type but PWLQ_I8, or left out (0); base.step a factor
 *          of each row, or NULL: with it the output of pwlq_linear_i8 on 8-bit rows
 *          is taken as it is
 *   out    N columns, any type but PWLQ_I8; may be base itself
 *   h      [T, R] binary32: kept for the backward pass
 * Rows without an adapter, and rows of another adapter, are not touched by an
 * adapter's infinities or NaN (its own rows get NaN where the product of such a
 * value may have been an infinity).  1 <= R <= 256, 1 <= adapters <= 65535, K, N
 * and strides up to 2^20, an adapter (R K or R N values) below 2 GiB.
 * Workspace: device, 256-byte aligned, pwlq_adapter_workspace_bytes(T, K, R).
 */
typedef struct {
    int64_t T, K, N;
    int R, adapters, weight_type;
    const void *down, *up;
    const int32_t *ids;
    const float *scale;
    pwlq_rows x, base, out;
    float *h;
} pwlq_adapter_args;

size_t pwlq_adapter_workspace_bytes(int64_t T, int64_t K, int R);
int pwlq_adapter(const pwlq_adapter_args *args, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Its backward pass from dy, the gradient with respect to out (weight_type):
 *     dh[t]     = scale[a] * dy[t] up[a]^T
 *     d_up[a]   = sum over rows of a: h[t] (x) dy[t]       [adapters, R, N]
 *     d_down[a] = sum over rows of a: dh[t] (x) x[t]       [adapters, R, K]
 *     dx[t]     = dx_base[t] + dh[t] down[a]
 * x is read as pwlq_adapter read it, or from an 8-bit checkpoint of it.
 * dx_base (the gradient that the shared projection passes on) and dx are of any
 * type but PWLQ_I8; dx_base may be left out (0), or be dx itself.  d_down and
 * d_up are binary32; an adapter without rows gets zeros.
 * Workspace: device, 256-byte aligned,
 * pwlq_adapter_backward_workspace_bytes(T, K, N, R, adapters) bytes.
 */
typedef struct {
    int64_t T, K, N;
    int R, adapters, weight_type;
    const void *down, *up;
    const int32_t *ids;
    const float *scale;
    pwlq_rows dy, x, dx_base, dx;
    const float *h;
    float *d_down, *d_up;
} pwlq_adapter_backward_args;

size_t pwlq_adapter_backward_workspace_bytes(int64_t T, int64_t K, int64_t N, int R, int adapters);
int pwlq_adapter_backward(const pwlq_adapter_backward_args *args, void *workspace, size_t workspace_bytes,
                          void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PWLQ_BLOCK_H */
