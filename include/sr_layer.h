/*
 * sr_layer.h -- layers over pixels or tokens, their gradients, and the clipping of all gradients: an
 * extension beyond the paper.  What stands between a network's features and the coefficients that the
 * other headers take (SR_COEFF_PIXEL_MAJOR), and behind the gradients that sr_list_route_grad and
 * sr_dict_assemble_list_grad send back.
 *
 * A row is the features of one pixel or token.  Rows are stored one after the other: [N][H][W][C], a
 * tensor described with n = N, h = H, w = W, c = C as SR_COEFF_PIXEL_MAJOR asks; only N*H*W, the number
 * of rows, matters.  With x_p the C features of row p, weight W, bias b:
 *
 *     linear   z = x W^T + b                     y = act(z) + residual
 *     gated    g = x Wg^T + bg, u = x Wu^T + bu  y = act(g) u         (W = Wg on top of Wu, b = bg, bu)
 *
 * All tensors of a call have one type, f32, f16 or bf16.  Products are summed in fp32 or better; those of 16-bit values
 * are exact, those of f32 values are within 2^-24 of themselves (large calls hold an f32 value below 2^-110 to 2^-134, as
 * three bfloat16 numbers).  Bias, activation and the rest are fp32; each output is rounded once.  Silu and sigmoid are within
 * (1.75 |z| + 8) 2^-24 of themselves, gelu within 0.75e-7 |z| (Abramowitz and Stegun 7.1.26), in its tail 5e-5 of its value at
 * z = -3, 2e-3 at -5, 3e-2 at -8.
 *
 * z's gradient, where an activation or a gate makes it, is an operand of two more products: f16 and bf16 calls of up to
 * 2e9 operations a product (2 rows x in x rows of the weight) hold it in two numbers of their type, to 2^-17 of itself or better
 * (f16: or 2^-25), larger ones round it once, as the next layer of a training step does with what it is given; the
 * bias's gradient is summed before that where it is rounded once.  An f16 gradient of z beyond 65504 is an infinity on that
 * way.  Infinities and NaN in the inputs stay in the rows and columns to which the formulas take them; what an infinity
 * makes there may be NaN.
 *
 * All rules of sr_dict.h hold: contiguous device memory of the caller at any address aligned to its elements (off 16-byte
 * boundaries large layers of 16 bits take some twice as long), every check on the host before anything is launched, its
 * statuses, no allocation, no synchronisation, work
 * enqueued on `stream` of the current device.  Outputs and workspace must not overlap inputs or one
 * another (but see sr_grad_clip).  The result of a call does not change from run to run: every sum has a
 * fixed order.  Calls that are in flight together need workspaces of their own (so do captured graphs
 * that may replay together).
 */
#ifndef SR_LAYER_H
#define SR_LAYER_H

#include <stddef.h>

#include "sr_dict.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SR_MAX_FEATURES 65536    /* most features of a row, in or out         */
#define SR_MAX_GRADS    4096     /* most tensors of a sr_grad_clip call       */

typedef enum {
    SR_ACT_NONE    = 0,        /* z                                             */
    SR_ACT_RELU    = 1,        /* max(z, 0); its slope at 0 is 0                */
    SR_ACT_GELU    = 2,        /* z (1 + erf(z / sqrt 2)) / 2                   */
    SR_ACT_SILU    = 3,        /* z / (1 + exp(-z))                             */
    SR_ACT_SIGMOID = 4         /* 1 / (1 + exp(-z))                             */
} sr_act;

/* Bytes of DEVICE scratch sr_layer_linear needs for rows of `in` features to `out` (0 where a size or the type is out of range, or where
 * none is needed). */
size_t sr_layer_linear_workspace_bytes(long long rows, int in, int out, int dtype);

/*
 *   x         [N][H][W][C]       features
 *   weight    [1][1][O][C]
 *   bias      [1][1][1][O], or NULL: none
 *   act       sr_act
 *   residual  [N][H][W][O], or NULL: none
 *   y         [N][H][W][O]       written
 *   workspace, workspace_bytes   DEVICE scratch, 16-byte aligned; may be NULL where none is needed
 *
 * 1 <= C, O <= SR_MAX_FEATURES, less than 2^31 - 256 rows.  No rows: a no-op returning SR_OK.
 */
int sr_layer_linear(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* residual,
                    sr_tensor* y, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of DEVICE scratch sr_layer_linear_grad needs (0 where a size, the type or act is out of range). */
size_t sr_layer_linear_grad_workspace_bytes(long long rows, int in, int out, int dtype, int act);

/*
 * Gradient of sr_layer_linear.  z is made anew from x; the residual's gradient is dy itself.
 *
 *     dz = dy act'(z)    dx = dz W    dweight = sum_p dz_p^T x_p    dbias = sum_p dz_p
 *
 *   x, weight, bias, act   as in the forward call (bias is not looked at for SR_ACT_NONE)
 *   dy        [N][H][W][O]
 *   dx        as x, written, or NULL
 *   dweight   as weight, written, or NULL
 *   dbias     [1][1][1][O], written, or NULL; at least one of the three is asked for
 *
 * No rows: dweight and dbias are set to zero.
 */
int sr_layer_linear_grad(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* dy,
                         sr_tensor* dx, sr_tensor* dweight, sr_tensor* dbias,
                         void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of DEVICE scratch sr_layer_gated needs for rows of `in` features to `out`, 2 * out rows of weights (0 as above). */
size_t sr_layer_gated_workspace_bytes(long long rows, int in, int out, int dtype);

/*
 *   weight    [1][1][2F][C]      the gate's F rows, then the other projection's
 *   bias      [1][1][1][2F], or NULL: none
 *   act       sr_act, of the gate
 *   y         [N][H][W][F]       written
 *
 * 1 <= C, F <= SR_MAX_FEATURES; the rest as for sr_layer_linear.
 */
int sr_layer_gated(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, sr_tensor* y,
                   void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of DEVICE scratch sr_layer_gated_grad needs (0 where a size or the type is out of range). */
size_t sr_layer_gated_grad_workspace_bytes(long long rows, int in, int out, int dtype);

/*
 * Gradient of sr_layer_gated: dg = dy u act'(g), du = dy act(g), and dx, dweight, dbias from dz = (dg, du) as for
 * sr_layer_linear_grad.  dy is [N][H][W][F], dweight as weight, dbias [1][1][1][2F]; each of the three may be NULL, not all.
 */
int sr_layer_gated_grad(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* dy,
                        sr_tensor* dx, sr_tensor* dweight, sr_tensor* dbias,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of DEVICE scratch sr_grad_clip needs for so many tensors (0 if there are none or too many). */
size_t sr_grad_clip_workspace_bytes(int tensors);

/*
 * The norm over all elements of all gradients, and the gradients scaled down to a largest norm:
 *
 *     norm = sqrt(sum over all elements of g^2)    factor = max_norm / norm if norm is finite and above max_norm, else 1
 *     out = factor g
 *
 *   grads     HOST array of `tensors` descriptors, any sizes (none too; 2^40 elements at most), each f32, f16 or bf16; the same tensor
 *             twice counts twice.  Where no axes hold its elements (more than 2^31 - 1 in one), a tensor is described as several
 *   outs      HOST array of as many, each with its gradient's type and sizes; a gradient's own memory (in place) or
 *             memory that no gradient and no other output overlaps; or NULL: the norm alone
 *   max_norm  not negative; infinity: nothing is scaled
 *   norm      DEVICE, 2 floats, written: norm, factor
 *   workspace, workspace_bytes   DEVICE scratch, 16-byte aligned
 *
 * The squares are summed so that no finite gradients overflow or vanish.  A norm that is finite but beyond fp32 is written as infinity, with the factor
 * that it has.  Gradients that hold infinities or NaN are left as they are, with a norm that is not finite and a factor of 1, so that a program
 * may skip its step.  1 <= tensors <= SR_MAX_GRADS.  Both arrays are read before the call returns.
 */
int sr_grad_clip(const sr_tensor* grads, const sr_tensor* outs, int tensors, double max_norm, float* norm,
                 void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SR_LAYER_H */
