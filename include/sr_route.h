/*
 * sr_route.h -- per-pixel lists, made and trained: an extension beyond the paper, beside
 * sr_dict_assemble_list (sr_dict.h), which folds such lists.
 *
 * A list keeps `entries` of a pixel's L atoms: a mixture of experts with the dictionary's
 * atoms as the experts.  Here are the router that makes the lists from what the coefficient
 * network hands over, the counts and losses that tell whether the atoms share the load, and
 * the gradients of both steps.  Nothing here knows of images but sr_dict_assemble_list_grad:
 * a pixel may as well be a token (SR_COEFF_PIXEL_MAJOR, one row of W tokens).
 *
 * For a pixel with logits z_l, l < L:
 *     m = max_l z_l,  e_l = exp(z_l - m),  s = sum_l e_l,  p_l = e_l / s,  lse = m + ln s
 *     index_t, t < entries: the atoms by decreasing z, equal ones by increasing l
 * A logit of -infinity masks its atom: p_l = 0, and the atom is listed only where fewer than
 * `entries` others are there, with the value 0.  A pixel with no other logit has values 0 and the
 * atoms 0, 1, ...; it takes no part in counts, shares and losses, and its gradient is 0.
 * -0 and +0 are equal, and either may be listed for the other.  NaN or +infinity logits give unspecified values (and, through the sums,
 * shares and losses), but always different atoms below L.
 *
 * All rules of sr_dict.h hold: device memory of the caller, every check on the host before
 * anything is launched, its statuses, no allocation, no synchronisation, work enqueued on `stream`
 * of the current device.  Outputs must not overlap inputs or one another.  The result of a call
 * does not change from run to run: every sum has a fixed order.  Calls that are in
 * flight together need workspaces of their own (so do captured graphs that may replay together).
 */
#ifndef SR_ROUTE_H
#define SR_ROUTE_H

#include <stddef.h>

#include "sr_dict.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What a list's values are. */
typedef enum {
    SR_ROUTE_SOFTMAX = 0,      /* p of the listed atoms (softmax over all L)       */
    SR_ROUTE_CHOSEN  = 1,      /* softmax over the listed atoms alone              */
    SR_ROUTE_VALUES  = 2       /* the stored values themselves: `coeff` holds
                                  coefficients, the largest are listed as they are
                                  (-infinity too: no atom is masked)               */
} sr_route_kind;

/*
 * The lists of every pixel.
 *
 *   coeff   the network's output, f32, f16 or bf16, in the order coeff_layout says (sr_dict.h):
 *           SR_COEFF_PLANAR [N][L][H][W]; SR_COEFF_PIXEL_MAJOR [N][H][W][L], described with c = L,
 *           h = H, w = W; SR_COEFF_PRE_SHUFFLE [N][L*scale*scale][H/scale][W/scale]
 *   scale   2, 3 or 4 for SR_COEFF_PRE_SHUFFLE; not read otherwise
 *   mask    [N][1][H][W]  SR_U8, or NULL: pixels whose byte is 0 are padding.  Their logits are not
 *           looked at; they get the atoms 0, 1, ... with the value 0
 *   index   [N][entries][H][W]  SR_U8        written, largest first
 *   value   [N][entries][H][W]  f32 or f16   written; computed in fp32 and rounded once
 *
 * 1 <= entries <= L <= SR_MAX_ATOMS.  N = 0 or an empty image is a no-op returning SR_OK.
 * SR_COEFF_BLOCKED and f8 coefficients are SR_ERR_UNSUPPORTED.
 */
int sr_list_route(const sr_tensor* coeff, int L, int scale, int entries, int kind, int coeff_layout,
                  const sr_tensor* mask, sr_tensor* index, sr_tensor* value, void* stream);

/* Bytes of DEVICE scratch sr_list_route_balance needs for L atoms (0 if L is out of range). */
size_t sr_list_route_workspace_bytes(int L);

/*
 * sr_list_route (SR_ROUTE_SOFTMAX or SR_ROUTE_CHOSEN), and in the same pass how the atoms share the load.  With
 * M the number of live pixels (not masked, and with a logit above -infinity):
 *
 *   counts  DEVICE, L + 1 64-bit integers, written: the live pixels whose list holds atom l (with a logit above
 *           -infinity); M
 *   share   DEVICE, L floats, written: (1/M) sum over live pixels of p_l (over all atoms, whatever the kind)
 *   loss    DEVICE, 2 floats, written: the balance loss L sum_l counts_l / (M entries) share_l, which is 1 where
 *           the load is spread evenly; and (1/M) sum over live pixels of lse^2
 *   workspace, workspace_bytes   DEVICE scratch, 16-byte aligned; its contents before and after are meaningless
 *
 * p and lse are formed in fp32; the sums over pixels run in fp32 over at most 4096 pixels and in double from there on.
 * Without a live pixel all of it is 0; an empty call writes that too.
 */
int sr_list_route_balance(const sr_tensor* coeff, int L, int scale, int entries, int kind, int coeff_layout,
                          const sr_tensor* mask, sr_tensor* index, sr_tensor* value,
                          long long* counts, float* share, float* loss,
                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gradient of the two calls above with respect to the logits.  The choice of the atoms, and the counts, are constants.
 *
 *   index   as the forward call wrote it: atoms below L, different within a pixel (else: unspecified values at that
 *           pixel, never an access outside)
 *   dvalue  [N][entries][H][W]  f32 or f16: gradient of the values, or NULL (none)
 *   counts  as sr_list_route_balance wrote it, and
 *   dloss   DEVICE, 2 floats: gradients of the two losses; both NULL: no part of the losses
 *   dcoeff  as coeff, same type and order; written
 *
 *     dz_l = q_l (G_l - sum_j q_j G_j) + dloss_0 (L / M) p_l (f_l - sum_j f_j p_j) + dloss_1 (2 / M) lse p_l
 *
 * with G_l the gradient of atom l's value (0 where it is not listed), q = p for SR_ROUTE_SOFTMAX and the softmax over the
 * listed atoms for SR_ROUTE_CHOSEN, f_l = counts_l / (M entries).  For SR_ROUTE_VALUES it is G_l, and counts must be NULL.
 * Computed in fp32 from the logits, rounded once.  Masked pixels (whose dvalue and index are not looked at) and masked atoms
 * get 0.  dvalue is finite at the other pixels (else: unspecified values at that pixel).
 */
int sr_list_route_grad(const sr_tensor* coeff, const sr_tensor* index, const sr_tensor* dvalue,
                       int L, int scale, int entries, int kind, int coeff_layout, const sr_tensor* mask,
                       const long long* counts, const float* dloss, sr_tensor* dcoeff, void* stream);

/* Bytes of DEVICE scratch sr_dict_assemble_list_grad needs (0 if L or k is out of range). */
size_t sr_dict_assemble_list_grad_workspace_bytes(int L, int k);

/*
 * Gradient of sr_dict_assemble_list with respect to the values and to the dictionary.  With B_ic the k x k neighbourhood of
 * the up-sampled image and E_i = sum_c dout_ic B_ic, the gradient of pixel i's filter:
 *
 *     dvalue[t][i] = D[index[t][i]] . E_i          ddict[l] = sum over i, t with index[t][i] = l of value[t][i] E_i
 *
 *   lr, index, value, dict, L, k, scale, channels, entries   as in the forward call
 *   mask    [N][1][H][W]  SR_U8, or NULL: where it is 0, dout and value are taken as 0 and dvalue is written as 0
 *   dout    [N][C][H][W]  gradient of the image, dtype of lr
 *   dvalue  as value, same type; written; or NULL
 *   ddict   [1][L][k][k]  f32; written; or NULL (not both)
 *   workspace, workspace_bytes   DEVICE scratch, 16-byte aligned; not needed (may be NULL) where ddict is NULL
 *
 * index: atoms below L (others count as atom L - 1); an atom that is listed twice gets both terms.  Finite values only: infinities and NaN in
 * dict, lr, dout or value give unspecified results.  Arithmetic is fp32 or equivalent (fp16 matrix-core products of operands split
 * in two, which hold all but 2^-23 of a pixel's largest E, an atom's largest tap and a value); ddict is summed in fp32 over runs of at
 * most 4096 pixels and in double from there on, and what a pixel whose E is below 2^-100 of the largest in its run adds to it may be lost.
 * An empty call writes zeros to ddict.
 */
int sr_dict_assemble_list_grad(const sr_tensor* lr, const sr_tensor* index, const sr_tensor* value, const sr_tensor* dict,
                               int L, int k, int scale, int channels, int entries, const sr_tensor* mask,
                               const sr_tensor* dout, sr_tensor* dvalue, sr_tensor* ddict,
                               void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SR_ROUTE_H */
