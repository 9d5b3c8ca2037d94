/* Operators that stand around the attention and the scan in a layer, for AMD MI355X (gfx950) -- C ABI
 * of libfla_seq.so.
 *
 *   residual + root-mean-square norm   forward, forward with an 8-bit output and its scales, backward
 *   rotary positions of q and k        outside the attention kernel: any head layout, one or two axes
 *   gated linear recurrence            over the tokens: forward with kept state, single steps, backward
 *
 * Conventions are those of fla_swin.h: device pointers owned by the caller, asynchronous launches on
 * `stream` (NULL = the null stream), nothing allocated, freed, copied or synchronised, fla_status
 * return values, the same call giving the same bits every time.  An empty problem (a size of 0)
 * returns FLA_OK and ignores the pointers.  Each entry point checks in the order FLA_ERR_SHAPE,
 * FLA_ERR_UNSUPPORTED (type, group, eps), FLA_ERR_HEAD_DIM, FLA_ERR_ROPE, (empty problem), FLA_ERR_NULL,
 * FLA_ERR_ALIGN, FLA_ERR_TOO_LARGE, FLA_ERR_WORKSPACE, FLA_ERR_ALIAS, FLA_ERR_ARCH, FLA_ERR_LAUNCH,
 * and on error launches nothing and touches no output.
 *
 * Types: dtype is FLA_F32 or FLA_BF16, the type of every tensor given as void* unless said otherwise.
 * Sums, norms, angles and states are held in 32 bits or more.  Pointers are aligned to their element
 * (FLA_ERR_ALIGN); no wider alignment is asked for.  Strides are in elements, 0 or positive
 * (FLA_ERR_SHAPE); the innermost dimension is contiguous.  Outputs are contiguous unless they have a
 * stride argument.  Overlap is judged by the whole range from a tensor's first to its last element.
 */
#ifndef FLA_SEQ_H
#define FLA_SEQ_H

#include <stddef.h>
#include <stdint.h>

#include "fla_swin.h"   /* fla_status, hipStream_t */

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FLA_F32 = 0, FLA_BF16 = 1 } fla_dtype;

/* ---- residual + root-mean-square norm --------------------------------------------------
 *
 * For each of `rows` rows of D channels:
 *   s = x + residual,   rstd = 1 / sqrt(mean(s^2) + eps),   y = s * rstd * weight.
 * residual may be NULL (s = x).  The norm is that of the unrounded s.  x, residual: rows x_stride /
 * residual_stride elements apart.  weight [D], of type weight_dtype (FLA_F32 or dtype).
 * Outputs, contiguous [rows, D]: y; sum (s rounded to dtype: the next layer's residual; NULL: not
 * kept); rstd [rows] fp32 (for the backward; NULL: not kept).  y and sum may each be exactly x or
 * residual (same address, rows D apart: in place); any other overlap is FLA_ERR_ALIAS.
 * eps must be finite and >= 0 (FLA_ERR_UNSUPPORTED).  D up to 2^24, tensors below 2^40 elements
 * (FLA_ERR_TOO_LARGE). */
int fla_add_rms_norm_fwd(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                         const void* weight, void* y, void* sum, float* rstd, int64_t rows, int D, float eps,
                         int dtype, int weight_dtype, hipStream_t stream);

/* The same with y in 8 bits (OCP e4m3, round to nearest even) and fp32 scales: a scale for each
 * `group` consecutive channels of a row (32, 64 or 128; the last group may be shorter), or one per row
 * (group = 0): scale = max|y| / 448, not below the least normal fp32 (2^-126); 1 where max|y| is 0;
 * q = y / scale.  A NaN in a group makes its scale and all its q NaN.
 * q: [rows, D] bytes; scales: [rows, ceil(D / group)] (group 0: [rows]).  q must not overlap anything. */
int fla_add_rms_norm_q8(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                        const void* weight, void* q, float* scales, void* sum, int64_t rows, int D, int group,
                        float eps, int dtype, int weight_dtype, hipStream_t stream);

/* Backward.  With n = s * rstd and dn = dy * weight, for the s and rstd given:
 *   dx = rstd * (dn - n * mean(dn * n)) + dsum     (the gradient of x and of residual alike),
 *   dweight = sum over rows of dy * n              (fp32).
 * s: the forward's sum (or x where there was no residual), rows s_stride apart; rounded to dtype, so
 * the gradients are those at the rounded sum.  dsum: the gradient that reaches `sum` from the layers
 * behind (NULL: none).  dx contiguous [rows, D]; it may be exactly dy or dsum.  The rows' shares of
 * dweight are added in a fixed order.  rows = 0 with D > 0 sets dweight to 0. */
int fla_add_rms_norm_bwd_workspace(int64_t rows, int D, size_t* bytes);
int fla_add_rms_norm_bwd(const void* dy, int64_t dy_stride, const void* s, int64_t s_stride, const void* weight,
                         const float* rstd, const void* dsum, int64_t dsum_stride, void* dx, float* dweight,
                         void* workspace, size_t workspace_bytes, int64_t rows, int D, int dtype, int weight_dtype,
                         hipStream_t stream);

/* ---- rotary positions -------------------------------------------------------------------
 *
 * q [B, L, hq, d] and k [B, L, hk, d] (hk may be 0): the first rot channels of every head turn, pair j
 * (j < rot / 2) by the angle position * freqs[j] and scaled by mscale:
 *   (a, b) -> mscale (a cos - b sin, b cos + a sin);
 * inverse != 0 turns back (the angle negated; mscale kept): the gradient of the rotation.
 * Pairs: interleaved != 0: channels (2j, 2j + 1); else (j, j + rot / 2).  Channels from rot on are
 * copied.  rot is even, 2 <= rot <= d, d <= 512 (FLA_ERR_HEAD_DIM).
 * positions: int32 or (pos64 != 0) int64, [B, L] or, with axes = 2, [B, L, 2] (axis contiguous), with
 * the strides pos_batch and pos_token: pairs of the first half (j < rot / 4) then turn with axis 0,
 * the others with axis 1 (rot divisible by 4).  Any value is a position, negative ones too.
 * freqs [rot / 2]: float64, radians per unit of position.  Angles are formed in 64 bits (off by about 2^-52 of
 * their size), so far positions keep their place in the turn; cosine and sine are rounded to fp32 once.
 * B * L up to 2^31 - 1024, hq + hk up to 2^20, tensors below 2^40 elements (FLA_ERR_TOO_LARGE).
 * Strides per tensor: batch, token, head (the last below 2^32: FLA_ERR_TOO_LARGE).  q_out may be exactly q (same strides), k_out exactly k:
 * in place.  Tokens may not overlap in an output. */
int fla_rotary(const void* q, int64_t q_batch, int64_t q_token, int64_t q_head,
               const void* k, int64_t k_batch, int64_t k_token, int64_t k_head,
               void* q_out, int64_t qo_batch, int64_t qo_token, int64_t qo_head,
               void* k_out, int64_t ko_batch, int64_t ko_token, int64_t ko_head,
               const void* positions, int pos64, int64_t pos_batch, int64_t pos_token, int axes,
               const double* freqs, int B, int L, int hq, int hk, int d, int rot, int interleaved,
               double mscale, int inverse, int dtype, hipStream_t stream);

/* Frequencies, on the host: freqs[j] = theta^(-2j / rot), j < rot / 2, changed for contexts longer than
 * the trained one by `factor`:
 *   FLA_ROPE_PLAIN   as they are;
 *   FLA_ROPE_LINEAR  freqs / factor (positions interpolated);
 *   FLA_ROPE_BASE    theta * factor^(rot / (rot - 2)) in place of theta (rot > 2);
 *   FLA_ROPE_PARTS   by the turns t a pair makes within trained_len positions: pairs of less than one turn
 *                    get freqs / factor, of more than 32 keep theirs, linear in t between;
 *                    *mscale = 0.1 ln(factor) + 1.
 * *mscale is 1 otherwise (mscale may be NULL).  theta finite and > 0, factor finite and >= 1, trained_len
 * finite and > 0 (FLA_ERR_ROPE, FLA_ERR_ROPE also for an unknown scaling); rot even and >= 2
 * (FLA_ERR_HEAD_DIM). */
typedef enum { FLA_ROPE_PLAIN = 0, FLA_ROPE_LINEAR = 1, FLA_ROPE_BASE = 2, FLA_ROPE_PARTS = 3 } fla_rope_scaling;
int fla_rotary_freqs(int rot, double theta, int scaling, double factor, double trained_len, double* freqs,
                     double* mscale);

/* ---- gated linear recurrence -------------------------------------------------------------
 *
 * Every channel of a sequence of L tokens by itself, from its state h_{-1} = h0 (NULL: 0), with a
 * decay gate r and an input gate i given per token before their sigmoids:
 *   z_t = c softplus(lam) sigmoid(r_t),   a_t = exp(-z_t),
 *   h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t.
 * x, r, i: [B, L, D] with batch and token strides; lam [D] fp32; h0 [B, D] fp32, contiguous.
 * lengths [B] int32 (device; NULL: all L): tokens from lengths[b] on are no tokens of sequence b: they
 * are not looked at, h keeps what it held there; a length below 0 counts as 0, above L as L.
 * Outputs: h [B, L, D] contiguous, h_last [B, D] fp32: the state behind each sequence's last token
 * (h0 for an empty one; NULL: not kept; it may be exactly h0), states: for the backward (NULL: not
 * kept), fla_gated_scan_states() bytes, contents private to the pair.
 * c finite and > 0 (FLA_ERR_UNSUPPORTED).  D up to 2^24, fewer than 2^22 tiles of 128 tokens by 64 channels, tensors
 * below 2^40 elements (FLA_ERR_TOO_LARGE).  L = 1 is a step of a kept state.  A sequence's h does not depend on
 * the others of its batch.
 * L = 0 with B, D > 0 copies h0 (or zeros) to h_last.
 * workspace: fla_gated_scan_workspace() bytes (may be NULL where that is 0); contents ignored on
 * entry.  Calls that may run at the same time need workspaces of their own. */
int fla_gated_scan_states(int B, int L, int D, size_t* bytes);
int fla_gated_scan_workspace(int B, int L, int D, size_t* bytes);
int fla_gated_scan_fwd(const void* x, int64_t x_batch, int64_t x_token, const void* r, int64_t r_batch,
                       int64_t r_token, const void* i, int64_t i_batch, int64_t i_token, const float* lam,
                       const float* h0, const int* lengths, void* h, float* h_last, float* states,
                       void* workspace, size_t workspace_bytes, int B, int L, int D, float c, int dtype,
                       hipStream_t stream);

/* Backward: with g_t = dh_t + a_{t+1} g_{t+1} (behind the last token: d_last),
 *   dx_t = g_t sqrt(1 - a_t^2) sigmoid(i_t),   di_t, dr_t accordingly,   dlam (fp32, summed over B and
 *   the tokens in a fixed order),   dh0 = a_0 g_0 (fp32; NULL: not wanted).
 * dh [B, L, D] with strides (NULL: zero), d_last [B, D] fp32 (NULL: zero).  dx, dr, di contiguous
 * [B, L, D], 0 in rows from lengths[b] on (every row is written).  states as the forward wrote them
 * for the same x, r, i, lam, h0 and lengths. */
int fla_gated_scan_bwd_workspace(int B, int L, int D, size_t* bytes);
int fla_gated_scan_bwd(const void* x, int64_t x_batch, int64_t x_token, const void* r, int64_t r_batch,
                       int64_t r_token, const void* i, int64_t i_batch, int64_t i_token, const float* lam,
                       const float* states, const int* lengths, const void* dh, int64_t dh_batch,
                       int64_t dh_token, const float* d_last, void* dx, void* dr, void* di, float* dlam,
                       float* dh0, void* workspace, size_t workspace_bytes, int B, int L, int D, float c,
                       int dtype, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FLA_SEQ_H */
