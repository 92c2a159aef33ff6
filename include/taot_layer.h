/*
 * taot_layer.h -- operators of a mixture-of-experts layer around the planner of taot.h, for one NVIDIA B200 (sm_100a).
 *
 * In the order in which a layer runs them:
 *   taot_rms_norm          residual's addition, RMS norm, the normalised rows in the inputs' type and / or in 8 bits with scales
 *   taot_route             router logits -> the routing table that taot_histogram and taot_plan read, and the experts' weights
 *   (taot_plan, taot_dispatch)
 *   taot_send              rows (and their scales) -> the send buffer, by the positions that taot_dispatch gives
 *   taot_combine           weighted sum of the rows that came back, and the residual
 * and their gradients: taot_combine_backward, taot_route_backward, taot_rms_norm_backward; the gradient of taot_send is
 * taot_combine without weights.
 *
 * Conventions: those of taot.h (device pointers d_*, `stream`, status codes; calls only enqueue), without a handle: every
 * call takes its sizes in a struct whose struct_size is sizeof of it, and launches on the current device, to which the
 * pointers and the stream belong.  A call with no rows checks its arguments and launches nothing.  All can be captured in a CUDA
 * graph.  Matrices are row-major with dense columns; ld_* is the distance between rows in elements, at least the number of columns.
 * Arrays are aligned to their elements; 16-byte aligned arrays with rows of a multiple of 16 bytes take the wide loads.
 * Sums, norms and scores are held in 32 bits or more and rounded once, at the end.  Same inputs give the same output bits.
 * Errors of every call: TAOT_ERR_NULL, TAOT_ERR_PARAM (struct_size, ranges, an output that overlaps an input or another
 * output where that is not allowed below; different columns of one wider array, the same ld apart, do not), TAOT_ERR_UNSUPPORTED,
 * TAOT_ERR_ALIGN, TAOT_ERR_CUDA.
 */
#ifndef TAOT_LAYER_H
#define TAOT_LAYER_H

#include "taot.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TAOT_F32 = 0, TAOT_BF16 = 1, TAOT_F16 = 2 };            /* element types */
enum { TAOT_SOFTMAX = 0, TAOT_SIGMOID = 1 };                    /* scores */

/*
 * h = x + residual (rounded to the type; h = x without a residual), rstd = (mean(h^2) + eps)^-1/2, y = h * rstd * weight,
 * and per group of `group` consecutive columns (the last group of a row may be short)
 *   scale = max(max |y| * (1 / 448), 2^-126),  q = y / scale rounded to nearest in e4m3 (4 exponent and 3 mantissa bits, ties to even),
 * both from the 32-bit y: the reciprocal of 448, the product with it and the quotients are fp32 numbers, rounded to nearest.  A NaN or an infinity in a row spreads as that arithmetic has it, and to no other row; so do squares
 * beyond the largest fp32: values of up to 2^60 in rows of up to 2^16 columns are safe.  Squares below 2^-126 lose digits, which
 * shows only with an eps as small (eps = 0 and a row of values below 2^-60).
 *   d_x, d_residual (or NULL), d_weight [D]: of the type.  d_h: required with a residual, else NULL.  May be d_x or d_residual
 *   itself (with the same ld), d_y may be d_x.
 *   d_y, d_q with d_scales [N, ceil(D / group)], d_rstd [N]: each optional, but at least one of d_y and d_q.
 * Ranges: N < 2^31, 1 <= D <= 2^20, eps >= 0 and finite, group 32, 64, 128 or 256 with d_q, 0 without.
 */
typedef struct {
    int32_t struct_size;
    int32_t dtype;
    int64_t N;
    int32_t D;
    int32_t group;
    float eps;
    int32_t reserved;                                       /* 0 */
    int64_t ld_x, ld_residual, ld_h, ld_y, ld_q;            /* those of absent arrays are not looked at */
} taot_norm_params;

int taot_rms_norm(const taot_norm_params* params, const void* d_x, const void* d_residual, const void* d_weight,
                  void* d_h, void* d_y, uint8_t* d_q, float* d_scales, float* d_rstd, void* stream);

/*
 * Gradients of y = h * rstd(h) * weight, h = x + residual (the 8-bit rows count as y):  with g = dy * weight,
 *   dx = rstd * (g - h rstd mean(g h rstd)) + dh      the gradient of x and of the residual alike
 *   dweight = sum over rows of dy * h * rstd          fp32, overwritten
 *   d_dy, d_h, d_weight, d_rstd as taot_rms_norm had or gave them; d_dh (or NULL): what reaches h from elsewhere.
 *   d_dx may be d_dy or d_dh (with the same ld), but not d_h.  d_dweight may be NULL.  With no rows dweight is set to zero.
 *   ws: taot_rms_norm_backward_workspace bytes of device memory, 16-byte aligned, the same for any N (4.8 MB for 4096 columns, 512 bytes for each
 *   column beyond 16384); not needed without d_dweight.
 * In the params ld_x is that of dx, ld_residual that of dh, ld_y that of dy; eps, group and ld_q are not looked at.
 */
int taot_rms_norm_backward_workspace(const taot_norm_params* params, size_t* bytes);
int taot_rms_norm_backward(const taot_norm_params* params, const void* d_dy, const void* d_dh, const void* d_h,
                           const void* d_weight, const float* d_rstd, void* d_dx, float* d_dweight, void* ws, void* stream);

/*
 * Routing of L * T tokens to k of E experts each.
 * An expert is closed to a token if its logit is NaN or at most the lowest finite value of the type (-infinity among them), or
 * if its bias is not finite; an infinite logit counts as the largest finite one.  Over the open experts
 *   score  s = softmax(logit) or 1 / (1 + exp(-logit)); the softmax's sum is over all experts with an open logit, whatever the
 *          biases, which take part in the choice only (so the gradient needs none);
 *   key    s + bias, or without a bias the logit itself;
 *   groups > 1: experts [g E/groups, (g+1) E/groups) are a group; its score is the sum of the group_top largest s (+ bias) of its
 *   open experts; only the groups_kept groups of the highest scores stay (a group without open experts comes last);
 *   topk   the k experts of the largest keys, largest first, all ties (of groups too) to the lowest index, decided as by
 *          arithmetic in 64 bits;
 *   weight scale * s, or with `renormalise` scale * s / (sum of the token's chosen s).
 * The choice is settled in 64 bits where fp32 leaves it open; weights are fp32 arithmetic.
 * Places that no open expert fills get expert -1 and weight 0; so do all places of a token whose d_mask byte is 0 (padding).
 * (The planner skips such entries and reports TAOT_INFO_BAD_INDEX; taot_dispatch puts them behind all others.)
 *   d_logits [L*T, E] with ld_logits; d_bias [L, E] fp32 or NULL; d_mask [L*T] bytes or NULL
 *   d_topk [L, T, k] int32, d_weights [L, T, k] fp32 or NULL
 * Ranges: L, T >= 0 with L * T < 2^31, 1 <= E <= 1024, 1 <= k <= min(E, 64), 1 <= groups <= 64 dividing E, 1 <= groups_kept <= groups
 * with k <= groups_kept * E / groups, group_top 1 or 2, scale finite.
 */
typedef struct {
    int32_t struct_size;
    int32_t dtype;                                          /* of the logits and of their gradient */
    int64_t L, T;
    int32_t E, k;
    int32_t score;
    int32_t groups, groups_kept, group_top;
    int32_t renormalise;
    float scale;
    int64_t ld_logits, ld_dlogits;                          /* ld_dlogits: taot_route_backward only */
} taot_route_params;

int taot_route(const taot_route_params* params, const void* d_logits, const float* d_bias, const uint8_t* d_mask,
               int32_t* d_topk, float* d_weights, void* stream);

/*
 * Gradient of the weights with respect to the logits (the choice itself has none): with c = scale and g = d_dweights
 *   softmax:              dl_e = c p_e ([e chosen] g_e - sum_j g_j p_j)
 *   softmax, renormalise: dl_i = c q_i (g_i - sum_j g_j q_j) for the chosen experts, q = their softmax among themselves
 *   sigmoid:              dl_i = c g_i s_i (1 - s_i)
 *   sigmoid, renormalise: dl_i = c q_i (1 - s_i) (g_i - sum_j g_j q_j), q = s / (sum of the chosen s)
 * and zero elsewhere.  Entries of d_topk outside [0, E) do not count; an expert that a token holds twice counts twice.
 *   d_dlogits [L*T, E] with ld_dlogits, fully written; must not overlap d_logits.
 * Of the params, groups, groups_kept and group_top are not looked at; k <= 64 may exceed E.
 */
int taot_route_backward(const taot_route_params* params, const void* d_logits, const int32_t* d_topk,
                        const float* d_dweights, void* d_dlogits, void* stream);

/*
 * Rows to the send buffer and back.  B send buffers (one per layer and source rank) of n tokens with k entries each: entry
 * (b, t, j) has the position d_perm[b][t][j] in [0, n*k), each position once per buffer, as taot_dispatch writes them for
 * B = L * R, n = T / R.  d_counts [B, C] (NULL with C = 0: all positions are in use), e.g. taot_dispatch's d_send_counts with C = R: only the first
 * sum_c d_counts[b][c] positions of buffer b are in use; entries behind them are not delivered: their rows are neither
 * written nor read.  A position outside [0, n*k) is left out too and sets TAOT_INFO_BAD_INDEX in d_info[b] (OR-ed; NULL: not
 * reported).
 * Ranges: B, n, k >= 0 with B * n * k < 2^31, k <= 64, 1 <= D <= 2^20, 0 <= C <= 4096.
 */
typedef struct {
    int32_t struct_size;
    int32_t dtype;
    int64_t B, n;
    int32_t k, D, C;
    int32_t reserved;                                       /* 0 */
    int64_t ld_rows;                                        /* of the send buffer: y, dy, and taot_send's output */
    int64_t ld_tokens;                                      /* of the tokens' rows: x, out, dout */
    int64_t ld_residual;
} taot_rows_params;

/*
 * d_rows[b][d_perm[b][t][j]][:] = d_x[b][t][:] for rows of D elements of elem_bytes (1, 2 or 4) bytes, whatever their type
 * (dtype is not looked at).  d_scales [B, n, scale_cols] fp32 -> d_row_scales [B, n*k, scale_cols] in the same way, both NULL
 * without scales.  1 <= scale_cols <= 2^20.
 */
int taot_send(const taot_rows_params* params, int32_t elem_bytes, const void* d_x, const float* d_scales, int32_t scale_cols,
              const int32_t* d_perm, const int32_t* d_counts, void* d_rows, float* d_row_scales, int32_t* d_info, void* stream);

/*
 * d_out[b][t][:] = d_residual[b][t][:] + sum_j d_weights[b][t][j] * d_y[b][d_perm[b][t][j]][:], summed in fp32 in the order of j.
 *   d_weights [B, n, k] fp32, NULL: all one.  d_residual: NULL, or rows of the type; d_out may be d_residual (with the same ld).
 */
int taot_combine(const taot_rows_params* params, const void* d_y, const int32_t* d_perm, const int32_t* d_counts,
                 const float* d_weights, const void* d_residual, void* d_out, int32_t* d_info, void* stream);

/*
 * Gradients of taot_combine (that of the residual is d_dout itself):
 *   d_dy[b][d_perm[b][t][j]][:] = d_weights[b][t][j] * d_dout[b][t][:]
 *   d_dweights[b][t][j] = sum over columns of d_dout[b][t] * d_y[b][d_perm[b][t][j]], 0 for entries that are not delivered
 * d_dy or d_dweights may be NULL (not both); d_y is needed for d_dweights only, and d_dy may be d_y itself (same ld).
 */
int taot_combine_backward(const taot_rows_params* params, const void* d_dout, const void* d_y, const int32_t* d_perm,
                          const int32_t* d_counts, const float* d_weights, void* d_dy, float* d_dweights, int32_t* d_info,
                          void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TAOT_LAYER_H */
