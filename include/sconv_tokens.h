/*
 * sconv, token operators: what a network runs behind its convolution stages when it goes on with attention, on AMD MI355X
 * (gfx950) - layer norm (from a feature map or from tokens), rotary positions over several axes, differential
 * attention -, each with its gradient.
 *
 * As for sconv.h: every pointer marked "device" is HIP device memory owned by the caller, the library allocates none, work is
 * enqueued on the given stream (a hipStream_t as void*, NULL = the default stream) and the call returns without
 * synchronising, outputs are overwritten, and every int function returns 0 or a negative SCONV_E* code.  Argument checks are
 * host code and run before any GPU call.  Nothing is kept between calls.  Results do not depend on timing: no
 * sum's order does.
 *
 * Types: SCONV_F32 and SCONV_BF16.  Whatever the type, sums, softmax statistics and norms are held in 32 bits and results are
 * rounded once.  (16-bit half is left out: a training program's small gradients leave its range without a scale that
 * follows the loss.)  Strides count elements; the last axis of a strided tensor is contiguous.
 * Sizes of zero are allowed where a call says so; such a call does what is left to do (it clears gradients, say).
 * SCONV_EUNSUPPORTED, before anything is enqueued, where a size passes a limit given below or a kernel's grid would have 2^32 threads:
 * that takes 2^24 rows of layer norm, tokens of rotary, tiles of 16 (query, head) pairs or of 128 keys at least.
 */
#ifndef SCONV_TOKENS_H
#define SCONV_TOKENS_H

#include "sconv.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SCONV_F32 = 0, SCONV_BF16 = 1 };

/*
 * Layer norm.  Every place (n, s) of C channels is normalised for itself:
 *   mean = sum_c x / C;  rstd = 1 / sqrt(sum_c (x - mean)^2 / C + eps);  y = (x - mean) * rstd * w[c] + b[c].
 * x is a feature map as sconv_forward leaves it, x[n][c][s] (s = the H*W places, contiguous), or tokens x[n][s][c]; y is tokens.
 */
enum { SCONV_LAYOUT_TOKENS = 0, SCONV_LAYOUT_MAP = 1 };
typedef struct {
    int32_t N, S, C;           /* N, S >= 0; 1 <= C <= 65536                                                      */
    int32_t layout;            /* of x (and dx)                                                                   */
    int32_t x_type, y_type;    /* y_type: x_type, or SCONV_BF16 under an fp32 x                                   */
    int32_t w_type;            /* of w, b and their gradients                                                     */
    float eps;                 /* >= 0, finite                                                                    */
    int64_t x_n, x_s;          /* strides of x: images, and places (tokens) or channels (map)                     */
    int64_t y_n, y_s;          /* strides of y (and dy): images, places                                           */
} sconv_layernorm_desc_t;
/*
 *   x_dev    device, in;  w_dev, b_dev: device, in, [C], optional (NULL: 1 and 0)
 *   y_dev    device, out
 *   mean_dev, rstd_dev  device, out, fp32 [N][S], both or neither: what the backward call reads
 */
int sconv_layernorm_forward(const sconv_layernorm_desc_t* desc, const void* x_dev, const void* w_dev, const void* b_dev,
                            void* y_dev, float* mean_dev, float* rstd_dev, void* hip_stream);
/*
 * Its gradient.  With g = dy * w and u = (x - mean) * rstd:
 *   dx = rstd * (g - mean_c(g) - u * mean_c(g * u));  dw[c] = sum over places of dy * u;  db[c] = sum over places of dy.
 *   dx_dev   device, out, optional: contiguous, in x's layout and type
 *   dw_dev, db_dev  device, out, both or neither: [C] of w_type
 *   ws_dev   device, scratch, ws_bytes: at least sconv_layernorm_workspace_size (read only with dw_dev; 16-byte aligned):
 *            partial sums of the weight's gradient, one row a workgroup, added in a fixed order by a second kernel
 */
int sconv_layernorm_backward(const sconv_layernorm_desc_t* desc, const void* dy_dev, const void* x_dev,
                             const float* mean_dev, const float* rstd_dev, const void* w_dev, void* dx_dev, void* dw_dev,
                             void* db_dev, void* ws_dev, size_t ws_bytes, void* hip_stream);
int sconv_layernorm_workspace_size(const sconv_layernorm_desc_t* desc, size_t* bytes);

/*
 * Rotary positions over several axes (rows and columns of a map, frames of a video).  Pair p of every head turns by the
 * angle pos[axis[p]] * freq[p]:
 *   (u, v) -> (u cos t - v sin t, u sin t + v cos t),
 * u, v being elements p and p + pairs of the head, or 2p and 2p + 1 (interleaved).  Elements from 2 * pairs on are copied.  Queries
 * and keys go through one launch.  Angles are formed in 64 bits, so a place far out on an axis keeps its
 * angle; the gradient is the turn by -t (inverse).
 */
enum { SCONV_ROTARY_MAX_AXES = 8, SCONV_ROTARY_MAX_PAIRS = 256 };
typedef struct {
    int32_t B, S, Hq, Hk, D;   /* B, S, Hq, Hk >= 0 (Hk 0: no keys); 1 <= D <= 1024                               */
    int32_t type;              /* of q and k                                                                      */
    int32_t pairs, axes;       /* 1 <= pairs <= min(D / 2, 256); 1 <= axes <= 8                                   */
    int32_t interleaved, inverse;
    int64_t q_b, q_s, q_h, k_b, k_s, k_h;       /* strides of q and k                                             */
    int64_t qo_b, qo_s, qo_h, ko_b, ko_s, ko_h; /* strides of the outputs                                         */
    int64_t pos_b;             /* stride of pos between requests: S * axes, or 0 for the same places in all       */
    uint8_t axis[SCONV_ROTARY_MAX_PAIRS];       /* of every pair, < axes                                          */
} sconv_rotary_desc_t;
/*
 *   q_dev, k_dev     device, in;  pos_dev: device, in, int32 [B or 1][S][axes];  freq_dev: device, in, fp32 [pairs]
 *   qo_dev, ko_dev   device, out; may be q_dev and k_dev with the same strides (in place), must not overlap them otherwise
 */
int sconv_rotary(const sconv_rotary_desc_t* desc, const void* q_dev, const void* k_dev, const int32_t* pos_dev,
                 const float* freq_dev, void* qo_dev, void* ko_dev, void* hip_stream);

/*
 * Differential attention: the difference of two softmax maps over the same values, weighed by a learned number of each
 * head.  Query head h has two queries (rows 2h, 2h+1 of q), key head g = h / (H / Hkv) two keys and one value:
 *   S_m = scale * Q_m K_m^T,  A_m = softmax over the keys that the query sees,  out = (A_1 - lam[h] A_2) V.
 * Query i of request b sees key j where j < n_b (k_lengths[b], or Sk), k_mask[b][j] is not 0, and - causal - j <= i + n_b - Sq: the
 * last query stands at the request's last key.  A query that sees nothing gives zeros and takes no gradient.  Keys and values
 * that k_lengths or k_mask leave out are never part of a sum, whatever they hold (Inf, NaN); one that causal alone hides from a
 * query has to be finite, as 0 * NaN may stand in the query's sum.
 * Inf in what a query sees goes through the formulas: a score of -Inf has no weight (a query with no other sees nothing), +Inf or NaN
 * makes the query's results NaN, an Inf in V is Inf or NaN in its column.  Gradients through such places are not finite.
 * One token of every request over a long cache (Sq = 1) is the same call: its keys are split over workgroups, whose parts a
 * second kernel joins.
 */
typedef struct {
    int32_t B, Sq, Sk;         /* >= 0                                                                            */
    int32_t H, Hkv;            /* H % Hkv == 0                                                                    */
    int32_t D, Dv;             /* of a query or key, 1..128; of a value, 1..256                                   */
    int32_t type;              /* of q, k, v, out and their gradients                                             */
    int32_t causal;
    float scale;               /* > 0, finite                                                                     */
    int64_t q_b, q_s, q_h, k_b, k_s, k_h, v_b, v_s, v_h;   /* strides                                             */
    int64_t mask_b;            /* stride of k_mask between requests                                               */
} sconv_diffattn_desc_t;
/*
 *   q_dev [B][Sq][2H][D], k_dev [B][Sk][2Hkv][D], v_dev [B][Sk][Hkv][Dv]  device, in (strided);  lam_dev: device, in, fp32 [H]
 *   k_lengths_dev    device, in, int32 [B], optional; taken as 0 below 0 and as Sk above Sk
 *   k_mask_dev       device, in, bytes [B][Sk], optional
 *   out_dev          device, out, [B][Sq][H][Dv], contiguous
 *   second_dev       device, out, [B][Sq][H][Dv]: A_2 V; lse_dev: device, out, fp32 [2][B][H][Sq]: ln of the sums of the two
 *                    softmaxes (-inf where nothing is seen).  Both or neither: what the backward call reads
 *   ws_dev, ws_bytes device, scratch, optional (NULL, 0), 16-byte aligned: parts of calls of few queries; with less than
 *                    sconv_diffattn_workspace_size(backward 0) the keys are split less or not at all
 */
int sconv_diffattn_forward(const sconv_diffattn_desc_t* desc, const void* q_dev, const void* k_dev, const void* v_dev,
                           const float* lam_dev, const int32_t* k_lengths_dev, const uint8_t* k_mask_dev, void* out_dev,
                           void* second_dev, float* lse_dev, void* ws_dev, size_t ws_bytes, void* hip_stream);
/*
 * Its gradient, from the weights formed again out of lse:
 *   G = dout V^T;  d_m = rows of dout . (A_m V);  dS_1 = A_1 (G - d_1);  dS_2 = -lam A_2 (G - d_2);
 *   dq_m = scale dS_m K_m;  dk_m = scale dS_m^T Q_m;  dv = (A_1 - lam A_2)^T dout;  dlam[h] = -sum A_2 G.
 *   dout_dev, out_dev, second_dev: [B][Sq][H][Dv], contiguous;  dq_dev, dk_dev, dv_dev: device, out, contiguous, in the shapes
 *   of q, k, v;  dlam_dev: device, out, fp32 [H].  Keys' and values' gradients are sums over the query heads that share them.
 *   ws_dev   device, scratch, 16-byte aligned, at least sconv_diffattn_workspace_size(backward 1)
 */
int sconv_diffattn_backward(const sconv_diffattn_desc_t* desc, const void* dout_dev, const void* q_dev, const void* k_dev,
                            const void* v_dev, const float* lam_dev, const int32_t* k_lengths_dev,
                            const uint8_t* k_mask_dev, const void* out_dev, const void* second_dev, const float* lse_dev,
                            void* dq_dev, void* dk_dev, void* dv_dev, float* dlam_dev, void* ws_dev, size_t ws_bytes,
                            void* hip_stream);
int sconv_diffattn_workspace_size(const sconv_diffattn_desc_t* desc, int backward, size_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* SCONV_TOKENS_H */
