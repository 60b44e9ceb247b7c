/*
 * gt_layer.h -- operators around the sparse attention of a graph transformer's
 * layer, for AMD Instinct MI355X (gfx950): differential attention over a CSR
 * graph, rotary positions with several axes, and layer norm, each with its
 * backward pass.  Part of the library that gt_attn.h declares; types, status
 * codes, error messages, CSR layout, streams and workspaces are those of
 * gt_attn.h, as are these rules: every pointer argument is DEVICE memory of the
 * calling thread's current device unless it is said to be host memory, `stream`
 * belongs to that device, arrays are row-major and dense, calls are asynchronous
 * on `stream` and may be captured into a graph, arguments are validated on the
 * host before any device work, and N == 0 enqueues nothing (except that the
 * gradients of parameters are then set to 0).  Results are bitwise reproducible
 * for fixed arguments.
 */
#ifndef GT_LAYER_H
#define GT_LAYER_H

#include "gt_attn.h"

#ifdef __cplusplus
extern "C" {
#define GT_ENUM_BASE : int
#else
#define GT_ENUM_BASE
#endif

/*
 * Differential attention, forward: each value head h has two maps over the
 * row's entries, with query and key heads 2h and 2h + 1, and its output is the
 * first map's sum less lambda[h] times the second's:
 *
 *   s_m,e      = scale * sum_d Q[i,2h+m,d] * K[j_e,2h+m,d]           m = 0, 1
 *   out[i,h,:] = sum_e (softmax_e(s_0) - lambda[h] softmax_e(s_1)) V[j_e,h,:]
 *
 * Layouts: Q, K [N][2H][D]; V, out [N][H][2D], in `dtype`, 16-byte aligned;
 * lambda float [H], any values; lse (may be NULL) float [N][2H], receives
 * ln(sum_e exp(s_m,e)).  An entry whose score is -inf (or below -2.35e38: scores
 * are held in units of ln 2) has weight 0 (its value row still enters, times 0);
 * a row without entries, or with none but such, counts as empty in that map: the
 * map's sum is 0 and its lse -inf.  Inf and NaN in the K or V row of a node reach
 * only the rows whose entries name that node.
 * Supported shapes: H in {1, 2, 4, 8} with D in {32, 64, 128}, and for bf16
 * features also D = 256 (a value head's 2D elements must fit 64 lanes of 16
 * bytes); 0 <= E < 2^31; 0 <= N < 2^31.
 * Accumulates in fp32; bf16 outputs are rounded to nearest even.  tuning:
 * light_max_deg, heavy_min_deg, chunk_edges and grid_blocks as for
 * gt_attn_fwd_ex (may be NULL); dense_tiles and bf16_weights are ignored.
 * out must not overlap an input, lse none of the other buffers.
 */
gt_status gt_diff_attn_fwd(gt_dtype dtype, const int64_t* rowptr, const int32_t* colidx, const void* Q,
                           const void* K, const void* V, const float* lambda, void* out, float* lse,
                           int64_t N, int64_t E, int32_t H, int32_t D, float scale,
                           const gt_tuning* tuning, hipStream_t stream);

/*
 * Differential attention, backward: gradients of sum(out * dout) for the
 * forward above.  With a_m,e = exp(s_m,e - lse_m) recomputed from the forward's
 * lse, c_e = <dout[i,h,:], V[j_e,h,:]>, Delta_m = sum_e a_m,e c_e, g_0 = 1 and
 * g_1 = -lambda[h]:
 *
 *   ds_m,e = g_m a_m,e (c_e - Delta_m)
 *   dQ[i,2h+m] = scale sum_e ds_m,e K[j_e,2h+m]    (entries of row i)
 *   dK[j,2h+m] = scale sum_e ds_m,e Q[i_e,2h+m]    (entries that name j)
 *   dV[j,h]    = sum_e (a_0,e - lambda[h] a_1,e) dout[i_e,h]
 *   dlambda[h] = -sum_i Delta_1 of row i
 *
 * rowptr_t / colidx_t is the transposed structure, as for gt_attn_bwd.  The
 * forward's out is not needed.  Layouts and shapes as for the forward; dQ, dK
 * [N][2H][D], dV [N][H][2D] in `dtype`, 16-byte aligned; dlambda (may be NULL)
 * float [H].  Gradients must not overlap the inputs or each other.  N == 0 sets
 * dlambda to 0.
 */
gt_status gt_diff_attn_bwd(gt_dtype dtype, const int64_t* rowptr, const int32_t* colidx,
                           const int64_t* rowptr_t, const int32_t* colidx_t, const void* Q, const void* K,
                           const void* V, const float* lambda, const void* dout, const float* lse,
                           void* dQ, void* dK, void* dV, float* dlambda, int64_t N, int64_t E, int32_t H,
                           int32_t D, float scale, hipStream_t stream);

/*
 * Rotary positions with several axes (time, height and width of a video's
 * tokens, coordinates of points or mesh nodes): pairs (x, y) of a head's
 * elements are turned by the angle that their node's position on one axis and
 * their frequency give, in every head alike:
 *
 *   (x, y) <- (x cos t - y sin t, x sin t + y cos t),   t = pos[n][axis] theta^-e
 *
 * The spec (host memory) has `axes` axes, 1 to 4; axis a turns dims[a] elements
 * (even, at least 2), together at most D; the head's other elements pass
 * through.  Which elements make the pair k of axis a, and its exponent e:
 *   GT_ROPE_PAIRS    the axes' sections follow one another; neighbours 2k and
 *                    2k + 1 of the section; e = 2k / dims[a]
 *   GT_ROPE_HALVES   sections likewise; elements k and dims[a] / 2 + k of the
 *                    section; e = 2k / dims[a]
 *   GT_ROPE_SECTIONS one spectrum over all R = sum of dims elements: elements p
 *                    and R / 2 + p of the head, e = 2p / R, and axis a has the
 *                    dims[a] / 2 pairs p after those of the axes before it
 * theta > 0, finite.  The angle is reduced to a part of a turn in 64 bits, so
 * far positions keep their accuracy; the turned values are computed in fp32 and
 * rounded once (bf16: to nearest even).  A node whose angle is not finite (its
 * position is not, or it overflows) gets NaN in that axis' elements.  inverse !=
 * 0 turns by -t: the inverse, which is also the operator's gradient.
 * Layouts: pos float [N][axes], 4-byte aligned; Q, K, outQ, outK [N][H][D] in
 * `dtype`, 16-byte aligned; K and outK may both be NULL.  outQ may be Q itself
 * and outK K itself (in place); other overlaps are refused, as are outputs that
 * overlap pos.  H >= 1; D even, 2 to 512; H * D <= 65536; 0 <= N < 2^31.
 */
typedef enum gt_rope_layout GT_ENUM_BASE {
    GT_ROPE_PAIRS = 0,
    GT_ROPE_HALVES = 1,
    GT_ROPE_SECTIONS = 2
} gt_rope_layout;

typedef struct gt_rope_spec {
    int32_t axes;
    int32_t dims[4];
    int32_t layout; /* gt_rope_layout */
    double theta;
} gt_rope_spec;

gt_status gt_rope(gt_dtype dtype, const float* pos, const void* Q, const void* K, void* outQ, void* outK,
                  int64_t N, int32_t H, int32_t D, const gt_rope_spec* spec, int32_t inverse,
                  hipStream_t stream);

/*
 * Layer norm over rows of F elements:
 *
 *   mean_i = sum_f X[i,f] / F,  rstd_i = 1 / sqrt(sum_f (X[i,f] - mean_i)^2 / F + eps)
 *   out[i,f] = (X[i,f] - mean_i) rstd_i gamma[f] + beta[f]
 *
 * and its backward, for g = dout * gamma and x^ = (X - mean) rstd:
 *
 *   dX = rstd (g - sum_f g / F - x^ sum_f (g x^) / F)
 *   dgamma[f] = sum_i dout[i,f] x^[i,f],  dbeta[f] = sum_i dout[i,f]
 *
 * A per-head norm is the same call with a row for each node and head.
 * Layouts: X, out, dout, dX [N][F] in `dtype`, 16-byte aligned; gamma, beta,
 * dgamma, dbeta float [F], each of which may be NULL (gamma: 1, beta: 0,
 * gradients: not wanted); mean, rstd float [N], which the forward writes if they
 * are not NULL and the backward reads.  1 <= F <= 16384, any F (rows of whole
 * 16-byte vectors are read fastest); 0 <= N < 2^31; eps >= 0, finite (with
 * eps = 0 a constant row gives 0 / 0).  Sums are fp32, the parameters' gradients
 * summed over rows in a fixed order; bf16 outputs are rounded to nearest even.
 * out may be X itself and dX may be X or dout itself; other overlaps are
 * refused.  N == 0 sets dgamma and dbeta to 0.
 */
gt_status gt_layernorm_fwd(gt_dtype dtype, const void* X, const float* gamma, const float* beta, void* out,
                           float* mean, float* rstd, int64_t N, int32_t F, float eps, hipStream_t stream);

gt_status gt_layernorm_bwd(gt_dtype dtype, const void* X, const void* dout, const float* gamma,
                           const float* mean, const float* rstd, void* dX, float* dgamma, float* dbeta,
                           int64_t N, int32_t F, hipStream_t stream);

#undef GT_ENUM_BASE

#ifdef __cplusplus
}
#endif

#endif /* GT_LAYER_H */
