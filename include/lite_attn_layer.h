/*
 * lite_attn_layer.h -- C ABI of what stands before and behind the attention call (lite_attn.h) in a transformer block:
 *
 *   lite_attn_rotary_fwd / _bwd         queries and keys as their projection leaves them -> normalised, turned by their
 *                                       tokens' positions (time, height, width), in the layout the attention call takes
 *   lite_attn_residual_norm_fwd / _bwd  a branch's output -> normalised, gated, added to the residual stream, and the
 *                                       stream's norm, scaled and shifted: the next branch's input
 *
 * Conventions of lite_attn.h: every pointer but the descriptors, argument structs and host_* is a DEVICE pointer on the
 * device that is current; calls are enqueued on `hip_stream` of that device and return at once; nothing is allocated,
 * synchronised or kept from one call for the next; only kernels are launched, so calls may be captured in a HIP graph;
 * nothing throws or aborts; 0 or a negative lite_attn_error is returned, and arguments are checked before anything is
 * launched.  Two calls may run at once, also on two streams, unless they write the same memory (a workspace counts).
 * All arithmetic is done in 32 bits, angles in 64, and every result is rounded once.  Infinities and NaNs spread as the
 * formulas have it, and no further: to their own token, and to the sums over tokens.  Results depend on the arguments
 * alone, to the bit.
 */
#ifndef LITE_ATTN_LAYER_H
#define LITE_ATTN_LAYER_H

#include "lite_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define LITE_ATTN_BF16 0
#define LITE_ATTN_F16 1
#define LITE_ATTN_F32 2

/* Norms. HEAD and ROW (rotary): x / sqrt(mean(x^2) + eps) over head_dim, or over all heads of the token.  RMS and LAYER
   (residual): the same over dim, LAYER after the mean is taken off. */
#define LITE_ATTN_NORM_NONE 0
#define LITE_ATTN_NORM_HEAD 1
#define LITE_ATTN_NORM_ROW 2
#define LITE_ATTN_NORM_RMS 3
#define LITE_ATTN_NORM_LAYER 4

/* ---- rotary positions -------------------------------------------------------------------------------------------------- */

typedef struct {
  int32_t batch, seqlen;    /* tokens of the call (>= 0: nothing to do), of each batch entry */
  int32_t heads_q, heads_k; /* heads of q, >= 1, and of k, >= 0: 0 = the call has no k */
  int32_t head_dim;         /* even, at most 512; under NORM_ROW max(heads_q, heads_k) times head_dim rounded up to a multiple
                               of 8 is at most 8192 (LITE_ATTN_EUNSUPPORTED otherwise) */
  int32_t dtype;            /* of q, k, the results and their gradients */
  int32_t weight_dtype;     /* of q_weight and k_weight */
  int32_t norm;             /* LITE_ATTN_NORM_NONE, _HEAD or _ROW */
  int32_t halves;           /* 0: pair i is the entries (2i, 2i + 1) of a head; 1: (i, i + pairs) */
  int32_t pairs;            /* pairs turned, 0 .. head_dim / 2; entries from 2 * pairs on are not turned */
  int32_t grid[3];          /* frames, height, width of the token grid, each >= 1 */
  float eps;                /* >= 0 */
} lite_attn_rotary_desc_t;

/* One of the tensors [batch, heads, seqlen, head_dim], head_dim contiguous, strides in elements and >= 0: results must not
   have two elements in one place, inputs may (stride 0).  `data` has the alignment of its type.  As many heads as
   fill 512 entries (four of 128) and one more lie within 4 GiB (LITE_ATTN_EUNSUPPORTED otherwise). */
typedef struct {
  void* data;
  int64_t stride_b, stride_h, stride_n;
} lite_attn_heads_t;

/* Where the tokens stand and how fast each pair turns:
     freqs        [3][pairs] 64-bit floats, radians per position: pair i of a token at (p0, p1, p2) turns by
                  p0 freqs[0][i] + p1 freqs[1][i] + p2 freqs[2][i], so a pair may belong to one axis
                  (lite_attn_rotary_freqs) or to several; may be null if pairs = 0
     positions    int32 [batch][3][seqlen], positions_stride_b elements from one batch entry to the next (>= 0; 0: the same
                  for all), or null: token n of the call is token token_start + n of the raster order of the grid, and
                  tokens behind the grid's last (text) stand at (0, 0, 0)
     token_start  >= 0; of use without positions only: a call may hold a part of the sequence, down to a single token */
typedef struct {
  const double* freqs;
  const int32_t* positions;
  int64_t positions_stride_b;
  int32_t token_start;
} lite_attn_positions_t;

typedef struct {
  lite_attn_heads_t q, k;         /* inputs */
  lite_attn_heads_t q_out, k_out; /* results; each either its input itself (same data and strides) or apart from all inputs */
  const void *q_weight, *k_weight; /* [head_dim] (NORM_HEAD) or [heads][head_dim] (NORM_ROW), or null: ones */
  lite_attn_positions_t at;
} lite_attn_rotary_fwd_t;

typedef struct {
  lite_attn_heads_t q, k;           /* the forward pass's inputs; read under a norm only (data may be null without) */
  lite_attn_heads_t dq_out, dk_out; /* gradients of its results */
  lite_attn_heads_t dq, dk;         /* results: gradients of its inputs; each may be its dq_out / dk_out itself */
  const void *q_weight, *k_weight;
  lite_attn_positions_t at;
  float *dq_weight, *dk_weight;     /* results, 32 bits, shaped like the weights, or null: not wanted */
  void* workspace;                  /* lite_attn_rotary_bwd_workspace() bytes, 16-byte aligned; null if that is 0 or no
                                       gradient of a weight is wanted */
  size_t workspace_bytes;
} lite_attn_rotary_bwd_t;

int lite_attn_rotary_fwd(const lite_attn_rotary_desc_t* desc, const lite_attn_rotary_fwd_t* args, void* hip_stream);
int lite_attn_rotary_bwd(const lite_attn_rotary_desc_t* desc, const lite_attn_rotary_bwd_t* args, void* hip_stream);
/* Bytes that lite_attn_rotary_bwd needs for the gradients of the weights; 0 also for a descriptor that is refused. */
size_t lite_attn_rotary_bwd_workspace(const lite_attn_rotary_desc_t* desc);
/* The usual frequencies, on the host: the pairs fall into three sections, axis_pairs[a] >= 0 of them for axis a, in order;
   pair i of an axis' n pairs turns by theta^(-i/n) per position of that axis (theta > 0).  host_freqs: [3][sum of axis_pairs]
   64-bit floats, to be brought to the device by the caller. */
int lite_attn_rotary_freqs(const int32_t axis_pairs[3], double theta, double* host_freqs);

/* ---- residual stream, gate and norms ----------------------------------------------------------------------------------- */

typedef struct {
  int32_t batch, seqlen;     /* seqlen >= 0 */
  int32_t dim;               /* 1 .. 8192 (LITE_ATTN_EUNSUPPORTED beyond) */
  int32_t tokens_per_mod;    /* >= 1: token n of a batch entry has row n / tokens_per_mod of gate, scale and shift: seqlen = one
                                row for a sample, the tokens of a frame = one for a frame, 1 = one for a token */
  int32_t dtype;             /* of y, h and their gradients */
  int32_t stream_dtype;      /* of x, x_out and their gradients: dtype or LITE_ATTN_F32 (else LITE_ATTN_EUNSUPPORTED) */
  int32_t param_dtype;       /* of gate, scale, shift, weights and bias */
  int32_t post_norm, pre_norm; /* LITE_ATTN_NORM_NONE, _RMS or _LAYER: of y, and of the stream */
  float post_eps, pre_eps;   /* >= 0 */
  float residual_scale;      /* finite; of the branch */
} lite_attn_residual_desc_t;

/* [batch, seqlen, dim] or, of gate, scale and shift, [batch, ceil(seqlen / tokens_per_mod), dim]: dim contiguous, strides in
   elements from one batch entry and from one row to the next, >= 0; results must not have two elements in one place. */
typedef struct {
  void* data;
  int64_t stride_b, stride_n;
} lite_attn_rows_t;

/*   p     = post_norm(y) * post_weight
     x_out = x + residual_scale * gate * p
     h     = (pre_norm(x_out) * pre_weight + pre_bias) * (1 + scale) + shift
   h comes from x_out as computed, before it is rounded to stream_dtype.  Left out (data = null): y, and x_out = x; gate: 1;
   scale, shift: 0; post_weight, pre_weight: 1; pre_bias: 0; x_out or h: not wanted (not both). */
typedef struct {
  lite_attn_rows_t x, y;         /* inputs */
  lite_attn_rows_t x_out, h;     /* results; x_out may be x itself and h y itself (same data and strides) */
  lite_attn_rows_t gate, scale, shift;
  const void *post_weight, *pre_weight, *pre_bias; /* [dim] */
} lite_attn_residual_fwd_t;

/* x_out is what the forward pass stored.  Sums over tokens are in 32 bits and one fixed order; gate, scale and shift that
   batch entries share (stride 0) get a gradient for each.
   Needed: dh or dx_out (null: zero); x_out, if dh is there and pre_norm or a gradient of scale or pre_weight asks for it; y,
   if post_norm or a gradient of gate or post_weight asks for it. */
typedef struct {
  lite_attn_rows_t dh, dx_out;   /* gradients of the forward pass's results */
  lite_attn_rows_t x_out, y;
  lite_attn_rows_t dx, dy;       /* results, or null: not wanted; dx may be dx_out itself and dy be dh or y itself */
  lite_attn_rows_t gate, scale;
  const void *post_weight, *pre_weight, *pre_bias;
  float *dgate, *dscale, *dshift;                /* results [batch][ceil(seqlen / tokens_per_mod)][dim], or null */
  float *dpost_weight, *dpre_weight, *dpre_bias; /* results [dim], or null */
  void* workspace;               /* lite_attn_residual_norm_bwd_workspace() bytes, 16-byte aligned; null if none of the six is
                                    wanted */
  size_t workspace_bytes;
} lite_attn_residual_bwd_t;

int lite_attn_residual_norm_fwd(const lite_attn_residual_desc_t* desc, const lite_attn_residual_fwd_t* args, void* hip_stream);
int lite_attn_residual_norm_bwd(const lite_attn_residual_desc_t* desc, const lite_attn_residual_bwd_t* args, void* hip_stream);
size_t lite_attn_residual_norm_bwd_workspace(const lite_attn_residual_desc_t* desc);

#ifdef __cplusplus
}
#endif
#endif /* LITE_ATTN_LAYER_H */
