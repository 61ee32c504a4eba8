/*
 * hp_operators.h - C ABI of the operators of a cross-attention layer over a
 * boundary, for AMD MI355X (gfx950).
 *
 * The boundary transform (hp.h) puts an encoder's tokens into the language
 * model's sequence.  The other way for a language model to take them in is a
 * layer whose queries attend to the encoder's states.  Between the projections
 * of such a layer (plain matrix products) stand
 *   - rotary positions in the heads of queries and keys   (hp_rotary),
 *   - attention to packed states of another length        (hp_cross_attend),
 *   - norms before and after the block with its gate and
 *     the scale of the residual stream                    (hp_gated_norm),
 * each with its gradient, and attention for single tokens (hp_cross_attend_step).
 *
 * Conventions are hp.h's: element types HP_BF16 and HP_F32; every call enqueues
 * its kernels on the caller's stream (a hipStream_t as void*, NULL = the default
 * stream) of the current device, is ordered against that stream only, allocates
 * nothing and returns without synchronising; the caller owns all memory, scratch
 * memory among it, until the stream has passed the call; calls return HP_OK or a
 * negative HP_E* code, write nothing on failure, and neither throw nor abort.
 * All calls may be recorded into a HIP graph.  Structs are read during the call
 * only.  Strides count elements.  Pointers need the alignment of their element
 * type, no more.  Zero rows are in order: nothing is launched.
 *
 * Sums, softmax statistics and angles are held in binary32 or more whatever the
 * element type; results are rounded once, to nearest even.  Attention in HP_BF16
 * rounds two values on the way as well, the weights P and the gradients dS of the
 * scores, which are bfloat16 operands of a matrix product (HP_F32: none).  For equal
 * inputs the results are the same bits on every call: no sum depends on the order in
 * which workgroups finish.
 */
#ifndef HP_OPERATORS_H_
#define HP_OPERATORS_H_

#include "hp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of heads: element (row, head, channel) at data[row * row_stride + head * head_stride + channel]. */
typedef struct hp_heads {
    void *data;
    int64_t row_stride, head_stride;
} hp_heads_t;

/* ---- rotary positions ---------------------------------------------------- */

#define HP_ROTARY_PLAIN    0   /* f_i = base^(-2i/rot)                                           */
#define HP_ROTARY_LINEAR   1   /* f_i / factor: positions drawn together                         */
#define HP_ROTARY_BASE     2   /* base * factor^(rot/(rot-2)): the lowest frequency is divided by
                                  factor, the highest kept (rot >= 4)                            */
#define HP_ROTARY_BY_TURNS 3   /* pairs that turn low_turns times or fewer over original_length
                                  positions are divided by factor, those that turn high_turns
                                  times or more are kept, linear in the turns between            */

typedef struct hp_rotary_scaling {
    int32_t kind;
    int32_t reserved;
    double base;               /* > 0, 10000 as a rule                                           */
    double factor;             /* > 0; not read for HP_ROTARY_PLAIN                              */
    double original_length;    /* HP_ROTARY_BY_TURNS only: > 0                                   */
    double low_turns, high_turns;   /* HP_ROTARY_BY_TURNS only: low < high                       */
    double amplitude;          /* multiplies cosine and sine; 1 as a rule                        */
} hp_rotary_scaling_t;

/* hp_rotary_table - cosines and sines of positions first .. first + n - 1:
 * table[p][i] = amplitude * (cos, sin)((first + p) * f_i), i < rot/2, binary32
 * [n, rot/2, 2], computed in binary64 and rounded once, so that angles of
 * 131072 positions and more carry no error of their own. */
int hp_rotary_table(float *table, int64_t n, int64_t first, int32_t rot,
                    const hp_rotary_scaling_t *scaling, void *stream);

#define HP_ROTARY_MAX_TENSORS 4
#define HP_ROTARY_MAX_AXES    4

/* hp_rotary - turns the first `rot` channels of every head by its row's
 * positions: for pair i with channels a, b and (c, s) = table[position][i],
 *     out_a = x_a c - x_b s,   out_b = x_b c + x_a s.
 * interleaved = 0: a = i, b = i + rot/2; otherwise a = 2i, b = 2i + 1.  Channels
 * from rot on are copied.  inverse != 0 takes -s: the gradient of the call with
 * respect to x (and, with amplitude 1, its inverse).
 * With n_axes > 1 the pairs are split into sections[0..n_axes), whose sum is
 * rot/2, and each section goes by a position of its own:
 * positions[axis * axis_stride + row].
 * A position that is not in [0, table_rows) leaves NaN in the turned channels of
 * its row.  out[t] may be x[t] with the same strides (in place); otherwise no
 * output may overlap an input or another output. */
typedef struct hp_rotary_args {
    int32_t dtype, n_tensors;
    int32_t dim, rot;          /* channels of a head (up to 1024), of which the first rot are turned
                                  (rot even, 2..dim)                                             */
    int32_t interleaved, inverse;
    int32_t n_axes;
    int32_t sections[HP_ROTARY_MAX_AXES];   /* not read for n_axes = 1 */
    int32_t reserved;
    int64_t rows;
    const float *table;
    int64_t table_rows;
    const int32_t *positions;
    int64_t axis_stride;
    int32_t heads[HP_ROTARY_MAX_TENSORS];   /* up to 4096 each */
    hp_heads_t x[HP_ROTARY_MAX_TENSORS], out[HP_ROTARY_MAX_TENSORS];
} hp_rotary_args_t;
int hp_rotary(const hp_rotary_args_t *args, void *stream);

/* ---- norms around a block, its gate and the residual stream --------------- */

#define HP_NORM_MAX_HIDDEN 32768

/* hp_gated_norm - the residual stream behind one block and in front of the next:
 *     n = y * w_post / sqrt(mean(y^2) + eps)      (w_post NULL: n = y)
 *     h = residual_scale * x + t * n              (y NULL: h = residual_scale * x)
 *     z = h * w_pre / sqrt(mean(h^2) + eps)       (w_pre NULL: no z)
 * with t = gate or tanh(gate) (gate_tanh), one value or one for each channel
 * (gate_size 1 or hidden; gate NULL: t = 1).  unit_offset: weights are 1 + w.
 * z goes by h before its rounding.  rstd (binary32 [2, rows], may be NULL)
 * receives the factors 1/sqrt(..) of y and of h, 1 where there is no norm.
 * h or z may be NULL if not wanted (not both).  h may be x or y in place, z may
 * be x or y, with the same stride (HP_EINVAL); other overlaps are not allowed. */
typedef struct hp_norm_args {
    int32_t dtype;
    int32_t gate_size, gate_tanh, unit_offset;
    int64_t rows;
    int32_t hidden;
    float residual_scale, eps;
    int32_t reserved;
    const void *x, *y;         /* [rows, hidden], rows x_stride, y_stride apart                  */
    int64_t x_stride, y_stride;
    void *h, *z;
    int64_t h_stride, z_stride;
    const void *w_post, *gate, *w_pre;
    float *rstd;
} hp_norm_args_t;
int hp_gated_norm(const hp_norm_args_t *args, void *stream);

/* hp_gated_norm_backward - gradients of the above.  `f` is the forward's struct
 * (its h and z are not read; rstd, filled by the forward, is needed).
 *   dh, dz: gradients of h and z [rows, hidden]; one of them may be NULL (zero).
 *   dx, dy: [rows, hidden], each may be NULL; dx may be dh or dz in place, with the
 *     same stride (HP_EINVAL), dy too.
 *   dw_post, dgate, dw_pre: of the weights' shapes and type, overwritten; each may
 *     be NULL.  Sums over rows are in binary32, in an order that follows from the
 *     sizes alone.
 *   workspace: hp_gated_norm_workspace(rows, hidden) bytes, 16-byte aligned; may be
 *     NULL if dw_post, dgate and dw_pre are. */
typedef struct hp_norm_grads {
    const void *dh, *dz;
    int64_t dh_stride, dz_stride;
    void *dx, *dy;
    int64_t dx_stride, dy_stride;
    void *dw_post, *dgate, *dw_pre;
    void *workspace;
    int64_t workspace_bytes;
} hp_norm_grads_t;
int hp_gated_norm_backward(const hp_norm_args_t *f, const hp_norm_grads_t *g, void *stream);
int64_t hp_gated_norm_workspace(int64_t rows, int32_t hidden);

/* ---- cross attention ------------------------------------------------------- */

#define HP_ATTEND_MAX_DIM 256

/* hp_cross_attend - attention of packed query rows to packed states: query row r
 * sees the states ranges[2r] .. ranges[2r+1] - 1 (ranges NULL: all of them),
 *     out[r][h] = sum_j softmax_j(scale * q[r][h] . k[j][h']) v[j][h'],
 * h' = h / (heads_q / heads_k).  Samples of any lengths are rows and states one
 * behind the other; causal and image-by-image masks are ranges.  Parts of a range
 * outside [0, keys) count as not there; a row whose range is empty gets zeros.
 * What a row does not see has no influence on it, whatever the values there are
 * (infinities and NaN included).  Rows next to each other should see much the
 * same states: up to 128 / group of them share the pass over what any of them sees.
 *   q, out: [rows, heads_q, dim]; k, v: [keys, heads_k, dim]; dim 1..256, heads_q up to
 *           16384 and a multiple of heads_k.  rows * heads_q / heads_k up to 2^30 - 1024,
 *           keys up to 2^31 - 1025 (HP_ELAYOUT).
 *   lse:    binary32 [rows, heads_q], may be NULL: receives the natural logarithm
 *           of the sum of exponentials, -inf for an empty row.
 *   scale:  > 0.
 *   workspace: hp_cross_attend_workspace(args, HP_ATTEND_FORWARD) bytes, 16-byte
 *           aligned; that may be zero. */
typedef struct hp_attend_args {
    int32_t dtype;
    int32_t heads_q, heads_k, dim;
    int64_t rows, keys;
    float scale;
    int32_t reserved;
    hp_heads_t q, k, v, out;
    const int32_t *ranges;
    float *lse;
    void *workspace;
    int64_t workspace_bytes;
    hp_heads_t dout, dq, dk, dv;            /* hp_cross_attend_backward only */
} hp_attend_args_t;
int hp_cross_attend(const hp_attend_args_t *args, void *stream);

/* hp_cross_attend_step - the same function for rows that have nothing in common,
 * as the single tokens of many requests against a cache of their states: every
 * row makes its own pass over its range, long ranges in several parts.  Up to
 * 2^23 rows (HP_ELAYOUT). */
int hp_cross_attend_step(const hp_attend_args_t *args, void *stream);

/* hp_cross_attend_backward - gradients of hp_cross_attend (or _step) from its
 * inputs, out, lse and the gradient dout of out.  dq, dk and dv are overwritten
 * whole: states that no row sees get zeros.  Heads that share a state head add up
 * in binary32.  In bf16 keys up to 2^30 - 1024 (HP_ELAYOUT).
 * Workspace: hp_cross_attend_workspace(args, HP_ATTEND_BACKWARD). */
int hp_cross_attend_backward(const hp_attend_args_t *args, void *stream);

#define HP_ATTEND_FORWARD  0
#define HP_ATTEND_STEP     1
#define HP_ATTEND_BACKWARD 2
/* Bytes of scratch memory that a call needs; of the struct only dtype, heads, dim, rows and keys are read.
 * Negative HP_E* code on sizes that the call refuses. */
int64_t hp_cross_attend_workspace(const hp_attend_args_t *args, int32_t call);

/* hp_image_ranges - the ranges of a sequence's positions for hp_cross_attend when
 * the states are the image tokens of a token map, packed in its order (what a
 * source buffer of the boundary holds): ranges[2 * (b * seq + p)] and the entry
 * behind it for position p of sample b.  An image has as many states as places in
 * the sequence; where each place stands for n states, the ranges are n times these.
 * Host memory, no HIP call.
 *   HP_SEE_SAMPLE:   every image of the sample;
 *   HP_SEE_PREVIOUS: the sample's images that end at or before p;
 *   HP_SEE_LATEST:   the last of these alone.
 * The latter two need a sample's images in ascending places (HP_EMAP). */
#define HP_SEE_SAMPLE   0
#define HP_SEE_PREVIOUS 1
#define HP_SEE_LATEST   2
int hp_image_ranges(const hp_token_map_t *map, int32_t rule, int32_t *ranges);

#ifdef __cplusplus
}
#endif
#endif /* HP_OPERATORS_H_ */
