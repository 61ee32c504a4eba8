/*
 * hp_packed.h - C ABI of states and weights held in 4 bits, for AMD MI355X (gfx950).
 *
 * A language model that decodes through a cross-attention layer reads, for every
 * token, the states that its request keeps and the weights of the projections, and
 * computes next to nothing with them.  Here both are held packed:
 *   - hp_pack, hp_unpack      rows of heads (or of a matrix) to packed rows and back,
 *   - hp_packed_attend_step   hp_cross_attend_step against packed states,
 *   - hp_packed_linear        a few rows times a packed weight matrix.
 * They serve; there are no gradients.  Rows that have much in common, as a second
 * prompt against the states of the first, read the states back (hp_unpack) and go
 * through hp_cross_attend.
 *
 * Conventions are those of hp_operators.h: streams, memory, codes, strides, types.
 *
 * The packed form.  The channels of a row (and head) are groups of 32, the last one
 * shorter; a group has a step and a low value in bfloat16 and a code of 4 bits a
 * channel, and stands for
 *     value = low + step * code.
 *   codes:  16 bytes a group, one behind the other: four 32-bit words (little endian),
 *           of which word w has channel 8w + 2i in bits 4i .. 4i + 3 and channel
 *           8w + 2i + 1 in bits 16 + 4i .. 19 + 4i, i < 4.
 *   scales: [groups, 2] bfloat16, (step, low).
 * hp_pack takes, of a group's values, low = the largest bfloat16 that is not above the
 * least, step = the least bfloat16 that is not below (greatest - low) / 15 (zero where
 * that is below 2^-126), and for each value the code of the nearest level, of the lower
 * of two: no value is farther than step / 2 from its own.  A group with a value that is
 * not finite (or below -3.3895e38, which no bfloat16 is) has NaN for its step and low, and
 * all of it reads back as NaN.  (Where the greatest value is within step of the largest
 * binary32 number, 3.4028e38, its level may be beyond and read back as infinite.)  Codes
 * of channels that a shorter group lacks are zero and are not read for their value.
 */
#ifndef HP_PACKED_H_
#define HP_PACKED_H_

#include "hp_operators.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HP_PACKED_GROUP   32
#define HP_PACKED_MAX_DIM 65536

/* Packed rows of heads: codes of (row, head) at codes + row * code_row_stride + head *
 * code_head_stride, in bytes, scales at scales + row * scale_row_stride + head *
 * scale_head_stride, in bfloat16 elements.  Codes are 16-byte aligned with strides that
 * are multiples of 16, scales 4-byte aligned with even strides (HP_EALIGN).  Attention is
 * fastest where the rows of a head lie one behind the other. */
typedef struct hp_packed {
    void *codes, *scales;
    int64_t code_row_stride, code_head_stride;
    int64_t scale_row_stride, scale_head_stride;
} hp_packed_t;

/* ---- packing as states are written, and reading back ---------------------- */

#define HP_PACK_MAX_TENSORS 4

/* hp_pack:   packed[t] = x[t] [rows, heads[t], dim], of up to four tensors (keys and
 *            values); dim up to HP_PACKED_MAX_DIM, heads x groups up to 4194240 (HP_ELAYOUT).
 * hp_unpack: x[t] = the values of packed[t], in binary32 and rounded once to the type.
 * No output may overlap an input, another output or itself. */
typedef struct hp_pack_args {
    int32_t dtype, n_tensors, dim, reserved;
    int64_t rows;
    int32_t heads[HP_PACK_MAX_TENSORS];      /* up to 65536 each */
    hp_heads_t x[HP_PACK_MAX_TENSORS];
    hp_packed_t packed[HP_PACK_MAX_TENSORS];
} hp_pack_args_t;
int hp_pack(const hp_pack_args_t *args, void *stream);
int hp_unpack(const hp_pack_args_t *args, void *stream);

/* ---- attention of single tokens to packed states --------------------------- */

/* hp_packed_attend_step - hp_cross_attend_step with k and v packed: every row makes its
 * own pass over its range, and what it does not see has no influence on it.  The states'
 * values enter as they are, not rounded to the type.  In HP_BF16 two numbers on the way
 * are rounded to 16 bits, the weights P and P * step, operands of matrix products
 * (HP_F32: none).  Sums on the way may be 2^11 times the number of states times the largest
 * value of v: values from 2^90 on are not safe from overflow; nor are queries from 2^118 on
 * (HP_F32: 2^122), or those whose sum over the channels of |q| times the largest value of k
 * is 2^125 or more, before the scale.  A state that is seen and is NaN in a group of v leaves
 * NaN in that group's channels, whatever its weight; queries that are not finite, NaN in
 * their head's.
 * How a call is cut goes by its rows and by the rows of the cache, not by what ranges leave of
 * them: one row of up to 1023 states (dim above 128: 895) is one launch, longer caches and
 * several rows are shared out and joined by a second, where a row's last bits may go by the
 * other rows' ranges (up to 512 rows; of more, each is by itself).  A short request in a large cache is
 * faster if k and v are the rows that it sees (32 heads of 128 on 8, one row of 576 states:
 * 10.2 us, in a cache of 100000: 12.5).
 *   q, out: [rows, heads_q, dim]; k, v: [keys, heads_k, dim]; dim 1..HP_ATTEND_MAX_DIM.
 *   Limits are hp_cross_attend_step's; row strides of packed states up to 2^24 (HP_ELAYOUT),
 *   none negative.
 *   workspace: hp_packed_attend_workspace bytes, 16-byte aligned; that may be zero. */
typedef struct hp_packed_attend_args {
    int32_t dtype;
    int32_t heads_q, heads_k, dim;
    int64_t rows, keys;
    float scale;
    int32_t reserved;
    hp_heads_t q, out;
    hp_packed_t k, v;
    const int32_t *ranges;
    float *lse;
    void *workspace;
    int64_t workspace_bytes;
} hp_packed_attend_args_t;
int hp_packed_attend_step(const hp_packed_attend_args_t *args, void *stream);
/* Bytes of scratch memory; of the struct only dtype, heads, dim, rows and keys are read. */
int64_t hp_packed_attend_workspace(const hp_packed_attend_args_t *args);

/* ---- a few rows times packed weights ----------------------------------------- */

/* hp_packed_linear - out[r][n] = sum_k x[r][k] w[n][k] for x [rows, n_in], packed w
 * [n_out, n_in] (one head: head strides are not read) and out [rows, n_out].  Sums are in
 * binary32, the weights' values are not rounded (in HP_BF16 the part of the lows may be off
 * by 2^-18 of 16 step + |low| times a group's sum of x); out may not overlap x; a row of x that
 * is not finite gives NaN.  Sums on the way may be 32 times a group's sum of |x| (HP_F32: twice
 * it), and 8 times what these sums of |x|, each times its group's largest value in w's row, add
 * up to: values of x from 2^118 on (HP_F32: 2^122) are not safe from overflow, and the latter
 * has to stay below 2^128.
 * Made for the rows of a decoding step: up to 32 rows at a time share a pass over the
 * weights.  Fastest where x is 16-byte aligned and its rows and their stride
 * are multiples of 16 bytes.
 * n_in up to HP_PACKED_MAX_DIM, n_out up to 2^24, rows up to 2^20, row strides of w up
 * to 2^24 and not negative (HP_ELAYOUT). */
typedef struct hp_packed_linear_args {
    int32_t dtype, n_in, n_out, reserved;
    int64_t rows;
    const void *x;
    int64_t x_stride;
    hp_packed_t w;
    void *out;
    int64_t out_stride;
} hp_packed_linear_args_t;
int hp_packed_linear(const hp_packed_linear_args_t *args, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HP_PACKED_H_ */
