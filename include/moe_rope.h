/*
 * moe_rope.h -- C ABI of rotary positions for rows of queries and keys.
 *
 * The attention layer of moe_attn.h rotates inside its own kernels: whole heads, halves as pairs, one frequency base.  The
 * call here serves callers that bring q and k themselves (moe_kv8_attend, moe_latent_attend): any even part of a head, pairs that
 * lie side by side or half the part apart, and frequencies scaled for contexts longer than a model was trained on.
 *
 * Conventions: as in moe.h (status codes, "dev" / "host", caller-owned memory and streams, row-major).  The call enqueues
 * on `stream` (hipStream_t as void*; null = the default stream), allocates nothing, keeps nothing and never waits, so it can be
 * captured into a graph.  Every tensor must be on one device, which need not be the current one.  The error text of a failed call
 * is moe_rope_last_error() on the same thread.
 */
#ifndef KLOTSKI_MOE_ROPE_H
#define KLOTSKI_MOE_ROPE_H

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Pair i of rot_dim / 2 turns by position * w_i:
 *     (a, b) -> magnitude * (a cos - b sin, b cos + a sin)
 * with w_i = theta^(-2i / rot_dim), scaled by `factor`:
 *   original_len 0: w_i / factor (a longer context squeezed into the positions known);
 *   original_len L > 0: by parts, r_i = L * w_i / (2 pi) being the turns over the original length,
 *     g_i = (r_i - low_turns) / (high_turns - low_turns) cut to 0..1, and w_i * (g_i + (1 - g_i) / factor): pairs that turn often keep
 *     their frequency, those that turn less than low_turns are squeezed (arXiv 2309.00071).
 * Angles are formed and reduced in 64 bits and more; sine and cosine are exact to about a step of 32 bits as long as |position| * w_i is at
 * most 2^31, which theta and factor of 1 and more see to at any position.
 */
typedef struct {
    int32_t rot_dim;      /* elements of a head that turn: even, 2..256 */
    int32_t first;        /* where they begin; the others are copied, or left alone in place */
    int32_t interleaved;  /* 1: pairs (2i, 2i + 1), 0: (i, i + rot_dim / 2), counted from `first` */
    int32_t original_len; /* see above; 0..2^30 */
    double theta;         /* > 0 */
    double factor;        /* > 0; 1: unscaled */
    double low_turns;     /* only with original_len > 0: 0 <= low_turns < high_turns */
    double high_turns;
    double magnitude;     /* factor of what turns, finite in 32 bits; 1: lengths stay */
} moe_rope_config;

/* Rows of heads: element (row, head, i) at row * row_stride + head * head_stride + i. */
typedef struct {
    const void* in;
    void* out;       /* in (then with the same strides), or memory that shares no element with it; heads and rows do not overlap */
    int32_t n_heads; /* 0..1024; 0: nothing, no pointer is looked at */
    int32_t reserved;/* 0 */
    int64_t in_row, in_head, out_row, out_head; /* strides in elements, any that are not negative */
} moe_rope_rows;

/*
 * moe_rope_rotate -- turns the rows of q and, unless null, of k by their positions, in one launch.
 *   dtype: moe_dtype of all rows; head_dim: 2..1024; n_rows: 0..2^24.
 *   out of the one shares no element with in or out of the other.
 *   positions: int32 [n_rows], of any sign.  Negative ones turn back: the transposed rotation, which is also the gradient's, is that
 *     of the negated positions.
 * Products are formed in 32 bits and rounded once.  Rows and parts whose addresses and strides are multiples of 16 bytes move 16 bytes at
 * a time, others element by element, with the same results.
 */
moe_status moe_rope_rotate(void* stream, const moe_rope_config* cfg, int32_t dtype, int32_t n_rows, int32_t head_dim,
                           const int32_t* positions, const moe_rope_rows* q, const moe_rope_rows* k);

/* Error text of the last failed call on the calling thread. */
const char* moe_rope_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* KLOTSKI_MOE_ROPE_H */
