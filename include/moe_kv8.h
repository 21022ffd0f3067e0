/*
 * moe_kv8.h -- C ABI of the key-value cache held in 8 bits: filling it, attending over it, evicting from it.
 *
 * The attention layer of moe_attn.h is bound by the bytes of its bf16 caches, in HBM and over the host link.  The
 * calls here keep a cache in half the bytes and in a bounded number of slots, for sequences of different lengths,
 * for single tokens and for prompts.  moe_attn_forward_kv8 (moe_attn.h) runs the whole attention layer over such a cache;
 * the calls here serve callers that bring q, k and v themselves.
 *
 * The cache.  For every sequence and key-value head, max_len slots of head_dim elements as e4m3 codes (sign, 4
 * exponent bits with bias 7, 3 fraction bits; largest number 448, codes 0x7f and 0xff NaN, no infinity) and one scale for
 * each `block` consecutive slots, K and V apart.  The value of a code is code * scale.  A scale is a power of two,
 * from 2^-100 to 2^119: a value is then exact in bf16, and raising the scale of a block loses nothing but what falls
 * below the smallest codes.  What lies in slots a sequence does not hold is never used, whatever it is.
 * A sequence holds slots 0 .. held-1; attention does not depend on the order of the slots, so slots need not be in the
 * order of the positions (moe_kv8_evict fills the slots it frees from the end).
 *
 * Conventions: as in moe.h (status codes, "dev" / "host", caller-owned memory and streams, row-major).  All
 * tensors are device memory; the calls enqueue on `stream` (hipStream_t as void*; null = the default stream), allocate
 * nothing, keep nothing and never wait, so they can be captured into a graph.  The numbers of slots and rows
 * per sequence are read on the device when the kernels run; the host gives bounds of them, which size the launches.
 * A number outside its bounds is taken as the nearest one inside: it can give wrong results, never an access out of the
 * tensors.  Calls that share neither cache, workspace nor outputs may run at once; a workspace may be used again by
 * the next call on the same stream (not by two graphs that may run at once).  Every tensor must be on one device,
 * which need not be the current one.  The error text of a failed call is moe_kv8_last_error() on the same thread.
 * A launch has at most 2^24 - 1 workgroups; a call whose sizes and bounds ask for more is MOE_ERR_SHAPE.  With pairs = n_seq *
 * n_kv_heads, and divisions rounded up, calls are within that if these are:
 *   append  2 * pairs * (blocks of a sequence that min(max_new, n_rows) tokens can fall into)
 *   attend  pairs * (min(max_new, n_rows) * n_q_heads / n_kv_heads / 128), and with weight_out
 *           pairs * (min(max_cached + max_new, max_len) / 128), too
 *   evict   pairs * (keep / 512)
 */
#ifndef KLOTSKI_MOE_KV8_H
#define KLOTSKI_MOE_KV8_H

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The cache of one layer: device memory, owned by the caller. */
typedef struct {
    int32_t n_seq;      /* 1..65536 */
    int32_t n_kv_heads; /* 1..1024; n_seq * n_kv_heads at most 2^20 */
    int32_t head_dim;   /* 32, 64 or 128 */
    int32_t max_len;    /* slots of a sequence: a multiple of block, at most 2^20 */
    int32_t block;      /* slots that share a scale: 16, 32, 64 or 128 */
    int32_t reserved;   /* 0 */
    void* k;            /* codes, uint8 [n_seq, n_kv_heads, max_len, head_dim], 16-byte aligned */
    void* v;
    float* k_scale;     /* [n_seq, n_kv_heads, max_len / block] */
    float* v_scale;
    int32_t* position;  /* [n_seq, n_kv_heads, max_len]: position of the token in a slot; may be null (then not
                           recorded, and nothing can be evicted) */
} moe_kv8_cache;

/* The new tokens of one step, shared by the layers of a model.  Sequence s brings the rows row_offsets[s] ..
 * row_offsets[s+1]-1 of q, k, v and out; its tokens take the slots from cached[s] on.  The arrays stay as they are: after
 * the last layer the caller adds the new tokens to `cached`.  A token that would take a slot from max_len on does not
 * exist: it is not stored, and its rows of out are left as they were. */
typedef struct {
    int32_t n_rows;     /* rows of all sequences, 0..2^20 */
    int32_t max_new;    /* tokens a sequence brings, at most */
    int32_t max_cached; /* slots a sequence holds before them, at most; neither bound is over max_len */
    int32_t reserved;   /* 0 */
    const int32_t* row_offsets;   /* [n_seq + 1], non-decreasing; null: every sequence brings max_new rows */
    const int32_t* cached;        /* [n_seq] slots held before the step */
    const int32_t* next_position; /* [n_seq] position of the first new token; null: cached, for sequences that have never been
                                     evicted from (behind an eviction positions run ahead of the slots held) */
} moe_kv8_step;

/*
 * moe_kv8_append -- quantises the new tokens' k and v (bf16, element (row, head, i) at row * row_stride + head *
 * head_stride + i; 16-byte aligned, strides multiples of 8) into the cache, and writes their positions.
 * For each block a sequence's tokens fall into: a = the largest magnitude among the new finite elements; the scale
 * becomes the least power of two s with a <= 448 s, but no less than the block's scale if the block held slots
 * before; codes the block held are rounded to the new scale, new ones are x / s, to nearest even.  Infinities become the
 * largest code, NaN stays NaN (neither moves the scale).  Prompts and single tokens thus give the same values, but for
 * the roundings of codes that a later, larger token pushes below the smallest normal code.
 */
moe_status moe_kv8_append(void* stream, const moe_kv8_cache* cache, const moe_kv8_step* step,
                          const void* k_new, const void* v_new, int64_t row_stride, int64_t head_stride);

/*
 * moe_kv8_attend -- softmax attention of the new tokens over the cache, after moe_kv8_append of the same step: token i
 * of sequence s sees slots 0 .. cached[s] + i, so the whole past and the new tokens up to itself.
 *   q, out: bf16, element (row, head, i) at row * row_stride + head * head_stride + i; 16-byte aligned, strides
 *     multiples of 8; no two (row, head) of out may share an element.  Without weight_out, out may be q with the same
 *     strides; else they share no element.  n_q_heads: a multiple of n_kv_heads, at most 8 times it.
 *   softmax_scale: factor of the scores; 0 stands for 1 / sqrt(head_dim).
 *   weight_out (may be null): [n_seq, n_kv_heads, max_len] accumulated attention weights.  Slot j of sequence s
 *     gets weight_in's value (0 for new slots, or for all when weight_in is null) plus the softmax weights that the
 *     step's tokens and the head's query heads gave it; weight_in may be weight_out.  Slots a sequence does
 *     not hold are left as they were.
 * Rows of no sequence are left as they were; of a step without rows q and out are not looked at.  Scores, the softmax's
 * statistics and all sums are kept in 32 bits, and so are the accumulated weights.  The weights enter the matrix product with V
 * as bf16: as two of them, with 16 bits together, where min(max_new, n_rows) * n_q_heads / n_kv_heads is at most 16, rounded once
 * (by up to 2^-8 of each weight) where it is more, so that a token's output is more exact decoded than within a prompt.  The result of
 * a sequence does not depend on what the others hold; how its sums are split follows from the numbers in the structs
 * and its own length.
 * workspace: moe_kv8_attend_workspace_bytes() of device memory, 256-byte aligned (may be null when that is 0).  It
 * depends on the sizes and bounds only.
 */
moe_status moe_kv8_attend_workspace_bytes(const moe_kv8_cache* cache, const moe_kv8_step* step, int32_t n_q_heads,
                                          int32_t with_weights, int64_t* bytes_out);
moe_status moe_kv8_attend(void* stream, const moe_kv8_cache* cache, const moe_kv8_step* step, int32_t n_q_heads,
                          const void* q, int64_t q_row_stride, int64_t q_head_stride, float softmax_scale, void* out,
                          int64_t out_row_stride, int64_t out_head_stride, const float* weight_in,
                          float* weight_out, void* workspace, int64_t workspace_bytes);

/*
 * moe_kv8_evict -- brings every sequence that holds more than `keep` slots down to `keep`, per key-value head: the slots
 * whose position is at least next_position[s] - recent stay (recent 0: none for its position), and of the others those with
 * the largest weight (ties: the lower slot; NaN: last), `keep` in all.  Chosen slots below `keep` stay where they are; the i-th slot below `keep` that
 * was not chosen takes over the i-th chosen slot from `keep` on: codes, weight, position.  A block's scale becomes the
 * largest of its own and those that come in, and its codes are rounded to it.  The caller then sets the
 * sequence's number of slots to min(held, keep).  Sequences that hold `keep` or fewer keep everything.
 *   keep: a multiple of block, 1..max_len;  recent: 0..keep;  held: [n_seq], at most max_held <= max_len.
 *   next_position: [n_seq], position of the token to come; null: held, which is that position only in sequences that have
 *     never been evicted from and began at position 0.  Behind an eviction positions run ahead of the slots held: with null all
 *     of them would count as recent, and weights decide nothing.
 *   weight_in -> weight_out: as in moe_kv8_attend, the same tensor or two that do not overlap; of weight_out
 *     only slots below min(held, keep) are written.
 *   position_out: where the positions go (again only below min(held, keep)); null: into cache->position itself.
 *   kept (may be null): [n_seq, n_kv_heads, keep], the slot that each slot was before; -1 from `held` on.
 * workspace: moe_kv8_evict_workspace_bytes(), 256-byte aligned.
 */
moe_status moe_kv8_evict_workspace_bytes(const moe_kv8_cache* cache, int32_t keep, int64_t* bytes_out);
moe_status moe_kv8_evict(void* stream, const moe_kv8_cache* cache, const int32_t* held, int32_t max_held, int32_t keep,
                         int32_t recent, const int32_t* next_position, const float* weight_in, float* weight_out,
                         int32_t* position_out, int32_t* kept, void* workspace, int64_t workspace_bytes);

/* Error text of the last failed call on the calling thread. */
const char* moe_kv8_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* KLOTSKI_MOE_KV8_H */
