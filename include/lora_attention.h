/*
 * liblora_gfx950 -- between the adapted projections of a layer: rotary positions, a paged cache of keys and values, attention over it.
 *
 * q, k and v of a batch come from lora_apply_multi (or lora_linear_scaled and lora_apply); these calls take them to the input of the output
 * projection, on the same terms as the rest of the library (same status codes, lora_last_error, streams, pointers, no allocation, no
 * synchronisation; every argument is checked on the host before the device is touched, and nothing throws or aborts):
 *
 *     lora_rotary_turns    the frequencies of a rotary position, as the fraction of a turn that each pair makes in a position
 *     lora_rotary          rows turned by their positions, and the gradient of that
 *     lora_cache_append    keys and values into the cache, keys turned on the way, and the same tokens' queries with them
 *     lora_attention       softmax(q k^T) v over the cache: single tokens, drafted trees, prompts and mixtures of them
 *
 * The cache is cut into pages of page_size slots.  A slot holds the key and the value of one token, per key head: k and v are
 * [pages][kv_heads][page_size][head_dim], in bf16, or in OCP E4M3 with one fp32 scale per slot and head ([pages][kv_heads][page_size]) for each:
 * value = byte * scale.  Which pages are whose, and in what order, is the caller's; the calls read it on the device.
 *
 * Device data that the calls read as indices (positions, slots, starts, lengths, page numbers) is checked where it is used: what fits nothing
 * reaches no memory outside the buffers.
 */
#ifndef LORA_ATTENTION_GFX950_H
#define LORA_ATTENTION_GFX950_H

#include "lora.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LORA_MAX_HEAD_DIM 256
#define LORA_MAX_HEADS 4096
#define LORA_MAX_PAGE 1024

/* A rotary position.  Pair i of `dims` / 2 is turned by positions * turns[i] / 2^64 turns; turns: device, 8-byte aligned, [dims / 2].  The pairs are elements i and
 * i + dims / 2 of a head, or 2 i and 2 i + 1 where `interleaved`; elements from `dims` on stay as they are.  dims: a multiple of 16, up to head_dim.
 * With a the angle:  y1 = m (x1 cos a - x2 sin a),  y2 = m (x1 sin a + x2 cos a),  m = magnitude. */
typedef struct {
    const uint64_t *turns;
    int32_t dims;
    int32_t interleaved;
    float magnitude;
} lora_rotary_t;

typedef struct {
    void *k, *v;                 /* device, 16-byte aligned */
    float *k_scales, *v_scales;  /* device; 8 bits only */
    int32_t pages;
    int32_t page_size;           /* a power of two, 16 .. LORA_MAX_PAGE */
    int32_t kv_heads;
    int32_t head_dim;            /* 64 or 128 */
    int32_t bits;                /* 16 (bf16) or 8 (E4M3) */
} lora_cache_t;

/* Frequencies.  Pair i turns by f_i = base^(-2 i / dims) radians a position, changed for longer contexts by `scaling`:
 *   LORA_ROTARY_PLAIN       f_i
 *   LORA_ROTARY_LINEAR      f_i / factor
 *   LORA_ROTARY_WAVELENGTH  by how often a pair turns in the original `length`, n_i = length f_i / 2 pi:  s f_i + (1 - s) f_i / factor,
 *                           s = (n_i - low) / (high - low) held to 0 .. 1
 *   LORA_ROTARY_DIMENSION   by the pair's number: s f_i + (1 - s) f_i / factor,  s = 1 - (i - a) / max(b - a, 0.001) held to 0 .. 1, where
 *                           a = floor(pair that turns `high` times in `length`), at least 0, b = ceil(pair that turns `low` times), at most dims - 1;
 *                           that pair is dims ln(length / (2 pi n)) / (2 ln base).  The magnitude is then 0.1 ln(factor) + 1, else 1.
 * factor, low, high and length are of no account where the kind does not name them.  Host only: turns is host memory, [dims / 2], which the caller copies to the
 * device; turns[i] = f_i / 2 pi in units of 2^-64, so that an angle is exact to 2^-31 turns at any position of 32 bits.  magnitude may be NULL. */
#define LORA_ROTARY_PLAIN 0
#define LORA_ROTARY_LINEAR 1
#define LORA_ROTARY_WAVELENGTH 2
#define LORA_ROTARY_DIMENSION 3
lora_status_t lora_rotary_turns(int32_t dims, double base, int32_t scaling, double factor, double low, double high, double length,
                                uint64_t *turns, float *magnitude);

/* y[t][h] = x[t][h] turned by positions[t].  `inverse` != 0: by -positions[t], which is the gradient's way (dx of dy; the magnitude is applied all the same).
 * x, y: device, bf16, 16-byte aligned, [tokens][heads][head_dim]; strides of a token and of a head in elements, multiples of 8; y may be x with its
 * strides, and must not overlap it otherwise.  head_dim: a multiple of 16 up to LORA_MAX_HEAD_DIM.  positions: device, int32, [tokens]; a row whose position is
 * negative is passed over: y's stays as it is.  The arithmetic is fp32, y is rounded once. */
lora_status_t lora_rotary(const void *x, int64_t x_token, int64_t x_head, int32_t tokens, int32_t heads, int32_t head_dim,
                          const int32_t *positions, const lora_rotary_t *rotary, int32_t inverse, void *y, int64_t y_token, int64_t y_head,
                          void *stream);

/* Token t's key (turned by positions[t]) and value into slot slots[t] = page * page_size + place of the cache; in 8 bits each head's row is
 * rounded as lora_rows_quantize does it, from fp32 (the turned key is not rounded to bf16 first), its scale beside it: d = max(largest magnitude, 448 * 2^-126),
 * scale = d / 448.  A token whose slot is outside the cache, or whose position is negative, is passed over.  Two tokens with the same slot: the slot
 * holds some of either (nothing else is touched).
 * q (NULL: none): the same tokens' queries, turned on the way into y as lora_rotary does it (a token that is passed over leaves its row of y as it is).
 * k, v: device, bf16, 16-byte aligned, [tokens][kv_heads][head_dim], q and y [tokens][q_heads][head_dim], strides as above.  rotary NULL: nothing is
 * turned, positions may be NULL, and q must be.  slots: device, int32, [tokens]. */
lora_status_t lora_cache_append(const void *k, int64_t k_token, int64_t k_head, const void *v, int64_t v_token, int64_t v_head,
                                int32_t tokens, const int32_t *slots, const int32_t *positions, const lora_rotary_t *rotary,
                                const lora_cache_t *cache, const void *q, int64_t q_token, int64_t q_head, int32_t q_heads,
                                void *y, int64_t y_token, int64_t y_head, void *stream);

/* y[t][h] = sum over the keys j that t sees of w_j v_j,  w = softmax of scale q[t][h] . k_j;  key head h / (q_heads / kv_heads).
 * Request r has the rows starts[r] .. starts[r + 1] - 1 of q and y, n of them, and lengths[r] keys in the cache, key j in slot j mod page_size of page
 * page_table[r][j / page_size]; the last n keys are those of its own n rows, the others, its context, were there before.  Row i of a request sees the
 * context and
 *   tree NULL:  its own n keys up to i (a prompt, a piece of one, a single token);
 *   tree:       those of its own keys j for which bit j of tree[starts[r] + i] is set (a drafted token: its ancestors and itself); of a request's
 *               own keys only the first 64 can be seen.
 * A row that sees no key, or only keys whose score is -infinity, is zeros.  Keys that a row does not see have no part in it, whatever their slots hold; an infinity or
 * NaN among the values that it sees makes that dim of y an infinity or NaN, which of them is not said where its weight is too small for 32 bits.
 * Keys on pages outside 0 .. pages - 1 are seen by none; lengths behind page_table's width * page_size count as that; rows of q behind the last request's are
 * left as they are in y.  A request may have no rows, and lengths[r] may be less than n (key j of its own is then key lengths[r] - n + j, where there is one).
 * starts must not descend: the host counts tiles and work groups by that.  Where they do, requests share rows, the call still returns LORA_OK, and any row, also one of a request
 * that shares none, may stay as it was in y or hold, by element, what one of the requests that claim it gives; nothing outside y and the workspace is written.
 *
 * q, y: device, bf16, 16-byte aligned, [tokens][q_heads][head_dim], strides as above, not overlapping; q_heads a multiple of kv_heads.  starts: device, int32,
 * [requests + 1]; lengths: device, int32, [requests]; page_table: device, int32, [requests][width], row stride ld_table; tree: device, 8-byte aligned, [tokens].
 * most: the most rows of a request, as far as the host knows (0: it does not): with it the call chooses its tiles, and more rows are no error.
 * width says the same of keys: width * page_size stands for the longest request, the host knowing no length.  Where there is little to read, a narrower view of the table (width
 * less, ld_table as it is) can save a launch and a join: as wide as needed / 8192 slots and more, one prompt of 600 tokens 25 / 31 us, 4 of 300 to 900 26 / 43, 40 trees of up to 22
 * tokens 10 / 19, 8 single tokens beside a prompt 32 / 47; decode steps, long contexts and large batches are level.  The sums' order may be another then, within the same roundings.
 * workspace: device, 16-byte aligned, of lora_attention_workspace_bytes() or more; its contents are of no account, and calls that may run at the same time need one each.
 * Products are bf16 x bf16 (E4M3 is exact there) with fp32 sums; scores, weights' sum and the running maximum are fp32.  Weights are relative to a maximum that may lag behind the true
 * one by 2^8, and a weight (in 8 bits times its value's scale) is rounded to bf16 for its product with v; in bf16 the weights' sum is of the rounded ones; y is rounded once.
 * Sums are divided at the end, so finite values have to leave them room: 2^8 times the sum of a request's |v| in a dim is less than 2^128, or infinities come of it.  In 8 bits, v's scales
 * below 2^-100 cost the weights bits.
 * scale: finite, and so are its multiple by log2 e and that times any score; a negative one is one of -q.  The same call gives the same bits. */
lora_status_t lora_attention_workspace_bytes(int32_t tokens, int32_t q_heads, int32_t requests, int32_t width, const lora_cache_t *cache,
                                             size_t *bytes);
lora_status_t lora_attention(const void *q, int64_t q_token, int64_t q_head, int32_t tokens, int32_t q_heads, const int32_t *starts,
                             const int32_t *lengths, int32_t requests, const int32_t *page_table, int64_t ld_table, int32_t width,
                             const uint64_t *tree, int32_t most, const lora_cache_t *cache, float scale, void *y, int64_t y_token,
                             int64_t y_head, void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LORA_ATTENTION_GFX950_H */
