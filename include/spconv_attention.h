/*
 * spconv_attention.h - attention over listed blocks of a paged cache on MI355X
 * (gfx950). C ABI of libspconv.so beside spconv.h.
 *
 * What the CSR filter is to the convolution of spconv.h, a list of key blocks is
 * to attention here: a row (neighbouring query tokens of one key/value head)
 * names the blocks that it reads, a table lowers each block to where its keys
 * lie, and what a row does not name is never touched. The calls, in the order in
 * which one step of a sequence model makes them:
 *   spconv_rope             rotates the queries by their positions,
 *   spconv_cache_append     rotates the new keys, stores keys and values in the
 *                           cache and keeps the sum of every block's keys,
 *   spconv_block_scores     scores the blocks for each row by those sums,
 *   spconv_select_blocks    lists each row's best blocks,
 *   spconv_block_attention  softmax attention over the listed blocks.
 *
 * Status codes, ownership and ordering are those of spconv.h: every call returns
 * SPCONV_OK or a negative code and never throws, arguments are checked on the
 * host before any GPU work is queued, the caller owns every buffer (workspace
 * included), device calls are asynchronous on `stream`, which belongs to the
 * current device, and may be captured into a graph. The library keeps no state.
 *
 * Element types (dtype): keys, values, queries and outputs of one call have the
 * same type. Dot products, softmax statistics, sums, scores and partial outputs
 * are fp32, angles fp64 (their sines and cosines fp32); a value is rounded to its
 * type once, when it is stored. fp16 and bf16 attention rounds the softmax weights
 * to the type as well, for the matrix cores: half a step of the type for each
 * weight, on top of the output's own.
 */
#ifndef SPCONV_ATTENTION_H
#define SPCONV_ATTENTION_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "spconv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPCONV_F32 0
#define SPCONV_F16 1
#define SPCONV_BF16 2

/* Flags of spconv_rope and spconv_cache_append. Any other bit is SPCONV_EINVAL. */
#define SPCONV_ROPE_INTERLEAVED 1u /* pairs (2i, 2i+1); without it pairs (i, i + rot/2) */
#define SPCONV_ROPE_INVERSE 2u     /* angle -> -angle: the gradient with the same amplitude, undoes the rotation with 1 / amplitude (spconv_rope only) */

/*
 * The sequences of a step: where their tokens, keys and rows are.
 *
 * Tokens are packed: sequence b has tokens [q_start[b], q_start[b+1]) of the
 * call's `tokens`, the newest of its kv_len[b] keys, so its i-th token stands at
 * position p = kv_len[b] - (q_start[b+1] - q_start[b]) + i and sees the keys
 * 0 .. p. Without q_start every sequence has one token, token b, as with
 * q_start[b] = b (generation; then tokens must equal sequences).
 *
 * Keys lie in pages of `block` keys: key j of sequence b is slot j % block of
 * page table[b*table_stride + j/block].
 *
 * Rows group q_block neighbouring tokens of a sequence, which share a block
 * list. There are R = tokens rows with q_block 1 (row = token), otherwise
 * R = tokens/q_block + sequences (floor): tokens i*q_block .. of sequence b are row
 * q_start[b]/q_block + b + i. Some rows have no tokens.
 *
 * Tokens outside [q_start[0], q_start[sequences]) belong to no sequence: nothing
 * is computed or written for them. The device arrays are not checked by the host;
 * the kernels keep every access inside the buffers whatever they hold: q_start is
 * taken into [0, tokens], kv_len into [0, max_blocks*block], tokens at negative
 * positions see nothing, and a page outside [0, pages) counts as not there (its
 * keys are seen by nobody, and a token to be stored there is dropped).
 */
typedef struct spconv_batch {
    int32_t sequences;     /* >= 1 */
    int32_t block;         /* keys per page: a multiple of 16, 16 to 256 */
    int32_t max_blocks;    /* columns of the table, >= 1; max_blocks * block < 2^31 */
    int32_t q_block;       /* tokens per row, 1 to 128 */
    int64_t tokens;        /* 1 to 2^31 - 1 */
    int64_t pages;         /* pages of the cache, 1 to 2^31 - 1 */
    int64_t table_stride;  /* >= max_blocks */
    const int32_t *table;  /* device [sequences][table_stride]; may be shared or reordered pages */
    const int32_t *kv_len; /* device [sequences] */
    const int32_t *q_start; /* device [sequences + 1], non-decreasing, nullable */
} spconv_batch;

/*
 * spconv_batch_rows - R, the rows of a batch (host only). Errors: SPCONV_EINVAL for
 * NULL arguments or a batch out of the ranges above (its arrays are not looked at).
 */
int spconv_batch_rows(const spconv_batch *batch, int64_t *rows);

/* Scalings of the rotary frequencies for contexts longer than a model was trained on. */
#define SPCONV_ROPE_PLAIN 0
#define SPCONV_ROPE_LINEAR 1   /* f / factor: positions are squeezed */
#define SPCONV_ROPE_BASE 2     /* base * factor^(rot/(rot-2)): the slowest pair turns factor times slower, the fastest as before */
#define SPCONV_ROPE_BY_PARTS 3 /* by wavelength w = 2 pi / f: f where w < original / high, f / factor where
                                * w > original / low, between them (1-t) f / factor + t f with
                                * t = (original / w - low) / (high - low) */
typedef struct spconv_rope_scaling {
    int32_t kind;
    double factor;   /* >= 1, not used by SPCONV_ROPE_PLAIN */
    double low, high, original; /* SPCONV_ROPE_BY_PARTS: 0 < low < high, original > 0 */
} spconv_rope_scaling;

/*
 * spconv_rope_frequencies - the angle per position of each pair (host):
 *   freq[i] = base^(-2i/rot), i = 0 .. rot/2 - 1, scaled as scaling says (nullable: plain).
 * freq  host array of rot/2 doubles; spconv_rope and spconv_cache_append take a device copy.
 * Errors: SPCONV_EINVAL for a NULL freq, rot < 2 or odd, a base that is not above 0 or not
 * finite, a bad scaling (SPCONV_ROPE_BASE needs rot > 2).
 */
int spconv_rope_frequencies(int rot, double base, const spconv_rope_scaling *scaling, double *freq);

/*
 * spconv_rope - rotary positions (device, asynchronous).
 * For pair i of the first rot components of every head, with angle = positions[t] * freq[i]
 * (rounded to fp64; negated with SPCONV_ROPE_INVERSE), c = cos(angle), s = sin(angle), both fp32, within 2^-22.6:
 *   out1 = amplitude * (x1 c - x2 s),  out2 = amplitude * (x2 c + x1 s);
 * components from rot on are copied.
 * x, out     device; token t, head h, component d at t*token_stride + h*head_stride + d
 *            (elements). out may be x itself with x's strides (in place); otherwise they must
 *            not overlap, nor any two rows of out (strides below dim are refused). Moved by the widest vectors,
 *            16 bytes to one element, that dim, rot, pointers and strides fit.
 * positions  device int32 [tokens], any value.   freq  device fp64 [rot/2].
 * dim        1 to 1024; rot even, 0 to dim (freq may be NULL with rot 0).
 * Errors: SPCONV_EINVAL (NULL pointer, unknown dtype or flags, tokens outside [1, 2^31-1],
 * heads outside [1, 65535], dim or rot out of range, a negative stride, a stride of out below dim, an amplitude that is
 * not finite, x == out with other strides); SPCONV_EHIP when the launch fails.
 */
int spconv_rope(int dtype, const void *x, int64_t x_token, int64_t x_head, int64_t tokens, int heads, int dim,
                const int32_t *positions, const double *freq, int rot, uint32_t flags, float amplitude, void *out,
                int64_t out_token, int64_t out_head, hipStream_t stream);

/*
 * spconv_cache_append - store a step's keys and values in the paged cache (device,
 * asynchronous). Token at position p of sequence b goes to slot p % block of page
 * table[b][p / block]; kv_len counts the new keys. Keys are rotated on the way as by
 * spconv_rope with that position (or positions[t], if given), then rounded. With sums,
 * the sum of each page that got a key is set to that of all keys the page now holds of the
 * sequence (slots 0 up to the newest), read back as stored: appending again from an
 * earlier position, after drafted tokens were dropped, leaves no trace of them.
 * A page that gets keys must belong to one sequence of the batch (pages that are only
 * read may be shared); the slots of two sequences in one page are otherwise stored in an unspecified order.
 * k, v       device, [tokens][heads][dim] by strides as in spconv_rope. Moved by 16-byte vectors where dim, rot and
 *            both tensors' pointers and strides fit, otherwise one by one.
 * k_cache, v_cache  device [pages][heads][block][dim], 16-byte aligned.
 * sums       device fp32 [pages][heads][dim], 16-byte aligned, nullable. None of the outputs may overlap the inputs.
 * positions  device int32 [tokens], nullable.  freq  device fp64 [rot/2], nullable (no rotation; rot must be 0).
 * flags, amplitude  as spconv_rope, without SPCONV_ROPE_INVERSE.
 * heads      1 to 65535.   dim  a multiple of 8, 8 to 256.   batch->q_block is not used.
 * Errors: SPCONV_EINVAL as above, and for (tokens/block + 2*sequences)*heads >= 2^31; SPCONV_EHIP when the launch fails.
 */
int spconv_cache_append(int dtype, const spconv_batch *batch, const void *k, int64_t k_token, int64_t k_head,
                        const void *v, int64_t v_token, int64_t v_head, int heads, int dim, const int32_t *positions,
                        const double *freq, int rot, uint32_t flags, float amplitude, void *k_cache, void *v_cache,
                        float *sums, hipStream_t stream);

/*
 * spconv_block_scores - score of every block for every row (device, asynchronous):
 *   scores[r][h][j] = max over the row's tokens at positions p >= j*block, and over the q_heads/heads
 *                     query heads of key head h, of q . sums[page] / n
 * with page = table[b][j] and n = min(block, kv_len[b] - j*block) the keys that the block holds: the
 * best product of a query with the mean key. Products that are NaN do not count; blocks that no
 * token of the row sees, blocks without a page and rows without tokens get -infinity.
 * q        device, [tokens][q_heads][dim] by strides; query head g belongs to key head g / (q_heads/heads).
 * sums     device fp32 [pages][heads][dim], 16-byte aligned, as spconv_cache_append keeps them.
 * scores   device fp32 [R][heads][max_blocks]; every element is written, must not overlap the inputs.
 * Errors: SPCONV_EINVAL (NULL pointer, bad batch, unknown dtype, q_heads not a multiple of heads or
 * above 65535, dim not a multiple of 8 in [8, 256], R*heads*ceil(max_blocks/n) >= 2^31 with n = 64 for rows of 16
 * (token, query head) pairs or less and 256 for others, a negative stride); SPCONV_EHIP.
 */
int spconv_block_scores(int dtype, const spconv_batch *batch, const void *q, int64_t q_token, int64_t q_head,
                        int q_heads, int heads, int dim, const float *sums, float *scores, hipStream_t stream);

/*
 * spconv_select_blocks - the blocks that each row reads (device, asynchronous).
 * A row whose first and last tokens stand at p0 and p1 sees n = p1/block + 1 blocks. If n <= keep all are
 * listed. Otherwise keep of them: the first `sink`, those from p0/block - local + 1 on (none of these with
 * local 0), and, of the others, those of the highest score; equal scores go to the lower index, +0 equals
 * -0, NaN counts as -infinity.
 * scores   device fp32 [R][heads][max_blocks]; only visible blocks' are read.
 * blocks   device int32 [R][heads][keep]: the list, ascending, then -1.
 * counts   device int32 [R][heads]: blocks listed, 0 for a row without tokens.
 * Errors: SPCONV_EINVAL (NULL pointer, bad batch, heads outside [1, 65535], keep < 1, negative sink or local,
 * keep < sink + local + ceil((q_block-1)/block), which could not hold what is always listed, R*heads*keep >= 2^40
 * or R*heads >= 2^31); SPCONV_EHIP.
 */
int spconv_select_blocks(const spconv_batch *batch, int heads, const float *scores, int keep, int sink, int local,
                         int32_t *blocks, int32_t *counts, hipStream_t stream);

/*
 * spconv_attention_workspace - bytes of device scratch memory that spconv_block_attention needs for these
 * sizes (host only; 0 if none). keep = 0: without lists. Errors: as spconv_block_attention.
 */
int spconv_attention_workspace(int dtype, const spconv_batch *batch, int q_heads, int heads, int dim, int keep,
                               int64_t *bytes);

/*
 * spconv_block_attention - causal softmax attention over listed blocks (device, asynchronous).
 * For each token (at position p, in row r) and query head g of key head h:
 *   S = keys of the blocks listed in row r of head h, at positions <= p
 *   out = sum over S of w_j v_j,  w_j = exp(scale * q.k_j) / sum over S of exp(scale * q.k_i)
 *   lse = log of that sum
 * A token that sees no key gets out = 0 and lse = -infinity (one whose every scale * q.k is -infinity as well).
 * Keys that a token does not see take no part whatever they hold (infinities and NaN among it). Infinities and NaN of
 * keys that it sees come out by the formula, except that an infinite value whose weight is rounded to 0 (by less
 * than 2^-25 of the largest in fp16, 2^-126 in the others) may give NaN.
 * blocks   device int32 [R][heads][keep], any order; entries outside [0, max_blocks) and blocks without a page
 *          are passed over, a block that is listed twice counts twice. NULL (with keep 0 and counts NULL): every
 *          visible block (what batch->q_block says is then of no matter).
 * counts   device int32 [R][heads], nullable (then all keep entries are looked at); taken into [0, keep].
 * k_cache, v_cache  device [pages][heads][block][dim], 16-byte aligned.
 * out      device, [tokens][q_heads][dim] by strides, must not overlap the inputs, nor its rows each other (strides
 *          below dim are refused).
 * lse      device fp32 [tokens][q_heads], nullable.
 * workspace  device, 16-byte aligned, at least spconv_attention_workspace bytes (nullable if that is 0); its
 *          contents do not matter. Calls that may run at the same time (other streams, graphs that hold the
 *          call) need workspaces of their own.
 * Results are reproducible run to run for a given device and sizes.
 * Errors: SPCONV_EINVAL (NULL pointer, bad batch, unknown dtype, q_heads not a multiple of heads or above 65535,
 * dim not a multiple of 8 in [8, 256], a negative stride, a scale whose product with log2(e) is not finite, keep < 0,
 * blocks without keep or keep without blocks, counts without blocks, out == q, 2^27 tiles or more of 16 to 256 (token, head) pairs of a row, a workspace
 * that is too small or misaligned); SPCONV_EHIP.
 */
int spconv_block_attention(int dtype, const spconv_batch *batch, const void *q, int64_t q_token, int64_t q_head,
                           int q_heads, int heads, int dim, const void *k_cache, const void *v_cache, float scale,
                           const int32_t *blocks, const int32_t *counts, int keep, void *out, int64_t out_token,
                           int64_t out_head, float *lse, void *workspace, int64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SPCONV_ATTENTION_H */
