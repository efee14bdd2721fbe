/*
 * switchsd_target.h -- operators on the target model's side of a verification step, on one GB300 (sm_103a).
 *
 * The controller (switchsd.h) leaves lengths, drafts and accepted tokens in device memory.  The target model's
 * forward pass over a draft needs three things that depend on them, and one that turns its logits into the tokens
 * that the controller verifies:
 *
 *   switchsd_kv_map         pages for the new tokens: block tables and slot maps built from the device lengths;
 *   switchsd_kv4_append     the new tokens' keys and values into a paged cache held in 4 bits;
 *   switchsd_kv4_attention  attention of the new tokens (one, or a draft and its root) over that cache;
 *   switchsd_logits         penalties for repeated tokens, biases and grammar masks on the logits, and every
 *                           position's greedy token: the target_argmax of switchsd_verify;
 *   switchsd_kv4_read       the values that the cache holds for some tokens.
 *
 * The conventions of switchsd.h hold: caller-owned device pointers, asynchronous on `stream`, host codes before
 * anything is enqueued, per-row device status, capture into CUDA graphs, no allocation.
 *
 * Lengths.  `lens[b] + lens_add` is the number of tokens that row b's cache holds before the step, and
 * `new_lens[b] + new_add` (0 .. T) the number of its new tokens, which take the positions from there on.  With a
 * controller's context x[0 .. L-1], whose last token the target has not seen, and a draft of vlen tokens, the step's
 * tokens are x[L-1] and the draft: lens = ctx_lens with lens_add = -1, new_lens = vlen with new_add = 1, T = k + 1.
 */
#ifndef SWITCHSD_TARGET_H_
#define SWITCHSD_TARGET_H_

#include "switchsd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define SWITCHSD_BF16 0
#define SWITCHSD_F16 1
#define SWITCHSD_F32 2

#define SWITCHSD_MAP_ROWS 8192  /* largest B of switchsd_kv_map */
#define SWITCHSD_VMAX 262144    /* largest vocabulary of switchsd_logits */
#define SWITCHSD_BIAS_MAX 4096  /* largest number of biases a row */

/*
 * Block tables and slot maps.  A pool of `pages` pages of `page` tokens (16, 32, 64, 128 or 256) serves B rows.
 * Row b holds held[b] pages, block_table[b][0 .. held[b]); the pages that no row holds are a stack,
 * free_list[0 .. free_count).  One call brings every row to the ceil((len + new) / page) pages that its lengths ask for:
 *
 *   1. rows that hold more give pages back: in order of rows, and in a row in order of the table, each pushed on the
 *      stack;
 *   2. rows that hold fewer take pages off the stack's top in order of rows, and in a row in order of the table;
 *   3. new token t of row b gets the slot block_table[b][p / page] * page + p % page of its position p = len + t.
 *
 * A row that the stack is too short for, counting what all rows before it asked for, or that asks for more than
 * `blocks` pages keeps what it holds: its status is SWITCHSD_ROW_CAPACITY.  A row with a negative length, with new
 * tokens outside [0, T] or with held[b] outside [0, blocks] is left alone with SWITCHSD_ROW_BAD_LEN.  Both get no
 * slots.
 *
 * Such a row has no place for its new tokens, so the step has to leave it out altogether: switchsd_kv_map_granted also
 * writes granted[b] = new_lens[b] for the other rows and -1 - new_add for these.  Given as new_lens to the attention and
 * the logits, and as draft_len to the verification (with new_add >= 0), it is a bad length there: the row gets zeros, no
 * greedy token, and a context that stays as it is, until a later map has pages for it.
 *
 *   lens, new_lens  int32 [B];  lens_add, new_add  see above
 *   block_table     int32 [B, blocks] (modified; entries that no page backs are -1 after the call that freed them)
 *   held            int32 [B] (modified)
 *   free_list       int32 [pages] (modified; entries taken become -1);  free_count  int32 [1] (modified)
 *   slots           int32 [B, T] or NULL: out, -1 for t >= new and for rows without slots
 *   status          int32 [B] or NULL: out
 *   granted         int32 [B] or NULL: out; may be new_lens itself
 *   B 1 .. SWITCHSD_MAP_ROWS, T >= 1, blocks >= 1, pages >= 1, pages * page <= 2^31 - 1, B * T and B * blocks < 2^31
 */
typedef struct {
    int32_t B, T, page, blocks, pages;
    const int32_t *lens, *new_lens;
    int32_t lens_add, new_add;
    int32_t *block_table, *held, *free_list, *free_count;
    int32_t *slots;
    int32_t *status;
    void *stream;
} switchsd_kv_map_params;

int switchsd_kv_map(const switchsd_kv_map_params *params);
int switchsd_kv_map_granted(const switchsd_kv_map_params *params, int32_t *granted);

/*
 * The 4-bit cache of one layer: uint8 [pages][Hkv][switchsd_kv4_bytes(page, D)], 16-byte aligned, D = 64 or 128.  With
 * G = D / 64 groups of 64 dimensions, a (page, head) holds
 *
 *   key codes    [page][D / 8] 32-bit words: word c * 2G + 2g + i (c < 4, g < G, i < 2) has the token's dimensions
 *                64 g + 16 c + 8 i + 0 .. 7
 *   value codes  [page / 8][D] 32-bit words: the word of a dimension has eight consecutive tokens
 *   scales       [page][2 G] f16: the G of the token's key, then the G of its value
 *
 * and element j = 2 p + e of a word (p < 4, e < 2) is its bits 4 (p + 4 e) .. + 3: a code c that stands for
 * (c - 8) * scale.  Both the scale's 7 significant bits and the code are chosen so that this product is an f16 number.
 */
size_t switchsd_kv4_bytes(int32_t page, int32_t D);

/*
 * Append: the new tokens' keys and values into the cache.  A group of 64 values x of a token gets the scale
 * max(max x / 7, max -x / 8), computed in binary32, rounded up to 7 significant bits, at most 8128, rounded to f16; and
 * the codes clamp(round(x / scale), -8, 7) + 8, rounding half to even (8 where the scale is 0).  A NaN in a group makes
 * the group's scale NaN; values beyond what the largest scale reaches saturate.
 *
 *   k, v        dtype (SWITCHSD_BF16 or SWITCHSD_F16) [B, T, Hkv, D], strides in elements between rows, tokens and
 *               heads (multiples of 8, but for a dimension of one; a head's values are contiguous), 16-byte aligned
 *   slots       int32 [B, T]: as switchsd_kv_map writes them -- a row's slots are consecutive inside a page and begin
 *               a page at its first slot, and -1 past the row's new tokens.  Slots outside [0, pages * page) are
 *               skipped.
 *   B * T < 2^31, B * (T / 8 + 2) * Hkv < 2^30 (here and for the read)
 * Calls that write into one page must not overlap on the GPU (eight tokens share a word).
 */
typedef struct {
    int32_t B, T, Hkv, D, page, pages, dtype;
    const void *k, *v;
    int64_t k_stride[3], v_stride[3];
    const int32_t *slots;
    void *cache;
    void *stream;
} switchsd_kv4_append_params;

int switchsd_kv4_append(const switchsd_kv4_append_params *params);

/*
 * Read: what the cache holds for given slots, as f16 (exactly): out_k, out_v [B, T, Hkv, D], 16-byte aligned; zeros for
 * slots outside [0, pages * page).
 */
typedef struct {
    int32_t B, T, Hkv, D, page, pages;
    const void *cache;
    const int32_t *slots;
    void *out_k, *out_v;
    void *stream;
} switchsd_kv4_read_params;

int switchsd_kv4_read(const switchsd_kv4_read_params *params);

/*
 * Attention over the 4-bit cache.  New token t of row b (t < new) stands at position len + t and sees the keys of the
 * positions 0 .. len + t, its own among them (append first; a row that the map left without slots is left out here by
 * switchsd_kv_map_granted's lengths, or it would see what earlier steps left behind its last token):
 *
 *   out[b, t, h] = sum_j softmax_j(scale * q[b, t, h] . k_j) v_j,   k, v of the key head h / (Hq / Hkv)
 *
 * Tokens t >= new, rows with bad lengths (negative, new outside [0, T], len + new > blocks * page: status
 * SWITCHSD_ROW_BAD_LEN) and tokens that see nothing get zeros.  The tokens of a page whose table entry lies outside
 * [0, pages) are not seen.  What the cache holds in places that a token does not see never reaches its result, NaN
 * among it; a NaN that it does see makes its result NaN, in the value's 64 dimensions or, where a call has many query
 * rows, in all of the head's.  Scores, the softmax's maximum and sum and the output's sum are held in binary32; the
 * weights that multiply the values are rounded to 11 bits.  The elements of a query that lie 2^22 and more below its own
 * largest may lose bits; magnitudes from 2^116 on, which only bf16 has, count as infinite.
 *
 *   q             dtype (SWITCHSD_BF16 or SWITCHSD_F16) [B, T, Hq, D], strides in elements between rows, tokens and
 *                 heads (multiples of 8, but for a dimension of one; a head's values are contiguous), 16-byte aligned
 *   out           dtype [B, T, Hq, D] contiguous, 16-byte aligned
 *   Hq            a multiple of Hkv, at most 64 times it
 *   block_table   int32 [B, blocks]
 *   workspace     at least switchsd_kv4_attention_workspace_bytes(params) bytes, 16-byte aligned, caller-owned: partial
 *                 results between the call's two kernels.  Calls that share one must not overlap on the GPU.
 *   status        int32 [B] or NULL.  SWITCHSD_ROW_TIMEOUT in all rows: an on-chip wait ran out, and what the call wrote
 *                 does not count.
 */
typedef struct {
    int32_t B, T, Hq, Hkv, D, page, pages, blocks, dtype;
    const void *q;
    int64_t q_stride[3];
    const void *cache;
    const int32_t *block_table, *lens, *new_lens;
    int32_t lens_add, new_add;
    float scale;
    void *out;
    void *workspace;
    size_t workspace_bytes;
    int32_t *status;
    void *stream;
} switchsd_kv4_attention_params;

size_t switchsd_kv4_attention_workspace_bytes(const switchsd_kv4_attention_params *params);
int switchsd_kv4_attention(const switchsd_kv4_attention_params *params);

/*
 * Logits of B rows and T positions.  Position t of row b (t < new) follows the row's context x[0 .. L-1] and the
 * draft's first t tokens.  With n_v the number of times that token v occurs there, m_v the same without the context's
 * first prompt_lens[b] tokens, and every operation rounded to binary32,
 *
 *   n_v > 0:  l = l > 0 ? l / rep : l * rep
 *   m_v > 0:  l = (l - freq * m_v) - pres
 *   l = l + bias_v                                 (the last entry of bias_ids that names v)
 *   l = -inf where the position's mask has a 0 bit
 *
 * argmax is the smallest v with the largest l; l = -inf and NaN are never chosen, and it is -1 where nothing is.  (The
 * verification appends the token that it is given: a grammar that leaves a position nothing is the caller's to see to.)
 *
 *   logits        dtype (SWITCHSD_BF16, SWITCHSD_F16, SWITCHSD_F32) [B, T, V], strides in elements between rows and
 *                 positions (V values are contiguous), aligned to its elements
 *   ctx_tokens    int32 [B, cap] (16-byte aligned, cap a multiple of 4 below 2^28), ctx_lens int32 [B]; NULL (both): no context
 *   draft         int32 [B, draft_stride]: entries 0 .. new - 2 are read; NULL for T = 1 or to leave the draft out
 *   new_lens      int32 [B] or NULL: positions of each row, T when NULL.  new_add is added.
 *   rep, freq, pres  float [B] or NULL (1, 0, 0); rep > 0
 *   prompt_lens   int32 [B] or NULL (0)
 *   bias_ids, bias   int32, float [B, nbias], or NULL; ids outside [0, V) are skipped
 *   mask          int32 [B, T, mask_words], mask_words >= ceil(V / 32), or NULL; bit v % 32 of word v / 32
 *   out           dtype [B, T, V] with its own strides, or NULL; may be `logits` itself (with its strides); positions
 *                 t >= new are not written
 *   argmax        int32 [B, T] or NULL (not both); -1 for t >= new
 *   workspace     at least switchsd_logits_workspace_bytes(params) bytes, 16-byte aligned, caller-owned: the tokens that
 *                 penalties and biases name, and the positions' best so far.  Calls that share one must not overlap on
 *                 the GPU.  (The size goes by B, T, V, cap, nbias and which of the inputs are given.)
 *   status        int32 [B] or NULL: SWITCHSD_ROW_BAD_LEN for a context length outside [0, cap] or new outside [0, T]
 *                 (the row is left out: argmax -1)
 * Tokens of the context and the draft outside [0, V) count for nothing.  B 1 .. 65535, T 1 .. 262140, V 1 .. SWITCHSD_VMAX,
 * nbias up to SWITCHSD_BIAS_MAX.
 */
typedef struct {
    int32_t B, T, V, cap, dtype;
    const void *logits;
    int64_t stride_b, stride_t;
    const int32_t *ctx_tokens, *ctx_lens;
    const int32_t *draft;
    int32_t draft_stride;
    const int32_t *new_lens;
    int32_t new_add;
    const float *rep, *freq, *pres;
    const int32_t *prompt_lens;
    const int32_t *bias_ids;
    const float *bias;
    int32_t nbias;
    const int32_t *mask;
    int32_t mask_words;
    void *out;
    int64_t out_stride_b, out_stride_t;
    int32_t *argmax;
    int32_t *status;
    void *workspace;
    size_t workspace_bytes;
    void *stream;
} switchsd_logits_params;

size_t switchsd_logits_workspace_bytes(const switchsd_logits_params *params);
int switchsd_logits(const switchsd_logits_params *params);

#ifdef __cplusplus
}
#endif

#endif /* SWITCHSD_TARGET_H_ */
