/*
 * zo_tree.h -- C ABI of libzo's operators for several new tokens of each sequence at a time, on gfx950:
 * prompts, and drafted answers that one pass of the model verifies.
 *
 * An objective that scores sampled answers draws nearly the same answers for every probe. Drawn with the same
 * random numbers (zo_draw is exact), an earlier answer is a draft of the next one: the model reads
 * all drafted tokens at once, a token is drawn behind each, and the longest beginning that the draws
 * agree with is kept. The answers are those of one token at a time up to rounding: the logits of tokens that are read together
 * come of other sums than those of one token, in the model's products as in the attention, and a draw that this decides is another
 * one. Each token is a draw from the model's own logits behind the tokens before it.
 *
 * Conventions are those of zo_decode.h. The new tokens of all sequences lie packed, one sequence after another:
 * those of sequence s are starts[s] .. starts[s + 1] - 1 of `tokens`, its new token i is starts[s] + i. starts (int32 [seqs + 1])
 * does not fall; entries outside [0, tokens] count as the nearest, and a sequence that would end before it
 * begins has none. Rows in front of the first and behind the last sequence's are left as they were. lengths[s] counts the
 * tokens of sequence s that are in the cache before its new ones (negative: 0); new token i has its place, lengths[s] + i,
 * behind them.
 * The new tokens are a tree: parents[t] is the index, within its sequence, of the token that t comes behind; it is below t's own
 * index. Any other value (-1): t comes behind the cached tokens. parents NULL: a chain, each behind the one before it.
 */
#ifndef ZO_TREE_H_
#define ZO_TREE_H_

#include "zo_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most words of 64 new tokens in zo_tree_lay's masks. */
#define ZO_TREE_WORDS 8u

/*
 * zo_tree_lay -- what the other calls take, from the trees: for new token i of sequence s at row t
 *   seq_of[t] = s, places[t] = lengths[s] + i, positions[t] = lengths[s] + the tokens before it on its branch,
 *   seen[t][w], bit b: whether it sees new token 64 w + b (itself and those before it on its branch).
 * Rows of no sequence get seq_of = positions = places = -1 and see nothing; so do, with their seq_of, new tokens from index
 * 64 words on of a tree, which the masks have no room for (zo_tree_accept takes `words` to know of them). Sums saturate at 2^31 - 1. parents NULL (a chain): words may be 0 and
 * seen NULL; positions are the places, and chains may be of any length (with words > 0: masks as for a tree, with its limit).
 * seen: [tokens, words], contiguous. The outputs do not overlap each other or the inputs.
 * Errors: ZO_ERR_NULL; ZO_ERR_ARG (alignment, words above ZO_TREE_WORDS, 0 words with parents, 2^24 tokens or sequences or more);
 * ZO_ERR_HIP.
 */
typedef struct {
  const int32_t *starts, *lengths, *parents;
  int32_t *seq_of, *positions, *places;
  uint64_t* seen;
  uint32_t tokens, seqs, words;
} zo_tree;

int zo_tree_lay(const zo_tree* t, void* stream);

/*
 * zo_norm_rotate_put_at -- zo_norm_rotate_put whose rows go to token places[token] of their sequence and are turned by
 * positions[token]: tokens of different branches of a tree share positions and not places. A token whose position or
 * place is negative is not put.
 * places: [tokens]; NULL: the positions. Errors: as zo_norm_rotate_put.
 */
int zo_norm_rotate_put_at(const zo_rotate_put* p, const int32_t* places, void* stream);

/*
 * zo_tree_attend -- attention of the new tokens of each sequence, whose keys and values are in the cache at
 * their places. New token i of sequence s (row t of q) and query head h see, of the tokens whose page is present,
 *   j < lengths[s], and the new token at j = lengths[s] + e where bit e % 64 of seen[t][e / 64] is set (e < 64 words) or, with
 *   seen NULL, where e <= i:
 * x_j = scale q . k_j, out = sum_j softmax(x)_j v_j, lse = log sum_j exp x_j, with key head h / (q_heads / cache.heads).
 * Nothing seen: out = 0 and lse = -inf. What a token does not see has no part in its result, whatever it holds. Lengths that
 * pass the table end with it.
 * q and out: [tokens] rows of q_heads heads; lse: float [tokens * q_heads], contiguous, or NULL. q_heads is a multiple of
 * cache.heads. seen: [tokens] rows of `words` words, seen_stride words apart, or NULL (a chain).
 * The work is split evenly over the chip whatever the lengths are, as in zo_cache_attend, and parts are joined by a
 * second launch; lengths and starts, which every workgroup reads, do not change before the call is done. work: device memory of zo_tree_attend_work() bytes, aligned to 16, contents irrelevant, one
 * for each call in flight. Heads of 64, 128 and 256 in pages of whole sixteens of tokens, whose rows begin at multiples of 16 bytes (below
 * 2^28 bytes apart in a page), run on the matrix cores; every other size, page and stride takes a kernel that is several times slower.
 * Arithmetic as in zo_cache_attend. A value that is infinite or NaN reaches the outputs of the tokens that see it and of no other.
 * Errors: ZO_ERR_NULL; ZO_ERR_ARG (dtype, alignment, dim = 0 or above ZO_DIM_MAX, heads, pages or page_tokens 0, heads above 65,535, an out
 * that shares an element with q or lies in the memory that the keys or the values span, too little work, words above 2^20, tokens
 * times q_heads 2^24 or more, sequences times heads 2^23 or more, 2^31 tokens or more in a row of the table); ZO_ERR_NONFINITE
 * (scale); ZO_ERR_HIP.
 */
typedef struct {
  zo_heads q, out;
  zo_cache cache;
  zo_page_table table;
  const int32_t *lengths, *starts;
  const uint64_t* seen;
  int64_t seen_stride;
  float* lse;
  void* work;
  uint64_t work_bytes;
  uint32_t tokens, q_heads, words;
  float scale;
  int32_t dtype;
} zo_tree_attention;

uint64_t zo_tree_attend_work(uint32_t tokens, uint32_t seqs, uint32_t q_heads, uint32_t heads, uint32_t dim, int32_t dtype);
int zo_tree_attend(const zo_tree_attention* a, void* stream);

/*
 * zo_tree_accept -- the walk along the drafted tokens that the draws agree with. drafted[t] is the token of row t, drawn[t] the
 * token drawn behind it. Sequence s walks from its new token 0 (a token that is certain): from the one it is at to the
 * first new token that comes behind it and whose drafted token is the one drawn there; until there is none, or `most` tokens are walked.
 * A negative token (zo_draw's for logits without any weight, or a place of a tree that is not used) agrees with none.
 * words: those given to zo_tree_lay, which gave new tokens from index 64 words on no place: the walk does not come to them. 0: no limit (chains
 * without masks).
 * path[s][i] is the index (within the sequence) of the walk's i-th token, tokens_out[s][i] the token drawn behind it, both
 * -1 behind the walk's end; counts[s] the tokens walked (0 for a sequence without new ones): as many are won, and the last is the
 * next step's token 0. path and tokens_out: [seqs, most], contiguous. The outputs do not overlap each other or the inputs.
 * Errors: ZO_ERR_NULL; ZO_ERR_ARG (alignment, most = 0, words above ZO_TREE_WORDS, 2^24 tokens, sequences or entries of path or more);
 * ZO_ERR_HIP.
 */
typedef struct {
  const int32_t *drafted, *drawn, *starts, *parents;
  int32_t *path, *tokens_out, *counts;
  uint32_t tokens, seqs, most, words;
} zo_tree_walk;

int zo_tree_accept(const zo_tree_walk* w, void* stream);

/*
 * zo_tree_keep -- brings a walked path together: in each of n_tensors tensors (as in zo_cache_copy: the keys and the values of each
 * layer, all of the shape and strides of `shape`; a host array; one that is listed several times moves once) every head's row at token lengths[s] + path[s][i] of sequence
 * s goes to token lengths[s] + i. path (int32, rows path_stride apart) rises along a row and ends with its first negative
 * entry, or the first that does not rise. Rows of an absent page, or behind the table, are neither read nor written. Sequences do not
 * share pages that rows are moved in (ZoPages: extend() gives them pages of their own).
 * Errors: ZO_ERR_NULL; ZO_ERR_ARG (dtype, alignment, heads, pages, page_tokens or dim 0, heads above 65,535, tensors that overlap, 2^17
 * sequences or more); ZO_ERR_MEMORY; ZO_ERR_HIP (earlier tensors may already be enqueued).
 */
typedef struct {
  zo_cache shape;
  void* const* tensors;
  zo_page_table table;
  const int32_t *lengths, *path;
  int64_t path_stride;
  uint32_t n_tensors, most;
  int32_t dtype;
} zo_tree_moves;

int zo_tree_keep(const zo_tree_moves* m, void* stream);

/*
 * zo_pages_cut -- host: the sequence keeps its first `tokens` tokens, and pages that no other holds are free again: what was
 * extended for a draft and not walked goes back to the book.
 * Errors: ZO_ERR_NULL, ZO_ERR_ARG (no such sequence, more tokens than it has).
 */
int zo_pages_cut(zo_pages* book, uint32_t seq, uint32_t tokens);

#ifdef __cplusplus
}
#endif

#endif /* ZO_TREE_H_ */
