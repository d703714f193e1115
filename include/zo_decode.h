/*
 * zo_decode.h -- C ABI of libzo's operators of a decode step on gfx950: from the weights that
 * the sweeps of zo.h train to answers.
 *
 * 1.5-SPSA needs a number for each probe and nothing of how it came about, so the loss may be a
 * score of sampled answers. These calls are what lies between a model's matrix products on
 * that way: norms and rotation of queries and keys, a paged cache of keys and values, the
 * attention of one new token of each sequence over it, and the draw of the token.
 *
 * Conventions for every call, beyond those of zo.h (streams, device, status codes; nothing is
 * enqueued and nothing written where a call returns ZO_ERR_NULL, ZO_ERR_ARG or ZO_ERR_NONFINITE):
 *   - A call takes its arguments in one struct, read during the call. Pointers are device memory
 *     unless said otherwise, strides are in elements, tensors are aligned to their element size
 *     and may be views (any strides; the last dimension contiguous).
 *   - dtype: ZO_F32 or ZO_BF16, the type of every tensor of the call unless said otherwise.
 *     Arithmetic is fp32 (positions' angles and the draw's weights: fp64), rounded once.
 *   - What lies in device memory cannot be checked on the host. The kernels stay inside the
 *     given tensors whatever lengths, positions and page ids hold; each call says what an entry
 *     out of range means.
 *   - Results do not depend on the stream, the device's load or on chance: the same call on the
 *     same inputs gives the same bits.
 *   - The calls record only kernel launches, so they can be captured into a HIP graph; host
 *     arrays (frequencies, page lists) are copied into the launch.
 */
#ifndef ZO_DECODE_H_
#define ZO_DECODE_H_

#include <stdint.h>

#include "zo.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
  ZO_ERR_MEMORY = -5, /* host memory ran out (the page book) */
  ZO_ERR_FULL = -6    /* the page book has no page (or no list entry) left; it is unchanged */
};

/* Largest size of a head. */
#define ZO_DIM_MAX 256u

/* Rows of heads: element (token, head, i) lies at data + token * token_stride + head * head_stride + i. */
typedef struct {
  void* data;
  int64_t token_stride, head_stride;
} zo_heads;

/* The keys and values of one layer in pages of page_tokens tokens: element (page, head, token, i)
 * of the keys lies at k + page * page_stride + head * head_stride + token * token_stride + i, of the
 * values likewise from v. Any order of the page's axes; elements of different pages, heads and
 * tokens do not overlap. */
typedef struct {
  void *k, *v;
  int64_t page_stride, head_stride, token_stride;
  uint32_t pages, heads, page_tokens, dim;
} zo_cache;

/* The pages of each sequence: token j of sequence s lies at row j mod page_tokens of page
 * ids[s * stride + j / page_tokens], j / page_tokens < width. An id outside [0, pages) marks a page
 * that is absent. */
typedef struct {
  const int32_t* ids;
  int64_t stride;
  uint32_t seqs, width;
} zo_page_table;

/*
 * zo_rotary_turns -- host function: the rotation frequencies of a position code, in turns
 * (angle / 2 pi) per position, for zo_rotate.turns: turns[i] = f_i / 2 pi, i < rotary / 2, from
 *   plain (factor = 1):        f_i = base^(-2 i / rotary)
 *   ZO_ROTARY_LINEAR:          f_i / factor (positions pressed together)
 *   ZO_ROTARY_BASE:            base' = base factor^(rotary / (rotary - 2)): the slowest pair turns
 *                              factor times slower, the fastest as before
 *   ZO_ROTARY_BANDS:           pairs that turn often over the original length keep f_i, pairs that
 *                              turn rarely get f_i / factor, between them a blend: with
 *                              r = original f_i / 2 pi turns over the original length,
 *                              f_i (1 - s) / factor + f_i s, s = (r - low) / (high - low) in [0, 1]
 * Arithmetic is IEEE float64. turns: host array of rotary / 2 doubles. original, low and high are
 * used by ZO_ROTARY_BANDS alone.
 * Errors: ZO_ERR_NULL (turns), ZO_ERR_NONFINITE, ZO_ERR_ARG (an unknown kind, rotary odd, below 2
 * or above ZO_DIM_MAX, base <= 1, factor < 1, original <= 0, low < 0, high <= low; rotary = 2 with
 * ZO_ROTARY_BASE).
 */
typedef enum { ZO_ROTARY_LINEAR = 0, ZO_ROTARY_BASE = 1, ZO_ROTARY_BANDS = 2 } zo_rotary_kind;

int zo_rotary_turns(zo_rotary_kind kind, uint32_t rotary, double base, double factor, double original,
                    double low, double high, double* turns);

/*
 * zo_norm_rotate -- norm of each query and key head and rotation by the token's position, one pass.
 * Per row x (one head of one token) of q (q_heads of them) and of k:
 *   norm:      n_i = x_i / sqrt(mean(x^2) + norm_eps) * gamma_i; gamma NULL: n = x
 *   rotation:  of the first `rotary` dims, in pairs (a, b): (i, i + rotary / 2), or with interleaved
 *              (2 i, 2 i + 1), by the angle 2 pi * positions[token] * turns[i]:
 *              a' = magnitude (a cos - b sin), b' = magnitude (a sin + b cos)
 *   dims from `rotary` on keep n. A negative position marks padding: its rows become zeros.
 * q_out and k_out may be q and k themselves (the same data and strides), and otherwise overlap
 * neither. k_heads = 0 (or q_heads = 0): that side is not touched. The angle is reduced in fp64, so
 * that far positions cost no precision. gamma: `dim` elements of the call's dtype. turns: host array
 * of rotary / 2 doubles (zo_rotary_turns or the caller's own); rotary = 0: no rotation.
 * Errors: ZO_ERR_NULL; ZO_ERR_ARG (dtype, alignment, dim = 0 or above ZO_DIM_MAX, rotary odd or
 * above dim, in and out overlapping otherwise, more rows than a launch takes: at least 2^26);
 * ZO_ERR_NONFINITE (norm_eps, magnitude, a frequency); ZO_ERR_HIP.
 */
typedef struct {
  zo_heads q, k, q_out, k_out;
  const void *q_gamma, *k_gamma;
  const int32_t* positions; /* [tokens] */
  const double* turns;      /* host */
  uint32_t tokens, q_heads, k_heads, dim, rotary, interleaved;
  float norm_eps, magnitude;
  int32_t dtype;
} zo_rotate;

int zo_norm_rotate(const zo_rotate* a, void* stream);

/*
 * zo_norm_rotate_put -- zo_norm_rotate whose keys, with the values v, go into the paged cache: row
 * (token, head) of the rotated k and of v is written to token positions[token] of sequence
 * seqs[token] (seqs NULL: token t belongs to sequence t). a.k_out is not used. A token with a
 * negative position, a sequence or position outside the table, or an absent page is not put. Tokens
 * of one call have distinct places. v: a.k_heads heads of the same dim. q_heads = 0 puts alone.
 * Errors: as zo_norm_rotate; ZO_ERR_ARG also where the cache's heads or dim are not the keys', its pages or
 * page_tokens are 0, its keys and values share an element, or q, k, v or q_out lie in the memory that either spans.
 */
typedef struct {
  zo_rotate a;
  zo_heads v;
  zo_cache cache;
  zo_page_table table;
  const int32_t* seqs; /* [tokens] or NULL */
} zo_rotate_put;

int zo_norm_rotate_put(const zo_rotate_put* p, void* stream);

/*
 * zo_norm_rotate_back -- the gradient of zo_norm_rotate. a describes the forward call (a.q and a.k:
 * its inputs; read only where there is a gamma, and may be NULL otherwise); a.q_out and a.k_out hold
 * the gradients of its outputs. Writes dq, dk (which may be the gradients they come from) and, for
 * each gamma, its gradient in fp32, summed over tokens and heads in an order that the sizes alone
 * fix. With d = rotation transposed of the incoming gradient, r = 1 / sqrt(mean(x^2) + eps):
 *   dx = r (d gamma - x r^2 mean(d gamma x)),   dgamma = sum of d x r;   without gamma dx = d.
 * Padding tokens get zeros and add nothing. work: device memory of zo_norm_rotate_back_work()
 * bytes, aligned to 16, contents irrelevant; used where there is a gamma.
 * Errors: as zo_norm_rotate; ZO_ERR_ARG also for too little work, ZO_ERR_NULL for a missing one.
 */
typedef struct {
  zo_rotate a;
  zo_heads dq, dk;
  float *dq_gamma, *dk_gamma; /* [dim], with the gamma */
  void* work;
  uint64_t work_bytes;
} zo_rotate_back;

uint64_t zo_norm_rotate_back_work(uint32_t tokens, uint32_t q_heads, uint32_t k_heads, uint32_t dim);
int zo_norm_rotate_back(const zo_rotate_back* b, void* stream);

/*
 * zo_cache_attend -- attention of one new token of each sequence over its cached tokens.
 * For sequence s and query head h, over the tokens j < lengths[s] whose page is present (key head
 * h / (q_heads / cache.heads)): x_j = scale q . k_j, out = sum_j softmax(x)_j v_j, lse = log sum_j exp x_j.
 * No token left: out = 0 and lse = -inf. Nothing of the cache behind lengths[s] has a part in the
 * result, whatever it holds. A negative length is 0, a length beyond the table ends with it.
 * q and out: [seqs] rows of q_heads heads (zo_heads.token_stride is the stride of sequences); lse:
 * float [seqs * q_heads], contiguous, or NULL. q_heads is a multiple of cache.heads.
 * The work is split evenly over the chip whatever the lengths are, by tiles of tokens, and the parts
 * of a sequence that was split are joined by a second launch. work: device memory of
 * zo_cache_attend_work() bytes, aligned to 16, contents irrelevant, one for each call in flight.
 * Weights are exp2 in fp32; for bf16 each is split in two bf16 parts (16 bits of it) where it meets
 * the values, and sums are fp32. A value that is infinite or NaN reaches the outputs of its own sequence and
 * dim, and makes them what the formula says as long as its weight is above 2^-90 of the largest.
 * Errors: ZO_ERR_NULL; ZO_ERR_ARG (dtype, alignment, dim = 0 or above ZO_DIM_MAX, heads, pages or
 * page_tokens 0, an out that shares an element with q or lies in the memory that the keys or the values span,
 * too little work, 2^24 rows or more); ZO_ERR_NONFINITE (scale); ZO_ERR_HIP.
 */
typedef struct {
  zo_heads q, out;
  zo_cache cache;
  zo_page_table table;
  const int32_t* lengths; /* [seqs] */
  float* lse;
  void* work;
  uint64_t work_bytes;
  uint32_t q_heads;
  float scale;
  int32_t dtype;
} zo_attend;

uint64_t zo_cache_attend_work(uint32_t seqs, uint32_t q_heads, uint32_t heads, uint32_t dim);
int zo_cache_attend(const zo_attend* a, void* stream);

/*
 * zo_cache_copy -- copies tokens 0 .. rows - 1 of page src to page dst, every head, for each of n_moves
 * moves in each of n_tensors tensors: the keys and the values of each layer of a model, all of the shape
 * and strides of `shape` (whose k and v are not used). tensors (device addresses) and moves are host
 * arrays. All moves read what the pages held before the call: no dst is repeated or is the src of a
 * move.
 * Errors: ZO_ERR_NULL, ZO_ERR_ARG (dtype, alignment, a page or rows out of range, rows = 0, a
 * repeated dst, a dst that is a src, pages that overlap, two different tensors that do, pages of more than 2^23
 * elements), ZO_ERR_MEMORY,
 * ZO_ERR_HIP (earlier batches may already be enqueued).
 */
typedef struct {
  int32_t src, dst, rows;
} zo_page_move;

int zo_cache_copy(const zo_cache* shape, void* const* tensors, uint32_t n_tensors, const zo_page_move* moves,
                  uint32_t n_moves, zo_dtype dtype, void* stream);

/*
 * zo_draw -- draws a token for each row of logits from given random numbers.
 * Row b, logits l_i, i < vocab (NaN counts as -inf, +inf as the largest finite number of its type):
 * with m = max l_i the weight of token i is the whole number
 *   w_i = round(2^44 exp((l_i - m) / temperature[b])).
 * In the order of falling logits, ties by index, kept are: the first top_k[b] tokens (all if <= 0); of
 * these the fewest first ones that hold floor(W P / 2^24) of their weight W, P = round(2^24 top_p[b])
 * (at least one; all if top_p >= 1); of these those with w_i >= round(2^44 min(min_p[b], 1)). The token
 * is the lowest index i at which the kept weight of tokens 0 .. i exceeds floor(W' U / 2^24), W' the kept
 * weight, U = floor(2^24 u[b]) clipped to [0, 2^24). Every sum is of whole numbers, so the token is
 * exact. temperature <= 0 (or NaN) takes the lowest index of the largest logit (logprob 0). A row
 * without any weight (all -inf) gives token -1 and logprob -inf.
 * temperature, top_k, top_p and min_p: device arrays [rows] or NULL (1, all, all, all). u: float
 * [rows]. tokens: int32 [rows]; logprobs: float [rows] or NULL, log(w_token / W').
 * Errors: ZO_ERR_NULL, ZO_ERR_ARG (dtype, alignment, vocab = 0 or above 2^18, 2^22 rows or more), ZO_ERR_HIP.
 */
typedef struct {
  const void* logits; /* [rows, vocab], rows row_stride elements apart */
  int64_t row_stride;
  const float *u, *temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int32_t* tokens;
  float* logprobs;
  uint32_t rows, vocab;
  int32_t dtype;
} zo_draw_args;

int zo_draw(const zo_draw_args* a, void* stream);

/*
 * zo_draw_split -- zo_draw, its rows split over workgroups where they are few and long: the same
 * tokens sooner. work: zo_draw_work() bytes (top_k: whether the call has any), aligned to 16, contents irrelevant,
 * one for each call in flight; with 0 bytes (many or short rows) work is not used and the call is zo_draw.
 * Errors: as zo_draw; ZO_ERR_ARG, ZO_ERR_NULL for the workspace.
 */
int zo_draw_split(const zo_draw_args* a, void* work, uint64_t work_bytes, void* stream);
uint64_t zo_draw_work(uint32_t rows, uint32_t vocab, int top_k);

/*
 * The page book -- host bookkeeping of a cache's pages: which pages each sequence holds, which are
 * shared, which are free. It holds no device memory and never touches the GPU; what has to be copied
 * on the device it hands out as moves for zo_cache_copy (of every layer, before the next put). A book
 * is used from one thread at a time. Sequences are numbered from 0; numbers of dropped ones are
 * given again.
 *
 * zo_pages_open     a book of `pages` free pages of page_tokens tokens; NULL if out of memory or 0.
 * zo_pages_add      a new sequence of `tokens` tokens.
 * zo_pages_fork     a new sequence with the tokens of seq, sharing its pages.
 * zo_pages_extend   room for `tokens` more tokens. If they start in a page that others share, the
 *                   sequence gets a page of its own for it and *move says what to copy (rows = 0: nothing).
 * zo_pages_drop     ends a sequence; pages that no other holds are free again.
 * zo_pages_left     how many pages are free.
 * zo_pages_length   the tokens of a sequence, or -1.
 * zo_pages_table    writes the pages of n sequences to rows of `width` ids, `stride` apart (-1 behind
 *                   the last), and their lengths; either output may be NULL.
 * zo_pages_compact  moves the pages in use to the lowest ids: at most `room` moves are written to
 *                   `moves` and carried out in the book (*n of them; all that are needed if room >=
 *                   the pages in use). Their sources and destinations are distinct.
 * Errors: ZO_ERR_NULL, ZO_ERR_ARG (no such sequence, a table too narrow, tokens out of range),
 * ZO_ERR_FULL, ZO_ERR_MEMORY; a call that fails leaves the book as it was.
 */
typedef struct zo_pages zo_pages;

zo_pages* zo_pages_open(uint32_t pages, uint32_t page_tokens);
void zo_pages_close(zo_pages* book);
int zo_pages_add(zo_pages* book, uint32_t tokens, uint32_t* seq);
int zo_pages_fork(zo_pages* book, uint32_t seq, uint32_t* forked);
int zo_pages_extend(zo_pages* book, uint32_t seq, uint32_t tokens, zo_page_move* move);
int zo_pages_drop(zo_pages* book, uint32_t seq);
uint32_t zo_pages_left(const zo_pages* book);
int64_t zo_pages_length(const zo_pages* book, uint32_t seq);
int zo_pages_table(const zo_pages* book, const uint32_t* seqs, uint32_t n, int32_t* ids, uint64_t stride,
                   uint32_t width, int32_t* lengths);
int zo_pages_compact(zo_pages* book, zo_page_move* moves, uint32_t room, uint32_t* n);

#ifdef __cplusplus
}
#endif

#endif /* ZO_DECODE_H_ */
