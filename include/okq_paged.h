/*
 * okq_paged - an 8-bit KV cache in pages, next to the 2-bit cache of okq.h: rotary positions with three axes, alone or behind a norm of
 * every head, append, attention for prompts and single tokens, with a window, and for trees of drafted tokens, and the pages' bookkeeping.  Plain C ABI with the conventions of okq.h: every tensor
 * argument is a DEVICE pointer owned by the caller and aligned to 16 bytes; structs, `strides` and `sections` are HOST memory,
 * read before the call returns; calls are asynchronous on `stream` and allocate nothing; errors that the host can see are returned
 * before anything is launched, errors only the device can see go to the cache's sticky status word.
 *
 * What the cache holds.  The tokens of a (layer, sequence, KV head) are cut into blocks of 32 consecutive tokens.  A block's keys have
 * one scale and its values another:
 *     scale = amax / 127,  code = rint(x / scale) in [-127, 127],  x ~ code * scale
 * with amax the largest magnitude among the block's 32 x 128 numbers (of the tokens there are, while the block is not full), both
 * quotients rounded to fp32, ties to even.  A block of zeros has scale 0 and codes 0.  A block with an infinity or NaN has a NaN scale:
 * its values are NaN, and so are outputs that see one of its tokens.  8.0078 bits per element.
 *
 * A block that is not full is quantised again from its raw tokens (kept in `raw`) with every append, so that after each call that
 * brings a sequence tokens it holds what one call with all of them would have left, bit for bit.
 *
 * Pages.  A page has room for page_tokens tokens of one sequence in all layers and heads.  table[b][j] is the page with tokens
 * [j * page_tokens, (j + 1) * page_tokens) of sequence b, -1 where there is none; refs[p] counts the table entries that name page p, 0
 * = free.  okq_pages_* keep both; a caller with an allocator of its own may write them itself.  A page is written only through a
 * sequence's append behind its length, so pages that are full can be shared.
 */
#ifndef OKQ_PAGED_H
#define OKQ_PAGED_H

#include "okq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define OKQ_FP16 0
#define OKQ_BF16 1
#define OKQ_FP32 2 /* okq_rope_apply and the normed heads only */

typedef struct okq_paged {
  int32_t n_layers, batch, n_kv_heads, n_q_heads; /* GQA group n_q_heads / n_kv_heads: an integer <= 8; head_dim is 128 */
  int32_t page_tokens; /* 32, 64, 128 or 256 */
  int32_t n_pages;     /* pages of the pool */
  int32_t max_pages;   /* table entries per sequence */
  int32_t dtype;       /* OKQ_FP16 or OKQ_BF16: keys and values given, raw tokens, queries, outputs */
  int8_t* codes;       /* [n_layers][n_pages][n_kv_heads][2][page_tokens][128], keys before values */
  float* scales;       /* [n_layers][n_pages][n_kv_heads][2][page_tokens / 32] */
  void* raw;           /* [n_layers][batch][n_kv_heads][2][32][128] of dtype: token t of the unfinished block in slot t mod 32 */
  int32_t* table;      /* [batch][max_pages] */
  int32_t* refs;       /* [n_pages] */
  int32_t* seq_len;    /* [n_layers][batch] */
  int32_t* status;     /* [1] sticky first device-side error, 0 = none */
} okq_paged;

/* Byte sizes of the seven buffers for the given shape fields, in the order of the struct. */
okq_status okq_paged_sizes(const okq_paged* shape, size_t out_bytes[7]);

/* Bytes of scratch that the calls below need at most for `layer_count` layers and n_new queries per sequence, or fewer of either; 0 on a
 * shape error. */
size_t okq_paged_workspace_bytes(const okq_paged* cache, int32_t layer_count, int32_t n_new);

/*
 * Rotary positions with three axes (time, height, width).  Channels c and c + pairs of a head are turned by the angle
 * positions[axis(c)] * freq[c], pairs = sections[0] + sections[1] + sections[2] <= 64, a multiple of 8; channels from 2 * pairs on
 * stay as they are.
 *   interleaved 0  the first sections[0] pairs follow axis 0, the next sections[1] axis 1, the last sections[2] axis 2
 *   interleaved 1  pair c follows axis 1 if c mod 3 = 1 and c < 3 sections[1], axis 2 if c mod 3 = 2 and c < 3 sections[2], else axis 0
 *                  (OKQ_ERR_INVALID_ARG where 3 sections[1] - 2 or 3 sections[2] - 1 is not a pair)
 *   freq       device double [pairs], radians per position
 *   positions  device int32 [3][batch][n]
 * Text alone: three equal positions.  The angle is taken and reduced in 64 bits: cosine and sine are off by 2^-22 + |angle| * 2^-51 at
 * most (absolute), two units of fp32 up to 2^27 radians and 2^-20 more at 2^31.  |angle| < 2^51.
 */
typedef struct okq_rope {
  int32_t sections[3];
  int32_t interleaved;
  const double* freq;
  const int32_t* positions;
} okq_rope;

/* A tensor to rotate: element (b, h, i, c) at in[b*in_strides[0] + h*in_strides[1] + i*in_strides[2] + c], the result likewise;
 * strides in elements, multiples of 16 bytes.  in == out with equal strides is allowed, any other overlap is not. */
typedef struct okq_rope_tensor {
  const void* in;
  void* out;
  int64_t in_strides[3], out_strides[3];
  int32_t heads;
} okq_rope_tensor;

/* Rotates q and, unless null, k (both of `dtype`, fp16, bf16 or fp32) in one launch.  inverse != 0 turns back, which is the
 * rotation's transpose: applied to the gradients of the outputs it gives those of the inputs.  batch or n = 0 is a no-op. */
okq_status okq_rope_apply(const okq_rope* rope, int32_t dtype, int32_t batch, int32_t n, const okq_rope_tensor* q,
                          const okq_rope_tensor* k, int32_t inverse, void* stream);

/*
 * Norm of every head, then the rotation, in one pass: for a row x of 128 channels
 *     y = R (weight * x * r),  r = (mean(x^2) + eps)^(-1/2)
 * with R the rotation of okq_rope (none where `rope` is null); all of it in 32 bits, rounded to `dtype` once.  Rows whose squares have no
 * sum in 32 bits are taken care of.  A NaN makes its whole row NaN; an infinity its own channel, and the one that it is turned with, and zeros of
 * the others.
 */
typedef struct okq_norm_tensor {
  const void* in;       /* element (b, h, i, c) at in[b*in_strides[0] + h*in_strides[1] + i*in_strides[2] + c], the others likewise */
  const void* grad_out; /* okq_norm_rope_grad only: gradient of the result */
  void* out;            /* the result; of okq_norm_rope_grad the gradient of `in` */
  int64_t in_strides[3], grad_strides[3], out_strides[3]; /* in elements, multiples of 16 bytes */
  const void* weight;   /* [128] of weight_dtype, the same for all heads; null: ones */
  float* weight_grad;   /* okq_norm_rope_grad only: [128], overwritten; null: not wanted */
  int32_t weight_dtype; /* OKQ_FP16, OKQ_BF16 or OKQ_FP32 */
  int32_t heads;
} okq_norm_tensor;

/* q and, unless null, k (both of `dtype`, fp16, bf16 or fp32) in one launch.  1e-30 <= eps.  out == in with equal strides is allowed, any
 * other overlap is not.  batch or n = 0 is a no-op. */
okq_status okq_norm_rope_apply(const okq_rope* rope, float eps, int32_t dtype, int32_t batch, int32_t n, const okq_norm_tensor* q,
                               const okq_norm_tensor* k, void* stream);

/* The gradients of `in` and of the weights (sums over all rows in 32 bits, in an order that depends on the sizes alone) from `in`, as it
 * was given to okq_norm_rope_apply, and the gradient of its result.  out == grad_out or out == in with equal strides is allowed.
 * workspace: okq_norm_rope_workspace_bytes (0 on sizes that are refused); not needed without rows, where the weights' gradients are zeros,
 * and where no weight_grad is wanted. */
okq_status okq_norm_rope_grad(const okq_rope* rope, float eps, int32_t dtype, int32_t batch, int32_t n, const okq_norm_tensor* q,
                              const okq_norm_tensor* k, void* workspace, size_t workspace_bytes, void* stream);
size_t okq_norm_rope_workspace_bytes(int32_t batch, int32_t n, int32_t q_heads, int32_t k_heads);

/*
 * Appends up to n_new tokens per sequence to layers [layer, layer + layer_count): new_len[b] of them (clamped to [0, n_new]), all
 * where new_len is null; rows behind are not read.
 *   k, v     device, of the cache's dtype, element (l, b, h, i, c) at k[l*ks[0] + b*ks[1] + h*ks[2] + i*ks[3] + c], l counted from
 *            `layer`; strides in elements, multiples of 8
 *   new_len  device int32 [batch] or null
 *   rope     null, or the rotation that the keys are given first (positions [3][batch][n_new], the same for all layers): the same
 *            numbers, bit for bit, as okq_rope_apply into a tensor of the cache's dtype and this call without it
 * The pages must be there (okq_pages_reserve): a sequence whose tokens would need a table entry that is missing, or that have no
 * room in its row, is left as it was, and the status word becomes OKQ_ERR_CAPACITY.
 *
 * Taking tokens back.  seq_len may be lowered as far as the start of the unfinished block (the last multiple of 32 not above it): the
 * next append with a token quantises the block again without them; until then its codes keep the scale that they had a part in.
 * It must not be lowered further: `raw` holds that block's tokens alone, an append would quantise those of another one, and nothing can tell.
 * Drafted tokens that may be rejected across the end of a block are appended to a fork of the sequence (okq_pages_fork), which is released
 * with them; the accepted ones are appended to the original.
 */
okq_status okq_paged_append(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* k, const int64_t k_strides[4],
                            const void* v, const int64_t v_strides[4], int32_t n_new, const int32_t* new_len,
                            const okq_rope* rope, void* stream);

/* Values that tokens [begin, begin + n) of every sequence stand for, of the cache's dtype: k_out, v_out device
 * [layer_count][batch][n_kv_heads][n][128]; rows of tokens that a sequence does not hold are left as they were. */
okq_status okq_paged_read(const okq_paged* cache, int32_t layer, int32_t layer_count, int32_t begin, int32_t n, void* k_out,
                          void* v_out, void* stream);

/*
 * Attention of the newest tokens over the cache: query i of sequence b, i < q_len[b] (clamped to [0, n_new]; n_new where q_len is null),
 * belongs to token seq_len - q_len[b] + i and sees the tokens up to and including that one.  n_new = 1: one query per sequence that
 * sees all of it.  A query that sees nothing (an empty sequence, more queries than tokens) gives zeros; rows behind q_len[b] are left
 * as they were.
 *   q         device, of the cache's dtype, element (l, b, h, i, c) at q[l*qs[0] + b*qs[1] + h*qs[2] + i*qs[3] + c]; strides multiples of 8
 *   rope      null, or the rotation that the queries are given first (positions [3][batch][n_new]), as okq_rope_apply would
 *   sm_scale  softmax scale, normally 1/sqrt(128)
 *   out       device, of the cache's dtype, with strides of its own
 *   workspace device scratch of okq_paged_workspace_bytes(cache, layer_count, n_new); nothing in it is kept between calls
 * Numbers.  Scores, maxima, sums and normalisers have 32 bits.  With few rows (queries x group) to a head, queries are in fixed point, 2^-24 of
 * their row's largest channel, and numerators (weight x value scale) too, 2^-30 of the largest among the 128 tokens of a tile.  With many,
 * queries are fp16 numbers after a power of two, and numerators fp16: 11 bits (two such numbers, 22 bits, with a window and for a tree), and
 * not less than 2^-18 of the largest among 64 tokens; those 2^-68 below the row's largest, and what adds less than 2e-32 to an output, may be
 * lost.
 * Query rows without a magnitude above 1e-30 count as zeros.
 * A sequence with a page missing below its length gives NaN and the status OKQ_ERR_INVALID_ARG.  OKQ_ERR_UNSUPPORTED (and a workspace
 * of 0 bytes) where the work, were all sequences as long as their rows of the table, is 2^31 pieces of 128 tokens and 8 or 256 rows
 * or more.
 */
okq_status okq_paged_attention(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t q_strides[4],
                               int32_t n_new, const int32_t* q_len, const okq_rope* rope, float sm_scale, void* workspace,
                               size_t workspace_bytes, void* out, const int64_t out_strides[4], void* stream);

/*
 * The same with a window: a query of token p sees token t <= p where p - t < window (at least 1: itself) or t < sinks.  Tokens are counted as
 * the cache holds them, so that okq_pages_slide changes nothing.  Pages that no query of the call sees are not read, and need not be there.
 * A window or sinks as long as a row of the table: okq_paged_attention, bit for bit (its numerators of 11 bits included).  OKQ_ERR_UNSUPPORTED
 * where that gives it, however short the window is.
 */
okq_status okq_paged_attention_window(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t q_strides[4],
                                      int32_t n_new, const int32_t* q_len, const okq_rope* rope, float sm_scale, int32_t window, int32_t sinks,
                                      void* workspace, size_t workspace_bytes, void* out, const int64_t out_strides[4], void* stream);

/*
 * The same for drafted tokens that form a tree.  The newest q_len[b] tokens of sequence b are its nodes, node j being token seq_len - q_len + j,
 * and query i is node i's: it sees all tokens before the nodes, and node j where bit j mod 64 of seen[b][i][j / 64] is set (itself only if its own
 * is; bits from q_len[b] on do not count).  A query that sees nothing gives zeros.
 *   seen   device uint64 [batch][n_new][(n_new + 63) / 64], as okq_tree_ancestors makes it, or any other
 * The nodes are appended like other tokens, in any order that puts parents first, with positions of their own in `rope`; to a fork, since
 * they may be rejected.
 */
okq_status okq_paged_attention_tree(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t q_strides[4],
                                    int32_t n_new, const int32_t* q_len, const okq_rope* rope, float sm_scale, const uint64_t* seen,
                                    void* workspace, size_t workspace_bytes, void* out, const int64_t out_strides[4], void* stream);

/* What the nodes of each sequence's tree see, from their parents: bits of a node's ancestors and its own, and how many ancestors it has.
 *   parents  device int32 [batch][n_new]: a node before it, or -1 for one that follows the sequence itself.  Anything else: such a node counts
 *            as one without a parent, and the cache's status becomes OKQ_ERR_INVALID_ARG
 *   q_len    device int32 [batch] or null, nodes of each sequence (clamped to [0, n_new]); rows behind are left as they were
 *   seen     device uint64 [batch][n_new][(n_new + 63) / 64]
 *   depth    device int32 [batch][n_new], or null
 * n_new at most 4096. */
okq_status okq_tree_ancestors(const okq_paged* cache, const int32_t* parents, int32_t n_new, const int32_t* q_len, uint64_t* seen, int32_t* depth,
                              void* stream);

/* Testing aid for the bounded waits of okq_paged_attention, as okq_debug_bulk_timeout is for the 2-bit path's quantiser: nothing of a
 * sequence's codes is delivered and every wait is limited to `limit_clocks` SM clocks.  The kernel returns by itself, outputs of
 * sequences that hold tokens are NaN, the status word becomes OKQ_ERR_TIMEOUT. */
okq_status okq_debug_paged_timeout(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t q_strides[4],
                                   int32_t n_new, void* workspace, size_t workspace_bytes, void* out, const int64_t out_strides[4],
                                   int64_t limit_clocks, void* stream);

/* The same for okq_paged_attention_window (window > 0, seen null) and okq_paged_attention_tree (window 0, seen as there). */
okq_status okq_debug_paged_timeout_sight(const okq_paged* cache, int32_t layer, int32_t layer_count, const void* q, const int64_t q_strides[4],
                                         int32_t n_new, int32_t window, int32_t sinks, const uint64_t* seen, void* workspace,
                                         size_t workspace_bytes, void* out, const int64_t out_strides[4], int64_t limit_clocks, void* stream);

/* How okq_paged_attention would take a call; for tests of the rules.  Positive: the decode kernel with a cluster of so many blocks per
 * (layer, sequence, KV head); OKQ_PLAN_LINE: the decode kernel over even ranges, and the merge; OKQ_PLAN_PROMPT: the prompt kernel; 0:
 * refused.  Only sizes are looked at. */
enum { OKQ_PLAN_LINE = -1, OKQ_PLAN_PROMPT = -2 };
int32_t okq_debug_paged_plan(const okq_paged* cache, int32_t layer_count, int32_t n_new);   /* and okq_paged_attention_tree */
int32_t okq_debug_paged_plan_window(const okq_paged* cache, int32_t layer_count, int32_t n_new, int32_t window, int32_t sinks);

/*
 * The pages.  All of it happens on the device, in stream order, without the host; free pages are handed out lowest index first, to
 * sequences and entries in ascending order, so that results do not depend on timing.  Indices out of range are skipped and set the
 * status OKQ_ERR_INVALID_ARG.
 */

/* Entries for at least tokens[b] tokens (device int32 [batch]) in every sequence's row; entries that are there stay.  Without enough
 * free pages, or with tokens[b] > max_pages * page_tokens, nothing is changed and the status becomes OKQ_ERR_CAPACITY. */
okq_status okq_pages_reserve(const okq_paged* cache, const int32_t* tokens, void* stream);

/* For i = 0 .. count - 1 in order: sequence dst[i], which must have no pages, gets the tokens of sequence src[i] (device int32
 * [count] both).  Full pages are shared, the unfinished one is copied into a free page, raw tokens and lengths are copied; the
 * source must hold equally many tokens in all layers.  A pair that cannot be forked is skipped (OKQ_ERR_INVALID_ARG, or
 * OKQ_ERR_CAPACITY without a free page).  workspace: 16 * count bytes (okq_paged_workspace_bytes covers `batch` pairs). */
okq_status okq_pages_fork(const okq_paged* cache, const int32_t* src, const int32_t* dst, int32_t count, void* workspace,
                          size_t workspace_bytes, void* stream);

/* Sequences seqs[0 .. count) (device int32) give up their pages and become empty in all layers; naming one twice is naming it once. */
okq_status okq_pages_release(const okq_paged* cache, const int32_t* seqs, int32_t count, void* stream);

/* Gives back the pages that okq_paged_attention_window with this window and these sinks will not see again from any token that is still to
 * come: of tokens [sinks, seq_len - window], seq_len that of the shortest layer, the whole pages leave each sequence's row, the entries
 * behind them move down, and the lengths of all layers shrink by their tokens (multiples of page_tokens).  Keys stay as they were rotated:
 * positions go on counting what was dropped.  To be called when the attention of the tokens appended so far is through in all layers, and none of
 * them will be taken back: the tokens before them, come again, would see further back than these.
 * 1 <= window, 0 <= sinks.  dropped (device int32 [batch], may be null) receives the tokens that each sequence lost. */
okq_status okq_pages_slide(const okq_paged* cache, int32_t window, int32_t sinks, int32_t* dropped, void* stream);

/* Copies codes and scales of pages src[i] to pages dst[i] (device int32 [count]) in all layers; tables and counts stay.  A pair whose
 * destination is named by another pair, as source or destination, is skipped (OKQ_ERR_INVALID_ARG). */
okq_status okq_pages_copy(const okq_paged* cache, const int32_t* src, const int32_t* dst, int32_t count, void* stream);

/* Moves pages in use to the front of the pool: with n of them in use, those behind the first n go, in ascending order, to the free
 * ones among the first n; tables and counts follow.  n_live (device int32 [1], may be null) receives n.
 * workspace: okq_paged_workspace_bytes(cache, 1, 1). */
okq_status okq_pages_compact(const okq_paged* cache, int32_t* n_live, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* OKQ_PAGED_H */
