/*
 * jupiter_paged.h -- keys and values in pages: the operators of a step over many requests whose caches share one pool
 * (entry points of libjupiter_stage.so).
 *
 * A cache of jupiter_stage.h is one buffer per sequence, a fork of it shares one prefix, and a call advances all its
 * branches by the same number of tokens.  Here a POOL holds pages of page_size positions, a request's BLOCK TABLE names
 * the pages that hold its positions in order, and a call takes the rows of any number of requests, each with any number
 * of new tokens (a RAGGED batch): rows row_start[i] .. row_start[i+1]-1 belong to request i.  Requests (outline branches,
 * Jupiter paper Sec. V-B) that share a prefix name the same pages; only pages that the prefix fills may be shared, as a step's
 * tokens go into the last page of a request while that has room, and jup_paged_extend() copies no page (a branch that begins inside
 * a page needs a copy of it of its own: jup_paged_reorder() and jup_paged_copy()).  A speculative step (Sec. V-A) is
 *
 *     jup_paged_extend     lengths -> pages, positions, slots                       (once per step)
 *     jup_paged_append     rotary embedding, keys and values into their slots       (every layer; or, for a stage of
 *     jup_paged_attention  the new tokens over the pages                             this library, all of its layers:
 *                                                                                    jup_stage_prefill_paged)
 *     jup_verify_drafts    drafted tokens against the target's probabilities, the requests' new lengths (once per step)
 *
 * Lengths, tables and tokens stay on the GPU: the host waits for nothing, and a captured step can be replayed.
 *
 * A pool may hold 8-bit codes and scales in place of bf16 values (jup_paged_append8, jup_paged_attention8, jup_paged_read8,
 * jup_stage_prefill_paged8): half the bytes, which is what decoding behind long caches waits for.  Where requests are the beams
 * of a search, jup_beam_select() ends a step in place of jup_verify_drafts(), and jup_paged_reorder() with jup_paged_copy()
 * makes the tables that the next one begins with; the same two let a request branch inside a page.
 *
 * Conventions (beside those of jupiter_stage.h)
 *   - Pointers inside the argument structs are DEVICE pointers; the structs themselves are host memory, read during the
 *     call.  Strides count elements.
 *   - Arguments are validated on the host; a failing call enqueues nothing.  What only the GPU knows (lengths, tables,
 *     slots) is checked by the kernels: whatever these hold, nothing outside the given buffers is read or written.
 *   - dtype JUP_F32 or JUP_BF16 as in jupiter_stage.h: JUP_F32 is the check mode (plain kernels, any even head_dim up to
 *     256); JUP_BF16 needs head_dim 128, 16-byte aligned tensors and strides that are multiples of 8.
 *   - Sizes: page_size is a power of two, 8 .. 65536; n_blocks * page_size <= 2^31 - 1, table_width * page_size <= 2^31 - 256;
 *     n_seqs <= JUP_PAGED_MAX_SEQS.
 */
#ifndef JUPITER_PAGED_H
#define JUPITER_PAGED_H

#include "jupiter_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

#define JUP_PAGED_MAX_SEQS 16384

/* Element i of (block, head, slot) lies at block * block_stride + head * head_stride + slot * slot_stride + i, of k and of v. */
typedef struct {
    void *k, *v;
    int64_t block_stride, head_stride, slot_stride;
    int32_t n_blocks, page_size, n_kv_heads, head_dim;
    int32_t dtype; /* JUP_F32 or JUP_BF16; of the calls that take scales JUP_I8 or JUP_E4M3 */
} jup_paged_pool_t;

/*
 * Pools in 8 bits.  k and v hold codes of one byte (strides count them), JUP_I8: two's complement, JUP_E4M3: sign, 4 bits of
 * exponent, 3 of fraction, no infinities.  Code i of (block, head, slot) stands for code * scale, with the scale of that head and
 * slot at block * block_stride + head * head_stride + slot of scales->k or scales->v (fp32).  What jup_paged_append8() writes, of the
 * 128 values x_i of a head:
 *     m = max(2^-100, max_i |x_i|),  scale = m / T,  code_i = the one nearest to x_i * (T / m), ties to even
 * in fp32, with T = 127 (JUP_I8) or 448 (JUP_E4M3): a value is off by at most scale / 2 (JUP_I8), or the larger of 2^-4 of itself and
 * scale * 2^-10 (JUP_E4M3), and by 2^-22 m, the three roundings in fp32.  A head with an infinity or a NaN gets scale NaN and codes 0.
 * Such pools need head_dim 128, tensors that are 16-byte aligned, strides of codes that are multiples of 16 and strides of scales that
 * are multiples of 4; the rows that go with them (q, k, v and results) are JUP_BF16.
 */
typedef enum { JUP_I8 = 3, JUP_E4M3 = 4 } jup_code_t;
typedef struct {
    float *k, *v;
    int64_t block_stride, head_stride;
    int64_t layer_stride; /* between the layers of a stage; used by jup_stage_prefill_paged8() and jup_paged_copy() alone */
} jup_paged_scales_t;

/*
 * Block tables, positions and slots of a step.  Request i holds lengths[i] positions in the first owned[i] entries of its
 * table row and gets n_new[i] more (0: none).  Pages are taken from the top of a stack of free blocks, in request order:
 * with F = *free_count and s the number of pages taken before, the next entry is free_blocks[F - 1 - s].
 *   table           [n_seqs][table_stride], table_width entries used: the taken pages are entered behind the owned[i] first
 *                   entries; all other entries stay as they are
 *   free_blocks     [n_free], n_free <= 2^30;  free_count [1]
 *   row_start       out [n_seqs + 1]: prefix sums of n_new
 *   positions       out [max_rows]: position of every row (rows behind the last: 0)
 *   slots           out [max_rows]: block * page_size + place in the block (rows behind the last: -1)
 *   new_lengths     out [n_seqs]: lengths + n_new;  new_owned out [n_seqs];  new_free_count out [1]
 *   status          out [1]: 0, or why the step does not fit, the smallest of
 *                     1  a negative number, owned[i] > table_width, or *free_count outside [0, n_free]
 *                     2  a request needs more than table_width pages
 *                     3  more than max_rows rows
 *                     4  more pages than there are free blocks
 *                   Then no request gets anything: row_start is all 0, slots all -1, lengths, owned, free_count and table
 *                   are as before, and the other calls of the step do nothing for it.
 * new_lengths, new_owned and new_free_count may be the same buffers as lengths, owned and free_count (else nothing may
 * overlap).  A page is given back by pushing it on the stack; entries behind the pages of a shortened request stay owned
 * and are used again.  Errors: JUP_EINVAL, JUP_EDEVICE.
 */
typedef struct {
    int32_t n_seqs, page_size, table_width, n_free, max_rows;
    int64_t table_stride;
    const int32_t *lengths, *n_new, *owned;
    int32_t *table;
    const int32_t *free_blocks, *free_count;
    int32_t *row_start, *positions, *slots, *new_lengths, *new_owned, *new_free_count, *status;
} jup_paged_extend_t;
JUP_API jup_status_t jup_paged_extend(const jup_paged_extend_t *args, void *stream);

/*
 * Rows of a step into their slots (steps 2 and 3 of jupiter_stage.h): k is rotated at positions[r] and stored with v at
 * slots[r]; q, if given, is rotated into q_out (which may be q itself).  rope_theta 0: nothing is rotated (then q must be
 * NULL and positions may be).  A slot outside the pool (-1: a row behind the last) stores nothing; its q is rotated all
 * the same.  Two rows with the same slot: the one or the other, element by element.
 *   q, k, v, q_out  element i of (row, head) at row * row_stride + head * head_stride + i
 *   n_heads         of q and q_out; those of k and v are the pool's
 * Rotation: pairs (i, i + head_dim / 2), angle position * rope_theta^(-2i / head_dim) in 64 bits, negative positions too.
 * Errors: JUP_EINVAL, JUP_EDEVICE.
 */
typedef struct {
    int32_t n_rows, n_heads;
    const void *q, *k, *v;
    void *q_out;
    int64_t q_row_stride, q_head_stride, k_row_stride, k_head_stride, v_row_stride, v_head_stride, q_out_row_stride, q_out_head_stride;
    const int32_t *positions, *slots;
    float rope_theta;
} jup_paged_append_t;
JUP_API jup_status_t jup_paged_append(const jup_paged_pool_t *pool, const jup_paged_append_t *args, void *stream);

/*
 * Attention of the new tokens over the pages.  Token t of the m = row_start[i+1] - row_start[i] new ones of request i sees
 * the positions 0 .. lengths[i] - m + t (lengths count the new tokens, whose keys and values are in the pool), so lengths
 * and row_start are what jup_paged_extend() left.  Query head h reads key/value head h / (n_heads / n_kv_heads).
 *     out = sum_j p_j v_j,  p = softmax_j(scale * q . k_j)
 * JUP_BF16: p is rounded to bf16 as it meets v; sums are fp32 and divided by sum p at the end, so that they overflow where values
 * are larger than 2^120 / number of keys.
 * A position whose table entry is outside [0, n_blocks), or that lies behind table_width pages, is not there; a row that
 * sees no position gets zeros.  Values of positions a row does not see do not reach it, whatever they are.  Rows of q and
 * out outside [row_start[0], row_start[n_seqs]) are neither read nor written.
 *   out             may be q, with its strides
 *   n_rows          rows of q and out; max_new: the longest m expected.  It chooses between kernels and decides nothing
 *                   else: results are right whatever it says.
 *   workspace       >= jup_paged_workspace_bytes(...) bytes, 256-byte aligned, ZERO when first used; every call leaves it
 *                   ready for the next.  Calls that share one must not overlap in time (captured
 *                   graphs included).  Not needed in check mode
 *   scale           positive, at most 1e38
 * Results do not depend on what the pages' order in the pool is, nor on the run; they do depend, in the last bits of fp32
 * sums, on how the keys are divided among workgroups, which follows from all requests of the call.
 * Errors: JUP_EINVAL, JUP_EDEVICE.
 */
typedef struct {
    int32_t n_seqs, n_rows, n_heads, max_new, table_width;
    int64_t table_stride;
    const void *q;
    void *out;
    int64_t q_row_stride, q_head_stride, out_row_stride, out_head_stride;
    const int32_t *row_start, *lengths, *table;
    float scale;
    void *workspace;
    size_t workspace_bytes;
} jup_paged_attention_t;
JUP_API jup_status_t jup_paged_attention(const jup_paged_pool_t *pool, const jup_paged_attention_t *args, void *stream);

/*
 * The same for pools in 8 bits.  Append: k is rotated in fp32 and quantised without another rounding; of two rows with the same slot the codes may
 * be one's and the scale the other's.  Attention: the scale of a key multiplies its score, that of a value its probability, and the product meets the value
 * as two numbers of bf16, which hold it to 2^-15; as one, rounded, 2^-8, in calls of long chunks and prompts (of G = n_heads / n_kv_heads: max_new * G
 * above 96, and (n_rows * G / 32 + n_seqs) * n_kv_heads above 1536).  Codes are exact in bf16.  A score or a
 * value of a key that a row does not see does not reach it, whatever codes and scales hold.  A key that it sees, and whose codes or scales are no finite
 * numbers, may make all of the row NaN however small the key's probability is.  JUP_I8 codes of -128 and JUP_E4M3 codes that are no numbers, which
 * jup_paged_append8() does not write, count as what they are.  Errors: JUP_EINVAL, JUP_EDEVICE.
 */
JUP_API jup_status_t jup_paged_append8(const jup_paged_pool_t *pool, const jup_paged_scales_t *scales, const jup_paged_append_t *args, void *stream);
JUP_API jup_status_t jup_paged_attention8(const jup_paged_pool_t *pool, const jup_paged_scales_t *scales, const jup_paged_attention_t *args, void *stream);

/*
 * Rows out of their slots: row r of k and v is what the pool holds at slots[r], or zeros where that is outside the pool.
 *   k, v            element i of (row, head) at row * row_stride + head * head_stride + i.  JUP_BF16, or JUP_F32 of a JUP_F32 pool.  Each
 *                   may be NULL
 * jup_paged_read8(): code * scale, rounded once.  Errors: JUP_EINVAL, JUP_EDEVICE.
 */
typedef struct {
    int32_t n_rows;
    void *k, *v;
    int64_t k_row_stride, k_head_stride, v_row_stride, v_head_stride;
    const int32_t *slots;
} jup_paged_read_t;
JUP_API jup_status_t jup_paged_read(const jup_paged_pool_t *pool, const jup_paged_read_t *args, void *stream);
JUP_API jup_status_t jup_paged_read8(const jup_paged_pool_t *pool, const jup_paged_scales_t *scales, const jup_paged_read_t *args, void *stream);

/* Bytes of a workspace that serves every call of jup_paged_attention(), jup_paged_attention8(), jup_verify_drafts(), jup_beam_select() and
 * jup_paged_reorder(). */
JUP_API size_t jup_paged_workspace_bytes(void);

/*
 * The forward of a stage (steps 1-6 of jupiter_stage.h) over the rows of a ragged batch, with a pool in place of the caches: what
 * jup_stage_prefill_chunk() computes for every request's new tokens on its own cache, the weights read once for all of
 * them.  Enqueues what jup_paged_append() and jup_paged_attention() do in every layer.
 *   hidden_in, hidden_out   [n_rows, d_model], stage dtype; hidden_out may be hidden_in.  n_rows <= the stage's max_chunk_tokens.
 *                   Rows behind the last request's may be there (a captured step of fixed size): hidden_out is then unspecified in them
 *   pool            of the stage's first layer: n_kv_heads = n_heads, head_dim as the stage's; JUP_BF16 for the bf16 and 4-bit stages.
 *                   A layer's k and v lie layer_stride elements behind the one's before it
 *   others          as in jup_paged_extend() and jup_paged_attention()
 * Results are those of the calls on caches up to the summation order of fp32 sums and the rounding of probabilities to bf16.
 * Errors: JUP_EINVAL, JUP_ECAP, JUP_EDEVICE.
 */
typedef struct {
    jup_paged_pool_t pool;
    int64_t layer_stride;
    int32_t n_seqs, max_new, table_width;
    int64_t table_stride;
    const int32_t *row_start, *lengths, *table, *positions, *slots;
    void *workspace;
    size_t workspace_bytes;
} jup_paged_batch_t;
JUP_API jup_status_t jup_stage_prefill_paged(jup_stage_t *stage, const void *hidden_in, int32_t n_rows, const jup_paged_batch_t *batch,
                                             void *hidden_out, void *stream);

/* The same over a pool in 8 bits (of the bf16 and 4-bit stages); batch->pool.dtype JUP_I8 or JUP_E4M3. */
JUP_API jup_status_t jup_stage_prefill_paged8(jup_stage_t *stage, const void *hidden_in, int32_t n_rows, const jup_paged_batch_t *batch,
                                              const jup_paged_scales_t *scales, void *hidden_out, void *stream);

/*
 * Verification of drafted tokens (Sec. V-A step 4).  Row r of request i holds an input token of the step: the last one
 * decided, then the drafted ones.  Row r of target_probs is the target model's distribution of the token that follows row
 * r, row r of draft_probs the distribution that the token in row r + 1 was drawn from (the last row of a request is not read).  Drafted token
 * x = tokens[r + 1] is accepted while
 *     u_accept[r] * draft_probs[r][x] < target_probs[r][x]
 * (draft_probs NULL: drafts were taken for certain, 1 in place of their probability).  At the first row that rejects, or
 * the last one, the next token is drawn from w = max(target - draft, 0) there (draft_probs NULL: target without x), or from w = target behind the
 * last draft: the lowest j with w_0 + .. + w_j > u_sample[i] * (w_0 + .. + w_(vocab-1)).  The tokens that come out are then distributed
 * as the target's (uniform u in [0, 1)).  Comparisons and sums are in 64 bits.
 *   target_probs, draft_probs   [n_rows][vocab], n_rows and vocab <= 2^30, rows *_row_stride elements apart; probs_dtype JUP_F32 or
 *                   JUP_BF16
 *   n_accepted      out [n_seqs]: drafts accepted;  next_token out [n_seqs]
 *   emitted         out [n_rows], may be NULL: rows of a request: its accepted drafts, the next token, then -1
 *   lengths, new_lengths   [n_seqs], may both be NULL: cached positions before the step -> positions that are valid behind it,
 *                   lengths[i] + 1 + n_accepted[i] (the entries of rejected drafts are dropped); may be the same buffer
 * A weight that is not a positive finite number counts as 0; if all of w are (a rejected row with target <= draft
 * everywhere), target takes its place, and if those are 0 too the next token is -1.  A drafted token outside [0, vocab) is
 * rejected (and excludes nothing).  u_sample below 0 counts as 0; beyond 1, or NaN: the last token with w > 0.  A request without rows gets
 * n_accepted 0, next_token -1, its length.  Rows outside [row_start[0], row_start[n_seqs]) are not touched.  Outputs overlap
 * nothing else.
 *   workspace       as in jup_paged_attention()
 * Errors: JUP_EINVAL, JUP_EDEVICE.
 */
typedef struct {
    int32_t n_seqs, n_rows, vocab, probs_dtype;
    const int32_t *tokens, *row_start;
    const void *target_probs, *draft_probs;
    int64_t target_row_stride, draft_row_stride;
    const float *u_accept, *u_sample;
    int32_t *n_accepted, *next_token, *emitted;
    const int32_t *lengths;
    int32_t *new_lengths;
    void *workspace;
    size_t workspace_bytes;
} jup_verify_drafts_t;
JUP_API jup_status_t jup_verify_drafts(const jup_verify_drafts_t *args, void *stream);

/*
 * The end of a step of a beam search.  Request i has n_beams beams, rows i * n_beams .. of logits and scores.  Its candidates are
 * (beam b, token j) with score  scores[b] + logits[b][j] - log sum_k exp(logits[b][k]),  of a beam that has ended (ended[b] not 0)
 * the one candidate (b, end_token) with scores[b].  The n_keep best of them come out, best first; equal scores: the lower beam, then the
 * lower token.  Within a beam logits are compared, then tokens, however far from them its score is; else scores in 64 bits, where of two beams'
 * that are alike to 2^-44 of themselves either may come first.  Exponentials are fp32 with their sums in 64, the logarithm and the score too: a score is off
 * by at most 2^-21 + 2^-22 ln(vocab), mostly far less, and by the rounding of new_scores, 2^-24 of it.
 *   logits          [n_seqs * n_beams][vocab], rows row_stride apart; logits_dtype JUP_F32 or JUP_BF16.  One that is NaN or +infinity
 *                   counts as -infinity, and is no candidate
 *   scores          [n_seqs * n_beams]: sums of log probabilities.  A beam whose score is not finite has no candidates
 *   ended           [n_seqs * n_beams], may be NULL: none has.  Rows of beams that have ended are not read
 *   parents         out [n_seqs * n_keep]: the candidate's beam, as a row of logits (what jup_paged_reorder() takes);
 *   tokens, new_scores, new_ended  out [n_seqs * n_keep]: new_ended is 1 where ended was, or the token is end_token (-1: none is)
 *   Where a request has fewer than n_keep candidates the others are parent -1, token -1, score -infinity, new_ended 0.
 * n_beams and n_keep are 1 .. JUP_BEAM_MOST, vocab 1 .. 2^30, n_seqs * n_beams <= JUP_PAGED_MAX_SEQS.  new_ended may be NULL.  Outputs overlap nothing
 * else (scores and ended are read behind the first outputs).  workspace: as in jup_paged_attention().  Errors: JUP_EINVAL, JUP_EDEVICE.
 */
#define JUP_BEAM_MOST 64
typedef struct {
    int32_t n_seqs, n_beams, n_keep, vocab, logits_dtype, end_token;
    const void *logits;
    int64_t row_stride;
    const float *scores;
    const int32_t *ended;
    int32_t *parents, *tokens;
    float *new_scores;
    int32_t *new_ended;
    void *workspace;
    size_t workspace_bytes;
} jup_beam_select_t;
JUP_API jup_status_t jup_beam_select(const jup_beam_select_t *args, void *stream);

/*
 * Block tables of requests that go on from others: request i of n_out becomes what request parents[i] of n_in was (-1: an empty one).
 * With L positions, the L / page_size pages that these fill are shared.  A page that they fill in part is the parent's own: the lowest i with that
 * parent takes it over, every other one gets a free page and a copy of it is due (jup_paged_copy).  Pages that are in some request's
 * owned[] entries and in none of the new tables go back on the stack, behind what is left of it, in the order of their numbers.
 * So all requests that have pages of the pool are in the call (one that stays what it is: parents[i] = i), or their pages are marked in held.
 *   table           [n_in][table_stride], table_width entries used; new_table [n_out][new_table_stride], new_table_width entries: those
 *                   behind a request's pages are set to -1.  They do not overlap
 *   lengths, owned  [n_in]; new_lengths, new_owned out [n_out]: the parent's length, the pages that it fills or begins
 *   free_blocks     [n_free], n_free <= 2^26: the stack has room for every block, so blocks are numbers below n_free;  free_count [1]
 *   new_free_blocks out [n_free] (may be free_blocks: else all of it is copied);  new_free_count out [1] (may be free_count)
 *   held            [n_free] bytes, may be NULL: blocks that are not 0 there do not go back
 *   copy_from, copy_to  out [n_out]: the page to copy and its copy, or -1
 *   status          out [1]: 0, or the smallest of
 *                     1  a parent outside -1 .. n_in - 1, or of one of the parents: a negative length, owned outside 0 .. table_width, or fewer
 *                        pages than its length needs; *free_count outside [0, n_free]
 *                     2  a request needs more than new_table_width pages
 *                     4  more copies than there are free blocks
 *                   Then the new requests are empty (lengths and owned 0, tables and copies -1) and the stack is as before: the
 *                   old tables still hold.
 * Entries of a table that are no blocks are copied as they are and never go back.  Where the partly filled page is none, copies of it are due all the
 * same: copy_from is that entry, the page in copy_to is the new request's, and as jup_paged_copy() does nothing for it, holds what it held.
 * n_in, n_out <= JUP_PAGED_MAX_SEQS.
 * workspace: as in jup_paged_attention().  Errors: JUP_EINVAL, JUP_EDEVICE.
 */
typedef struct {
    int32_t n_in, n_out, page_size, table_width, new_table_width, n_free;
    int64_t table_stride, new_table_stride;
    const int32_t *parents, *table, *lengths, *owned, *free_blocks, *free_count;
    const uint8_t *held;
    int32_t *new_table, *new_lengths, *new_owned, *new_free_blocks, *new_free_count, *copy_from, *copy_to, *status;
    void *workspace;
    size_t workspace_bytes;
} jup_paged_reorder_t;
JUP_API jup_status_t jup_paged_reorder(const jup_paged_reorder_t *args, void *stream);

/*
 * Pages copied: of every layer's k and v (and scales), page copy_from[i] to page copy_to[i], all slots of it, or the first
 * lengths[i] mod page_size where lengths is given (none where that is 0).  Nothing happens where one of the two is outside the pool.  No page is
 * the target of two copies, or both source and target.
 *   pool, scales    of the first layer, any dtype (scales NULL for JUP_F32 and JUP_BF16); a layer's k and v lie layer_stride elements
 *                   behind the one's before it
 * Errors: JUP_EINVAL, JUP_EDEVICE.
 */
typedef struct {
    int32_t n_copies, n_layers;
    int64_t layer_stride;
    const int32_t *copy_from, *copy_to, *lengths;
} jup_paged_copy_t;
JUP_API jup_status_t jup_paged_copy(const jup_paged_pool_t *pool, const jup_paged_scales_t *scales, const jup_paged_copy_t *args, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* JUPITER_PAGED_H */
