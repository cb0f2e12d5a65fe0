/*
 * wq4_attn.h -- decode attention over a paged key/value cache (sm_103a),
 * part of the same library as wq4.h (libwq4.so).
 *
 * The paper's compiled models run PagedAttention (keys and values kept in
 * fixed-size pages reached through a per-sequence page table, Kwon et al.)
 * and FlashAttention (softmax computed in one pass with a running maximum,
 * Dao et al.) as their attention kernels (Section 2.3).  One decode step of
 * one layer computes, for sequence b and query head j (key/value head
 * h = j / G, G = n_q_heads / n_kv_heads: grouped-query attention),
 *
 *   s_t = scale * q[b][j] . K_t,   o[b][j] = sum_t softmax(s)_t * V_t,
 *
 * over the T = seq_lens[b] cached tokens t, token t being row t % page_size
 * of page page_table[b][t / page_size].
 *
 * Accuracy contract: |o - o_ref| <= 2e-3 * sum_t p_t |V_t| + 2^-40 * sum_t |V_t| +
 * ulp16(|o_ref|) per element, o_ref and p the exact (fp64) result and weights, the
 * sums over the tokens seen.  The path rounds each weight to fp16 for the value
 * product, in units in which the largest is 2^15: a weight of at least 2^-29 of
 * the largest is within 2^-11 of itself, a smaller one within 2^-40 of the largest
 * (the second term, felt only where nearly all the weight lies on tokens whose
 * values are far smaller than the others').  It normalises by the sum of the same
 * rounded weights; scores and all sums are fp32.  Valid while scale * sum_d |q_d
 * K_t,d| <= 64 and values are finite.
 *
 * Conventions are those of wq4.h: device pointers owned by the caller,
 * asynchronous on `stream`, no allocation, argument errors returned before
 * anything is enqueued, device-side problems (a page id outside the pool, a
 * length beyond the page table, a wait that gave up) recorded in the status
 * word that wq4_device_status() reads and clears.
 */
#ifndef WQ4_ATTN_H
#define WQ4_ATTN_H

#include <stddef.h>
#include <stdint.h>

#include "wq4.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The paged cache of one layer. */
typedef struct {
    uint16_t* k;                 /* fp16 [num_pages][n_kv_heads][page_size][head_dim], 16-byte aligned */
    uint16_t* v;                 /* same shape and alignment; must not overlap k */
    int num_pages;               /* pages in the pool, >= 1 */
    int n_kv_heads;              /* >= 1 */
    int page_size;               /* tokens per page: a multiple of 16 */
    int head_dim;                /* 128 */
    const int32_t* page_table;   /* int32 [batch][page_table_stride]: page ids of each sequence */
    int page_table_stride;       /* >= 1: entries per sequence (max pages of a sequence) */
} wq4_kv_cache;

/* Largest batch wq4_paged_attention accepts. */
#define WQ4_ATTN_MAX_BATCH 1024

/*
 * Workspace wq4_paged_attention needs for this geometry on the current
 * device: arrival counters (batch * n_kv_heads words, which must be zero
 * before the first call and are left zero by every call that completes) and
 * fp32 partial results of sequences split across thread blocks.  0 on bad
 * arguments.
 */
size_t wq4_paged_attention_workspace_bytes(int batch, int n_q_heads, int n_kv_heads, int head_dim);

/*
 * Decode attention of every sequence and query head (definition above).
 *   cache      : the layer's paged cache (pointers are device pointers).
 *   q          : fp16 [batch] rows of q_stride elements, each holding
 *                [n_q_heads][head_dim] (a row of the fused QKV projection
 *                output works: its first n_q_heads*head_dim entries are q);
 *                16-byte aligned, q_stride % 8 == 0.
 *   seq_lens   : int32 [batch] device array, tokens in the cache per
 *                sequence (the current token included); 0 gives o = 0;
 *                larger than page_table_stride * page_size is clamped and
 *                flagged.
 *   out        : fp16 [batch] rows of out_stride elements, [n_q_heads][head_dim]
 *                each; 4-byte aligned, out_stride even; must not overlap the
 *                inputs or the workspace.
 *   n_q_heads  : a multiple of n_kv_heads with n_q_heads / n_kv_heads <= 8.
 *   scale      : the score scale (1/sqrt(head_dim) for standard attention).
 *   workspace  : device memory of wq4_paged_attention_workspace_bytes(),
 *                16-byte aligned, its counters zero (see there), not shared by
 *                concurrent calls.
 * Sequences are split across the GPU's thread blocks by tokens in equal
 * shares and the shares are merged in a fixed order: the same inputs on the
 * same device give the same bits.  Launched with programmatic dependent
 * launch; everything is read after the previous kernel in `stream` has
 * completed.  Returns WQ4_OK, WQ4_ERR_INVALID,
 * WQ4_ERR_ALIGN, WQ4_ERR_UNSUPPORTED (head_dim != 128, group > 8) or
 * WQ4_ERR_CUDA.
 */
int wq4_paged_attention(const wq4_kv_cache* cache, const uint16_t* q, int q_stride, const int32_t* seq_lens,
                        uint16_t* out, int out_stride, int batch, int n_q_heads, float scale, void* workspace,
                        size_t workspace_bytes, void* stream);

/*
 * wq4_paged_attention under a sliding window with a few first tokens that stay
 * visible (sinks): the new token of sequence b, at position T - 1, sees
 *   t < T  with  t >= T - window  or  t < n_sinks.
 *   window  : tokens of the window, the new one included, >= 1; 0: no window
 *             (n_sinks is then without effect).
 *   n_sinks : >= 0.
 * Everything else is as for wq4_paged_attention, its workspace included.  Only
 * pages that hold a visible token are looked up and read: the others may have
 * been freed (wq4_kv_trim) and their page-table entries may be anything.
 * What masked rows of a visible page hold (NaN included) does not matter.
 */
int wq4_window_attention(const wq4_kv_cache* cache, const uint16_t* q, int q_stride, const int32_t* seq_lens,
                         uint16_t* out, int out_stride, int batch, int n_q_heads, float scale, int window,
                         int n_sinks, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Append step of a decode iteration: writes the new token's key and value of
 * every key/value head into the cache,
 *   cache.k[page_table[b][pos / page_size]][h][pos % page_size][:] = new_k[b][h][:]
 * (and likewise v) with pos = positions[b] (device int32 [batch]).
 *   new_k, new_v : fp16 [batch] rows of new_stride elements holding
 *                  [n_kv_heads][head_dim] (rows of the fused QKV output, offset
 *                  to their k and v parts, work); 16-byte aligned,
 *                  new_stride % 8 == 0.
 * A negative position, one beyond the page table, or a page id outside the
 * pool writes nothing for that sequence and is flagged.  Bit-exact copy.
 */
int wq4_kv_append(const wq4_kv_cache* cache, const uint16_t* new_k, const uint16_t* new_v, int new_stride,
                  const int32_t* positions, int batch, void* stream);

/* ------------------------------------------------------------------------ */
/* Prompts                                                                    */
/* ------------------------------------------------------------------------ */

/*
 * The new tokens of a batch of prompts (or of chunks of them) are rows laid end
 * to end: sequence b owns rows [row_starts[b], row_starts[b + 1]), n of them (0
 * allowed), and they are the last n of its seq_lens[b] tokens: the row r stands
 * at position seq_lens[b] - n + (r - row_starts[b]).
 *   row_starts : int32 [batch + 1] device array, not decreasing, within [0, rows].
 *   seq_lens   : int32 [batch] device array, tokens of each sequence, the new
 *                ones included.
 *   rows       : rows that the buffers hold (>= row_starts[batch]).  Rows that
 *                no sequence owns are left as they are.
 *
 * wq4_prompt_append: for each row of the fused QKV projection's output, the
 * rotation of q and k as in wq4_decode_attn (pairs (x_2i, x_2i+1) by
 * pos * rope_theta^(-2i / 128)) and the append of k and v at the row's position:
 *   q_out[r] = rope(qkv[r][: n_q_heads]),  cache.k <- rope(the next n_kv_heads),
 *   cache.v <- the last n_kv_heads.
 *   qkv   : fp16 rows of qkv_stride elements holding [n_q_heads + 2 *
 *           n_kv_heads][head_dim]; 16-byte aligned, qkv_stride % 8 == 0.
 *   q_out : fp16 rows of q_out_stride elements, [n_q_heads][head_dim] each; 16-byte
 *           aligned, q_out_stride % 8 == 0.  It may be qkv itself (the same
 *           pointer and stride: rotated in place); otherwise it must not overlap it.
 *   rope_theta : > 1, or 0 for no rotation (q is then copied, and left out with
 *           a null q_out).
 * Each rotated element is within half an fp16 ulp, plus 2^-22 of the pair's
 * larger element, of the exact rotation; values are copied bit for bit.  A
 * sequence whose rows have a position below 0, beyond the page table or on a
 * page id outside the pool: those rows' keys and values are not written, and
 * bit 5 is flagged (q is rotated by max(position, 0)).
 * Sequences must not map new positions to the same cache row.
 */
int wq4_prompt_append(const wq4_kv_cache* cache, const uint16_t* qkv, int qkv_stride, uint16_t* q_out,
                      int q_out_stride, const int32_t* row_starts, const int32_t* seq_lens, int batch, int rows,
                      int n_q_heads, double rope_theta, void* stream);

/*
 * Workspace wq4_prompt_attention needs on the current device for calls of at
 * most this batch and this many rows.  0 on bad arguments.
 */
size_t wq4_prompt_attention_workspace_bytes(int batch, int rows, int n_q_heads, int n_kv_heads, int head_dim);

/*
 * Attention of a prompt's rows over the cache, their own keys and values
 * (appended before) included: the row at position i sees
 *   t <= i  with  window == 0  or  t > i - window  or  t < n_sinks
 * and o is as for wq4_paged_attention over those tokens; a row that sees none
 * (position below 0), or only scores of -infinity, gets zeros.  Grouping, scale
 * and the accuracy contract are those of wq4_paged_attention, but that the largest
 * weight is at least 2^6 (weights of 2^-20 of it are within 2^-11 of themselves, and
 * the contract's second term is 2^-31 * sum_t |V_t|) and that the sum that
 * normalises is of the weights before their rounding.  A call whose key
 * tiles, were every row at the page table's end, pass 2^30 (without a window a
 * million rows of 8 key/value heads by 4 with room for a million tokens) returns
 * WQ4_ERR_UNSUPPORTED: split it into chunks.
 *   q, out : fp16 rows of q_stride, out_stride elements, [n_q_heads][head_dim]
 *            each; 16-byte aligned, strides % 8 == 0; out must not overlap the
 *            inputs or the workspace.
 *   workspace : device memory of wq4_prompt_attention_workspace_bytes(), 256-byte
 *            aligned, of any contents, not shared by calls that may overlap.  It is
 *            left with any contents too: wq4_paged_attention and wq4_window_attention,
 *            whose counters must be zero, may be given it only after it was set to 0
 *            (else their merges are wrong, and nothing is flagged).
 * Pages of which no row of the call sees a token are not read: their entries may
 * be anything.  What a row does not see (NaN included) does not reach it.  (An
 * infinite value that a row does see gives an infinity, or NaN where its weight
 * rounds to 0.)  Rows beside a value that is not finite and that some row of their
 * few dozen does not see are right, but computed one by one: milliseconds in place of
 * microseconds (16 rows of 32 heads over 4096 tokens 9 ms).
 * Positions at or beyond the page table's end: the length is clamped there for
 * keys and values and bit 3 flagged; a page id outside the pool among the seen
 * ones reads as zeros and flags bit 4.  Row starts that decrease anywhere: no row
 * is computed, bit 3 is flagged.  Deterministic on one device.
 */
int wq4_prompt_attention(const wq4_kv_cache* cache, const uint16_t* q, int q_stride, const int32_t* row_starts,
                         const int32_t* seq_lens, uint16_t* out, int out_stride, int batch, int rows, int n_q_heads,
                         float scale, int window, int n_sinks, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* Pages                                                                      */
/* ------------------------------------------------------------------------ */

#define WQ4_KV_MAX_SEQS 1024
#define WQ4_KV_MAX_LAYERS 128

/*
 * A pool of pages and the sequences that hold them, kept on the device.  Every
 * layer has its own cache of the same geometry; one page table serves them all.
 * What the calls below keep true, and need:
 *   - page_table[s][j] for j < ceil(seq_lens[s] / page_size) is a page id, or -1
 *     where wq4_kv_trim freed the page; every further entry is -1;
 *   - page_refs[p] is the number of entries that name page p; 0: free.
 * (All -1, 0 and 0 is an empty pool.)  A call that takes pages takes the
 * lowest-numbered free ones in order, so its result depends on the state alone.
 *   layers     : HOST array of num_layers caches, each with this page_table;
 *                at most WQ4_KV_MAX_LAYERS.
 *   page_table : device int32 [max_seqs][layers[0].page_table_stride], less than
 *                2^31 entries (and a page less than 2^26 rows of all its heads).
 *   seq_lens   : device int32 [max_seqs];  max_seqs <= WQ4_KV_MAX_SEQS.
 *   page_refs  : device int32 [num_pages].
 *   workspace  : device memory of wq4_kv_pool_workspace_bytes(), 16-byte aligned,
 *                of any contents.
 * The calls are asynchronous on `stream`, allocate nothing and can be captured;
 * calls on one pool must not overlap on the GPU.  Lists are device int32 [n], n
 * from 0 to WQ4_KV_MAX_SEQS.  What cannot be done is left undone as said at each
 * call and flagged in the status word (bit 7).
 */
typedef struct {
    const wq4_kv_cache* layers;
    int num_layers;
    int max_seqs;
    int32_t* page_table;
    int32_t* seq_lens;
    int32_t* page_refs;
    void* workspace;
    size_t workspace_bytes;
} wq4_kv_pool;

/* 0 on bad arguments. */
size_t wq4_kv_pool_workspace_bytes(int num_pages, int max_seqs);

/* Grows sequence seqs[i] to new_lens[i] tokens: takes the pages it lacks and sets
 * its length (the new tokens' rows hold whatever the pages held).  Refused:
 * an index out of range or listed before, a length below the present one or
 * beyond the page table.  Where the free pages run out, that sequence and all
 * later ones that need any stay as they were. */
int wq4_kv_reserve(const wq4_kv_pool* pool, const int32_t* seqs, const int32_t* new_lens, int n, void* stream);

/* Sequence children[i] becomes a copy of parents[i]: full pages are shared, a
 * last page that is not full is copied (its rows in use, in every layer) to a page
 * of the child's own, so that both can append.  What the child held is freed
 * first.  A parent may have many children.  Refused: an index out of range, a
 * child listed before, a child that is a parent in the list.  A child for whose
 * last page no free one is left stays empty (length 0). */
int wq4_kv_fork(const wq4_kv_pool* pool, const int32_t* parents, const int32_t* children, int n, void* stream);

/* Frees all pages of the listed sequences; their lengths become 0.  An index out
 * of range is refused; one listed twice is freed once. */
int wq4_kv_free(const wq4_kv_pool* pool, const int32_t* seqs, int n, void* stream);

/* Frees the pages of the listed sequences that their coming tokens do not see
 * under a window (>= 1) with n_sinks (>= 0) first tokens: those without a token t
 * < n_sinks or t > seq_lens - window.  Their entries become -1; lengths stay.
 * Refusals as for wq4_kv_free.  From then on the sequence is for wq4_window_attention
 * and wq4_prompt_attention under that window: wq4_paged_attention and wq4_decode_step
 * see the whole context and take its freed pages for ids outside the pool (bit 4). */
int wq4_kv_trim(const wq4_kv_pool* pool, const int32_t* seqs, int n, int window, int n_sinks, void* stream);

/* Moves the pages in use to the front of the pool: with m in use, the k-th one at
 * or behind page m moves to the k-th free one before it, in every layer, and
 * every table entry follows.  An entry that names a page without reference or
 * outside the pool becomes -1 and is flagged if it is at or behind m. */
int wq4_kv_compact(const wq4_kv_pool* pool, void* stream);

/* Copies page src[i] to page dst[i] in every layer (n up to num_pages; table and
 * references stay as they are).  Refused: a pair with an id outside the pool, with
 * a destination that is another's too, or with a source that is any pair's destination. */
int wq4_kv_copy_pages(const wq4_kv_pool* pool, const int32_t* src, const int32_t* dst, int n, void* stream);

/* ------------------------------------------------------------------------ */
/* Decode step with attention                                               */
/* ------------------------------------------------------------------------ */

/*
 * The attention of one decode step (Section 2.3: the compiled models run
 * PagedAttention and FlashAttention between their projections).  The paper
 * names no positional encoding; its models (Llama-3.1, Phi-3.5) rotate q and
 * k, and this library's reading of that rotation is: within each head the
 * adjacent pair (x_2i, x_2i+1) turns by pos * rope_theta^(-2i / head_dim),
 * computed in fp64 on the fp16 values and rounded once to fp16.
 *   layers     : HOST array of num_layers caches (device pointers inside),
 *                all with the table's n_kv_heads, head_dim 128 and one common
 *                page_size (a multiple of 16); page tables [batch][stride].
 *                Sequences of a batch must not map their new positions to
 *                the same cache row.  (One may map another's new position as
 *                a token that it has cached, as two consecutive tokens of one
 *                sequence do: it attends to the new key and value.)
 *   positions  : device int32 [batch]: the new token's place in its sequence
 *                (the number of tokens already cached).
 *   rope_theta : rotary base (> 1; Llama-3.x 500000, Phi-3.5 10000).
 *   scale      : attention score scale (> 0, normally 1/sqrt(head_dim)).
 */
typedef struct {
    const wq4_kv_cache* layers;
    const int32_t* positions;
    double rope_theta;
    float scale;
} wq4_decode_attn;

/* Workspace bytes (table->workspace_bytes) wq4_decode_step needs: the chain's
 * workspace plus the attention buffers (for batch 3-32 it includes
 * wq4_paged_attention's workspace, which depends on the current device).
 * 0 if the table is invalid or its heads are unsupported (head_dim != 128,
 * n_q_heads / n_kv_heads not a whole number <= 8). */
size_t wq4_decode_step_workspace_bytes(const wq4_layer_table* table);

/*
 * One decode step of every sequence of the batch: the chain of wq4_decode_chain
 * with the query-block stand-in replaced by attention.  For layer l and row b,
 * after the QKV projection:
 *   q = rope(qkv[:, :H]), k = rope(qkv[:, H:H + Hkv*128]), v = qkv[:, H + Hkv*128:]
 *   layers[l] gets k, v at position positions[b] (as wq4_kv_append)
 *   a = fp16( attention(q, layers[l], positions[b] + 1 tokens) )
 * and a is the O projection's input (o = r(a) W_o . a).  Batch 1-2 runs the
 * attention inside the persistent chain kernel (split over the GPU's blocks,
 * fp32 scores and softmax); batch 3-32 records wq4_paged_attention and a
 * rotation/append kernel into its CUDA graph.  Accuracy: rotated q and k
 * within one fp16 ulp of the exact rotation of the fp16 projection outputs;
 * a within the attention contract of wq4_paged_attention; the projections as
 * in wq4_decode_chain.  Device-side problems are flagged in the status word
 * (bit 5: a position or page id that makes the append impossible, nothing
 * written; bit 3: a length beyond the page table, clamped; bit 4: a page id
 * outside the pool, zeros read).  The plan is built at the first call (and
 * rebuilt when the table or this description changes) as for
 * wq4_decode_chain; table->workspace must hold
 * wq4_decode_step_workspace_bytes(table) bytes.
 * Returns WQ4_OK, WQ4_ERR_INVALID, WQ4_ERR_ALIGN, WQ4_ERR_UNSUPPORTED or
 * WQ4_ERR_CUDA.
 */
int wq4_decode_step(const wq4_layer_table* table, const wq4_decode_attn* attn, const uint16_t* x,
                    uint16_t* logits, void* stream);

/* The same step with HOST buffers (x_host fp16 [batch][hidden], logits_host
 * fp16 [batch][vocab]): copies x in, runs the step, copies the logits out and
 * synchronizes `stream`. */
int wq4_decode_step_host(const wq4_layer_table* table, const wq4_decode_attn* attn, const uint16_t* x_host,
                         uint16_t* logits_host, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WQ4_ATTN_H */
