/*
 * speccache.h -- C ABI of the paged KV cache around the verify step: what a
 * serving loop does with the cache that specverify.h reads.
 *
 * One request's life on the cache: its prompt comes in chunks (rows appended
 * to its pages, then attention of the chunk over everything cached so far),
 * each round appends its verify rows (a chain's, or a token tree's), verifies
 * them (spec_verify of specverify.h, on the same pools and block table) and
 * moves the accepted path's rows behind its context; requests are forked,
 * preempted (Sec. 3 of arXiv 2505.17074: a scheduler that switches between
 * them) and freed, and their pages with them.
 *
 * Conventions: those of specverify.h for streams, errors and argument checks
 * (every check runs on the host before any HIP call; on an error nothing is
 * enqueued and no output is touched), and
 *   - spec_cache_append, spec_cache_commit and spec_cache_copy_pages take no
 *     workspace and no staging: what the host knows travels in the kernels'
 *     arguments, so that a captured call holds all it needs.  A batch of more
 *     requests (or pages) than fit runs as several launches in order on the
 *     stream;
 *   - spec_chunk_attn stages its plan as spec_verify_attn does;
 *   - SPEC_ERR_WORKSPACE is also the answer where the host has no memory left
 *     for a plan or the bookkeeping;
 *   - nothing reads or writes a page outside the pools: page ids from the
 *     block table (device memory, the caller's contract) are clamped into
 *     [0, num_pages) where rows are read, and rows of a page id outside are
 *     not written.
 */
#ifndef SPECCACHE_H
#define SPECCACHE_H

#include "specverify.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A paged KV cache (device memory).
 *   num_layers    layers that k and v hold (>= 1), layer l's pools
 *                 layer_stride elements after layer l - 1's (ignored for one).
 *   k, v          [num_layers][num_pages, page_tokens, Hkv, d], strides
 *                 kv_stride_tok / kv_stride_head inside a page in elements
 *                 (a page spans page_tokens * kv_stride_tok elements, as in
 *                 spec_attn_args_t), last dim contiguous; rows 16-byte aligned.
 *   page_tokens   a positive multiple of 32.
 *   block_table   int32 [requests, block_stride]: request i's page ids at
 *                 block_table[i * block_stride + j], its logical row t being
 *                 row t % page_tokens of page block_table[i * block_stride +
 *                 t / page_tokens].  May be NULL for spec_cache_copy_pages.
 *   block_width   entries of a row that exist (1 .. block_stride; 0:
 *                 block_stride of them).  Lengths that need more are refused.
 */
typedef struct spec_cache {
  int32_t num_layers;
  int32_t num_kv_heads;
  int32_t head_dim;
  spec_dtype_t dtype;
  int32_t num_pages;
  int32_t page_tokens;
  void* k;
  void* v;
  int64_t layer_stride;
  int64_t kv_stride_tok;
  int64_t kv_stride_head;
  const int32_t* block_table;
  int32_t block_stride;
  int32_t block_width;
} spec_cache_t;

/*
 * The new tokens of a batch (host memory): request i has ctx_len[i] >= 0 rows
 * cached and new_len[i] >= 0 new ones, at its logical rows ctx_len[i] ..
 * ctx_len[i] + new_len[i] - 1.  Nq = sum new_len; request i's rows of every
 * packed array start at the running sum of new_len over requests < i.  A
 * request with new_len 0 takes no part.
 */
typedef struct spec_chunks {
  int32_t num_requests;
  int32_t pad0;
  const int32_t* ctx_len;
  const int32_t* new_len;
} spec_chunks_t;

/*
 * Attention of each request's new tokens over its paged cache (one layer).
 * New token j of request i sees the rows 0 .. ctx_len[i] + j of its request,
 * its own among them (the new rows are in the cache already:
 * spec_cache_append).
 *   layer      the layer of the cache that is read.
 *   q          [Nq, Hq, d] in the cache's dtype, strides in elements, last
 *              dim contiguous, 16-byte aligned rows.  Query head h reads KV
 *              head h / (Hq / Hkv).  scale <= 0 selects 1/sqrt(d).
 *   out        [Nq, Hq, d] contiguous, 16-byte aligned, in out_dtype:
 *              SPEC_BF16 or SPEC_F32.  For SPEC_F32 the probabilities
 *              enter the second product in three bf16 parts (off by 2^-24 of
 *              their value at most); for SPEC_BF16 in two (2^-16) where no
 *              request of the batch has more than 32 query rows a KV head
 *              (new_len Hq / Hkv), else in one (2^-8, as the output's own
 *              rounding).  Scores, maxima, sums and outputs accumulate in
 *              fp32 in all.  Rows past Nq are left as they are.
 *   d in {64, 128}; bf16 caches only (SPEC_ERR_UNSUPPORTED otherwise).
 * A value of K or V that a token does not see never reaches its output, NaN
 * and infinities included, whether it is a later token's row, a row behind
 * the request's end in its last page, or another request's page.
 * Where such values lie among keys that are read, the rows concerned are
 * computed a second time: a call takes up to about five times as long, or up
 * to 0.1 ms more where that is longer.  The sums over V are not normalised
 * before the last step and may reach 2^8 times the keys' number times V's
 * largest value, which has to stay in fp32's range.
 * Long key ranges are cut into pieces whose partial outputs a second kernel
 * joins, where the batch alone would leave compute units idle; the cut depends
 * on the lengths, the head counts and the device alone, and results are
 * deterministic.  out overlaps neither q nor the cache.
 * One token a request is decoding; spec_verify_attn with draft_len 0 computes
 * the same on one layer's pools (fp32 output).  This call is the one for
 * prompts, for decoding beside them and for decoding alone; spec_verify_attn
 * belongs to rounds with drafts, whose trees' masks and acceptance it knows.  One
 * token each, fp32 outputs, us here and there: 1 request over 1000 rows (32 / 8
 * heads, d = 128) 12 and 17, over 30000 38 and 35, 64 over 4000 183 and 184, 128
 * over 500 55 and 58, 32 over 2000 (32 / 32 heads) 169 and 178, 64 over 4000
 * (d = 64) 89 and 100.
 */
typedef struct spec_chunk_attn_args {
  int32_t num_q_heads;
  int32_t layer;
  float scale;
  spec_dtype_t out_dtype;
  const void* q;
  int64_t q_stride_tok;
  int64_t q_stride_head;
  void* out;
} spec_chunk_attn_args_t;

/* Workspace sizes for spec_chunk_attn (as spec_workspace_bytes). */
SPEC_API spec_status_t spec_chunk_workspace_bytes(const spec_chunks_t* chunks, const spec_cache_t* cache,
                                                  const spec_chunk_attn_args_t* args, size_t* device_bytes,
                                                  size_t* host_bytes);

SPEC_API spec_status_t spec_chunk_attn(const spec_chunks_t* chunks, const spec_cache_t* cache,
                                       const spec_chunk_attn_args_t* args, void* workspace, size_t workspace_bytes,
                                       void* host_staging, size_t host_staging_bytes, void* stream);

/*
 * New K/V rows into the cache's pages: row r of request i's new rows goes to
 * its logical row ctx_len[i] + r, in layers layer .. layer + num_layers - 1.
 *   k_new, v_new  [num_layers][Nq, Hkv, d] in the cache's dtype, strides in
 *                 elements (new_stride_layer ignored for one layer), last dim
 *                 contiguous, 16-byte aligned rows.  No row of them lies where
 *                 a row is written.
 * Two requests that name the same page (shared pages of a fork) must not
 * both append to it; spec_pages_resize sees to that.
 */
typedef struct spec_append_args {
  int32_t layer;
  int32_t num_layers;
  const void* k_new;
  const void* v_new;
  int64_t new_stride_layer;
  int64_t new_stride_tok;
  int64_t new_stride_head;
} spec_append_args_t;

SPEC_API spec_status_t spec_cache_append(const spec_chunks_t* chunks, const spec_cache_t* cache,
                                         const spec_append_args_t* args, void* stream);

/*
 * After a round: moves the rows of each request's accepted path behind its
 * context, in every layer of the cache.  Request i's verify rows sit at its
 * logical rows ctx_len[i] + node (as spec_verify_attn reads them); the path
 * from the root to accepted_node[i] (device memory: spec_accept_args_t's
 * output) at depth t goes to row ctx_len[i] + t.  The request then has
 * ctx_len[i] + accepted_len[i] + 1 valid rows; what the rows behind them hold
 * is unspecified.  Chains are in place already and nothing runs for them.  A
 * request whose accepted_node is not one of its nodes (-1: a sequential
 * sibling walk that gave up) keeps its rows as they are.
 */
SPEC_API spec_status_t spec_cache_commit(const spec_requests_t* req, const spec_cache_t* cache,
                                         const int32_t* accepted_node, void* stream);

/*
 * One page's copy: the first `tokens` rows (1 .. page_tokens) of page src to
 * the same rows of page dst.
 */
typedef struct spec_page_copy {
  int32_t src;
  int32_t dst;
  int32_t tokens;
} spec_page_copy_t;

/*
 * Copies pages (host list) in every layer of the cache, K and V.  No page may
 * be written twice, nor both read and written, in one call
 * (SPEC_ERR_INVALID_ARG): the copies run at the same time.
 */
SPEC_API spec_status_t spec_cache_copy_pages(const spec_cache_t* cache, const spec_page_copy_t* copies,
                                             int32_t num_copies, void* stream);

/*
 * Page bookkeeping (host only; no GPU call): which sequence holds which page
 * of a pool of num_pages pages of page_tokens rows.  Pages are shared by
 * forked sequences and counted.  A page is handed out lowest id first.  A
 * handle is used by one thread at a time.  Calls that fail change nothing.
 *
 *   spec_pages_open     a new, empty sequence (ids are reused lowest first).
 *   spec_pages_resize   the sequence has `tokens` rows from now on: pages are
 *                       added or given back.  Where rows are added behind a
 *                       partly filled page that a fork shares, the sequence
 *                       gets a page of its own instead, and *copy says what
 *                       has to be copied to it before the rows are written
 *                       (copy->tokens = 0: nothing).  SPEC_ERR_NO_PAGES when
 *                       the pool cannot hold it.
 *   spec_pages_fork     a new sequence with the same rows on the same pages.
 *   spec_pages_close    gives the sequence's pages back.
 *   spec_pages_table    its page ids, in order, into out[0 .. max); *count is
 *                       their number (SPEC_ERR_WORKSPACE if max is less).
 *   spec_pages_compact  moves the used pages with the highest ids to free
 *                       pages with the lowest, until the used ones are the
 *                       first of the pool: copies[0 .. *count) says which
 *                       (their number is at most half the pages;
 *                       SPEC_ERR_WORKSPACE if max is less than it).  The
 *                       tables hold the new ids from then on.
 *   spec_pages_free_count  free pages.
 */
typedef struct spec_pages spec_pages_t;

SPEC_API spec_status_t spec_pages_create(int32_t num_pages, int32_t page_tokens, spec_pages_t** out);
SPEC_API void spec_pages_destroy(spec_pages_t* pages);
SPEC_API spec_status_t spec_pages_open(spec_pages_t* pages, int32_t* sequence);
SPEC_API spec_status_t spec_pages_resize(spec_pages_t* pages, int32_t sequence, int32_t tokens,
                                         spec_page_copy_t* copy);
SPEC_API spec_status_t spec_pages_fork(spec_pages_t* pages, int32_t sequence, int32_t* child);
SPEC_API spec_status_t spec_pages_close(spec_pages_t* pages, int32_t sequence);
SPEC_API spec_status_t spec_pages_table(const spec_pages_t* pages, int32_t sequence, int32_t* out, int32_t max,
                                        int32_t* count);
SPEC_API spec_status_t spec_pages_compact(spec_pages_t* pages, spec_page_copy_t* copies, int32_t max,
                                          int32_t* count);
SPEC_API int32_t spec_pages_free_count(const spec_pages_t* pages);

#ifdef __cplusplus
}
#endif
#endif /* SPECCACHE_H */
