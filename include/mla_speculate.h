/*
 * mla_speculate.h -- C ABI of the speculative decode step of the low-bit MLA
 * library for AMD MI355X (gfx950), beside the decode calls of mla_lowbit.h.
 *
 * A drafting model proposes tokens behind a sequence, and the target model
 * looks at all of them in one step.  The step's calls:
 *
 *   1. the drafted tokens go into the paged cache behind the context, as any
 *      token does (mla_lowbit_quant_append, mla_lowbit_norm_rope_append, ...);
 *   2. mla_lowbit_tree_attn: their attention, in every layer;
 *   3. mla_verify_tree: which of them stay, and the next token, from the
 *      target's logits and given random numbers;
 *   4. mla_lowbit_commit: the cached rows of those that stay move up behind the
 *      context, in all layers.
 *
 * The conventions of mla_lowbit.h hold for every entry point: device buffers
 * of the current HIP device, owned by the caller; bf16 as uint16_t; work
 * enqueued on `stream`, no call synchronizes or allocates; arguments checked
 * on the host before any HIP call; its return codes.  A launch that would not
 * fit one dispatch is refused with MLA_ENOTSUP.  Device-resident values
 * (lengths, node ranges, masks, parents, page ids, tokens, paths, plans) are
 * preconditions; the kernels clamp every index that comes from them into its
 * buffer, or pass over it.  Every call can be captured into a graph, and none
 * needs a length on the host: a plan (split_tokens, split_indptr) made for
 * lengths that a sequence has not reached serves it too.  Positions count in 32
 * bits: a page table of more than 2^30 tokens, or a longer split, is refused with
 * MLA_ENOTSUP.  A workspace holds values only while its call runs; two calls that
 * may overlap need one each.
 *
 * Trees.  Sequence b has the nodes cu_nodes[b] .. cu_nodes[b+1]-1 of the
 * node-indexed arrays (device, int32 [B+1], non-decreasing from 0, the last at
 * most num_nodes), at most max_nodes <= 64 of them, and may have none.  Node i
 * below counts from the sequence's first.  Node 0 is the root: the last token
 * that is already part of the text, whose row is not yet in the cache; the
 * others are drafted behind it.  Node i's row is cached at position
 * ctx_lens[b] + i, whatever its depth in the tree (its rotation goes by its
 * depth: position ctx_lens[b] + depth).  A chain has parents[i] = i - 1.
 */
#ifndef MLA_SPECULATE_H
#define MLA_SPECULATE_H

#include "mla_lowbit.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Split size for mla_*_tree_attn over sequences of seq_lens tokens, drafted
 * ones included (host only; no HIP call): the multiple of 32 tokens, or 0
 * (unsplit), with the least estimated time of attention and merge.  The split
 * itself is mla_plan_splits's, and any size gives right results.
 *   seq_lens  host, int32 [B], each >= 1
 *   nodes     host, int32 [B], 0 .. max_nodes: of every sequence.  Without them
 *             (mla_tree_split_tokens) sequences of one length are taken to have
 *             max_nodes each, and in batches of several lengths an eighth of them
 *             to all: up to half more time where ragged contexts have equal trees.
 * Returns it, or -MLA_EINVAL / -MLA_ENOTSUP.
 */
int32_t mla_tree_split_tokens(const int32_t* seq_lens, int32_t B, int32_t max_nodes, int32_t H);
int32_t mla_tree_split_tokens_for(const int32_t* seq_lens, const int32_t* nodes, int32_t B, int32_t max_nodes, int32_t H);

/* Bytes of the workspace of a split call; -1 for a negative or too large size. */
int64_t mla_tree_workspace_bytes(int32_t num_splits, int32_t max_nodes, int32_t H);

/*
 * Attention of drafted tokens over the paged cache, absorbed form: as
 * mla_lowbit_decode_attn, with the queries of every node, for head h
 *   z_t = softmax_scale * (q_lat[i,h,:] . C_hat[t,:] + q_rope[i,h,:] . K_hat[t,:])
 *   out[i,h,:] = sum_t softmax(z)_t C_hat[t,:],   lse[i,h] = ln sum_t e^{z_t}
 * over the keys t < ctx_lens[b] and the keys t = ctx_lens[b] + j of the nodes j
 * whose bit is set in tree_mask[i].  (A node sees itself only if its own bit is
 * set.)  A row that sees no key gets 0 and -inf.  A key that a row does not see
 * has no part in the row, whatever its cached values; a row that sees a drafted
 * key with a channel that is not finite (as dequantized, in the low-bit
 * cache's fp16 or the BF16 cache's own values) is NaN.
 *   q_lat      device, bf16 [num_nodes][H][d_c];  q_rope device, bf16 [num_nodes][H][d_r]
 *   cache, num_pages, block_table, max_pages_per_seq  as for the decode
 *   ctx_lens   device, int32 [B]: tokens before the root, >= 0
 *   tree_mask  device, uint64 [num_nodes]: bit j, node j of the same sequence
 *   H          1 or more, max_nodes * H <= 2^20
 *   split_tokens  0: unsplit, else the splits of mla_plan_splits over the lengths
 *              with the nodes (split_indptr, num_splits; a sequence's splits past
 *              its length are passed over)
 *   out        device, bf16 [num_nodes][H][d_c];  lse device, fp32 [num_nodes][H] or NULL
 *   workspace  split only: at least mla_tree_workspace_bytes, 16-byte aligned
 * Rows of nodes from cu_nodes[B] on are neither read nor written.  Products and
 * weights as in the decode calls: fp16 operands over the low-bit cache, bf16
 * over the BF16 cache, fp32 sums, split partials in fp16 (not finite past its
 * range).  Scores of queries or context keys that are not finite, or past the
 * fp16 range over the low-bit cache: NaN or +inf makes the row NaN (out and lse),
 * split or not; a key of score -inf weighs nothing (0 times its values: NaN in a
 * channel that is not finite).  A call repeats itself bit for bit.  B = 0 or
 * num_nodes = 0 is a no-op.
 */
int mla_lowbit_tree_attn(const mla_cache_format* f, const uint16_t* q_lat, const uint16_t* q_rope,
                         const void* cache, int64_t num_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                         const int32_t* ctx_lens, const int32_t* cu_nodes, const uint64_t* tree_mask,
                         int32_t num_nodes, int32_t max_nodes, int32_t B, int32_t H, float softmax_scale,
                         int32_t split_tokens, const int32_t* split_indptr, int32_t num_splits,
                         uint16_t* out, float* lse, void* workspace, int64_t workspace_bytes, hipStream_t stream);
int mla_bf16_tree_attn(const mla_cache_format* f, const uint16_t* q_lat, const uint16_t* q_rope,
                       const void* cache, int64_t num_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                       const int32_t* ctx_lens, const int32_t* cu_nodes, const uint64_t* tree_mask,
                       int32_t num_nodes, int32_t max_nodes, int32_t B, int32_t H, float softmax_scale,
                       int32_t split_tokens, const int32_t* split_indptr, int32_t num_splits,
                       uint16_t* out, float* lse, void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* Bytes of mla_verify_tree's workspace; -1 for a negative or too large size. */
int64_t mla_verify_workspace_bytes(int32_t num_nodes, int32_t B, int32_t vocab);

/*
 * Verification of drafted tokens: the emitted tokens are distributed as the
 * target's own would be.  For every sequence, from the root down, with p the
 * softmax of the node's logits over the sequence's temperature (temperature 0:
 * all of p on the largest logit, the lowest index among equals):
 *   fixed drafts (draft_probs NULL): r = p; for the node's children in their
 *     order, child i with token x is taken if u_accept[i] * sum(r) < r(x), else
 *     r(x) = 0;
 *   drawn drafts: child i was drawn from q, the draft_probs row of its parent,
 *     independently of the node's other children (a token may come twice);
 *     r = p; child i is taken if u_accept[i] * q(x) < r(x), else r becomes
 *     max(r - q, 0) over its sum (r stays if that sum is 0).  With children drawn
 *     without replacement the emitted tokens would not be the target's: give those
 *     as fixed drafts, which may be chosen in any way that does not look at the
 *     random numbers;
 *   temperature 0, either way: a child is taken if its token is the largest
 *     logit's;
 * and with the child taken the walk goes on there.  With none taken the next
 * token is drawn from r: the first x with r(0) + .. + r(x) > u_draw[b] * sum(r)
 * (temperature 0: the largest logit's).  A walk that meets a row of logits with
 * a NaN, with +inf or with nothing above -inf ends there with the token -1.
 * Tokens outside [0, vocab) are never taken.  Where r has no weight left (the
 * fixed drafts name every token of p, or the last token's share is lost to
 * rounding), the token is drawn from p.
 * Everything is computed in fp64 from the logits as they are: errors of the
 * weights below 1e-12 (of those above 1e-300), and of sums below 1e-12 of the row's
 * whole sum, also of what rejections leave of it.  So an outcome differs from exact
 * arithmetic's only where a random number lies within 1e-12 / s of a border, s the
 * share of p that is left: 1 until a draft is rejected, and little after the
 * rejection of a token with nearly all of p, or of one drawn from a q next to p.
 *   logits       device, fp32 or bf16 (logits_type) [num_nodes][logits_stride], first vocab used
 *   vocab        1 .. 2^21
 *   draft_probs  device, fp32 [num_nodes][draft_stride], first vocab used, or NULL
 *   tokens       device, int32 [num_nodes] (a root's is not read)
 *   parents      device, int32 [num_nodes]: a node's parent in its sequence, below
 *                the node's own index (else the node is never reached; a root's is
 *                not read)
 *   temperature  device, fp32 [B], >= 0 (above 1e30: as 1e30), or NULL (1 for all)
 *   u_accept     device, fp32 [num_nodes], u_draw device, fp32 [B]: in [0, 1)
 *   path         device, int32 [B][max_nodes]: the nodes that stay, the root first, then -1
 *   out_tokens   device, int32 [B][max_nodes]: the emitted tokens (the taken children's,
 *                then the drawn one), then -1
 *   logprobs     device, fp32 [B][max_nodes] or NULL: ln p of the emitted tokens
 *                (0 at temperature 0), then 0
 *   keep         device, int32 [B]: nodes that stay, and tokens emitted (0 without nodes)
 *   workspace    at least mla_verify_workspace_bytes, 16-byte aligned
 * B = 0 is a no-op.
 */
enum { MLA_LOGITS_BF16 = 0, MLA_LOGITS_FP32 = 1 };
int mla_verify_tree(const void* logits, int32_t logits_type, int64_t logits_stride, int32_t vocab,
                    const float* draft_probs, int64_t draft_stride, const int32_t* tokens, const int32_t* parents,
                    const int32_t* cu_nodes, int32_t num_nodes, int32_t max_nodes, int32_t B,
                    const float* temperature, const float* u_accept, const float* u_draw,
                    int32_t* path, int32_t* out_tokens, float* logprobs, int32_t* keep,
                    void* workspace, int64_t workspace_bytes, hipStream_t stream);

/*
 * Commit: in each of num_layers caches, the row of position ctx_lens[b] + path[b][k]
 * goes to position ctx_lens[b] + k, for k < keep[b]; bytes move as they are.  All
 * rows are read before any of the sequence is written, so paths may be any.
 * Rows past the kept ones stay as they are.  new_lens[b] = ctx_lens[b] + keep[b].
 *   caches     device, [num_layers] pointers to caches of one format and size
 *              (256-byte aligned), none named twice
 *   path       device, int32 [B][max_nodes];  keep device, int32 [B]
 *   new_lens   device, int32 [B], or NULL; shares no memory with ctx_lens, path or keep
 * Entries outside [0, max_nodes), positions past the page table and page ids
 * outside the cache are passed over.  Sequences must own their pages from
 * position ctx_lens[b] on.  B = 0 or num_layers = 0 moves nothing.
 */
int mla_lowbit_commit(const mla_cache_format* f, void* const* caches, int32_t num_layers, int64_t num_pages,
                      const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                      const int32_t* path, const int32_t* keep, int32_t max_nodes, int32_t B, int32_t* new_lens,
                      hipStream_t stream);
int mla_bf16_commit(const mla_cache_format* f, void* const* caches, int32_t num_layers, int64_t num_pages,
                    const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                    const int32_t* path, const int32_t* keep, int32_t max_nodes, int32_t B, int32_t* new_lens,
                    hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MLA_SPECULATE_H */
