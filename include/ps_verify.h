/*
 * ps_verify.h - C ABI of the steps that follow the parallel draft step in Algorithm 1:
 * building the draft token tree from the drafter's top-k output, what the target model needs
 * around its pass over that tree (its KV cache in 8 bits, the attention of the tree's rows over
 * it, its distributions from its logits), and the acceptance walk over the tree against those
 * distributions.  Same library as ps_draft.h
 * (libps_draft.so), same conventions: extern "C", plain pointers and sizes, int status
 * (ps_status of ps_draft.h: 0 = OK, negative = error), nothing is enqueued on an error,
 * no allocation, no host synchronisation, asynchronous on the given hipStream_t.
 * Pointers marked DEVICE are device memory owned by the caller, HOST ones are read before
 * the call returns.
 */
#ifndef PS_VERIFY_H
#define PS_VERIFY_H
#include <stdint.h>
#include "ps_draft.h"
#ifdef __cplusplus
extern "C" {
#endif

#define PS_TREE_MAX_NODES 64

/*
 * The shape of a draft tree (Algorithm 1: the tree N; Section 4.2): node 0 is the root (the
 * last token of the prefix), parent[0] = -1, and 0 <= parent[s] < s for every other node, so
 * a node's children follow it and are tried in ascending index.  A node at depth t >= 1
 * carries a token proposed by draft row t-1, i.e. by q(. | x_<n, [MASK]_1..t-1); rank[s] says
 * which of that row's top-k tokens (0 = most probable; rank[0] is ignored).  Both arrays are
 * HOST memory of n_nodes entries, 1 <= n_nodes <= PS_TREE_MAX_NODES, and are copied.
 */
typedef struct ps_tree_shape {
    int32_t n_nodes;
    const int32_t* parent;
    const int32_t* rank;
} ps_tree_shape;

/*
 * Tree construction (Algorithm 1, "Draft future token tree N"): tokens[b][s] =
 * top_ids[b][depth(s) - 1][rank[s]] for s >= 1 and -1 for the root.
 *   top_ids  DEVICE [batch][rows][topk] int32: ps_draft_step's output (rows = k+1 draft rows)
 *   tokens   DEVICE [batch][n_nodes] int32, written
 * Errors: PS_ERR_NULL; PS_ERR_SHAPE (batch < 1, a malformed tree, a depth beyond rows, a rank
 * outside [0, topk)); PS_ERR_DEVICE.
 */
PS_API int ps_tree_tokens(const ps_tree_shape* tree, int32_t batch, int32_t rows, int32_t topk,
                   const int32_t* top_ids, int32_t* tokens, void* stream);

/*
 * The acceptance walk of Algorithm 1 (its inner loops and the final draw), once per sequence,
 * in float64 on the float32 inputs.  Starting at the root with P = p[0]: the children s of
 * the current node are tried in ascending index; child s with token x = tokens[s] at depth t is
 * accepted when r[s] < min(1, P(x) / q[t-1](x)) (a proposal with q(x) = 0 counts as ratio 1);
 * then the walk moves to s and P = p[s].  A rejected child leaves P = the positive part of
 * P - q[t-1], divided by its sum.  When the current node has no child left to try, the last
 * token is drawn from P by inversion with r[0]: the number of token ids whose cumulative sum
 * of P (in id order) is <= r[0] * sum(P), at most vocab-1.
 *   tokens      DEVICE [batch][n_nodes] int32 (entry 0 ignored); a token outside [0, vocab)
 *               is treated as rejected and leaves P unchanged.  May be NULL when top_ids is
 *               given: node s then carries top_ids[b][depth(s) - 1][rank[s]], what
 *               ps_tree_tokens would have written (tree->rank is needed then)
 *   top_ids     DEVICE [batch][rows][topk] int32 or NULL; read only when tokens is NULL
 *   q           DEVICE [batch][rows][vocab] float32: the drafter's distributions
 *               (ps_draft_step's probs); rows >= the tree's depth
 *   p           DEVICE [batch][n_nodes][vocab] float32: the target's next-token distribution
 *               after the path to each node (entry 0: after the prefix alone)
 *   r           DEVICE [batch][n_nodes] float32 uniform numbers in [0, 1)
 *   n_accepted  DEVICE [batch] int32, written: accepted draft tokens
 *   path        DEVICE [batch][rows] int32, written: the accepted nodes, then -1
 *   out_tokens  DEVICE [batch][rows + 1] int32, written: the accepted tokens, the last drawn
 *               token, then -1
 *   workspace   DEVICE, optional (NULL = none): exchange memory for large vocabularies, at least
 *               ps_verify_workspace_bytes(batch, vocab) bytes, 256-byte aligned, owned by the caller,
 *               set to zero once before its first use and then left to the library (it may be
 *               used with any batch up to the one it was sized for)
 * vocab may be at most 262144 (1048576 when vocab % 4 == 0 and q and p are 16-byte aligned).
 * For vocab > 32768 (vocab % 4 == 0, aligned rows, batch * workgroups per sequence <= compute units) several
 * workgroups share a sequence and exchange their partial sums through device memory: the workspace if one is
 * given (calls with different workspaces may overlap in time), else, for batch <= 64, about 1 MB that belongs to
 * the library: calls that use the library's memory on one device must not overlap in time (calls on one stream
 * never do).  Without either, one workgroup walks each sequence (slower, same results).  Should the exchange
 * ever time out (it cannot while every workgroup of the launch gets a compute unit), n_accepted[b] = -2 marks
 * the sequence and its other outputs are undefined.
 * Errors: PS_ERR_NULL; PS_ERR_SHAPE (batch < 1, vocab < 1, a malformed tree, a depth beyond
 * rows; without tokens: topk < 1 or a rank outside [0, topk)); PS_ERR_UNSUPPORTED (vocab too
 * large); PS_ERR_DEVICE.
 */
typedef struct ps_verify_args {
    int32_t batch, rows, vocab;
    const int32_t* tokens;
    const float* q;
    const float* p;
    const float* r;
    int32_t* n_accepted;
    int32_t* path;
    int32_t* out_tokens;
    const int32_t* top_ids;
    int32_t topk;
    void* workspace;
    size_t workspace_bytes;
} ps_verify_args;
PS_API int ps_verify_walk(const ps_tree_shape* tree, const ps_verify_args* args, void* stream);

/* Bytes of exchange memory ps_verify_walk can use for this batch and vocabulary (0: none needed).  Host only. */
PS_API size_t ps_verify_workspace_bytes(int32_t batch, int32_t vocab);

/*
 * ps_verify_walk for callers that cannot allocate device memory or hand any in: code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation.  Same arguments (args->workspace is
 * ignored), same results, same kernels; it allocates nothing, on the host or on the device.  The exchange
 * memory that large vocabularies need is a fixed array inside the library, 1,065,472 bytes, of which every GPU
 * the library runs on holds its own copy until the process ends.  Limits (beyond them PS_ERR_UNSUPPORTED, never
 * a silent slower path): when vocab > 32768 with vocab % 4 == 0 and aligned rows, batch <= 64 and
 * batch * workgroups per sequence (ceil(vocab / 16384), at most 16) <= compute units.  All calls on one GPU
 * share that array, which keeps what the last call left (tagged with a per-sequence launch count that lives in
 * the array too, so old contents are never taken for data): calls of this function, and calls of ps_verify_walk
 * without a workspace, that overlap in time on one GPU race with each other; calls on one stream never overlap.
 * The first call on a device asks the runtime for the array's address: make it outside graph capture.
 */
PS_API int ps_verify_walk_static(const ps_tree_shape* tree, const ps_verify_args* args, void* stream);

/*
 * The target's KV cache in 8 bits.  The unit is a block: 32 consecutive positions of one kv head, whose keys share one scale and
 * whose values share another, a power of two each; an element is an e4m3 number (4 exponent and 3 fraction bits, largest 448, no
 * infinities, 0x7F and 0xFF are NaN) and stands for code * scale.  The scale is the least 2^e, e >= -100, with which the block's
 * largest finite magnitude is at most 448; Inf and NaN are stored as NaN and do not count for the scale.
 *   k_codes, v_codes  DEVICE [blocks][n_kv_heads][32 * head_dim], 16-byte aligned.  A block is laid out as the attention's matrix
 *                     instructions take it: dim j of position t (0..31) is byte
 *                       keys    ((j/32 * 2 + j/16 % 2) * 32 + t) * 16 + j % 16
 *                       values  ((j/32 * 2 + t/4 % 2) * 32 + j % 32) * 16 + t/8 * 4 + t % 4
 *   k_scale, v_scale  DEVICE [blocks][n_kv_heads] float32
 *   kv_offsets        HOST [batch+1], in positions as in ps_draft_step_args, multiples of 32: sequence b owns the blocks
 *                     kv_offsets[b] / 32 .. kv_offsets[b+1] / 32 - 1
 * Nothing has to be initialised: a block is valid from the first position of it that is written.  Supported: head_dim 64 or 128,
 * n_kv_heads up to 1024, batch 1..PS_CACHE_MAX_BATCH, kv_offsets below 2^36.
 * For this and all that follows: the stream and the device pointers belong to the current device, outputs overlap nothing else.
 */
#define PS_CACHE_BLOCK 32
#define PS_CACHE_MAX_BATCH 64
typedef struct ps_cache {
    int32_t n_kv_heads, head_dim;
    uint8_t* k_codes;
    uint8_t* v_codes;
    float* k_scale;
    float* v_scale;
    const int64_t* kv_offsets;
} ps_cache;

/*
 * Writes rows of keys (after the rotary embedding) and values behind the kv_len[b] positions that sequence b has.
 *   k_rows, v_rows  DEVICE [batch][rows][n_kv_heads][head_dim], dtype
 *   row_stride      elements between consecutive rows, >= n_kv_heads * head_dim (0 stands for that): rows of a fused projection
 *                   are taken where they are; sequence b starts rows * row_stride elements after sequence b - 1
 *   kv_len          HOST [batch]: valid positions before the call;  kv_len_dev  DEVICE [batch] or NULL: the lengths themselves,
 *                   kv_len then holds upper bounds (a length outside 0..kv_len[b] counts as the nearer of the two)
 *   n_seq           HOST [batch] or NULL: only the first n_seq[b] rows (0..rows) of sequence b are written
 *   n_accepted, path  DEVICE [batch] and [batch][path_rows] int32, both or neither, not with n_seq: what ps_verify_walk left.  The
 *                   rows are then a tree's, and node 0 and the accepted nodes path[b][0 .. n_accepted[b]-1] are written, in that
 *                   order.  A path ends before an entry outside [0, rows); nothing is written where n_accepted[b] < 0.
 *                   1 <= path_rows < PS_TREE_MAX_NODES (more nodes than that are on no path); n_accepted[b] counts as at most path_rows
 *   len_out         DEVICE [batch] int32 or NULL, written: the new lengths.  May be kv_len_dev itself
 * In a block that has positions already the scale only grows; when it does, the codes that are there are rounded again to the new
 * scale.  Positions of the last block written that are behind the new length become zero codes; blocks behind it stay as they are.
 * Calls that write the same sequence must not overlap in time, and no other call may read what one writes.
 * Errors: PS_ERR_NULL; PS_ERR_SHAPE; PS_ERR_OFFSETS (kv_offsets negative, decreasing or no multiples of 32); PS_ERR_KV_CAPACITY
 * (kv_len[b] and the most rows that can follow exceed the sequence's blocks); PS_ERR_UNSUPPORTED (head_dim, batch, alignment: rows
 * and row_stride to 4 bytes; kv_len[b] and the rows above 2^31 - 1); PS_ERR_DEVICE.
 */
typedef struct ps_cache_write_args {
    int32_t batch, rows, dtype;
    const ps_cache* cache;
    const void* k_rows;
    const void* v_rows;
    int64_t row_stride;
    const int32_t* kv_len;
    const int32_t* kv_len_dev;
    const int32_t* n_seq;
    const int32_t* n_accepted;
    const int32_t* path;
    int32_t path_rows;
    int32_t* len_out;
} ps_cache_write_args;
PS_API int ps_cache_write(const ps_cache_write_args* args, void* stream);

/*
 * Reads positions start[b] .. start[b] + n_seq[b] - 1 of every sequence back: code * scale in dtype (exact in both types;
 * what rounds to 2^128 when it is written is Inf).
 *   k_rows, v_rows  DEVICE [batch][rows][n_kv_heads][head_dim], dtype, written; one of them may be NULL; row_stride as above.
 *                   Rows from n_seq[b] on and what lies between rows stay as they were
 *   start           HOST [batch] or NULL: 0;  n_seq  HOST [batch] or NULL: rows
 * Errors: as ps_cache_write.
 */
typedef struct ps_cache_read_args {
    int32_t batch, rows, dtype;
    const ps_cache* cache;
    void* k_rows;
    void* v_rows;
    int64_t row_stride;
    const int32_t* start;
    const int32_t* n_seq;
} ps_cache_read_args;
PS_API int ps_cache_read(const ps_cache_read_args* args, void* stream);

/*
 * Tree attention over that cache (Section 3, token tree verification: each token attends to its ancestors only): row s of a
 * sequence, node s of the tree, attends to the sequence's kv_len[b] cached positions, to itself and to its ancestors among the rows;
 *   out = softmax(scale * q k^T) v per head, query head h uses kv head h / (n_heads / n_kv_heads).
 * A single token is the tree of one node, a chain of rows the tree with parent[s] = s - 1 (tree->rank is not used).
 *   q               DEVICE [batch][n_nodes][n_heads][head_dim], dtype, after the rotary embedding
 *   k_rows, v_rows  DEVICE [batch][n_nodes][n_kv_heads][head_dim], dtype: the rows' own keys and values, used as they are (they reach
 *                   the cache when the walk has accepted them).  Both NULL: the rows attend to the cached positions only
 *   q_stride, kv_stride  elements between consecutive rows of q, and of k_rows and v_rows (0: no gap), as row_stride above
 *   scale           0 stands for 1 / sqrt(head_dim); else 2^-20 .. 2^20
 *   out             DEVICE [batch][n_nodes][n_heads][head_dim], dtype, written
 *   lse             DEVICE [batch][n_nodes][n_heads] float32 or NULL, written: log of the sum of exp(scale * q k)
 *   kv_len, kv_len_dev  as for ps_cache_write.  Work is divided by kv_len: bounds far above the lengths leave part of the card idle
 *   workspace       DEVICE, ps_tree_attention_workspace_bytes bytes, 256-byte aligned (NULL where that is 0); its contents do not
 *                   matter before or after the call.  Calls that overlap in time need one each
 * A row that sees nothing (no cached position, no own rows) has out = 0 and lse = -Inf.  A value row that is hidden from a row does
 * not enter that row's result, whatever it holds; a key row that is not finite leaves the rows that see it undefined, no others.
 * Scores, softmax and sums are float32.  bf16: probabilities are rounded to bf16 before they are multiplied with the values.
 * Errors: PS_ERR_NULL; PS_ERR_SHAPE (also a malformed tree, a scale that is negative or not finite); PS_ERR_OFFSETS;
 * PS_ERR_KV_CAPACITY (kv_len[b] exceeds the sequence's blocks); PS_ERR_WORKSPACE; PS_ERR_UNSUPPORTED (head_dim, batch, alignment
 * to 4 bytes, n_heads > 1024, scale, kv_len above 2^30); PS_ERR_DEVICE.
 */
typedef struct ps_tree_attn_args {
    int32_t batch, n_heads, dtype;
    float scale;
    const ps_cache* cache;
    const void* q;
    const void* k_rows;
    const void* v_rows;
    int64_t q_stride, kv_stride;
    void* out;
    float* lse;
    const int32_t* kv_len;
    const int32_t* kv_len_dev;
    void* workspace;
    size_t workspace_bytes;
} ps_tree_attn_args;
PS_API int ps_tree_attention(const ps_tree_shape* tree, const ps_tree_attn_args* args, void* stream);

/* Bytes of device scratch that call needs (0: none, or bad arguments).  Host only; reads no device pointer. */
PS_API size_t ps_tree_attention_workspace_bytes(const ps_tree_shape* tree, const ps_tree_attn_args* args);

/*
 * The target's distributions, as ps_verify_walk takes them (p), from its logits, and draws from them.  Per row, with the settings of
 * its sequence:  x_i = logits_i / temperature, e_i = exp(x_i - max x); kept are the top_k largest logits (of equal ones those with
 * the lowest ids), of these, in the same order, the shortest prefix whose sum of e is at least top_p times the sum over all of them,
 * and of these the ones with e_i >= min_p; at least the first one is kept.  probs_i = e_i / (sum of the kept e), 0 for the others.
 *   logits       DEVICE [batch][rows][vocab], dtype
 *   temperature  DEVICE [batch] float32 or NULL: 1.  Not above 0 (or NaN): greedy, all mass on the first of the largest logits
 *   top_k        DEVICE [batch] int32 or NULL: all.  Below 1: all
 *   top_p        DEVICE [batch] float32 or NULL: 1.  1 and above, or NaN: all
 *   min_p        DEVICE [batch] float32 or NULL: 0.  Above 1 counts as 1; NaN as 0
 *   r            DEVICE [batch][rows] float32 uniform numbers in [0, 1); needed with ids
 *   probs        DEVICE [batch][rows][vocab] float32 or NULL, written
 *   ids          DEVICE [batch][rows] int32 or NULL, written: drawn by inversion, the number of ids whose cumulative sum of kept
 *                e (in id order) is <= r * sum, at most the last kept id
 *   id_probs     DEVICE [batch][rows] float32 or NULL (needs ids), written: the drawn id's probability
 *   workspace    DEVICE, ps_target_probs_workspace_bytes bytes, 256-byte aligned (NULL where that is 0); its contents do not matter
 *                before or after the call.  Calls that overlap in time need one each
 * How rows are divided among workgroups goes by the sizes and by which of top_k and top_p are given, not by what they hold.  Which tokens
 * are kept and which one is drawn is decided with exponentials and sums that carry more than 40 bits.  A logit of -Inf has no mass; a row without any mass (all -Inf) has probs 0 and id -1, a row with a NaN or +Inf has probs NaN and id -1, id_probs
 * likewise.  Supported: vocab <= 2^20, batch * rows <= 2^20.
 * Errors: PS_ERR_NULL (args, logits, ids without r, neither probs nor ids); PS_ERR_SHAPE; PS_ERR_WORKSPACE; PS_ERR_UNSUPPORTED
 * (sizes; alignment: logits to their type, everything else to 4 bytes); PS_ERR_DEVICE.
 */
typedef struct ps_target_probs_args {
    int32_t batch, rows, vocab, dtype;
    const void* logits;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* r;
    float* probs;
    int32_t* ids;
    float* id_probs;
    void* workspace;
    size_t workspace_bytes;
} ps_target_probs_args;
PS_API int ps_target_probs(const ps_target_probs_args* args, void* stream);

/* Bytes of device scratch that call needs (0: none, or bad arguments).  Host only; reads no device pointer. */
PS_API size_t ps_target_probs_workspace_bytes(const ps_target_probs_args* args);

#ifdef __cplusplus
}
#endif
#endif /* PS_VERIFY_H */
