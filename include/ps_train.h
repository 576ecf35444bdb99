/*
 * ps_train.h - C ABI of group-wise parallel training: the layout's embeddings, its attention, the loss, and their gradients
 * (same library, libps_draft.so, same conventions as ps_draft.h: extern "C", plain pointers and sizes, int ps_status
 * results, nothing is enqueued on an argument error, no allocation, asynchronous on the given hipStream_t, which
 * has to belong to the current device, as every pointer has).
 *
 * Section 4.1, "Group-wise Parallel Training": a training sequence of T real tokens is laid out as T parallel
 * groups, each an input token followed by k [MASK] tokens,
 *     x_0 m_1 .. m_k | x_1 m_1 .. m_k | ... | x_{T-1} m_1 .. m_k            rows = T (k + 1),
 * and attention over this layout uses a customised causal mask under which every token ignores the [MASK]
 * tokens of previous groups (caption of Figure 3), with position indices adjusted so that training and
 * inference see the same thing (caption of Figure 2): row (group g, slot s) attends to the real tokens of
 * groups 0..g and to the [MASK] tokens 1..s of its own group, and stands at position g + s - what the same
 * token sees and where it stands in ps_draft_step when x_0..x_g are the prefix.
 */
#ifndef PS_TRAIN_H
#define PS_TRAIN_H
#include <stddef.h>
#include <stdint.h>
#include "ps_draft.h"
#ifdef __cplusplus
extern "C" {
#endif

/*
 * One forward pass of that attention for `seqs` independent sequences of the same length.
 *   q          DEVICE [seqs, rows, n_heads, head_dim], dtype, BEFORE the rotary embedding
 *   k, v       DEVICE [seqs, rows, n_kv_heads, head_dim], dtype (k before the rotary embedding)
 *   out        DEVICE [seqs, rows, n_heads, head_dim] float32, written: softmax(q k^T / sqrt(head_dim)) v per head
 *              under the mask above; query head h uses kv head h / (n_heads / n_kv_heads)
 *              (a key or value row that the mask hides from a row does not enter that row's result, whatever it
 *              holds: Inf and NaN in it stay with the rows that see it)
 *              (q, k, v and out need to be aligned to 4 bytes only)
 *   workspace  DEVICE, at least ps_group_attention_workspace_bytes(args) bytes, 256-byte aligned, owned by the
 *              caller: the rotary table and the rotated k (dtype: keys are rounded to the storage type after
 *              the rotary embedding, as the inference path caches them; queries are rotated in float32 on chip)
 * The rotary embedding (pairs (j, j + head_dim / 2), angle position * rope_base^(-2j / head_dim), computed in
 * double precision) is applied inside.  Supported: head_dim 64 or 128; k + 1 <= 16; n_heads a multiple of
 * n_kv_heads; dtype PS_F32 or PS_BF16; tokens + k <= 2^20; (k + 1) * n_kv_heads * head_dim <= 2^25.  Errors: PS_ERR_NULL, PS_ERR_SHAPE (a size < 1,
 * k < 0), PS_ERR_UNSUPPORTED, PS_ERR_WORKSPACE, PS_ERR_DEVICE.
 */
typedef struct ps_group_attn_args {
    int32_t seqs;       /* >= 1 */
    int32_t tokens;     /* T >= 1 real tokens per sequence */
    int32_t k;          /* [MASK] tokens per parallel group, 0 <= k <= 15 (0: ordinary causal attention) */
    int32_t n_heads, n_kv_heads, head_dim;
    int32_t dtype;      /* ps_dtype of q, k, v */
    float rope_base;
    const void* q;
    const void* k_;
    const void* v;
    float* out;
    void* workspace;
    size_t workspace_bytes;
} ps_group_attn_args;

/* Bytes of workspace ps_group_attention needs (0 if the arguments are invalid or unsupported).  Host only. */
PS_API size_t ps_group_attention_workspace_bytes(const ps_group_attn_args* args);

PS_API int ps_group_attention(const ps_group_attn_args* args, void* stream);

/*
 * The same forward pass for training: also writes what the backward pass needs,
 *   lse        DEVICE [seqs, rows, n_heads] float32: the logarithm of the row's sum of exp(q k^T / sqrt(head_dim)) over
 *              the keys it sees (natural logarithm), aligned to 4 bytes
 * out is bit for bit that of ps_group_attention; workspace as there.  Errors as there (lse NULL: PS_ERR_NULL).
 */
PS_API int ps_group_attention_lse(const ps_group_attn_args* args, float* lse, void* stream);

/*
 * The backward pass of that attention: the gradients of q, k and v (before the rotary embedding, as they were passed
 * in) from the gradient of out.  The probabilities are worked out again from q, k and lse; nothing of the size
 * rows x rows is kept.  The rounding of a rotated key to the storage type counts as the identity.
 *   q, k, v    DEVICE, as they were passed to ps_group_attention_lse
 *   out, lse   DEVICE, as it left them
 *   d_out      DEVICE [seqs, rows, n_heads, head_dim], dtype: gradient of out
 *   d_q        DEVICE [seqs, rows, n_heads, head_dim], dtype, written
 *   d_k, d_v   DEVICE [seqs, rows, n_kv_heads, head_dim], dtype, written: sums over the query heads that share the kv
 *              head and over all rows that see the key
 *   workspace  DEVICE, at least ps_group_attention_grad_workspace_bytes(args) bytes, 256-byte aligned, owned by the caller
 * All sums are held in float32 and added in an order that depends on the sizes alone: the same call gives the
 * same bits.  PS_BF16: probabilities and their gradients, P and dS, are rounded to bf16, once each, before the products that make the
 * gradients; relative to the gradients' 2-norm the error is 0.0024, where the rounding of the results alone leaves 0.0017.  What a row holds that the mask hides from another (Inf and NaN among it) does not enter the other's d_q,
 * and d_out, q and out of rows that do not see a key do not enter the key's d_k and d_v; where the mask lets Inf and NaN through, they
 * enter as the formulas have it (a probability times Inf is Inf, also one so small that it is taken for zero).  The inputs must not overlap the
 * outputs.  (q, k, v, out, lse, d_out and the gradients need to be aligned to 4 bytes only.)  Sizes and
 * errors are those of ps_group_attention; also PS_ERR_UNSUPPORTED for rows / 128 * n_heads >= 2^24 and for 2^23 or more
 * tiles of 64 real or up to 128 [MASK] keys over all sequences and kv heads.
 */
typedef struct ps_group_attn_grad_args {
    int32_t seqs, tokens, k;
    int32_t n_heads, n_kv_heads, head_dim;
    int32_t dtype;      /* ps_dtype of q, k, v, d_out and the gradients */
    float rope_base;
    const void* q;
    const void* k_;
    const void* v;
    const float* out;
    const float* lse;
    const void* d_out;
    void* d_q;
    void* d_k;
    void* d_v;
    void* workspace;
    size_t workspace_bytes;
} ps_group_attn_grad_args;

/* Bytes of workspace ps_group_attention_grad needs (0 if the arguments are invalid or unsupported).  Host only. */
PS_API size_t ps_group_attention_grad_workspace_bytes(const ps_group_attn_grad_args* args);

PS_API int ps_group_attention_grad(const ps_group_attn_grad_args* args, void* stream);

/*
 * The rows of the training layout from token ids (Section 4.3: the [MASK] tokens are added to the embedding layer):
 *   x[b, g (k + 1)] = scale * embed[token_ids[b, g]],   x[b, g (k + 1) + s] = scale * mask_emb[s - 1], s = 1..k
 * computed in float32, rounded once to dtype.
 *   token_ids  DEVICE [seqs, tokens] int32.  An id outside [0, vocab) (a padded position) gives a row of zeros.
 *   embed      DEVICE [vocab, hidden], dtype;  mask_emb  DEVICE [k, hidden], dtype (may be NULL if k == 0)
 *   x          DEVICE [seqs, rows, hidden], dtype, written; must not overlap the inputs
 * (all aligned to 4 bytes).  Supported: hidden a multiple of 32 (PS_BF16) or 16 (PS_F32) up to 2^16; k <= 15;
 * seqs * tokens <= 2^22; vocab <= 2^23.  Errors: PS_ERR_NULL, PS_ERR_SHAPE (a size < 1, k < 0, scale not finite), PS_ERR_UNSUPPORTED,
 * PS_ERR_DEVICE.
 */
typedef struct ps_group_embed_args {
    int32_t seqs, tokens, k;
    int32_t hidden, vocab;
    int32_t dtype;
    float scale;
    const int32_t* token_ids;
    const void* embed;
    const void* mask_emb;
    void* x;
} ps_group_embed_args;

PS_API int ps_group_embed(const ps_group_embed_args* args, void* stream);

/*
 * The gradients of both tables from the gradient of x:
 *   d_embed[v] = scale * (sum of d_x[b, g (k + 1)] over the positions with token_ids[b, g] == v), zeros for a v that none has
 *   d_mask[s - 1] = scale * (sum of d_x[b, g (k + 1) + s] over all b and g)
 *   d_x        DEVICE [seqs, rows, hidden], dtype
 *   d_embed    DEVICE [vocab, hidden], dtype, written whole; NULL: not wanted (a frozen table)
 *   d_mask     DEVICE [k, hidden], dtype, written; NULL: not wanted, or k == 0
 *   workspace  DEVICE, at least ps_group_embed_grad_workspace_bytes(args) bytes (which covers both outputs, whatever
 *              of them is NULL), 256-byte aligned, owned by the caller
 * Sums are held in float32, in an order that depends on the sizes and the token ids alone (positions are sorted by
 * token, equal tokens by position), and rounded once to dtype.  Positions with an id outside [0, vocab) enter d_mask
 * as the others do, and no row of d_embed.  Sizes and errors as ps_group_embed; also PS_ERR_WORKSPACE, and
 * PS_ERR_NULL where neither output is wanted.
 */
typedef struct ps_group_embed_grad_args {
    int32_t seqs, tokens, k;
    int32_t hidden, vocab;
    int32_t dtype;
    float scale;
    const int32_t* token_ids;
    const void* d_x;
    void* d_embed;
    void* d_mask;
    void* workspace;
    size_t workspace_bytes;
} ps_group_embed_grad_args;

/* Bytes of workspace ps_group_embed_grad needs (0 if the arguments are invalid or unsupported).  Host only. */
PS_API size_t ps_group_embed_grad_workspace_bytes(const ps_group_embed_grad_args* args);

PS_API int ps_group_embed_grad(const ps_group_embed_grad_args* args, void* stream);

/*
 * Cross entropy of rows against the LM head, which the drafter shares with the target, frozen (Section 4.3; Eq. 3 with a
 * weight for every row), and its gradient with respect to the rows:
 *   logits[i, v] = h[i] . w_lm[v]
 *   loss[i]      = weights[i] * (log(sum_v exp(logits[i, v])) - logits[i, targets[i]])
 *   d_hidden[i]  = weights[i] * (sum_v softmax(logits[i])[v] w_lm[v] - w_lm[targets[i]])     (the gradient of the losses' sum)
 * The logits are never kept: the vocabulary is gone through in pieces, whose size bounds the workspace.
 *   h          DEVICE [rows, hidden], dtype
 *   w_lm       DEVICE [vocab, hidden], dtype
 *   targets    DEVICE [rows] int32.  A row whose target lies outside [0, vocab) (the label -100 of an ignored position), or
 *              whose weight is 0, has loss 0 and a gradient of zeros, whatever its row of h holds.
 *   weights    DEVICE [rows] float32, or NULL: 1 for every row
 *   loss       DEVICE [rows] float32, written
 *   d_hidden   DEVICE [rows, hidden], dtype, written; NULL: the losses only (half of the work)
 *   workspace  DEVICE, at least ps_vocab_loss_workspace_bytes(args) bytes, 256-byte aligned, owned by the caller
 * A row's Inf and NaN stay with its own loss and gradient; a target's logit of Inf or NaN makes both NaN.  |weights| below 2^63.
 * Products and sums are held in float32 and added in an order that depends on the sizes alone; PS_BF16: the
 * exponentials are rounded to bf16 before they are multiplied with w_lm, and d_hidden once at the end.  A probability below 2^-62 of
 * the target's may be taken for zero.
 * A row with a logit more than some 99 above its target's is worked out by itself, by one workgroup that reads w_lm three times (once if
 * only the losses are wanted): exact, but slow (tens of milliseconds at vocab 32000, for one such row or for hundreds).
 * Supported: hidden a multiple of 32 (PS_BF16) or 16 (PS_F32) up to 2^16; vocab <= 2^23; rows <= 2^22.  (h, w_lm and d_hidden
 * aligned to 16 bytes, the others to 4.)  Errors: PS_ERR_NULL, PS_ERR_SHAPE (a size < 1, a dtype that is none),
 * PS_ERR_UNSUPPORTED (sizes, alignment), PS_ERR_WORKSPACE, PS_ERR_DEVICE.
 */
typedef struct ps_vocab_loss_args {
    int32_t rows, hidden, vocab;
    int32_t dtype;
    const void* h;
    const void* w_lm;
    const int32_t* targets;
    const float* weights;
    float* loss;
    void* d_hidden;
    void* workspace;
    size_t workspace_bytes;
} ps_vocab_loss_args;

/* Bytes of workspace ps_vocab_loss needs for these sizes, with d_hidden NULL or not as in the call (0 if the arguments
 * are invalid or unsupported).  Host only. */
PS_API size_t ps_vocab_loss_workspace_bytes(const ps_vocab_loss_args* args);

PS_API int ps_vocab_loss(const ps_vocab_loss_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PS_TRAIN_H */
