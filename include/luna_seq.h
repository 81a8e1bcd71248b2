/*
 * luna_seq.h -- causal attention over sequences of different lengths on AMD Instinct
 * MI355X (gfx950): linear attention whose weights decay by a factor of each head's own,
 * and softmax attention with grouped heads.  Part of libluna.so beside luna.h, whose
 * conventions (status codes, luna_last_error(), streams, caller-owned device memory and
 * workspaces, validation before anything is enqueued) hold here too.
 *
 * These are the two kinds of causal attention layer of a hybrid decoder: a converted model
 * keeps some softmax layers, eq. (1) of Section 2, beside linear ones, eq. (9) of
 * Section 3.1, here with the prefix sums of the streaming form discounted per token.
 *
 * Tensors are rows of `width` contiguous elements reached by strides (luna_rows); the
 * sequences that the rows belong to are described once (luna_seqs).  All row tensors of a
 * call share one element type (luna_dtype); numbers per row, states and statistics are
 * fp32.
 */
#ifndef LUNA_SEQ_H_
#define LUNA_SEQ_H_

#include "luna.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A tensor of rows.  Row i of sequence b, head h starts at element
 *   b * seq + h * head + i * row      (equal or padded sequences), or
 *   (offsets[b] + i) * row + h * head (packed sequences; seq is not read).
 * data is 16-byte aligned and every stride a multiple of 16 bytes; row is at least the
 * width and at most 2^20 elements.  head or seq may be 0 for inputs whose heads or
 * sequences share their rows.  An output overlaps no other tensor of the call.
 */
typedef struct luna_rows {
  void* data;
  int64_t seq, head, row;
} luna_rows;

/*
 * The sequences of a call, in one of three forms:
 *   offsets == NULL, lens == NULL  `count` sequences of `rows` rows each;
 *   lens (device, [count])         `count` sequences with room for `rows` rows of which the
 *                                  first lens[b] are used: a padded batch, or a cache;
 *   offsets (device, [count + 1])  packed: sequence b has rows offsets[b] .. offsets[b + 1] - 1
 *                                  of `rows` rows in all (offsets not decreasing).
 * A sequence may be empty.  Rows of no sequence (behind a length, before the first or behind
 * the last offset) are neither read nor written.  The kernels clamp what they read from offsets
 * and lens to [0, rows], so other contents give undefined results, but no access outside the
 * tensors.  1 <= count <= 65535, 0 <= rows <= 2^30
 * (2^30 rows in all where every sequence has its own), 1 <= H <= 65535, and no launch of a call may have
 * 2^32 threads or more: one has 256 to 512 per sequence, head and 64 tokens or more (luna_softmax_fwd of few queries over
 * long keys: 256 per 512 keys of a key head, and d per query row), and a call beyond that is refused (LUNA_ERR_UNSUPPORTED).
 * NaN and infinities.  In the forward calls what is not finite in a row's query, or in the keys and
 * values of tokens that the row sees, reaches that row alone: nothing comes from later tokens, other sequences or
 * other (key) heads, or from rows of no sequence.  In luna_decay_fwd a value that is not finite makes its column
 * NaN from its token on (in out, and in the state).  Gradients are defined for finite inputs: one that is not may reach every
 * gradient row of its own sequence and (key) head, and no other.
 */
typedef struct luna_seqs {
  int64_t count, rows;
  const int32_t* offsets;
  const int32_t* lens;
} luna_seqs;

/* Numbers per row (denominators, log-sums) are contiguous [count][H][rows], or [H][rows] for
 * packed sequences; entries of rows of no sequence are left as they were. */

/* Operation codes of luna_seq_workspace_bytes(). */
enum {
  LUNA_OP_DECAY_FWD = 0,
  LUNA_OP_DECAY_BWD = 1,
  LUNA_OP_SOFTMAX_FWD = 2,
  LUNA_OP_SOFTMAX_BWD = 3
};

/*
 * Bytes of device workspace of an operation (256-byte aligned; no initialisation; untouched
 * until the call's kernels have finished; 0 on invalid arguments).  Dq, Dv: widths of queries
 * and values (softmax: both d).  Hk: key heads (softmax; H otherwise).  keys: the key
 * sequences of softmax calls, NULL where they are the query ones.
 */
size_t luna_seq_workspace_bytes(int32_t op, luna_dtype dtype, const luna_seqs* seqs, const luna_seqs* keys, int64_t H,
                                int64_t Hk, int64_t Dq, int64_t Dv);

/*
 * Causal linear attention with a decay for each head, over whole sequences (prompts,
 * training), in chunks.  With f_h = exp(log_decay[h]) (log_decay fp32 device memory [H];
 * values above 0 count as 0, -infinity forgets everything at every token), per sequence and head
 *   S_i = f_h S_{i-1} + k_i v_i^T,   z_i = f_h z_{i-1} + k_i   (fp32, [D][d] and [D]),
 *   normalize 0: out_i = scale q_i^T S_i
 *   normalize 1: out_i = scale q_i^T S_i / (den_i + eps), den_i = scale q_i^T z_i.
 * Q, K: width D in {32, 64, 128, 256}; V, out: width d in {32, 64, 128}.  Queries and keys are
 * used as given: features of luna_featuremap or luna_featuremap_variant (normalize 1 needs
 * weights whose sums stay away from -eps: features that are not negative), or projections.
 * S [count][H][D][d], z [count][H][D] (z only with normalize 1): the state before the
 * first token, overwritten by the state after the last one (unchanged for an empty
 * sequence); S is 16-byte aligned; S == NULL starts from zero and returns no state.
 * den (normalize 1, may be NULL): denominators per row, without eps, which the backward
 * pass takes.
 * Precision: LUNA_F32 computes in fp32.  LUNA_BF16 takes products of the bf16 operands with fp32
 * accumulation; the weights of a chunk of 64 tokens (in two parts with normalize 1) and the state are
 * rounded to bf16 as operands of the products that form out, whose sums are fp32.  The state that the call
 * returns and den have fp32 accuracy for both types.
 */
luna_status luna_decay_fwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype,
                           const luna_seqs* seqs, int64_t H, int64_t D, int64_t d, const float* log_decay,
                           int32_t normalize, float scale, float eps, float* S, float* z, const luna_rows* out,
                           float* den, void* ws, size_t ws_bytes, void* stream);

/*
 * The same for the m next tokens of every sequence, token by token in fp32 from the state
 * (S, z), which is read and updated in place: the recurrent form for decoding.  Q, K, V, out
 * hold `count` sequences of m rows (packed and padded forms are not taken); count * H <= 2^19.
 * It needs no workspace.
 */
luna_status luna_decay_step(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype, int64_t count,
                            int64_t m, int64_t H, int64_t D, int64_t d, const float* log_decay, int32_t normalize,
                            float scale, float eps, float* S, float* z, const luna_rows* out, void* stream);

/*
 * Gradients of luna_decay_fwd from S == NULL: for dO = dL/dout writes dQ, dK (width D) and
 * dV (width d); log_decay gets none.  With normalize 1, out and den are what the forward call
 * wrote (out in the call's type); with normalize 0 they are not read and may be NULL.
 * Precision as in the forward call; the weights and their gradients are rounded to bf16 once as operands, dO.out
 * meets the sums before a chunk in parts (2^-17).
 */
luna_status luna_decay_bwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, const luna_rows* dO,
                           luna_dtype dtype, const luna_seqs* seqs, int64_t H, int64_t D, int64_t d,
                           const float* log_decay, int32_t normalize, float scale, float eps, const luna_rows* out,
                           const float* den, const luna_rows* dQ, const luna_rows* dK, const luna_rows* dV, void* ws,
                           size_t ws_bytes, void* stream);

/*
 * Causal softmax attention, eq. (1) of Section 2 with the causal mask, grouped heads: query
 * head h reads key head h / (H / Hk).  keys == NULL: the keys are the queries' own tokens.
 * Otherwise keys describes key sequences of their own (the same count), whose last rows
 * are the queries' tokens: query i of a sequence of Lq queries and Lk keys sees the keys
 *   j <= i + Lk - Lq;
 * a row that sees none has out = 0 and lse = -infinity.
 *   P_ij = exp(scale q_i.k_j - lse_i),  lse_i = ln sum_j exp(scale q_i.k_j),  out_i = sum_j P_ij v_j.
 * Q, K, V, out: width d in {32, 64, 128}; K and V have Hk heads (H a multiple of Hk).
 * lse (may be NULL): fp32 per query row, which the backward pass takes.
 * LUNA_BF16 rounds P to bf16 as an operand of the product with V; scores, maxima and
 * sums are fp32.
 * Calls of equal or padded query sequences with at most 64 query rows per key head (rows * H / Hk: the next tokens
 * over a cache) and room for more than 128 keys read the keys in pieces of 512 side by side, each once for all
 * query heads of a key head.  All others, among them packed queries and larger groups, take the keys one
 * block after the other for 128 query rows of a head (64: LUNA_F32 and d = 32), however few of these there are.
 */
luna_status luna_softmax_fwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype,
                             const luna_seqs* seqs, const luna_seqs* keys, int64_t H, int64_t Hk, int64_t d,
                             float scale, const luna_rows* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Gradients of luna_softmax_fwd: from its out and lse and dO = dL/dout writes dQ (H heads)
 * and dK, dV (Hk heads, summed over the query heads of each).  Sums are taken in a fixed
 * order: the same call gives the same bits.  Scores and lse are fp32, so a P_ij carries about
 * 2^-22 |score| of itself; it is never taken as more than 1.  (Scores from 2^31 on are outside
 * of what either call is made for.)
 */
luna_status luna_softmax_bwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, const luna_rows* out,
                             const float* lse, const luna_rows* dO, luna_dtype dtype, const luna_seqs* seqs,
                             const luna_seqs* keys, int64_t H, int64_t Hk, int64_t d, float scale, const luna_rows* dQ,
                             const luna_rows* dK, const luna_rows* dV, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LUNA_SEQ_H_ */
