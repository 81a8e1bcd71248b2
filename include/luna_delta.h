/*
 * luna_delta.h -- causal linear attention by the gated delta rule on AMD Instinct MI355X (gfx950):
 * chunked over prompts and in training, token by token in decoding, and its gradients.  Part of
 * libluna.so beside luna_seq.h, whose tensors (luna_rows), sequences (luna_seqs), numbers per row and
 * conventions hold here too.
 *
 * Where luna_decay_fwd only adds to its state, this layer first takes out what the state already answers
 * to a key: per sequence and value head, with a_t = exp(log_decay_t),
 *   u_t = beta_t (v_t - a_t S_{t-1}^T k_t),  S_t = a_t S_{t-1} + k_t u_t^T,  out_t = scale S_t^T q_t
 * (S fp32, [D][d]).  Q and K have Hk heads (H a multiple of Hk): value head h reads key head h / (H / Hk).
 * log_decay and beta are fp32 numbers per row and value head, contiguous [count][H][rows], or [H][rows] for packed
 * sequences; log decays above 0 count as 0, and below -128 as -128 (a factor of 0: the token forgets everything before
 * it).  The recurrence is stable, and meant to be used, where beta |k|^2 <= 2: keys of norm 1 and beta
 * in [0, 2].  Elsewhere its values may grow without bound; past the range of fp32 they are not defined.
 */
#ifndef LUNA_DELTA_H_
#define LUNA_DELTA_H_

#include "luna_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Operation codes of luna_delta_workspace_bytes(). */
enum {
  LUNA_OP_DELTA_FWD = 0,
  LUNA_OP_DELTA_BWD = 1
};

/*
 * Bytes of device workspace of an operation (as luna_seq_workspace_bytes; 0 where it needs none, which is the forward call in
 * LUNA_BF16, and on invalid arguments, with a reason in luna_last_error()).  It grows with the chunks of 64 tokens, of which packed
 * sequences count rows / 64 + count (each has one at least, however short) and others count * ceil(rows / 64).  Per chunk and value
 * head the gradients take 8 D d + 512 d + 50688 bytes in LUNA_BF16 and 8 D d + 512 d + 34304 in LUNA_F32, the forward call in
 * LUNA_F32 takes 34304: 247 KB with D = d = 128, 8.1 GB for 8 x 16 heads of 16384 tokens, 44.5 GB for 16 heads of 10000 packed
 * sequences of 8.  A batch that this is too much for is handed over in parts: sequences do not depend on one another.
 */
size_t luna_delta_workspace_bytes(int32_t op, luna_dtype dtype, const luna_seqs* seqs, int64_t H, int64_t Hk, int64_t D,
                                  int64_t d);

/*
 * The layer over whole sequences, in chunks of 64 tokens.  Q, K: Hk heads of width D; V, out: H heads of width d; D and d
 * in {32, 64, 128}.  S [count][H][D][d], 16-byte aligned: the state before the first token, overwritten by the state after
 * the last one (unchanged for an empty sequence); S == NULL starts from zero and returns no state.
 * A value that is not finite makes its column of out and S NaN from its token on; so does a key or a gate (log_decay
 * NaN, beta NaN or infinite) for all columns of the heads that read it; a query reaches its own row alone.  Nothing
 * comes from later tokens, other sequences or heads, or rows of no sequence.
 * Precision: LUNA_F32 computes in fp32.  LUNA_BF16 takes products of bf16 operands with fp32 accumulation, in which what is
 * not given in bf16 (the state, the chunk's corrections) counts in parts: to 2^-17 of each, and to 2^-24 with S, which
 * then has fp32 accuracy.  The weights q.k of a chunk are rounded to bf16 once.
 */
luna_status luna_delta_fwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype,
                           const luna_seqs* seqs, int64_t H, int64_t Hk, int64_t D, int64_t d, const float* log_decay,
                           const float* beta, float scale, float* S, const luna_rows* out, void* ws, size_t ws_bytes,
                           void* stream);

/*
 * The same for the m next tokens of every sequence, token by token in fp32 from the state S, which is read and updated in
 * place.  Q, K, V, out hold `count` sequences of m rows, log_decay and beta [count][H][m]; count * H <= 2^19.  It needs no
 * workspace.
 */
luna_status luna_delta_step(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype, int64_t count,
                            int64_t m, int64_t H, int64_t Hk, int64_t D, int64_t d, const float* log_decay,
                            const float* beta, float scale, float* S, const luna_rows* out, void* stream);

/*
 * Gradients of luna_delta_fwd from S == NULL: for dO = dL/dout writes dQ, dK (Hk heads, summed over the value heads of
 * each), dV, and per row and value head dlog_decay (0 where log_decay is above 0) and dbeta, laid out as the gates are.
 * Precision as in luna_delta_fwd with S: the gates' gradients have fp32 accuracy relative to the terms of their sums.
 * Sums are taken in a fixed order: the same call gives the same bits.  Gradients are defined for finite inputs: one that
 * is not may reach every gradient row of its own sequence and key head, and no other.
 */
luna_status luna_delta_bwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, const luna_rows* dO,
                           luna_dtype dtype, const luna_seqs* seqs, int64_t H, int64_t Hk, int64_t D, int64_t d,
                           const float* log_decay, const float* beta, float scale, const luna_rows* dQ,
                           const luna_rows* dK, const luna_rows* dV, float* dlog_decay, float* dbeta, void* ws,
                           size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LUNA_DELTA_H_ */
