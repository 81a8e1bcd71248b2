/*
 * luna_paged.h -- softmax attention over a cache in pages on AMD Instinct MI355X (gfx950): new keys and
 * values into the pages, with the rotation of their positions on the way, and attention of new tokens over
 * them.  Part of libluna.so beside luna_seq.h, whose tensors (luna_rows), sequences (luna_seqs), numbers
 * per row and conventions hold here too.
 *
 * A pool of `pool` pages holds `rows` tokens each, of Hk heads; keys and values are luna_rows whose seq is the stride of a
 * page: token i of sequence b, head h lies at element
 *   p * seq + h * head + (i % rows) * row,  p = table[b * width + i / rows].
 * lens[b] counts the tokens of sequence b in the cache, those of the call included: the m new tokens of a sequence are its
 * last ones, with positions lens[b] - m .. lens[b] - 1.  Sequences may share pages that are only read.
 * rows is a power of two from 16 to 65536, width * rows at most 2^30.  The kernels read lens as
 * within [0, width * rows] where they read the cache, and no page outside of the pool: what a table entry outside of [0, pool)
 * stands for is not written, and seen by no row.  So other contents give other results, but no access outside the tensors.
 */
#ifndef LUNA_PAGED_H_
#define LUNA_PAGED_H_

#include "luna_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct luna_pages {
  int64_t pool, rows, width;
  const int32_t* table; /* device, [count][width] */
  const int32_t* lens;  /* device, [count] */
} luna_pages;

/*
 * Appends the new tokens' keys and values (K, V: Hk heads of width d in {32, 64, 128}, sequences as seqs says) to
 * the pages.  Of each key the first rot components are rotated by its position p: pairs of components turn by the angles
 * p * inv_freq[j], j = 0 .. rot / 2 - 1 (device, fp32; angles are formed in 64 bits),
 *   (x, y) -> (x cos - y sin, x sin + y cos),
 * components j and j + rot / 2 (interleaved 0) or 2 j and 2 j + 1 (interleaved 1).  rot is a multiple of 16 up to d; 0
 * rotates nothing (inv_freq NULL).  Q (may be NULL): the same tokens' queries, H heads, rotated alike into q_out, which may be Q
 * itself.  Positions below 0 (more new tokens than lens says) and from width * rows on are not appended.  Of two new
 * tokens at one place of a page each element there comes from one of them, not all from the same.  It needs no workspace.
 */
luna_status luna_paged_append(const luna_rows* K, const luna_rows* V, const luna_rows* Q, luna_dtype dtype,
                              const luna_seqs* seqs, const luna_pages* pages, int64_t H, int64_t Hk, int64_t d, int64_t rot,
                              const float* inv_freq, int32_t interleaved, const luna_rows* k_pages,
                              const luna_rows* v_pages, const luna_rows* q_out, void* stream);

/* Bytes of device workspace of luna_paged_fwd (as luna_seq_workspace_bytes; 0 where it needs none, and on invalid arguments,
 * with a reason in luna_last_error()). */
size_t luna_paged_workspace_bytes(luna_dtype dtype, const luna_seqs* seqs, const luna_pages* pages, int64_t H, int64_t Hk,
                                  int64_t d);

/*
 * Causal softmax attention as luna_softmax_fwd over the keys and values in the pages (those of the new tokens among them):
 * query i of a sequence's m sees the keys j <= i + lens[b] - m.  A row that sees none has out = 0 and lse = -infinity.
 * Of equal or padded query sequences with at most 64 query rows per key head (rows * H / Hk: the next tokens) the cached
 * keys of all sequences are shared out equally among the workgroups, whatever their lengths, each read once for all query
 * heads of a key head (LUNA_F32: for 32 of its rows).  So are those of LUNA_F32 calls of more rows whose tables have room for
 * four keys a new token and which make less than 512 tiles of 64 rows, or tiles that are at most half full.  All others take
 * the keys one block after the other for tiles of 128 query rows of a head (64: LUNA_F32 and d = 32); of equal or padded
 * LUNA_BF16 calls with d >= 64 and at most 512 tiles the keys are shared out as well.  Packed queries, whose lengths the host
 * does not see, always take such tiles, each with all keys of its sequence: next tokens are faster as [count][H][1][d].  Sums
 * are taken in a fixed order.  What is not finite is treated as luna_softmax_fwd does.
 */
luna_status luna_paged_fwd(const luna_rows* Q, const luna_rows* k_pages, const luna_rows* v_pages, luna_dtype dtype,
                           const luna_seqs* seqs, const luna_pages* pages, int64_t H, int64_t Hk, int64_t d, float scale,
                           const luna_rows* out, float* lse, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LUNA_PAGED_H_ */
