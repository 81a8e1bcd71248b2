// luna_seq.hpp -- sequences of different lengths: what the host and the kernels of the
// operators of luna_seq.h share (luna_decay*.hip, luna_softmax*.hip, luna_seq_api.cpp).
//
// Work over sequences is cut in pieces of equal length, numbered by slots that the host can
// count without knowing the lengths.  Equal and padded sequences have ceil(rows / piece)
// slots each.  Packed ones take slot floor(offsets[b] / piece) + b and the ones after it: a
// sequence's ceil(len / piece) pieces always fit before the next one's first slot, and
// floor(rows / piece) + count slots hold all of them.  The sequence of a slot is the last
// whose first slot is not behind it.
#pragma once

#include "luna_device.hpp"
#include "luna_kernels.hpp"

namespace luna {

struct SeqRows {  // luna_rows
  char* data;
  int64_t seq, head, row;
};

struct SeqSet {  // luna_seqs
  int64_t count, rows;
  const int32_t* offsets;
  const int32_t* lens;
};

inline int64_t seq_slots(const SeqSet& s, int64_t piece) {
  return s.offsets ? s.rows / piece + s.count : s.count * ((s.rows + piece - 1) / piece);
}

// States of pieces are numbered apart from the slots, so that short packed sequences take none: only sequences longer than a
// piece have them, a state per piece.  With u = offsets[b] / piece, one's first state is floor(u) + min(b, floor(u)).  The next
// such sequence starts len / piece > 1 pieces later or more and is a later one, so that its first state is at least
// floor(len / piece) + 1 >= ceil(len / piece) further; and with u + len / piece <= rows / piece no state reaches
// floor(rows / piece) + min(count, floor(rows / piece)).  Equal and padded sequences have theirs in the place of their slots.
__host__ __device__ inline int64_t seq_first_state(const SeqSet& s, int64_t b, int64_t first, int piece) {
  if (!s.offsets) return b * ((s.rows + piece - 1) / piece);
  const int u = (int)first / piece;  // (at most 2^30 rows)
  return u + (b < u ? b : u);
}
inline int64_t seq_states(const SeqSet& s, int piece) { return seq_first_state(s, s.count, s.rows, piece); }

// One piece of one sequence.
struct SeqPiece {
  int seq;      // -1: the slot holds no piece
  int index;    // piece of its sequence
  int len;      // rows of the sequence
  int64_t first;  // its first row in packed tensors, else 0
};

__device__ __forceinline__ int seq_clamp(int64_t x, int64_t lo, int64_t hi) {
  return (int)(x < lo ? lo : x > hi ? hi : x);
}

__device__ __forceinline__ SeqPiece seq_of(const SeqSet& s, int b) {
  SeqPiece p;
  p.seq = b;
  p.index = 0;
  p.first = 0;
  if (s.offsets) {
    p.first = seq_clamp(s.offsets[b], 0, s.rows);
    p.len = seq_clamp((int64_t)s.offsets[b + 1], p.first, s.rows) - (int)p.first;
  } else {
    p.len = s.lens ? seq_clamp(s.lens[b], 0, s.rows) : (int)s.rows;
  }
  return p;
}

// The last packed sequence b with holds(b, offsets[b]), which holds up to some sequence and no further; -1: none (the whole
// wave calls this).  64 guesses at a time: every 4096th, 64th and single sequence.  (One look at each 64 after the other
// took 24 ms for 16384 sequences of 8 tokens in 16 heads, of 1.6 ms for the same sequences without offsets.)
template <typename Holds>
__device__ __forceinline__ int seq_last(const SeqSet& s, Holds holds) {
  const int lane = threadIdx.x % kWave, count = (int)s.count;
  int below = 0, step = 1;  // sequences known to hold
  while (step * kWave < count) step *= kWave;
  for (; step > 0; step /= kWave) {
    const int b = below + step * (lane + 1) - 1;
    below += step * __popcll(__ballot(b < count && holds(b, seq_clamp(s.offsets[min(b, count)], 0, s.rows))));
  }
  return __builtin_amdgcn_readfirstlane(below - 1);
}

// The piece of a slot (the whole wave calls this with one slot).
__device__ __forceinline__ SeqPiece seq_piece(const SeqSet& s, int slot, int piece) {
  SeqPiece p;
  int first_slot;
  if (s.offsets) {
    p.seq = seq_last(s, [&](int b, int first) { return first / piece + b <= slot; });
    if (p.seq < 0) return p;
    p = seq_of(s, p.seq);
    first_slot = (int)(p.first / piece) + p.seq;
  } else {
    const int each = (int)((s.rows + piece - 1) / piece);
    p = seq_of(s, slot / each);
    first_slot = p.seq * each;
  }
  p.index = __builtin_amdgcn_readfirstlane(slot - first_slot);
  if (p.index < 0 || (int64_t)p.index * piece >= p.len) p.seq = -1;
  return p;
}

// The same with the longest work first, where a piece's work grows with its distance from the end of its
// sequence (late: from the start): all pieces at the largest distance, then those at the next, so that no long one
// begins when the others end.  Up to 64 sequences, one a lane; more fill the device one after the other.
__device__ __forceinline__ SeqPiece seq_piece_by_work(const SeqSet& s, int slot, int slots, int piece, bool late) {
  if (s.count > kWave) return seq_piece(s, late ? slots - 1 - slot : slot, piece);
  SeqPiece p;
  p.seq = -1;
  const int lane = threadIdx.x % kWave, count = (int)s.count;
  const int mine = lane < count ? (int)(((int64_t)seq_of(s, lane).len + piece - 1) / piece) : 0;  // pieces
  // the largest distance with more than `slot` pieces at it or beyond, from 64 guesses at a time
  int far = 0, step = 1;
  while (s.rows / piece >= (int64_t)step * kWave) step *= kWave;
  for (; step > 0; step /= kWave) {
    int beyond = 0;
    for (int b = 0; b < count; ++b) beyond += max(0, __builtin_amdgcn_readlane(mine, b) - (far + step * lane));
    const int most = __popcll(__ballot(beyond > slot));
    if (most == 0) return p;
    far += step * (most - 1);
  }
  for (int b = 0; b < count; ++b) slot -= max(0, __builtin_amdgcn_readlane(mine, b) - far - 1);
  const uint64_t have = __ballot(mine > far);
  const bool hit = mine > far && __popcll(have & (((uint64_t)1 << lane) - 1)) == slot;
  p = seq_of(s, __builtin_ctzll(__ballot(hit)));
  p.index = late ? far : __builtin_amdgcn_readlane(mine, p.seq) - 1 - far;
  return p;
}

// Address of row i of a sequence and head.
__device__ __forceinline__ char* seq_row(const SeqRows& r, const SeqPiece& p, bool packed, int head, int64_t i, int esz) {
  return r.data + (packed ? (p.first + i) * r.row + head * r.head : p.seq * r.seq + head * r.head + i * r.row) * esz;
}
// Index of row i among numbers per row.
__device__ __forceinline__ int64_t seq_num(const SeqSet& s, const SeqPiece& p, int H, int head, int64_t i) {
  return s.offsets ? head * s.rows + p.first + i : ((int64_t)p.seq * H + head) * s.rows + i;
}

// 2^x in one instruction (1 ulp; results below 2^-126 are 0).  Also where a result is not wanted: what
// follows a matrix product and precedes the first reads of its result holds no branch, not
// even around an exponential or a load.  (Where a short conditional block stood there, the
// compiler left out the wait states on the path around it, and the reads came too early.)
__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// x summed over the four lane groups of 16
__device__ __forceinline__ float groups_sum(float x) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// Decay factor's exponent: log_decay within [-1e30, 0], so that multiples of it stay defined (0 times it
// is 0), in base 2; NaN stays NaN.
__device__ __forceinline__ float decay_log2(float g) {
  g = g > 0.0f ? 0.0f : g < -1e30f ? -1e30f : g;
  return g * 1.44269504088896340736f;
}

// ---------------------------------------------------------------------------
// decay (luna_decay.hip, luna_decay_step.hip)
// ---------------------------------------------------------------------------

// How the sums are formed (luna_decay.hip): plain; with denominators; with one more key
// component that is given per row.
constexpr int kDecayPlain = 0, kDecayNorm = 1, kDecayAug = 2;

struct DecayArgs {
  SeqRows q, k, v, o;  // widths dk, dk, dv, dv
  SeqSet s;
  const float* log_decay;  // [H]
  int H, dk, dv;
  int piece, slots;        // tokens per piece (a multiple of 64), and slots of pieces (workgroups)
  int nstates;             // states (seq_states)
  int reverse;             // sums over later tokens instead of earlier ones
  int exact_state;         // the state to fp32 accuracy (it is returned)
  float* states;           // [nstates][H][decay_state_floats]: state before each piece; null: one piece per sequence
  int transposed;          // states: of k and v exchanged
  int guard;               // values that are not finite reach no earlier token
  float* S;                // [count][H][dk][dv] and z [count][H][dk], in and out, or null
  float* z;
  float* den;              // per row, out (kDecayNorm), or null
  const float* kw;         // per row: weight of the row as a key, or null
  const float* ka;         // per row: the key's further component (kDecayAug; null: 1)
  const float* qa;         // per row: the query's (null: 1)
  const float* ow;         // per row: factor of the output row, or null
  float scale, eps;
};
__host__ __device__ inline int64_t decay_state_floats(int dk, int dv) {
  return (int64_t)dk * dv + (dk > dv ? dk : dv);
}
bool decay_supported(int dk, int dv);
// Columns of v of a workgroup, and its threads (16 columns a wave; two waves where more than 128 features meet few columns).
constexpr int decay_columns(int dv) { return dv <= 64 ? 64 : 128; }
constexpr int decay_threads(int dk, int dv) { return 4 * decay_columns(dv) * (dk > 128 && dv <= 64 ? 2 : 1); }
// Workgroups of a pass.
inline int64_t decay_groups(int64_t slots, int64_t H, int dv) { return slots * H * ((dv + decay_columns(dv) - 1) / decay_columns(dv)); }
// What every piece but its sequence's last adds to the state, then the states before the pieces in their place.  (A row
// pass that adds up the pieces before its own by itself, without the second launch, waits for them one after the
// other: LUNA backward 256 -> 455 us.)
hipError_t launch_decay_states(Dt dt, int mode, const DecayArgs& a, hipStream_t s);
hipError_t launch_decay_scan(const DecayArgs& a, hipStream_t s);
hipError_t launch_decay_out(Dt dt, int mode, const DecayArgs& a, hipStream_t s);

// w = 1 / (den + eps) and wd = -dO.out per row
struct DecayWeightsArgs {
  SeqRows dO, out;
  SeqSet s;
  const float* den;
  float* w;
  float* delta;
  int H, d;
  float eps;
};
hipError_t launch_decay_weights(Dt dt, const DecayWeightsArgs& a, hipStream_t s);

struct DecayStepArgs {
  SeqRows q, k, v, o;
  const float* log_decay;
  int64_t count;
  int m, H, D, d, normalize;
  float scale, eps;
  float* S;
  float* z;
};
hipError_t launch_decay_step(Dt dt, const DecayStepArgs& a, hipStream_t s);

// ---------------------------------------------------------------------------
// softmax (luna_softmax*.hip)
// ---------------------------------------------------------------------------

struct SoftmaxArgs {
  SeqRows q, k, v, o;
  SeqSet qs, ks;
  int H, Hk, d;
  float scale;
  float* lse;  // per query row, out (forward: may be null) or in (backward)
  // backward
  SeqRows dO, dq, dk, dv;
  float* parts;  // few queries over long keys: [slots][Hk][rows][d + 2], see luna_softmax_split.hip;
                 // backward: [H] numbers per key row of 2 d floats, see softmax_head_parts
  float* delta;  // per query row: dO.out, written by the query pass and read by the key pass
};
// Query rows of a workgroup of the forward call and of the backward pass over queries, and key rows of one of the pass over
// keys: four waves of 32 or 16.
constexpr int softmax_tile(Dt dt, int64_t d) { return dt == Dt::BF16 && d >= 64 ? 128 : 64; }
hipError_t launch_softmax_fwd(Dt dt, const SoftmaxArgs& a, hipStream_t s);
// Few queries over long keys: m tokens of equal or padded sequences, up to 64 rows per key head, whose keys
// then share one read of the cache; cut in pieces of kSplitKeys keys.  (Packed queries, whose lengths the host does not see,
// and more rows take the tile kernels, a chain of all key blocks each.)
constexpr int kSplitKeys = 512, kSplitRows = 64;
inline bool softmax_splits(const SeqSet& qs, const SeqSet& ks, int64_t H, int64_t Hk) {
  return !qs.offsets && qs.rows * (H / Hk) <= kSplitRows && ks.rows > 128;
}
hipError_t launch_softmax_split(Dt dt, const SoftmaxArgs& a, hipStream_t s);
hipError_t launch_softmax_bwd(Dt dt, const SoftmaxArgs& a, hipStream_t s);

}  // namespace luna
