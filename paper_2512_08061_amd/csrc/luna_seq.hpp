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

// The same in scalar registers (a sequence that the whole workgroup has: what is read from memory lies in vector registers, and a
// buffer whose address does is tried lane by lane).
__device__ __forceinline__ SeqPiece seq_uniform(SeqPiece p) {
  p.seq = __builtin_amdgcn_readfirstlane(p.seq);
  p.index = __builtin_amdgcn_readfirstlane(p.index);
  p.len = __builtin_amdgcn_readfirstlane(p.len);
  p.first = __builtin_amdgcn_readfirstlane((int)p.first);  // (at most 2^30)
  return p;
}

// The same number, of which the compiler knows nothing: what is worked out from it is worked out there, not once before a
// loop, where 100 such numbers and more would be written to memory and read back in every turn.
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
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

// The sequence of a rank by length, the longest first, of up to 64 sequences (the whole wave calls this with one rank); of more:
// of that number.
__device__ __forceinline__ int seq_by_length(const SeqSet& s, int rank) {
  if (s.count > kWave) return rank;
  const int lane = threadIdx.x % kWave, count = (int)s.count;
  const int mine = lane < count ? seq_of(s, lane).len : -1;
  int before = 0;
  for (int b = 0; b < count; ++b) {
    const int other = __builtin_amdgcn_readlane(mine, b);
    before += other > mine || (other == mine && b < lane);
  }
  return __builtin_ctzll(__ballot(lane < count && before == rank));
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
// softmax (luna_softmax*.hip, luna_paged_*.hip)
// ---------------------------------------------------------------------------

// luna_pages: token i of sequence b lies in row i % 2^shift of page table[b][i / 2^shift].  A page has at least 16 rows, so that
// 16 keys from a multiple of 16 on lie in one.
struct PageSet {
  const int32_t* table;  // [count][width]
  int64_t pool;
  int width, shift;
};
// The page of a token of a sequence (which has room for it), or -1 where the table holds none of the pool.
__host__ __device__ inline int page_of(const PageSet& p, int seq, int token) {
  const int page = p.table[(int64_t)seq * p.width + (token >> p.shift)];
  return page >= 0 && page < p.pool ? page : -1;
}

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
  PageSet pages;  // calls over pages: k.seq and v.seq are those of pages
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
// Over pages: the tile kernels, and the kernel for few rows of a key head (luna_paged_split.hip).
hipError_t launch_paged_tiles(Dt dt, const SoftmaxArgs& a, hipStream_t s);
// Workgroups of that kernel that share a key head's rows: in fp32 32 rows each (64 spilled, and one wave's products were the whole time
// of a short call: 2 tokens of 32 heads on one, 3 keys, d = 128, 44.0 and 23.9 us).  In bf16 one takes up to 64, though 33 and more of
// d = 128 spill 19 registers too: the cache is read once.
inline int64_t paged_row_groups(Dt dt, int64_t rows) { return dt == Dt::BF16 || rows < 1 ? 1 : (rows + 31) / 32; }
// In fp32 it takes more rows as well, where the room for keys is long beside the new tokens (else shares and their join cost more than
// the causal tiles: 90 tokens of 100 and 200 keys, 30.9 and 18.3 us) and the tiles of 64 rows of a head are too few for the device or
// at least half empty.  d = 128, us, tiles first: 70 tokens of caches of 4096 and 1999, 8 heads, 465 and 85; 64 tokens of 16 caches of
// 1500, 16 heads (256 tiles), 490 and 241; d = 64, 17 tokens of 12 caches of up to 6175, 32 heads on 2, 427 and 94.  With 512 full
// tiles of long keys the tiles lead: 1000 tokens of a cache of 8000, 32 heads on 8, 1308 and 1760.
inline bool paged_splits(Dt dt, const SeqSet& qs, int64_t H, int64_t Hk, int64_t room) {
  if (qs.offsets) return false;
  const int64_t rows = qs.rows * (H / Hk);
  if (rows <= kSplitRows) return true;
  if (dt == Dt::BF16 || room / 4 < qs.rows) return false;
  const int64_t tiles = qs.count * H * ((qs.rows + 63) / 64);
  return tiles < 512 || qs.count * Hk * paged_row_groups(dt, rows) <= tiles;  // (32 rows and 64)
}
// Tiles (bf16 with d = 64 and 128) whose keys are cut in shares as well: calls of so few tiles that the longest sequence alone would keep
// some of the device busy to the end.  Shares of the keys, in units of kPagedTileUnit; 0: no cut.
constexpr int kPagedTileUnit = 512;
inline int paged_tile_shares(Dt dt, const SeqSet& qs, int64_t H, int64_t Hk, int64_t d) {
  if (dt != Dt::BF16 || d < 64 || qs.offsets || paged_splits(dt, qs, H, Hk, 0)) return 0;
  const int64_t tiles = (qs.rows + 127) / 128;
  return qs.count * tiles * H > 512 ? 0 : (int)(512 / (tiles * H));
}
hipError_t launch_paged_tile_join(const SoftmaxArgs& a, int shares, hipStream_t s);
// Keys of a unit of work of that kernel, which a wave takes at a time, and the workgroups that share the units of a key
// head (room: of the sequences' rows of the table).
constexpr int paged_unit(Dt dt) { return dt == Dt::BF16 ? 64 : 32; }
int64_t paged_shares(Dt dt, int64_t count, int64_t room, int64_t Hk, int64_t rows);
hipError_t launch_paged_split(Dt dt, const SoftmaxArgs& a, hipStream_t s);

// The line of all sequences' units in equal shares: units of a share; the units u0 .. u1 - 1 of a sequence with `before` units
// before it that a share holds; the shares that hold units of a sequence; the number of a share's part of a sequence, below
// shares + count (from part to part of the line the share or the sequence grows, or both).
struct PagedUnits {
  int u0, u1;
};
// (at least `least` units: a share of fewer costs more than it saves)
constexpr int kPagedLeast = 4;  // of the kernel for few rows
__host__ __device__ inline int64_t paged_per(int64_t all, int shares, int least = kPagedLeast) {
  const int64_t per = (all + shares - 1) / shares;
  return per < least ? least : per;
}
__host__ __device__ inline PagedUnits paged_held(int64_t before, int units, int64_t per, int share, int64_t all) {
  const int64_t begin = share * per, end = begin + per < all ? begin + per : all;
  return PagedUnits{(int)(begin > before ? begin - before : 0), (int)(end - before < units ? end - before : units)};
}
__host__ __device__ inline PagedUnits paged_holders(int64_t before, int units, int64_t per) {  // (first, last; none: last = first - 1)
  const int first = (int)(before / per);
  return PagedUnits{first, units ? (int)((before + units - 1) / per) : first - 1};
}
__host__ __device__ inline int64_t paged_part(int share, int seq) { return (int64_t)share + seq; }

struct AppendArgs {
  SeqRows k, v, q, o;     // new rows, o: rotated queries; q.data null: no queries
  SeqRows kp, vp;         // pages
  SeqSet s;               // the new tokens
  PageSet pages;
  const int32_t* lens;    // [count], these tokens included
  const float* inv_freq;  // [rot / 2]
  int H, Hk, d, rot, interleaved;
};
hipError_t launch_append(Dt dt, const AppendArgs& a, hipStream_t s);
bool append_launchable(const SeqSet& s);

}  // namespace luna
