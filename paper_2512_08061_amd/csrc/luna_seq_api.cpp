// luna_seq_api.cpp -- host side of the C ABI declared in include/luna_seq.h: checks, the plan of
// a call and its workspace, launches on the caller's stream.
#include "luna_seq.h"

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "luna_error.hpp"
#include "luna_seq.hpp"

namespace {

using luna::set_error;

constexpr int64_t kMaxRows = (int64_t)1 << 30, kMaxRow = (int64_t)1 << 20;

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// A launch has fewer than 2^32 threads.
bool launchable(int64_t groups, int threads) { return groups < ((int64_t)1 << 32) / threads; }

luna::SeqRows rows_of(const luna_rows* r) {
  return r ? luna::SeqRows{static_cast<char*>(r->data), r->seq, r->head, r->row} : luna::SeqRows{};
}
luna::SeqSet set_of(const luna_seqs* s) { return luna::SeqSet{s->count, s->rows, s->offsets, s->lens}; }

luna_status check_seqs(const luna_seqs* s, const char* what) {
  char why[128];
  if (!s) {
    snprintf(why, sizeof why, "%s is NULL", what);
    return set_error(LUNA_ERR_INVALID_ARG, why);
  }
  if (s->count < 1 || s->rows < 0) {
    snprintf(why, sizeof why, "%s: count must be >= 1 and rows >= 0", what);
    return set_error(LUNA_ERR_INVALID_ARG, why);
  }
  if (s->offsets && s->lens) {
    snprintf(why, sizeof why, "%s: offsets and lens exclude each other", what);
    return set_error(LUNA_ERR_INVALID_ARG, why);
  }
  if (s->count > 65535 || s->rows > kMaxRows || (!s->offsets && s->count * s->rows > kMaxRows)) {
    snprintf(why, sizeof why, "%s: more than 65535 sequences or 2^30 rows", what);
    return set_error(LUNA_ERR_UNSUPPORTED, why);
  }
  return LUNA_OK;
}

// heads and sequences of an output must not share rows; those of an input may (stride 0)
luna_status check_rows(const luna_rows* r, const char* what, luna_dtype dt, const luna_seqs& s, int64_t heads, int64_t width,
                       bool output) {
  char why[160];
  const int64_t e = dt == LUNA_BF16 ? 8 : 4;  // elements of 16 bytes
  const char* bad = nullptr;
  if (!r || (!r->data && s.rows > 0)) bad = "is NULL";
  else if (((uintptr_t)r->data & 15) != 0) bad = "must be 16-byte aligned";
  else if (r->row < width) bad = "has rows closer than their width";
  else if (r->head < 0 || r->seq < 0) bad = "has a negative stride";
  else if (r->row % e || r->head % e || (!s.offsets && r->seq % e)) bad = "has strides that are no multiple of 16 bytes";
  else if (output && ((heads > 1 && r->head < width) || (!s.offsets && s.count > 1 && r->seq < width))) bad = "has rows that overlap";
  if (bad) {
    snprintf(why, sizeof why, "%s %s", what, bad);
    return set_error(LUNA_ERR_INVALID_ARG, why);
  }
  if (r->row > kMaxRow || r->head > ((int64_t)1 << 40) || r->seq > ((int64_t)1 << 40)) {
    snprintf(why, sizeof why, "%s: strides above 2^20 elements (rows) or 2^40", what);
    return set_error(LUNA_ERR_UNSUPPORTED, why);
  }
  return LUNA_OK;
}

luna_status check_ws(size_t need, const void* ws, size_t ws_bytes) {
  if (need == 0) return LUNA_OK;
  if (!ws || ((uintptr_t)ws & 255) != 0) return set_error(LUNA_ERR_INVALID_ARG, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < need) {
    char why[96];
    snprintf(why, sizeof why, "workspace holds %zu bytes, %zu are needed", ws_bytes, need);
    return set_error(LUNA_ERR_WORKSPACE, why);
  }
  return LUNA_OK;
}

luna_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return LUNA_OK;
  char why[160];
  snprintf(why, sizeof why, "%s: %s", what, hipGetErrorString(e));
  return set_error(LUNA_ERR_HIP, why);
}

luna::Dt type_of(luna_dtype dt) { return dt == LUNA_BF16 ? luna::Dt::BF16 : luna::Dt::F32; }
luna_status check_type(luna_dtype dt) {
  return dt == LUNA_F32 || dt == LUNA_BF16 ? LUNA_OK : set_error(LUNA_ERR_INVALID_ARG, "dtype must be LUNA_F32 or LUNA_BF16");
}

// ---------------------------------------------------------------------------
// decay
// ---------------------------------------------------------------------------

struct DecayPlan {
  int piece = 0, slots = 0, nstates = 0;
  bool many = false;  // some sequence may have more than one piece
  size_t states = 0, w = 0, delta = 0, total = 0;  // workspace offsets
};

// Tokens per piece.  A piece is a serial chain of chunks, so cutting sequences fills the device; but pieces cost a pass
// over the keys and values of all but each sequence's last one, and their states written, scanned and read.  Estimated
// from: a 64-token chunk about 4 us with 128 features and d = 128 in bf16, three times as much in fp32, one workgroup
// a compute unit (two with 64 features; the plain bf16 pass of 128 features and columns, which also runs two, is counted as
// one), and a sixth more while no second one fills its waits; 4.5 TB/s.  Measured, us a
// call by piece: 8 x 16 heads of 16384 tokens, D = d = 128, one 1070, 4096 683, 2048 726, 1024 783; backward of 2 x 16
// heads of 2048 tokens with 256 features 128 289, 256 214, 384 244, 512 222; fp32 backward of 4096 tokens in 12 heads, 64
// features, 64 114, 128 101, 256 118.  How lengths fall into pieces is on the device and not known here (six packed prompts
// with 256 features: 384 us by the estimate's 512, 353 by 576): packed sequences are taken as of their mean length, one of
// them as long as a piece.
luna_status plan_decay(luna_dtype dt, const luna_seqs& s, int64_t H, int64_t D, int64_t d, bool backward, bool normalize,
                       DecayPlan* p) {
  const int64_t per = s.rows, all = s.offsets ? s.rows : s.count * s.rows;
  const int64_t longest = ceil_div(per > 0 ? per : 1, 64) * 64;
  const luna::SeqSet set = set_of(&s);
  const double chunk = (1.5 + 1.5e-4 * (double)(D * d)) * (dt == LUNA_BF16 ? 1.0 : 3.0);
  const double state = (double)luna::decay_state_floats((int)D, (int)d) * 4;
  const int64_t room = D <= 64 ? 512 : 256;
  double best = 0.0;
  for (int64_t piece = longest; piece >= 64; piece = piece > 64 && piece < 128 ? 64 : piece / 128 * 64) {
    // sequences of the same length, or packed ones, with half a piece left over at the end of each
    const int64_t whole = s.offsets ? ceil_div(all, piece) : s.count * ceil_div(per, piece);
    const int64_t pieces = whole + (s.offsets ? s.count / 2 : 0), full = ceil_div(piece, 64);
    const double groups = (double)(pieces * H);
    const double mean = s.offsets ? std::min((double)full, ((double)all / 64 + (double)(s.count / 2)) / (double)pieces) : (double)full;
    const double chunks = (double)ceil_div(pieces * H, room) * mean + ((double)full - mean);
    const double one = chunks * chunk * (groups < 2 * room ? 1.17 : 1.0);
    const double cost = piece == longest ? one : 1.4 * one + 8.0 + 4.0 * (double)(whole * H) * state / 4.5e6;
    if (p->piece == 0 || cost < best) {
      best = cost;
      p->piece = (int)piece;
    }
  }
  p->many = per > p->piece;
  const int64_t slots = luna::seq_slots(set, p->piece);
  const int dk = (int)D, dv = (int)d;  // (the other way round: dQ and dK)
  if (!launchable(luna::decay_groups(slots, H, dv), luna::decay_threads(dk, dv)) ||
      (backward && !launchable(luna::decay_groups(slots, H, dk), luna::decay_threads(dv, dk))) ||
      (backward && normalize && !launchable(luna::seq_slots(set, 64), 256)))
    return set_error(LUNA_ERR_UNSUPPORTED, "too many pieces of sequences and heads");
  p->slots = (int)slots;
  size_t off = 0;
  auto take = [&](size_t& at, size_t bytes) {
    at = off;
    off = align256(off + bytes);
  };
  if (p->many) {
    p->nstates = (int)luna::seq_states(set, p->piece);
    take(p->states, (size_t)p->nstates * H * luna::decay_state_floats((int)D, (int)d) * 4);
  }
  if (backward && normalize) {
    take(p->w, (size_t)all * H * 4);
    take(p->delta, (size_t)all * H * 4);
  }
  p->total = off;
  return LUNA_OK;
}

luna_status check_decay(luna_dtype dt, int64_t H, int64_t D, int64_t d, const float* log_decay, int32_t normalize, float scale,
                        float eps) {
  luna_status st = check_type(dt);
  if (st != LUNA_OK) return st;
  if (H < 1) return set_error(LUNA_ERR_INVALID_ARG, "H must be >= 1");
  if (H > 65535) return set_error(LUNA_ERR_UNSUPPORTED, "H must be <= 65535");
  if (D < 1 || d < 1) return set_error(LUNA_ERR_INVALID_ARG, "D and d must be >= 1");
  if (D > 256 || d > 128 || !luna::decay_supported((int)D, (int)d))
    return set_error(LUNA_ERR_UNSUPPORTED, "D must be 32, 64, 128 or 256 and d 32, 64 or 128");
  if (!log_decay) return set_error(LUNA_ERR_INVALID_ARG, "log_decay is NULL");
  if (normalize != 0 && normalize != 1) return set_error(LUNA_ERR_INVALID_ARG, "normalize must be 0 or 1");
  if (!std::isfinite(scale)) return set_error(LUNA_ERR_INVALID_ARG, "scale must be finite");
  if (!(std::isfinite(eps) && eps >= 0.0f)) return set_error(LUNA_ERR_INVALID_ARG, "eps must be finite and >= 0");
  return LUNA_OK;
}

luna_status check_state(const float* S, const float* z, int32_t normalize) {
  if (((uintptr_t)S & 15) != 0) return set_error(LUNA_ERR_INVALID_ARG, "S must be 16-byte aligned");
  if ((S != nullptr && normalize) != (z != nullptr))
    return set_error(LUNA_ERR_INVALID_ARG, "z goes with S and normalize 1, and only with them");
  return LUNA_OK;
}

void set_plan(const DecayPlan& p, luna::DecayArgs& a, void* ws) {
  a.piece = p.piece;
  a.slots = p.slots;
  a.nstates = p.nstates;
  a.states = p.many ? reinterpret_cast<float*>(static_cast<char*>(ws) + p.states) : nullptr;
}
luna_status run_decay_states(luna::Dt dt, int mode, const luna::DecayArgs& a, hipStream_t s) {
  if (!a.states) return LUNA_OK;
  const luna_status st = hip_status(luna::launch_decay_states(dt, mode, a, s), "decay state launch");
  if (st != LUNA_OK) return st;
  return hip_status(luna::launch_decay_scan(a, s), "decay scan launch");
}
luna_status run_decay_rows(luna::Dt dt, int mode, const luna::DecayArgs& a, hipStream_t s) {
  return hip_status(luna::launch_decay_out(dt, mode, a, s), "decay launch");
}

// ---------------------------------------------------------------------------
// softmax
// ---------------------------------------------------------------------------

// Pairs of a query and a key that it sees.
double seen_pairs(double nq, double nk) { return nq <= nk ? nq * nk - nq * nq / 2 : nk * nk / 2; }

// Whether dK and dV are formed per query head, in fp32 parts that are added up.  Without parts a workgroup walks the queries
// of a key tile for every head of the group: the longest chain is group * n / 64 steps of about 2.1 us (d = 128; 1.35 with 64).
// Parts divide the chains by the group, down to the mean of all steps over 256 compute units.  They cost their bytes
// (written and read, 1.7 MB a us), or at least the sum's chain of 32 (16) rounds of loads per head of the group, and 8 us per
// workgroup and compute unit.  Of packed sequences one is taken as three times as long as the mean (by this estimate the pass
// then takes 1.04 times the better form's time in the mean of 750 random packings; 1.15 with all taken as equal, 1.57 with parts
// up to 1024 key tiles).  Measured, us of the call without and with parts, d = 128: 8192 tokens, 16 heads on 4 1482 and 1097;
// 32 heads on 4, 4096 tokens 1261 and 637, 1024 tokens 313 and 173, but 256 tokens 93 and 121, 16 x 512 tokens 259 and 459,
// 6 x 4096 3339 and 3780, 64 queries behind 16000 keys 598 and 915; packed, 8192 and 50 times 100 tokens 1526 and 1207 (taken
// without).  Parts hold the rows of 512 key tiles at most: 64 MiB (d = 128) times the query heads of a group.
bool softmax_head_parts(luna::Dt dt, const luna::SeqSet& qs, const luna::SeqSet& ks, int64_t H, int64_t Hk, int64_t d) {
  if (dt != luna::Dt::BF16 || d < 64 || H == Hk) return false;
  const double count = (double)qs.count, group = (double)(H / Hk), width = (double)d / 128, step = d == 64 ? 1.35 : 2.1;
  const auto all = [](const luna::SeqSet& s) { return (double)s.rows * (s.offsets ? 1.0 : (double)s.count); };
  const auto longest = [&](const luna::SeqSet& s) { return s.offsets ? std::min(3.0 / count, 1.0) * (double)s.rows : (double)s.rows; };
  const auto other = [&](const luna::SeqSet& s) { return s.count > 1 ? (all(s) - longest(s)) / (count - 1) : 0.0; };
  const double tiles = count * std::ceil(all(ks) / count / 128);
  const double pairs = seen_pairs(longest(qs), longest(ks)) + (count - 1) * seen_pairs(other(qs), other(ks));
  const double chain = group * std::min(longest(qs), longest(ks)) / 64 * step, mean = pairs / (128 * 64) * (double)H / 256 * step;
  const double bytes = all(ks) * (double)H * 2 * (double)d * 4;
  return tiles * (double)Hk <= 512 && chain - std::max(chain / group, mean) >
                                          std::max(bytes / 1.7e6, 11.5 * width * group) + 8.0 * tiles * (double)H / 256 + 6.0;
}

luna_status check_softmax(luna_dtype dt, const luna_seqs* seqs, const luna_seqs* keys, int64_t H, int64_t Hk, int64_t d,
                          float scale, bool backward) {
  luna_status st = check_type(dt);
  if (st == LUNA_OK) st = check_seqs(seqs, "seqs");
  if (st == LUNA_OK && keys) st = check_seqs(keys, "keys");
  if (st != LUNA_OK) return st;
  if (keys && keys->count != seqs->count) return set_error(LUNA_ERR_INVALID_ARG, "seqs and keys differ in count");
  if (H < 1 || Hk < 1 || H % Hk) return set_error(LUNA_ERR_INVALID_ARG, "H must be a positive multiple of Hk");
  if (H > 65535) return set_error(LUNA_ERR_UNSUPPORTED, "H must be <= 65535");
  if (d != 32 && d != 64 && d != 128) return set_error(LUNA_ERR_UNSUPPORTED, "d must be 32, 64 or 128");
  if (!std::isfinite(scale)) return set_error(LUNA_ERR_INVALID_ARG, "scale must be finite");
  const luna::SeqSet qs = set_of(seqs), ks = set_of(keys ? keys : seqs);
  const luna::Dt t = type_of(dt);
  const int tile = luna::softmax_tile(t, d);
  const int64_t qtiles = luna::seq_slots(qs, tile), ktiles = luna::seq_slots(ks, tile);
  bool fits;
  if (backward) {
    fits = launchable(qtiles * H, 256) &&
           launchable(ktiles * (softmax_head_parts(t, qs, ks, H, Hk, d) ? H : Hk), tile == 128 ? 512 : 256);
  } else if (luna::softmax_splits(qs, ks, H, Hk)) {
    fits = launchable(luna::seq_slots(ks, luna::kSplitKeys) * Hk, 256) && launchable(qs.count * H * qs.rows, (int)d);
  } else {
    fits = launchable(qtiles * H, 256);
  }
  return fits ? LUNA_OK : set_error(LUNA_ERR_UNSUPPORTED, "too many tiles of sequences and heads");
}

luna::SoftmaxArgs softmax_args(const luna_rows* Q, const luna_rows* K, const luna_rows* V, const luna_rows* out,
                               const luna_seqs* seqs, const luna_seqs* keys, int64_t H, int64_t Hk, int64_t d, float scale) {
  luna::SoftmaxArgs a{};
  a.q = rows_of(Q);
  a.k = rows_of(K);
  a.v = rows_of(V);
  a.o = rows_of(out);
  a.qs = set_of(seqs);
  a.ks = set_of(keys ? keys : seqs);
  a.H = (int)H;
  a.Hk = (int)Hk;
  a.d = (int)d;
  a.scale = scale;
  return a;
}

int64_t all_rows(const luna_seqs& s) { return s.offsets ? s.rows : s.count * s.rows; }

// bytes of the backward pass's dO.out per query row, and of the key rows' parts behind them
size_t delta_bytes(const luna_seqs* seqs, int64_t H) { return align256((size_t)all_rows(*seqs) * H * 4); }
size_t head_part_bytes(luna_dtype dt, const luna_seqs* seqs, const luna_seqs* keys, int64_t H, int64_t Hk, int64_t d) {
  const luna_seqs* ks = keys ? keys : seqs;
  if (!softmax_head_parts(type_of(dt), set_of(seqs), set_of(ks), H, Hk, d)) return 0;
  return align256((size_t)all_rows(*ks) * H * 2 * d * 4);
}

// bytes of the split call's partial rows, or 0 where the call is not split
size_t split_bytes(const luna_seqs* seqs, const luna_seqs* keys, int64_t H, int64_t Hk, int64_t d) {
  const luna::SeqSet qs = set_of(seqs), ks = set_of(keys ? keys : seqs);
  if (!luna::softmax_splits(qs, ks, H, Hk)) return 0;
  return align256((size_t)luna::seq_slots(ks, luna::kSplitKeys) * H * qs.rows * (d + 2) * 4);
}


}  // namespace

extern "C" {

size_t luna_seq_workspace_bytes(int32_t op, luna_dtype dtype, const luna_seqs* seqs, const luna_seqs* keys, int64_t H,
                                int64_t Hk, int64_t Dq, int64_t Dv) {
  luna::clear_error();
  if (op == LUNA_OP_DECAY_FWD || op == LUNA_OP_DECAY_BWD) {
    const float one = 1.0f;
    if (check_seqs(seqs, "seqs") != LUNA_OK || check_decay(dtype, H, Dq, Dv, &one, 1, 1.0f, 0.0f) != LUNA_OK) return 0;
    DecayPlan p;
    if (plan_decay(dtype, *seqs, H, Dq, Dv, op == LUNA_OP_DECAY_BWD, true, &p) != LUNA_OK) return 0;
    return p.total;
  }
  if (op == LUNA_OP_SOFTMAX_FWD || op == LUNA_OP_SOFTMAX_BWD) {
    if (check_softmax(dtype, seqs, keys, H, Hk, Dq, 1.0f, op == LUNA_OP_SOFTMAX_BWD) != LUNA_OK) return 0;
    if (Dv != Dq) {
      set_error(LUNA_ERR_INVALID_ARG, "Dq and Dv differ");
      return 0;
    }
    return op == LUNA_OP_SOFTMAX_BWD ? delta_bytes(seqs, H) + head_part_bytes(dtype, seqs, keys, H, Hk, Dq)
                                     : split_bytes(seqs, keys, H, Hk, Dq);
  }
  set_error(LUNA_ERR_INVALID_ARG, "unknown operation");
  return 0;
}

luna_status luna_decay_fwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype,
                           const luna_seqs* seqs, int64_t H, int64_t D, int64_t d, const float* log_decay,
                           int32_t normalize, float scale, float eps, float* S, float* z, const luna_rows* out,
                           float* den, void* ws, size_t ws_bytes, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_decay(dtype, H, D, d, log_decay, normalize, scale, eps)) != LUNA_OK) return st;
  if ((st = check_seqs(seqs, "seqs")) != LUNA_OK) return st;
  if ((st = check_state(S, z, normalize)) != LUNA_OK) return st;
  if (den && !normalize) return set_error(LUNA_ERR_INVALID_ARG, "den goes with normalize 1");
  if ((st = check_rows(Q, "Q", dtype, *seqs, H, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(K, "K", dtype, *seqs, H, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(out, "out", dtype, *seqs, H, d, true)) != LUNA_OK) return st;
  DecayPlan p;
  if ((st = plan_decay(dtype, *seqs, H, D, d, false, normalize, &p)) != LUNA_OK) return st;
  if ((st = check_ws(p.total, ws, ws_bytes)) != LUNA_OK) return st;
  if (seqs->rows == 0) return LUNA_OK;
  luna::DecayArgs a{};
  a.q = rows_of(Q);
  a.k = rows_of(K);
  a.v = rows_of(V);
  a.o = rows_of(out);
  a.s = set_of(seqs);
  a.log_decay = log_decay;
  a.H = (int)H;
  a.dk = (int)D;
  a.dv = (int)d;
  a.S = S;
  a.z = z;
  a.exact_state = S != nullptr;
  a.guard = 1;
  a.den = den;
  a.scale = scale;
  a.eps = eps;
  const int mode = normalize ? luna::kDecayNorm : luna::kDecayPlain;
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  set_plan(p, a, ws);
  if ((st = run_decay_states(type_of(dtype), mode, a, hs)) != LUNA_OK) return st;
  return run_decay_rows(type_of(dtype), mode, a, hs);
}

luna_status luna_decay_step(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype, int64_t count,
                            int64_t m, int64_t H, int64_t D, int64_t d, const float* log_decay, int32_t normalize,
                            float scale, float eps, float* S, float* z, const luna_rows* out, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_decay(dtype, H, D, d, log_decay, normalize, scale, eps)) != LUNA_OK) return st;
  const luna_seqs seqs{count, m, nullptr, nullptr};
  if (m < 1) return set_error(LUNA_ERR_INVALID_ARG, "m must be >= 1");
  if ((st = check_seqs(&seqs, "the tokens")) != LUNA_OK) return st;
  if (!S) return set_error(LUNA_ERR_INVALID_ARG, "S is NULL");
  if ((st = check_state(S, z, normalize)) != LUNA_OK) return st;
  if ((st = check_rows(Q, "Q", dtype, seqs, H, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(K, "K", dtype, seqs, H, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(out, "out", dtype, seqs, H, d, true)) != LUNA_OK) return st;
  if (count * H * 4 > (int64_t)1 << 21) return set_error(LUNA_ERR_UNSUPPORTED, "count * H must be <= 2^19");
  luna::DecayStepArgs a{};
  a.q = rows_of(Q);
  a.k = rows_of(K);
  a.v = rows_of(V);
  a.o = rows_of(out);
  a.log_decay = log_decay;
  a.count = count;
  a.m = (int)m;
  a.H = (int)H;
  a.D = (int)D;
  a.d = (int)d;
  a.normalize = normalize;
  a.scale = scale;
  a.eps = eps;
  a.S = S;
  a.z = z;
  return hip_status(luna::launch_decay_step(type_of(dtype), a, reinterpret_cast<hipStream_t>(stream)), "decay step launch");
}

luna_status luna_decay_bwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, const luna_rows* dO,
                           luna_dtype dtype, const luna_seqs* seqs, int64_t H, int64_t D, int64_t d,
                           const float* log_decay, int32_t normalize, float scale, float eps, const luna_rows* out,
                           const float* den, const luna_rows* dQ, const luna_rows* dK, const luna_rows* dV, void* ws,
                           size_t ws_bytes, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_decay(dtype, H, D, d, log_decay, normalize, scale, eps)) != LUNA_OK) return st;
  if ((st = check_seqs(seqs, "seqs")) != LUNA_OK) return st;
  if (normalize && !den) return set_error(LUNA_ERR_INVALID_ARG, "den is NULL");
  if ((st = check_rows(Q, "Q", dtype, *seqs, H, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(K, "K", dtype, *seqs, H, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(dO, "dO", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if (normalize && (st = check_rows(out, "out", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(dQ, "dQ", dtype, *seqs, H, D, true)) != LUNA_OK) return st;
  if ((st = check_rows(dK, "dK", dtype, *seqs, H, D, true)) != LUNA_OK) return st;
  if ((st = check_rows(dV, "dV", dtype, *seqs, H, d, true)) != LUNA_OK) return st;
  DecayPlan p;
  if ((st = plan_decay(dtype, *seqs, H, D, d, true, normalize, &p)) != LUNA_OK) return st;
  if ((st = check_ws(p.total, ws, ws_bytes)) != LUNA_OK) return st;
  if (seqs->rows == 0) return LUNA_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const luna::Dt dt = type_of(dtype);
  float* w = nullptr;
  float* delta = nullptr;
  if (normalize) {
    w = reinterpret_cast<float*>(static_cast<char*>(ws) + p.w);
    delta = reinterpret_cast<float*>(static_cast<char*>(ws) + p.delta);
    luna::DecayWeightsArgs r{rows_of(dO), rows_of(out), set_of(seqs), den, w, delta, (int)H, (int)d, eps};
    if ((st = hip_status(luna::launch_decay_weights(dt, r, s), "row weight launch")) != LUNA_OK) return st;
  }
  luna::DecayArgs a{};
  a.s = set_of(seqs);
  a.log_decay = log_decay;
  a.H = (int)H;
  a.scale = scale;
  set_plan(p, a, ws);
  const int mode = normalize ? luna::kDecayAug : luna::kDecayPlain;
  // dQ: dO against V, with K as values
  a.q = rows_of(dO);
  a.k = rows_of(V);
  a.v = rows_of(K);
  a.o = rows_of(dQ);
  a.dk = (int)d;
  a.dv = (int)D;
  a.qa = delta;
  a.ow = w;
  if ((st = run_decay_states(dt, mode, a, s)) != LUNA_OK) return st;
  if ((st = run_decay_rows(dt, mode, a, s)) != LUNA_OK) return st;
  // over later tokens: dV, K against Q with dO as values (whose states, and z of weights delta, are dK's, too)
  a.reverse = 1;
  a.q = rows_of(K);
  a.k = rows_of(Q);
  a.v = rows_of(dO);
  a.o = rows_of(dV);
  a.dk = (int)D;
  a.dv = (int)d;
  a.qa = nullptr;
  a.ka = delta;
  a.kw = w;
  a.ow = nullptr;
  if ((st = run_decay_states(dt, normalize ? luna::kDecayNorm : luna::kDecayPlain, a, s)) != LUNA_OK) return st;
  if ((st = run_decay_rows(dt, luna::kDecayPlain, a, s)) != LUNA_OK) return st;
  // dK: V against dO, with Q as values
  a.q = rows_of(V);
  a.k = rows_of(dO);
  a.v = rows_of(Q);
  a.o = rows_of(dK);
  a.dk = (int)d;
  a.dv = (int)D;
  a.transposed = 1;
  return run_decay_rows(dt, mode, a, s);
}

luna_status luna_softmax_fwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype,
                             const luna_seqs* seqs, const luna_seqs* keys, int64_t H, int64_t Hk, int64_t d,
                             float scale, const luna_rows* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_softmax(dtype, seqs, keys, H, Hk, d, scale, false)) != LUNA_OK) return st;
  const luna_seqs& ks = keys ? *keys : *seqs;
  if ((st = check_rows(Q, "Q", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(K, "K", dtype, ks, Hk, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, ks, Hk, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(out, "out", dtype, *seqs, H, d, true)) != LUNA_OK) return st;
  const size_t need = split_bytes(seqs, keys, H, Hk, d);
  if ((st = check_ws(need, ws, ws_bytes)) != LUNA_OK) return st;
  if (seqs->rows == 0) return LUNA_OK;
  luna::SoftmaxArgs a = softmax_args(Q, K, V, out, seqs, keys, H, Hk, d, scale);
  a.lse = lse;
  if (need) {
    a.parts = static_cast<float*>(ws);
    return hip_status(luna::launch_softmax_split(type_of(dtype), a, reinterpret_cast<hipStream_t>(stream)), "split softmax launch");
  }
  return hip_status(luna::launch_softmax_fwd(type_of(dtype), a, reinterpret_cast<hipStream_t>(stream)), "softmax launch");
}

luna_status luna_softmax_bwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, const luna_rows* out,
                             const float* lse, const luna_rows* dO, luna_dtype dtype, const luna_seqs* seqs,
                             const luna_seqs* keys, int64_t H, int64_t Hk, int64_t d, float scale, const luna_rows* dQ,
                             const luna_rows* dK, const luna_rows* dV, void* ws, size_t ws_bytes, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_softmax(dtype, seqs, keys, H, Hk, d, scale, true)) != LUNA_OK) return st;
  const luna_seqs& ks = keys ? *keys : *seqs;
  if (!lse) return set_error(LUNA_ERR_INVALID_ARG, "lse is NULL");
  if ((st = check_rows(Q, "Q", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(K, "K", dtype, ks, Hk, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, ks, Hk, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(out, "out", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(dO, "dO", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(dQ, "dQ", dtype, *seqs, H, d, true)) != LUNA_OK) return st;
  if ((st = check_rows(dK, "dK", dtype, ks, Hk, d, true)) != LUNA_OK) return st;
  if ((st = check_rows(dV, "dV", dtype, ks, Hk, d, true)) != LUNA_OK) return st;
  const size_t deltas = delta_bytes(seqs, H), parts = head_part_bytes(dtype, seqs, keys, H, Hk, d);
  if ((st = check_ws(deltas + parts, ws, ws_bytes)) != LUNA_OK) return st;
  luna::SoftmaxArgs a = softmax_args(Q, K, V, out, seqs, keys, H, Hk, d, scale);
  a.lse = const_cast<float*>(lse);
  a.dO = rows_of(dO);
  a.dq = rows_of(dQ);
  a.dk = rows_of(dK);
  a.dv = rows_of(dV);
  a.delta = static_cast<float*>(ws);
  if (parts) a.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + deltas);
  return hip_status(luna::launch_softmax_bwd(type_of(dtype), a, reinterpret_cast<hipStream_t>(stream)), "softmax backward launch");
}

}  // extern "C"
