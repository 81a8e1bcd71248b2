// luna_delta_api.cpp -- host side of the C ABI declared in include/luna_delta.h: checks, the workspace, launches on the
// caller's stream.
#include "luna_delta.h"

#include <cmath>

#include "luna_checks.hpp"
#include "luna_delta.hpp"

namespace {

using luna::set_error;
using namespace luna::checks;

luna_status check_delta(luna_dtype dt, int64_t H, int64_t Hk, int64_t D, int64_t d, float scale) {
  const luna_status st = check_type(dt);
  if (st != LUNA_OK) return st;
  if (H < 1 || Hk < 1 || H % Hk) return set_error(LUNA_ERR_INVALID_ARG, "H must be a positive multiple of Hk");
  if (H > 65535) return set_error(LUNA_ERR_UNSUPPORTED, "H must be <= 65535");
  if (D < 1 || d < 1) return set_error(LUNA_ERR_INVALID_ARG, "D and d must be >= 1");
  if ((D != 32 && D != 64 && D != 128) || (d != 32 && d != 64 && d != 128))
    return set_error(LUNA_ERR_UNSUPPORTED, "D and d must be 32, 64 or 128");
  if (!std::isfinite(scale)) return set_error(LUNA_ERR_INVALID_ARG, "scale must be finite");
  return LUNA_OK;
}

// numbers per row: of no rows they may be NULL
luna_status check_numbers(const float* x, const char* what, const luna_seqs& s) {
  char why[64];
  if (x || s.rows == 0) return LUNA_OK;
  snprintf(why, sizeof why, "%s is NULL", what);
  return set_error(LUNA_ERR_INVALID_ARG, why);
}

struct DeltaPlan {
  int64_t slots = 0;
  size_t n = 0, p = 0, gates = 0, before = 0, after = 0, e = 0, x = 0, total = 0;  // workspace offsets
};

luna_status plan_delta(luna_dtype dt, const luna_seqs& s, int64_t H, int64_t Hk, int64_t D, int64_t d, bool backward, DeltaPlan* p) {
  const luna::SeqSet set = set_of(&s);
  p->slots = luna::seq_slots(set, luna::kDeltaChunk);
  if (!launchable(p->slots * Hk, 512) || p->slots >= ((int64_t)1 << 31) ||
      !launchable((backward ? 2 : 1) * s.count * H * (d / 32), 512))
    return set_error(LUNA_ERR_UNSUPPORTED, "too many chunks of sequences and heads");
  const size_t all = (size_t)p->slots * H, matrix = (size_t)luna::kDeltaChunk * luna::kDeltaChunk * (dt == LUNA_BF16 ? 2 : 4);
  const auto parts = [&](int n) { return (size_t)(dt == LUNA_BF16 ? n : 1); };
  const auto take = [&](size_t& at, size_t bytes) {
    at = p->total;
    p->total = align256(p->total + all * bytes);
  };
  if (!backward && dt == LUNA_BF16) return LUNA_OK;  // (one launch, all in LDS)
  take(p->n, parts(luna::kDeltaBackParts) * matrix);
  take(p->p, parts(luna::kDeltaBackParts) * matrix);
  take(p->gates, luna::kDeltaGates * 4);
  if (backward) {
    take(p->before, (size_t)(D * d) * 4);
    take(p->after, (size_t)(D * d) * 4);
    take(p->e, (size_t)luna::kDeltaChunk * d * 4);
    take(p->x, (size_t)luna::kDeltaChunk * d * 4);
  }
  return LUNA_OK;
}

luna::DeltaArgs delta_args(const luna_rows* Q, const luna_rows* K, const luna_rows* V, const luna_rows* o, const luna_seqs* seqs,
                           int64_t H, int64_t Hk, int64_t D, int64_t d, const float* log_decay, const float* beta, float scale,
                           const DeltaPlan& p, void* ws) {
  luna::DeltaArgs a{};
  a.q = rows_of(Q);
  a.k = rows_of(K);
  a.v = rows_of(V);
  a.o = rows_of(o);
  a.s = set_of(seqs);
  a.log_decay = log_decay;
  a.beta = beta;
  a.H = (int)H;
  a.Hk = (int)Hk;
  a.D = (int)D;
  a.d = (int)d;
  a.slots = (int)p.slots;
  a.scale = scale;
  char* at = static_cast<char*>(ws);
  a.n = at + p.n;
  a.p = at + p.p;
  a.gates = reinterpret_cast<float*>(at + p.gates);
  a.before = reinterpret_cast<float*>(at + p.before);
  a.after = reinterpret_cast<float*>(at + p.after);
  a.e = reinterpret_cast<float*>(at + p.e);
  a.x = reinterpret_cast<float*>(at + p.x);
  return a;
}

}  // namespace

extern "C" {

size_t luna_delta_workspace_bytes(int32_t op, luna_dtype dtype, const luna_seqs* seqs, int64_t H, int64_t Hk, int64_t D,
                                  int64_t d) {
  luna::clear_error();
  if (op != LUNA_OP_DELTA_FWD && op != LUNA_OP_DELTA_BWD) {
    set_error(LUNA_ERR_INVALID_ARG, "unknown operation");
    return 0;
  }
  DeltaPlan p;
  if (check_seqs(seqs, "seqs") != LUNA_OK || check_delta(dtype, H, Hk, D, d, 1.0f) != LUNA_OK ||
      plan_delta(dtype, *seqs, H, Hk, D, d, op == LUNA_OP_DELTA_BWD, &p) != LUNA_OK)
    return 0;
  return p.total;
}

luna_status luna_delta_fwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype,
                           const luna_seqs* seqs, int64_t H, int64_t Hk, int64_t D, int64_t d, const float* log_decay,
                           const float* beta, float scale, float* S, const luna_rows* out, void* ws, size_t ws_bytes,
                           void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_delta(dtype, H, Hk, D, d, scale)) != LUNA_OK) return st;
  if ((st = check_seqs(seqs, "seqs")) != LUNA_OK) return st;
  if ((st = check_numbers(log_decay, "log_decay", *seqs)) != LUNA_OK) return st;
  if ((st = check_numbers(beta, "beta", *seqs)) != LUNA_OK) return st;
  if (((uintptr_t)S & 15) != 0) return set_error(LUNA_ERR_INVALID_ARG, "S must be 16-byte aligned");
  if ((st = check_rows(Q, "Q", dtype, *seqs, Hk, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(K, "K", dtype, *seqs, Hk, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(out, "out", dtype, *seqs, H, d, true)) != LUNA_OK) return st;
  DeltaPlan p;
  if ((st = plan_delta(dtype, *seqs, H, Hk, D, d, false, &p)) != LUNA_OK) return st;
  if ((st = check_ws(p.total, ws, ws_bytes)) != LUNA_OK) return st;
  if (seqs->rows == 0) return LUNA_OK;
  luna::DeltaArgs a = delta_args(Q, K, V, out, seqs, H, Hk, D, d, log_decay, beta, scale, p, ws);
  a.S = S;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const luna::Dt dt = type_of(dtype);
  if (dt == luna::Dt::BF16) return hip_status(luna::launch_delta_fwd_bf16(S != nullptr, a, s), "delta launch");
  if ((st = hip_status(luna::launch_delta_gates(dt, a, s), "delta gate launch")) != LUNA_OK) return st;
  return hip_status(luna::launch_delta_fwd_f32(a, s), "delta launch");
}

luna_status luna_delta_step(const luna_rows* Q, const luna_rows* K, const luna_rows* V, luna_dtype dtype, int64_t count,
                            int64_t m, int64_t H, int64_t Hk, int64_t D, int64_t d, const float* log_decay,
                            const float* beta, float scale, float* S, const luna_rows* out, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_delta(dtype, H, Hk, D, d, scale)) != LUNA_OK) return st;
  const luna_seqs seqs{count, m, nullptr, nullptr};
  if (m < 1) return set_error(LUNA_ERR_INVALID_ARG, "m must be >= 1");
  if ((st = check_seqs(&seqs, "the tokens")) != LUNA_OK) return st;
  if ((st = check_numbers(log_decay, "log_decay", seqs)) != LUNA_OK) return st;
  if ((st = check_numbers(beta, "beta", seqs)) != LUNA_OK) return st;
  if (!S) return set_error(LUNA_ERR_INVALID_ARG, "S is NULL");
  if (((uintptr_t)S & 15) != 0) return set_error(LUNA_ERR_INVALID_ARG, "S must be 16-byte aligned");
  if ((st = check_rows(Q, "Q", dtype, seqs, Hk, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(K, "K", dtype, seqs, Hk, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(out, "out", dtype, seqs, H, d, true)) != LUNA_OK) return st;
  if (count * H > (int64_t)1 << 19) return set_error(LUNA_ERR_UNSUPPORTED, "count * H must be <= 2^19");
  luna::DeltaStepArgs a{};
  a.q = rows_of(Q);
  a.k = rows_of(K);
  a.v = rows_of(V);
  a.o = rows_of(out);
  a.log_decay = log_decay;
  a.beta = beta;
  a.count = count;
  a.m = (int)m;
  a.H = (int)H;
  a.Hk = (int)Hk;
  a.D = (int)D;
  a.d = (int)d;
  a.scale = scale;
  a.S = S;
  return hip_status(luna::launch_delta_step(type_of(dtype), a, reinterpret_cast<hipStream_t>(stream)), "delta step launch");
}

luna_status luna_delta_bwd(const luna_rows* Q, const luna_rows* K, const luna_rows* V, const luna_rows* dO,
                           luna_dtype dtype, const luna_seqs* seqs, int64_t H, int64_t Hk, int64_t D, int64_t d,
                           const float* log_decay, const float* beta, float scale, const luna_rows* dQ,
                           const luna_rows* dK, const luna_rows* dV, float* dlog_decay, float* dbeta, void* ws,
                           size_t ws_bytes, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_delta(dtype, H, Hk, D, d, scale)) != LUNA_OK) return st;
  if ((st = check_seqs(seqs, "seqs")) != LUNA_OK) return st;
  if ((st = check_numbers(log_decay, "log_decay", *seqs)) != LUNA_OK) return st;
  if ((st = check_numbers(beta, "beta", *seqs)) != LUNA_OK) return st;
  if ((st = check_numbers(dlog_decay, "dlog_decay", *seqs)) != LUNA_OK) return st;
  if ((st = check_numbers(dbeta, "dbeta", *seqs)) != LUNA_OK) return st;
  if ((st = check_rows(Q, "Q", dtype, *seqs, Hk, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(K, "K", dtype, *seqs, Hk, D, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(dO, "dO", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(dQ, "dQ", dtype, *seqs, Hk, D, true)) != LUNA_OK) return st;
  if ((st = check_rows(dK, "dK", dtype, *seqs, Hk, D, true)) != LUNA_OK) return st;
  if ((st = check_rows(dV, "dV", dtype, *seqs, H, d, true)) != LUNA_OK) return st;
  DeltaPlan p;
  if ((st = plan_delta(dtype, *seqs, H, Hk, D, d, true, &p)) != LUNA_OK) return st;
  if ((st = check_ws(p.total, ws, ws_bytes)) != LUNA_OK) return st;
  if (seqs->rows == 0) return LUNA_OK;
  luna::DeltaArgs a = delta_args(Q, K, V, dO, seqs, H, Hk, D, d, log_decay, beta, scale, p, ws);
  a.dq = rows_of(dQ);
  a.dk = rows_of(dK);
  a.dv = rows_of(dV);
  a.dlog_decay = dlog_decay;
  a.dbeta = dbeta;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const luna::Dt dt = type_of(dtype);
  if ((st = hip_status(luna::launch_delta_gates(dt, a, s), "delta gate launch")) != LUNA_OK)
    return st;
  if ((st = hip_status(luna::launch_delta_both(dt, a, s), "delta state launch")) != LUNA_OK) return st;
  return hip_status(luna::launch_delta_grads(dt, a, s), "delta gradient launch");
}

}  // extern "C"
