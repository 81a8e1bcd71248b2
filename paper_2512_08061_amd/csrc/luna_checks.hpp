// luna_checks.hpp -- the checks that the host files of the operators over sequences share (luna_seq_api.cpp,
// luna_delta_api.cpp, luna_paged_api.cpp).
#pragma once

#include <cstdio>

#include "luna_error.hpp"
#include "luna_seq.h"
#include "luna_seq.hpp"

namespace luna {
namespace checks {

constexpr int64_t kMaxRows = (int64_t)1 << 30, kMaxRow = (int64_t)1 << 20;

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// A launch has fewer than 2^32 threads.
inline bool launchable(int64_t groups, int threads) { return groups < ((int64_t)1 << 32) / threads; }

inline luna::SeqRows rows_of(const luna_rows* r) {
  return r ? luna::SeqRows{static_cast<char*>(r->data), r->seq, r->head, r->row} : luna::SeqRows{};
}
inline luna::SeqSet set_of(const luna_seqs* s) { return luna::SeqSet{s->count, s->rows, s->offsets, s->lens}; }

inline luna_status check_seqs(const luna_seqs* s, const char* what) {
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
inline luna_status check_rows(const luna_rows* r, const char* what, luna_dtype dt, const luna_seqs& s, int64_t heads, int64_t width,
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

inline luna_status check_ws(size_t need, const void* ws, size_t ws_bytes) {
  if (need == 0) return LUNA_OK;
  if (!ws || ((uintptr_t)ws & 255) != 0) return set_error(LUNA_ERR_INVALID_ARG, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < need) {
    char why[96];
    snprintf(why, sizeof why, "workspace holds %zu bytes, %zu are needed", ws_bytes, need);
    return set_error(LUNA_ERR_WORKSPACE, why);
  }
  return LUNA_OK;
}

inline luna_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return LUNA_OK;
  char why[160];
  snprintf(why, sizeof why, "%s: %s", what, hipGetErrorString(e));
  return set_error(LUNA_ERR_HIP, why);
}

inline luna::Dt type_of(luna_dtype dt) { return dt == LUNA_BF16 ? luna::Dt::BF16 : luna::Dt::F32; }
inline luna_status check_type(luna_dtype dt) {
  return dt == LUNA_F32 || dt == LUNA_BF16 ? LUNA_OK : set_error(LUNA_ERR_INVALID_ARG, "dtype must be LUNA_F32 or LUNA_BF16");
}

}  // namespace checks
}  // namespace luna
