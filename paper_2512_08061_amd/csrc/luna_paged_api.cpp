// luna_paged_api.cpp -- host side of the C ABI declared in include/luna_paged.h: checks, the workspace, launches on the
// caller's stream.
#include "luna_paged.h"

#include <cmath>

#include "luna_checks.hpp"

namespace {

using luna::set_error;
using namespace luna::checks;

int log2_of(int64_t x) {
  int n = 0;
  while (((int64_t)1 << n) < x) ++n;
  return n;
}
luna::PageSet pages_of(const luna_pages& p) { return luna::PageSet{p.table, p.pool, (int)p.width, log2_of(p.rows)}; }
// the cached keys as sequences
luna::SeqSet cache_of(const luna_seqs& s, const luna_pages& p) { return luna::SeqSet{s.count, p.width * p.rows, nullptr, p.lens}; }

luna_status check_paged(luna_dtype dt, const luna_seqs* seqs, const luna_pages* p, int64_t H, int64_t Hk, int64_t d) {
  luna_status st = check_type(dt);
  if (st == LUNA_OK) st = check_seqs(seqs, "seqs");
  if (st != LUNA_OK) return st;
  if (!p) return set_error(LUNA_ERR_INVALID_ARG, "pages is NULL");
  if (H < 1 || Hk < 1 || H % Hk) return set_error(LUNA_ERR_INVALID_ARG, "H must be a positive multiple of Hk");
  if (H > 65535) return set_error(LUNA_ERR_UNSUPPORTED, "H must be <= 65535");
  if (d != 32 && d != 64 && d != 128) return set_error(LUNA_ERR_UNSUPPORTED, "d must be 32, 64 or 128");
  if (p->pool < 1 || p->width < 1 || p->rows < 1) return set_error(LUNA_ERR_INVALID_ARG, "pages: pool, rows and width must be >= 1");
  if (p->rows < 16 || p->rows > 65536 || (p->rows & (p->rows - 1)))
    return set_error(LUNA_ERR_UNSUPPORTED, "pages: rows must be a power of two from 16 to 65536");
  if (p->pool > ((int64_t)1 << 31) || p->width > kMaxRows / p->rows)
    return set_error(LUNA_ERR_UNSUPPORTED, "pages: more than 2^31 pages or 2^30 tokens of a sequence");
  if (!p->table || !p->lens) return set_error(LUNA_ERR_INVALID_ARG, "pages: table or lens is NULL");
  return LUNA_OK;
}

// pages as the sequences of a tensor of rows
luna_status check_pages(const luna_rows* r, const char* what, luna_dtype dt, const luna_pages& p, int64_t Hk, int64_t d, bool output) {
  const luna_seqs as{p.pool, p.rows, nullptr, nullptr};
  return check_rows(r, what, dt, as, Hk, d, output);
}

// bytes of the parts of rows whose keys lie in several shares, or 0 where the tile kernels take the call
size_t part_bytes(luna_dtype dt, const luna_seqs& s, const luna_pages& p, int64_t H, int64_t Hk, int64_t d) {
  const int64_t shares = luna::paged_splits(type_of(dt), set_of(&s), H, Hk, p.width * p.rows)
                             ? luna::paged_shares(type_of(dt), s.count, p.width * p.rows, Hk, s.rows * (H / Hk))
                             : luna::paged_tile_shares(type_of(dt), set_of(&s), H, Hk, d);
  if (!shares) return 0;
  return align256((size_t)(shares + s.count) * H * (s.rows < 1 ? 1 : s.rows) * (d + 2) * 4);
}

luna_status check_attn(luna_dtype dt, const luna_seqs* seqs, const luna_pages* pages, int64_t H, int64_t Hk, int64_t d) {
  const luna_status st = check_paged(dt, seqs, pages, H, Hk, d);
  if (st != LUNA_OK) return st;
  const luna::SeqSet qs = set_of(seqs);
  const int64_t rows = qs.rows * (H / Hk);
  bool fits;
  if (luna::paged_splits(type_of(dt), qs, H, Hk, pages->width * pages->rows)) {  // (a join takes two rows of a key head or more)
    fits = launchable(qs.count * H * qs.rows, 256) &&
           launchable((luna::paged_shares(type_of(dt), qs.count, pages->width * pages->rows, Hk, rows) + qs.count) * Hk *
                          luna::paged_row_groups(type_of(dt), rows),
                      256);
  } else {
    fits = launchable(luna::seq_slots(qs, luna::softmax_tile(type_of(dt), d)) * H, 256);
  }
  return fits ? LUNA_OK : set_error(LUNA_ERR_UNSUPPORTED, "too many tiles of sequences and heads");
}

}  // namespace

extern "C" {

size_t luna_paged_workspace_bytes(luna_dtype dtype, const luna_seqs* seqs, const luna_pages* pages, int64_t H, int64_t Hk,
                                  int64_t d) {
  luna::clear_error();
  if (check_attn(dtype, seqs, pages, H, Hk, d) != LUNA_OK) return 0;
  return part_bytes(dtype, *seqs, *pages, H, Hk, d);
}

luna_status luna_paged_append(const luna_rows* K, const luna_rows* V, const luna_rows* Q, luna_dtype dtype,
                              const luna_seqs* seqs, const luna_pages* pages, int64_t H, int64_t Hk, int64_t d, int64_t rot,
                              const float* inv_freq, int32_t interleaved, const luna_rows* k_pages,
                              const luna_rows* v_pages, const luna_rows* q_out, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_paged(dtype, seqs, pages, H, Hk, d)) != LUNA_OK) return st;
  if (rot < 0 || rot > d || rot % 16) return set_error(LUNA_ERR_INVALID_ARG, "rot must be a multiple of 16 from 0 to d");
  if ((rot > 0) != (inv_freq != nullptr)) return set_error(LUNA_ERR_INVALID_ARG, "inv_freq goes with rot > 0");
  if (interleaved != 0 && interleaved != 1) return set_error(LUNA_ERR_INVALID_ARG, "interleaved must be 0 or 1");
  if ((Q != nullptr) != (q_out != nullptr)) return set_error(LUNA_ERR_INVALID_ARG, "Q and q_out go together");
  if ((st = check_rows(K, "K", dtype, *seqs, Hk, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(V, "V", dtype, *seqs, Hk, d, false)) != LUNA_OK) return st;
  if (Q && (st = check_rows(Q, "Q", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if (Q && (st = check_rows(q_out, "q_out", dtype, *seqs, H, d, true)) != LUNA_OK) return st;
  if ((st = check_pages(k_pages, "k_pages", dtype, *pages, Hk, d, true)) != LUNA_OK) return st;
  if ((st = check_pages(v_pages, "v_pages", dtype, *pages, Hk, d, true)) != LUNA_OK) return st;
  const luna::SeqSet set = set_of(seqs);
  if (!luna::append_launchable(set)) return set_error(LUNA_ERR_UNSUPPORTED, "too many new tokens");
  if (seqs->rows == 0) return LUNA_OK;
  luna::AppendArgs a{};
  a.k = rows_of(K);
  a.v = rows_of(V);
  a.q = rows_of(Q);
  a.o = rows_of(q_out);
  a.kp = rows_of(k_pages);
  a.vp = rows_of(v_pages);
  a.s = set;
  a.pages = pages_of(*pages);
  a.lens = pages->lens;
  a.inv_freq = inv_freq;
  a.H = (int)H;
  a.Hk = (int)Hk;
  a.d = (int)d;
  a.rot = (int)rot;
  a.interleaved = interleaved;
  return hip_status(luna::launch_append(type_of(dtype), a, reinterpret_cast<hipStream_t>(stream)), "append launch");
}

luna_status luna_paged_fwd(const luna_rows* Q, const luna_rows* k_pages, const luna_rows* v_pages, luna_dtype dtype,
                           const luna_seqs* seqs, const luna_pages* pages, int64_t H, int64_t Hk, int64_t d, float scale,
                           const luna_rows* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  luna::clear_error();
  luna_status st;
  if ((st = check_attn(dtype, seqs, pages, H, Hk, d)) != LUNA_OK) return st;
  if (!std::isfinite(scale)) return set_error(LUNA_ERR_INVALID_ARG, "scale must be finite");
  if ((st = check_rows(Q, "Q", dtype, *seqs, H, d, false)) != LUNA_OK) return st;
  if ((st = check_pages(k_pages, "k_pages", dtype, *pages, Hk, d, false)) != LUNA_OK) return st;
  if ((st = check_pages(v_pages, "v_pages", dtype, *pages, Hk, d, false)) != LUNA_OK) return st;
  if ((st = check_rows(out, "out", dtype, *seqs, H, d, true)) != LUNA_OK) return st;
  const size_t need = part_bytes(dtype, *seqs, *pages, H, Hk, d);
  if ((st = check_ws(need, ws, ws_bytes)) != LUNA_OK) return st;
  if (seqs->rows == 0) return LUNA_OK;
  luna::SoftmaxArgs a{};
  a.q = rows_of(Q);
  a.k = rows_of(k_pages);
  a.v = rows_of(v_pages);
  a.o = rows_of(out);
  a.qs = set_of(seqs);
  a.ks = cache_of(*seqs, *pages);
  a.pages = pages_of(*pages);
  a.H = (int)H;
  a.Hk = (int)Hk;
  a.d = (int)d;
  a.scale = scale;
  a.lse = lse;
  a.parts = static_cast<float*>(ws);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return hip_status(luna::paged_splits(type_of(dtype), a.qs, H, Hk, a.ks.rows) ? luna::launch_paged_split(type_of(dtype), a, s)
                                                                                   : luna::launch_paged_tiles(type_of(dtype), a, s),
                    "paged attention launch");
}

}  // extern "C"
