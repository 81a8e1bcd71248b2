// luna_paged_append.hip -- new keys and values into the pages of a cache, keys (and the queries beside them) rotated on the way.
//
// Token i of a sequence's m new ones has position p = len - m + i.  With angle a_j = p inv_freq_j the pair (x, y) of components j
// becomes (x cos a_j - y sin a_j, x sin a_j + y cos a_j); components behind the rotated ones stay.  Angles are formed in 64 bits as
// turns, of which only the fraction goes on in fp32.
//
// A workgroup takes TOKENS tokens of one sequence: the turns' sines and cosines and the tokens' pages once into LDS, then the rows of all
// heads, eight pairs (or eight elements that only move) a thread.  What bounds it is reading and writing each row once: a thread asks
// for the rows of several items before it writes the first (packed prompts of 16384 tokens, 16 heads on 4, d = 128, 201 MB: 52.8 us, 3.8 TB/s;
// with two items 54.4, with eight 73.4, one after the other 62.7).
#include "luna_seq.hpp"

namespace luna {

namespace {

constexpr int kMaxPairs = 64;  // d / 2

template <typename T, int TOKENS>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  constexpr int esz = (int)sizeof(T), AHEAD = TOKENS == 1 ? 2 : 4;
  __shared__ __attribute__((aligned(16))) float cs[TOKENS][2][kMaxPairs];
  __shared__ int page_at[TOKENS];  // (-1: none)
  const SeqPiece sp = seq_piece(a.s, blockIdx.x, TOKENS);
  if (sp.seq < 0) return;
  const bool packed = a.s.offsets != nullptr;
  const int t0 = sp.index * TOKENS, m = min(TOKENS, sp.len - t0), pairs = a.rot / 2;
  const int64_t first = (int64_t)a.lens[sp.seq] - sp.len + t0;  // position of the piece's first token
  for (int i = threadIdx.x; i < m * pairs; i += 256) {
    const int t = i / pairs, j = i % pairs;
    const double turns = (double)(first + t) * (double)a.inv_freq[j] * 0.15915494309189535;  // 1 / (2 pi)
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[t][0][j] = c;
    cs[t][1][j] = s;
  }
  const int64_t room = (int64_t)a.pages.width << a.pages.shift;
  if ((int)threadIdx.x < m) {
    const int64_t pos = first + threadIdx.x;
    page_at[threadIdx.x] = pos >= 0 && pos < room ? page_of(a.pages, sp.seq, (int)pos) : -1;
  }
  __syncthreads();

  // per token and head of Q and K: rot / 16 pieces of 8 pairs, then what is not rotated; of V: all
  const int turned = a.rot / 16, still = (a.d - a.rot) / 8, each = turned + still, vs = a.d / 8;
  const int qh = a.q.data ? a.H : 0, items = (qh + a.Hk) * each + a.Hk * vs, all = m * items;
  const int step = (a.interleaved ? 16 : 8) * esz, next = (a.interleaved ? 8 : pairs) * esz;
  for (int i0 = threadIdx.x; i0 < all; i0 += 256 * AHEAD) {
    Frag<T> x[AHEAD], y[AHEAD];
    char* to[AHEAD];   // null: nothing to write
    int piece[AHEAD];  // of the turned ones, or -1
    int token[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) {
      const int i = min(i0 + 256 * n, all - 1), t = i / items, item = i % items;
      const bool is_v = item >= (qh + a.Hk) * each;
      const int r = is_v ? item - (qh + a.Hk) * each : item;
      const int head = r / (is_v ? vs : each), p = r % (is_v ? vs : each);
      const bool is_q = !is_v && head < qh, turns = !is_v && p < turned;
      const SeqRows from = is_v ? a.v : is_q ? a.q : a.k;
      const SeqRows pages = is_v ? a.vp : a.kp;
      const int hk = is_v ? head : head - qh, page = page_at[t];
      // x: the pairs' first components and y their second, or both in turn
      const int at = turns ? step * p : (is_v ? 8 * p : a.rot + (p - turned) * 8) * esz;
      const char* src = seq_row(from, sp, packed, is_q ? head : hk, t0 + t, esz) + at;
      char* dst = is_q ? seq_row(a.o, sp, packed, head, t0 + t, esz)
                       : pages.data + (max(page, 0) * pages.seq + hk * pages.head + ((first + t) & ((1 << a.pages.shift) - 1)) * pages.row) * esz;
      to[n] = i0 + 256 * n < all && (is_q || page >= 0) ? dst + at : nullptr;
      piece[n] = turns ? p : -1;
      token[n] = t;
      load8(x[n], reinterpret_cast<const T*>(src));
      if (turns) load8(y[n], reinterpret_cast<const T*>(src + next));
    }
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) {
      if (!to[n]) continue;
      if (piece[n] < 0) {
        store8(reinterpret_cast<T*>(to[n]), x[n]);
        continue;
      }
      float c[8], s[8], u[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = cs[token[n]][0][8 * piece[n] + e], s[e] = cs[token[n]][1][8 * piece[n] + e];
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          u[e] = x[n].get(e) * c[e / 2] - x[n].get(e + 1) * s[e / 2];
          u[e + 1] = x[n].get(e) * s[e / 2] + x[n].get(e + 1) * c[e / 2];
          v[e] = y[n].get(e) * c[4 + e / 2] - y[n].get(e + 1) * s[4 + e / 2];
          v[e + 1] = y[n].get(e) * s[4 + e / 2] + y[n].get(e + 1) * c[4 + e / 2];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] = x[n].get(e) * c[e] - y[n].get(e) * s[e];
          v[e] = x[n].get(e) * s[e] + y[n].get(e) * c[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; e += 2) x[n].set2(e, u[e], u[e + 1]), y[n].set2(e, v[e], v[e + 1]);
      store8(reinterpret_cast<T*>(to[n]), x[n]);
      store8(reinterpret_cast<T*>(to[n] + next), y[n]);
    }
  }
}

// Tokens of a workgroup: one where all of them together are few workgroups.
constexpr int kManyTokens = 8;
bool append_many(const SeqSet& s) { return (s.offsets ? s.rows : s.count * s.rows) >= 4096; }

template <typename T>
hipError_t launch_typed(const AppendArgs& a, hipStream_t s) {
  if (append_many(a.s))
    hipLaunchKernelGGL((append_kernel<T, kManyTokens>), dim3((unsigned)seq_slots(a.s, kManyTokens)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((append_kernel<T, 1>), dim3((unsigned)seq_slots(a.s, 1)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

bool append_launchable(const SeqSet& s) { return seq_slots(s, append_many(s) ? kManyTokens : 1) < ((int64_t)1 << 24); }

hipError_t launch_append(Dt dt, const AppendArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_typed<__bf16>(a, s) : launch_typed<float>(a, s);
}

}  // namespace luna
