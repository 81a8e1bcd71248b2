// luna_paged_append.hip -- new keys and values into the pages of a cache, keys (and the queries beside them) rotated on the way.
//
// Token i of a sequence's m new ones has position p = len - m + i.  With angle a_j = p inv_freq_j the pair (x, y) of components j
// becomes (x cos a_j - y sin a_j, x sin a_j + y cos a_j); components behind the rotated ones stay.  Angles are formed in 64 bits as
// turns, of which only the fraction goes on in fp32.
//
// A workgroup takes TOKENS tokens of one sequence: the turns' sines and cosines once into LDS, then the rows of all heads, eight
// pairs (or 16 bytes that only move) a thread.  What bounds it is reading and writing each row once.
#include "luna_seq.hpp"

namespace luna {

namespace {

constexpr int kMaxPairs = 64;  // d / 2

// Eight consecutive elements, whatever the type.
template <typename T>
__device__ __forceinline__ void get8(float (&x)[8], const char* p) {
  Frag<T> f;
  load8(f, reinterpret_cast<const T*>(p));
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = f.get(e);
}
template <typename T>
__device__ __forceinline__ void put8(char* p, const float (&x)[8]) {
  Frag<T> f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) f.set2(e, x[e], x[e + 1]);
  store8(reinterpret_cast<T*>(p), f);
}

template <typename T, int TOKENS>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  constexpr int esz = (int)sizeof(T);
  __shared__ __attribute__((aligned(16))) float cs[TOKENS][2][kMaxPairs];
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
  __syncthreads();

  // per token and head of Q and K: rot / 16 pieces of 8 pairs, then what is not rotated; of V: all
  const int turned = a.rot / 16, still = (a.d - a.rot) / 8, each = turned + still, vs = a.d / 8;
  const int qh = a.q.data ? a.H : 0, items = (qh + a.Hk) * each + a.Hk * vs;
  const int64_t room = (int64_t)a.pages.width << a.pages.shift;
  for (int i = threadIdx.x; i < m * items; i += 256) {
    const int t = i / items, item = i % items;
    const int64_t pos = first + t;
    int page = -1;
    if (pos >= 0 && pos < room) page = page_of(a.pages, sp.seq, (int)pos);
    const int64_t slot = pos & ((1 << a.pages.shift) - 1);
    const bool is_v = item >= (qh + a.Hk) * each;
    const int r = is_v ? item - (qh + a.Hk) * each : item;
    const int head = r / (is_v ? vs : each), piece = r % (is_v ? vs : each);
    const bool is_q = !is_v && head < qh;
    if (!is_q && page < 0) continue;
    const SeqRows& from = is_v ? a.v : is_q ? a.q : a.k;
    const int hk = is_v ? head : head - qh;
    const char* src = seq_row(from, sp, packed, is_q ? head : hk, t0 + t, esz);
    char* dst = is_q ? seq_row(a.o, sp, packed, head, t0 + t, esz)
                     : (is_v ? a.vp : a.kp).data + (page * (is_v ? a.vp : a.kp).seq + hk * (is_v ? a.vp : a.kp).head + slot * (is_v ? a.vp : a.kp).row) * esz;
    if (is_v || piece >= turned) {
      const int at = (is_v ? piece * 8 : a.rot + (piece - turned) * 8) * esz;
      Frag<T> f;
      load8(f, reinterpret_cast<const T*>(src + at));
      store8(reinterpret_cast<T*>(dst + at), f);
      continue;
    }
    // x: the pairs' first components and y their second, or both in turn
    const int at = (a.interleaved ? 16 : 8) * piece * esz, next = (a.interleaved ? 8 : pairs) * esz;
    float x[8], y[8], c[8], s[8];
    get8<T>(x, src + at);
    get8<T>(y, src + at + next);
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = cs[t][0][8 * piece + e], s[e] = cs[t][1][8 * piece + e];
    float u[8], v[8];
    if (a.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        u[e] = x[e] * c[e / 2] - x[e + 1] * s[e / 2];
        u[e + 1] = x[e] * s[e / 2] + x[e + 1] * c[e / 2];
        v[e] = y[e] * c[4 + e / 2] - y[e + 1] * s[4 + e / 2];
        v[e + 1] = y[e] * s[4 + e / 2] + y[e + 1] * c[4 + e / 2];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = x[e] * c[e] - y[e] * s[e];
        v[e] = x[e] * s[e] + y[e] * c[e];
      }
    }
    put8<T>(dst + at, u);
    put8<T>(dst + at + next, v);
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
