// luna_softmax.hpp -- tiles shared by the forward and backward kernels of causal softmax
// attention (luna_softmax.hip, luna_softmax_bwd.hip).
#pragma once

#include "luna_seq.hpp"

namespace luna {

// `m` rows (at most R) of width DH into LDS rows of pitch P; rows past m as zeros.
template <typename T, int R, int DH, int P>
__device__ __forceinline__ void softmax_load_rows(T* dst, const char* base, int64_t row, int m) {
  constexpr int E = 16 / (int)sizeof(T), PER = DH / E;
  static_assert(R * PER % 256 == 0, "whole pieces per thread");
  const Buf b = buffer(base, m > 0 ? (int)(((m - 1) * row + DH) * (int)sizeof(T)) : 0);
#pragma unroll
  for (int i = 0; i < R * PER / 256; ++i) {
    const int idx = threadIdx.x + 256 * i, r = idx / PER, c = (idx % PER) * E;
    const auto x = __builtin_amdgcn_raw_buffer_load_b128(b, r < m ? (r * (int)row + c) * (int)sizeof(T) : kPastEnd, 0, 0);
    *reinterpret_cast<i32x4*>(&dst[r * P + c]) = __builtin_bit_cast(i32x4, x);
  }
}

// The pages of N groups of 16 keys from k0 (a multiple of 16) on, up to kend; none: a bit for each group without one.
template <int N>
struct KeyPages {
  int page[N], none;
  __device__ __forceinline__ int at(int i) const {
    int p = 0;  // (selects became a load at an address that depends on i, and the pages went to scratch memory)
#pragma unroll
    for (int k = 0; k < N; ++k) p |= page[k] & -(int)(i == k);
    return p;
  }
};
template <int N>
__device__ __forceinline__ KeyPages<N> key_pages(const SoftmaxArgs& a, int seq, int k0, int kend) {
  KeyPages<N> p;
  p.none = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int key = k0 + 16 * i;
    p.page[i] = __builtin_amdgcn_readfirstlane(page_of(a.pages, seq, max(min(key, kend - 1), 0)));
    if (p.page[i] < 0 && key < kend) p.none |= 1 << i;
  }
  return p;
}
// Rows key .. key + 15 (key a multiple of 16) of a page, up to kend; none of a page that is none of the pool.
__device__ __forceinline__ Buf key_group(const SoftmaxArgs& a, const SeqRows& r, int page, int hk, int key, int kend, int width, int esz) {
  const int n = page < 0 ? 0 : min(16, kend - key);
  const char* base = r.data + (max(page, 0) * r.seq + hk * r.head + (key & ((1 << a.pages.shift) - 1)) * r.row) * esz;
  return buffer(base, n > 0 ? (int)(((n - 1) * r.row + width) * esz) : 0);
}
// As softmax_load_rows, group(i): rows 16 i .. 16 i + 15.
template <typename T, int R, int DH, int P, typename F>
__device__ __forceinline__ void softmax_load_pages(T* dst, F group, int64_t row) {
  constexpr int E = 16 / (int)sizeof(T), PER = DH / E;
  static_assert(R * PER % 256 == 0 && (kWave <= 16 * PER), "a wave's rows lie in one group");
#pragma unroll
  for (int i = 0; i < R * PER / 256; ++i) {
    const int idx = threadIdx.x + 256 * i, r = idx / PER, c = (idx % PER) * E;
    const Buf b = group((kWave * wave_id() + 256 * i) / PER / 16);
    const auto x = __builtin_amdgcn_raw_buffer_load_b128(b, (r % 16 * (int)row + c) * (int)sizeof(T), 0, 0);
    *reinterpret_cast<i32x4*>(&dst[r * P + c]) = __builtin_bit_cast(i32x4, x);
  }
}

// This lane's row (of m, from base) as operand fragments; a row past m as zeros.
template <typename T, int DH>
__device__ __forceinline__ void softmax_load_frags(Frag<T> (&f)[DH / 32], const char* base, int64_t row, int m, int r, int g) {
  const Buf b = buffer(base, m > 0 ? (int)(((m - 1) * row + DH) * (int)sizeof(T)) : 0);
  const int off = r < m ? (r * (int)row + 8 * g) * (int)sizeof(T) : kPastEnd;
#pragma unroll
  for (int t = 0; t < DH / 32; ++t) buf_load8(f[t], b, r < m ? off + 32 * t * (int)sizeof(T) : kPastEnd);
}

// x over the four lane groups
__device__ __forceinline__ float groups_max(float x) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

typedef __attribute__((ext_vector_type(16))) float f32x16;

// Head of a workgroup of H consecutive ones: consecutive workgroups go to the eight dies in turn, so that heads
// i, i + 8, ... meet on one; it gets neighbours, which share key heads.
__device__ __forceinline__ int head_of(int i, int H) { return H % 8 == 0 ? i % 8 * (H / 8) + i / 8 : i; }

// A tile of 64 bf16 rows in LDS.  The 16-byte pieces of a row are swapped among each other by the row's number, so
// that eight rows' pieces of one column, and the two pieces by four rows of a transposing read, lie in different banks.
// Rows come through registers: a thread's pieces are asked for a tile ahead and stored when the tile is free.  (Loads
// that go to LDS directly save those registers and stores, but the compiler waits for all of them before
// any transposing read.)
template <int DH, int THREADS = 256>
struct TileRegs {
  i32x4 x[64 * DH / 8 / THREADS];
};
template <int DH>
struct Tile {
  static constexpr int PIECES = DH / 8;
  __bf16 x[64 * DH];

  static __device__ __forceinline__ int swap(int row) {
    return DH == 128 ? (row % 4) * 2 + (row / 4) % 2 : ((row / 2) % 4) * 2;
  }
  // `n` rows from `base`, the others as zeros, by THREADS threads of which this is tid
  template <int THREADS>
  static __device__ __forceinline__ void load(TileRegs<DH, THREADS>& t, int tid, const char* base, int64_t row, int n) {
    const Buf b = buffer(base, n > 0 ? (int)(((n - 1) * row + DH) * 2) : 0);
#pragma unroll
    for (int j = 0; j < 64 * PIECES / THREADS; ++j) {
      const int at = tid + THREADS * j, r = at / PIECES, piece = at % PIECES;
      t.x[j] = __builtin_bit_cast(
          i32x4, __builtin_amdgcn_raw_buffer_load_b128(b, r < n ? (r * (int)row + piece * 8) * 2 : kPastEnd, 0, 0));
    }
  }
  // by four waves, group(i): rows 16 i .. 16 i + 15
  template <typename F>
  static __device__ __forceinline__ void load_pages(TileRegs<DH, 256>& t, int wave, int lane, F group, int64_t row) {
#pragma unroll
    for (int j = 0; j < 64 * PIECES / 256; ++j) {
      const int first = kWave * wave + 256 * j, at = first + lane, r = at / PIECES, piece = at % PIECES;
      t.x[j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(group(first / PIECES / 16),
                                                                               (r % 16 * (int)row + piece * 8) * 2, 0, 0));
    }
  }
  template <int THREADS>
  __device__ __forceinline__ void store(const TileRegs<DH, THREADS>& t, int tid) {
#pragma unroll
    for (int j = 0; j < 64 * PIECES / THREADS; ++j) {
      const int at = tid + THREADS * j, r = at / PIECES, piece = at % PIECES;
      *reinterpret_cast<i32x4*>(&x[r * DH + ((piece ^ swap(r)) * 8)]) = t.x[j];
    }
  }
  // elements 8 piece .. 8 piece + 7 of a row
  __device__ __forceinline__ bf16x8 row8(int row, int piece) const {
    return *reinterpret_cast<const bf16x8*>(&x[row * DH + ((piece ^ swap(row)) * 8)]);
  }
  // transposed: rows k0 .. k0 + 3 of column c0 + lane % 16 into slots e0 .. e0 + 3 (see load_tr4)
  __device__ __forceinline__ void tr4(Frag<__bf16>& f, int e0, int k0, int c0, int lane) const {
    const int i = lane % 16, row = k0 + i / 4, col = c0 + 4 * (i % 4);
    typedef __attribute__((ext_vector_type(4))) short i16x4;
    const __bf16* src = &x[row * DH + (((col / 8) ^ swap(row)) * 8) + col % 8];
    const i16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) i16x4*)(__attribute__((address_space(3))) void*)(src));
    const bf16x4 b = __builtin_bit_cast(bf16x4, v);
    f.v[e0 + 0] = b[0]; f.v[e0 + 1] = b[1]; f.v[e0 + 2] = b[2]; f.v[e0 + 3] = b[3];
  }
};
// x over the two halves of a wave
__device__ __forceinline__ float halves_sum(float x) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int e = 0; e < 16; ++e) z[e] = 0.0f;
  return z;
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// query rows (key rows) of a workgroup: 16 x 16 products, and 32 x 32 ones (bf16 with d = 64 and 128)
constexpr int kSoftmaxTile = softmax_tile(Dt::F32, 128), kSoftmaxTile32 = softmax_tile(Dt::BF16, 128);
static_assert(kSoftmaxTile == 64 && softmax_tile(Dt::BF16, 32) == 64 && softmax_tile(Dt::BF16, 64) == kSoftmaxTile32, "tiles");
static_assert(kSoftmaxTile32 == 128, "four waves of 32 rows");

// keys per step of the tile kernels: the staged rows of two tensors fit 64 KiB and a bit
template <typename T>
constexpr int kSoftmaxStep = sizeof(T) == 2 ? 64 : 32;

__device__ __forceinline__ bool not_finite(float x) { return !(fabsf(x) < __builtin_inff()); }

// In a tile's product with V a hidden key weighs 0, and 0 times an infinity or a NaN of its values is NaN.  So where a
// row's result is not finite and values of keys that are hidden from it (or rows beside it) are not either, softmax_row
// forms it again from the keys that it sees.  Tiles of finite values pay one test of their results, and rows that see what
// is not finite, far from the tile where it lies, one more.  (The log-sum is right as it is: scores are masked one by one.)

// Row of a key among keys or values; null where its page is none of the pool (whose keys no row sees).
template <bool PAGED>
__device__ __forceinline__ char* softmax_key_row(const SoftmaxArgs& a, const SeqRows& r, const SeqPiece& sk, int hk, int key, int esz) {
  if constexpr (!PAGED) {
    return seq_row(r, sk, a.ks.offsets != nullptr, hk, key, esz);
  } else {
    const int page = page_of(a.pages, sk.seq, key);
    return page < 0 ? nullptr : r.data + (page * r.seq + hk * r.head + (key & ((1 << a.pages.shift) - 1)) * r.row) * esz;
  }
}

// Whether the values of keys first .. end - 1 hold any that is not finite (for all lanes).
template <typename T, int DH, int LANES, bool PAGED = false>
__device__ __forceinline__ bool softmax_odd_values(const SoftmaxArgs& a, const SeqPiece& sk, int hk, int first, int end) {
  bool odd = false;
#pragma unroll 1
  for (int key = max(first, 0) + (int)threadIdx.x % LANES; key < end; key += LANES) {
    const T* v = reinterpret_cast<const T*>(softmax_key_row<PAGED>(a, a.v, sk, hk, key, (int)sizeof(T)));
    if (PAGED && !v) continue;
#pragma unroll 4
    for (int c = 0; c < DH; c += 8) {
      Frag<T> f;
      load8(f, v + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) odd |= not_finite(f.get(e));
    }
  }
  return __any(odd);
}

// The same for the LANES lanes of a row, where a wave may have rows of its own in each.
template <typename T, int DH, int LANES>
__device__ __forceinline__ bool softmax_odd_row(const SoftmaxArgs& a, const SeqPiece& sk, int hk, int first, int end) {
  if constexpr (LANES == kWave) {
    return softmax_odd_values<T, DH, LANES, true>(a, sk, hk, first, end);
  } else {
    return true;  // (two rows of a wave may go different ways: formed again in any case)
  }
}

// One query row by itself, key by key in fp32, by LANES lanes of a wave.
template <typename T, int DH, int LANES, bool PAGED = false>
__device__ __forceinline__ void softmax_row(const SoftmaxArgs& a, const SeqPiece& sq, const SeqPiece& sk, int head, int i) {
  constexpr int PER = (DH + LANES - 1) / LANES, esz = (int)sizeof(T);
  const bool pq = a.qs.offsets != nullptr;
  const int lane = threadIdx.x % LANES, hk = head / (a.H / a.Hk), last = min(sk.len - 1, i + sk.len - sq.len);
  const T* q = reinterpret_cast<const T*>(seq_row(a.q, sq, pq, head, i, esz));
  float top = -__builtin_inff(), sum = 0.0f, acc[PER];
#pragma unroll
  for (int c = 0; c < PER; ++c) acc[c] = 0.0f;
#pragma unroll 1
  for (int k0 = 0; k0 <= last; k0 += LANES) {
    const int n = min(LANES, last - k0 + 1);
    const T* k = reinterpret_cast<const T*>(softmax_key_row<PAGED>(a, a.k, sk, hk, k0 + min(lane, n - 1), esz));
    const bool seen = lane < n && (!PAGED || k);
    if (PAGED && !k) k = q;
    float s = 0.0f;
#pragma unroll 4
    for (int c = 0; c < DH; c += 8) {
      Frag<T> qf, kf;
      load8(qf, q + c);
      load8(kf, k + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(qf.get(e), kf.get(e), s);
    }
    s = seen ? s * (a.scale * kLog2e) : -__builtin_inff();
    float most = fmaxf(top, s);
#pragma unroll
    for (int x = LANES / 2; x > 0; x /= 2) most = fmaxf(most, __shfl_xor(most, x));
    const float base = most == -__builtin_inff() ? 0.0f : most, f = exp2_raw(top - base), p = exp2_raw(s - base);
    top = most;
    sum = fmaf(sum, f, p);
#pragma unroll
    for (int c = 0; c < PER; ++c) acc[c] *= f;
#pragma unroll 1
    for (int j0 = 0; j0 < n; j0 += 8)
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // (behind the last key: the last one again, times 0)
        const T* v = reinterpret_cast<const T*>(softmax_key_row<PAGED>(a, a.v, sk, hk, k0 + min(j0 + j, n - 1), esz));
        const float pj = __shfl(p, j0 + j, LANES);
        if (PAGED && !v) continue;
#pragma unroll
        for (int c = 0; c < PER; ++c) acc[c] = fmaf(pj, (float)v[min(lane + LANES * c, DH - 1)], acc[c]);
      }
    bool lost = true;
#pragma unroll
    for (int c = 0; c < PER; ++c) lost &= isnan(acc[c]);
    if (__all(lost)) break;  // nothing but NaN is left of the row
  }
#pragma unroll
  for (int x = LANES / 2; x > 0; x /= 2) sum += __shfl_xor(sum, x);
  const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
  T* o = reinterpret_cast<T*>(seq_row(a.o, sq, pq, head, i, esz));
#pragma unroll
  for (int c = 0; c < PER; ++c)
    if (lane + LANES * c < DH) o[lane + LANES * c] = (T)(acc[c] * inv);
}

// The keys of padded sequences as one line of units of `unit` keys, cut in equal shares (see PagedUnits).
__device__ __forceinline__ int units_of(const SeqSet& s, int b, int unit) {
  return (seq_clamp(s.lens[b], 0, s.rows) + unit - 1) / unit;
}
__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int w = 1; w < kWave; w *= 2) x += __shfl_xor(x, w);
  return x;
}
template <typename I>
__device__ __forceinline__ I lanes_up_to(I x) {
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int w = 1; w < kWave; w *= 2) {
    const I other = __shfl_up(x, w);
    x += lane >= w ? other : 0;
  }
  return x;
}
// The parts of the line (what a share holds of a sequence) by size: whole shares first, then the others.  The sequence of the part
// of a rank, its share and the units that this holds; -1: no such part (the whole wave calls this; units of all below 2^31).
__device__ __forceinline__ int sequence_of_part(const SeqSet& s, int rank, int shares, int unit, int* share, PagedUnits* held) {
  const int lane = threadIdx.x % kWave, count = (int)s.count;
  int64_t sum = 0;
  for (int b = lane; b < count; b += kWave) sum += units_of(s, b, unit);
  const int all = (int)wave_sum(sum), per = (int)paged_per(all, shares, 1);
#pragma unroll 1
  for (int rest = 0; rest < 2; ++rest) {
    int before0 = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < count; b0 += kWave) {
      const int b = b0 + lane, mine = b < count ? units_of(s, b, unit) : 0, to = before0 + lanes_up_to(mine), before = to - mine;
      const PagedUnits in = paged_holders(before, mine, per);
      const int lo = (before + per - 1) / per, hi = to / per;  // whole ones: lo .. hi - 1
      const int whole = hi > lo ? hi - lo : 0, n = rest ? in.u1 - in.u0 + 1 - whole : whole;
      const int until = lanes_up_to(n);
      const uint64_t found = __ballot(rank < until);
      if (found) {
        const int i = __builtin_ctzll(found), k = rank - (until - n);
        const int mine_share = !rest ? lo + k : !whole ? in.u0 + k : k == 0 && in.u0 < lo ? in.u0 : in.u1;
        const PagedUnits u = paged_held(before, mine, per, mine_share, all);
        *share = __builtin_amdgcn_readlane(mine_share, i);
        held->u0 = __builtin_amdgcn_readlane(u.u0, i);
        held->u1 = __builtin_amdgcn_readlane(u.u1, i);
        return b0 + i;
      }
      rank -= __builtin_amdgcn_readlane(until, kWave - 1);
      before0 = __builtin_amdgcn_readlane(to, kWave - 1);
    }
  }
  return -1;
}
// The sequence b of which share number - b holds units, and the units before it; -1: none (the whole wave calls this).
__device__ __forceinline__ int sequence_of_number(const SeqSet& s, int number, int shares, int unit, int64_t per, int64_t all, int64_t* first) {
  const int lane = threadIdx.x % kWave, count = (int)s.count;
  int64_t sum = 0;
  for (int b0 = 0; b0 < count && b0 <= number; b0 += kWave) {
    const int b = b0 + lane, mine = b < count ? units_of(s, b, unit) : 0, share = number - b;
    const int64_t to = sum + lanes_up_to((int64_t)mine);
    const PagedUnits u = paged_held(to - mine, mine, per, share, all);
    const uint64_t found = __ballot(mine > 0 && share >= 0 && share < shares && share * per < all && u.u0 < u.u1);
    if (found) {
      const int i = __builtin_ctzll(found);
      *first = __shfl(to - mine, i);
      return __builtin_amdgcn_readfirstlane(b0 + i);
    }
    sum = __shfl(to, kWave - 1);
  }
  return -1;
}
// Sum over the threads of a workgroup.
template <int THREADS>
__device__ __forceinline__ int64_t group_sum(int64_t x, int64_t* scan) {
  x = wave_sum(x);
  __syncthreads();
  if (threadIdx.x % kWave == 0) scan[threadIdx.x / kWave] = x;
  __syncthreads();
  int64_t sum = 0;
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) sum += scan[w];
  return sum;
}
// Units of the sequences before `end`, by the whole workgroup.
template <int THREADS = 256>
__device__ __forceinline__ int64_t units_before(const SeqSet& s, int end, int unit, int64_t* scan) {
  int64_t x = 0;
  for (int b = threadIdx.x; b < end; b += THREADS) x += units_of(s, b, unit);
  return group_sum<THREADS>(x, scan);
}

// The last sequence with at most `at` units before it, and these units (at is below the sum of all).
__device__ __forceinline__ int sequence_at(const SeqSet& s, int64_t at, int unit, int64_t* before) {
  const int lane = threadIdx.x % kWave, count = (int)s.count;
  int64_t sum = 0;
  for (int b0 = 0; b0 < count; b0 += kWave) {
    const int64_t mine = b0 + lane < count ? units_of(s, b0 + lane, unit) : 0;
    int64_t to = mine;  // units up to this sequence's end
#pragma unroll
    for (int w = 1; w < kWave; w *= 2) {
      const int64_t other = __shfl_up(to, w);
      to += lane >= w ? other : 0;
    }
    const uint64_t behind = __ballot(b0 + lane < count && sum + to > at);
    if (behind) {
      const int i = __builtin_ctzll(behind);
      *before = sum + __shfl(to - mine, i);
      return __builtin_amdgcn_readfirstlane(b0 + i);
    }
    sum += __shfl(to, kWave - 1);
  }
  *before = sum;
  return count;
}

}  // namespace luna
