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

// Whether the values of keys first .. end - 1 hold any that is not finite (for all lanes).
template <typename T, int DH, int LANES>
__device__ __forceinline__ bool softmax_odd_values(const SoftmaxArgs& a, const SeqPiece& sk, int hk, int first, int end) {
  bool odd = false;
#pragma unroll 1
  for (int key = max(first, 0) + (int)threadIdx.x % LANES; key < end; key += LANES) {
    const T* v = reinterpret_cast<const T*>(seq_row(a.v, sk, a.ks.offsets != nullptr, hk, key, (int)sizeof(T)));
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

// One query row by itself, key by key in fp32, by LANES lanes of a wave.
template <typename T, int DH, int LANES>
__device__ __forceinline__ void softmax_row(const SoftmaxArgs& a, const SeqPiece& sq, const SeqPiece& sk, int head, int i) {
  constexpr int PER = (DH + LANES - 1) / LANES, esz = (int)sizeof(T);
  const bool pq = a.qs.offsets != nullptr, pk = a.ks.offsets != nullptr;
  const int lane = threadIdx.x % LANES, hk = head / (a.H / a.Hk), last = min(sk.len - 1, i + sk.len - sq.len);
  const T* q = reinterpret_cast<const T*>(seq_row(a.q, sq, pq, head, i, esz));
  float top = -__builtin_inff(), sum = 0.0f, acc[PER];
#pragma unroll
  for (int c = 0; c < PER; ++c) acc[c] = 0.0f;
#pragma unroll 1
  for (int k0 = 0; k0 <= last; k0 += LANES) {
    const int n = min(LANES, last - k0 + 1);
    const T* k = reinterpret_cast<const T*>(seq_row(a.k, sk, pk, hk, k0 + min(lane, n - 1), esz));
    float s = 0.0f;
#pragma unroll 4
    for (int c = 0; c < DH; c += 8) {
      Frag<T> qf, kf;
      load8(qf, q + c);
      load8(kf, k + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(qf.get(e), kf.get(e), s);
    }
    s = lane < n ? s * (a.scale * kLog2e) : -__builtin_inff();
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
        const T* v = reinterpret_cast<const T*>(seq_row(a.v, sk, pk, hk, k0 + min(j0 + j, n - 1), esz));
        const float pj = __shfl(p, j0 + j);
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

}  // namespace luna
