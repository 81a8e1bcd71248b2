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
__device__ __forceinline__ float groups_sum(float x) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
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

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kSoftmaxTile = 64;  // query rows (key rows) of a workgroup

// keys per step of the tile kernels: the staged rows of two tensors fit 64 KiB and a bit
template <typename T>
constexpr int kSoftmaxStep = sizeof(T) == 2 ? 64 : 32;

}  // namespace luna
