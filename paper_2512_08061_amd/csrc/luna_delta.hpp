// luna_delta.hpp -- linear attention by the gated delta rule: what its kernels and the host share
// (luna_delta_*.hip, luna_delta_api.cpp).
//
// Per sequence and head, with a_t = exp(log_decay) of the token and its beta,
//
//   u_t = beta_t (v_t - a_t S_{t-1}^T k_t),  S_t = a_t S_{t-1} + k_t u_t^T,  out_t = scale S_t^T q_t.
//
// A chunk of C = 64 tokens from the state S before it, with G the sums of log decays within it:
//
//   M_ij = e^(G_i - G_j) k_i.k_j  (j < i),   P_ij = scale e^(G_i - G_j) q_i.k_j  (j <= i),
//   R = V - e^G K S,   E = R - M U,  U = beta E   =>   E = R + N (beta R),   N = -M (I + beta M)^-1,
//   out = scale e^G Q S + P U,   S' = e^(G_C) S + K^T (e^(G_C - G) U).
//
// N is strictly lower triangular and so are its factors; it serves the backward pass as well, where from dS' (of the
// state behind the chunk)
//
//   dU = P^T dO + e^(G_C - G) K dS',   X = dU + N^T (beta dU),   dV = beta X,   dbeta = X.E,
//   dS = e^(G_C) dS' + Q^T (scale e^G dO) - K^T (e^G beta X).
//
// N, P and the factors of the gates need no state; what is left is serial in the chunks but independent for each value
// column, so a wave takes 16 columns of one head from the first chunk to the last.  The bf16 forward pass forms the matrices in
// the workgroups that use them (luna_delta_fwd.hip); the fp32 and backward passes for all chunks at once before
// (luna_delta_gates.hip, luna_delta_scan.hpp, luna_delta_grads.hip).
#pragma once

#include "luna_decay.hpp"

namespace luna {

constexpr int kDeltaChunk = 64;

// Per chunk and head: rows of 64 numbers.
constexpr int kDeltaFirst = 0;  // e^G
constexpr int kDeltaLast = 1;   // e^(G_C - G)
constexpr int kDeltaBeta = 2;
constexpr int kDeltaMisc = 3;  // e^(G_C), then (an int) the first token with a key or gate that is not finite, or 64
constexpr int kDeltaHigh = 4, kDeltaLow = 5;  // G / ln 2 in two parts, so that differences keep their accuracy
constexpr int kDeltaGateRows = 6, kDeltaGates = kDeltaGateRows * kDeltaChunk;

// Parts of bf16 that fp32 operands of bf16 calls are split in: two (2^-17 of each operand), three (2^-24) where the
// state is returned and in the backward pass, whose gradients of the gates are fp32 sums that cancel in part.  P is an operand
// of `out` alone in the forward pass and is rounded once there.
constexpr int kDeltaParts = 2, kDeltaExactParts = 3, kDeltaBackParts = 3;

// Workgroups of the gradients' kernel, and of the serial ones in fp32 and of the backward pass, that run at once: one a compute unit.
constexpr int64_t kDeltaUnits = 256;
// Whether each value head of a key head's chunks has a workgroup of its own there (luna_delta_grads.hip), where its states have room for
// its dQ and dK: where the compute units then take at most three quarters of the turns that they take when a workgroup adds up its
// heads one after the other.  The whole backward pass, D = d = 128, us, one after the other first: 176 tokens, 32 heads on 4, 345 and
// 124 in fp32, 214 and 96 in bf16; 2000 tokens, 32 on 1, 1528 and 620, 945 and 430; 4800 tokens, 16 on 4 (300 chunks and key heads:
// 8 turns and 5), 961 and 893, 514 and 480; but two of 3600 (452: 8 and 8) 826 and 873, 474 and 514, two of 4800 (600: 12 and 10) 1130
// and 1125, 648 and 665.
inline bool delta_grads_apart(int64_t chunks, int64_t group) {
  const auto turns = [](int64_t groups) { return (groups + kDeltaUnits - 1) / kDeltaUnits; };
  return 4 * turns(chunks * group) <= 3 * turns(chunks) * group && chunks * group < ((int64_t)1 << 22);  // (within a launch)
}

// Whether these serial kernels take 32 value columns a workgroup, with two waves that load, or 64, of which all waves load (groups:
// workgroups of 32): the first where they run at once, since a chunk passes in less time; with D < 128 and lengths that may differ up to
// twice as many, since the longest sequence's chain counts then and short ones leave room.  us, 32 columns first, backward unless said:
//   equal lengths, 16 heads of 2048 tokens, D = d = 128: two in bf16 282 and 338, three 428 and 426, eight 1028 and 931; in fp32 488
//     and 562, 756 and 682, 1692 and 1456;
//   8 x 1000, 12 heads, d = 64 (384): D = 64 in fp32 286 and 258, in bf16 202 and 193; D = 32 207 and 206, 188 and 181; forward in fp32,
//     384 of 1024 tokens, D = 64 267 and 204, D = 32 181 and 156;
//   packed 33 to 1500, 12 heads, d = 64 (384): D = 64 in fp32 227 and 259, in bf16 156 and 185; D = 32 185 and 206, 142 and 173; forward
//     in fp32, 20 to 1500, 16 heads (384), D = 64 181 and 211, D = 32 141 and 159; but packed 800 to 1100 (384) 288 and 272 in fp32.
inline bool delta_narrow(int64_t D, int64_t d, int64_t groups, bool equal) {
  return d == 32 || groups <= kDeltaUnits * (D < 128 && !equal ? 2 : 1);
}

struct DeltaArgs {
  SeqRows q, k, v, o;  // widths D, D, d, d; o: out, or dO in the backward pass
  SeqSet s;
  const float* log_decay;  // per row
  const float* beta;
  int H, Hk, D, d;
  int slots;    // chunks of all sequences (seq_slots)
  float scale;
  float* S;     // [count][H][D][d], in and out, or null
  // workspace, per slot and head
  char* n;      // [parts][64][64] of the call's type
  char* p;      // the same
  float* gates; // [kDeltaGates]
  float* before;  // backward: [d][D] state before the chunk
  float* after;   // [d][D] gradient of the state behind it
  float* e;       // [d][64]
  float* x;       // [d][64]
  // gradients
  SeqRows dq, dk, dv;
  float* dlog_decay;
  float* dbeta;
};

// Slot of the first chunk of a sequence.
__device__ __forceinline__ int delta_first_slot(const SeqSet& s, const SeqPiece& p) {
  return s.offsets ? (int)(p.first / kDeltaChunk) + p.seq : p.seq * (int)((s.rows + kDeltaChunk - 1) / kDeltaChunk);
}

// x of the lanes of a row of 16, or of a row's last lane, that a DPP control names; zeros where there is none.  (No LDS, unlike a shuffle.)
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, ROWS == 0xf));
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CTRL, ROWS, 0xf, ROWS == 0xf);
  const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CTRL, ROWS, 0xf, ROWS == 0xf);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Sums over the lanes up to this one.
template <typename F>
__device__ __forceinline__ F lane_sums(F x) {
  x += dpp<0x111>(x);       // a lane before in the row
  x += dpp<0x112>(x);       // two
  x += dpp<0x114>(x);       // four
  x += dpp<0x118>(x);       // eight
  x += dpp<0x142, 0xa>(x);  // the last lane of the row before, for rows 1 and 3
  x += dpp<0x143, 0xc>(x);  // lane 31, for rows 2 and 3
  return x;
}
// Sum over the 16 lanes of a row.
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xb1>(x);   // lane 1, 0, 3, 2 of four
  x += dpp<0x4e>(x);   // lane 2, 3, 0, 1
  x += dpp<0x141>(x);  // the other four of eight
  x += dpp<0x140>(x);  // the other eight
  return x;
}
__device__ __forceinline__ double of_lane(double x, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const unsigned lo = __builtin_amdgcn_readlane((int)(unsigned)u, lane), hi = __builtin_amdgcn_readlane((int)(unsigned)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float of_lane(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }

// An fp32 operand as products of type T take it: itself, or P parts in bf16.
template <typename T, int P>
struct DeltaOp;
template <int P>
struct DeltaOp<float, P> {
  Frag<float> x;
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = v[e];
  }
};
template <int P>
struct DeltaOp<__bf16, P> {
  Frag<__bf16> p[P];
  __device__ __forceinline__ void set(const float (&v)[8]) {
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = v[e];
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        p[k].set2(e, r[e], r[e + 1]);
        r[e] -= p[k].get(e);
        r[e + 1] -= p[k].get(e + 1);
      }
  }
};
template <typename T, int P>
__device__ __forceinline__ void set_tiles(DeltaOp<T, P>& o, const f32x4& lo, const f32x4& hi) {
  const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  o.set(v);
}
template <int P>
__device__ __forceinline__ void mma(f32x4& c, const Frag<float>& a, const DeltaOp<float, P>& b) { mma(c, a, b.x); }
template <int P>
__device__ __forceinline__ void mma(f32x4& c, const DeltaOp<float, P>& a, const Frag<float>& b) { mma(c, a.x, b); }
template <int P>
__device__ __forceinline__ void mma(f32x4& c, const Frag<__bf16>& a, const DeltaOp<__bf16, P>& b) {
#pragma unroll
  for (int k = P - 1; k >= 0; --k) mma(c, a, b.p[k]);
}
template <int P>
__device__ __forceinline__ void mma(f32x4& c, const DeltaOp<__bf16, P>& a, const Frag<__bf16>& b) {
#pragma unroll
  for (int k = P - 1; k >= 0; --k) mma(c, a.p[k], b);
}
template <int P, int Q>
__device__ __forceinline__ void mma(f32x4& c, const DeltaOp<float, P>& a, const DeltaOp<float, Q>& b) { mma(c, a.x, b.x); }
// (products of parts that are below what the others leave out are left out)
template <int P, int Q>
__device__ __forceinline__ void mma(f32x4& c, const DeltaOp<__bf16, P>& a, const DeltaOp<__bf16, Q>& b) {
  constexpr int MOST = (P > Q ? P : Q) - 1;
#pragma unroll
  for (int k = MOST; k >= 0; --k)
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (k - i >= 0 && k - i < Q) mma(c, a.p[i], b.p[k - i]);
}

// LDS by byte addresses: what differs between lanes is worked out once, the rest lies in the instructions' offsets.
__device__ __forceinline__ unsigned lds_address(const void* p) {
  return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
__device__ __forceinline__ void lds8(Frag<__bf16>& f, unsigned at) {
  f.v = *(__attribute__((address_space(3))) const bf16x8*)(uintptr_t)at;
}
__device__ __forceinline__ void lds8_store(unsigned at, const Frag<__bf16>& f) { *(__attribute__((address_space(3))) bf16x8*)(uintptr_t)at = f.v; }
__device__ __forceinline__ f32x4 lds4(unsigned at) { return *(__attribute__((address_space(3))) const f32x4*)(uintptr_t)at; }
// eight rows of a column, four and four `step` bytes apart
__device__ __forceinline__ void lds_tr(Frag<__bf16>& f, unsigned at, int step) {
  typedef __attribute__((ext_vector_type(4))) short i16x4;
  const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)at);
  const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)(at + step));
  f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The parts of an operand in LDS: [parts][rows][pitch].
template <typename T>
constexpr int delta_parts(int p) { return sizeof(T) == 2 ? p : 1; }
template <int P>
__device__ __forceinline__ void load_op(DeltaOp<float, P>& o, const float* x, int) { load8(o.x, x); }
template <int P>
__device__ __forceinline__ void load_op(DeltaOp<__bf16, P>& o, const __bf16* x, int part) {
#pragma unroll
  for (int k = 0; k < P; ++k) load8(o.p[k], x + k * part);
}
// slots e0 .. e0 + 3 from four rows of a column (see load_tr4_at)
template <int P, typename F>
__device__ __forceinline__ void load_op_tr4(DeltaOp<float, P>& o, int e0, int lane, int, F at) { load_tr4_at(o.x, e0, lane, at); }
template <int P, typename F>
__device__ __forceinline__ void load_op_tr4(DeltaOp<__bf16, P>& o, int e0, int lane, int part, F at) {
#pragma unroll
  for (int k = 0; k < P; ++k) load_tr4_at(o.p[k], e0, lane, [&](int kk, int col) { return at(kk, col) + k * part; });
}
// four consecutive elements as parts
template <int P>
__device__ __forceinline__ void store_parts4(float* x, int, float a, float b, float c, float d) { store4(x, a, b, c, d); }
template <int P>
__device__ __forceinline__ void store_parts4(__bf16* x, int part, float a, float b, float c, float d) {
#pragma unroll
  for (int k = 0; k < P; ++k) {
    store4(x + k * part, a, b, c, d);
    a -= (float)(__bf16)a, b -= (float)(__bf16)b, c -= (float)(__bf16)c, d -= (float)(__bf16)d;
  }
}

// N, P and the gates' factors of all chunks to the workspace
hipError_t launch_delta_gates(Dt dt, const DeltaArgs& a, hipStream_t s);
// out and the state: in bf16 all in one launch (exact: the state to fp32 accuracy), in fp32 behind the gates' launch
hipError_t launch_delta_fwd_bf16(bool exact, const DeltaArgs& a, hipStream_t s);
hipError_t launch_delta_fwd_f32(const DeltaArgs& a, hipStream_t s);
// the backward pass: E and the states before the chunks, X and the gradients of the states behind them; the gradients
hipError_t launch_delta_both(Dt dt, const DeltaArgs& a, hipStream_t s);
hipError_t launch_delta_grads(Dt dt, const DeltaArgs& a, hipStream_t s);
struct DeltaStepArgs {
  SeqRows q, k, v, o;
  const float* log_decay;  // [count][H][m]
  const float* beta;
  int64_t count;
  int m, H, Hk, D, d;
  float scale;
  float* S;
};
hipError_t launch_delta_step(Dt dt, const DeltaStepArgs& a, hipStream_t s);

}  // namespace luna
