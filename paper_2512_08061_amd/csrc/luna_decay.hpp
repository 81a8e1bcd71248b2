// luna_decay.hpp -- causal linear attention with a decay for each head, in chunks: the
// kernel behind luna_decay_fwd and, with other operands, every pass of luna_decay_bwd.
//
// For row weights w_j (or 1) and, in kDecayAug, one more component a_i, b_j of queries and keys:
//
//   P_ij = f^(i - j) w_j (q_i.k_j + a_i b_j)   (j <= i; reverse: j >= i and f^(j - i)),
//   out_i = c_i sum_j P_ij v_j                 (kDecayNorm: over sum_j P_ij + eps).
//
//   forward        q = Q,  k = K,  v = V
//   dQ             q = dO, k = V,  v = K,  a_i = -dO_i.out_i, b = 1, c_i = 1 / (den_i + eps)
//   dK  (reverse)  q = V,  k = dO, v = Q,  a = 1, b_j = -dO_j.out_j, w_j = 1 / (den_j + eps)
//   dV  (reverse)  q = K,  k = Q,  v = dO, w_j as before
//
// A workgroup of four waves takes one piece of one sequence and head (and up to 128 columns
// of v) in chunks of C tokens, with the discounted state S of the tokens before the chunk
// in registers: wave w holds its columns of S (all features), as accumulator tiles.  Per chunk
//
//   P = mask(Q K^T)                    each wave 16 queries' rows, rounded to T, through LDS
//   out^T = f^(i+1) S^T Q^T + V^T P^T  each wave its columns: S's accumulator tiles are the A
//                                      operand as they are (features 4g + j of two tiles are
//                                      the 8 k-slots of a lane group; Q is read in that order)
//   S = f^C S + K^T (f^(C-1-j) w_j V)  the V operand of P's product, scaled
//
// With S returned (exact_state) the scaled V is split in three bf16 parts, so that S has fp32
// accuracy; else it is rounded to bf16 (2^-9 of each term, as S itself is as an operand).
// Denominators are sums of P before its rounding plus q.z with z in fp32 (LDS), so they have
// fp32 accuracy.
#pragma once

#include "luna_seq.hpp"
#include "luna_split.hpp"

namespace luna {

template <typename T>
constexpr int kDecayChunk = sizeof(T) == 2 ? 64 : 32;

// LDS of a workgroup: the chunk's q, k, v and P rows (padded by 16 bytes), then fp32 tables.
template <typename T, int DK, int DVW>
struct DecayLds {
  static constexpr int C = kDecayChunk<T>, PAD = 16 / (int)sizeof(T);
  static constexpr int PK = DK + PAD, PV = DVW + PAD, PA = C + PAD;
  T q[C][PK], k[C][PK], v[C][PV], p[C][PA];
  float pw[C + 4];                         // f^0 .. f^C
  float dec[C], kw[C], ka[C], qa[C], den[C];  // f^(m-1-j) w_j, w_j, b_j, a_i, denominators
  float z[DK];
};

// `m` rows of width w (at most W) into LDS rows of pitch P; rows past m and columns past w as zeros.
template <typename T, int C, int W, int P>
__device__ __forceinline__ void decay_load_rows(T* dst, const char* base, int64_t row, int m, int w, bool reverse) {
  constexpr int E = 16 / (int)sizeof(T), PER = W / E;
  static_assert(C * PER % 256 == 0, "whole pieces per thread");
  const Buf b = buffer(base, m > 0 ? (int)(((m - 1) * row + w) * (int)sizeof(T)) : 0);
#pragma unroll
  for (int i = 0; i < C * PER / 256; ++i) {
    const int idx = threadIdx.x + 256 * i, r = idx / PER, c = (idx % PER) * E;
    const int at = (reverse ? m - 1 - r : r) * (int)row + c;
    const auto x = __builtin_amdgcn_raw_buffer_load_b128(b, r < m && c < w ? at * (int)sizeof(T) : kPastEnd, 0, 0);
    *reinterpret_cast<i32x4*>(&dst[r * P + c]) = __builtin_bit_cast(i32x4, x);
  }
}

// x summed over the four lane groups
__device__ __forceinline__ float sum_groups(float x) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// The scaled values of a fragment as one operand, and their split in parts.
template <typename T>
struct DecayScaled;
template <>
struct DecayScaled<float> {
  Frag<float> x;
  __device__ __forceinline__ void set(const Frag<float>& v, const float (&w)[8], bool) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = v.v[e] * w[e];
  }
  __device__ __forceinline__ void mma_into(f32x4& c, const Frag<float>& a, bool) const { mma(c, a, x); }
};
template <>
struct DecayScaled<__bf16> {
  Split3 x;
  __device__ __forceinline__ void set(const Frag<__bf16>& v, const float (&w)[8], bool exact) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = v.get(e) * w[e];
    if (exact) {
      split3(x, y);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e += 2) x.p[0].set2(e, y[e], y[e + 1]);
    }
  }
  __device__ __forceinline__ void mma_into(f32x4& c, const Frag<__bf16>& a, bool exact) const {
    if (exact) {
      mma(c, a, x.p[2]);
      mma(c, a, x.p[1]);
    }
    mma(c, a, x.p[0]);
  }
};

template <typename T, int DK, int DVW, int MODE, bool OUT>
__global__ __launch_bounds__(256) void decay_kernel(DecayArgs a) {
  using Lds = DecayLds<T, DK, DVW>;
  constexpr int C = Lds::C, FT = DK / 16, CT = DVW / 64, KT = C / 16, KS = C / 32;
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);

  const int tid = threadIdx.x, lane = tid % kWave, wave = wave_id();
  const int g = lane / 16, c = lane % 16;
  const int slices = (a.dv + DVW - 1) / DVW;
  const int slice = blockIdx.x % slices, head = (blockIdx.x / slices) % a.H, slot = blockIdx.x / slices / a.H;
  const SeqPiece sp = seq_piece(a.s, slot, a.piece);
  if (sp.seq < 0) return;
  const bool packed = a.s.offsets != nullptr, rev = a.reverse;
  const int begin = sp.index * a.piece, end = min(sp.len, begin + a.piece);
  if (!OUT && end == sp.len) return;  // (nothing starts from the state after the last piece)
  const int col0 = slice * DVW, cols = min(DVW, a.dv - col0);
  const int wcol = 16 * CT * wave;  // this wave's first column of the slice
  const bool exact = a.exact_state;

  const float g2 = decay_log2(a.log_decay[head]);
  for (int i = tid; i <= C; i += 256) l.pw[i] = exp2f(g2 * (float)i);

  // the state before the piece
  const int64_t sf = decay_state_floats(a.dk, a.dv);
  float* st = a.states ? a.states + ((int64_t)slot * a.H + head) * sf : nullptr;
  f32x4 S[FT][CT], za[CT];  // za: row 0 is the further key component's row of S (kDecayAug)
  const float* S0 = nullptr;
  const float* z0 = nullptr;
  if (OUT) {
    const int64_t at = (int64_t)sp.seq * a.H + head;
    if (a.states) {
      if (begin > 0 || a.S) S0 = st, z0 = st + (int64_t)a.dk * a.dv;
    } else if (a.S) {
      S0 = a.S + at * a.dk * a.dv;
      z0 = MODE == kDecayNorm ? a.z + at * a.dk : nullptr;
    }
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = wcol + 16 * ct + c;
#pragma unroll
    for (int ft = 0; ft < FT; ++ft)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int f = 16 * ft + 4 * g + j;
        S[ft][ct][j] = S0 && f < a.dk && col < cols ? S0[(int64_t)f * a.dv + col0 + col] : 0.0f;
      }
    za[ct] = zero4();
    if (MODE == kDecayAug && S0 && g == 0 && col < cols) za[ct][0] = z0[col0 + col];
  }
  if (MODE == kDecayNorm)
    for (int f = tid; f < DK; f += 256) l.z[f] = S0 && f < a.dk ? z0[f] : 0.0f;

  for (int t0 = begin; t0 < end; t0 += C) {
    const int m = min(C, end - t0);
    const int64_t lo = rev ? sp.len - t0 - m : t0;  // the chunk's first row in memory
    constexpr int esz = (int)sizeof(T);
    __syncthreads();  // the chunk before is no longer read
    if (OUT) decay_load_rows<T, C, DK, Lds::PK>(&l.q[0][0], seq_row(a.q, sp, packed, head, lo, esz), a.q.row, m, a.dk, rev);
    decay_load_rows<T, C, DK, Lds::PK>(&l.k[0][0], seq_row(a.k, sp, packed, head, lo, esz), a.k.row, m, a.dk, rev);
    decay_load_rows<T, C, DVW, Lds::PV>(&l.v[0][0], seq_row(a.v, sp, packed, head, lo, esz) + col0 * esz, a.v.row, m, cols, rev);
    if (tid < C) {
      const bool in = tid < m;
      const int64_t num = seq_num(a.s, sp, a.H, head, lo + (rev ? m - 1 - tid : tid));
      const float w = !in ? 0.0f : a.kw ? a.kw[num] : 1.0f;
      l.kw[tid] = w;
      l.dec[tid] = in ? w * exp2f(g2 * (float)(m - 1 - tid)) : 0.0f;
      if (MODE == kDecayAug) {
        l.ka[tid] = !in ? 0.0f : a.ka ? a.ka[num] : 1.0f;
        l.qa[tid] = !in ? 0.0f : a.qa ? a.qa[num] : 1.0f;
      }
    }
    __syncthreads();

    f32x4 o[KT][CT];
    if (OUT) {
      // P: wave w forms the rows of query tile w, over the keys before them
      if (wave < KT) {
        const int qt = wave, i = 16 * qt + c;
        Frag<T> qf[DK / 32];
#pragma unroll
        for (int t = 0; t < DK / 32; ++t) load8(qf[t], &l.q[i][32 * t + 8 * g]);
        float den = 0.0f;
        if (MODE == kDecayNorm) {
#pragma unroll
          for (int t = 0; t < DK / 32; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) den = fmaf(qf[t].get(e), l.z[32 * t + 8 * g + e], den);
          den *= l.pw[i + 1];
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          f32x4 acc = zero4();
          if (kt <= qt) {
#pragma unroll
            for (int t = 0; t < DK / 32; ++t) {
              Frag<T> kf;
              load8(kf, &l.k[16 * kt + c][32 * t + 8 * g]);
              mma(acc, kf, qf[t]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int key = 16 * kt + 4 * g + j;
              float x = acc[j];
              if (MODE == kDecayAug) x = fmaf(l.qa[i], l.ka[key], x);
              x *= l.pw[max(i - key, 0)] * l.kw[key];
              acc[j] = key <= i ? x : 0.0f;
              if (MODE == kDecayNorm) den += acc[j];
            }
          }
          if (kt <= qt + 1) store4(&l.p[i][16 * kt + 4 * g], acc[0], acc[1], acc[2], acc[3]);
        }
        if (MODE == kDecayNorm) {
          den = sum_groups(den);
          if (g == 0) l.den[i] = den;
        }
      }
      // f^(i+1) S^T Q^T
#pragma unroll
      for (int qt = 0; qt < KT; ++qt)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) o[qt][ct] = zero4();
#pragma unroll
      for (int t = 0; t < FT / 2; ++t) {
        Frag<T> sf_[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            sf_[ct].set2(e, S[2 * t][ct][e], S[2 * t][ct][e + 1]);
            sf_[ct].set2(4 + e, S[2 * t + 1][ct][e], S[2 * t + 1][ct][e + 1]);
          }
#pragma unroll
        for (int qt = 0; qt < KT; ++qt) {
          Frag<T> qf;
          load4(qf, 0, &l.q[16 * qt + c][32 * t + 4 * g]);
          load4(qf, 4, &l.q[16 * qt + c][32 * t + 16 + 4 * g]);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) mma(o[qt][ct], sf_[ct], qf);
        }
      }
      if (MODE == kDecayAug) {
#pragma unroll
        for (int qt = 0; qt < KT; ++qt) {
          Frag<T> qf;
          qf.zero();
          qf.set(0, g == 0 ? l.qa[16 * qt + c] : 0.0f);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            Frag<T> zf;
            zf.zero();
            zf.set(0, g == 0 ? za[ct][0] : 0.0f);
            mma(o[qt][ct], zf, qf);
          }
        }
      }
#pragma unroll
      for (int qt = 0; qt < KT; ++qt) {
        const float f = l.pw[16 * qt + c + 1];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[qt][ct][j] *= f;
      }
      __syncthreads();  // P is whole; z has been read
    }

    // V^T P^T, and the state after the chunk
    {
      const float f = l.pw[m];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
        for (int ft = 0; ft < FT; ++ft)
#pragma unroll
          for (int j = 0; j < 4; ++j) S[ft][ct][j] *= f;
        za[ct][0] *= f;
      }
    }
    f32x4 zacc[(FT + 3) / 4];
    if (MODE == kDecayNorm)
#pragma unroll
      for (int i = 0; i < (FT + 3) / 4; ++i) zacc[i] = zero4();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float dec[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) dec[e] = l.dec[32 * ks + 8 * g + e];
      Frag<T> vf[CT];
      DecayScaled<T> vs[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        load_tr4(vf[ct], 0, &l.v[0][0], Lds::PV, 32 * ks + 8 * g, wcol + 16 * ct, lane);
        load_tr4(vf[ct], 4, &l.v[0][0], Lds::PV, 32 * ks + 8 * g + 4, wcol + 16 * ct, lane);
        vs[ct].set(vf[ct], dec, exact);
      }
      if (OUT) {
#pragma unroll
        for (int qt = 2 * ks; qt < KT; ++qt) {
          Frag<T> pf;
          load8(pf, &l.p[16 * qt + c][32 * ks + 8 * g]);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) mma(o[qt][ct], vf[ct], pf);
        }
      }
      DecayScaled<T> one;  // columns 0 .. 2: the parts of the discounts
      if (MODE == kDecayNorm) {
        if constexpr (sizeof(T) == 2) {
          Split3 parts;
          split3(parts, dec);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            one.x.p[0].v[e] = c == 0 ? parts.p[0].v[e] : c == 1 ? parts.p[1].v[e] : c == 2 ? parts.p[2].v[e] : (__bf16)0.0f;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) one.x.v[e] = c == 0 ? dec[e] : 0.0f;
        }
      }
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) {
        Frag<T> kf;
        load_tr4(kf, 0, &l.k[0][0], Lds::PK, 32 * ks + 8 * g, 16 * ft, lane);
        load_tr4(kf, 4, &l.k[0][0], Lds::PK, 32 * ks + 8 * g + 4, 16 * ft, lane);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) vs[ct].mma_into(S[ft][ct], kf, exact);
        if (MODE == kDecayNorm)
          if (ft % 4 == wave) one.mma_into(zacc[ft / 4], kf, false);
      }
      if (MODE == kDecayAug) {
        Frag<T> kf;
        kf.zero();
#pragma unroll
        for (int e = 0; e < 8; ++e) kf.set(e, c == 0 ? l.ka[32 * ks + 8 * g + e] : 0.0f);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) vs[ct].mma_into(za[ct], kf, exact);
      }
    }
    if (MODE == kDecayNorm) {
#pragma unroll
      for (int i = 0; i < (FT + 3) / 4; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // the three parts' columns, in every quad of lanes
          float x = zacc[i][j];
          x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xf, 0xf, true));
          x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xf, 0xf, true));
          const int f = 16 * (4 * i + wave) + 4 * g + j;
          if (c == 0 && f < DK) l.z[f] = fmaf(l.pw[m], l.z[f], x);
        }
      }
    }

    if (OUT) {
      const Buf b = buffer(seq_row(a.o, sp, packed, head, lo, esz) + col0 * esz, (int)(((m - 1) * a.o.row + cols) * esz));
#pragma unroll
      for (int qt = 0; qt < KT; ++qt) {
        const int i = 16 * qt + c, r = rev ? m - 1 - i : i;
        float f = a.scale;
        if (MODE == kDecayNorm) {
          const float den = a.scale * l.den[i];
          f = a.scale / (den + a.eps);
          if (a.den && wave == 0 && g == 0 && slice == 0 && i < m) a.den[seq_num(a.s, sp, a.H, head, lo + r)] = den;
        }
        if (a.ow && i < m) f *= a.ow[seq_num(a.s, sp, a.H, head, lo + r)];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const int col = wcol + 16 * ct + 4 * g;
          buf_store4<T>(b, i < m && col < cols ? (r * (int)a.o.row + col) * esz : kPastEnd, f * o[qt][ct][0],
                        f * o[qt][ct][1], f * o[qt][ct][2], f * o[qt][ct][3]);
        }
      }
    }
  }

  // the state after the piece: to the next piece's prefix (state pass), or after the sequence's last token
  float* S1 = nullptr;
  float* z1 = nullptr;
  if (!OUT) {
    S1 = st;
    z1 = st + (int64_t)a.dk * a.dv;
  } else if (a.S && end == sp.len) {
    const int64_t at = (int64_t)sp.seq * a.H + head;
    S1 = a.S + at * a.dk * a.dv;
    z1 = MODE == kDecayNorm ? a.z + at * a.dk : nullptr;
  }
  if (!S1) return;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = wcol + 16 * ct + c;
    if (col < cols) {
#pragma unroll
      for (int ft = 0; ft < FT; ++ft)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int f = 16 * ft + 4 * g + j;
          if (f < a.dk) S1[(int64_t)f * a.dv + col0 + col] = S[ft][ct][j];
        }
      if (MODE == kDecayAug && g == 0) z1[col0 + col] = za[ct][0];
    }
  }
  if (MODE == kDecayNorm && slice == 0) {
    __syncthreads();
    for (int f = tid; f < a.dk; f += 256) z1[f] = l.z[f];
  }
}

template <typename T, int DK, int DVW, int MODE, bool OUT>
hipError_t launch_decay_one(const DecayArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(DecayLds<T, DK, DVW>);
  static_assert(bytes <= 160 * 1024, "one workgroup's LDS");
  const hipError_t e = allow_lds<decay_kernel<T, DK, DVW, MODE, OUT>>(bytes);
  if (e != hipSuccess) return e;
  const int slices = (a.dv + DVW - 1) / DVW;
  hipLaunchKernelGGL((decay_kernel<T, DK, DVW, MODE, OUT>), dim3((unsigned)((int64_t)a.slots * a.H * slices)), dim3(256),
                     bytes, s, a);
  return hipGetLastError();
}

template <typename T, int DK, int MODE, bool OUT>
hipError_t launch_decay_width(const DecayArgs& a, hipStream_t s) {
  return a.dv <= 64 ? launch_decay_one<T, DK, 64, MODE, OUT>(a, s) : launch_decay_one<T, DK, 128, MODE, OUT>(a, s);
}

template <typename T, int MODE, bool OUT>
hipError_t launch_decay_mode(const DecayArgs& a, hipStream_t s) {
  return a.dk <= 64    ? launch_decay_width<T, 64, MODE, OUT>(a, s)
         : a.dk <= 128 ? launch_decay_width<T, 128, MODE, OUT>(a, s)
                       : launch_decay_width<T, 256, MODE, OUT>(a, s);
}

// one translation unit per element type and mode (luna_decay_*.hip)
template <typename T, int MODE>
hipError_t launch_decay_typed(const DecayArgs& a, bool out, hipStream_t s);
#define LUNA_DECAY_TYPED(T, MODE)                                                     \
  template <>                                                                         \
  hipError_t launch_decay_typed<T, MODE>(const DecayArgs& a, bool out, hipStream_t s) { \
    return out ? launch_decay_mode<T, MODE, true>(a, s) : launch_decay_mode<T, MODE, false>(a, s); \
  }

}  // namespace luna
