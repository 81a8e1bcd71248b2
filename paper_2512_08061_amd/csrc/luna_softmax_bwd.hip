// luna_softmax_bwd.hip -- causal softmax attention, backward.  With P_ij = exp(s_ij - lse_i) and
// D_i = dO_i.out_i:
//
//   dS_ij = P_ij (dO_i.v_j - D_i),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
//
// Two kernels, each forming the scores again, so that every sum belongs to one workgroup: no
// atomics, the same bits at every call.  The query pass owns 64 queries of a head and meets their
// keys (S^T = K Q^T and dP^T = V dO^T as in the forward pass; dS^T is the B operand of
// dQ^T = K^T dS^T); it also forms D and leaves it for the key pass, which owns 64 keys of a key
// head and meets the queries that see them, for every query head of the group in turn (S = Q K^T and
// dP = dO V^T, lane (g, c): queries 4g + j of key c; P and dS are the B operands of dV^T = dO^T P
// and dK^T = Q^T dS).
#include "luna_softmax.hpp"

namespace luna {

namespace {

// A weight 2^x times 2^SHIFT, at most 2^SHIFT (NaN stays NaN).  lse carries a few roundings to 2^-24 of itself, which for
// scores of millions is no longer a small number: without the limit rows of scores about 10^7 had weights above 2,
// infinite in fp16, and larger ones any factor too much.
template <int SHIFT = 0>
__device__ __forceinline__ float weight(float x) {
  return exp2_raw(__builtin_elementwise_minimum(x, (float)SHIFT));
}

template <typename T, int DH>
struct SoftmaxBwdLds {
  static constexpr int KB = kSoftmaxStep<T>, P = DH + 16 / (int)sizeof(T);
  T x[KB][P], y[KB][P];
  float lse[KB], delta[KB];
};

template <typename T, int DH>
__global__ __launch_bounds__(256) void softmax_dq_kernel(SoftmaxArgs a) {
  using Lds = SoftmaxBwdLds<T, DH>;
  constexpr int KB = Lds::KB, P = Lds::P, KT = KB / 16, CT = DH / 16, esz = (int)sizeof(T);
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id(), g = lane / 16, c = lane % 16;
  const int head = blockIdx.x % a.H;
  const SeqPiece sq = seq_piece_by_work(a.qs, blockIdx.x / a.H, gridDim.x / a.H, kSoftmaxTile, true);
  if (sq.seq < 0) return;
  const SeqPiece sk = seq_of(a.ks, sq.seq);
  const bool pq = a.qs.offsets != nullptr, pk = a.ks.offsets != nullptr;
  const int q0 = sq.index * kSoftmaxTile, m = min(kSoftmaxTile, sq.len - q0);
  const int shift = sk.len - sq.len;
  const int kend = min(sk.len, max(0, q0 + m + shift));
  const int i = 16 * wave + c, last = q0 + i + shift;
  const int hk = head / (a.H / a.Hk);
  const int64_t num = seq_num(a.qs, sq, a.H, head, q0 + i);

  Frag<T> qf[DH / 32], gf[DH / 32], of[DH / 32];
  softmax_load_frags<T, DH>(qf, seq_row(a.q, sq, pq, head, q0, esz), a.q.row, m, i, g);
  softmax_load_frags<T, DH>(gf, seq_row(a.dO, sq, pq, head, q0, esz), a.dO.row, m, i, g);
  softmax_load_frags<T, DH>(of, seq_row(a.o, sq, pq, head, q0, esz), a.o.row, m, i, g);
  float delta = 0.0f;
#pragma unroll
  for (int t = 0; t < DH / 32; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) delta = fmaf(gf[t].get(e), of[t].get(e), delta);
  delta = groups_sum(delta);
  if (g == 0 && i < m) a.delta[num] = delta;
  const float lse = i < m ? a.lse[num] * kLog2e : 0.0f;
  const float scale = a.scale * kLog2e;
  f32x4 dq[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) dq[t] = zero4();

  for (int k0 = 0; k0 < kend; k0 += KB) {
    const int kn = min(KB, kend - k0);
    __syncthreads();
    softmax_load_rows<T, KB, DH, P>(&l.x[0][0], seq_row(a.k, sk, pk, hk, k0, esz), a.k.row, kn);
    softmax_load_rows<T, KB, DH, P>(&l.y[0][0], seq_row(a.v, sk, pk, hk, k0, esz), a.v.row, kn);
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < KT / 2; ++ks) {
      Frag<T> ds;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int kt = 2 * ks + h;
        f32x4 s = zero4(), dp = zero4();
#pragma unroll
        for (int t = 0; t < DH / 32; ++t) {
          Frag<T> kf, vf;
          load8(kf, &l.x[16 * kt + c][32 * t + 8 * g]);
          load8(vf, &l.y[16 * kt + c][32 * t + 8 * g]);
          mma(s, kf, qf[t]);
          mma(dp, vf, gf[t]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = k0 + 16 * kt + 4 * g + j;
          const bool seen = key <= last && key < kend;
          const float e = weight(fmaf(s[j], scale, -lse)) * (dp[j] - delta);
          s[j] = seen ? e : 0.0f;
        }
        ds.set2(4 * h, s[0], s[1]);
        ds.set2(4 * h + 2, s[2], s[3]);
      }
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        Frag<T> kf;
        load_tr4(kf, 0, &l.x[0][0], P, 32 * ks + 4 * g, 16 * t, lane);
        load_tr4(kf, 4, &l.x[0][0], P, 32 * ks + 16 + 4 * g, 16 * t, lane);
        mma(dq[t], kf, ds);
      }
    }
  }
  const Buf b = buffer(seq_row(a.dq, sq, pq, head, q0, esz), (int)(((m - 1) * a.dq.row + DH) * esz));
#pragma unroll
  for (int t = 0; t < CT; ++t)
    buf_store4<T>(b, i < m ? (i * (int)a.dq.row + 16 * t + 4 * g) * esz : kPastEnd, dq[t][0] * a.scale, dq[t][1] * a.scale,
                  dq[t][2] * a.scale, dq[t][3] * a.scale);
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void softmax_dkdv_kernel(SoftmaxArgs a) {
  using Lds = SoftmaxBwdLds<T, DH>;
  constexpr int KB = Lds::KB, P = Lds::P, KT = KB / 16, CT = DH / 16, esz = (int)sizeof(T);
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id(), g = lane / 16, c = lane % 16;
  const int hk = blockIdx.x % a.Hk;
  const SeqPiece sk = seq_piece_by_work(a.ks, blockIdx.x / a.Hk, gridDim.x / a.Hk, kSoftmaxTile, false);
  if (sk.seq < 0) return;
  const SeqPiece sq = seq_of(a.qs, sk.seq);
  const bool pq = a.qs.offsets != nullptr, pk = a.ks.offsets != nullptr;
  const int k0 = sk.index * kSoftmaxTile, m = min(kSoftmaxTile, sk.len - k0);
  const int shift = sk.len - sq.len;
  const int key = k0 + 16 * wave + c, i = 16 * wave + c;
  const int qbegin = max(0, k0 - shift) / KB * KB;  // the first query that sees the tile's first key

  Frag<T> kf[DH / 32], vf[DH / 32];
  softmax_load_frags<T, DH>(kf, seq_row(a.k, sk, pk, hk, k0, esz), a.k.row, m, i, g);
  softmax_load_frags<T, DH>(vf, seq_row(a.v, sk, pk, hk, k0, esz), a.v.row, m, i, g);
  const float scale = a.scale * kLog2e;
  f32x4 dk[CT], dv[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) dk[t] = dv[t] = zero4();

  const int group = a.H / a.Hk;
  for (int head = hk * group; head < (hk + 1) * group; ++head) {
    for (int q0 = qbegin; q0 < sq.len; q0 += KB) {
      const int qn = min(KB, sq.len - q0);
      __syncthreads();
      softmax_load_rows<T, KB, DH, P>(&l.x[0][0], seq_row(a.q, sq, pq, head, q0, esz), a.q.row, qn);
      softmax_load_rows<T, KB, DH, P>(&l.y[0][0], seq_row(a.dO, sq, pq, head, q0, esz), a.dO.row, qn);
      if (threadIdx.x < KB) {
        const bool in = threadIdx.x < qn;
        const int64_t num = seq_num(a.qs, sq, a.H, head, q0 + (int)threadIdx.x);
        l.lse[threadIdx.x] = in ? a.lse[num] * kLog2e : 0.0f;
        l.delta[threadIdx.x] = in ? a.delta[num] : 0.0f;
      }
      __syncthreads();
#pragma unroll
      for (int ks = 0; ks < KT / 2; ++ks) {
        Frag<T> pf, ds;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int qt = 2 * ks + h;
          f32x4 s = zero4(), dp = zero4(), p;
          const f32x4 lse = *reinterpret_cast<const f32x4*>(&l.lse[16 * qt + 4 * g]);
          const f32x4 delta = *reinterpret_cast<const f32x4*>(&l.delta[16 * qt + 4 * g]);
#pragma unroll
          for (int t = 0; t < DH / 32; ++t) {
            Frag<T> qf, gf;
            load8(qf, &l.x[16 * qt + c][32 * t + 8 * g]);
            load8(gf, &l.y[16 * qt + c][32 * t + 8 * g]);
            mma(s, qf, kf[t]);
            mma(dp, gf, vf[t]);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int r = 16 * qt + 4 * g + j, query = q0 + r;
            const bool seen = key <= query + shift && r < qn && i < m;
            const float e = weight(fmaf(s[j], scale, -lse[j]));
            p[j] = seen ? e : 0.0f;
            s[j] = seen ? e * (dp[j] - delta[j]) : 0.0f;
          }
          pf.set2(4 * h, p[0], p[1]);
          pf.set2(4 * h + 2, p[2], p[3]);
          ds.set2(4 * h, s[0], s[1]);
          ds.set2(4 * h + 2, s[2], s[3]);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          Frag<T> f;
          load_tr4(f, 0, &l.y[0][0], P, 32 * ks + 4 * g, 16 * t, lane);
          load_tr4(f, 4, &l.y[0][0], P, 32 * ks + 16 + 4 * g, 16 * t, lane);
          mma(dv[t], f, pf);
          load_tr4(f, 0, &l.x[0][0], P, 32 * ks + 4 * g, 16 * t, lane);
          load_tr4(f, 4, &l.x[0][0], P, 32 * ks + 16 + 4 * g, 16 * t, lane);
          mma(dk[t], f, ds);
        }
      }
    }
  }
  const Buf bk = buffer(seq_row(a.dk, sk, pk, hk, k0, esz), (int)(((m - 1) * a.dk.row + DH) * esz));
  const Buf bv = buffer(seq_row(a.dv, sk, pk, hk, k0, esz), (int)(((m - 1) * a.dv.row + DH) * esz));
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const int col = 16 * t + 4 * g;
    buf_store4<T>(bk, i < m ? (i * (int)a.dk.row + col) * esz : kPastEnd, dk[t][0] * a.scale, dk[t][1] * a.scale,
                  dk[t][2] * a.scale, dk[t][3] * a.scale);
    buf_store4<T>(bv, i < m ? (i * (int)a.dv.row + col) * esz : kPastEnd, dv[t][0], dv[t][1], dv[t][2], dv[t][3]);
  }
}

// bf16 with d = 64 and 128: 32 x 32 x 16 products (lane (h, c) of a result holds rows 8 (i / 4) + 4 h + i % 4 of column
// c), 32 rows of a workgroup's 128 to a wave.
template <int DH>
struct SoftmaxBwdLds32 {
  Tile<DH> x[2], y[2];
};

// this lane's row as B operands
template <int DH>
__device__ __forceinline__ void row_operands(bf16x8 (&f)[DH / 16], const char* base, int64_t row, int m, int r, int h) {
  const Buf b = buffer(base, m > 0 ? (int)(((m - 1) * row + DH) * 2) : 0);
#pragma unroll
  for (int t = 0; t < DH / 16; ++t)
    f[t] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(
                                          b, r < m ? (r * (int)row + 16 * t + 8 * h) * 2 : kPastEnd, 0, 0));
}

template <int DH>
__device__ __forceinline__ void store_rows(char* base, int64_t row, int m, int r, int h, const f32x16 (&x)[DH / 32], float f) {
  const Buf b = buffer(base, (int)(((m - 1) * row + DH) * 2));
#pragma unroll
  for (int t = 0; t < DH / 32; ++t)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      buf_store4<__bf16>(b, r < m ? (r * (int)row + 32 * t + 2 * e + 4 * h) * 2 : kPastEnd, x[t][e] * f, x[t][e + 1] * f,
                         x[t][e + 2] * f, x[t][e + 3] * f);
}

template <int DH>
__global__ __launch_bounds__(256, 2) void softmax_dq32_kernel(SoftmaxArgs a) {
  constexpr int KB = 64, KS = DH / 16, CT = DH / 32, esz = 2;
  extern __shared__ __attribute__((aligned(16))) char raw[];
  SoftmaxBwdLds32<DH>& l = *reinterpret_cast<SoftmaxBwdLds32<DH>*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id(), h = lane / 32, c = lane % 32;
  const int head = head_of(blockIdx.x % a.H, a.H);
  const SeqPiece sq = seq_piece_by_work(a.qs, blockIdx.x / a.H, gridDim.x / a.H, 128, true);
  if (sq.seq < 0) return;
  const SeqPiece sk = seq_of(a.ks, sq.seq);
  const bool pq = a.qs.offsets != nullptr, pk = a.ks.offsets != nullptr;
  const int q0 = sq.index * 128, m = min(128, sq.len - q0);
  const int shift = sk.len - sq.len;
  const int kend = min(sk.len, max(0, q0 + m + shift));
  const int i = 32 * wave + c, last = q0 + i + shift;
  const int wfirst = q0 + 32 * wave + shift, wlast = min(wfirst + 31, kend - 1);
  const int hk = head / (a.H / a.Hk);
  const int64_t num = seq_num(a.qs, sq, a.H, head, q0 + i);

  bf16x8 qf[KS], gf[KS];
  row_operands<DH>(qf, seq_row(a.q, sq, pq, head, q0, esz), a.q.row, m, i, h);
  row_operands<DH>(gf, seq_row(a.dO, sq, pq, head, q0, esz), a.dO.row, m, i, h);
  float delta = 0.0f;
  {
    bf16x8 of[KS];
    row_operands<DH>(of, seq_row(a.o, sq, pq, head, q0, esz), a.o.row, m, i, h);
#pragma unroll
    for (int t = 0; t < KS; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[t][e], (float)of[t][e], delta);
  }
  delta = halves_sum(delta);
  if (h == 0 && i < m) a.delta[num] = delta;
  if (a.scale < 0.0f)  // (the sign of the scale goes to q, as in the forward pass)
#pragma unroll
    for (int t = 0; t < KS; ++t) qf[t] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(i32x4, qf[t]) ^ (int)0x80008000);
  const float scale = fmaxf(fabsf(a.scale) * kLog2e, 1e-37f);
  float lse = i < m ? a.lse[num] * kLog2e : 0.0f;
  if (lse == -__builtin_inff()) lse = __builtin_inff();  // (a row that sees nothing: exp2(-infinity - infinity) below)
  f32x16 dq[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) dq[t] = zero16();

  TileRegs<DH> kr, vr;
  const auto load = [&](int k0) {
    Tile<DH>::load(kr, threadIdx.x, seq_row(a.k, sk, pk, hk, k0, esz), a.k.row, min(KB, kend - k0));
    Tile<DH>::load(vr, threadIdx.x, seq_row(a.v, sk, pk, hk, k0, esz), a.v.row, min(KB, kend - k0));
  };
  load(0);
  l.x[0].store(kr, threadIdx.x);
  l.y[0].store(vr, threadIdx.x);
  int buf = 0;
  for (int k0 = 0; k0 < kend; k0 += KB, buf ^= 1) {
    __syncthreads();  // this block is whole, and the one before no longer read
    load(k0 + KB);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int kb = k0 + 32 * half;
      if (kb > wlast) break;
      f32x16 s = zero16(), dp = zero16();
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(l.x[buf].row8(32 * half + c, 2 * t + h), qf[t], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(l.y[buf].row8(32 * half + c, 2 * t + h), gf[t], dp, 0, 0, 0);
      }
      // K^T operands of 16 keys, read a step before their products
      Frag<__bf16> kf[2][CT];
      const auto read_k = [&](int ks) {
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          const int row = 32 * half + 16 * ks + 4 * h, col = 32 * t + 16 * ((lane / 16) % 2);
          l.x[buf].tr4(kf[ks][t], 0, row, col, lane);
          l.x[buf].tr4(kf[ks][t], 4, row + 8, col, lane);
        }
      };
      read_k(0);
      if (kb + 31 > wfirst) {  // some row does not see some key
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = kb + 8 * (e / 4) + 4 * h + e % 4;
          s[e] = key <= last && key < kend ? s[e] : -__builtin_inff();
        }
      }
      Frag<__bf16> ds[2];
#pragma unroll
      for (int e = 0; e < 16; e += 2)
        ds[e / 8].set2(e % 8, weight(fmaf(s[e], scale, -lse)) * (dp[e] - delta),
                       weight(fmaf(s[e + 1], scale, -lse)) * (dp[e + 1] - delta));
      read_k(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int t = 0; t < CT; ++t) dq[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks][t].v, ds[ks].v, dq[t], 0, 0, 0);
    }
    l.x[buf ^ 1].store(kr, threadIdx.x);
    l.y[buf ^ 1].store(vr, threadIdx.x);
  }
  store_rows<DH>(seq_row(a.dq, sq, pq, head, q0, esz), a.dq.row, m, i, h, dq, a.scale);
}

// Two waves share 32 keys: one forms S, P and dV, the other, a step of 64 queries behind it, dP, dS and dK from the same
// P, which comes through LDS, lane for lane as both need it: times 2^15 in fp16 (2^-12 of P, down to 2^-29; in bf16 it
// would be a third rounding to 2^-9 of dK's terms: error 0.0030 instead of 0.0025, 1% less time).  P keeps
// that factor until the gradients are stored.  Either wave does the same two products (its rows against a tile, a
// transposed tile against its result) with half of the operands and gradients, so that two
// waves fit a SIMD; one wave with all of them took 490 registers, moved half of them about and reached 20% of the matrix
// cores' time.  8192 tokens, 16 heads of 128 on 4: 590 to 627 us on different cards (the query pass 425 to 456, the sum 46),
// matrix cores 37% busy; with d = 128 3 registers spill (query pass: 5).  With parts a
// workgroup takes one query head and leaves fp32 rows there, which softmax_sum_kernel adds up.
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr int kKeyShift = 15;  // P times 2^15 in the key pass

template <int DH>
struct SoftmaxKeyLds {
  Tile<DH> x[3], y[3];
  f16x8 p[2][4][4][kWave];  // per step parity, key tile and 16 queries
  float lse[3][64], delta[3][64];
};

template <int DH>
__global__ __launch_bounds__(512, 2) void softmax_dkdv32_kernel(SoftmaxArgs a) {
  constexpr int KB = 64, KS = DH / 16, CT = DH / 32, esz = 2;
  extern __shared__ __attribute__((aligned(16))) char raw[];
  SoftmaxKeyLds<DH>& l = *reinterpret_cast<SoftmaxKeyLds<DH>*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id() % 4, h = lane / 32, c = lane % 32;
  const bool second = wave_id() >= 4;  // dP, dS, dK
  const int group = a.H / a.Hk, heads = a.parts ? a.H : a.Hk;
  const int unit = head_of(blockIdx.x % heads, heads);
  const int hk = a.parts ? unit / group : unit, head0 = a.parts ? unit : unit * group, each = a.parts ? 1 : group;
  const SeqPiece sk = seq_piece_by_work(a.ks, blockIdx.x / heads, gridDim.x / heads, 128, false);
  if (sk.seq < 0) return;
  const SeqPiece sq = seq_of(a.qs, sk.seq);
  const bool pq = a.qs.offsets != nullptr, pk = a.ks.offsets != nullptr;
  const int k0 = sk.index * 128, m = min(128, sk.len - k0);
  const int shift = sk.len - sq.len;
  const int i = 32 * wave + c, key = k0 + i;
  const int wfirst = k0 + 32 * wave, wlast = wfirst + 31;  // the wave's keys
  const int qbegin = max(0, k0 - shift) / KB * KB;  // the first query that sees the tile's first key
  const int blocks = qbegin < sq.len ? (sq.len - qbegin + KB - 1) / KB : 0, steps = each * blocks;

  bf16x8 rf[KS];  // K rows (with the scale's sign, as in the forward pass) or V rows
  row_operands<DH>(rf, seq_row(second ? a.v : a.k, sk, pk, hk, k0, esz), second ? a.v.row : a.k.row, m, i, h);
  if (!second && a.scale < 0.0f)
#pragma unroll
    for (int t = 0; t < KS; ++t) rf[t] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(i32x4, rf[t]) ^ (int)0x80008000);
  const float scale = fmaxf(fabsf(a.scale) * kLog2e, 1e-37f);
  f32x16 acc[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) acc[t] = zero16();

  TileRegs<DH, 512> xr, yr;
  float lse = 0.0f, delta = 0.0f;  // of query threadIdx.x of the step
  const auto load = [&](int step) {
    const int head = head0 + step / blocks, q0 = qbegin + step % blocks * KB, qn = min(KB, sq.len - q0);
    Tile<DH>::load(xr, threadIdx.x, seq_row(a.q, sq, pq, head, q0, esz), a.q.row, qn);
    Tile<DH>::load(yr, threadIdx.x, seq_row(a.dO, sq, pq, head, q0, esz), a.dO.row, qn);
    const int64_t num = seq_num(a.qs, sq, a.H, head, q0 + min((int)threadIdx.x % KB, qn - 1));
    lse = a.lse[num];
    delta = a.delta[num];
  };
  const auto store = [&](int buf) {
    l.x[buf].store(xr, threadIdx.x);
    l.y[buf].store(yr, threadIdx.x);
    if (threadIdx.x < KB) {  // (a row that sees nothing: exp2(-infinity - infinity) below)
      l.lse[buf][threadIdx.x] = lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e - kKeyShift;
      l.delta[buf][threadIdx.x] = delta;
    }
  };
  if (steps > 0) {
    load(0);
    store(0);
  }
  for (int step = 0; step <= steps && steps > 0; ++step) {
    __syncthreads();  // the tiles of this step and P of the one before are whole
    load(min(step + 1, steps - 1));
    const int at = second ? step - 1 : step;  // this wave's step
    const int q0 = qbegin + at % blocks * KB, qn = min(KB, sq.len - q0), buf = at % 3;
    if (at >= 0 && at < steps && q0 + KB - 1 + shift >= wfirst) {  // (uniform) some query sees a key of the wave
      const Tile<DH>& rows = second ? l.y[buf] : l.x[buf];
      const Tile<DH>& cols = second ? l.x[buf] : l.y[buf];
      f32x16 s[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) s[half] = zero16();
#pragma unroll
      for (int t = 0; t < KS; ++t)
#pragma unroll
        for (int half = 0; half < 2; ++half)
          s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.row8(32 * half + c, 2 * t + h), rf[t], s[half], 0, 0, 0);
      // transposed operands of 16 queries, read a step before their products
      Frag<__bf16> f[2][CT], pf[4];
      const auto read = [&](int ks) {
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          const int row = 16 * ks + 4 * h, col = 32 * t + 16 * ((lane / 16) % 2);
          cols.tr4(f[ks % 2][t], 0, row, col, lane);
          cols.tr4(f[ks % 2][t], 4, row + 8, col, lane);
        }
      };
      read(0);
      if (!second) {
        f16x8 ph[4];
        if (q0 + shift < wlast || qn < KB || m < 128) {
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int r = 32 * half + 8 * (e / 4) + 4 * h + e % 4;
              s[half][e] = key <= q0 + r + shift && r < qn && i < m ? s[half][e] : -__builtin_inff();
            }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const f32x4 ls = *reinterpret_cast<const f32x4*>(&l.lse[buf][32 * half + 2 * e + 4 * h]);
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
              const float x = weight<kKeyShift>(fmaf(s[half][e + j], scale, -ls[j]));
              const float y = weight<kKeyShift>(fmaf(s[half][e + j + 1], scale, -ls[j + 1]));
              pf[2 * half + e / 8].set2(e % 8 + j, x, y);
              ph[2 * half + e / 8][e % 8 + j] = (_Float16)x;
              ph[2 * half + e / 8][e % 8 + j + 1] = (_Float16)y;
            }
          }
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) l.p[at % 2][wave][ks][lane] = ph[ks];
      } else {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const f16x8 p = l.p[at % 2][wave][ks][lane];
          const f32x4 d0 = *reinterpret_cast<const f32x4*>(&l.delta[buf][16 * ks + 4 * h]);
          const f32x4 d1 = *reinterpret_cast<const f32x4*>(&l.delta[buf][16 * ks + 8 + 4 * h]);
#pragma unroll
          for (int e = 0; e < 8; e += 2)
            pf[ks].set2(e, (float)p[e] * (s[ks / 2][8 * (ks % 2) + e] - (e < 4 ? d0[e] : d1[e - 4])),
                        (float)p[e + 1] * (s[ks / 2][8 * (ks % 2) + e + 1] - (e < 4 ? d0[e + 1] : d1[e - 3])));
        }
      }
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        if (ks < 3) read(ks + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < CT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[ks % 2][t].v, pf[ks].v, acc[t], 0, 0, 0);
      }
    }
    if (step + 1 < steps) store((step + 1) % 3);
  }
  if (a.parts) {
    if (i >= m) return;
    float* part = a.parts + seq_num(a.ks, sk, a.H, unit, k0 + i) * (2 * DH) + (second ? 0 : DH);
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int e = 0; e < 16; e += 4) store4(part + 32 * t + 2 * e + 4 * h, acc[t][e], acc[t][e + 1], acc[t][e + 2], acc[t][e + 3]);
    return;
  }
  constexpr float unit_p = 1.0f / (1 << kKeyShift);
  if (second) store_rows<DH>(seq_row(a.dk, sk, pk, hk, k0, esz), a.dk.row, m, i, h, acc, a.scale * unit_p);
  else store_rows<DH>(seq_row(a.dv, sk, pk, hk, k0, esz), a.dv.row, m, i, h, acc, unit_p);
}

// dK and dV of a key head from its query heads' rows in a.parts, in order of the heads.
template <int DH>
__global__ __launch_bounds__(256) void softmax_sum_kernel(SoftmaxArgs a) {
  constexpr int PER = DH / 4;  // threads per row of each gradient
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
  const SeqPiece sk = seq_piece(a.ks, slot, 128);
  if (sk.seq < 0) return;
  const bool pk = a.ks.offsets != nullptr;
  const int k0 = sk.index * 128, m = min(128, sk.len - k0), group = a.H / a.Hk;
  for (int idx = threadIdx.x; idx < m * 2 * PER; idx += 256) {
    const int r = idx / (2 * PER), at = idx % (2 * PER), which = at / PER, col = at % PER * 4;
    f32x4 sum = zero4();
    for (int g = 0; g < group; ++g)
      sum += *reinterpret_cast<const f32x4*>(a.parts + seq_num(a.ks, sk, a.H, hk * group + g, k0 + r) * (2 * DH) + which * DH + col);
    const float f = (which ? 1.0f : a.scale) / (1 << kKeyShift);
    __bf16* to = reinterpret_cast<__bf16*>(seq_row(which ? a.dv : a.dk, sk, pk, hk, k0 + r, 2)) + col;
    store4(to, sum[0] * f, sum[1] * f, sum[2] * f, sum[3] * f);
  }
}

template <int DH>
hipError_t launch_width32(const SoftmaxArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(SoftmaxBwdLds32<DH>), key_bytes = (int)sizeof(SoftmaxKeyLds<DH>);
  hipError_t e = allow_lds<softmax_dq32_kernel<DH>>(bytes);
  if (e == hipSuccess) e = allow_lds<softmax_dkdv32_kernel<DH>>(key_bytes);
  if (e != hipSuccess) return e;
  const int64_t qt = seq_slots(a.qs, 128), kt = seq_slots(a.ks, 128);
  if (qt > 0) hipLaunchKernelGGL((softmax_dq32_kernel<DH>), dim3((unsigned)(qt * a.H)), dim3(256), bytes, s, a);
  if ((e = hipGetLastError()) != hipSuccess || kt == 0) return e;
  hipLaunchKernelGGL((softmax_dkdv32_kernel<DH>), dim3((unsigned)(kt * (a.parts ? a.H : a.Hk))), dim3(512), key_bytes, s, a);
  if ((e = hipGetLastError()) != hipSuccess || !a.parts) return e;
  hipLaunchKernelGGL((softmax_sum_kernel<DH>), dim3((unsigned)(kt * a.Hk)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t launch_width(const SoftmaxArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(SoftmaxBwdLds<T, DH>);
  hipError_t e = allow_lds<softmax_dq_kernel<T, DH>>(bytes);
  if (e == hipSuccess) e = allow_lds<softmax_dkdv_kernel<T, DH>>(bytes);
  if (e != hipSuccess) return e;
  if (seq_slots(a.qs, kSoftmaxTile) > 0)
    hipLaunchKernelGGL((softmax_dq_kernel<T, DH>), dim3((unsigned)(seq_slots(a.qs, kSoftmaxTile) * a.H)), dim3(256), bytes, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (seq_slots(a.ks, kSoftmaxTile) > 0)
    hipLaunchKernelGGL((softmax_dkdv_kernel<T, DH>), dim3((unsigned)(seq_slots(a.ks, kSoftmaxTile) * a.Hk)), dim3(256), bytes, s,
                       a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_bwd(const SoftmaxArgs& a, hipStream_t s) {
  return a.d == 32 ? launch_width<T, 32>(a, s) : a.d == 64 ? launch_width<T, 64>(a, s) : launch_width<T, 128>(a, s);
}

}  // namespace

hipError_t launch_softmax_bwd(Dt dt, const SoftmaxArgs& a, hipStream_t s) {
  if (dt == Dt::F32) return launch_bwd<float>(a, s);
  return a.d == 32 ? launch_width<__bf16, 32>(a, s) : a.d == 64 ? launch_width32<64>(a, s) : launch_width32<128>(a, s);
}

}  // namespace luna
