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
  const int head = blockIdx.x % a.H, slot = gridDim.x / a.H - 1 - blockIdx.x / a.H;
  const SeqPiece sq = seq_piece(a.qs, slot, kSoftmaxTile);
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
          const float e = exp2_raw(fmaf(s[j], scale, -lse)) * (dp[j] - delta);
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
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;  // (earlier tiles are seen by more queries)
  const SeqPiece sk = seq_piece(a.ks, slot, kSoftmaxTile);
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
            const float e = exp2_raw(fmaf(s[j], scale, -lse[j]));
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
  return dt == Dt::BF16 ? launch_bwd<__bf16>(a, s) : launch_bwd<float>(a, s);
}

}  // namespace luna
