// luna_softmax.hip -- causal softmax attention over sequences of different lengths, forward.
//
//   s_ij = scale q_i.k_j (j <= i + Lk - Lq),  out_i = sum_j exp(s_ij - lse_i) v_j.
//
// One pass over the keys with the running maximum and sum of each row.  A workgroup of four waves
// takes 64 queries of one head, a wave 16 of them.  Scores are formed transposed, S^T = K Q^T:
// lane (g, c) of a block of 16 keys holds keys 4g + j of query c, so a row's maximum and
// sum are four registers and two lane exchanges, and two blocks of probabilities are
// the B operand of out^T = V^T P^T as they are (keys 4g + j of both as the 8 k-slots; V is read
// in that order with transposing reads).  Maxima and sums are fp32, in base 2; P is rounded to
// the element type as an operand after its sum is taken.
#include "luna_softmax.hpp"

namespace luna {

namespace {

template <typename T, int DH>
struct SoftmaxLds {
  static constexpr int KB = kSoftmaxStep<T>, P = DH + 16 / (int)sizeof(T);
  T k[KB][P], v[KB][P];
};

template <typename T, int DH>
__global__ __launch_bounds__(256) void softmax_fwd_kernel(SoftmaxArgs a) {
  using Lds = SoftmaxLds<T, DH>;
  constexpr int KB = Lds::KB, P = Lds::P, KT = KB / 16, CT = DH / 16, esz = (int)sizeof(T);
  __shared__ __attribute__((aligned(16))) char raw[sizeof(Lds)];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id(), g = lane / 16, c = lane % 16;
  const int head = blockIdx.x % a.H, slot = gridDim.x / a.H - 1 - blockIdx.x / a.H;  // (later tiles have more keys)
  const SeqPiece sq = seq_piece(a.qs, slot, kSoftmaxTile);
  if (sq.seq < 0) return;
  const SeqPiece sk = seq_of(a.ks, sq.seq);
  const bool pq = a.qs.offsets != nullptr, pk = a.ks.offsets != nullptr;
  const int q0 = sq.index * kSoftmaxTile, m = min(kSoftmaxTile, sq.len - q0);
  const int shift = sk.len - sq.len;  // query i sees keys up to i + shift
  const int kend = min(sk.len, max(0, q0 + m + shift));
  const int i = 16 * wave + c;        // this lane's query of the tile
  const int last = q0 + i + shift;    // its last key
  const int hk = head / (a.H / a.Hk);

  Frag<T> qf[DH / 32];
  softmax_load_frags<T, DH>(qf, seq_row(a.q, sq, pq, head, q0, esz), a.q.row, m, i, g);
  const float scale = a.scale * kLog2e;
  f32x4 o[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) o[t] = zero4();
  float top = -__builtin_inff(), sum = 0.0f;

  for (int k0 = 0; k0 < kend; k0 += KB) {
    const int kn = min(KB, kend - k0);
    __syncthreads();
    softmax_load_rows<T, KB, DH, P>(&l.k[0][0], seq_row(a.k, sk, pk, hk, k0, esz), a.k.row, kn);
    softmax_load_rows<T, KB, DH, P>(&l.v[0][0], seq_row(a.v, sk, pk, hk, k0, esz), a.v.row, kn);
    __syncthreads();
    f32x4 s[KT];
    float most = top;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      s[kt] = zero4();
#pragma unroll
      for (int t = 0; t < DH / 32; ++t) {
        Frag<T> kf;
        load8(kf, &l.k[16 * kt + c][32 * t + 8 * g]);
        mma(s[kt], kf, qf[t]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = k0 + 16 * kt + 4 * g + j;
        const float x = s[kt][j] * scale;
        s[kt][j] = key <= last && key < kend ? x : -__builtin_inff();
        most = fmaxf(most, s[kt][j]);
      }
    }
    most = groups_max(most);
    const float base = most == -__builtin_inff() ? 0.0f : most;  // (no key seen yet)
    const float f = exp2_raw(top - base);
    top = most;
    float part = 0.0f;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[kt][j] = exp2_raw(s[kt][j] - base);
        part += s[kt][j];
      }
    sum = fmaf(sum, f, part);
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[t][j] *= f;
#pragma unroll
    for (int ks = 0; ks < KT / 2; ++ks) {
      Frag<T> pf;
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        pf.set2(j, s[2 * ks][j], s[2 * ks][j + 1]);
        pf.set2(4 + j, s[2 * ks + 1][j], s[2 * ks + 1][j + 1]);
      }
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        Frag<T> vf;
        load_tr4(vf, 0, &l.v[0][0], P, 32 * ks + 4 * g, 16 * t, lane);
        load_tr4(vf, 4, &l.v[0][0], P, 32 * ks + 16 + 4 * g, 16 * t, lane);
        mma(o[t], vf, pf);
      }
    }
  }
  sum = groups_sum(sum);
  const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;  // (NaN stays)
  const Buf b = buffer(seq_row(a.o, sq, pq, head, q0, esz), (int)(((m - 1) * a.o.row + DH) * esz));
#pragma unroll
  for (int t = 0; t < CT; ++t)
    buf_store4<T>(b, i < m ? (i * (int)a.o.row + 16 * t + 4 * g) * esz : kPastEnd, o[t][0] * inv, o[t][1] * inv,
                  o[t][2] * inv, o[t][3] * inv);
  if (a.lse && g == 0 && i < m) a.lse[seq_num(a.qs, sq, a.H, head, q0 + i)] = (top + log2f(sum)) * kLn2;
}

template <typename T>
hipError_t launch_fwd(const SoftmaxArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(seq_slots(a.qs, kSoftmaxTile) * a.H));
  if (a.d == 32) hipLaunchKernelGGL((softmax_fwd_kernel<T, 32>), grid, dim3(256), 0, s, a);
  else if (a.d == 64) hipLaunchKernelGGL((softmax_fwd_kernel<T, 64>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((softmax_fwd_kernel<T, 128>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_softmax_fwd(Dt dt, const SoftmaxArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_fwd<__bf16>(a, s) : launch_fwd<float>(a, s);
}

}  // namespace luna
