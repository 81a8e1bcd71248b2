// luna_delta_gates.hip -- the gated delta rule's matrices of each chunk: N = -M (I + beta M)^-1, P and the factors of its gates
// (luna_delta.hpp), for all chunks, side by side.
//
// A workgroup of four waves takes a chunk of one key head: K K^T and Q K^T once on the matrix cores, wave w the rows 16 w ..
// 16 w + 15, then for each value head of the group its gates, M and P.  N in blocks of 16: the diagonal blocks by forward
// substitution, a wave each and a column a lane,
//   N_rc = -M_rc - sum_{p < r} M_rp beta_p N_pc,
// and wave j the blocks below the diagonal of block column j, on the fp32 matrix cores,
//   Z = M_ij + sum_{j <= p < i} M_ip beta_p N_pj,   N_ij = -(Z + N_ii beta_i Z).
// What bounds it is these chains: 1024 chunks in bf16, D = 128, 26 us.
#include "luna_delta.hpp"

namespace luna {

namespace {

constexpr int C = kDeltaChunk, PM = C + 4;

template <typename T, int DK>
struct GatesLds {
  static constexpr int PK = DK + 16 / (int)sizeof(T);
  union {
    T k[C][PK];
    float n[C][PM];
  };
  float m[C][PM];
  float high[C], low[C], beta[C];
  int key, gate;  // first row that is not finite
};

// c += A B of fp32 blocks of 16: row c of A (four numbers from 4 g on), and B as a sum's registers are.
__device__ __forceinline__ void mma16(f32x4& c, const float* row, const f32x4& b) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(row);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
}

__device__ __forceinline__ bool odd(const Frag<__bf16>& f) { return not_finite(f); }
__device__ __forceinline__ bool odd(const Frag<float>& f) {
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) bad |= !(fabsf(f.v[e]) < __builtin_inff());
  return bad;
}

template <typename T, int DK, int NP>
__global__ __launch_bounds__(256) void delta_gates_kernel(DeltaArgs a) {
  using Lds = GatesLds<T, DK>;
  constexpr int esz = (int)sizeof(T), KS = DK / 32;
  __shared__ __attribute__((aligned(16))) char raw[sizeof(Lds)];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int tid = threadIdx.x, lane = tid % kWave, wave = wave_id(), g = lane / 16, c = lane % 16;
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk, group = a.H / a.Hk;
  const SeqPiece sp = seq_uniform(seq_piece(a.s, slot, C));
  if (sp.seq < 0) return;
  const bool packed = a.s.offsets != nullptr;
  const int t0 = sp.index * C, m = min(C, sp.len - t0);

  if (tid == 0) l.key = C;
  __syncthreads();
  {
    DecayRows<T, C, DK, Lds::PK, 256> kr;
    kr.load(seq_row(a.k, sp, packed, hk, t0, esz), a.k.row, m, DK, false);
    kr.store(&l.k[0][0]);
  }
  Frag<T> qf[KS];
  {
    const Buf b = buffer(seq_row(a.q, sp, packed, hk, t0, esz), (int)(((m - 1) * a.q.row + DK) * esz));
    const int i = 16 * wave + c;
#pragma unroll
    for (int t = 0; t < KS; ++t) buf_load8(qf[t], b, i < m ? (i * (int)a.q.row + 32 * t + 8 * g) * esz : kPastEnd);
  }
  __syncthreads();
  f32x4 kk[4], qk[4];  // rows j of block jt (4 g + e), column i = 16 wave + c
  {
    Frag<T> kf[KS];
    bool bad = false;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      load8(kf[t], &l.k[16 * wave + c][32 * t + 8 * g]);
      bad |= odd(kf[t]);
    }
    if (bad) atomicMin(&l.key, 16 * wave + c);
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      kk[jt] = zero4();
      qk[jt] = zero4();
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        Frag<T> kj;
        load8(kj, &l.k[16 * jt + c][32 * t + 8 * g]);
        mma(kk[jt], kj, kf[t]);
        mma(qk[jt], kj, qf[t]);
      }
    }
  }

  for (int h = 0; h < group; ++h) {
    const int head = hk * group + h;
    const int64_t at = (int64_t)slot * a.H + head;
    float* gates = a.gates + at * kDeltaGates;
    __syncthreads();  // K, or the head before, is no longer read
    if (wave == 0) {
      const int64_t num = seq_num(a.s, sp, a.H, head, t0 + min(lane, m - 1));
      float x = lane < m ? a.log_decay[num] : 0.0f, beta = lane < m ? a.beta[num] : 0.0f;
      const uint64_t lost = __ballot(isnan(x) || !(fabsf(beta) < __builtin_inff()));
      const int bad = min(l.key, lost ? (int)__builtin_ctzll(lost) : C);
      if (lane >= bad) x = beta = 0.0f;
      // (e^-128 is 0 in fp32; in base 2)
      double sum = (double)fminf(fmaxf(x, -128.0f), 0.0f) * 1.4426950408889634;
#pragma unroll
      for (int w = 1; w < kWave; w *= 2) {
        const double other = __shfl_up(sum, w);
        sum += lane >= w ? other : 0.0;
      }
      const double whole = __shfl(sum, kWave - 1);
      const float high = (float)sum, low = (float)(sum - (double)high);
      l.high[lane] = high;
      l.low[lane] = low;
      l.beta[lane] = beta;
      if (lane == 0) l.gate = bad;
      gates[kDeltaFirst * C + lane] = exp2_raw(high);
      gates[kDeltaLast * C + lane] = exp2_raw((float)(whole - sum));
      gates[kDeltaBeta * C + lane] = beta;
      gates[kDeltaHigh * C + lane] = high;
      gates[kDeltaLow * C + lane] = low;
      gates[kDeltaMisc * C + lane] = lane == 0 ? exp2_raw((float)whole) : __int_as_float(lane == 1 ? bad : 0);
    }
    __syncthreads();
    const int bad = l.gate, i = 16 * wave + c;
    const float high = l.high[i], low = l.low[i];
    T* p = reinterpret_cast<T*>(a.p) + at * delta_parts<T>(NP) * C * C;
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      f32x4 mm, pp;
      const f32x4 hj = *reinterpret_cast<const f32x4*>(&l.high[16 * jt + 4 * g]);
      const f32x4 lj = *reinterpret_cast<const f32x4*>(&l.low[16 * jt + 4 * g]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = 16 * jt + 4 * g + e;
        const float f = exp2_raw((high - hj[e]) + (low - lj[e]));
        mm[e] = j < i && i < bad ? kk[jt][e] * f : 0.0f;
        pp[e] = j <= i && j < bad ? a.scale * qk[jt][e] * f : 0.0f;
      }
      *reinterpret_cast<f32x4*>(&l.m[i][16 * jt + 4 * g]) = mm;
      store_parts4<NP>(p + i * C + 16 * jt + 4 * g, C * C, pp[0], pp[1], pp[2], pp[3]);
    }
    __syncthreads();
    {  // diagonal blocks
      const int r0 = 16 * wave;
      float n[16], bn[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float sum = l.m[r0 + r][r0 + c];
#pragma unroll
        for (int p4 = 0; p4 < r; p4 += 4) {
          const f32x4 row = *reinterpret_cast<const f32x4*>(&l.m[r0 + r][r0 + p4]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (p4 + e < r) sum = fmaf(row[e], bn[p4 + e], sum);
        }
        n[r] = -sum;
        bn[r] = l.beta[r0 + r] * n[r];
      }
      if (g == 0)
#pragma unroll
        for (int r = 0; r < 16; ++r) l.n[r0 + r][r0 + c] = n[r];
    }
    __syncthreads();
    {  // block column `wave`
      f32x4 bn[4];
#pragma unroll
      for (int i2 = 0; i2 < 4; ++i2) {
        f32x4 n = zero4();
        const f32x4 beta = *reinterpret_cast<const f32x4*>(&l.beta[16 * i2 + 4 * g]);
        if (i2 == wave) {
#pragma unroll
          for (int e = 0; e < 4; ++e) n[e] = l.n[16 * i2 + 4 * g + e][16 * wave + c];
        } else if (i2 > wave) {
          f32x4 z;
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = l.m[16 * i2 + 4 * g + e][16 * wave + c];
#pragma unroll
          for (int p2 = 0; p2 < i2; ++p2)  // (blocks before the column's own are zeros)
            mma16(z, &l.m[16 * i2 + c][16 * p2 + 4 * g], bn[p2]);
          mma_settle();
          f32x4 bz, y = z;
#pragma unroll
          for (int e = 0; e < 4; ++e) bz[e] = beta[e] * z[e];
          mma16(y, &l.n[16 * i2 + c][16 * i2 + 4 * g], bz);
          mma_settle();
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            n[e] = -y[e];
            l.n[16 * i2 + 4 * g + e][16 * wave + c] = n[e];
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) bn[i2][e] = beta[e] * n[e];
      }
    }
    __syncthreads();
    T* n = reinterpret_cast<T*>(a.n) + at * delta_parts<T>(NP) * C * C;
    const int r = tid / 4;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int j = 16 * (tid % 4) + 4 * b;
      f32x4 x = *reinterpret_cast<const f32x4*>(&l.n[r][j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = j + e < r ? x[e] : 0.0f;
      store_parts4<NP>(n + r * C + j, C * C, x[0], x[1], x[2], x[3]);
    }
  }
}

template <typename T, int NP>
hipError_t launch_gates(const DeltaArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.slots * a.Hk)), block(256);
  switch (a.D) {
    case 32: hipLaunchKernelGGL((delta_gates_kernel<T, 32, NP>), grid, block, 0, s, a); break;
    case 64: hipLaunchKernelGGL((delta_gates_kernel<T, 64, NP>), grid, block, 0, s, a); break;
    case 128: hipLaunchKernelGGL((delta_gates_kernel<T, 128, NP>), grid, block, 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_gates(Dt dt, const DeltaArgs& a, hipStream_t s) {
  return dt == Dt::F32 ? launch_gates<float, 1>(a, s) : launch_gates<__bf16, kDeltaBackParts>(a, s);
}

}  // namespace luna
