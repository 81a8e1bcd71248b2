// luna_decay_step.hip -- the recurrent form of linear attention with a decay for each head: m
// new tokens per sequence from the state (S, z), token by token in fp32,
//
//   S = f S + k_t v_t^T,  z = f z + k_t,  out_t = scale q_t^T S [/ (scale q_t^T z + eps)].
//
// One workgroup per sequence, head and COLS value columns: thread (quad, group) holds four columns of
// S for the features group + 32 i in registers for the whole step, so that a call reads the state
// once and writes it once with 16-byte accesses, which is what bounds it.  Every group has its
// share of each sum over features; the shares are added within a wave by lane exchanges and over the
// waves through LDS, in a fixed order.  Measured: 64 sequences of 16 heads, states of 256 x 128: 60 us for 270 MB (4.5 TB/s)
// with other states in between, 48 us again and again on one state, half of which then lies in the last-level cache;
// 8 sequences, 128 x 128: 5.5 us.  Normalised calls take all columns of a head in one
// workgroup: each of several would read z while one of them writes it.
#include "luna_seq.hpp"

namespace luna {

namespace {

constexpr int kStepGroups = 32;  // feature groups
constexpr int kStepStage = 4;    // tokens staged in LDS at a time

template <typename T, int COLS, int FEAT, bool NORM>
__global__ __launch_bounds__(8 * COLS) void decay_step_kernel(DecayStepArgs a) {
  constexpr int QUADS = COLS / 4, THREADS = QUADS * kStepGroups, WAVES = THREADS / kWave, D = FEAT * kStepGroups;
  __shared__ float sq[kStepStage][D], sk[kStepStage][D];
  __shared__ __attribute__((aligned(16))) float sv[kStepStage][COLS];
  __shared__ float red[kStepStage][WAVES][QUADS][5];
  const int blocks = a.d / COLS;
  const int64_t at = blockIdx.x / blocks;
  const int col0 = (blockIdx.x % blocks) * COLS;
  const int64_t b = at / a.H;
  const int head = (int)(at % a.H);
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int quad = tid % QUADS, grp = tid / QUADS;
  float* S = a.S + at * D * a.d + col0 + 4 * quad;
  float* z = NORM ? a.z + at * D : nullptr;
  const auto rows = [&](const SeqRows& r) { return reinterpret_cast<T*>(r.data) + b * r.seq + head * r.head; };
  const T *Q = rows(a.q), *K = rows(a.k), *V = rows(a.v) + col0;
  T* O = rows(a.o) + col0;
  const float f = exp2f(decay_log2(a.log_decay[head]));

  float4 s[FEAT];
  float zz[FEAT];
#pragma unroll
  for (int i = 0; i < FEAT; ++i) {
    const int c = grp + kStepGroups * i;
    s[i] = *reinterpret_cast<const float4*>(S + (int64_t)c * a.d);
    zz[i] = NORM ? z[c] : 0.0f;
  }
  for (int t0 = 0; t0 < a.m; t0 += kStepStage) {
    const int tn = min(kStepStage, a.m - t0);
    __syncthreads();  // the stage before is no longer read
    for (int i = tid; i < tn * D; i += THREADS) {
      sq[i / D][i % D] = (float)Q[(int64_t)(t0 + i / D) * a.q.row + i % D];
      sk[i / D][i % D] = (float)K[(int64_t)(t0 + i / D) * a.k.row + i % D];
    }
    for (int i = tid; i < tn * COLS; i += THREADS) sv[i / COLS][i % COLS] = (float)V[(int64_t)(t0 + i / COLS) * a.v.row + i % COLS];
    __syncthreads();
    for (int t = 0; t < tn; ++t) {
      const float4 v = *reinterpret_cast<const float4*>(&sv[t][4 * quad]);
      float n[5] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < FEAT; ++i) {
        const int c = grp + kStepGroups * i;
        const float k = sk[t][c], q = sq[t][c];
        s[i].x = fmaf(f, s[i].x, k * v.x);
        s[i].y = fmaf(f, s[i].y, k * v.y);
        s[i].z = fmaf(f, s[i].z, k * v.z);
        s[i].w = fmaf(f, s[i].w, k * v.w);
        n[0] = fmaf(q, s[i].x, n[0]);
        n[1] = fmaf(q, s[i].y, n[1]);
        n[2] = fmaf(q, s[i].z, n[2]);
        n[3] = fmaf(q, s[i].w, n[3]);
        if (NORM) {
          zz[i] = fmaf(f, zz[i], k);
          n[4] = fmaf(q, zz[i], n[4]);
        }
      }
#pragma unroll
      for (int w = QUADS; w < kWave; w *= 2)
#pragma unroll
        for (int i = 0; i < (NORM ? 5 : 4); ++i) n[i] += __shfl_xor(n[i], w);
      if (lane < QUADS)
#pragma unroll
        for (int i = 0; i < 5; ++i) red[t][wave][quad][i] = n[i];
    }
    __syncthreads();
    for (int i = tid; i < tn * COLS; i += THREADS) {
      const int t = i / COLS, c = i % COLS;
      float num = 0.0f, den = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        num += red[t][w][c / 4][c % 4];
        if (NORM) den += red[t][w][c / 4][4];
      }
      num *= a.scale;
      O[(int64_t)(t0 + t) * a.o.row + c] = (T)(NORM ? num / (a.scale * den + a.eps) : num);
    }
  }
#pragma unroll
  for (int i = 0; i < FEAT; ++i) {
    const int c = grp + kStepGroups * i;
    *reinterpret_cast<float4*>(S + (int64_t)c * a.d) = s[i];
    if (NORM && quad == 0) z[c] = zz[i];
  }
}

template <typename T, int COLS, bool NORM>
hipError_t launch_step(const DecayStepArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.count * a.H * (a.d / COLS))), block(8 * COLS);
  switch (a.D) {
    case 32: hipLaunchKernelGGL((decay_step_kernel<T, COLS, 1, NORM>), grid, block, 0, s, a); break;
    case 64: hipLaunchKernelGGL((decay_step_kernel<T, COLS, 2, NORM>), grid, block, 0, s, a); break;
    case 128: hipLaunchKernelGGL((decay_step_kernel<T, COLS, 4, NORM>), grid, block, 0, s, a); break;
    case 256: hipLaunchKernelGGL((decay_step_kernel<T, COLS, 8, NORM>), grid, block, 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_step_typed(const DecayStepArgs& a, hipStream_t s) {
  if (!a.normalize) return launch_step<T, 32, false>(a, s);
  return a.d == 32 ? launch_step<T, 32, true>(a, s) : a.d == 64 ? launch_step<T, 64, true>(a, s) : launch_step<T, 128, true>(a, s);
}

}  // namespace

hipError_t launch_decay_step(Dt dt, const DecayStepArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_step_typed<__bf16>(a, s) : launch_step_typed<float>(a, s);
}

}  // namespace luna
