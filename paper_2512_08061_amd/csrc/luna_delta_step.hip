// luna_delta_step.hip -- the recurrent form of the gated delta rule: m new tokens per sequence from the state S, token by
// token in fp32,
//
//   S = a S,  u = beta (v - S^T k),  S = S + k u^T,  out = scale S^T q.
//
// One workgroup per sequence, head and 32 value columns: thread (quad, group) holds four columns of S for the features
// group + 32 i in registers for the whole step, so that a call reads the state once and writes it once with 16-byte
// accesses, which is what bounds it (64 x 32 heads, D = d = 128, 270 MB: 54.2 us, the rate of a copy).  S^T k, S^T q and k.q are summed side by side, before the update, of which
// S'^T q = S^T q + (k.q) u follows; the shares of the groups are added within a wave by lane exchanges and over the
// waves through LDS, in a fixed order.
//
// Infinities among keys, values and beta count as NaN, which every sum hands on: from its token on the head's or column's state and
// rows are NaN (infinities by themselves would stay, beside the NaN of 0 times them).
#include "luna_seq.hpp"
#include "luna_delta.hpp"

namespace luna {

namespace {

constexpr int kStepGroups = 32;  // feature groups
constexpr int kStepStage = 4;    // tokens staged in LDS at a time
constexpr int kStepCols = 32;

__device__ __forceinline__ float finite_or_nan(float x) { return fmaf(0.0f, x, x); }  // (0 times an infinity is NaN)

template <typename T, int FEAT>
__global__ __launch_bounds__(8 * kStepCols) void delta_step_kernel(DeltaStepArgs a) {
  constexpr int COLS = kStepCols, QUADS = COLS / 4, THREADS = QUADS * kStepGroups, WAVES = THREADS / kWave, D = FEAT * kStepGroups;
  __shared__ float sq[kStepStage][D], sk[kStepStage][D];
  __shared__ __attribute__((aligned(16))) float sv[kStepStage][COLS];
  __shared__ float gates[2][kStepStage];
  __shared__ float red[2][WAVES][QUADS][9];
  const int blocks = a.d / COLS;
  const int64_t at = blockIdx.x / blocks;
  const int col0 = (blockIdx.x % blocks) * COLS;
  const int64_t b = at / a.H;
  const int head = (int)(at % a.H), hk = head / (a.H / a.Hk);
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int quad = tid % QUADS, grp = tid / QUADS;
  float* S = a.S + at * D * a.d + col0 + 4 * quad;
  const T* Q = reinterpret_cast<const T*>(a.q.data) + b * a.q.seq + hk * a.q.head;
  const T* K = reinterpret_cast<const T*>(a.k.data) + b * a.k.seq + hk * a.k.head;
  const T* V = reinterpret_cast<const T*>(a.v.data) + b * a.v.seq + head * a.v.head + col0;
  T* O = reinterpret_cast<T*>(a.o.data) + b * a.o.seq + head * a.o.head + col0;

  float4 s[FEAT];
#pragma unroll
  for (int i = 0; i < FEAT; ++i) s[i] = *reinterpret_cast<const float4*>(S + (int64_t)(grp + kStepGroups * i) * a.d);
  for (int t0 = 0; t0 < a.m; t0 += kStepStage) {
    const int tn = min(kStepStage, a.m - t0);
    __syncthreads();  // the stage before is no longer read
    for (int i = tid; i < tn * D; i += THREADS) {
      sq[i / D][i % D] = (float)Q[(int64_t)(t0 + i / D) * a.q.row + i % D];
      sk[i / D][i % D] = finite_or_nan((float)K[(int64_t)(t0 + i / D) * a.k.row + i % D]);
    }
    for (int i = tid; i < tn * COLS; i += THREADS) sv[i / COLS][i % COLS] = finite_or_nan((float)V[(int64_t)(t0 + i / COLS) * a.v.row + i % COLS]);
    if (tid < tn) {
      gates[0][tid] = exp2f(decay_log2(a.log_decay[at * a.m + t0 + tid]));
      gates[1][tid] = finite_or_nan(a.beta[at * a.m + t0 + tid]);
    }
    __syncthreads();
    for (int t = 0; t < tn; ++t) {
      const float f = gates[0][t], beta = gates[1][t];
      float n[9] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < FEAT; ++i) {
        const int c = grp + kStepGroups * i;
        const float k = sk[t][c], q = sq[t][c];
        s[i].x *= f, s[i].y *= f, s[i].z *= f, s[i].w *= f;
        n[0] = fmaf(k, s[i].x, n[0]);
        n[1] = fmaf(k, s[i].y, n[1]);
        n[2] = fmaf(k, s[i].z, n[2]);
        n[3] = fmaf(k, s[i].w, n[3]);
        n[4] = fmaf(q, s[i].x, n[4]);
        n[5] = fmaf(q, s[i].y, n[5]);
        n[6] = fmaf(q, s[i].z, n[6]);
        n[7] = fmaf(q, s[i].w, n[7]);
        n[8] = fmaf(k, q, n[8]);
      }
#pragma unroll
      for (int w = QUADS; w < kWave; w *= 2)
#pragma unroll
        for (int i = 0; i < 9; ++i) n[i] += __shfl_xor(n[i], w);
      if (lane < QUADS)
#pragma unroll
        for (int i = 0; i < 9; ++i) red[t % 2][wave][quad][i] = n[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 9; ++i) {
        n[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) n[i] += red[t % 2][w][quad][i];
      }
      const float4 v = *reinterpret_cast<const float4*>(&sv[t][4 * quad]);
      const float4 u = {beta * (v.x - n[0]), beta * (v.y - n[1]), beta * (v.z - n[2]), beta * (v.w - n[3])};
#pragma unroll
      for (int i = 0; i < FEAT; ++i) {
        const float k = sk[t][grp + kStepGroups * i];
        s[i].x = fmaf(k, u.x, s[i].x);
        s[i].y = fmaf(k, u.y, s[i].y);
        s[i].z = fmaf(k, u.z, s[i].z);
        s[i].w = fmaf(k, u.w, s[i].w);
      }
      if (grp == 0)
        store4(O + (int64_t)(t0 + t) * a.o.row + 4 * quad, a.scale * fmaf(n[8], u.x, n[4]), a.scale * fmaf(n[8], u.y, n[5]),
               a.scale * fmaf(n[8], u.z, n[6]), a.scale * fmaf(n[8], u.w, n[7]));
    }
  }
#pragma unroll
  for (int i = 0; i < FEAT; ++i) *reinterpret_cast<float4*>(S + (int64_t)(grp + kStepGroups * i) * a.d) = s[i];
}

template <typename T>
hipError_t launch_step(const DeltaStepArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.count * a.H * (a.d / kStepCols))), block(8 * kStepCols);
  switch (a.D) {
    case 32: hipLaunchKernelGGL((delta_step_kernel<T, 1>), grid, block, 0, s, a); break;
    case 64: hipLaunchKernelGGL((delta_step_kernel<T, 2>), grid, block, 0, s, a); break;
    case 128: hipLaunchKernelGGL((delta_step_kernel<T, 4>), grid, block, 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_step(Dt dt, const DeltaStepArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_step<__bf16>(a, s) : launch_step<float>(a, s);
}

}  // namespace luna
