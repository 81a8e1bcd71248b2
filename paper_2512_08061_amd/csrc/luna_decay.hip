// luna_decay.hip -- around the chunked decay kernel (luna_decay.hpp): the discounted prefixes
// of the pieces' states, the row weights of the backward pass, and which instantiation runs.
#include "luna_seq.hpp"

namespace luna {

namespace {

// Before: state p of a sequence and head is what piece p adds (all but the last piece).  After: the state before piece p,
// S_p = f^piece S_{p-1} + X_{p-1}, from the caller's state or zero.  Four elements per thread; loads of the next piece do
// not wait for the sums.  A workgroup per sequence, or, where the sequences are more than the states, per state: the
// sequence whose first one it is, which is the last whose first state is not behind it, if that is longer than a piece.
__global__ __launch_bounds__(256) void decay_scan_kernel(DecayArgs a, int64_t elems) {
  const int head = blockIdx.y;
  int b = blockIdx.z;
  if (gridDim.z < a.s.count) {
    b = seq_last(a.s, [&](int64_t i, int64_t first) { return seq_first_state(a.s, i, first, a.piece) <= blockIdx.z; });
    if (b < 0) return;
  }
  const int64_t e = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (e >= elems) return;
  const SeqPiece sp = seq_of(a.s, b);
  const int pieces = (int)(((int64_t)sp.len + a.piece - 1) / a.piece);
  const int64_t at0 = seq_first_state(a.s, b, sp.first, a.piece);
  if (pieces < 2 || (gridDim.z < a.s.count && at0 != blockIdx.z)) return;
  const int64_t step = a.H * decay_state_floats(a.dk, a.dv);
  float* x = a.states + at0 * step + head * decay_state_floats(a.dk, a.dv) + e;
  const auto at = [&](int p) { return reinterpret_cast<f32x4*>(x + p * step); };
  const float f = exp2_raw(decay_log2(a.log_decay[head]) * (float)a.piece);
  f32x4 run = zero4(), next = *at(0);
  if (a.S) {
    const int64_t zat = (int64_t)a.dk * a.dv, user = (int64_t)b * a.H + head;
    if (e < zat) run = *reinterpret_cast<const f32x4*>(a.S + user * zat + e);
    else if (a.z && e - zat < a.dk)
#pragma unroll
      for (int j = 0; j < 4; ++j) run[j] = a.z[user * a.dk + e - zat + j];
  }
  for (int p = 0; p < pieces; ++p) {
    const f32x4 add = next;
    if (p + 2 < pieces) next = *at(p + 1);
    *at(p) = run;
    run = f * run + add;
  }
}

// w_i = 1 / (den_i + eps), delta_i = -dO_i.out_i: a quarter wave per row.
template <typename T>
__global__ __launch_bounds__(256) void decay_weights_kernel(DecayWeightsArgs a) {
  const int head = blockIdx.y;
  const SeqPiece sp = seq_piece(a.s, blockIdx.x, 64);
  if (sp.seq < 0) return;
  const bool packed = a.s.offsets != nullptr;
  const int sub = threadIdx.x % 16;
  constexpr int E = 16 / (int)sizeof(T);
  for (int r = threadIdx.x / 16; r < 64; r += 16) {
    const int i = sp.index * 64 + r;
    if (i >= sp.len) break;
    const char* g = seq_row(a.dO, sp, packed, head, i, sizeof(T));
    const char* o = seq_row(a.out, sp, packed, head, i, sizeof(T));
    float x = 0.0f;
    for (int c = sub * E; c < a.d; c += 16 * E) {
      const i32x4 gv = *reinterpret_cast<const i32x4*>(g + c * sizeof(T)), ov = *reinterpret_cast<const i32x4*>(o + c * sizeof(T));
      const T* gt = reinterpret_cast<const T*>(&gv);
      const T* ot = reinterpret_cast<const T*>(&ov);
#pragma unroll
      for (int e = 0; e < E; ++e) x = fmaf((float)gt[e], (float)ot[e], x);
    }
    x += __shfl_xor(x, 1);
    x += __shfl_xor(x, 2);
    x += __shfl_xor(x, 4);
    x += __shfl_xor(x, 8);
    if (sub == 0) {
      const int64_t num = seq_num(a.s, sp, a.H, head, i);
      a.w[num] = 1.0f / (a.den[num] + a.eps);
      a.delta[num] = -x;
    }
  }
}

}  // namespace

template <typename T, int MODE>
hipError_t launch_decay_typed(const DecayArgs& a, bool out, hipStream_t s);
extern template hipError_t launch_decay_typed<__bf16, kDecayPlain>(const DecayArgs&, bool, hipStream_t);
extern template hipError_t launch_decay_typed<__bf16, kDecayNorm>(const DecayArgs&, bool, hipStream_t);
extern template hipError_t launch_decay_typed<__bf16, kDecayAug>(const DecayArgs&, bool, hipStream_t);
extern template hipError_t launch_decay_typed<float, kDecayPlain>(const DecayArgs&, bool, hipStream_t);
extern template hipError_t launch_decay_typed<float, kDecayNorm>(const DecayArgs&, bool, hipStream_t);
extern template hipError_t launch_decay_typed<float, kDecayAug>(const DecayArgs&, bool, hipStream_t);

bool decay_supported(int dk, int dv) {
  return (dk == 32 || dk == 64 || dk == 128 || dk == 256) && (dv == 32 || dv == 64 || dv == 128);
}

static hipError_t launch_decay(Dt dt, int mode, const DecayArgs& a, bool out, hipStream_t s) {
  if (dt == Dt::BF16)
    return mode == kDecayPlain ? launch_decay_typed<__bf16, kDecayPlain>(a, out, s)
           : mode == kDecayNorm ? launch_decay_typed<__bf16, kDecayNorm>(a, out, s)
                                : launch_decay_typed<__bf16, kDecayAug>(a, out, s);
  return mode == kDecayPlain ? launch_decay_typed<float, kDecayPlain>(a, out, s)
         : mode == kDecayNorm ? launch_decay_typed<float, kDecayNorm>(a, out, s)
                              : launch_decay_typed<float, kDecayAug>(a, out, s);
}
hipError_t launch_decay_states(Dt dt, int mode, const DecayArgs& a, hipStream_t s) {
  return launch_decay(dt, mode, a, false, s);
}
hipError_t launch_decay_out(Dt dt, int mode, const DecayArgs& a, hipStream_t s) { return launch_decay(dt, mode, a, true, s); }

hipError_t launch_decay_scan(const DecayArgs& a, hipStream_t s) {
  const int64_t elems = decay_state_floats(a.dk, a.dv);  // (a multiple of 4; unused ones of z too)
  const int64_t sequences = a.s.count < a.nstates ? a.s.count : a.nstates;
  const dim3 grid((unsigned)((elems / 4 + 255) / 256), (unsigned)a.H, (unsigned)sequences);
  hipLaunchKernelGGL(decay_scan_kernel, grid, dim3(256), 0, s, a, elems);
  return hipGetLastError();
}

hipError_t launch_decay_weights(Dt dt, const DecayWeightsArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)seq_slots(a.s, 64), (unsigned)a.H);
  if (dt == Dt::BF16) hipLaunchKernelGGL(decay_weights_kernel<__bf16>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(decay_weights_kernel<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace luna
