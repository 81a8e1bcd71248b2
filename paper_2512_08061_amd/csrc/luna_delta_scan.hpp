// luna_delta_scan.hpp -- the passes of the gated delta rule that are serial in the chunks (luna_delta.hpp): a wave takes 16
// value columns of one sequence and head from the first chunk to the last (the backward pass: from the last to the first),
// with its columns of the state in registers, as the accumulator tiles of S' = .. + K^T U.
//
// Every product's result is the next one's operand as it lies in the registers, so that a chunk needs no exchange between
// lanes: rows 4g + e of a pair of tiles 2s, 2s + 1 stand for features (and tokens) 32 s + 8 g + e and 32 s + 8 g + 4 + e, the
// eight k-slots of lane group g.  K S and N (beta R) take such pairs as their B operand, out^T = S^T Q^T + U^T P^T the same
// registers as its A operand.  K and Q lie in LDS as their rows; K^T is read transposed.  What bounds them is the chain of a
// chunk, 4.1 us for the gradients' of bf16 with D = d = 128 (2 x 16 heads of 2048 tokens: 132 us for both, side by side).
#pragma once

#include "luna_delta.hpp"

namespace luna {

// The tiles of a chunk.
template <typename T, int DK, int DVW, int NP, int PP, bool OUT>
struct ScanLds {
  static constexpr int C = kDeltaChunk, PAD = 16 / (int)sizeof(T), PK = DK + PAD, PV = DVW + PAD, PN = C + PAD;
  T k[C][PK];
  T q[OUT ? C : 1][PK];
  T v[C][PV];
  T n[NP][C][PN];
  T p[OUT ? PP : 1][OUT ? C : 1][PN];
  float gates[4][C];
  int since[DVW];  // per column: the first token with a value that is not finite
};

// Token (feature) of row r of tile i of such pairs, and of rows 4 g .. 4 g + 3.
__device__ __forceinline__ int pair_row(int i, int r) { return 32 * (i / 2) + 8 * (r / 4) + 4 * (i % 2) + r % 4; }
__device__ __forceinline__ int pair_rows(int i, int g) { return 32 * (i / 2) + 8 * g + 4 * (i % 2); }

// N x [64][64] from the workspace to LDS, a chunk ahead.
template <typename T, int N, int PN, int THREADS>
struct ScanMatrix {
  DecayRows<T, kDeltaChunk, kDeltaChunk, PN, THREADS> x[N];
  __device__ __forceinline__ void load(const char* from) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      x[i].load(from + (int64_t)i * kDeltaChunk * kDeltaChunk * sizeof(T), kDeltaChunk, kDeltaChunk, kDeltaChunk, false);
  }
  __device__ __forceinline__ void store(T (*to)[kDeltaChunk][PN]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i].store(&to[i][0][0]);
  }
};

// rows from `first` on as zeros
template <typename T, int C, int W, int P, int THREADS>
__device__ __forceinline__ void clear_rows(DecayRows<T, C, W, P, THREADS>& x, int first) {
  using R = DecayRows<T, C, W, P, THREADS>;
#pragma unroll
  for (int i = 0; i < R::N; ++i)
    if ((threadIdx.x + THREADS * i) / R::PER >= (unsigned)first) x.x[i] = i32x4{0, 0, 0, 0};
}

// The transposed operand of tile i (16 features or tokens as pair_row says) over rows k0 + 8 g .. + 7 of an LDS tile.
template <typename T>
__device__ __forceinline__ void load_pair_tr(Frag<T>& f, const T* x, int pitch, int i, int k0, int lane) {
  const int first = 32 * (i / 2) + 4 * (i % 2), row = k0 + 8 * (lane / 16);
#pragma unroll
  for (int half = 0; half < 2; ++half)
    load_tr4_at(f, 4 * half, lane, [&](int kk, int col) { return x + (row + 4 * half + kk) * pitch + first + 8 * (col / 4) + col % 4; });
}
template <typename T, int P>
__device__ __forceinline__ void load_op_pair_tr(DeltaOp<T, P>& f, const T* x, int part, int pitch, int i, int k0, int lane) {
  const int first = 32 * (i / 2) + 4 * (i % 2), row = k0 + 8 * (lane / 16);
#pragma unroll
  for (int half = 0; half < 2; ++half)
    load_op_tr4(f, 4 * half, lane, part,
                [&](int kk, int col) { return x + (row + 4 * half + kk) * pitch + first + 8 * (col / 4) + col % 4; });
}

// From the first chunk to the last.  OUT: writes out and returns the state, else leaves E and the states before the chunks for the
// backward pass.  HELP: waves that only load, a chunk ahead (0: all load).
template <typename T, int DK, int DVW, int NP, int HELP, bool OUT>
__device__ __forceinline__ void delta_scan(const DeltaArgs& a, int block, char* raw) {
  using Lds = ScanLds<T, DK, DVW, NP, 1, OUT>;
  constexpr int C = Lds::C, FT = DK / 16, FS = DK / 32, KT = C / 16, KS = C / 32, esz = (int)sizeof(T), THREADS = HELP ? 64 * HELP : 4 * DVW;  // (those that load)
  constexpr int TI = FT < 4 ? FT : 4, TN = FT * KS / TI;  // tiles of a batch of transposed reads, and batches
  static_assert(!OUT || sizeof(T) == 4, "bf16 has a forward kernel of its own");
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int tid = threadIdx.x, lane = tid % kWave, wave = wave_id() - HELP, g = lane / 16, c = lane % 16;
  const int slices = a.d / DVW;
  const int slice = block % slices, head = (block / slices) % a.H, b = block / slices / a.H;
  const SeqPiece sp = seq_uniform(seq_of(a.s, b));
  if (sp.len == 0) return;
  const bool packed = a.s.offsets != nullptr;
  const int hk = head / (a.H / a.Hk), col0 = slice * DVW, wcol = 16 * wave;
  const int slot0 = delta_first_slot(a.s, sp), chunks = (sp.len + C - 1) / C;
  constexpr int64_t nbytes = (int64_t)delta_parts<T>(NP) * C * C * esz, pbytes = (int64_t)C * C * esz;
  constexpr int kNever = 1 << 30;

  DecayRows<T, C, DK, Lds::PK, THREADS> kr, qr;
  DecayRows<T, C, DVW, Lds::PV, THREADS> vr;
  ScanMatrix<T, NP, Lds::PN, THREADS> nr;
  ScanMatrix<T, 1, Lds::PN, THREADS> pr;
  constexpr int GN = 4 * C / THREADS;
  float gr[GN];
  int br = C;
  const auto load = [&](int chunk) {
    const int t0 = chunk * C, m = min(C, sp.len - t0);
    const int64_t at = (int64_t)(slot0 + chunk) * a.H + head;
    kr.load(seq_row(a.k, sp, packed, hk, t0, esz), a.k.row, m, DK, false);
    vr.load(seq_row(a.v, sp, packed, head, t0, esz) + col0 * esz, a.v.row, m, DVW, false);
    nr.load(a.n + at * nbytes);
    if constexpr (OUT) {
      qr.load(seq_row(a.q, sp, packed, hk, t0, esz), a.q.row, m, DK, false);
      pr.load(a.p + at * pbytes);
    }
    const float* gates = a.gates + at * kDeltaGates;
#pragma unroll
    for (int i = 0; i < GN; ++i) gr[i] = gates[tid + THREADS * i];
    br = __float_as_int(gates[kDeltaMisc * C + 1]);
  };
  for (int i = tid; i < DVW; i += THREADS) l.since[i] = kNever;

  const auto put = [&](int t0) {
    const int bad = __builtin_amdgcn_readfirstlane(br);
    if (bad < C) clear_rows(kr, bad);
    kr.store(&l.k[0][0]);
    if constexpr (OUT) {
      vr.clean(l.since, t0);
      qr.store(&l.q[0][0]);
      pr.store(l.p);
    }
    vr.store(&l.v[0][0]);
    nr.store(l.n);
#pragma unroll
    for (int i = 0; i < GN; ++i) (&l.gates[0][0])[tid + THREADS * i] = gr[i];
  };
  if (!HELP || wave < 0) load(0);
  if (HELP && wave < 0) {
    for (int chunk = 0; chunk < chunks; ++chunk) {
      __syncthreads();
      put(chunk * C);
      __syncthreads();
      if (chunk + 1 < chunks) load(chunk + 1);
    }
    return;
  }

  f32x4 S[FT];
  const int64_t state = ((int64_t)b * a.H + head) * a.D * a.d + col0 + wcol + c;
#pragma unroll
  for (int ft = 0; ft < FT; ++ft)
#pragma unroll
    for (int j = 0; j < 4; ++j) S[ft][j] = OUT && a.S ? a.S[state + (int64_t)(pair_rows(ft, g) + j) * a.d] : 0.0f;

  int lost = kNever;  // the first token with a key or gate that is not finite
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const int t0 = chunk * C, m = min(C, sp.len - t0);
    const int64_t at = (int64_t)(slot0 + chunk) * a.H + head;
    __syncthreads();  // the chunk before is no longer read
    if constexpr (!HELP) {
      put(t0);
      if (chunk + 1 < chunks) load(chunk + 1);
    }
    __syncthreads();
    if constexpr (OUT) {
      const int bad = __builtin_amdgcn_readfirstlane(reinterpret_cast<const int&>(l.gates[kDeltaMisc][1]));
      if (bad < C) lost = min(lost, t0 + bad);
    }

    if (!OUT) {  // the state before the chunk, [d][D]
      float* to = a.before + (at * a.d + col0 + wcol + c) * DK;
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) *reinterpret_cast<f32x4*>(to + pair_rows(ft, g)) = S[ft];
    }
    // (operands are read from LDS a batch before their products)
    f32x4 r[KT], o[KT];
    Frag<T> kf[2][KT], qf[2][OUT ? KT : 1], tf[2][TI];
    DeltaOp<T, NP> nf[KT][KS];
    const auto read_k = [&](int t) {
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        load8(kf[t % 2][i], &l.k[pair_row(i, c)][32 * t + 8 * g]);
        if constexpr (OUT) load8(qf[t % 2][i], &l.q[16 * i + c][32 * t + 8 * g]);
      }
    };
    const auto read_t = [&](int n) {
#pragma unroll
      for (int i = 0; i < TI; ++i) load_pair_tr(tf[n % 2][i], &l.k[0][0], Lds::PK, (TI * n + i) % FT, 32 * ((TI * n + i) / FT), lane);
    };
    const auto gate4 = [&](int which, int i) { return *reinterpret_cast<const f32x4*>(&l.gates[which][pair_rows(i, g)]); };
    f32x4 first[KT], beta[KT], last[KT];
    Frag<T> v[KT];
    read_k(0);
#pragma unroll
    for (int i = 0; i < KT; ++i) r[i] = zero4(), o[i] = zero4();
#pragma unroll
    for (int t = 0; t < FS; ++t) {
      if (t + 1 < FS) read_k(t + 1);
      else
#pragma unroll
        for (int i = 0; i < KT; ++i) {
          first[i] = gate4(kDeltaFirst, i);
          beta[i] = gate4(kDeltaBeta, i);
          last[i] = gate4(kDeltaLast, i);
          load_tr4(v[i], 0, &l.v[0][0], Lds::PV, pair_rows(i, g), wcol, lane);
#pragma unroll
          for (int s = 0; s <= i / 2; ++s) load_op(nf[i][s], &l.n[0][pair_row(i, c)][32 * s + 8 * g], C * Lds::PN);
        }
      DeltaOp<T, NP> sf;
      set_tiles(sf, S[2 * t], S[2 * t + 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        mma(r[i], kf[t % 2][i], sf);
        if constexpr (OUT) mma(o[i], sf, qf[t % 2][i]);
      }
    }
    // R and beta R
    DeltaOp<T, NP> br[KS];
    {
      f32x4 x[KT];
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          r[i][e] = fmaf(-first[i][e], r[i][e], v[i].get(e));
          x[i][e] = beta[i][e] * r[i][e];
        }
#pragma unroll
      for (int s = 0; s < KS; ++s) set_tiles(br[s], x[2 * s], x[2 * s + 1]);
    }
    read_t(0);
    __builtin_amdgcn_sched_barrier(0);
    // E = R + N (beta R), of whose rows 32 s .. the columns up to 32 s + 31
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 2 * s; i < KT; ++i) mma(r[i], nf[i][s], br[s]);
    if (!OUT) {
      float* to = a.e + (at * a.d + col0 + wcol + c) * C;
#pragma unroll
      for (int i = 0; i < KT; ++i) *reinterpret_cast<f32x4*>(to + pair_rows(i, g)) = r[i];
    }
    // U, and U discounted to the chunk's end
    DeltaOp<T, NP> uf[KS];
    DeltaOp<T, NP> ul[KS];
    {
      f32x4 x[KT];
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          r[i][e] *= beta[i][e];
          x[i][e] = last[i][e] * r[i][e];
        }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        if constexpr (OUT) set_tiles(uf[s], r[2 * s], r[2 * s + 1]);
        set_tiles(ul[s], x[2 * s], x[2 * s + 1]);
      }
    }
    {
      const float whole = l.gates[kDeltaMisc][0];
#pragma unroll
      for (int ft = 0; ft < FT; ++ft)
#pragma unroll
        for (int j = 0; j < 4; ++j) S[ft][j] *= whole;
    }
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      if (n + 1 < TN) read_t(n + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TI; ++i) mma(S[(TI * n + i) % FT], tf[n % 2][i], ul[(TI * n + i) / FT]);
    }
    if constexpr (OUT) {
      const Buf to = buffer(seq_row(a.o, sp, packed, head, t0, esz) + col0 * esz, (int)(((m - 1) * a.o.row + DVW) * esz));
      const i32x4 since = *reinterpret_cast<const i32x4*>(&l.since[wcol + 4 * g]);
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        const int row = 16 * i + c;
        const float first = a.scale * l.gates[kDeltaFirst][row];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] *= first;
#pragma unroll
        for (int s = 0; s <= i / 2; ++s) {
          Frag<T> f;
          load8(f, &l.p[0][row][32 * s + 8 * g]);
          mma(o[i], uf[s], f);
        }
      }
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        const int row = 16 * i + c;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] = t0 + row >= min(since[e], lost) ? __builtin_nanf("") : o[i][e];
        buf_store4<T>(to, row < m ? (row * (int)a.o.row + wcol + 4 * g) * esz : kPastEnd, o[i][0], o[i][1], o[i][2], o[i][3]);
      }
    }
  }
  if (OUT && a.S) {
    const bool gone = min(l.since[wcol + c], lost) != kNever;
#pragma unroll
    for (int ft = 0; ft < FT; ++ft)
#pragma unroll
      for (int j = 0; j < 4; ++j) a.S[state + (int64_t)(pair_rows(ft, g) + j) * a.d] = gone ? __builtin_nanf("") : S[ft][j];
  }
}

// The gradients of the states and X, from the last chunk to the first.
template <typename T, int DK, int DVW, int NP, int HELP>
__device__ __forceinline__ void delta_back(const DeltaArgs& a, int block, char* raw) {
  using Lds = ScanLds<T, DK, DVW, NP, NP, true>;
  constexpr int C = Lds::C, FT = DK / 16, FS = DK / 32, KT = C / 16, KS = C / 32, esz = (int)sizeof(T), THREADS = HELP ? 64 * HELP : 4 * DVW;  // (those that load)
  constexpr int TI = FT < 4 ? FT : 4, TN = FT * KS / TI;  // tiles of a batch of transposed reads, and batches
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int tid = threadIdx.x, lane = tid % kWave, wave = wave_id() - HELP, g = lane / 16, c = lane % 16;
  const int slices = a.d / DVW;
  const int slice = block % slices, head = (block / slices) % a.H, b = block / slices / a.H;
  const SeqPiece sp = seq_uniform(seq_of(a.s, b));
  if (sp.len == 0) return;
  const bool packed = a.s.offsets != nullptr;
  const int hk = head / (a.H / a.Hk), col0 = slice * DVW, wcol = 16 * wave;
  const int slot0 = delta_first_slot(a.s, sp), chunks = (sp.len + C - 1) / C;
  constexpr int64_t nbytes = (int64_t)NP * C * C * esz;

  DecayRows<T, C, DK, Lds::PK, THREADS> kr, qr;
  DecayRows<T, C, DVW, Lds::PV, THREADS> vr;
  ScanMatrix<T, NP, Lds::PN, THREADS> nr, pr;
  constexpr int GN = 4 * C / THREADS;
  float gr[GN];
  const auto load = [&](int chunk) {
    const int t0 = chunk * C, m = min(C, sp.len - t0);
    const int64_t at = (int64_t)(slot0 + chunk) * a.H + head;
    kr.load(seq_row(a.k, sp, packed, hk, t0, esz), a.k.row, m, DK, false);
    qr.load(seq_row(a.q, sp, packed, hk, t0, esz), a.q.row, m, DK, false);
    vr.load(seq_row(a.o, sp, packed, head, t0, esz) + col0 * esz, a.o.row, m, DVW, false);
    nr.load(a.n + at * nbytes);
    pr.load(a.p + at * nbytes);
    const float* gates = a.gates + at * kDeltaGates;
#pragma unroll
    for (int i = 0; i < GN; ++i) gr[i] = gates[tid + THREADS * i];
  };
  const auto put = [&] {
    kr.store(&l.k[0][0]);
    qr.store(&l.q[0][0]);
    vr.store(&l.v[0][0]);
    nr.store(l.n);
    pr.store(l.p);
#pragma unroll
    for (int i = 0; i < GN; ++i) (&l.gates[0][0])[tid + THREADS * i] = gr[i];
  };
  if (!HELP || wave < 0) load(chunks - 1);
  if (HELP && wave < 0) {
    for (int chunk = chunks - 1; chunk >= 0; --chunk) {
      __syncthreads();
      put();
      __syncthreads();
      if (chunk > 0) load(chunk - 1);
    }
    return;
  }
  f32x4 S[FT];
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) S[ft] = zero4();
  for (int chunk = chunks - 1; chunk >= 0; --chunk) {
    const int64_t at = (int64_t)(slot0 + chunk) * a.H + head;
    __syncthreads();  // the chunk behind is no longer read
    if constexpr (!HELP) {
      put();
      if (chunk > 0) load(chunk - 1);
    }
    __syncthreads();

    {  // [d][D]
      float* to = a.after + (at * a.d + col0 + wcol + c) * DK;
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) *reinterpret_cast<f32x4*>(to + pair_rows(ft, g)) = S[ft];
    }
    // (operands are read from LDS a batch before their products)
    f32x4 x[KT];
    Frag<T> kf[2][KT], qt[2][TI], kt[2][TI], of[KS];
    DeltaOp<T, NP> pf[KT][KS], nf[KT][KS], os[KS];
    const auto read_k = [&](int t) {
#pragma unroll
      for (int i = 0; i < KT; ++i) load8(kf[t % 2][i], &l.k[pair_row(i, c)][32 * t + 8 * g]);
    };
    const auto read_t = [&](int n) {
#pragma unroll
      for (int i = 0; i < TI; ++i) {
        load_pair_tr(qt[n % 2][i], &l.q[0][0], Lds::PK, (TI * n + i) % FT, 32 * ((TI * n + i) / FT), lane);
        load_pair_tr(kt[n % 2][i], &l.k[0][0], Lds::PK, (TI * n + i) % FT, 32 * ((TI * n + i) / FT), lane);
      }
    };
    const auto gate4 = [&](int which, int i) { return *reinterpret_cast<const f32x4*>(&l.gates[which][pair_rows(i, g)]); };
    f32x4 first[KT], beta[KT], last[KT];
    read_k(0);
#pragma unroll
    for (int i = 0; i < KT; ++i) x[i] = zero4();
#pragma unroll
    for (int t = 0; t < FS; ++t) {
      if (t + 1 < FS) {
        read_k(t + 1);
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          load_tr4(of[s], 0, &l.v[0][0], Lds::PV, 32 * s + 8 * g, wcol, lane);
          load_tr4(of[s], 4, &l.v[0][0], Lds::PV, 32 * s + 8 * g + 4, wcol, lane);
        }
#pragma unroll
        for (int i = 0; i < KT; ++i) {
          first[i] = gate4(kDeltaFirst, i);
          beta[i] = gate4(kDeltaBeta, i);
          last[i] = gate4(kDeltaLast, i);
#pragma unroll
          for (int s = i / 2; s < KS; ++s) load_op_pair_tr(pf[i][s], &l.p[0][0][0], C * Lds::PN, Lds::PN, i, 32 * s, lane);
        }
      }
      DeltaOp<T, NP> sf;
      set_tiles(sf, S[2 * t], S[2 * t + 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < KT; ++i) mma(x[i], kf[t % 2][i], sf);
    }
    // dU
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      x[i] *= last[i];
#pragma unroll
      for (int s = i / 2; s < KS; ++s) load_op_pair_tr(nf[i][s], &l.n[0][0][0], C * Lds::PN, Lds::PN, i, 32 * s, lane);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < 2 * s + 2; ++i) mma(x[i], pf[i][s], of[s]);
    // scale e^G dO
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = a.scale * first[2 * s + e / 4][e % 4] * of[s].get(e);
      os[s].set(y);
    }
    // X = dU + N^T (beta dU)
    DeltaOp<T, NP> bu[KS];
    {
      f32x4 y[KT];
#pragma unroll
      for (int i = 0; i < KT; ++i) y[i] = beta[i] * x[i];
#pragma unroll
      for (int s = 0; s < KS; ++s) set_tiles(bu[s], y[2 * s], y[2 * s + 1]);
    }
    read_t(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < 2 * s + 2; ++i) mma(x[i], nf[i][s], bu[s]);
    {
      float* to = a.x + (at * a.d + col0 + wcol + c) * C;
#pragma unroll
      for (int i = 0; i < KT; ++i) *reinterpret_cast<f32x4*>(to + pair_rows(i, g)) = x[i];
    }
    // - e^G beta X
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] *= -first[i][e] * beta[i][e];
#pragma unroll
    for (int s = 0; s < KS; ++s) set_tiles(bu[s], x[2 * s], x[2 * s + 1]);
    {
      const float whole = l.gates[kDeltaMisc][0];
#pragma unroll
      for (int ft = 0; ft < FT; ++ft)
#pragma unroll
        for (int j = 0; j < 4; ++j) S[ft][j] *= whole;
    }
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      if (n + 1 < TN) read_t(n + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TI; ++i) mma(S[(TI * n + i) % FT], qt[n % 2][i], os[(TI * n + i) / FT]);
#pragma unroll
      for (int i = 0; i < TI; ++i) mma(S[(TI * n + i) % FT], kt[n % 2][i], bu[(TI * n + i) / FT]);
    }
  }
}

template <typename T, int DK, int DVW, int HELP>
__global__ __launch_bounds__(4 * DVW + 64 * HELP, 1) void delta_scan_kernel(DeltaArgs a) {
  extern __shared__ __attribute__((aligned(16))) char raw[];
  delta_scan<T, DK, DVW, 1, HELP, true>(a, blockIdx.x, raw);
}
// Both passes of the backward half: neither needs what the other writes, and each alone has few workgroups.
template <typename T, int DK, int DVW, int NP, int HELP>
__global__ __launch_bounds__(4 * DVW + 64 * HELP, 1) void delta_both_kernel(DeltaArgs a) {
  extern __shared__ __attribute__((aligned(16))) char raw[];
  const int half = gridDim.x / 2;
  if ((int)blockIdx.x < half) delta_back<T, DK, DVW, NP, HELP>(a, blockIdx.x, raw);
  else delta_scan<T, DK, DVW, NP, HELP, false>(a, blockIdx.x - half, raw);
}

template <typename T, int DK, int DVW, int HELP>
hipError_t launch_scan_one(const DeltaArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(ScanLds<T, DK, DVW, 1, 1, true>);
  static_assert(bytes <= 160 * 1024, "one workgroup's LDS");
  const hipError_t e = allow_lds<delta_scan_kernel<T, DK, DVW, HELP>>(bytes);
  if (e != hipSuccess) return e;
  const int64_t groups = a.s.count * a.H * (a.d / DVW);
  hipLaunchKernelGGL((delta_scan_kernel<T, DK, DVW, HELP>), dim3((unsigned)groups), dim3(4 * DVW + 64 * HELP), bytes, s, a);
  return hipGetLastError();
}
template <typename T, int DK, int DVW, int NP, int HELP>
hipError_t launch_both_one(const DeltaArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(ScanLds<T, DK, DVW, NP, NP, true>);
  static_assert(bytes <= 160 * 1024 && bytes >= (int)sizeof(ScanLds<T, DK, DVW, NP, 1, false>), "one workgroup's LDS");
  const hipError_t e = allow_lds<delta_both_kernel<T, DK, DVW, NP, HELP>>(bytes);
  if (e != hipSuccess) return e;
  const int64_t groups = 2 * a.s.count * a.H * (a.d / DVW);
  hipLaunchKernelGGL((delta_both_kernel<T, DK, DVW, NP, HELP>), dim3((unsigned)groups), dim3(4 * DVW + 64 * HELP), bytes, s, a);
  return hipGetLastError();
}

constexpr int kScanHelp = 2;  // waves that load, beside those of 32 columns (see delta_narrow)
template <typename T, int DK, int DVW, int NP, bool BOTH>
hipError_t launch_scan_width(const DeltaArgs& a, hipStream_t s) {
  constexpr int help = DVW == 32 ? kScanHelp : 0;
  if constexpr (BOTH) return launch_both_one<T, DK, DVW, NP, help>(a, s);
  else return launch_scan_one<T, DK, DVW, help>(a, s);
}
template <typename T, int DK, int NP, bool BOTH>
hipError_t launch_scan_feature(const DeltaArgs& a, hipStream_t s) {
  const bool equal = !a.s.offsets && !a.s.lens;
  return delta_narrow(DK, a.d, (BOTH ? 2 : 1) * a.s.count * a.H * (a.d / 32), equal) ? launch_scan_width<T, DK, 32, NP, BOTH>(a, s)
                                                                                     : launch_scan_width<T, DK, 64, NP, BOTH>(a, s);
}
template <typename T, int NP, bool BOTH>
hipError_t launch_scan_all(const DeltaArgs& a, hipStream_t s) {
  return a.D == 32 ? launch_scan_feature<T, 32, NP, BOTH>(a, s) : a.D == 64 ? launch_scan_feature<T, 64, NP, BOTH>(a, s)
                                                                            : launch_scan_feature<T, 128, NP, BOTH>(a, s);
}

}  // namespace luna
