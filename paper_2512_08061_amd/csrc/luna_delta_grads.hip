// luna_delta_grads.hip -- the gradients of the gated delta rule within each chunk (luna_delta.hpp), for all chunks side by side,
// from the states before the chunks S, the gradients of the states behind them dS', E and X.  With U = beta E and
// dR = beta X (dV), Gamma_ij = e^(G_i - G_j):
//
//   dbeta_i = X_i.E_i,   dP_ij = dO_i.U_j (j <= i),   dM_ij = -dR_i.U_j (j < i),
//   dQ = scale e^G (dO S^T) + (scale dP Gamma) K,
//   dK = e^(G_C - G) (U dS'^T) - e^G (dR S^T) + (scale dP Gamma)^T Q + (dM Gamma) K + (dM Gamma)^T K,
//   dG_i = q_i.(scale e^G dO S^T)_i - k_i.(e^G dR S^T)_i - k_i.(e^(G_C - G) U dS'^T)_i
//          + sum_j w_ij - sum_j w_ji,   w = dP P + dM M,
//   dG_C = sum_i k_i.(e^(G_C - G) U dS'^T)_i + e^(G_C) <dS', S>,
//   dlog_decay_t = sum_{i >= t} dG_i + dG_C.
//
// A workgroup takes a chunk of one key head and adds up over the value heads of its group, in their order (with few chunks each value
// head has a workgroup, and a launch behind adds up); a wave has 16 features of dQ and dK, formed transposed, so that a lane holds
// four neighbouring features of a token.  What bounds it is one workgroup a compute unit (eight waves of 256 registers fill the
// register files, U and dR in parts the LDS) in phases that wait for memory, for the LDS and for one another: bf16, 2 x 16 heads of
// 2048 tokens, D = d = 128, 114 us for 0.33 GB.
#include "luna_delta.hpp"

namespace luna {

namespace {

constexpr int C = kDeltaChunk, KT = C / 16, KS = C / 32;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

template <int DK>
constexpr int kGradWaves = DK == 128 ? 8 : 4;
template <typename T, int DK, int DV, int NP>
struct GradLds {
  static constexpr int PAD = 16 / (int)sizeof(T), PK = DK + PAD, PA = C + PAD, PT = sizeof(T) == 2 ? C : PA, W = kGradWaves<DK>;
  T k[C][PK], q[C][PK];
  union {
    struct {
      T u[NP][DV][PT], r[NP][DV][PT];  // U and dR, transposed
    };
    struct {
      T ap[NP][C][PA], am[NP][C][PA];  // scale dP Gamma and dM Gamma
    };
  };
  // Place of a column's token in u and r: in bf16 the 16-byte pieces are swapped by the row's number, so that the two pieces of eight
  // rows that half a wave of transposing reads meets lie in different banks (padded rows: 40% of the LDS's cycles were conflicts).
  static __device__ __forceinline__ int at(int row, int col) {
    return sizeof(T) == 2 ? row * PT + ((col / 8 ^ (4 * (row / 2 % 2) + 2 * (row / 8 % 2))) * 8) + col % 8 : row * PT + col;
  }
  float gates[kDeltaGateRows][C];
  union {
    float beta[4 * W][C];  // shares of dbeta
    struct {
      float row[KT][C], col[KT][C];  // sums of w over the columns of block jt, and over the rows of block it
      float dots[W][2][C];
    };
  };
  float state[W];               // shares of <dS', S>
};

// A tile of 16 tokens of U or dR as an operand over the columns 32 s + 8 g .. + 7 of d.
template <typename Lds, typename T, int NP, int DV>
struct GradTile {
  unsigned at;  // this lane's place in tile `it` of u, or of r
  __device__ __forceinline__ GradTile(const T* x, int it, int lane) {
    const int g = lane / 16, c = lane % 16;
    at = lds_address(x) + (sizeof(T) == 2 ? Lds::at(8 * g + c / 4, 16 * it + 4 * (c % 4)) : Lds::at(8 * g, 16 * it + c)) * (int)sizeof(T);
  }
  __device__ __forceinline__ void read(DeltaOp<T, NP>& f, int s) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < NP; ++k) lds_tr(f.p[k], at + (k * DV + 32 * s) * Lds::PT * 2, 4 * Lds::PT * 2);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f.x.v[e] = *(__attribute__((address_space(3))) const float*)(uintptr_t)(at + (32 * s + e) * Lds::PT * 4);
    }
  }
};

template <typename T, int DK, int DV, int NP>
__global__ __launch_bounds__(64 * kGradWaves<DK>, 1) void delta_grads_kernel(DeltaArgs a, int shares) {
  using Lds = GradLds<T, DK, DV, NP>;
  constexpr int W = Lds::W, THREADS = 64 * W, PK = Lds::PK, PA = Lds::PA, PT = Lds::PT, esz = (int)sizeof(T), FS = DK / 32, VS = DV / 32;
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int tid0 = threadIdx.x, wave = wave_id();
  const int hk = blockIdx.x / shares % a.Hk, slot = blockIdx.x / shares / a.Hk, group = a.H / a.Hk;
  const int h0 = blockIdx.x % shares * (group / shares), h1 = h0 + group / shares;  // the value heads
  const SeqPiece sp = seq_uniform(seq_piece(a.s, slot, C));
  if (sp.seq < 0) return;
  const bool packed = a.s.offsets != nullptr, mine = wave < DK / 16;
  const int t0 = sp.index * C, m = min(C, sp.len - t0), feat = mine ? 16 * wave : 0;
  constexpr bool PARK = DK == 128 && DV == 128;  // (registers are short)
  // What a head needs from memory is asked for before the head before it is done, or as early in it as registers allow: a load
  // takes 2000 cycles and more.
  constexpr int NC = DV * 16 / THREADS, NG = (kDeltaGates + THREADS - 1) / THREADS;
  f32x4 ev[NC], xv[NC];
  float gv[NG], lv = 0.0f;
  const auto load_head = [&](int head) {
    const int tid = anew(tid0), lane = tid % kWave, i4 = 4 * (tid % 16);  // U, dR and dbeta: four tokens of a column a thread
    const int64_t at = (int64_t)slot * a.H + head;
    const Buf be = buffer(a.e + at * DV * C, DV * C * 4), bx = buffer(a.x + at * DV * C, DV * C * 4);
    const Buf bg = buffer(a.gates + at * kDeltaGates, kDeltaGates * 4);
    const int off = (tid / 16 * C + i4) * 4;
#pragma unroll
    for (int n = 0; n < NG; ++n) gv[n] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(bg, (tid + THREADS * n) * 4, 0, 0));
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      ev[n] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(be, off, n * (THREADS / 16) * C * 4, 0));
      xv[n] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(bx, off, n * (THREADS / 16) * C * 4, 0));
    }
    lv = a.log_decay[seq_num(a.s, sp, a.H, head, t0 + min(kWave - 1 - lane, m - 1))];
  };
  {
    DecayRows<T, C, DK, PK, THREADS> x, y;
    x.load(seq_row(a.k, sp, packed, hk, t0, esz), a.k.row, m, DK, false);
    y.load(seq_row(a.q, sp, packed, hk, t0, esz), a.q.row, m, DK, false);
    load_head(hk * group + h0);
    x.store(&l.k[0][0]);
    y.store(&l.q[0][0]);
  }
  // The sums over the value heads, in registers or, where these do not suffice for them beside the rest, from head to head in
  // the place of the first one's states, which have been read by then.
  static_assert(!PARK || DV * DK >= 2 * C * DK, "room for both");
  f32x4 dq[KT], dk[KT];
  const Buf parked = buffer(a.before + ((int64_t)slot * a.H + hk * group) * DV * DK, PARK ? 2 * KT * THREADS * 16 : 0);
#pragma unroll
  for (int i = 0; i < KT; ++i) dq[i] = zero4(), dk[i] = zero4();

  for (int h = h0; h < h1; ++h) {
    const int tid = anew(tid0), lane = tid % kWave, g = lane / 16, c = lane % 16, i4 = 4 * (tid % 16);
    const int head = hk * group + h;
    const int64_t at = (int64_t)slot * a.H + head;
    const Buf bo = buffer(seq_row(a.o, sp, packed, head, t0, esz), (int)(((m - 1) * a.o.row + DV) * esz));
    const int orow = (c * (int)a.o.row + 8 * g) * esz;
    const auto load_do = [&](Frag<T>& f, int it, int s) {  // (rows from m on lie behind the buffer)
      buf_load8(f, bo, orow + 16 * it * (int)a.o.row * esz + 32 * s * esz);
    };
    // this wave's features of the states, 32 columns of d at a time, and rows of dO
    const Buf before = buffer(a.before + at * DV * DK, DV * DK * 4), after = buffer(a.after + at * DV * DK, DV * DK * 4);
    const int state = (feat + c + 8 * g * DK) * 4;
    float sx[8], sy[8];
    Frag<T> of[2];
    const auto load_states = [&](int s) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sx[e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(before, state, (32 * s + e) * DK * 4, 0));
        sy[e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(after, state, (32 * s + e) * DK * 4, 0));
      }
    };
    if (PARK && h > h0) load_head(head);
    __syncthreads();  // the head before is no longer read
#pragma unroll
    for (int n = 0; n < NG; ++n)
      if (tid + THREADS * n < kDeltaGates) (&l.gates[0][0])[tid + THREADS * n] = gv[n];
    const float log_decay = lv;
    __syncthreads();
    {
      const f32x4 beta = *reinterpret_cast<const f32x4*>(&l.gates[kDeltaBeta][i4]);
      f32x4 sum = zero4();
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        const int col = tid / 16 + n * (THREADS / 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = fmaf(ev[n][j], xv[n][j], sum[j]);
        store_parts4<NP>(&l.u[0][0][0] + Lds::at(col, i4), DV * PT, beta[0] * ev[n][0], beta[1] * ev[n][1], beta[2] * ev[n][2], beta[3] * ev[n][3]);
        store_parts4<NP>(&l.r[0][0][0] + Lds::at(col, i4), DV * PT, beta[0] * xv[n][0], beta[1] * xv[n][1], beta[2] * xv[n][2], beta[3] * xv[n][3]);
      }
      *reinterpret_cast<f32x4*>(&l.beta[tid / 16][i4]) = sum;
    }
    load_states(0);
    load_do(of[0], 0, 0);
    __syncthreads();
    float dbeta = 0.0f;
    if (wave == 0)
#pragma unroll
      for (int w = 0; w < 4 * W; ++w) dbeta += l.beta[w][kWave - 1 - lane];
    __syncthreads();  // the shares are no longer read
    {  // dV
      const Buf b = buffer(seq_row(a.dv, sp, packed, head, t0, esz), (int)(((m - 1) * a.dv.row + DV) * esz));
#pragma unroll
      for (int n = 0; n < C * DV / 4 / THREADS; ++n) {
        const int idx = tid + n * THREADS, i = idx % C, col = idx / C * 4;
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] = 0.0f;
#pragma unroll
          for (int p = delta_parts<T>(NP) - 1; p >= 0; --p) x[j] += (float)(&l.r[p][0][0])[Lds::at(col + j, i)];
        }
        buf_store4<T>(b, i < m ? (i * (int)a.dv.row + col) * esz : kPastEnd, x[0], x[1], x[2], x[3]);
      }
    }
    // this wave's features of dO S^T, dR S^T and U dS'^T, transposed
    f32x4 zq[KT], zr[KT], zk[KT];
    float both = 0.0f;
#pragma unroll
    for (int i = 0; i < KT; ++i) zq[i] = zero4(), zr[i] = zero4(), zk[i] = zero4();
    {
      const int lane = anew(tid0) % kWave, g = lane / 16, c = lane % 16;
      DeltaOp<T, NP> rf[2], uf[2];
      const GradTile<Lds, T, NP, DV> r0(&l.r[0][0][0], 0, lane), r1(&l.r[0][0][0], 1, lane), r2(&l.r[0][0][0], 2, lane), r3(&l.r[0][0][0], 3, lane);
      const GradTile<Lds, T, NP, DV> u0(&l.u[0][0][0], 0, lane), u1(&l.u[0][0][0], 1, lane), u2(&l.u[0][0][0], 2, lane), u3(&l.u[0][0][0], 3, lane);
      const auto read = [&](int n) {  // of tile n % KT and columns 32 (n / KT) ..
        (n % KT == 0 ? r0 : n % KT == 1 ? r1 : n % KT == 2 ? r2 : r3).read(rf[n % 2], n / KT);
        (n % KT == 0 ? u0 : n % KT == 1 ? u1 : n % KT == 2 ? u2 : u3).read(uf[n % 2], n / KT);
      };
      read(0);
#pragma unroll
      for (int s = 0; s < VS; ++s) {
        DeltaOp<T, NP> sf, df;
        sf.set(sx);
        df.set(sy);
#pragma unroll
        for (int e = 0; e < 8; ++e) both = fmaf(sx[e], sy[e], both);
        if (s + 1 < VS) load_states(s + 1);
#pragma unroll
        for (int it = 0; it < KT; ++it) {
          const int n = s * KT + it;
          if (n + 1 < VS * KT) {
            read(n + 1);
            load_do(of[(n + 1) % 2], (n + 1) % KT, (n + 1) / KT);
          }
          __builtin_amdgcn_sched_barrier(0);
          mma(zq[it], sf, of[n % 2]);
          mma(zr[it], sf, rf[n % 2]);
          mma(zk[it], df, uf[n % 2]);
        }
      }
    }
    // blocks of dP and dM: rows j of block jt (4 g + e), column i of block it
    constexpr int ROUNDS = (10 + W - 1) / W;
    f32x4 ap[ROUNDS], am[ROUNDS];
    int its[ROUNDS], jts[ROUNDS];
#pragma unroll
    for (int n = 0; n < ROUNDS; ++n) {
      const int lane = anew(tid0) % kWave, g = lane / 16, c = lane % 16;
      const int tile = wave + W * n;  // (0,0) (1,0) (1,1) (2,0) ..; behind the last one: again, unused
      const int it = tile >= 6 ? 3 : tile >= 3 ? 2 : tile >= 1 ? 1 : 0, jt = min(tile - it * (it + 1) / 2, it);
      its[n] = it;
      jts[n] = jt;
      f32x4 p = zero4(), r = zero4(), kk = zero4(), qk = zero4();
      Frag<T> oi[VS];
      DeltaOp<T, NP> rf[2], uf[2];
      const GradTile<Lds, T, NP, DV> ri(&l.r[0][0][0], it, lane), uj(&l.u[0][0][0], jt, lane);
      const auto read = [&](int s) {
        ri.read(rf[s % 2], s);
        uj.read(uf[s % 2], s);
      };
#pragma unroll
      for (int s = 0; s < VS; ++s) load_do(oi[s], it, s);
      read(0);
#pragma unroll
      for (int s = 0; s < VS; ++s) {
        if (s + 1 < VS) read(s + 1);
        __builtin_amdgcn_sched_barrier(0);
        mma(r, uf[s % 2], rf[s % 2]);
        mma(p, uf[s % 2], oi[s]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < FS; ++t) {
        Frag<T> kj, ki, qi;
        load8(kj, &l.k[16 * jt + c][32 * t + 8 * g]);
        load8(ki, &l.k[16 * it + c][32 * t + 8 * g]);
        load8(qi, &l.q[16 * it + c][32 * t + 8 * g]);
        mma(kk, kj, ki);
        mma(qk, kj, qi);
      }
      const int i = 16 * it + c, j0 = 16 * jt + 4 * g;
      const float high = l.gates[kDeltaHigh][i], low = l.gates[kDeltaLow][i];
      const f32x4 hj = *reinterpret_cast<const f32x4*>(&l.gates[kDeltaHigh][j0]);
      const f32x4 lj = *reinterpret_cast<const f32x4*>(&l.gates[kDeltaLow][j0]);
      f32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = j0 + e;
        const float f = exp2_raw((high - hj[e]) + (low - lj[e]));
        ap[n][e] = j <= i ? a.scale * p[e] * f : 0.0f;
        am[n][e] = j < i ? -r[e] * f : 0.0f;
        w[e] = fmaf(ap[n][e], qk[e], am[n][e] * kk[e]);
      }
      const float over = groups_sum(w[0] + w[1] + w[2] + w[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = row_sum(w[e]);
      if (tile < 10) {
        if (g == 0) l.row[jt][i] = over;
        if (c == 0) *reinterpret_cast<f32x4*>(&l.col[it][j0]) = w;
      }
    }
    __syncthreads();  // U and dR are no longer read
#pragma unroll
    for (int n = 0; n < ROUNDS; ++n) {
      if (wave + W * n < 10) {
        const int i = 16 * its[n] + c, j = 16 * jts[n] + 4 * g;
        store_parts4<NP>(&l.ap[0][i][j], C * PA, ap[n][0], ap[n][1], ap[n][2], ap[n][3]);
        store_parts4<NP>(&l.am[0][i][j], C * PA, am[n][0], am[n][1], am[n][2], am[n][3]);
      }
    }
    if (wave < 2) {  // the blocks beside the diagonal that products of 32 columns meet
      const int i = 32 * wave + c, j = 32 * wave + 16 + 4 * g;
      const float z = __int_as_float(anew(0));
      store_parts4<NP>(&l.ap[0][i][j], C * PA, z, z, z, z);
      store_parts4<NP>(&l.am[0][i][j], C * PA, z, z, z, z);
    }
    __syncthreads();
    {
      const int lane = anew(tid0) % kWave, g = lane / 16, c = lane % 16;
      if constexpr (PARK) {
#pragma unroll
        for (int i = 0; i < KT; ++i) dq[i] = zero4(), dk[i] = zero4();
        if (h > h0) {
          const int off = anew(tid0) * 16;
#pragma unroll
          for (int i = 0; i < KT; ++i) {
            dq[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(parked, off, i * THREADS * 16, 0));
            dk[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(parked, off, (KT + i) * THREADS * 16, 0));
          }
        }
      }
#pragma unroll
      for (int it = 0; it < KT; ++it) {
        const int i = 16 * it + c;
        const float first = l.gates[kDeltaFirst][i], last = l.gates[kDeltaLast][i];
        Frag<T> qf, kf;
        load4(qf, 0, &l.q[i][feat + 4 * g]);
        load4(kf, 0, &l.k[i][feat + 4 * g]);
        float sum = 0.0f, ends = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = a.scale * first * zq[it][e], y = first * zr[it][e], z = last * zk[it][e];
          dq[it][e] += x;
          dk[it][e] += z - y;
          sum = fmaf(qf.get(e), x, sum);
          sum = fmaf(-kf.get(e), y, sum);
          ends = fmaf(kf.get(e), z, ends);
        }
        sum = groups_sum(sum);
        ends = groups_sum(ends);
        if (mine && g == 0) {
          l.dots[wave][0][i] = sum - ends;
          l.dots[wave][1][i] = ends;
        }
      }
      both = groups_sum(row_sum(both));
      if (mine && lane == 0) l.state[wave] = both;
    }
    if (!PARK && h + 1 < h1) load_head(head + 1);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int lane = anew(tid0) % kWave, g = lane / 16, c = lane % 16;
      Frag<T> kf, qf;  // features (rows) over the tokens 32 s + 8 g ..
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        load_tr4(kf, 4 * half, &l.k[0][0], PK, 32 * s + 8 * g + 4 * half, feat, lane);
        load_tr4(qf, 4 * half, &l.q[0][0], PK, 32 * s + 8 * g + 4 * half, feat, lane);
      }
#pragma unroll
      for (int it = 0; it < KT; ++it) {
        if (it / 2 >= s) {  // over j
          DeltaOp<T, NP> pf, mf;
          load_op(pf, &l.ap[0][16 * it + c][32 * s + 8 * g], C * PA);
          load_op(mf, &l.am[0][16 * it + c][32 * s + 8 * g], C * PA);
          mma(dq[it], kf, pf);
          mma(dk[it], kf, mf);
        }
        if (it / 2 <= s) {  // over i
          DeltaOp<T, NP> pf, mf;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int row = 32 * s + 8 * g + 4 * half;
            load_op_tr4(pf, 4 * half, lane, C * PA, [&](int kk, int col) { return &l.ap[0][row + kk][16 * it + col]; });
            load_op_tr4(mf, 4 * half, lane, C * PA, [&](int kk, int col) { return &l.am[0][row + kk][16 * it + col]; });
          }
          mma(dk[it], qf, pf);
          mma(dk[it], kf, mf);
        }
      }
    }
    if (PARK && h + 1 < h1) {
      const int off = anew(tid0) * 16;
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, dq[i]), parked, off, i * THREADS * 16, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, dk[i]), parked, off, (KT + i) * THREADS * 16, 0);
      }
    }
    if (mine && shares > 1) {  // (one head: its sums, in the place of its states, which have been read by then)
      const int lane = anew(tid0) % kWave, g = lane / 16, c = lane % 16;
#pragma unroll
      for (int it = 0; it < KT; ++it) {
        const int off = ((16 * it + c) * DK + feat + 4 * g) * 4;
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, dq[it]), before, off, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, dk[it]), after, off, 0, 0);
      }
    } else if (mine && h + 1 == h1) {
      const int lane = anew(tid0) % kWave, g = lane / 16, c = lane % 16;
      const Buf bq = buffer(seq_row(a.dq, sp, packed, hk, t0, esz), (int)(((m - 1) * a.dq.row + DK) * esz));
      const Buf bk = buffer(seq_row(a.dk, sp, packed, hk, t0, esz), (int)(((m - 1) * a.dk.row + DK) * esz));
#pragma unroll
      for (int it = 0; it < KT; ++it) {
        const int i = 16 * it + c;
        buf_store4<T>(bq, i < m ? (i * (int)a.dq.row + feat + 4 * g) * esz : kPastEnd, dq[it][0], dq[it][1], dq[it][2], dq[it][3]);
        buf_store4<T>(bk, i < m ? (i * (int)a.dk.row + feat + 4 * g) * esz : kPastEnd, dk[it][0], dk[it][1], dk[it][2], dk[it][3]);
      }
    }
    __syncthreads();  // the sums are whole
    if (wave == 0) {  // (the last token in lane 0: sums over the later tokens are those up to a lane)
      const int token = kWave - 1 - anew(tid0) % kWave;
      float sum = 0.0f, ends = 0.0f, whole = 0.0f;
#pragma unroll
      for (int w = 0; w < DK / 16; ++w) {
        sum += l.dots[w][0][token];
        ends += l.dots[w][1][token];
        whole += l.state[w];
      }
#pragma unroll
      for (int b = 0; b < KT; ++b) {
        const float row = l.row[b][token], col = l.col[b][token];  // (not all of them formed)
        sum += b <= token / 16 ? row : 0.0f;
        sum -= b >= token / 16 ? col : 0.0f;
      }
      sum = lane_sums(sum);
      ends = of_lane(lane_sums(ends), kWave - 1);
      if (token < m) {
        const int64_t num = seq_num(a.s, sp, a.H, head, t0 + token);
        // (above 0 a log decay counts as 0)
        a.dlog_decay[num] = log_decay > 0.0f ? 0.0f : sum + ends + l.gates[kDeltaMisc][0] * whole;
        a.dbeta[num] = dbeta;
      }
    }
  }
}

// dQ and dK of chunks whose value heads had a workgroup each, added up in the heads' order.
template <typename T, int DK>
__global__ __launch_bounds__(256) void delta_grads_join_kernel(DeltaArgs a) {
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk, group = a.H / a.Hk;
  const SeqPiece sp = seq_piece(a.s, slot, C);
  if (sp.seq < 0) return;
  const bool packed = a.s.offsets != nullptr;
  const int t0 = sp.index * C, m = min(C, sp.len - t0);
  const float* from = blockIdx.y ? a.after : a.before;
  const SeqRows& rows = blockIdx.y ? a.dk : a.dq;
  const int64_t head0 = (int64_t)slot * a.H + hk * group;
  for (int at = 4 * threadIdx.x; at < m * DK; at += 4 * 256) {
    f32x4 sum = zero4();
#pragma unroll 4
    for (int h = 0; h < group; ++h) sum += *reinterpret_cast<const f32x4*>(from + (head0 + h) * a.d * DK + at);
    store4(reinterpret_cast<T*>(seq_row(rows, sp, packed, hk, t0 + at / DK, (int)sizeof(T))) + at % DK, sum[0], sum[1], sum[2], sum[3]);
  }
}

template <typename T, int DK, int DV, int NP>
hipError_t launch_one(const DeltaArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(GradLds<T, DK, DV, NP>);
  static_assert(bytes <= 160 * 1024, "one workgroup's LDS");
  const hipError_t e = allow_lds<delta_grads_kernel<T, DK, DV, NP>>(bytes);
  if (e != hipSuccess) return e;
  const int64_t groups = (int64_t)a.slots * a.Hk;
  const int group = a.H / a.Hk, shares = DV >= C && delta_grads_apart(groups, group) ? group : 1;
  hipLaunchKernelGGL((delta_grads_kernel<T, DK, DV, NP>), dim3((unsigned)(groups * shares)), dim3(64 * kGradWaves<DK>), bytes, s, a, shares);
  if (shares > 1) hipLaunchKernelGGL((delta_grads_join_kernel<T, DK>), dim3((unsigned)groups, 2), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T, int DK, int NP>
hipError_t launch_columns(const DeltaArgs& a, hipStream_t s) {
  return a.d == 32 ? launch_one<T, DK, 32, NP>(a, s) : a.d == 64 ? launch_one<T, DK, 64, NP>(a, s) : launch_one<T, DK, 128, NP>(a, s);
}
template <typename T, int NP>
hipError_t launch_grads(const DeltaArgs& a, hipStream_t s) {
  return a.D == 32 ? launch_columns<T, 32, NP>(a, s) : a.D == 64 ? launch_columns<T, 64, NP>(a, s) : launch_columns<T, 128, NP>(a, s);
}

}  // namespace

hipError_t launch_delta_grads(Dt dt, const DeltaArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_grads<__bf16, kDeltaBackParts>(a, s) : launch_grads<float, 1>(a, s);
}

}  // namespace luna
