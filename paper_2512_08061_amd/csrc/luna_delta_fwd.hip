// luna_delta_fwd.hip -- the gated delta rule over whole sequences in bf16, forward, in one launch (luna_delta.hpp).
//
// A workgroup takes DVW value columns of one sequence and head.  Four gate waves form the matrices of the next chunk (N in
// parts, P, the factors of the gates) in LDS while the scan waves, 16 columns each, carry the state through the present one, so
// that the matrices never go to memory and the state's chain waits for nothing but itself.  Tiles and matrices lie in LDS
// twice.  Three barriers a chunk:
//
//   gate waves                                             scan waves
//   K, Q of the next chunk, 16 rows each, to LDS           K S, half of it
//   K K^T, Q K^T, M, P, N's diagonal blocks; loads         K S, Q S, R, E = R + N (beta R)
//   N below its diagonal blocks; the next gates            S = e^(G_C) S + K^T (..), out
//
// The scan waves' products are chained in registers as luna_delta_scan.hpp says.  Operands are read from LDS a batch before
// their products (by itself the compiler reads each right before its use and waits out the LDS 80 times a chunk).  16-byte pieces
// of a row are swapped among each other by the row's number, so that the rows of pairs of tiles do not meet in a bank.  What bounds it
// is the chain of a chunk: 8 x 16 heads of 16384 tokens, D = d = 128, 1012 to 1031 us, 4 us a chunk (LDS active 50% of all cycles, half of
// them bank conflicts of the transposing reads, which touch every other 8 bytes; matrix cores 28%).  Tiles of 16 consecutive rows and
// features have no such conflicts, but need two 8-byte reads for each 16-byte one of an operand's row: 1078 us (of 1012).
#include "luna_delta_scan.hpp"

namespace luna {

namespace {

constexpr int C = kDeltaChunk, KT = C / 16, KS = C / 32;
constexpr int kNever = 1 << 30;

// Rows of W bf16 in LDS: 16-byte pieces swapped by a number of the row that pair_row(i, c) and the rows of a transposing read
// of lane (g, c) have for all i alike.
template <int W>
struct Rows {
  static constexpr int PIECES = W / 8;
  static __device__ __forceinline__ int swap(int row) {
    return PIECES == 16 ? 4 * (row % 4) + row / 8 % 4 : PIECES == 8 ? 4 * (row / 2 % 2) + row / 8 % 4 : row / 8 % 4;
  }
  static __device__ __forceinline__ int at(int row, int col) { return row * W + ((col / 8 ^ swap(row)) * 8) + col % 8; }
  // bytes
  static __device__ __forceinline__ int byte(int row, int col) { return 2 * at(row, col); }
  static constexpr int pair(int i) { return (32 * (i / 2) + 4 * (i % 2)) * W * 2; }  // from pair_row(0, c) to pair_row(i, c)
};

template <int DK, int NP>
struct FwdLds {
  __bf16 k[2][C * DK], q[2][C * DK];
  __bf16 n[2][NP][C * C], p[2][C * C];  // N transposed
  // M below its diagonal blocks, in parts: of a row the first two parts of four columns, and the third of them
  __bf16 m[C][2 * C + 8], m3[NP == 3 ? C : 2][C + 4];
  alignas(16) float gates[3][4][C];  // (formed while the two chunks before are at work)
  float high[C], low[C];
  float from[KT][C];  // e^(G_i0 - G_j) for the rows i0 = 16 w
  float to[C];        // e^(G_i - G_i0) for i's block's first row i0
  int since[64];      // per column: the first token with a value that is not finite
  int key[2], gate;   // the first row with a key, or gate, that is not finite
};

// Four numbers in parts.
template <int NP>
struct Parts4 {
  bf16x4 p[NP];
};
template <int NP>
__device__ __forceinline__ Parts4<NP> parts_of(f32x4 x) {
  Parts4<NP> r;
#pragma unroll
  for (int k = 0; k < NP; ++k) {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.p[k][e] = (__bf16)x[e];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] -= (float)r.p[k][e];
  }
  return r;
}
// c += A B of fp32 blocks of 16, both in parts: row c of A (four numbers from 4 g on), and B as a sum's registers are.  A bf16
// product has room for two of the products of parts.  (As fp32 products, 128 cycles each instead of 32 or 48, the blocks of N
// below its diagonal ones took 4100 cycles a chunk beside the scan's products.)
template <int NP>
__device__ __forceinline__ void mma16(f32x4& c, const Parts4<NP>& a, const Parts4<NP>& b) {
  const auto two = [](const bf16x4& x, const bf16x4& y) {
    Frag<__bf16> f;
    f.v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    return f;
  };
  if constexpr (NP == 3) mma(c, two(a.p[0], a.p[2]), two(b.p[2], b.p[0]));
  mma(c, two(a.p[0], a.p[1]), two(b.p[1], b.p[1]));
  mma(c, two(a.p[0], a.p[1]), two(b.p[0], b.p[0]));
}
// four rows of a column
__device__ __forceinline__ bf16x4 lds_tr4(unsigned at) {
  typedef __attribute__((ext_vector_type(4))) short i16x4;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)at));
}
__device__ __forceinline__ bf16x4 lds_b4(unsigned at) { return *(__attribute__((address_space(3))) const bf16x4*)(uintptr_t)at; }

// What every gate wave has.
template <int DK, int NP>
struct GateWave {
  using Lds = FwdLds<DK, NP>;
  static constexpr int FS = DK / 32;
  const DeltaArgs& a;
  Lds& l;
  const int g0, c0;
  unsigned rows[2][FS];  // row c of tiles 0 and 1 of K

  // Of K K^T and Q K^T, M and P: the diagonal block W (kf, qf: its rows of K and Q) and one or two of those below the
  // diagonal, (3, 0) | (1, 0) | (2, 0), (2, 1) | (3, 1), (3, 2), so that no wave has more than three.  Returns N's diagonal block
  // (rows 4 g + e of column c).
  template <int W>
  __device__ __forceinline__ f32x4 blocks_of(int buf, const float (&gates)[4][C], const Frag<__bf16> (&kf)[FS],
                                             const Frag<__bf16> (&qf)[FS]) const {
    constexpr int OFF = W < 2 ? 1 : 2, I = W == 0 ? KT - 1 : W, J0 = W == 3 ? 1 : 0;  // blocks (I, J0 ..)
    const int g = anew(g0), c = anew(c0);
    const unsigned kb = lds_address(l.k[buf]), qb = lds_address(l.q[buf]);
    const auto row = [&](Frag<__bf16>& f, unsigned base, int tile, int t) { lds8(f, base + rows[tile % 2][t] + tile / 2 * 32 * DK * 2); };
    const int i = 16 * I + c;
    Frag<__bf16> ki[FS], qi[FS], kj[OFF][FS];
#pragma unroll
    for (int t = 0; t < FS; ++t) {
      if (W == 0) {
        row(ki[t], kb, I, t);
        row(qi[t], qb, I, t);
        kj[0][t] = kf[t];
      } else {
        ki[t] = kf[t];
        qi[t] = qf[t];
        row(kj[0][t], kb, J0, t);
      }
    }
    const int key = l.key[buf], gate = l.gate;
    const f32x4 hj = lds4(lds_address(&l.high[16 * W + 4 * g])), lj = lds4(lds_address(&l.low[16 * W + 4 * g]));
    const float high = l.high[16 * W + c], low = l.low[16 * W + c];
    const f32x4 beta = lds4(lds_address(&gates[kDeltaBeta][16 * W + 4 * g]));
    const float to_row = l.to[i];
    f32x4 from[OFF], kk[OFF], qk[OFF], kd = zero4(), qd = zero4();
#pragma unroll
    for (int n = 0; n < OFF; ++n) from[n] = lds4(lds_address(&l.from[I][16 * (J0 + n) + 4 * g]));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < FS; ++t) {
      mma(kd, kf[t], kf[t]);
      mma(qd, kf[t], qf[t]);
    }
#pragma unroll
    for (int n = 0; n < OFF; ++n) {
      kk[n] = zero4();
      qk[n] = zero4();
      if (n + 1 < OFF)
#pragma unroll
        for (int t = 0; t < FS; ++t) row(kj[n + 1][t], kb, J0 + n + 1, t);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < FS; ++t) {
        mma(kk[n], kj[n][t], ki[t]);
        mma(qk[n], kj[n][t], qi[t]);
      }
    }
    const int bad = __builtin_amdgcn_readfirstlane(min(key, gate));
    // e^(G_i - G_j): in the diagonal block directly, below it as a product over the first row of i's block.  M's diagonal block comes
    // as M^T and, K K^T being symmetric, as M.
    f32x4 md, pd, mm[OFF], pp[OFF], z;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float d = (high - hj[e]) + (low - lj[e]), f = exp2_raw(fminf(d, 0.0f)), f2 = exp2_raw(fminf(-d, 0.0f));
      md[e] = 4 * g + e < c ? kd[e] * f : 0.0f;
      pd[e] = 4 * g + e <= c ? a.scale * f * qd[e] : 0.0f;
      z[e] = 4 * g + e > c ? kd[e] * f2 : 0.0f;
    }
#pragma unroll
    for (int n = 0; n < OFF; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float f = to_row * from[n][e];
        mm[n][e] = kk[n][e] * f;
        pp[n][e] = qk[n][e] * (a.scale * f);
      }
    if (bad < C) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        md[e] = 16 * W + c < bad ? md[e] : 0.0f;
        pd[e] = 16 * W + 4 * g + e < bad ? pd[e] : 0.0f;
        z[e] = 16 * W + 4 * g + e < bad ? z[e] : 0.0f;
#pragma unroll
        for (int n = 0; n < OFF; ++n) {
          mm[n][e] = i < bad ? mm[n][e] : 0.0f;
          pp[n][e] = 16 * (J0 + n) + 4 * g + e < bad ? pp[n][e] : 0.0f;
        }
      }
    }
    // M's blocks of 4 on the diagonal: of this lane group's, row e
    f32x4 m4[4];
#pragma unroll
    for (int e = 1; e < 4; ++e)
#pragma unroll
      for (int k = 0; k < e; ++k) m4[e][k] = __shfl(z[e], 20 * g + k);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < OFF; ++n) {
      const Parts4<NP> x = parts_of<NP>(mm[n]);
      Frag<__bf16> f;
      f.v = __builtin_shufflevector(x.p[0], x.p[1], 0, 1, 2, 3, 4, 5, 6, 7);
      *reinterpret_cast<bf16x8*>(&l.m[i][32 * (J0 + n) + 8 * g]) = f.v;
      if constexpr (NP == 3) *reinterpret_cast<bf16x4*>(&l.m3[i][16 * (J0 + n) + 4 * g]) = x.p[2];
      store4(&l.p[buf][Rows<C>::at(i, 16 * (J0 + n) + 4 * g)], pp[n][0], pp[n][1], pp[n][2], pp[n][3]);
    }
    store4(&l.p[buf][Rows<C>::at(16 * W + c, 16 * W + 4 * g)], pd[0], pd[1], pd[2], pd[3]);
    // The diagonal block by substitution, four rows at a time: lane group p's rows are solved among themselves, and
    // all rows take what these contribute as a product (its own among them).
    const Parts4<NP> mp = parts_of<NP>(md);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      f32x4 t = z, bn;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int k = 0; k < e; ++k) t[e] = fmaf(m4[e][k], bn[k], t[e]);
        bn[e] = -beta[e] * t[e];
      }
      if (p == 3) {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = g == p ? t[e] : z[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) bn[e] = g == p ? bn[e] : 0.0f;
        mma16(z, mp, parts_of<NP>(bn));
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = -z[e];
    store_parts4<NP>(&l.n[buf][0][Rows<C>::at(16 * W + c, 16 * W + 4 * g)], C * C, z[0], z[1], z[2], z[3]);
    return z;
  }

  // The blocks of N below the diagonal one (x) of block column W: what each takes from the finished ones above it.
  template <int W>
  __device__ __forceinline__ void column_of(int buf, const float (&gates)[4][C], const f32x4& x) const {
    const int g = anew(g0), c = anew(c0), tr = 4 * g + c / 4, q = c % 4;
    const auto block = [&](Parts4<NP>& y, int i, int p) {  // row c of a block of M
      Frag<__bf16> f;
      lds8(f, lds_address(&l.m[c][8 * g]) + 16 * i * (2 * C + 8) * 2 + 16 * p * 4);
      y.p[0] = __builtin_shufflevector(f.v, f.v, 0, 1, 2, 3);
      y.p[1] = __builtin_shufflevector(f.v, f.v, 4, 5, 6, 7);
      if constexpr (NP == 3) y.p[2] = lds_b4(lds_address(&l.m3[c][4 * g]) + 16 * i * (C + 4) * 2 + 16 * p * 2);
    };
    Parts4<NP> an[KT], am[KT][KT], zp[KT];
    f32x4 z[KT], beta[KT], bn;
    z[W] = x;
    beta[W] = lds4(lds_address(&gates[kDeltaBeta][16 * W + 4 * g]));
#pragma unroll
    for (int i = W + 1; i < KT; ++i) block(am[i][W], i, W);
#pragma unroll
    for (int i = W + 1; i < KT; ++i) {  // four rows of column c
      const unsigned at = lds_address(&l.m[tr][8 * q]) + 16 * i * (2 * C + 8) * 2 + 16 * W * 4;
      zp[i].p[0] = lds_tr4(at);
      zp[i].p[1] = lds_tr4(at + 8);
      if constexpr (NP == 3) zp[i].p[2] = lds_tr4(lds_address(&l.m3[tr][4 * q]) + 16 * i * (C + 4) * 2 + 16 * W * 2);
    }
#pragma unroll
    for (int i = W + 1; i < KT; ++i) {
      beta[i] = lds4(lds_address(&gates[kDeltaBeta][16 * i + 4 * g]));
#pragma unroll
      for (int k = 0; k < NP; ++k) an[i].p[k] = lds_tr4(lds_address(&l.n[buf][k][Rows<C>::at(16 * i + tr, 16 * i + 4 * q)]));
#pragma unroll
      for (int p = W + 1; p < i; ++p) block(am[i][p], i, p);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = W + 1; i < KT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[i][e] = (float)zp[i].p[0][e] + (float)zp[i].p[1][e];
        if constexpr (NP == 3) z[i][e] = (float)zp[i].p[0][e] + ((float)zp[i].p[1][e] + (float)zp[i].p[2][e]);
      }
#pragma unroll
    for (int p = W; p < KT; ++p) {
      if (p == W) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bn[e] = beta[p][e] * z[p][e];
      } else {  // N of block p
        f32x4 bz, y = z[p];
#pragma unroll
        for (int e = 0; e < 4; ++e) bz[e] = beta[p][e] * z[p][e];
        mma16(y, an[p], parts_of<NP>(bz));
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = -y[e], bn[e] = beta[p][e] * y[e];
        store_parts4<NP>(&l.n[buf][0][Rows<C>::at(16 * W + c, 16 * p + 4 * g)], C * C, y[0], y[1], y[2], y[3]);
      }
      if (p + 1 < KT) {
        const Parts4<NP> b = parts_of<NP>(bn);
#pragma unroll
        for (int i = p + 1; i < KT; ++i) mma16(z[i], am[i][p], b);
      }
    }
  }
};

template <int DK, int DVW, int NP>
__global__ __launch_bounds__(4 * DVW + 256, 2) void delta_fwd_kernel(DeltaArgs a) {
  using Lds = FwdLds<DK, NP>;
  constexpr int FT = DK / 16, FS = DK / 32, SCAN = DVW / 16;  // feature tiles, and scan waves
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id(), g = lane / 16, c = lane % 16;
  const int slices = a.d / DVW, heads = (int)(a.s.count * a.H);
  // (slices of a head eight workgroups apart where that is possible: on one die, whose cache then holds its rows once)
  int slice, item;
  if (heads % 8 == 0) {
    slice = blockIdx.x / 8 % slices;
    item = blockIdx.x / (8 * slices) * 8 + blockIdx.x % 8;
  } else {
    slice = blockIdx.x % slices;
    item = blockIdx.x / slices;
  }
  const int head = item % a.H, b = seq_by_length(a.s, item / a.H);
  const SeqPiece sp = seq_uniform(seq_of(a.s, b));
  if (sp.len == 0) return;
  const bool packed = a.s.offsets != nullptr;
  const int hk = head / (a.H / a.Hk), col0 = slice * DVW, chunks = (sp.len + C - 1) / C;

  for (int i = threadIdx.x; i < DVW; i += 4 * DVW + 256) l.since[i] = kNever;
  if (threadIdx.x < 2) l.key[threadIdx.x] = C;
  // the blocks beside the diagonal ones that products of 32 columns meet stay zeros
  for (int i = threadIdx.x; i < 2 * 2 * 16 * 16; i += 4 * DVW + 256) {
    const int r = i % 16, col = i / 16 % 16, block = i / 256 % 2, buf = i / 512;
    for (int p = 0; p < NP; ++p) l.n[buf][p][Rows<C>::at(32 * block + 16 + col, 32 * block + r)] = (__bf16)0.0f;
    l.p[buf][Rows<C>::at(32 * block + r, 32 * block + 16 + col)] = (__bf16)0.0f;
  }
  __syncthreads();

  if (wave >= SCAN) {
    // ------------------------------------------------------------------ gate waves
    const int w = wave - SCAN, tid = threadIdx.x - 64 * SCAN;
    // (before the scan waves, where these have the shorter chain: 1.04 -> 1.01 ms with two parts, but 537 -> 570 us with three)
    if constexpr (NP == 2) __builtin_amdgcn_s_setprio(3);
    GateWave<DK, NP> gate{a, l, g, c, {}};
#pragma unroll
    for (int t = 0; t < FS; ++t) {
      gate.rows[0][t] = Rows<DK>::byte(c, 32 * t + 8 * g);
      gate.rows[1][t] = Rows<DK>::byte(16 + c, 32 * t + 8 * g);
    }
    unsigned to_row[FS];
#pragma unroll
    for (int t = 0; t < FS; ++t) to_row[t] = Rows<DK>::byte(16 * w + c, 32 * t + 8 * g);
    Frag<__bf16> kr[FS], qr[FS];  // this wave's 16 rows
    const int kat = ((16 * w + c) * (int)a.k.row + 8 * g) * 2, qat = ((16 * w + c) * (int)a.q.row + 8 * g) * 2;
    float gr = 0.0f, br = 0.0f;
    const auto load = [&](int chunk) {
      const int t0 = chunk * C, m = min(C, sp.len - t0);  // (rows from m on lie behind the buffers)
      const Buf bk = buffer(seq_row(a.k, sp, packed, hk, t0, 2), (int)(((m - 1) * a.k.row + DK) * 2));
      const Buf bq = buffer(seq_row(a.q, sp, packed, hk, t0, 2), (int)(((m - 1) * a.q.row + DK) * 2));
#pragma unroll
      for (int t = 0; t < FS; ++t) {
        buf_load8(kr[t], bk, kat + 64 * t);
        buf_load8(qr[t], bq, qat + 64 * t);
      }
    };
    const auto load_gates = [&](int chunk) {  // (a chunk before the last wave forms them)
      const int64_t num = seq_num(a.s, sp, a.H, head, min(chunk * C + lane, sp.len - 1));
      gr = a.log_decay[num];
      br = a.beta[num];
    };
    const auto form_gates = [&](int chunk, int slot) {
      float(&gates)[4][C] = l.gates[slot];
      const bool in = chunk * C + lane < sp.len;
      float x = in ? gr : 0.0f, beta = in ? br : 0.0f;
      const uint64_t lost = __ballot(isnan(x) || !(fabsf(beta) < __builtin_inff()));
      const int bad = lost ? (int)__builtin_ctzll(lost) : C;
      if (lane >= bad) x = beta = 0.0f;
      // (e^-128 is 0 in fp32; in base 2)
      const double sum = lane_sums((double)fminf(fmaxf(x, -128.0f), 0.0f) * 1.4426950408889634), whole = of_lane(sum, kWave - 1);
      const float high = (float)sum;
      l.high[lane] = high;
      l.low[lane] = (float)(sum - (double)high);
      gates[kDeltaFirst][lane] = exp2_raw(high);
      gates[kDeltaLast][lane] = exp2_raw((float)(whole - sum));
      gates[kDeltaBeta][lane] = beta;
#pragma unroll
      for (int t = 1; t < KT; ++t) l.from[t][lane] = exp2_raw((float)fmin(of_lane(sum, 16 * t) - sum, 0.0));
      double row0 = of_lane(sum, 0);
#pragma unroll
      for (int t = 1; t < KT; ++t) row0 = lane >= 16 * t ? of_lane(sum, 16 * t) : row0;
      l.to[lane] = exp2_raw((float)(sum - row0));
      if (lane == 0) {
        gates[kDeltaMisc][0] = exp2_raw((float)whole);
        l.gate = bad;
      }
    };
    load(0);
    load_gates(0);
    if (w == KT - 1) form_gates(0, 0);
    load_gates(min(1, chunks - 1));
    int slot = 0;
    for (int chunk = 0; chunk <= chunks; ++chunk) {  // (beside the scan of chunk - 1)
      const int buf = chunk % 2, next = slot == 2 ? 0 : slot + 1;
      float(&gates)[4][C] = l.gates[slot];
      __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
      if (chunk < chunks) {
        bool odd = false;
#pragma unroll
        for (int t = 0; t < FS; ++t) {
          odd |= not_finite(kr[t]);
          lds8_store(lds_address(l.k[buf]) + to_row[t], kr[t]);
          lds8_store(lds_address(l.q[buf]) + to_row[t], qr[t]);
        }
        if (__any(odd) && odd) atomicMin(&l.key[buf], 16 * w + c);
      }
      __syncthreads();
      f32x4 diag = zero4();
      if (chunk < chunks) {
        if (tid == 0) {
          l.key[1 - buf] = C;
          reinterpret_cast<int&>(gates[kDeltaMisc][1]) = min(l.key[buf], l.gate);
        }
        diag = w == 0 ? gate.template blocks_of<0>(buf, gates, kr, qr) : w == 1 ? gate.template blocks_of<1>(buf, gates, kr, qr)
             : w == 2 ? gate.template blocks_of<2>(buf, gates, kr, qr) : gate.template blocks_of<3>(buf, gates, kr, qr);
        if (chunk + 1 < chunks) load(chunk + 1);
      }
      __syncthreads();
      if (chunk < chunks) {
        if (w == 0) {
          gate.template column_of<0>(buf, gates, diag);
        } else if (w == 1) {
          gate.template column_of<1>(buf, gates, diag);
        } else if (w == 2) {
          gate.template column_of<2>(buf, gates, diag);
        } else if (chunk + 1 < chunks) {
          form_gates(chunk + 1, next);
        }
        load_gates(min(chunk + 2, chunks - 1));
      }
      __syncthreads();
      slot = next;
    }
    return;
  }

  // -------------------------------------------------------------------- scan waves
  const int wcol = 16 * wave;
  f32x4 S[FT];
  const int64_t state = ((int64_t)b * a.H + head) * a.D * a.d + col0 + wcol + c;
#pragma unroll
  for (int ft = 0; ft < FT; ++ft)
#pragma unroll
    for (int j = 0; j < 4; ++j) S[ft][j] = a.S ? a.S[state + (int64_t)(pair_rows(ft, g) + j) * a.d] : 0.0f;
  unsigned short vr[C / 4];  // this lane's tokens of its column, as pairs of tiles have them
  const int vat = (8 * g * (int)a.v.row + wcol + c) * 2, vrow = (int)a.v.row * 2, orow = (int)a.o.row * 2;
  const int oat = (8 * (c / 4) + c % 4) * orow + (wcol + 4 * g) * 2;
  const auto load_v = [&](int chunk) {
    const int t0 = chunk * C, m = min(C, sp.len - t0);  // (rows from m on lie behind the buffer)
    const Buf bv = buffer(seq_row(a.v, sp, packed, head, t0, 2) + col0 * 2, (int)(((m - 1) * a.v.row + DVW) * 2));
    const int at = anew(vat);
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) vr[4 * i + e] = __builtin_amdgcn_raw_buffer_load_b16(bv, at + (pair_rows(i, 0) + e) * vrow, 0, 0);
  };
  // this lane's places in the tiles
  unsigned rk[FS], tk[FS], tn[KS], rp[KS];
  {
    const int row = 8 * (c / 4) + c % 4, tr = 8 * g + c / 4, q = c % 4;
#pragma unroll
    for (int t = 0; t < FS; ++t) {
      rk[t] = lds_address(l.k[0]) + Rows<DK>::byte(row, 32 * t + 8 * g);
      tk[t] = lds_address(l.k[0]) + Rows<DK>::byte(tr, 32 * t + 8 * q);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      tn[s] = lds_address(l.n[0]) + Rows<C>::byte(tr, 32 * s + 8 * q);
      rp[s] = lds_address(l.p[0]) + Rows<C>::byte(row, 32 * s + 8 * g);
    }
  }
  constexpr int QK = 2 * C * DK * 2;  // from K's tiles to Q's
  load_v(0);
  __syncthreads();
  __syncthreads();
  __syncthreads();
  int lost = kNever;    // the first token with a key or gate that is not finite
  bool poison = false;  // whether anything was not finite so far
  int slot = 0;
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const int t0 = chunk * C, m = min(C, sp.len - t0);
    const float(&gates)[4][C] = l.gates[slot];
    const unsigned ga = lds_address(&gates[0][0]) + 32 * g;  // the gates of rows 8 g ..
    const auto gate4 = [&](int which, int i) { return lds4(ga + which * C * 4 + (32 * (i / 2) + 4 * (i % 2)) * 4); };
    // K S
    DeltaOp<__bf16, NP> sf[FS];
    Frag<__bf16> kf[2][KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) lds8(kf[0][i], rk[0] + Rows<DK>::pair(i));
    f32x4 r[KT], o[KT], first[KT], beta[KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) r[i] = zero4(), o[i] = zero4();
#pragma unroll
    for (int t = 0; t < FS; ++t) {
#pragma unroll
      for (int i = 0; i < KT; ++i) lds8(kf[(t + 1) % 2][i], (t + 1 < FS ? rk[t + 1 < FS ? t + 1 : 0] : rk[0] + QK) + Rows<DK>::pair(i));
      set_tiles(sf[t], S[2 * t], S[2 * t + 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < KT; ++i) mma(r[i], kf[t % 2][i], sf[t]);
      if (t == (FS - 1) / 2) __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < KT; ++i) first[i] = gate4(kDeltaFirst, i), beta[i] = gate4(kDeltaBeta, i);
    const int bad = __builtin_amdgcn_readfirstlane(reinterpret_cast<const int&>(gates[kDeltaMisc][1]));
    // R and beta R
    DeltaOp<__bf16, NP> br[KS];
    {
      f32x4 v[KT];
      float most = 0.0f;
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = __uint_as_float((unsigned)vr[4 * i + e] << 16);
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = __builtin_elementwise_maximum(most, fabsf(v[i][e]));
      if (__any(!(most < __builtin_inff()))) {  // (values that are not finite enter as zeros)
        poison = true;
        int first_odd = kNever;
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(fabsf(v[i][e]) < __builtin_inff())) {
              first_odd = min(first_odd, t0 + pair_rows(i, g) + e);
              v[i][e] = 0.0f;
            }
        atomicMin(&l.since[wcol + c], first_odd);
        wave_lds_fence();
      }
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) r[i][e] = fmaf(-first[i][e], r[i][e], v[i][e]);
      if (bad < C) {  // (so do the rows from a key or gate on that is not)
        poison = true;
        lost = min(lost, t0 + bad);
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (pair_rows(i, g) + e >= bad) r[i][e] = 0.0f;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) set_tiles(br[s], beta[2 * s] * r[2 * s], beta[2 * s + 1] * r[2 * s + 1]);
    }
    if (chunk + 1 < chunks) load_v(chunk + 1);
    // Q S (two parts of S suffice for out), and meanwhile N
    DeltaOp<__bf16, NP> nf[2][KS];
    const auto read_n = [&](int i) {
#pragma unroll
      for (int s = 0; s <= i / 2; ++s)
#pragma unroll
        for (int p = 0; p < NP; ++p) lds_tr(nf[i % 2][s].p[p], tn[i / 2] + 32 * s * C * 2 + 8 * (i % 2) + p * C * C * 2, 4 * C * 2);
    };
#pragma unroll
    for (int t = 0; t < FS; ++t) {
      const int at = (t + FS) % 2;
      if (t + 1 < FS)
#pragma unroll
        for (int i = 0; i < KT; ++i) lds8(kf[1 - at][i], rk[t + 1 < FS ? t + 1 : 0] + QK + Rows<DK>::pair(i));
      else
        read_n(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        mma(o[i], sf[t].p[1], kf[at][i]);
        mma(o[i], sf[t].p[0], kf[at][i]);
      }
    }
    // E = R + N (beta R), of whose rows 32 s .. the columns up to 32 s + 31
    constexpr int TI = FT < 4 ? FT : 4, TN = FT * KS / TI;  // tiles of a batch of K^T, and batches
    Frag<__bf16> tf[2][TI];
    const auto read_t = [&](int n) {
#pragma unroll
      for (int i = 0; i < TI; ++i) {
        const int ft = (TI * n + i) % FT, s = (TI * n + i) / FT;
        lds_tr(tf[n % 2][i], tk[ft / 2] + 32 * s * DK * 2 + 8 * (ft % 2), 4 * DK * 2);
      }
    };
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      if (i + 1 < KT) read_n(i + 1);
      else read_t(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s <= i / 2; ++s) mma(r[i], nf[i % 2][s], br[s]);
    }
    f32x4 last[KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) last[i] = gate4(kDeltaLast, i);
    const float whole = gates[kDeltaMisc][0];
    float row_first[KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) row_first[i] = gates[kDeltaFirst][pair_row(i, c)];
    __syncthreads();
    // U, and U discounted to the chunk's end
    DeltaOp<__bf16, 2> uf[KS];
    DeltaOp<__bf16, NP> ul[KS];
#pragma unroll
    for (int i = 0; i < KT; ++i) r[i] *= beta[i];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      set_tiles(ul[s], last[2 * s] * r[2 * s], last[2 * s + 1] * r[2 * s + 1]);
      set_tiles(uf[s], r[2 * s], r[2 * s + 1]);
    }
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) S[ft] *= whole;
    Frag<__bf16> pf[KT][KS];
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      if (n + 1 < TN) read_t(n + 1);
      else
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
          for (int s = 0; s <= i / 2; ++s) lds8(pf[i][s], rp[s] + Rows<C>::pair(i));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TI; ++i) mma(S[(TI * n + i) % FT], tf[n % 2][i], ul[(TI * n + i) / FT]);
    }
    // out
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      o[i] *= a.scale * row_first[i];
#pragma unroll
      for (int s = 0; s <= i / 2; ++s) mma(o[i], uf[s], pf[i][s]);
    }
    if (poison) {
      const i32x4 since = *reinterpret_cast<const i32x4*>(&l.since[wcol + 4 * g]);
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t0 + pair_row(i, c) >= min(since[e], lost)) o[i][e] = __builtin_nanf("");
    }
    const Buf to = buffer(seq_row(a.o, sp, packed, head, t0, 2) + col0 * 2, (int)(((m - 1) * a.o.row + DVW) * 2));
    const int at = anew(oat);
#pragma unroll
    for (int i = 0; i < KT; ++i) buf_store4<__bf16>(to, at + pair_rows(i, 0) * orow, o[i][0], o[i][1], o[i][2], o[i][3]);
    __syncthreads();
    slot = slot == 2 ? 0 : slot + 1;
    const int way = chunk % 2 ? -1 : 1;  // to the other tiles
#pragma unroll
    for (int t = 0; t < FS; ++t) rk[t] += way * C * DK * 2, tk[t] += way * C * DK * 2;
#pragma unroll
    for (int s = 0; s < KS; ++s) tn[s] += way * NP * C * C * 2, rp[s] += way * C * C * 2;
  }
  if (a.S) {
    const bool gone = min(l.since[wcol + c], lost) != kNever;
#pragma unroll
    for (int ft = 0; ft < FT; ++ft)
#pragma unroll
      for (int j = 0; j < 4; ++j) a.S[state + (int64_t)(pair_rows(ft, g) + j) * a.d] = gone ? __builtin_nanf("") : S[ft][j];
  }
}

template <int DK, int DVW, int NP>
hipError_t launch_one(const DeltaArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(FwdLds<DK, NP>);
  static_assert(bytes <= 160 * 1024, "one workgroup's LDS");
  const hipError_t e = allow_lds<delta_fwd_kernel<DK, DVW, NP>>(bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((delta_fwd_kernel<DK, DVW, NP>), dim3((unsigned)(a.s.count * a.H * (a.d / DVW))), dim3(4 * DVW + 256), bytes, s, a);
  return hipGetLastError();
}
template <int DK, int NP>
hipError_t launch_columns(const DeltaArgs& a, hipStream_t s) {
  // 32 columns where workgroups of 64 would leave half of the device idle: a chunk passes in less time (2000 tokens, 16 heads, D = d = 128:
  // 118 and 127 us, with a state 141 and 162)
  return a.d == 32 || a.s.count * a.H * (a.d / 64) <= 128 ? launch_one<DK, 32, NP>(a, s) : launch_one<DK, 64, NP>(a, s);
}
template <int NP>
hipError_t launch_parts(const DeltaArgs& a, hipStream_t s) {
  return a.D == 32 ? launch_columns<32, NP>(a, s) : a.D == 64 ? launch_columns<64, NP>(a, s) : launch_columns<128, NP>(a, s);
}

}  // namespace

hipError_t launch_delta_fwd_bf16(bool exact, const DeltaArgs& a, hipStream_t s) {
  return exact ? launch_parts<kDeltaExactParts>(a, s) : launch_parts<kDeltaParts>(a, s);
}

}  // namespace luna
