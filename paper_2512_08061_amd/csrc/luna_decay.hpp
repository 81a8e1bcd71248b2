// luna_decay.hpp -- causal linear attention with a decay for each head, in chunks: the
// kernel behind luna_decay_fwd and, with other operands, every pass of luna_decay_bwd.
//
// For row weights w_j (or 1) and, in kDecayAug, one more component a_i, b_j of queries and keys:
//
//   P_ij = f^(i - j) w_j (q_i.k_j + a_i b_j)   (j <= i; reverse: j >= i and f^(j - i)),
//   out_i = c_i sum_j P_ij v_j                 (kDecayNorm: over sum_j P_ij + eps).
//
//   forward        q = Q,  k = K,  v = V
//   dQ             q = dO, k = V,  v = K,  a_i = -dO_i.out_i, b = 1, c_i = 1 / (den_i + eps)
//   dK  (reverse)  q = V,  k = dO, v = Q,  a = 1, b_j = -dO_j.out_j, w_j = 1 / (den_j + eps)
//   dV  (reverse)  q = K,  k = Q,  v = dO, w_j as before
//
// The states of dK are those of dV transposed (with z of weights b_j as their further row), so one state pass serves both.
//
// A workgroup takes one piece of one sequence and head (and up to 128 columns of v) in chunks of C
// tokens, with the discounted state S of the tokens before the chunk in registers: a wave for 16
// columns of S (all features), as accumulator tiles.  Per chunk
//
//   P = mask(Q K^T)                    16 x 16 blocks shared out among the waves, rounded to T, through LDS
//   out^T = f^(i+1) S^T Q^T + V^T P^T  each wave its columns: S's accumulator tiles are the A
//                                      operand as they are (features 4g + j of two tiles are
//                                      the 8 k-slots of a lane group; Q is read in that order)
//   S = f^C S + K^T (f^(C-1-j) w_j V)  the V operand of P's product, scaled
//
// The next chunk's rows are on their way to registers while a chunk is worked on.  A wave holds few registers (16
// columns), so that up to four share a SIMD: a chunk is a chain of dependent steps with three barriers, whose waits
// other waves and workgroups fill.  The scaled V is split in bf16 parts, two (2^-17 of each term), or three with S
// returned (exact_state), so that S then has fp32 accuracy.
// A hidden token weighs 0 in the product with V, and 0 times an infinity or NaN of its value would reach the rows before
// it: in the forward pass such values enter as zeros, and from their token on the column is NaN (3% of the time).
// Denominators are sums of P before its rounding plus q.z with z in fp32 (LDS), so they have
// fp32 accuracy.  With 256 features and up to 64 columns two waves share the features of 16 columns (four waves alone
// leave a SIMD one each: 249 -> 157 us for 4 x 16 heads of 4096 tokens); with 128 columns that was no faster (384 -> 390).
//
// Measured: 8 x 16 heads of 16384 tokens, D = d = 128: 708 us, of which state pass 190, scan 11, row pass 500 (2.1 GB at
// 4.2 TB/s; LDS active 61% of all cycles).  Six packed prompts, 16 heads, 256 features, with denominators: 341 us (77, 23,
// 242); matrix cores 14% busy, bound by the chain of a chunk, one workgroup a compute unit, and 560 pieces over 256
// compute units.
#pragma once

#include "luna_seq.hpp"
#include "luna_split.hpp"

namespace luna {

template <typename T>
constexpr int kDecayChunk = sizeof(T) == 2 ? 64 : 32;

// Parts of P in the product with V: in bf16 with denominators two, P and what its rounding left (out's error on packed LUNA
// prompts 0.0023 -> 0.0017 of its norm, 385 -> 391 us).  One elsewhere: two workgroups a compute unit would not have
// the registers (128 features: 704 -> 787 us).
template <typename T, int MODE, bool OUT>
constexpr int kDecayParts = sizeof(T) == 2 && MODE == kDecayNorm && OUT ? 2 : 1;

// LDS of a workgroup: the chunk's q, k, v and P rows (padded by 16 bytes), then fp32 tables.
template <typename T, int DK, int DVW, int PP>
struct DecayLds {
  static constexpr int FS = DK > 128 && DVW <= 64 ? 2 : 1;  // waves that share the features of 16 columns
  static constexpr int C = kDecayChunk<T>, PAD = 16 / (int)sizeof(T);
  static constexpr int PK = DK + PAD, PV = DVW + PAD, PA = C + PAD;
  T q[C][PK], k[C][PK], v[C][PV], p[PP][C][PA];
  float pw[C + 4];                               // f^0 .. f^C
  float dec[C], kw[C], ka[C], qa[C], ow[C];      // f^(m-1-j) w_j, w_j, b_j, a_i, c_i
  float den[2][C];                               // two waves' shares of the denominators
  float z[DK];
  int since[DVW];  // per column: the first token with a value that is not finite
  f32x4 o[FS > 1 ? DVW / 16 : 1][FS][C / 32][kWave];  // half of out's tiles, from one such wave to the other
  T one[4][C];  // three parts and zeros: of f^(m-1-j) w_j, times b_j in state passes; kDecayAug: of b_j
};

// Rows of one tensor on their way from memory to LDS: C rows of width w (at most W), rows past m and columns past w as
// zeros.
template <typename T, int C, int W, int P, int THREADS>
struct DecayRows {
  static constexpr int E = 16 / (int)sizeof(T), PER = W / E, N = (C * PER + THREADS - 1) / THREADS;
  i32x4 x[N];
  __device__ __forceinline__ void load(const char* base, int64_t row, int m, int w, bool reverse) {
    const Buf b = buffer(base, m > 0 ? (int)(((m - 1) * row + w) * (int)sizeof(T)) : 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = threadIdx.x + THREADS * i, r = idx / PER, c = (idx % PER) * E;
      const int at = (reverse ? m - 1 - r : r) * (int)row + c;
      x[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                           b, r < m && c < w ? at * (int)sizeof(T) : kPastEnd, 0, 0));
    }
  }
  __device__ __forceinline__ void store(T* dst) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = threadIdx.x + THREADS * i, r = idx / PER, c = (idx % PER) * E;
      if (N * THREADS == C * PER || r < C) *reinterpret_cast<i32x4*>(&dst[r * P + c]) = x[i];
    }
  }
  // Infinities and NaN as zeros; since[column]: the first token, t0 + row, that had one.
  __device__ __forceinline__ void clean(int* since, int t0) {
    constexpr uint32_t ALL = sizeof(T) == 2 ? 0x7fff7fff : 0x7fffffff, ONE = sizeof(T) == 2 ? 0x00800080 : 0x00800000;
    constexpr uint32_t TOP = sizeof(T) == 2 ? 0x80008000 : 0x80000000;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= ((uint32_t)x[i][e] & ALL) + ONE;  // (an exponent of ones carries into the sign's place)
    if (!(any & TOP)) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = threadIdx.x + THREADS * i, r = idx / PER, c = (idx % PER) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int word = e * (int)sizeof(T) / 4, shift = sizeof(T) == 2 ? 16 * (e % 2) : 0;
        const uint32_t part = sizeof(T) == 2 ? 0xffffu << shift : 0xffffffffu;
        if ((((uint32_t)x[i][word] & ALL) + ONE) & TOP & part) {
          x[i][word] &= (int)~part;
          atomicMin(&since[c + e], t0 + r);
        }
      }
    }
  }
};

// The scaled values of a fragment as one operand (fp32) or in parts (bf16: two, or three where exact).
template <typename T>
struct DecayScaled;
template <>
struct DecayScaled<float> {
  Frag<float> x;
  __device__ __forceinline__ void set(const Frag<float>& v, const float (&w)[8], bool) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = v.v[e] * w[e];
  }
  __device__ __forceinline__ void mma_into(f32x4& c, const Frag<float>& a, bool) const { mma(c, a, x); }
};
template <>
struct DecayScaled<__bf16> {
  Split3 x;
  __device__ __forceinline__ void set(const Frag<__bf16>& v, const float (&w)[8], bool) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = v.get(e) * w[e];
    split3(x, y);
  }
  __device__ __forceinline__ void mma_into(f32x4& c, const Frag<__bf16>& a, bool exact) const {
    if (exact) mma(c, a, x.p[2]);
    mma(c, a, x.p[1]);
    mma(c, a, x.p[0]);
  }
};

template <int DK, int DVW>
constexpr int kDecayThreads = decay_threads(DK, DVW);

// Waves per SIMD: two workgroups of a compute unit where the registers suffice or nearly so (128 features without
// denominators: 546 -> 487 us of the long batch's row pass, with 2 registers spilled; of those with 64 features up to 3 spill,
// 10 of 64 plain bf16 columns that return a state).  The others would spill more (128 features and 64 columns, whose half as
// many waves carry twice the rows in flight: 254 -> 517 us for 8 x 16 heads of 8192 tokens).
template <typename T, int DK, int DVW, int MODE, bool EXACT>
constexpr int kDecayWaves = DK <= 64 || (DK == 128 && DVW == 128 && MODE == kDecayPlain && !EXACT) ? 4 : 2;

template <typename T, int DK, int DVW, int MODE, bool OUT, bool EXACT>
__global__ __launch_bounds__((kDecayThreads<DK, DVW>), (kDecayWaves<T, DK, DVW, MODE, EXACT>)) void decay_kernel(DecayArgs a) {
  constexpr int PP = kDecayParts<T, MODE, OUT>;
  using Lds = DecayLds<T, DK, DVW, PP>;
  constexpr int C = Lds::C, FS = Lds::FS, FT = DK / 16 / FS, KT = C / 16, KS = C / 32, NW = DVW / 16;
  constexpr int THREADS = kDecayThreads<DK, DVW>, SHARE = FS * NW >= 2 * KT ? 2 : 1;  // SHARE: waves per 16 queries of P
  constexpr int UNROLL = DK > 128 ? 1 : 8;  // (registers)
  static_assert(FS == 1 || MODE != kDecayAug, "za is one wave's");
  constexpr int esz = (int)sizeof(T);
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);

  const int tid = threadIdx.x, lane = tid % kWave, wave = wave_id();
  const int g = lane / 16, c = lane % 16;
  const int slices = (a.dv + DVW - 1) / DVW;
  const int slice = blockIdx.x % slices, head = (blockIdx.x / slices) % a.H, slot = blockIdx.x / slices / a.H;
  const SeqPiece sp = seq_piece(a.s, slot, a.piece);
  if (sp.seq < 0) return;
  const bool packed = a.s.offsets != nullptr, rev = a.reverse;
  const int begin = sp.index * a.piece, end = min(sp.len, begin + a.piece);
  if (!OUT && end == sp.len) return;  // (nothing starts from the state after the last piece)
  const int col0 = slice * DVW, cols = min(DVW, a.dv - col0);
  const int cw = wave % NW, half = FS == 1 ? 0 : wave / NW;
  const int wcol = 16 * cw, wfeat = half * (DK / FS);  // this wave's first column of the slice and first feature

  const float g2 = decay_log2(a.log_decay[head]);
  for (int i = tid; i <= C; i += THREADS) l.pw[i] = exp2_raw(g2 * (float)i);
  constexpr int kNever = 1 << 30;  // (behind any token)
  for (int i = tid; i < DVW; i += THREADS) l.since[i] = kNever;

  // a chunk's rows, and thread tid's numbers of row tid, a chunk ahead
  DecayRows<T, C, DK, Lds::PK, THREADS> qr, kr;
  DecayRows<T, C, DVW, Lds::PV, THREADS> vr;
  float kw = 1.0f, ka = 1.0f, qa = 1.0f, ow = 1.0f;
  const auto load = [&](int t0) {
    const int m = min(C, end - t0);
    const int64_t lo = rev ? sp.len - t0 - m : t0;  // the chunk's first row in memory
    if (OUT) qr.load(seq_row(a.q, sp, packed, head, lo, esz), a.q.row, m, a.dk, rev);
    kr.load(seq_row(a.k, sp, packed, head, lo, esz), a.k.row, m, a.dk, rev);
    vr.load(seq_row(a.v, sp, packed, head, lo, esz) + col0 * esz, a.v.row, m, cols, rev);
    const int r = min(tid, m - 1);
    const int64_t num = seq_num(a.s, sp, a.H, head, lo + (rev ? m - 1 - r : r));
    if (a.kw) kw = a.kw[num];
    if ((MODE == kDecayAug || (MODE == kDecayNorm && !OUT)) && a.ka) ka = a.ka[num];
    if (MODE == kDecayAug && OUT && a.qa) qa = a.qa[num];
    if (OUT && a.ow) ow = a.ow[num];
  };
  load(begin);

  // the state before the piece
  const int64_t sf = decay_state_floats(a.dk, a.dv), sheads = (int64_t)a.H * sf;
  const int state = __builtin_amdgcn_readfirstlane(packed ? (int)seq_first_state(a.s, sp.seq, sp.first, a.piece) + sp.index : slot);
  float* st = a.states ? a.states + ((int64_t)state * a.H + head) * sf : nullptr;  // (not touched where the sequence has one piece)
  const int64_t user = (int64_t)sp.seq * a.H + head;
  const int mycol = wcol + c;
  f32x4 S[FT], za = zero4();  // za: rows 0 to 2 add up to the further key component's row of S (kDecayAug; its parts, in bf16)
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) S[ft] = zero4();
  if (MODE == kDecayNorm) {
    for (int f = tid; f < DK; f += THREADS) l.z[f] = 0.0f;
  }
  const int64_t zat = (int64_t)a.dk * a.dv;
  {
    const float* x = nullptr;
    const float* xz = nullptr;
    if (OUT && a.states && (begin > 0 || end < sp.len)) {
      if (begin > 0 || a.S) x = st, xz = st + zat;
    } else if (OUT && a.S) {
      x = a.S + user * zat;
      if (MODE == kDecayNorm) xz = a.z + user * a.dk;
    }
    if (x) {
      const int64_t row = a.transposed ? 1 : a.dv, col = (int64_t)(col0 + mycol) * (a.transposed ? a.dk : 1);
      if (mycol < cols) {
#pragma unroll
        for (int ft = 0; ft < FT; ++ft)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int k = wfeat + 16 * ft + 4 * g + j;
            if (k < a.dk) S[ft][j] = x[k * row + col];
          }
        if (MODE == kDecayAug && g == 0) za[0] = xz[col0 + mycol];
      }
      if (MODE == kDecayNorm)
        for (int k = tid; k < a.dk; k += THREADS) l.z[k] = xz[k];
    }
  }
  const auto write_state = [&](float* S1, float* z1) {
    if (mycol < cols) {
      const bool lost = l.since[mycol] != kNever;
#pragma unroll
      for (int ft = 0; ft < FT; ++ft)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k = wfeat + 16 * ft + 4 * g + j;
          if (k < a.dk) S1[(int64_t)k * a.dv + col0 + mycol] = lost ? __builtin_nanf("") : S[ft][j];
        }
      if (MODE == kDecayAug && g == 0) z1[col0 + mycol] = lost ? __builtin_nanf("") : za[0] + za[1] + za[2];
    }
    if (MODE == kDecayNorm && slice == 0)
      for (int k = tid; k < a.dk; k += THREADS) z1[k] = l.z[k];
  };
  for (int t0 = begin; t0 < end; t0 += C) {
    const int m = min(C, end - t0);
    __syncthreads();  // the chunk before is no longer read (at first: f^i are written)
    if (OUT) qr.store(&l.q[0][0]);
    kr.store(&l.k[0][0]);
    if (MODE != kDecayAug && a.guard) vr.clean(l.since, t0);
    vr.store(&l.v[0][0]);
    if (tid < C) {
      const bool in = tid < m;
      l.kw[tid] = in ? kw : 0.0f;
      l.dec[tid] = in ? kw * l.pw[max(m - 1 - tid, 0)] : 0.0f;
      if (MODE == kDecayAug) {
        l.ka[tid] = in ? ka : 0.0f;
        if (OUT) l.qa[tid] = in ? qa : 0.0f;
      }
      if (MODE != kDecayPlain) {  // the discounts of z (times b_j) or b_j, bf16: in three parts
        const float x = MODE == kDecayAug ? l.ka[tid] : l.dec[tid] * (OUT ? 1.0f : ka);
        const T part0 = (T)x, part1 = (T)(x - (float)part0);
        l.one[0][tid] = part0;
        l.one[1][tid] = part1;
        l.one[2][tid] = (T)(x - (float)part0 - (float)part1);
        l.one[3][tid] = (T)0.0f;
      }
      if (OUT) l.ow[tid] = ow;
    }
    if (t0 + C < end) load(t0 + C);
    __syncthreads();

    f32x4 o[KT];
    if (OUT) {
      // P: SHARE waves form the rows of a query tile, over the keys before them
      if (wave < SHARE * KT) {
        const int qt = wave / SHARE, share = wave % SHARE, i = 16 * qt + c;
        float den = 0.0f;
        if (MODE == kDecayNorm) {
#pragma unroll UNROLL
          for (int t = 0; t < DK / 32; t += SHARE) {
            const int f = 32 * (t + share) + 8 * g;
            Frag<T> x;
            load8(x, &l.q[i][f]);
#pragma unroll
            for (int e = 0; e < 8; ++e) den = fmaf(x.get(e), l.z[f + e], den);
          }
          den *= l.pw[i + 1];
        }
        Frag<T> qf[DK / 32];
#pragma unroll
        for (int t = 0; t < DK / 32; ++t) load8(qf[t], &l.q[i][32 * t + 8 * g]);
        const float qai = MODE == kDecayAug ? l.qa[i] : 0.0f;
        for (int kt = share; kt < KT && kt <= qt + 1; kt += SHARE) {  // (a block behind the diagonal as zeros)
          f32x4 acc = zero4();
          const f32x4 w = *reinterpret_cast<const f32x4*>(&l.kw[16 * kt + 4 * g]);
          const f32x4 b = MODE == kDecayAug ? *reinterpret_cast<const f32x4*>(&l.ka[16 * kt + 4 * g]) : zero4();
          float f[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = l.pw[max(i - (16 * kt + 4 * g + j), 0)] * w[j];
#pragma unroll
          for (int t = 0; t < DK / 32; ++t) {
            Frag<T> kf;
            load8(kf, &l.k[16 * kt + c][32 * t + 8 * g]);
            mma(acc, kf, qf[t]);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = (MODE == kDecayAug ? fmaf(qai, b[j], acc[j]) : acc[j]) * f[j];
            acc[j] = 16 * kt + 4 * g + j <= i ? x : 0.0f;
            if (MODE == kDecayNorm) den += acc[j];
          }
          store4(&l.p[0][i][16 * kt + 4 * g], acc[0], acc[1], acc[2], acc[3]);
          if constexpr (PP == 2)
            store4(&l.p[1][i][16 * kt + 4 * g], acc[0] - (float)(T)acc[0], acc[1] - (float)(T)acc[1],
                   acc[2] - (float)(T)acc[2], acc[3] - (float)(T)acc[3]);
        }
        if (MODE == kDecayNorm) {
          den = groups_sum(den);
          if (g == 0) l.den[share][i] = den;
        }
      }
      // f^(i+1) S^T Q^T
#pragma unroll
      for (int qt = 0; qt < KT; ++qt) o[qt] = zero4();
#pragma unroll
      for (int t = 0; t < FT / 2; ++t) {
        Frag<T> sf_;
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          sf_.set2(e, S[2 * t][e], S[2 * t][e + 1]);
          sf_.set2(4 + e, S[2 * t + 1][e], S[2 * t + 1][e + 1]);
        }
#pragma unroll
        for (int qt = 0; qt < KT; ++qt) {
          Frag<T> qf;
          load4(qf, 0, &l.q[16 * qt + c][wfeat + 32 * t + 4 * g]);
          load4(qf, 4, &l.q[16 * qt + c][wfeat + 32 * t + 16 + 4 * g]);
          mma(o[qt], sf_, qf);
        }
      }
      if (MODE == kDecayAug) {
        const float z = g == 0 ? za[0] + za[1] + za[2] : 0.0f;
        Frag<T> zf;  // (z and a_i in two parts each: one rounding of either would be 2^-9 of sums that nearly cancel)
        zf.zero();
        zf.set(0, z);
        zf.set(1, z);
        zf.set(2, z - (float)(T)z);
#pragma unroll
        for (int qt = 0; qt < KT; ++qt) {
          Frag<T> qf;
          const float x = l.qa[16 * qt + c];
          qf.zero();
          qf.set(0, x);
          qf.set(1, x - (float)(T)x);
          qf.set(2, x);
          mma(o[qt], zf, qf);
        }
      }
#pragma unroll
      for (int qt = 0; qt < KT; ++qt) {
        const float f = l.pw[16 * qt + c + 1];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[qt][j] *= f;
      }
      __syncthreads();  // P is whole; z has been read
    }

    // V^T P^T, and the state after the chunk
    {
      const float f = l.pw[m];
#pragma unroll
      for (int ft = 0; ft < FT; ++ft)
#pragma unroll
        for (int j = 0; j < 4; ++j) S[ft][j] *= f;
#pragma unroll
      for (int j = 0; j < 3; ++j) za[j] *= f;
    }
    constexpr int ZT = (FT + NW - 1) / NW;  // tiles of z per wave
    f32x4 zacc[ZT];
    if (MODE == kDecayNorm)
#pragma unroll
      for (int i = 0; i < ZT; ++i) zacc[i] = zero4();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float dec[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) dec[e] = l.dec[32 * ks + 8 * g + e];
      Frag<T> vf;
      load_tr4(vf, 0, &l.v[0][0], Lds::PV, 32 * ks + 8 * g, wcol, lane);
      load_tr4(vf, 4, &l.v[0][0], Lds::PV, 32 * ks + 8 * g + 4, wcol, lane);
      DecayScaled<T> vs;
      vs.set(vf, dec, EXACT);
      if (OUT && ks % FS == half) {
#pragma unroll
        for (int qt = 2 * ks; qt < KT; ++qt) {
#pragma unroll
          for (int part = PP - 1; part >= 0; --part) {
            Frag<T> pf;
            load8(pf, &l.p[part][16 * qt + c][32 * ks + 8 * g]);
            mma(o[qt], vf, pf);
          }
        }
      }
      Frag<T> one;  // columns 0 .. 2: the parts
      if (MODE == kDecayNorm) load8(one, &l.one[min(c, 3)][32 * ks + 8 * g]);
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) {
        Frag<T> kf;
        load_tr4(kf, 0, &l.k[0][0], Lds::PK, 32 * ks + 8 * g, wfeat + 16 * ft, lane);
        load_tr4(kf, 4, &l.k[0][0], Lds::PK, 32 * ks + 8 * g + 4, wfeat + 16 * ft, lane);
        vs.mma_into(S[ft], kf, EXACT);
      }
      if (MODE == kDecayNorm) {  // (read again, so that no wave's products stand behind a branch)
#pragma unroll
        for (int i = 0; i < ZT; ++i) {
          const int f = wfeat + 16 * min(NW * i + cw, FT - 1);
          Frag<T> kf;
          load_tr4(kf, 0, &l.k[0][0], Lds::PK, 32 * ks + 8 * g, f, lane);
          load_tr4(kf, 4, &l.k[0][0], Lds::PK, 32 * ks + 8 * g + 4, f, lane);
          mma(zacc[i], kf, one);
        }
      }
      if (MODE == kDecayAug) {
        Frag<T> kf;
        load8(kf, &l.one[min(c, 3)][32 * ks + 8 * g]);
        vs.mma_into(za, kf, EXACT);
      }
    }
    if (MODE == kDecayNorm) {
#pragma unroll
      for (int i = 0; i < ZT; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // the three parts' columns, in every quad of lanes
          float x = zacc[i][j];
          x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xf, 0xf, true));
          x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xf, 0xf, true));
          const int f = 16 * (NW * i + cw) + 4 * g + j;
          if (c == 0 && f < DK / FS) l.z[wfeat + f] = fmaf(l.pw[m], l.z[wfeat + f], x);
        }
      }
    }

    if (OUT) {
      const int64_t lo = rev ? sp.len - t0 - m : t0;
      const Buf b = buffer(seq_row(a.o, sp, packed, head, lo, esz) + col0 * esz, (int)(((m - 1) * a.o.row + cols) * esz));
      constexpr int QT = KT / FS;  // query tiles that this wave writes
      const i32x4 since = *reinterpret_cast<const i32x4*>(&l.since[wcol + 4 * g]);
      f32x4 x[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) x[t] = half ? o[KT - QT + t] : o[t];
      if constexpr (FS == 2) {
#pragma unroll
        for (int t = 0; t < QT; ++t) l.o[cw][half][t][lane] = half ? o[t] : o[KT - QT + t];
        __syncthreads();
#pragma unroll
        for (int t = 0; t < QT; ++t) x[t] += l.o[cw][1 - half][t][lane];
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const int i = 16 * (QT * half + t) + c, r = rev ? m - 1 - i : i;
        float f = a.scale * l.ow[i];
        if (MODE == kDecayNorm) {
          const float den = a.scale * (SHARE == 2 ? l.den[0][i] + l.den[1][i] : l.den[0][i]);
          f = a.scale / (den + a.eps);
          if (a.den && cw == 0 && g == 0 && slice == 0 && i < m) a.den[seq_num(a.s, sp, a.H, head, lo + r)] = den;
        }
        const int col = wcol + 4 * g;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t][e] = MODE != kDecayAug && t0 + i >= since[e] ? __builtin_nanf("") : f * x[t][e];
        buf_store4<T>(b, i < m && col < cols ? (r * (int)a.o.row + col) * esz : kPastEnd, x[t][0], x[t][1], x[t][2], x[t][3]);
      }
    }
  }

  // the state after the piece (state pass), or after the sequence's last token
  if (MODE == kDecayNorm) __syncthreads();  // z is whole
  if (!OUT) write_state(st, st + zat);
  else if (a.S && end == sp.len) write_state(a.S + user * a.dk * a.dv, MODE == kDecayNorm ? a.z + user * a.dk : nullptr);
}

template <typename T, int DK, int DVW, int MODE, bool OUT, bool EXACT>
hipError_t launch_decay_one(const DecayArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(DecayLds<T, DK, DVW, kDecayParts<T, MODE, OUT>>);
  static_assert(bytes <= 160 * 1024, "one workgroup's LDS");
  const hipError_t e = allow_lds<decay_kernel<T, DK, DVW, MODE, OUT, EXACT>>(bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((decay_kernel<T, DK, DVW, MODE, OUT, EXACT>), dim3((unsigned)decay_groups(a.slots, a.H, a.dv)),
                     dim3(kDecayThreads<DK, DVW>), bytes, s, a);
  return hipGetLastError();
}

// (fp32 has one form; gradients return no state)
template <typename T, int DK, int DVW, int MODE, bool OUT>
hipError_t launch_decay_exact(const DecayArgs& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2 && MODE != kDecayAug)
    if (a.exact_state) return launch_decay_one<T, DK, DVW, MODE, OUT, true>(a, s);
  return launch_decay_one<T, DK, DVW, MODE, OUT, false>(a, s);
}

template <typename T, int DK, int MODE, bool OUT>
hipError_t launch_decay_width(const DecayArgs& a, hipStream_t s) {
  return decay_columns(a.dv) == 64 ? launch_decay_exact<T, DK, 64, MODE, OUT>(a, s) : launch_decay_exact<T, DK, 128, MODE, OUT>(a, s);
}

template <typename T, int MODE, bool OUT>
hipError_t launch_decay_mode(const DecayArgs& a, hipStream_t s) {
  if constexpr (MODE != kDecayAug)  // (whose keys are V or dO)
    if (a.dk > 128) return launch_decay_width<T, 256, MODE, OUT>(a, s);
  return a.dk <= 64 ? launch_decay_width<T, 64, MODE, OUT>(a, s) : launch_decay_width<T, 128, MODE, OUT>(a, s);
}

// one translation unit per element type and mode (luna_decay_*.hip)
template <typename T, int MODE>
hipError_t launch_decay_typed(const DecayArgs& a, bool out, hipStream_t s);
#define LUNA_DECAY_TYPED(T, MODE)                                                     \
  template <>                                                                         \
  hipError_t launch_decay_typed<T, MODE>(const DecayArgs& a, bool out, hipStream_t s) { \
    return out ? launch_decay_mode<T, MODE, true>(a, s) : launch_decay_mode<T, MODE, false>(a, s); \
  }

}  // namespace luna
