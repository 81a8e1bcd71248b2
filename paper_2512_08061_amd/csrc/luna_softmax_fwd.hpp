// luna_softmax_fwd.hpp -- causal softmax attention over sequences of different lengths, forward (luna_softmax.hip; over pages:
// luna_paged_tiles.hip).
//
//   s_ij = scale q_i.k_j (j <= i + Lk - Lq),  out_i = sum_j exp(s_ij - lse_i) v_j.
//
// One pass over the keys with the running maximum and sum of each row.  A workgroup of four waves
// takes 64 queries of one head, a wave 16 of them.  Scores are formed transposed, S^T = K Q^T:
// lane (g, c) of a block of 16 keys holds keys 4g + j of query c, so a row's maximum and
// sum are four registers and two lane exchanges, and two blocks of probabilities are
// the B operand of out^T = V^T P^T as they are (keys 4g + j of both as the 8 k-slots; V is read
// in that order with transposing reads).  Maxima and sums are fp32, in base 2; P is rounded to
// the element type as an operand after its sum is taken.  fp32 with d = 128, 4 x 16 heads of 2048 tokens: 601 us, 114
// TFLOP/s of the 144 that a large fp32 product reaches.
#pragma once

#include "luna_softmax.hpp"

namespace luna {

template <typename T, int DH>
struct SoftmaxLds {
  static constexpr int KB = kSoftmaxStep<T>, P = DH + 16 / (int)sizeof(T);
  T k[KB][P], v[KB][P];
};

template <typename T, int DH, bool PAGED>
__global__ __launch_bounds__(256) void softmax_fwd_kernel(SoftmaxArgs a) {
  using Lds = SoftmaxLds<T, DH>;
  constexpr int KB = Lds::KB, P = Lds::P, KT = KB / 16, CT = DH / 16, esz = (int)sizeof(T);
  __shared__ __attribute__((aligned(16))) char raw[sizeof(Lds)];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id(), g = lane / 16, c = lane % 16;
  const int head = blockIdx.x % a.H;
  const SeqPiece sq = seq_piece_by_work(a.qs, blockIdx.x / a.H, gridDim.x / a.H, kSoftmaxTile, true);
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
    int none = 0;  // keys whose page is none of the pool
    if constexpr (PAGED) {
      const KeyPages<KB / 16> pages = key_pages<KB / 16>(a, sk.seq, k0, kend);
      none = pages.none;
      softmax_load_pages<T, KB, DH, P>(&l.k[0][0], [&](int i) { return key_group(a, a.k, pages.at(i), hk, k0 + 16 * i, kend, DH, esz); }, a.k.row);
      softmax_load_pages<T, KB, DH, P>(&l.v[0][0], [&](int i) { return key_group(a, a.v, pages.at(i), hk, k0 + 16 * i, kend, DH, esz); }, a.v.row);
    } else {
      softmax_load_rows<T, KB, DH, P>(&l.k[0][0], seq_row(a.k, sk, pk, hk, k0, esz), a.k.row, kn);
      softmax_load_rows<T, KB, DH, P>(&l.v[0][0], seq_row(a.v, sk, pk, hk, k0, esz), a.v.row, kn);
    }
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
        s[kt][j] = key <= last && key < kend && (!PAGED || !(none >> kt & 1)) ? x : -__builtin_inff();
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
  bool bad = false;
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[t][j] *= inv;
      bad |= not_finite(o[t][j]);
    }
  uint64_t rows = __ballot(bad && i < m);
  rows = (rows | rows >> 32) & 0xffffffff;
  rows = (rows | rows >> 16) & 0xffff;
  if (rows && !softmax_odd_values<T, DH, kWave, PAGED>(a, sk, hk, q0 + 16 * wave + shift + 1, kend)) rows = 0;
  const bool good = i < m && !(rows >> c & 1);
  const Buf b = buffer(seq_row(a.o, sq, pq, head, q0, esz), (int)(((m - 1) * a.o.row + DH) * esz));
#pragma unroll
  for (int t = 0; t < CT; ++t)
    buf_store4<T>(b, good ? (i * (int)a.o.row + 16 * t + 4 * g) * esz : kPastEnd, o[t][0], o[t][1], o[t][2],
                  o[t][3]);
  if (a.lse && g == 0 && i < m) a.lse[seq_num(a.qs, sq, a.H, head, q0 + i)] = (top + log2f(sum)) * kLn2;
  for (; rows; rows &= rows - 1) softmax_row<T, DH, kWave, PAGED>(a, sq, sk, head, q0 + 16 * wave + __builtin_ctzll(rows));
}

// bf16 with d = 64 and 128: 32 x 32 x 16 products, a wave with 32 queries of a workgroup's 128, keys in blocks of 64.
// Lane (h, c) of a 32-key block of S^T holds keys 8 (i / 4) + 4 h + i % 4 of query c; eight of the sixteen
// are the k-slots of its half for the product with V.  The next block is on its way to registers while one is worked on.
// The output is rescaled only when some row's maximum has grown by more than 2^8 since its last rescaling (a sum of
// at most 2^8 times larger terms keeps its relative accuracy), which most blocks skip.
// Packed prompts of up to 16384 tokens, 16 heads of 128 on 4: 1450 to 1550 us on different cards, 925 to 970 TFLOP/s over the
// visible pairs; matrix cores 47% busy, the rest the exponentials and maxima between the two products, at two waves a SIMD.
// With GROUPS = 2 two groups of four waves take the key blocks in turn, each with its own maxima, sums and rows, which are
// joined at the end: the last tile of a sequence is a chain half as long.
template <int DH, int GROUPS>
struct SoftmaxLds32 {
  Tile<DH> k[GROUPS][2], v[GROUPS][2];  // per group of waves, twice
};

// A tile and the keys first (a multiple of 64) .. end - 1 that it sees; part: where its rows go that are part of the sequence's
// ([token][head of the key head][d + 2]: unnormalised, then the sum and the maximum), null: to out.
template <int DH, int GROUPS, bool PAGED>
__device__ __forceinline__ void softmax_tile32(const SoftmaxArgs& a, char* raw, int head, const SeqPiece& sq, const SeqPiece& sk,
                                               int first, int end, float* part_rows) {
  constexpr int KB = 64, KS = DH / 16, CT = DH / 32, esz = 2;
  SoftmaxLds32<DH, GROUPS>& l = *reinterpret_cast<SoftmaxLds32<DH, GROUPS>*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id() % 4, h = lane / 32, c = lane % 32;
  const int group = GROUPS == 1 ? 0 : wave_id() / 4, tid = threadIdx.x % 256;
  const bool pq = a.qs.offsets != nullptr, pk = a.ks.offsets != nullptr;
  const int q0 = sq.index * 128, m = min(128, sq.len - q0);
  const int shift = sk.len - sq.len;
  const int kend = min(end, max(0, q0 + m + shift));
  const int i = 32 * wave + c, last = q0 + i + shift;
  const int wfirst = q0 + 32 * wave + shift, wlast = min(wfirst + 31, kend - 1);  // the wave's rows see all keys up to / none behind
  const int hk = head / (a.H / a.Hk);

  // scores are taken with |scale|, the sign going to q (0 as a tiny scale, so that masked scores stay -infinity)
  bf16x8 qf[KS];
  {
    const Buf b = buffer(seq_row(a.q, sq, pq, head, q0, esz), (int)(((m - 1) * a.q.row + DH) * esz));
    const int flip = a.scale < 0.0f ? (int)0x80008000 : 0;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      i32x4 x = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                              b, i < m ? (i * (int)a.q.row + 16 * t + 8 * h) * esz : kPastEnd, 0, 0));
      qf[t] = __builtin_bit_cast(bf16x8, x ^ flip);
    }
  }
  const float scale = fmaxf(fabsf(a.scale) * kLog2e, 1e-37f);
  f32x16 o[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;
  float base = -__builtin_inff(), sum = 0.0f;

  TileRegs<DH> kr, vr;
  int none = 0;  // of the block on its way: keys whose page is none of the pool, a bit for 16
  const auto load = [&](int k0) {
    if constexpr (PAGED) {
      const KeyPages<4> pages = key_pages<4>(a, sk.seq, k0, kend);
      none = pages.none;
      Tile<DH>::load_pages(kr, wave, lane, [&](int i) { return key_group(a, a.k, pages.at(i), hk, k0 + 16 * i, kend, DH, esz); }, a.k.row);
      Tile<DH>::load_pages(vr, wave, lane, [&](int i) { return key_group(a, a.v, pages.at(i), hk, k0 + 16 * i, kend, DH, esz); }, a.v.row);
      return;
    }
    Tile<DH>::load(kr, tid, seq_row(a.k, sk, pk, hk, k0, esz), a.k.row, min(KB, kend - k0));
    Tile<DH>::load(vr, tid, seq_row(a.v, sk, pk, hk, k0, esz), a.v.row, min(KB, kend - k0));
  };
  load(first + KB * group);
  l.k[group][0].store(kr, tid);
  l.v[group][0].store(vr, tid);
  int buf = 0;
  for (int k0 = first + KB * group; k0 - KB * group < kend; k0 += GROUPS * KB, buf ^= 1) {
    __syncthreads();  // this block is whole, and the one before no longer read
    const int without = none;
    load(k0 + GROUPS * KB);
    if (k0 <= wlast) {
      f32x16 s[2];
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[half][e] = 0.0f;
#pragma unroll
      for (int t = 0; t < KS; ++t)
#pragma unroll
        for (int half = 0; half < 2; ++half)
          s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(l.k[group][buf].row8(32 * half + c, 2 * t + h), qf[t], s[half], 0, 0, 0);
      // V operands of 16 keys, read one step before their products (by itself the compiler reads each right before
      // its use and waits out the LDS 16 times a block)
      Frag<__bf16> vf[2][CT];
      const auto read_v = [&](int ks) {
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          const int row = 16 * ks + 4 * h, col = 32 * t + 16 * ((lane / 16) % 2);
          l.v[group][buf].tr4(vf[ks % 2][t], 0, row, col, lane);
          l.v[group][buf].tr4(vf[ks % 2][t], 4, row + 8, col, lane);
        }
      };
      read_v(0);
      if constexpr (PAGED) mma_settle<12>();  // (the test of `without` is a path around the masking)
      if (k0 + KB - 1 > wfirst || k0 + KB > kend || (PAGED && without)) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = k0 + 32 * half + 8 * (e / 4) + 4 * h + e % 4;
            const bool seen = key <= last && key < kend && (!PAGED || !(without >> (2 * half + e / 8) & 1));
            s[half][e] = seen ? s[half][e] : -__builtin_inff();
          }
      }
      float most = fmaxf(s[0][0], s[1][0]);
#pragma unroll
      for (int e = 1; e < 16; ++e) most = fmaxf(fmaxf(most, s[0][e]), s[1][e]);
      {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(most), __float_as_uint(most), false, false);
        most = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])) * scale;
      }
      const bool grow = most > base + 8.0f;  // (base -inf: any key seen; NaN: no)
      if (__any(grow)) {
        const float to = grow ? most : base;
        const float f = exp2_raw(base - (to == -__builtin_inff() ? 0.0f : to));
        base = to;
        sum *= f;
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[t][e] *= f;
      }
      const float b = base == -__builtin_inff() ? 0.0f : base;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        Frag<__bf16> pf;
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float x = exp2_raw(fmaf(s[ks / 2][8 * (ks % 2) + e], scale, -b));
          const float y = exp2_raw(fmaf(s[ks / 2][8 * (ks % 2) + e + 1], scale, -b));
          part += x + y;
          pf.set2(e, x, y);
        }
        sum += part;
        if (ks < 3) read_v(ks + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < CT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ks % 2][t].v, pf.v, o[t], 0, 0, 0);
      }
    }
    l.k[group][buf ^ 1].store(kr, tid);
    l.v[group][buf ^ 1].store(vr, tid);
  }
  sum = halves_sum(sum);
  if constexpr (GROUPS == 2) {  // the second group's rows join the first's
    constexpr int ROWS = 4 * kWave * CT * 16;
    static_assert(sizeof(l) >= (ROWS + 256) * sizeof(float), "a group's rows fit the tiles");
    float* part = reinterpret_cast<float*>(raw);
    f32x4* rows = reinterpret_cast<f32x4*>(raw);
    __syncthreads();
    if (group == 1) {
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          rows[((t * 4 + e) * 4 + wave) * kWave + lane] = f32x4{o[t][4 * e], o[t][4 * e + 1], o[t][4 * e + 2], o[t][4 * e + 3]};
      if (h == 0) {
        part[ROWS + i] = base;
        part[ROWS + 128 + i] = sum;
      }
    }
    __syncthreads();
    if (group == 1) return;
    const float other = part[ROWS + i], most = fmaxf(base, other), to = most == -__builtin_inff() ? 0.0f : most;
    const float f = exp2_raw(base - to), g = exp2_raw(other - to);
    base = most;
    sum = sum * f + part[ROWS + 128 + i] * g;
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[t][e] = fmaf(o[t][e], f, g * rows[((t * 4 + e / 4) * 4 + wave) * kWave + lane][e % 4]);
  }
  if (PAGED && part_rows) {
    const int heads = a.H / a.Hk;
    float* to = part_rows + (int64_t)((q0 + i) * heads + head % heads) * (DH + 2);
    if (i < m) {
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 2)  // (rows of d + 2 numbers begin at multiples of 8 bytes)
          *reinterpret_cast<float2*>(to + 32 * t + 2 * (e - e % 4) + 4 * h + e % 4) = float2{o[t][e], o[t][e + 1]};
      if (h == 0) to[DH] = sum, to[DH + 1] = base;
    }
    return;
  }
  const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;  // (NaN stays)
  bool bad = false;
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      o[t][e] *= inv;
      bad |= not_finite(o[t][e]);
    }
  uint64_t rows = __ballot(bad && i < m);
  rows = (rows | rows >> 32) & 0xffffffff;
  if (rows && !softmax_odd_values<__bf16, DH, kWave, PAGED>(a, sk, hk, wfirst + 1, kend)) rows = 0;
  const bool good = i < m && !(rows >> c & 1);
  const Buf b = buffer(seq_row(a.o, sq, pq, head, q0, esz), (int)(((m - 1) * a.o.row + DH) * esz));
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      buf_store4<__bf16>(b, good ? (i * (int)a.o.row + 32 * t + 2 * e + 4 * h) * esz : kPastEnd, o[t][e], o[t][e + 1], o[t][e + 2],
                         o[t][e + 3]);
  if (a.lse && h == 0 && i < m) a.lse[seq_num(a.qs, sq, a.H, head, q0 + i)] = (base + log2f(sum)) * kLn2;
  for (; rows; rows &= rows - 1) softmax_row<__bf16, DH, kWave, PAGED>(a, sq, sk, head, q0 + 32 * wave + __builtin_ctzll(rows));
}

template <int DH, int GROUPS, bool PAGED>
__global__ __launch_bounds__(256 * GROUPS, 2) void softmax_fwd32_kernel(SoftmaxArgs a) {
  extern __shared__ __attribute__((aligned(16))) char raw[];
  const int head = head_of(blockIdx.x % a.H, a.H);
  const SeqPiece sq = seq_piece_by_work(a.qs, blockIdx.x / a.H, gridDim.x / a.H, 128, true);
  if (sq.seq < 0) return;
  const SeqPiece sk = seq_of(a.ks, sq.seq);
  softmax_tile32<DH, GROUPS, PAGED>(a, raw, head, sq, sk, 0, sk.len, nullptr);
}

// Over pages, what a share of the line of all sequences' keys holds of one sequence (see PagedUnits), for the tiles of one number
// and head: whole sequences are finished here, the parts of others are joined by a launch behind it.  (512 new tokens of caches of 4096,
// 1999, 700 and 16384, 16 heads on 4, d = 128: 138 and 27 us; without shares the longest cache kept 64 of 256 compute units busy
// for 348.)
template <int DH>
__global__ __launch_bounds__(256, 2) void softmax_part32_kernel(SoftmaxArgs a, int shares) {
  extern __shared__ __attribute__((aligned(16))) char raw[];
  const int tiles = (int)((a.qs.rows + 127) / 128), tile = blockIdx.x / a.H % tiles, rank = blockIdx.x / (tiles * a.H);
  const int head = head_of(blockIdx.x % a.H, a.H), heads = a.H / a.Hk;
  int share;
  PagedUnits held;
  const int b = sequence_of_part(a.ks, rank, shares, kPagedTileUnit, &share, &held);
  if (b < 0) return;
  const SeqPiece sk = seq_uniform(seq_of(a.ks, b));
  SeqPiece sq = seq_uniform(seq_of(a.qs, b));
  if (128 * tile >= sq.len) return;
  sq.index = tile;
  const bool whole = held.u0 == 0 && held.u1 * kPagedTileUnit >= sk.len;
  float* rows = a.parts + (paged_part(share, b) * a.Hk + head / heads) * (a.qs.rows * heads) * (DH + 2);
  softmax_tile32<DH, 1, true>(a, raw, head, sq, sk, kPagedTileUnit * held.u0, min(sk.len, kPagedTileUnit * held.u1), whole ? nullptr : rows);
}

template <int DH, int GROUPS, bool PAGED>
hipError_t launch_groups(const SoftmaxArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(SoftmaxLds32<DH, GROUPS>);
  const hipError_t e = allow_lds<softmax_fwd32_kernel<DH, GROUPS, PAGED>>(bytes);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(seq_slots(a.qs, 128) * a.H));
  hipLaunchKernelGGL((softmax_fwd32_kernel<DH, GROUPS, PAGED>), grid, dim3(256 * GROUPS), bytes, s, a);
  return hipGetLastError();
}

// Two groups where the longest chain counts: up to two workgroups a compute unit (of which one with two groups, or
// two with one, run at once).  d = 128, one group and two: 16 heads of 1999 tokens 46.6 and 41.9 us, 32 heads 57.2 and
// 55.1, 16 heads of 4000 tokens 98 and 88, but 8 x 512 tokens 25.0 and 33.2, 12 heads of 8000 tokens 228 and 247.
template <int DH, bool PAGED>
hipError_t launch_fwd32(const SoftmaxArgs& a, hipStream_t s) {
  return seq_slots(a.qs, 128) * a.H <= 512 ? launch_groups<DH, 2, PAGED>(a, s) : launch_groups<DH, 1, PAGED>(a, s);
}

template <int DH>
hipError_t launch_shares(const SoftmaxArgs& a, int shares, hipStream_t s) {
  constexpr int bytes = (int)sizeof(SoftmaxLds32<DH, 1>);
  hipError_t e = allow_lds<softmax_part32_kernel<DH>>(bytes);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)((shares + a.qs.count) * ((a.qs.rows + 127) / 128) * a.H));
  hipLaunchKernelGGL((softmax_part32_kernel<DH>), grid, dim3(256), bytes, s, a, shares);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  return launch_paged_tile_join(a, shares, s);
}

template <typename T, int DH, bool PAGED>
hipError_t launch_fwd(const SoftmaxArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((softmax_fwd_kernel<T, DH, PAGED>), dim3((unsigned)(seq_slots(a.qs, kSoftmaxTile) * a.H)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <bool PAGED>
hipError_t launch_tiles(Dt dt, const SoftmaxArgs& a, hipStream_t s) {
  if (dt == Dt::F32)
    return a.d == 32 ? launch_fwd<float, 32, PAGED>(a, s) : a.d == 64 ? launch_fwd<float, 64, PAGED>(a, s) : launch_fwd<float, 128, PAGED>(a, s);
  if constexpr (PAGED)
    if (const int shares = paged_tile_shares(dt, a.qs, a.H, a.Hk, a.d))
      return a.d == 64 ? launch_shares<64>(a, shares, s) : launch_shares<128>(a, shares, s);
  return a.d == 32 ? launch_fwd<__bf16, 32, PAGED>(a, s) : a.d == 64 ? launch_fwd32<64, PAGED>(a, s) : launch_fwd32<128, PAGED>(a, s);
}

}  // namespace luna
