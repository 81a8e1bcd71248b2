// luna_paged_split.hip -- softmax attention of few rows per key head over the pages of a cache (the next tokens of
// sequences): what bounds it is reading the keys and values once (32 caches of up to 8192 tokens, 16 heads on 4, d = 128, 258 MB:
// 69.9 us, 3.7 TB/s, and 7.4 to join), and for few tokens the chain of dependent loads (one cache of 3001: 11.0 and 6.2 us).
//
// The rows of a key head, m tokens of its H / Hk heads each, are one operand of up to RT tiles of 16, so that the cache is
// read once for the whole group (in fp32 once for 32 rows, a workgroup each).  The keys of all sequences, in units of paged_unit(), are one line that is cut in equal shares,
// a workgroup each (lengths are on the device: every workgroup adds them up by itself), so that long and short sequences
// load the device alike.  A share may hold the end of one sequence, several, and the beginning of another; within each
// its four waves take the units in turn, each with a running maximum, sum and unnormalised output of its own, which are joined
// through LDS.  A sequence that lies in one share is finished there; the parts of others are joined by a second launch, in
// a fixed order.  Parts are numbered share + sequence: along the line one of the two grows from part to part.
// Keys go from memory straight to the matrix operand (no other wave reads them); values pass through LDS, in the wave's own
// part of it, to be read transposed.  16 keys from a multiple of 16 on lie in one page, whose number is the same for all lanes.
#include "luna_softmax.hpp"

namespace luna {

namespace {

template <typename T, int DH>
struct PagedLds {
  static constexpr int KB = sizeof(T) == 2 ? 64 : 32, P = DH + (sizeof(T) == 2 ? 16 : 4);
  union {
    T v[4][KB][P];
    float o[4][16][DH + 1];  // at the join: a row tile of every wave
  };
  float top[4][16], sum[4][16];
  int64_t scan[4];
};

template <typename T, int DH, int RT>
__global__ __launch_bounds__(256) void paged_split_kernel(SoftmaxArgs a, int shares, int row_groups) {
  using Lds = PagedLds<T, DH>;
  constexpr int KB = Lds::KB, P = Lds::P, KT = KB / 16, CT = DH / 16, DT = DH / 32, esz = (int)sizeof(T), E = 16 / esz;
  constexpr int PER = DH / E, VL = KB * PER / kWave;  // 16-byte pieces of a row, and of a unit's values per lane
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id(), g = lane / 16, c = lane % 16;
  const int hk = blockIdx.x % a.Hk, row0 = blockIdx.x / a.Hk % row_groups * (16 * RT), number = blockIdx.x / a.Hk / row_groups;
  const int64_t all = units_before(a.ks, (int)a.ks.count, KB, l.scan), per = paged_per(all, shares, kPagedLeast);
  int64_t first;  // units before sequence b
  int b, share, stop = (int)a.ks.count;
  if (per > kPagedLeast || gridDim.x == (unsigned)(shares * a.Hk * row_groups)) {  // a share
    share = number;
    if (share >= shares || share * per >= all) return;
    b = sequence_at(a.ks, share * per, KB, &first);
  } else {  // of a short line what a share holds of one sequence, so that no sequence waits for another
    b = sequence_of_number(a.ks, number, shares, KB, per, all, &first);
    if (b < 0) return;
    share = number - b;
    stop = b + 1;
  }
  const int64_t end = min(all, (share + 1) * per);
  const int group = a.H / a.Hk, rows = (int)a.qs.rows * group;
  const float scale = a.scale * kLog2e;

  for (; b < stop && first < end; ++b) {
    const SeqPiece sk = seq_uniform(seq_of(a.ks, b)), sq = seq_uniform(seq_of(a.qs, b));
    const int units = (sk.len + KB - 1) / KB, shift = sk.len - sq.len;
    const PagedUnits held = paged_held(first, units, per, share, all);
    const int u0 = held.u0, u1 = held.u1;
    first += units;
    if (u0 >= u1) continue;
    Frag<T> qf[RT][DT];
    int last[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = row0 + 16 * rt + c, t = r / group;
      const bool in = r < rows && t < sq.len;
      last[rt] = in ? t + shift : -1;
      const T* q = reinterpret_cast<const T*>(a.q.data) + (in ? b * a.q.seq + (hk * group + r % group) * a.q.head + t * a.q.row : 0);
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        if (in) load8(qf[rt][i], q + 32 * i + 8 * g);
        else qf[rt][i].zero();
      }
    }
    f32x4 o[RT][CT];
    float top[RT], sum[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      top[rt] = -__builtin_inff();
      sum[rt] = 0.0f;
#pragma unroll
      for (int i = 0; i < CT; ++i) o[rt][i] = zero4();
    }
    const int seen = min(u1, ((min(row0 + 16 * RT, rows) - 1) / group + shift) / KB + 1);  // (the units that the last of the rows sees)
    for (int u = u0 + wave; u < seen; u += 4) {
      const int k0 = u * KB;
      const KeyPages<KT> pages = key_pages<KT>(a, b, k0, sk.len);
      Frag<T> kf[KT][DT];
      i32x4 vr[VL];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const Buf bk = key_group(a, a.k, pages.page[kt], hk, k0 + 16 * kt, sk.len, DH, esz);
#pragma unroll
        for (int i = 0; i < DT; ++i) buf_load8(kf[kt][i], bk, (c * (int)a.k.row + 32 * i + 8 * g) * esz);
      }
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        const int idx = lane + kWave * i, r = idx / PER, col = (idx % PER) * E;
        static_assert(kWave / PER <= 16, "a load's rows lie in one group");
        const Buf bv = key_group(a, a.v, pages.page[kWave * i / PER / 16], hk, k0 + kWave * i / PER / 16 * 16, sk.len, DH, esz);
        vr[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(bv, (r % 16 * (int)a.v.row + col) * esz, 0, 0));
      }
      f32x4 s[RT][KT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          s[rt][kt] = zero4();
#pragma unroll
          for (int i = 0; i < DT; ++i) mma(s[rt][kt], kf[kt][i], qf[rt][i]);
        }
      wave_lds_fence();  // the unit before has been read
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        const int idx = lane + kWave * i;
        *reinterpret_cast<i32x4*>(&l.v[wave][idx / PER][(idx % PER) * E]) = vr[i];
      }
      wave_lds_fence();
      Frag<T> pf[RT][KT / 2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float most = top[rt];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int key = k0 + 16 * kt + 4 * g + j;
            const float x = s[rt][kt][j] * scale;
            s[rt][kt][j] = key < sk.len && key <= last[rt] && !(pages.none >> kt & 1) ? x : -__builtin_inff();
            most = fmaxf(most, s[rt][kt][j]);
          }
        most = groups_max(most);
        const float base = most == -__builtin_inff() ? 0.0f : most;
        const float f = exp2_raw(top[rt] - base);
        top[rt] = most;
        float part = 0.0f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[rt][kt][j] = exp2_raw(s[rt][kt][j] - base);
            part += s[rt][kt][j];
          }
        sum[rt] = fmaf(sum[rt], f, part);
#pragma unroll
        for (int i = 0; i < CT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[rt][i][j] *= f;
#pragma unroll
        for (int ks = 0; ks < KT / 2; ++ks)
#pragma unroll
          for (int j = 0; j < 4; j += 2) {
            pf[rt][ks].set2(j, s[rt][2 * ks][j], s[rt][2 * ks][j + 1]);
            pf[rt][ks].set2(4 + j, s[rt][2 * ks + 1][j], s[rt][2 * ks + 1][j + 1]);
          }
      }
#pragma unroll
      for (int ks = 0; ks < KT / 2; ++ks)
#pragma unroll
        for (int i = 0; i < CT; ++i) {
          Frag<T> vf;
          load_tr4(vf, 0, &l.v[wave][0][0], P, 32 * ks + 4 * g, 16 * i, lane);
          load_tr4(vf, 4, &l.v[wave][0][0], P, 32 * ks + 16 + 4 * g, 16 * i, lane);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) mma(o[rt][i], vf, pf[rt][ks]);
        }
    }

    // the four waves' rows joined: the rows themselves, or of this part the maximum, the sum and the unnormalised output
    const bool whole = u0 == 0 && u1 == units;
    float* part = a.parts + (paged_part(share, b) * a.Hk + hk) * rows * (DH + 2);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float mine = groups_sum(sum[rt]);
      __syncthreads();
      if (g == 0) {
        l.top[wave][c] = top[rt];
        l.sum[wave][c] = mine;
      }
#pragma unroll
      for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) l.o[wave][c][16 * i + 4 * g + j] = o[rt][i][j];
      __syncthreads();
      constexpr int LANES = DH < kWave ? DH : kWave;  // a row's threads
      for (int r0 = 0; r0 < 16; r0 += 256 / LANES) {
        const int r = r0 + (int)threadIdx.x / LANES, x = threadIdx.x % LANES, row = row0 + 16 * rt + r;
        const float most = fmaxf(fmaxf(l.top[0][r], l.top[1][r]), fmaxf(l.top[2][r], l.top[3][r]));
        const float base = most == -__builtin_inff() ? 0.0f : most;
        float f[4], y[DH / LANES], total = 0.0f;
#pragma unroll
        for (int e = 0; e < DH / LANES; ++e) y[e] = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          f[w] = exp2_raw(l.top[w][r] - base);
          total = fmaf(f[w], l.sum[w][r], total);
#pragma unroll
          for (int e = 0; e < DH / LANES; ++e) y[e] = fmaf(f[w], l.o[w][r][x + LANES * e], y[e]);
        }
        const int t = row / group, head = hk * group + row % group;
        const bool in = row < rows && t < sq.len;
        if (!whole) {
          if (row < rows) {
#pragma unroll
            for (int e = 0; e < DH / LANES; ++e) part[row * (DH + 2) + x + LANES * e] = y[e];
            if (x == 0) part[row * (DH + 2) + DH] = total, part[row * (DH + 2) + DH + 1] = most;
          }
          continue;
        }
        const float inv = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < DH / LANES; ++e) odd |= not_finite(y[e] * inv);
        // (uniform for a row's threads where a wave has one)
        uint64_t lost = __ballot(in && odd);
        if constexpr (LANES < kWave) lost = lost >> (lane / LANES * LANES) & (((uint64_t)1 << LANES) - 1);
        if (in && a.lse && x == 0) a.lse[seq_num(a.qs, sq, a.H, head, t)] = (most + log2f(total)) * kLn2;
        if (in && lost && softmax_odd_row<T, DH, LANES>(a, sk, hk, t + shift + 1, sk.len)) {
          softmax_row<T, DH, LANES, true>(a, sq, sk, head, t);
        } else if (in) {
          T* to = reinterpret_cast<T*>(seq_row(a.o, sq, false, head, t, esz));
#pragma unroll
          for (int e = 0; e < DH / LANES; ++e) to[x + LANES * e] = (T)(y[e] * inv);
        }
      }
    }
    __syncthreads();  // (the next sequence's values take the rows' place)
  }
}

// Rows whose keys lie in several shares joined, `times` rows a thread group; rows of sequences without any key as zeros.
template <typename T, int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(SoftmaxArgs a, int shares, int unit, int least, int times) {
  constexpr int LANES = DH < kWave ? DH : kWave, ROWS = 256 / LANES, N = DH / LANES;
  __shared__ int64_t scan[4];
  const int group = a.H / a.Hk, rows = (int)a.qs.rows * group, tiles = (rows + ROWS * times - 1) / (ROWS * times);
  const int tile = blockIdx.x % tiles, hk = blockIdx.x / tiles % a.Hk, b = blockIdx.x / tiles / a.Hk;
  const SeqPiece sq = seq_of(a.qs, b), sk = seq_of(a.ks, b);
  const int64_t all = units_before(a.ks, (int)a.ks.count, unit, scan), before = units_before(a.ks, b, unit, scan);
  const PagedUnits holders = paged_holders(before, (sk.len + unit - 1) / unit, paged_per(all, shares, least));
  const int s0 = holders.u0, s1 = holders.u1;
  if (s0 == s1) return;  // (finished there)
  const int x = threadIdx.x % LANES, lane = threadIdx.x % kWave;
  const int64_t step = (int64_t)a.Hk * rows * (DH + 2);
  for (int n = 0; n < times; ++n) {
    const int row = (tile * times + n) * ROWS + (int)threadIdx.x / LANES, t = row / group, head = hk * group + row % group;
    if (row >= rows || t >= sq.len) return;
    const float* part = a.parts + (paged_part(s0, b) * a.Hk + hk) * rows * (DH + 2) + (int64_t)row * (DH + 2);
    float most = -__builtin_inff(), total = 0.0f, y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = 0.0f;
#pragma unroll 4
    for (int i = 0; i <= s1 - s0; ++i) most = fmaxf(most, part[i * step + DH + 1]);
    const float base = most == -__builtin_inff() ? 0.0f : most;
#pragma unroll 4
    for (int i = 0; i <= s1 - s0; ++i) {
      const float f = exp2_raw(part[i * step + DH + 1] - base);
      total = fmaf(f, part[i * step + DH], total);
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = fmaf(f, part[i * step + x + LANES * e], y[e]);
    }
    const float inv = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
    bool odd = false;
#pragma unroll
    for (int e = 0; e < N; ++e) odd |= not_finite(y[e] * inv);
    uint64_t lost = __ballot(odd);
    if constexpr (LANES < kWave) lost = lost >> (lane / LANES * LANES) & (((uint64_t)1 << LANES) - 1);
    if (a.lse && x == 0) a.lse[seq_num(a.qs, sq, a.H, head, t)] = (most + log2f(total)) * kLn2;
    if (lost && softmax_odd_row<T, DH, LANES>(a, sk, hk, t + sk.len - sq.len + 1, sk.len)) {
      softmax_row<T, DH, LANES, true>(a, sq, sk, head, t);
      continue;
    }
    T* to = reinterpret_cast<T*>(seq_row(a.o, sq, false, head, t, (int)sizeof(T)));
#pragma unroll
    for (int e = 0; e < N; ++e) to[x + LANES * e] = (T)(y[e] * inv);
  }
}

template <typename T, int DH, int RT>
hipError_t launch_rows(const SoftmaxArgs& a, int shares, hipStream_t s) {
  constexpr int bytes = (int)sizeof(PagedLds<T, DH>);
  const hipError_t e = allow_lds<paged_split_kernel<T, DH, RT>>(bytes);
  if (e != hipSuccess) return e;
  // Of a short line a sequence of a share each, as long as these run side by side: caches of 11, 10, 510 and 19 tokens, d = 128, 15.5
  // instead of 27.3 us; eight of up to 3371, 12 heads, fp32, 21 and 42; but 200 of 30 tokens, four key heads, 44 and 35.
  const int row_groups = (int)paged_row_groups(sizeof(T) == 2 ? Dt::BF16 : Dt::F32, a.qs.rows * (a.H / a.Hk));
  const int64_t groups = (shares + (a.ks.count * a.Hk * row_groups <= 512 ? a.ks.count : 0)) * a.Hk * row_groups;
  hipLaunchKernelGGL((paged_split_kernel<T, DH, RT>), dim3((unsigned)groups), dim3(256), bytes, s, a, shares, row_groups);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t launch_join(const SoftmaxArgs& a, int rows, int shares, int unit, int least, int times, hipStream_t s) {
  const int each = 256 / (DH < kWave ? DH : kWave) * times;
  const int64_t groups = a.qs.count * a.Hk * ((rows + each - 1) / each);
  hipLaunchKernelGGL((paged_join_kernel<T, DH>), dim3((unsigned)groups), dim3(256), 0, s, a, shares, unit, least, times);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t launch_width(const SoftmaxArgs& a, hipStream_t s) {
  const int rows = (int)a.qs.rows * (a.H / a.Hk);
  const int shares = (int)paged_shares(sizeof(T) == 2 ? Dt::BF16 : Dt::F32, a.ks.count, a.ks.rows, a.Hk, rows);
  hipError_t e;
  if (rows <= 16) e = launch_rows<T, DH, 1>(a, shares, s);
  else if (rows <= 32 || sizeof(T) == 4) e = launch_rows<T, DH, 2>(a, shares, s);
  else if constexpr (sizeof(T) == 2) e = launch_rows<T, DH, 4>(a, shares, s);
  return e != hipSuccess ? e : launch_join<T, DH>(a, rows, shares, PagedLds<T, DH>::KB, kPagedLeast, 1, s);
}

template <typename T>
hipError_t launch_split(const SoftmaxArgs& a, hipStream_t s) {
  return a.d == 32 ? launch_width<T, 32>(a, s) : a.d == 64 ? launch_width<T, 64>(a, s) : launch_width<T, 128>(a, s);
}

}  // namespace

int64_t paged_shares(Dt dt, int64_t count, int64_t room, int64_t Hk, int64_t rows) {
  const int64_t unit = paged_unit(dt), units = count * ((room + unit - 1) / unit);
  const int64_t sets = Hk * paged_row_groups(dt, rows), most = (512 + sets - 1) / sets, full = (units + 3) / 4;
  return full < 1 ? 1 : full < most ? full : most;
}

hipError_t launch_paged_split(Dt dt, const SoftmaxArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_split<__bf16>(a, s) : launch_split<float>(a, s);
}

hipError_t launch_paged_tile_join(const SoftmaxArgs& a, int shares, hipStream_t s) {
  const int rows = (int)a.qs.rows * (a.H / a.Hk);
  return a.d == 64 ? launch_join<__bf16, 64>(a, rows, shares, kPagedTileUnit, 1, 8, s) : launch_join<__bf16, 128>(a, rows, shares, kPagedTileUnit, 1, 8, s);
}

}  // namespace luna
