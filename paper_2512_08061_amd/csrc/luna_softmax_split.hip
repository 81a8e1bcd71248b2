// luna_softmax_split.hip -- softmax attention of few queries over long keys (the next tokens of sequences
// with a cache): what bounds it is reading the keys and values once.
//
// The query rows of a key head, m tokens of its H / Hk heads each, are one operand of up to RT tiles of 16, so
// that the cache is read once for the whole group.  The keys of a sequence are cut in pieces of
// kSplitKeys, a workgroup each: its waves take blocks of a piece in turn, each with a running maximum,
// sum and unnormalised output of its own, which are joined through LDS.  Keys go from memory straight to
// the matrix operand (no other wave reads them); values pass through LDS, in the wave's own part of it, to
// be read transposed, so waves never wait for one another before the join.  A second launch joins the
// pieces of every row.  Sums are taken in a fixed order.  Measured: the next token of 32 sequences with 125000 cached
// tokens in all, 16 heads of 128 on 4: 61 us for 257 MB (4.2 TB/s), and 6 us for the join.
#include "luna_softmax.hpp"

namespace luna {

namespace {

template <typename T>
constexpr int kSplitBlock = sizeof(T) == 2 ? 64 : 32;  // keys of a wave at a time

template <typename T, int DH>
struct SplitLds {
  static constexpr int KB = kSplitBlock<T>, P = DH + (sizeof(T) == 2 ? 16 : 4);
  union {
    T v[4][KB][P];
    float o[4][16][DH + 1];  // at the join: a row tile of every wave
  };
  float top[4][16], sum[4][16];
};

template <typename T, int DH, int RT>
__global__ __launch_bounds__(256) void softmax_split_kernel(SoftmaxArgs a) {
  using Lds = SplitLds<T, DH>;
  constexpr int KB = Lds::KB, P = Lds::P, KT = KB / 16, CT = DH / 16, DT = DH / 32, esz = (int)sizeof(T), E = 16 / esz;
  constexpr int VL = KB * DH / E / kWave;  // 16-byte pieces of a block's values per lane
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const int lane = threadIdx.x % kWave, wave = wave_id(), g = lane / 16, c = lane % 16;
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
  const SeqPiece sk = seq_piece(a.ks, slot, kSplitKeys);
  if (sk.seq < 0) return;
  const SeqPiece sq = seq_of(a.qs, sk.seq);
  const int group = a.H / a.Hk, rows = (int)a.qs.rows * group, shift = sk.len - sq.len;
  const bool pk = a.ks.offsets != nullptr;
  const int begin = sk.index * kSplitKeys, end = min(sk.len, begin + kSplitKeys);

  Frag<T> qf[RT][DT];
  int last[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = 16 * rt + c, t = r / group;
    const bool in = r < rows && t < sq.len;
    last[rt] = in ? t + shift : -1;
    const T* q = reinterpret_cast<const T*>(a.q.data) + (in ? sk.seq * a.q.seq + (hk * group + r % group) * a.q.head + t * a.q.row : 0);
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      if (in) load8(qf[rt][i], q + 32 * i + 8 * g);
      else qf[rt][i].zero();
    }
  }
  const float scale = a.scale * kLog2e;
  f32x4 o[RT][CT];
  float top[RT], sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    top[rt] = -__builtin_inff();
    sum[rt] = 0.0f;
#pragma unroll
    for (int i = 0; i < CT; ++i) o[rt][i] = zero4();
  }

  for (int k0 = begin + KB * wave; k0 < end; k0 += 4 * KB) {
    const int kn = min(KB, end - k0);
    const Buf bk = buffer(seq_row(a.k, sk, pk, hk, k0, esz), (int)(((kn - 1) * a.k.row + DH) * esz));
    const Buf bv = buffer(seq_row(a.v, sk, pk, hk, k0, esz), (int)(((kn - 1) * a.v.row + DH) * esz));
    Frag<T> kf[KT][DT];
    i32x4 vr[VL];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int r = 16 * kt + c;
        buf_load8(kf[kt][i], bk, r < kn ? (r * (int)a.k.row + 32 * i + 8 * g) * esz : kPastEnd);
      }
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int idx = lane + kWave * i, r = idx / (DH / E), col = (idx % (DH / E)) * E;
      vr[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                            bv, r < kn ? (r * (int)a.v.row + col) * esz : kPastEnd, 0, 0));
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
    wave_lds_fence();  // the block before has been read
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int idx = lane + kWave * i;
      *reinterpret_cast<i32x4*>(&l.v[wave][idx / (DH / E)][(idx % (DH / E)) * E]) = vr[i];
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
          const int key = 16 * kt + 4 * g + j;
          const float x = s[rt][kt][j] * scale;
          s[rt][kt][j] = key < kn && k0 + key <= last[rt] ? x : -__builtin_inff();
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

  // the four waves' rows joined: of every piece the maximum, the sum and the unnormalised output
  float* part = a.parts + ((int64_t)slot * a.Hk + hk) * rows * (DH + 2);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float whole = groups_sum(sum[rt]);
    __syncthreads();
    if (g == 0) {
      l.top[wave][c] = top[rt];
      l.sum[wave][c] = whole;
    }
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) l.o[wave][c][16 * i + 4 * g + j] = o[rt][i][j];
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * (DH + 1); idx += 256) {
      const int r = idx / (DH + 1), x = idx % (DH + 1);
      if (16 * rt + r >= rows) continue;
      const float most = fmaxf(fmaxf(l.top[0][r], l.top[1][r]), fmaxf(l.top[2][r], l.top[3][r]));
      const float base = most == -__builtin_inff() ? 0.0f : most;
      float y = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) y = fmaf(exp2_raw(l.top[w][r] - base), x < DH ? l.o[w][r][x] : l.sum[w][r], y);
      part[(16 * rt + r) * (DH + 2) + x] = y;
      if (x == DH) part[(16 * rt + r) * (DH + 2) + DH + 1] = most;
    }
  }
}

// Rows of all pieces of a sequence joined; rows that see no key, and sequences without any, as zeros.
template <typename T, int DH>
__global__ __launch_bounds__(DH) void softmax_join_kernel(SoftmaxArgs a) {
  const int group = a.H / a.Hk, rows = (int)a.qs.rows * group;
  const int r = blockIdx.x % rows, hk = (blockIdx.x / rows) % a.Hk, b = blockIdx.x / rows / a.Hk;
  const int head = hk * group + r % group, t = r / group, x = threadIdx.x;
  const SeqPiece sq = seq_of(a.qs, b), sk = seq_of(a.ks, b);
  if (t >= sq.len) return;
  const int pieces = (sk.len + kSplitKeys - 1) / kSplitKeys;
  const int64_t slot = a.ks.offsets ? sk.first / kSplitKeys + b : b * ((a.ks.rows + kSplitKeys - 1) / kSplitKeys);
  const int64_t step = (int64_t)a.Hk * rows * (DH + 2);
  const float* part = a.parts + ((slot * a.Hk + hk) * rows + r) * (DH + 2);
  // the pieces' maxima and factors a thread each; then their rows, whose loads do not wait for one another
  __shared__ float w[DH], part_sum[DH];
  float most = -__builtin_inff();
  for (int p = x; p < pieces; p += DH) most = fmaxf(most, part[p * step + DH + 1]);
  w[x] = most;
  __syncthreads();
  for (int i = 0; i < min(pieces, DH); ++i) most = fmaxf(most, w[i]);
  const float base = most == -__builtin_inff() ? 0.0f : most;
  float y = 0.0f, sum = 0.0f;
  for (int p0 = 0; p0 < pieces; p0 += DH) {
    const int n = min(DH, pieces - p0);
    __syncthreads();  // the weights before are no longer read
    if (x < n) {
      w[x] = exp2_raw(part[(p0 + x) * step + DH + 1] - base);
      part_sum[x] = w[x] * part[(p0 + x) * step + DH];
    }
    __syncthreads();
#pragma unroll 8
    for (int i = 0; i < n; ++i) {
      y = fmaf(w[i], part[(p0 + i) * step + x], y);
      sum += part_sum[i];
    }
  }
  const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
  if (a.lse && x == 0) a.lse[seq_num(a.qs, sq, a.H, head, t)] = (most + log2f(sum)) * kLn2;
  if (__syncthreads_or(not_finite(y * inv))) {  // (uniform)
    constexpr int LANES = DH < kWave ? DH : kWave;
    if (softmax_odd_values<T, DH, LANES>(a, sk, hk, t + sk.len - sq.len + 1, sk.len)) {
      if (x < kWave) softmax_row<T, DH, LANES>(a, sq, sk, head, t);
      return;
    }
  }
  reinterpret_cast<T*>(seq_row(a.o, sq, false, head, t, (int)sizeof(T)))[x] = (T)(y * inv);
}

template <typename T, int DH, int RT>
hipError_t launch_rows(const SoftmaxArgs& a, hipStream_t s) {
  constexpr int bytes = (int)sizeof(SplitLds<T, DH>);
  const hipError_t e = allow_lds<softmax_split_kernel<T, DH, RT>>(bytes);
  if (e != hipSuccess) return e;
  const int64_t slots = seq_slots(a.ks, kSplitKeys);
  if (slots > 0)
    hipLaunchKernelGGL((softmax_split_kernel<T, DH, RT>), dim3((unsigned)(slots * a.Hk)), dim3(256), bytes, s, a);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t launch_width(const SoftmaxArgs& a, hipStream_t s) {
  const int rows = (int)a.qs.rows * (a.H / a.Hk);
  const hipError_t e = rows <= 16 ? launch_rows<T, DH, 1>(a, s) : rows <= 32 ? launch_rows<T, DH, 2>(a, s) : launch_rows<T, DH, 4>(a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((softmax_join_kernel<T, DH>), dim3((unsigned)(a.qs.count * a.Hk * rows)), dim3(DH), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_split(const SoftmaxArgs& a, hipStream_t s) {
  return a.d == 32 ? launch_width<T, 32>(a, s) : a.d == 64 ? launch_width<T, 64>(a, s) : launch_width<T, 128>(a, s);
}

}  // namespace

hipError_t launch_softmax_split(Dt dt, const SoftmaxArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_split<__bf16>(a, s) : launch_split<float>(a, s);
}

}  // namespace luna
