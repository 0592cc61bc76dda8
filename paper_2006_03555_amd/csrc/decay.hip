// decay.hip - linear attention with a decay per head, in chunks of 64 tokens.
//
//   S_t = a S_{t-1} + k_t v_t^T,   o_t = c q_t^T S_t,   a = exp(log_decay of the head)
//
// A workgroup takes one (batch, head), a slice of the value columns and one segment of
// the sequence, and carries X = S (kd x slice, fp32, in matrix-core accumulators) over
// the segment's chunks. Of one chunk with rows i, j in [0, 64):
//   O   = (Q K^T o D) V + diag(a^(i + 1)) Q X     D_ij = a^(i - j) for j <= i, else 0
//   X  <- a^64 X + K^T diag(a^(63 - j)) V
// Every power has an exponent >= 0 and comes from a table, so a decay of 0 and one of 1
// are the same code and nothing overflows that the formula does not.
//
// The products are taken transposed, so that no result has to change lanes: with X's
// rows (k columns) as accumulator rows, two adjacent tiles of X are the A operand of
// O^T = X^T Q^T in loaded order (accumulator row r of tile nb stands for k column
// perm_col(nb, r)), and the tiles of P^T = K Q^T (rows j, columns i) are in chained order
// the B operand of V^T P^T. Only V^T and K^T need a transpose; bf16 tiles get it from
// the LDS transpose read. Each wave holds all of X's rows for its own value columns and
// builds P^T for itself: two barriers per chunk, both for the staging.
//
// Precision (bf16): X, and all sums, are fp32. The weighted values diag(a^(..)) V enter
// K^T V as three bf16 terms (24 bits: exact), so X is as exact as fp32 inputs would make
// it; X enters Q X as two terms and the pair weights P as one, one rounding of 2^-9 each
// beside the output's own.
#include "decay.hpp"
#include "tile_common.hpp"

namespace favor {
namespace {

constexpr int kChunkT = 64;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Rows of an LDS tile are padded by 16 bytes, so that 16 rows at one column fall into
// different banks.
template <typename T> constexpr int kPad = 16 / (int)sizeof(T);

// Eight fp32 values as N operand fragments whose sum they are: all but the last term
// truncated (no term of a finite value overflows, and the remainder is exact), the last
// rounded.
template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&f)[N]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int n = 0; n + 1 < N; ++n) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned a = __float_as_uint(r[2 * i]), b = __float_as_uint(r[2 * i + 1]);
      w[i] = __builtin_amdgcn_perm(b, a, 0x07060302);
      r[2 * i] -= __uint_as_float(a & 0xffff0000u);
      r[2 * i + 1] -= __uint_as_float(b & 0xffff0000u);
    }
    f[n] = __builtin_bit_cast(bf16x8, w);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[N - 1][i] = (bf16)r[i];
}
template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], f32x8 (&f)[N]) {
  static_assert(N == 1, "fp32 operands are whole");
#pragma unroll
  for (int i = 0; i < 8; ++i) f[0][i] = x[i];
}
template <typename T> constexpr int kSumTerms = sizeof(T) == 2 ? 3 : 1;
template <typename T> constexpr int kStateTerms = sizeof(T) == 2 ? 2 : 1;

// Operand fragment of the transpose of an LDS tile [64][ld]: the lane's row (lane % 16 =
// 4 q + r) is tile column c0 + step q + r, its k positions tokens 32 m + (chained order).
__device__ __forceinline__ bf16x8 load_tr(const bf16 *tile, int ld, int m, int c0, int step) {
  const int l = lane_id();
  const bf16 *p = tile + (32 * m + 4 * (l >> 4) + ((l >> 2) & 3)) * ld + c0 + step * (l & 3);
  using lds4 = __attribute__((address_space(3))) s16x4;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p + 16 * ld));
  struct Two { s16x4 a, b; };
  return __builtin_bit_cast(bf16x8, Two{lo, hi});
}
__device__ __forceinline__ f32x8 load_tr(const float *tile, int ld, int m, int c0, int step) {
  const int l = lane_id();
  const float *p = tile + (32 * m + 4 * (l >> 4)) * ld + c0 + step * ((l >> 2) & 3) + (l & 3);
  f32x8 f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = p[(16 * (i >> 2) + (i & 3)) * ld];
  return f;
}

// A chunk's rows on their way from global memory to an LDS tile [64][W + pad]: 16-byte
// units, zero past the chunk's n rows and the tensor's `width` columns.
template <typename T, int W, int NT>
struct Staged {
  static constexpr int kPer = 16 / (int)sizeof(T);
  static constexpr int kUnits = W / kPer;
  static constexpr int N = kChunkT * kUnits / NT;
  static_assert(kChunkT * kUnits % NT == 0, "whole passes");
  u32x4 r[N];
  __device__ __forceinline__ void load(const T *base, int64_t stride, int n, int width) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int u = threadIdx.x + k * NT;
      const int row = u / kUnits, col = u % kUnits * kPer;
      r[k] = row < n && col < width
                 ? *reinterpret_cast<const u32x4 *>(base + row * stride + col)
                 : u32x4{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ void store(T *tile) const {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int u = threadIdx.x + k * NT;
      const int row = u / kUnits, col = u % kUnits * kPer;
      *reinterpret_cast<u32x4 *>(tile + row * (W + kPad<T>) + col) = r[k];
    }
  }
};

// a^e for e = 0 .. 64 as a sum of two floats: a chunk's a^64 meets X thousands of times,
// and one float's rounding would be raised to that power.
struct Powers {
  float hi[kChunkT + 1], lo[kChunkT + 1];
};
__device__ __forceinline__ void power(double g, int e, float &hi, float &lo) {
  const double d = e == 0 ? 1.0 : exp(g * e);   // 0^0 = 1
  hi = (float)d;
  lo = isfinite(hi) ? (float)(d - hi) : 0.f;
}
__device__ __forceinline__ void fill_powers(Powers &p, float g) {
  if (threadIdx.x <= kChunkT) power(g, threadIdx.x, p.hi[threadIdx.x], p.lo[threadIdx.x]);
}

// What a workgroup works on.
struct Item {
  int bh, b, h, slice, seg;
  int len;    // tokens of the sequence
  int first;  // the segment's first row (in the scan's order)
  int n;      // its tokens
};

__device__ __forceinline__ Item item_of(const DecayScan &a, int id, int nslice, int nseg) {
  Item it;
  it.slice = id % nslice;
  id /= nslice;
  it.seg = id % nseg;
  it.bh = id / nseg;
  it.b = it.bh / a.H;
  it.h = it.bh % a.H;
  it.len = a.lengths ? min(max(a.lengths[it.b], 0), a.L) : a.L;
  it.first = it.seg * a.seg_len;
  it.n = min(max(it.len - it.first, 0), a.seg_len);
  return it;
}
// The segment of the sequence's last token: it ends with X_n.
__device__ __forceinline__ int last_seg(const DecayScan &a, int len) {
  return len == 0 ? 0 : (len - 1) / a.seg_len;
}

// Start of row r of the scan's order, and the step to the next row.
template <typename T>
__device__ __forceinline__ const T *row_ptr(const void *p, const Rows &s, const Item &it,
                                            bool reverse, int r) {
  const int64_t t = reverse ? it.len - 1 - r : r;
  return static_cast<const T *>(p) + it.b * s.b + it.h * s.h + t * s.t;
}

// X's tiles of one wave: [k rows / 16][value columns / 16].
template <int KD, int NCT>
struct State {
  f32x4 x[KD / 16][NCT];
};

// The first value column of a wave's columns, and the place of lane column c (0 .. 15) of
// tile ct among them: with two tiles a lane's rows of both are eight consecutive columns.
template <int NCT>
__device__ __forceinline__ int value_col(int ct, int c) {
  return NCT == 2 ? perm_col(ct, c) : c;
}

// Slice partials in the workspace: the accumulators as they are, 16 bytes per lane.
template <int KD, int NW, int NCT>
__device__ __forceinline__ size_t part_at(const DecayScan &a, int bh, int seg, int slice, int nb,
                                          int ct) {
  const int nslice = (a.vd + 16 * NW * NCT - 1) / (16 * NW * NCT);
  const size_t x = ((size_t)bh * (a.nseg - 1) + seg) * nslice + slice;
  return x * (KD * 16 * NW * NCT) +
         4 * ((size_t)(((threadIdx.x >> 6) * (KD / 16) + nb) * NCT + ct) * 64 + lane_id());
}

template <int KD, int NW, int NCT>
__device__ __forceinline__ void load_state(const DecayScan &a, const Item &it,
                                           State<KD, NCT> &s) {
  const int w = threadIdx.x >> 6, l = lane_id(), g = l >> 4, c = l & 15;
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb)
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      f32x4 x{0.f, 0.f, 0.f, 0.f};
      if (it.seg > 0) {
        x = *reinterpret_cast<const f32x4 *>(
            a.part + part_at<KD, NW, NCT>(a, it.bh, it.seg - 1, it.slice, nb, ct));
      } else if (a.x_in) {
        const int vc = 16 * NW * NCT * it.slice + 16 * NCT * w + value_col<NCT>(ct, c);
        const int kc = perm_col(nb, 4 * g);
        if (vc < a.vd && kc < a.kd) {
          const float *p = a.x_in + (size_t)it.bh * a.kd * a.vd;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[j] = a.x_t ? p[(size_t)vc * a.kd + kc + j] : p[(size_t)(kc + j) * a.vd + vc];
        }
      }
      s.x[nb][ct] = x;
    }
}

template <int KD, int NW, int NCT>
__device__ __forceinline__ void store_state(const DecayScan &a, const Item &it,
                                            const State<KD, NCT> &s) {
  const int w = threadIdx.x >> 6, l = lane_id(), g = l >> 4, c = l & 15;
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb)
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      const int vc = 16 * NW * NCT * it.slice + 16 * NCT * w + value_col<NCT>(ct, c);
      const int kc = perm_col(nb, 4 * g);
      if (vc < a.vd && kc < a.kd) {
        float *p = a.x_out + (size_t)it.bh * a.kd * a.vd;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          p[a.x_t ? (size_t)vc * a.kd + kc + j : (size_t)(kc + j) * a.vd + vc] = s.x[nb][ct][j];
      }
    }
}

// X <- a^n X + sum_scale K^T diag(a^(n - shift - j)) V of a chunk with n tokens. vt: the
// wave's value columns transposed, tokens in chained order.
template <typename T, int KD, int NCT>
__device__ __forceinline__ void update_state(State<KD, NCT> &s, const T *Ks,
                                             const typename Mma<T>::frag (&vt)[NCT][2],
                                             const Powers &pw, int n, int shift,
                                             float sum_scale) {
  using P = Mma<T>;
  constexpr int N = kSumTerms<T>;
  const int g = lane_id() >> 4;
  typename P::frag vw[2][NCT][N];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    float wt[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = n - shift - (32 * m + 16 * (i >> 2) + 4 * g + (i & 3));
      wt[i] = e >= 0 ? pw.hi[max(e, 0)] * sum_scale : 0.f;
    }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = to_f32(vt[ct][m][i]) * wt[i];
      split8<N>(x, vw[m][ct]);
    }
  }
  // The chunk's sum starts from zero and joins X in one rounded step: the bf16 matrix
  // core cuts off what its accumulator cannot hold, always downwards, which over the
  // chunks of a long memory (8192 positive terms, a = 1) put X off by 6e-6.
  const float hi = pw.hi[n], lo = pw.lo[n];
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb) {
    f32x4 u[NCT];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) u[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const auto kt = load_tr(Ks, KD + kPad<T>, m, perm_col(nb, 0), 8);
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int t = N - 1; t >= 0; --t) u[ct] = P::mma(kt, vw[m][ct][t], u[ct]);
    }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = s.x[nb][ct][j];
        s.x[nb][ct][j] = fmaf(x, hi, fmaf(x, lo, u[ct][j]));
      }
  }
}

template <typename T, int NW, int NCT>
__device__ __forceinline__ void load_values(const T *Vs, typename Mma<T>::frag (&vt)[NCT][2]) {
  const int w = threadIdx.x >> 6;
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int m = 0; m < 2; ++m)
      vt[ct][m] = load_tr(Vs, 16 * NW * NCT + kPad<T>, m,
                          16 * NCT * w + value_col<NCT>(ct, 0), NCT == 2 ? 8 : 4);
}

// The sums of one segment of 64 * chunks tokens, from X = 0.
template <typename T, int KD, int NW, int NCT>
__global__ __launch_bounds__(64 * NW) void k_decay_sums(DecayScan a) {
  constexpr int NT = 64 * NW, VS = 16 * NW * NCT;
  __shared__ __align__(16) T Ks[kChunkT * (KD + kPad<T>)];
  __shared__ __align__(16) T Vs[kChunkT * (VS + kPad<T>)];
  __shared__ Powers pw;
  const int nslice = (a.vd + VS - 1) / VS;
  const Item it = item_of(a, xcd_item(blockIdx.x, gridDim.x), nslice, a.nseg - 1);
  if (it.seg >= last_seg(a, it.len)) return;   // X_n comes from the scan
  fill_powers(pw, a.log_decay[it.h]);
  const int v0 = VS * it.slice;
  const int64_t sgn = a.reverse ? -1 : 1;
  State<KD, NCT> s;
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb)
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) s.x[nb][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  Staged<T, KD, NT> kr;
  Staged<T, VS, NT> vr;
  const auto fetch = [&](int c) {
    const int r = it.first + c, n = min(kChunkT, it.n - c);
    kr.load(row_ptr<T>(a.k, a.ks, it, a.reverse, r), sgn * a.ks.t, n, a.kd);
    vr.load(row_ptr<T>(a.v, a.vs, it, a.reverse, r) + v0, sgn * a.vs.t, n, a.vd - v0);
  };
  fetch(0);
  for (int c = 0; c < it.n; c += kChunkT) {
    kr.store(Ks);
    vr.store(Vs);
    __syncthreads();
    if (c + kChunkT < it.n) fetch(c + kChunkT);
    typename Mma<T>::frag vt[NCT][2];
    load_values<T, NW, NCT>(Vs, vt);
    update_state<T, KD, NCT>(s, Ks, vt, pw, kChunkT, a.shift, a.sum_scale);
    __syncthreads();
  }
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb)
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
      *reinterpret_cast<f32x4 *>(
          a.part + part_at<KD, NW, NCT>(a, it.bh, it.seg, it.slice, nb, ct)) = s.x[nb][ct];
}

// part of a head's segments: X before segment s + 1 = a^seg_len (X before s) + sums of s,
// one accumulator quadruple per thread, in the slices' own order.
template <int KD, int NW, int NCT>
__global__ __launch_bounds__(256) void k_decay_prefix(DecayScan a) {
  constexpr int VS = 16 * NW * NCT, Q = KD * VS / 4;
  const int nslice = (a.vd + VS - 1) / VS;
  const int e = (blockIdx.x % (Q / 256)) * 256 + threadIdx.x;
  const int id = blockIdx.x / (Q / 256);
  const Item it = item_of(a, id, nslice, 1);
  const int last = last_seg(a, it.len);
  if (last == 0) return;
  const int l = e & 63, g = l >> 4, c = l & 15;
  const int ct = (e >> 6) % NCT, nb = (e >> 6) / NCT % (KD / 16), w = (e >> 6) / NCT / (KD / 16);
  f32x4 x{0.f, 0.f, 0.f, 0.f};
  if (a.x_in) {
    const int vc = VS * it.slice + 16 * NCT * w + value_col<NCT>(ct, c);
    const int kc = perm_col(nb, 4 * g);
    if (vc < a.vd && kc < a.kd) {
      const float *p = a.x_in + (size_t)it.bh * a.kd * a.vd;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[j] = a.x_t ? p[(size_t)vc * a.kd + kc + j] : p[(size_t)(kc + j) * a.vd + vc];
    }
  }
  float hi, lo;
  power(a.log_decay[it.h], a.seg_len, hi, lo);
  f32x4 *p = reinterpret_cast<f32x4 *>(a.part) +
             ((size_t)it.bh * (a.nseg - 1) * nslice + it.slice) * Q + e;
  for (int s = 0; s < last; ++s, p += (size_t)nslice * Q) {
    const f32x4 u = *p;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = fmaf(x[j], hi, fmaf(x[j], lo, u[j]));
    *p = x;
  }
}

template <typename T, int KD, int NW, int NCT>
__global__ __launch_bounds__(64 * NW) void k_decay_scan(DecayScan a) {
  using P = Mma<T>;
  using frag = typename P::frag;
  constexpr int NT = 64 * NW, VS = 16 * NW * NCT, NP = KD / 32, LD = KD + kPad<T>;
  __shared__ __align__(16) T Qs[kChunkT * LD];
  __shared__ __align__(16) T Ks[kChunkT * LD];
  __shared__ __align__(16) T Vs[kChunkT * (VS + kPad<T>)];
  __shared__ Powers pw;
  const int nslice = (a.vd + VS - 1) / VS;
  const Item it = item_of(a, xcd_item(blockIdx.x, gridDim.x), nslice, a.nseg);
  const int w = threadIdx.x >> 6, l = lane_id(), g = l >> 4, c16 = l & 15;
  const int v0 = VS * it.slice;
  const int64_t sgn = a.reverse ? -1 : 1;
  fill_powers(pw, a.log_decay[it.h]);
  State<KD, NCT> s;
  load_state<KD, NW, NCT>(a, it, s);
  Staged<T, KD, NT> qr, kr;
  Staged<T, VS, NT> vr;
  const auto fetch = [&](int c) {
    const int r = it.first + c, n = min(kChunkT, it.n - c);
    qr.load(row_ptr<T>(a.q, a.qs, it, a.reverse, r), sgn * a.qs.t, n, a.kd);
    kr.load(row_ptr<T>(a.k, a.ks, it, a.reverse, r), sgn * a.ks.t, n, a.kd);
    vr.load(row_ptr<T>(a.v, a.vs, it, a.reverse, r) + v0, sgn * a.vs.t, n, a.vd - v0);
  };
  if (it.n > 0) fetch(0);
  for (int c = 0; c < it.n; c += kChunkT) {
    const int n = min(kChunkT, it.n - c);
    qr.store(Qs);
    kr.store(Ks);
    vr.store(Vs);
    __syncthreads();
    if (c + kChunkT < it.n) fetch(c + kChunkT);

    // X^T Q^T
    f32x4 o[4][NCT];
#pragma unroll
    for (int ib = 0; ib < 4; ++ib)
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) o[ib][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      frag xf[NCT][kStateTerms<T>];
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] = s.x[2 * p][ct][j];
          x[4 + j] = s.x[2 * p + 1][ct][j];
        }
        split8<kStateTerms<T>>(x, xf[ct]);
      }
#pragma unroll
      for (int ib = 0; ib < 4; ++ib) {
        const frag qf = load_frag<T>(&Qs[(16 * ib + c16) * LD + 32 * p + 8 * g]);
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
          for (int t = kStateTerms<T> - 1; t >= 0; --t) o[ib][ct] = P::mma(xf[ct][t], qf, o[ib][ct]);
      }
    }
#pragma unroll
    for (int ib = 0; ib < 4; ++ib) {
      const float f = pw.hi[16 * ib + c16 + a.shift] * a.row_scale;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[ib][ct][j] *= f;
    }

    // + V^T (D o K Q^T), the pairs j <= i
    frag vt[NCT][2];
    load_values<T, NW, NCT>(Vs, vt);
#pragma unroll
    for (int ib = 0; ib < 4; ++ib) {
      frag qf[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p)
        qf[p] = load_frag<T>(&Qs[(16 * ib + c16) * LD + 32 * p + 8 * g]);
#pragma unroll
      for (int m = 0; m <= ib / 2; ++m) {
        f32x4 pt[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int jb = 2 * m + h;
          f32x4 x{0.f, 0.f, 0.f, 0.f};
          if (jb <= ib) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
              x = P::mma(load_frag<T>(&Ks[(16 * jb + c16) * LD + 32 * p + 8 * g]), qf[p], x);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int e = 16 * (ib - jb) + c16 - 4 * g - j;
              x[j] = e >= 0 ? x[j] * (pw.hi[max(e, 0)] * a.pair_scale) : 0.f;
            }
          }
          pt[h] = x;
        }
        const frag pf = P::pack(pt[0], pt[1]);
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) o[ib][ct] = P::mma(vt[ct][m], pf, o[ib][ct]);
      }
      const int i = 16 * ib + c16;
      if (i < n) {
        T *op = const_cast<T *>(row_ptr<T>(a.o, a.os, it, a.reverse, it.first + c + i));
        const int vc = v0 + 16 * NCT * w + 4 * NCT * g;
        if (vc < a.vd) {
          if constexpr (NCT == 2) store8(op + vc, o[ib][0], o[ib][1]);
          else store4(op + vc, o[ib][0]);
        }
      }
    }
    update_state<T, KD, NCT>(s, Ks, vt, pw, n, a.shift, a.sum_scale);
    __syncthreads();
  }

  if (a.x_out && it.seg == last_seg(a, it.len)) store_state<KD, NW, NCT>(a, it, s);
  // the rows of the segment past the sequence's end
  const int end = min(a.L, it.first + a.seg_len);
  constexpr int kPer = 16 / (int)sizeof(T), kUnits = VS / kPer;
  for (int r = it.first + it.n + threadIdx.x / kUnits; r < end; r += NT / kUnits) {
    const int col = v0 + threadIdx.x % kUnits * kPer;
    if (col < a.vd)
      *reinterpret_cast<u32x4 *>(static_cast<T *>(a.o) + it.b * a.os.b + it.h * a.os.h +
                                 r * a.os.t + col) = u32x4{0, 0, 0, 0};
  }
}

enum class Which { Sums, Prefix, Scan };

template <typename T, int KD, int NW, int NCT>
hipError_t launch(const DecayScan &a, Which which, hipStream_t st) {
  const int nslice = decay_slices(a.kd, a.vd);
  if (which == Which::Sums) {
    k_decay_sums<T, KD, NW, NCT><<<a.BH * (a.nseg - 1) * nslice, 64 * NW, 0, st>>>(a);
  } else if (which == Which::Prefix) {
    k_decay_prefix<KD, NW, NCT>
        <<<a.BH * nslice * (KD * 16 * NW * NCT / 4 / 256), 256, 0, st>>>(a);
  } else {
    k_decay_scan<T, KD, NW, NCT><<<a.BH * a.nseg * nslice, 64 * NW, 0, st>>>(a);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t dispatch(const DecayScan &a, Which which, hipStream_t st) {
  const bool wide = decay_slice(a.kd, a.vd) == 128;
  if (a.kd <= 64) return wide ? launch<T, 64, 4, 2>(a, which, st) : launch<T, 64, 2, 2>(a, which, st);
  if (a.kd <= 128)
    return wide ? launch<T, 128, 4, 2>(a, which, st) : launch<T, 128, 2, 2>(a, which, st);
  return launch<T, 256, 4, 1>(a, which, st);
}

hipError_t dispatch(const DecayScan &a, Dt dt, Which which, hipStream_t st) {
  return dt == Dt::BF16 ? dispatch<bf16>(a, which, st) : dispatch<float>(a, which, st);
}

}  // namespace

// 64 columns for narrow values, and with more than 128 k columns, whose X would not
// leave room for the operands in registers.
int decay_slice(int kd, int vd) { return kd > 128 || vd <= 64 ? 64 : 128; }

hipError_t launch_decay_sums(const DecayScan &a, Dt dt, hipStream_t st) {
  return dispatch(a, dt, Which::Sums, st);
}
hipError_t launch_decay_prefix(const DecayScan &a, hipStream_t st) {
  return dispatch(a, Dt::F32, Which::Prefix, st);
}
hipError_t launch_decay_scan(const DecayScan &a, Dt dt, hipStream_t st) {
  return dispatch(a, dt, Which::Scan, st);
}

}  // namespace favor
