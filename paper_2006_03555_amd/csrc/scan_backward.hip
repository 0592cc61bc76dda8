// scan_backward.hip - gradients of the selective scan. With a_t = exp(s_t A) and
// e_t = dy_t silu(z_t), per channel and state
//
//   g_t = C_t e_t + q_{t+1},  q_t = a_t g_t        (from the last token back; q_L = dh_out)
//   dC_t = sum_d e_t h_t,  dB_t = sum_d g_t s_t x_t,  dA = sum_t s_t q_t h_{t-1},
//   d(s x)_t = sum_n g_t B_t,  ds_t = sum_n A q_t h_{t-1} + x_t d(s x)_t,  dx_t = s_t d(s x)_t + skip e_t
//
// Every chunk of 128 tokens is a workgroup of its own (or a few tiles of channels of it): a first
// pass takes each chunk's sums of h (from the left) and of q (from the right), a second chains
// them, and the third recomputes h and q inside the chunk from the two states around it. Bound by
// the vector unit: about 25 issue slots per (token, channel, state) in the third pass, 9 in the
// first. dB and dC are sums over channels: the wave's four rows of lanes are joined by exchanging
// halves and rows (each exchange leaves half as many values), and the waves add into LDS in turns,
// wave w at state i + w, so that the order is fixed. What the workgroups of a group of channels
// leave is added up last. Rows reach the lanes through two tiles of LDS, two values to a word in
// bf16, and their gradients leave the same way. B4 L4096 D2048 N16 in bf16: 196 to 216 us, 18 and
// 515 to 530; the vector unit is busy for 91% and 90% of the first and the third.
#include <algorithm>

#include "scan_common.hpp"

namespace favor {
namespace {

constexpr int W = kScanBackTile;   // channels of a tile, one per lane
static_assert(W == 4 * kScanWaves && kLoads<W> == 1, "one unit of a thread");
template <typename T> constexpr bool kBoth = sizeof(T) == 2;   // two tiles hold all four rows

// The rows x, dt, dy and z of a thread's unit (z: x stands in where there is none), by way of two
// tiles to the lanes, where the four come again as often as they are asked for: in 16 bits they
// stay in the tiles, else they are put there in turn.
template <typename T> struct Rows4 {
  RowVec<T, 8> x, dt, dy, z;

  __device__ __forceinline__ void load(const Scan &a, const ScanPlace &p, int64_t t0, const Unit &w) {
    x = get_row<T>(a.x, a.xs, p, t0, w);
    dt = get_row<T>(a.dt, a.dts, p, t0, w);
    dy = get_row<T>(a.dy, a.dys, p, t0, w);
    z = get_row<T>(a.z ? a.z : a.x, a.z ? a.zs : a.xs, p, t0, w);
  }
  __device__ __forceinline__ void put(float *tiles, const Unit &w) const {
    put_pair<W>(tiles, w, x, dt);
    if (kBoth<T>) put_pair<W>(tiles + W * kTok, w, dy, z);
  }
  __device__ __forceinline__ void put_rest(float *tiles, const Unit &w) const {   // for whole workgroups
    if (kBoth<T>) return;
    __syncthreads();
    put_pair<W>(tiles, w, dy, z);
    __syncthreads();
  }
  static __device__ __forceinline__ void get(const float *tiles, int c, int tl, float (&v0)[8], float (&v1)[8]) {
    get_pair<T, W>(tiles, c, tl, v0, v1);
  }
  static __device__ __forceinline__ void get_rest(const float *tiles, int c, int tl, float (&v0)[8], float (&v1)[8]) {
    get_pair<T, W>(tiles + (kBoth<T> ? W * kTok : 0), c, tl, v0, v1);
  }
};
// e = dy silu(z); zeros from token `left` on.
__device__ __forceinline__ void lane_gated(const Scan &a, int left, float (&e)[8], const float (&z)[8]) {
  if (a.z)
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] *= z[j] * sigmoid(z[j]);
  if (left < 8)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= left) e[j] = 0.f;
}

template <typename T> __global__ __launch_bounds__(kScanThreads, 4) void k_scan_parts(Scan a) {
  extern __shared__ __align__(16) float lds[];
  float *tiles = lds, *tb = tiles + 2 * W * kTok, *tc = tb + kStates * kTok;
  float *tA = tc + kStates * kTok, *th = tA + kStates * W, *tq = th + kStates * W;
  const ScanPlace p = scan_place(a, W);
  int tid = threadIdx.x;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, tl = lane % 16;
  const int cl = 4 * wave + lane / 16, c = p.c0 + cl;   // this lane's channel
  const int64_t at_part = ((int64_t)p.b * a.nseg + p.seg) * a.D * a.N;
  const int64_t t0 = (int64_t)p.seg * kTok;
  const int first_n = blockIdx.z * a.sum_states, end_n = min(first_n + a.sum_states, a.N);
  if (t0 >= p.n) {   // no token: nothing is added
    if (blockIdx.z) return;
    for (int i = threadIdx.x; i < min(W, p.cend - p.c0) * a.N; i += kScanThreads)
      a.part[at_part + (int64_t)p.c0 * a.N + i] = a.part_r[at_part + (int64_t)p.c0 * a.N + i] = 0.f;
    if (threadIdx.x < min(W, p.cend - p.c0))
      a.steps[((int64_t)p.b * a.nseg + p.seg) * a.D + p.c0 + threadIdx.x] = 0.f;
    return;
  }
  const Unit w = unit_of<W>(p, t0, 0, tid);
  Rows4<T> rows;
  States<T> low_b, low_c;
  rows.load(a, p, t0, w);
  low_b.load(a.b, a.bs, p, t0, first_n, min(kStates, end_n - first_n), tid);
  low_c.load(a.c, a.cs, p, t0, first_n, min(kStates, end_n - first_n), tid);
  const float bias = a.bias ? a.bias[min(c, p.cend - 1)] : 0.f;
  float s[8], sx[8], e[8], ssum = 0.f;
  for (int n0 = first_n; n0 < end_n; n0 += kStates) {
    const int count = min(kStates, end_n - n0);
    if (n0 > first_n) {
      low_b.load(a.b, a.bs, p, t0, n0, count, tid);
      low_c.load(a.c, a.cs, p, t0, n0, count, tid);
    } else {
      rows.put(tiles, w);
    }
    low_b.put(tb, p, t0, count, tid);
    low_c.put(tc, p, t0, count, tid);
    load_channels<W>(a.A, p, a.N, n0, count, kLog2e, tA, tid);
    __syncthreads();
    if (n0 == first_n) {
      float z[8];
      rows.get(tiles, cl, tl, sx, s);
      rows.put_rest(tiles, w);
      rows.get_rest(tiles, cl, tl, e, z);
      lane_gated(a, lane_left(p, t0, tl), e, z);
      ssum = lane_steps(a, lane_left(p, t0, tl), bias, s, sx);
#pragma unroll
      for (int j = 0; j < 8; ++j) sx[j] *= s[j];
      const float total = row_sum(ssum);
      if (first_n == 0 && tl == 15 && c < p.cend) a.steps[((int64_t)p.b * a.nseg + p.seg) * a.D + c] = total;
    }
    for (int n = 0; n < count; n += 2) {   // two states at once; one behind the last is zeros
      float Bv[2][8], Cv[2][8], S[2], Q[2], P[2], P2[2], h[2] = {}, q[2] = {};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        lane_load(tb + (n + i) * kTok, tl, Bv[i]);
        lane_load(tc + (n + i) * kTok, tl, Cv[i]);
        const float A = tA[(n + i) * W + cl];
        float at[8];
        S[i] = Q[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          at[j] = exp2_hw(s[j] * A);
          S[i] = fmaf(at[j], S[i], sx[j] * Bv[i][j]);
        }
#pragma unroll
        for (int j = 7; j >= 0; --j) Q[i] = at[j] * fmaf(e[j], Cv[i][j], Q[i]);
        P[i] = P2[i] = exp2_hw(ssum * A);
      }
      row_scan2<false>(S[0], P[0], h[0], S[1], P[1], h[1]);
      row_scan2<true>(Q[0], P2[0], q[0], Q[1], P2[1], q[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (tl == 15) th[(n + i) * W + cl] = S[i];
        if (tl == 0) tq[(n + i) * W + cl] = Q[i];
      }
    }
    __syncthreads();
    tid = fresh_thread();
    store_channels<W>(a.part + at_part, p, a.N, n0, count, th, tid);
    store_channels<W>(a.part_r + at_part, p, a.N, n0, count, tq, tid);
  }
}

// Two values in a word, the first in its low half.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const bf16 v[2] = {from_f32<bf16>(lo), from_f32<bf16>(hi)};
  return __builtin_bit_cast(uint32_t, v);
}
// The low or the high halves of eight words as a row.
__device__ __forceinline__ void put_halves(void *base, const Rows &r, const ScanPlace &p, int64_t t0, const Unit &w,
                                           const uint32_t (&d)[8], uint32_t halves) {
  uint4 v;
  v.x = __builtin_amdgcn_perm(d[1], d[0], halves);
  v.y = __builtin_amdgcn_perm(d[3], d[2], halves);
  v.z = __builtin_amdgcn_perm(d[5], d[4], halves);
  v.w = __builtin_amdgcn_perm(d[7], d[6], halves);
  *reinterpret_cast<uint4 *>(row_out<bf16>(base, r, p, t0, w)) = v;
}

// The sums of 16 values over the wave's four rows of lanes; row r keeps values 4 r' .. 4 r' + 3
// of (v: first eight, then the others): rows 0, 1 the first eight's halves, rows 2, 3 the
// others'.
__device__ __forceinline__ f32x4 join_rows(const float (&v)[8], const float (&w)[8]) {
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[j]), __float_as_uint(w[j]), false, false);
    x[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  f32x4 o;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[j]), __float_as_uint(x[j + 4]), false, false);
    o[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return o;
}

// The lane's channel, formed anew: addresses of it are few and far between.
__device__ __forceinline__ int fresh_channel(const ScanPlace &p) {
  const int t = fresh_thread();
  return p.c0 + 4 * (t / 64) + t % 64 / 16;
}

// A workgroup takes a.subs tiles of W channels one after the other, so that dB and dC are
// sums over all of them before they leave it. kGate: there is a z, whose gradient needs y again.
template <typename T, bool kGate> __global__ __launch_bounds__(kScanThreads, 4) void k_scan_backward(Scan a) {
  extern __shared__ __align__(16) float lds[];
  float *tiles = lds, *tb = tiles + 2 * W * kTok, *tc = tb + kStates * kTok;
  float *tlow = tc + kStates * kTok;   // dB, then dC
  float *tA = tlow + 2 * kStates * kTok, *th = tA + kStates * W, *tq = th + kStates * W;
  ScanPlace p = scan_place(a, W * a.subs);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, tl = lane % 16;
  const int cl = 4 * wave + lane / 16;
  const int64_t at_part = ((int64_t)p.b * a.nseg + p.seg) * a.D * a.N;
  const int64_t at_sum = ((int64_t)p.b * a.nseg + p.seg) * a.D;
  const int64_t t0 = (int64_t)p.seg * kTok;
  const bool some = t0 < p.n;
  for (int sub = 0; sub < a.subs && p.c0 < p.cend; ++sub, p.c0 += W) {
    const int c = p.c0 + cl;   // this lane's channel
    const bool channel = c < p.cend;
    if (!some) {
      for (int i = threadIdx.x; i < min(W, p.cend - p.c0) * a.N; i += kScanThreads)
        a.part_a[at_part + (int64_t)p.c0 * a.N + i] = 0.f;
      if (tl == 15 && channel) {
        if (a.dskip) a.part_d[at_sum + c] = 0.f;
        if (a.dbias) a.part_s[at_sum + c] = 0.f;
      }
      const Unit w = unit_of<W>(p, t0, 0, fresh_thread());
      const float none[8] = {};
      if (w.t >= a.L - t0 || w.c >= p.cend) continue;
      put_row<T>(a.dx, a.dxs, p, t0, w, none);
      put_row<T>(a.ddt, a.ddts, p, t0, w, none);
      if (kGate) put_row<T>(a.dz, a.dzs, p, t0, w, none);
    } else {
      // a lane without a channel adds nothing to dB and dC
      const int left = channel ? lane_left(p, t0, tl) : 0;
      float s[8], sx[8], e[8], ds[8], dsx[8], y[8], ssum = 0.f;
      States<T> low_b, low_c;
      Rows4<T> rows;
      int tid = fresh_thread();
      if (sub == 0) {
        low_b.load(a.b, a.bs, p, t0, 0, min(kStates, a.N), tid);
        low_c.load(a.c, a.cs, p, t0, 0, min(kStates, a.N), tid);
        low_b.put(tb, p, t0, min(kStates, a.N), tid);
        low_c.put(tc, p, t0, min(kStates, a.N), tid);
        tid = fresh_thread();
      }
      rows.load(a, p, t0, unit_of<W>(p, t0, 0, tid));
      rows.put(tiles, unit_of<W>(p, t0, 0, tid));   // the last tile's readers are behind a barrier
      for (int n0 = 0; n0 < a.N; n0 += kStates) {
        const int count = min(kStates, a.N - n0);
        if (n0) {
          tid = fresh_thread();
          low_b.load(a.b, a.bs, p, t0, n0, count, tid);
          low_c.load(a.c, a.cs, p, t0, n0, count, tid);
          low_b.put(tb, p, t0, count, tid);
          low_c.put(tc, p, t0, count, tid);
        }
        load_channels<W>(a.A, p, a.N, n0, count, 1.f, tA, tid);
        load_channels<W>(a.part + at_part, p, a.N, n0, count, 1.f, th, tid);
        load_channels<W>(a.part_r + at_part, p, a.N, n0, count, 1.f, tq, tid);
        __syncthreads();
        if (n0 == 0) {
          float z[8], skip = 0.f;
          rows.get(tiles, cl, tl, sx, s);
          rows.put_rest(tiles, unit_of<W>(p, t0, 0, tid));
          rows.get_rest(tiles, cl, tl, e, z);
          lane_gated(a, left, e, z);
          ssum = lane_steps(a, left, a.bias ? a.bias[min(fresh_channel(p), p.cend - 1)] : 0.f, s, sx);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            skip = fmaf(e[j], sx[j], skip);
            sx[j] *= s[j];
            ds[j] = dsx[j] = y[j] = 0.f;
          }
          if (a.dskip) {
            const float total = row_sum(skip);
            if (tl == 15 && channel) a.part_d[at_sum + fresh_channel(p)] = total;
          }
        }
        const int each = (count + kScanWaves - 1) / kScanWaves;   // states of a wave's turn
        for (int turn = 0; turn < kScanWaves; ++turn) {
          for (int k = 0; k < each; ++k) {
            const int n = ((turn + wave) % kScanWaves) * each + k, at_c = n * W + cl;
            float Bv[8], Cv[8], at[8], bx[8], ce[8], dB[8], dC[8];
            lane_load(tb + n * kTok, tl, Bv);
            lane_load(tc + n * kTok, tl, Cv);
            const float A = tA[at_c], A2 = kLog2e * A;
            float h = th[at_c], q = tq[at_c];
            float S = tl == 0 ? h : 0.f, Q = tl == 15 ? q : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              at[j] = exp2_hw(s[j] * A2);
              bx[j] = sx[j] * Bv[j];
              ce[j] = e[j] * Cv[j];
              S = fmaf(at[j], S, bx[j]);
            }
#pragma unroll
            for (int j = 7; j >= 0; --j) Q = at[j] * (ce[j] + Q);
            float P = exp2_hw(ssum * A2), P2 = P;
            row_scan_both(S, P, h, Q, P2, q);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float before = h;
              h = fmaf(at[j], h, bx[j]);
              dC[j] = e[j] * h;
              if (kGate) y[j] = fmaf(Cv[j], h, y[j]);
              bx[j] = before;
            }
            float dA = 0.f;
#pragma unroll
            for (int j = 7; j >= 0; --j) {
              const float g = ce[j] + q;
              q = at[j] * g;
              dB[j] = g * sx[j];
              dsx[j] = fmaf(g, Bv[j], dsx[j]);
              const float u = q * bx[j];
              ds[j] = fmaf(A, u, ds[j]);
              dA = fmaf(s[j], u, dA);
            }
            dA = row_sum(dA);
            if (tl == 15) th[at_c] = dA;   // h before the chunk has been read
            f32x4 low = join_rows(dB, dC);
            f32x4 *to = reinterpret_cast<f32x4 *>(tlow + (lane / 32 * kStates + n) * kTok + 4 * tl +
                                                  (lane / 16 % 2) * 64);
            if (turn || sub) low += *to;
            *to = low;
          }
          __syncthreads();
        }
        tid = fresh_thread();
        if (sub + 1 == a.subs || p.c0 + W >= p.cend) {
          const int n = tid % kStates, first = tid / kStates;
          const int64_t base = ((((int64_t)p.tile * a.B + p.b) * a.L + t0) * a.G + p.g) * a.N + n0 + n;
          const int64_t stride = (int64_t)a.G * a.N;
          const int left = (int)min((int64_t)kTok, p.n - t0);
#pragma unroll
          for (int i = 0; i < kTok * kStates / kScanThreads; ++i) {
            const int t = first + i * (kScanThreads / kStates);
            if (n >= count || t >= left) continue;
            a.part_b[base + t * stride] = tlow[n * kTok + token_at(t)];
            a.part_c[base + t * stride] = tlow[(kStates + n) * kTok + token_at(t)];
          }
        }
        store_channels<W>(a.part_a + at_part, p, a.N, n0, count, th, tid);
        if (n0 + kStates < a.N) __syncthreads();
      }
      // the rows' gradients, where the lanes have the sums; in place of what only the lane reads
      const float bias = a.bias ? a.bias[min(fresh_channel(p), p.cend - 1)] : 0.f;
      const float skip = a.skip ? a.skip[min(fresh_channel(p), p.cend - 1)] : 0.f;
      float x[8], raw[8], dy[8], z[8], dbias = 0.f;
      if (!kBoth<T>) {
        tid = fresh_thread();
        rows.load(a, p, t0, unit_of<W>(p, t0, 0, tid));
        rows.put(tiles, unit_of<W>(p, t0, 0, tid));
        __syncthreads();
      }
      rows.get(tiles, cl, tl, x, raw);
      rows.put_rest(tiles, unit_of<W>(p, t0, 0, tid));
      rows.get_rest(tiles, cl, tl, dy, z);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ds[j] = fmaf(x[j], dsx[j], ds[j]);
        dsx[j] = fmaf(s[j], dsx[j], skip * e[j]);
      }
      if (a.softplus)
#pragma unroll
        for (int j = 0; j < 8; ++j) ds[j] *= softplus_slope(raw[j] + bias, s[j]);
      if (kGate)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float g = sigmoid(z[j]);
          y[j] = dy[j] * fmaf(skip, x[j], y[j]) * (g * fmaf(z[j], 1.f - g, 1.f));
        }
#pragma unroll
      for (int j = 0; j < 8; ++j) dbias += j < left ? ds[j] : 0.f;
      if (a.dbias) {
        dbias = row_sum(dbias);
        if (tl == 15 && channel) a.part_s[at_sum + fresh_channel(p)] = dbias;
      }
      tid = fresh_thread();
      const Unit w = unit_of<W>(p, t0, 0, tid);
      const bool mine = w.t < a.L - t0 && w.c < p.cend;
      if constexpr (kBoth<T>) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(pack_bf16(dsx[j], ds[j]));
        tile_store(tiles, cl, tl, x);
        if (kGate) tile_store(tiles + W * kTok, cl, tl, y);
        __syncthreads();
        uint32_t d[8];
        float o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int at = tile_at(8 * w.u + k, w.t);
          d[k] = w.live ? __float_as_uint(tiles[at]) : 0;
          o[k] = kGate && w.live ? tiles[W * kTok + at] : 0.f;
        }
        if (mine) {
          put_halves(a.dx, a.dxs, p, t0, w, d, 0x05040100u);
          put_halves(a.ddt, a.ddts, p, t0, w, d, 0x07060302u);
          if (kGate) put_row<T>(a.dz, a.dzs, p, t0, w, o);
        }
      } else {
        const auto rows_out = [&](void *dst, const Rows &r, const float *tile) {
          float o[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = w.live ? tile[tile_at(8 * w.u + k, w.t)] : 0.f;
          if (mine) put_row<T>(dst, r, p, t0, w, o);
        };
        tile_store(tiles, cl, tl, dsx);
        tile_store(tiles + W * kTok, cl, tl, ds);
        __syncthreads();
        rows_out(a.dx, a.dxs, tiles);
        rows_out(a.ddt, a.ddts, tiles + W * kTok);
        if (kGate) {
          __syncthreads();
          tile_store(tiles, cl, tl, y);
          __syncthreads();
          rows_out(a.dz, a.dzs, tiles);
        }
      }
      __syncthreads();
    }
  }
}

// dB and dC: over the workgroups of a group of channels.
constexpr int kLowThreads = 256;
template <typename T> __global__ __launch_bounds__(kLowThreads) void k_scan_low(Scan a, int tiles) {
  const int64_t GN = (int64_t)a.G * a.N, per = (int64_t)a.L * GN;
  const int b = blockIdx.y;
  const float *part = blockIdx.z ? a.part_c : a.part_b;
  const Rows &r = blockIdx.z ? a.dcs : a.dbs;
  for (int64_t i = (int64_t)blockIdx.x * kLowThreads + threadIdx.x; i < per; i += (int64_t)gridDim.x * kLowThreads) {
    const int t = (int)(i / GN), gn = (int)(i - t * GN), g = gn / a.N, n = gn - g * a.N;
    float sum = 0.f;
    if (t < clamped_length(a.lengths, b, a.L))
#pragma unroll 8
      for (int k = 0; k < tiles; ++k) sum += part[((int64_t)k * a.B + b) * per + i];
    static_cast<T *>(blockIdx.z ? a.dc : a.db)[b * r.b + g * r.h + t * r.t + n] = from_f32<T>(sum);
  }
}

// dA, dskip and dbias: over sequences and chunks. 64 columns by 16 row lanes, joined in order.
constexpr int kSumCols = 64, kSumLanes = 16;
__global__ __launch_bounds__(kSumCols *kSumLanes) void k_scan_params(Scan a, int rows) {
  __shared__ float part[kSumLanes][kSumCols];
  const int64_t DN = (int64_t)a.D * a.N;
  const int lane = threadIdx.x / kSumCols;
  int64_t col = (int64_t)blockIdx.x * kSumCols + threadIdx.x % kSumCols;
  const float *src = a.part_a;
  float *dst = a.dA;
  int64_t cols = DN;
  if (col >= DN) {
    col -= DN;
    cols = a.D;
    src = a.part_d;
    dst = a.dskip;
    if (col >= a.D) {
      col -= a.D;
      src = a.part_s;
      dst = a.dbias;
    }
  }
  const bool live = col < cols && dst;
  float s = 0.f;
  if (live)
#pragma unroll 8
    for (int r = lane; r < rows; r += kSumLanes) s += src[r * cols + col];
  part[lane][threadIdx.x % kSumCols] = s;
  __syncthreads();
  if (lane || !live) return;
  for (int i = 1; i < kSumLanes; ++i) s += part[i][threadIdx.x];
  dst[col] = s;
}

template <typename K>
hipError_t launch_tiles(K kernel, const Scan &a, int width, int parts, size_t lds, hipStream_t st) {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  const int tiles = a.G * ((a.D / a.G + width - 1) / width), each = kScanBlocks / tiles;
  Scan part = a;
  for (part.seg0 = 0; part.seg0 < a.nseg; part.seg0 += each) {
    const int segments = std::min(each, a.nseg - part.seg0);
    kernel<<<dim3((unsigned)(tiles * segments), a.B, parts), kScanThreads, lds, st>>>(part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_scan_backward_parts(const Scan &a, Dt dt, hipStream_t st) {
  const size_t lds = sizeof(float) * (2 * W * kTok + 2 * kStates * kTok + 3 * kStates * W);
  const int parts = (a.N + a.sum_states - 1) / a.sum_states;
  return dt == Dt::BF16 ? launch_tiles(k_scan_parts<bf16>, a, W, parts, lds, st)
                        : launch_tiles(k_scan_parts<float>, a, W, parts, lds, st);
}

hipError_t launch_scan_backward(const Scan &a, Dt dt, hipStream_t st) {
  const size_t lds = sizeof(float) * (2 * W * kTok + 4 * kStates * kTok + 3 * kStates * W);
  const auto launch = [&](auto kernel) { return launch_tiles(kernel, a, W * a.subs, 1, lds, st); };
  if (dt == Dt::BF16) return a.z ? launch(k_scan_backward<bf16, true>) : launch(k_scan_backward<bf16, false>);
  return a.z ? launch(k_scan_backward<float, true>) : launch(k_scan_backward<float, false>);
}

hipError_t launch_scan_backward_sums(const Scan &a, Dt dt, hipStream_t st) {
  const int64_t low = (int64_t)a.L * a.G * a.N;
  if (low > 0) {
    const int tiles = (a.D / a.G + W * a.subs - 1) / (W * a.subs);
    const dim3 grid((unsigned)std::min<int64_t>(kLowBlocks, (low + kLowThreads - 1) / kLowThreads), a.B, 2);
    if (dt == Dt::BF16) k_scan_low<bf16><<<grid, kLowThreads, 0, st>>>(a, tiles);
    else k_scan_low<float><<<grid, kLowThreads, 0, st>>>(a, tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t cols = (int64_t)a.D * a.N + 2 * a.D;
  k_scan_params<<<(unsigned)((cols + kSumCols - 1) / kSumCols), kSumCols * kSumLanes, 0, st>>>(a, a.B * a.nseg);
  return hipGetLastError();
}

}  // namespace favor
