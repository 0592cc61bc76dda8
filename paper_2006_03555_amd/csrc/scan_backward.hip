// scan_backward.hip - gradients of the selective scan. With a_t = exp(s_t A) and
// e_t = dy_t silu(z_t), per channel and state
//
//   g_t = C_t e_t + q_{t+1},  q_t = a_t g_t        (from the last token back; q_L = dh_out)
//   dC_t = sum_d e_t h_t,  dB_t = sum_d g_t s_t x_t,  dA = sum_t s_t q_t h_{t-1},
//   d(s x)_t = sum_n g_t B_t,  ds_t = sum_n A q_t h_{t-1} + x_t d(s x)_t,  dx_t = s_t d(s x)_t + skip e_t
//
// Every chunk of 128 tokens is a workgroup of its own: a first pass takes each chunk's sums of
// h (from the left) and of q (from the right), a second chains them, and the third recomputes
// h and q inside the chunk from the two states around it. Bound by the vector unit: about 23
// issue slots per (token, channel, state) in the third pass. dB and dC are sums over channels: a
// lane adds its two, the wave's four rows are joined by exchanging halves and rows (each exchange
// leaves half as many values), and the waves add into LDS in turns, wave w at state i + w, so
// that the order is fixed. What the workgroups of a group of channels leave is added up last.
#include "scan_common.hpp"

namespace favor {
namespace {

// Channels per lane and workgroup of the first pass and of the third.
constexpr int kCh = 2, W = 4 * kScanWaves * kCh;
constexpr int kTile = kScanBackTile;
static_assert(kTile == 4 * kScanWaves, "one channel per lane");

// dy and z of a thread's units as they lie in memory; then e = dy silu(z). Zeros behind the
// sequence and the group.
template <typename T, int kWidth> struct Gated {
  RowVec<T, 8> dy[kLoads<kWidth>], z[kLoads<kWidth>];

  __device__ __forceinline__ void load(const Scan &a, const ScanPlace &p, int64_t t0, int tid) {
#pragma unroll
    for (int i = 0; i < kLoads<kWidth>; ++i) {
      const Unit w = unit_of<kWidth>(p, t0, i, tid);
      dy[i] = get_row<T>(a.dy, a.dys, p, t0, w);
      if (a.z) z[i] = get_row<T>(a.z, a.zs, p, t0, w);
    }
  }
  __device__ __forceinline__ void get(const Scan &a, const Unit &w, int i, float *e) const {
    float g[8];
    dy[i].get(e);
    if (a.z) {
      z[i].get(g);
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] *= g[k] * sigmoid(g[k]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) e[k] = w.live ? e[k] : 0.f;
  }
};

template <typename T> __global__ __launch_bounds__(kScanThreads, 4) void k_scan_parts(Scan a) {
  extern __shared__ __align__(16) float lds[];
  float *tile = lds, *tb = tile + W * kTok, *tc = tb + kStates * kTok;
  float *tA = tc + kStates * kTok, *th = tA + kStates * W, *tq = th + kStates * W;
  const ScanPlace p = scan_place(a, W);
  int tid = threadIdx.x;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, tl = lane % 16;
  const int cl = 4 * kCh * wave + lane / 16;
  const int64_t at_part = ((int64_t)p.b * a.nseg + p.seg) * a.D * a.N;
  const int64_t t0 = (int64_t)p.seg * kTok;
  if (t0 >= p.n) {   // no token: nothing is added
    for (int i = threadIdx.x; i < min(W, p.cend - p.c0) * a.N; i += kScanThreads)
      a.part[at_part + (int64_t)p.c0 * a.N + i] = a.part_r[at_part + (int64_t)p.c0 * a.N + i] = 0.f;
    if (threadIdx.x < min(W, p.cend - p.c0))
      a.steps[((int64_t)p.b * a.nseg + p.seg) * a.D + p.c0 + threadIdx.x] = 0.f;
    return;
  }
  float s[kCh][8], sx[kCh][8], e[kCh][8], ssum[kCh];
  States<T> low_b, low_c;
  {
    // everything is requested at once; the tile holds the steps, then s x, then e
    Steps<T, W> steps;
    Gated<T, W> gated;
    float in[kLoads<W>][8];
    steps.load(a, p, t0, tid);
    gated.load(a, p, t0, tid);
    low_b.load(a.b, a.bs, p, t0, 0, min(kStates, a.N), tid);
    low_c.load(a.c, a.cs, p, t0, 0, min(kStates, a.N), tid);
#pragma unroll
    for (int i = 0; i < kLoads<W>; ++i) {
      const Unit w = unit_of<W>(p, t0, i, tid);
      float own[8];
      steps.template get<true>(a, w, i, own, in[i]);
      put_unit(tile, w, own);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kCh; ++i) tile_load(tile, cl + 4 * i, tl, s[i]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLoads<W>; ++i) put_unit(tile, unit_of<W>(p, t0, i, tid), in[i]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kCh; ++i) tile_load(tile, cl + 4 * i, tl, sx[i]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLoads<W>; ++i) {
      const Unit w = unit_of<W>(p, t0, i, tid);
      gated.get(a, w, i, in[i]);
      put_unit(tile, w, in[i]);
    }
  }
  for (int n0 = 0; n0 < a.N; n0 += kStates) {
    const int count = min(kStates, a.N - n0);
    if (n0) {
      low_b.load(a.b, a.bs, p, t0, n0, count, tid);
      low_c.load(a.c, a.cs, p, t0, n0, count, tid);
    }
    low_b.put(tb, p, t0, count, tid);
    low_c.put(tc, p, t0, count, tid);
    load_channels<W>(a.A, p, a.N, n0, count, kLog2e, tA, tid);
    __syncthreads();
    if (n0 == 0) {
#pragma unroll
      for (int i = 0; i < kCh; ++i) {
        tile_load(tile, cl + 4 * i, tl, e[i]);
        ssum[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) ssum[i] += s[i][j];
        const float total = row_sum(ssum[i]);
        const int c = p.c0 + cl + 4 * i;
        if (tl == 15 && c < p.cend) a.steps[((int64_t)p.b * a.nseg + p.seg) * a.D + c] = total;
      }
    }
    for (int n = 0; n < count; ++n) {
      float Bv[8], Cv[8], S[kCh], Q[kCh], P[kCh], P2[kCh], h[kCh], q[kCh];
      lane_load(tb + n * kTok, tl, Bv);
      lane_load(tc + n * kTok, tl, Cv);
#pragma unroll
      for (int i = 0; i < kCh; ++i) {
        const float A = tA[n * W + cl + 4 * i];
        float at[8];
        S[i] = Q[i] = h[i] = q[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          at[j] = exp2_hw(s[i][j] * A);
          S[i] = fmaf(at[j], S[i], sx[i][j] * Bv[j]);
        }
#pragma unroll
        for (int j = 7; j >= 0; --j) Q[i] = at[j] * fmaf(e[i][j], Cv[j], Q[i]);
        P[i] = P2[i] = exp2_hw(ssum[i] * A);
      }
      row_scan2<false>(S[0], P[0], h[0], S[1], P[1], h[1]);
      row_scan2<true>(Q[0], P2[0], q[0], Q[1], P2[1], q[1]);
#pragma unroll
      for (int i = 0; i < kCh; ++i) {
        if (tl == 15) th[n * W + cl + 4 * i] = S[i];
        if (tl == 0) tq[n * W + cl + 4 * i] = Q[i];
      }
    }
    __syncthreads();
    tid = fresh_thread();
    store_channels<W>(a.part + at_part, p, a.N, n0, count, th, tid);
    store_channels<W>(a.part_r + at_part, p, a.N, n0, count, tq, tid);
  }
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

// A workgroup takes a.subs tiles of kTile channels one after the other, so that dB and dC are
// sums over all of them before they leave it.
template <typename T> __global__ __launch_bounds__(kScanThreads, 4) void k_scan_backward(Scan a) {
  extern __shared__ __align__(16) float lds[];
  float *t1 = lds, *t2 = t1 + kTile * kTok, *tb = t2 + kTile * kTok, *tc = tb + kStates * kTok;
  float *tlow = tc + kStates * kTok;   // dB, then dC
  float *tA = tlow + 2 * kStates * kTok, *th = tA + kStates * kTile, *tq = th + kStates * kTile;
  ScanPlace p = scan_place(a, kTile * a.subs);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, tl = lane % 16;
  const int cl = 4 * wave + lane / 16;
  const int64_t at_part = ((int64_t)p.b * a.nseg + p.seg) * a.D * a.N;
  const int64_t at_sum = ((int64_t)p.b * a.nseg + p.seg) * a.D;
  const int64_t t0 = (int64_t)p.seg * kTok;
  const bool some = t0 < p.n;
  for (int sub = 0; sub < a.subs && p.c0 < p.cend; ++sub, p.c0 += kTile) {
    const int c = p.c0 + cl;   // this lane's channel
    const bool channel = c < p.cend;
    static_assert(kLoads<kTile> == 1, "one unit of a thread");
    if (!some) {
      for (int i = threadIdx.x; i < min(kTile, p.cend - p.c0) * a.N; i += kScanThreads)
        a.part_a[at_part + (int64_t)p.c0 * a.N + i] = 0.f;
      if (tl == 15 && channel) {
        if (a.dskip) a.part_d[at_sum + c] = 0.f;
        if (a.dbias) a.part_s[at_sum + c] = 0.f;
      }
      const Unit w = unit_of<kTile>(p, t0, 0, threadIdx.x);
      const float none[8] = {};
      if (w.t >= a.L - t0 || w.c >= p.cend) continue;
      put_row<T>(a.dx, a.dxs, p, t0, w, none);
      put_row<T>(a.ddt, a.ddts, p, t0, w, none);
      if (a.z) put_row<T>(a.dz, a.dzs, p, t0, w, none);
    } else {
      float s[8], sx[8], e[8], ds[8], dsx[8], y[8], ssum = 0.f;
      States<T> low_b, low_c;
      int tid = fresh_thread();
      {
        const Unit w = unit_of<kTile>(p, t0, 0, tid);
        Steps<T, kTile> steps;
        Gated<T, kTile> gated;
        float own[8], x[8];
        steps.load(a, p, t0, tid);
        gated.load(a, p, t0, tid);
        if (sub == 0) {
          low_b.load(a.b, a.bs, p, t0, 0, min(kStates, a.N), tid);
          low_c.load(a.c, a.cs, p, t0, 0, min(kStates, a.N), tid);
        }
        steps.template get<false>(a, w, 0, own, x);
        put_unit(t1, w, own);   // the last tile's readers are behind a barrier
        put_unit(t2, w, x);
        __syncthreads();
        tile_load(t1, cl, tl, s);
        tile_load(t2, cl, tl, sx);
        __syncthreads();
        gated.get(a, w, 0, x);
        put_unit(t1, w, x);
      }
      for (int n0 = 0; n0 < a.N; n0 += kStates) {
        const int count = min(kStates, a.N - n0);
        if (n0) {
          tid = fresh_thread();
          low_b.load(a.b, a.bs, p, t0, n0, count, tid);
          low_c.load(a.c, a.cs, p, t0, n0, count, tid);
        }
        if (sub == 0) {
          low_b.put(tb, p, t0, count, tid);
          low_c.put(tc, p, t0, count, tid);
        }
        load_channels<kTile>(a.A, p, a.N, n0, count, 1.f, tA, tid);
        load_channels<kTile>(a.part + at_part, p, a.N, n0, count, 1.f, th, tid);
        load_channels<kTile>(a.part_r + at_part, p, a.N, n0, count, 1.f, tq, tid);
        __syncthreads();
        if (n0 == 0) {
          tile_load(t1, cl, tl, e);
          float skip = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            skip = fmaf(e[j], sx[j], skip);
            sx[j] *= s[j];
            ssum += s[j];
            ds[j] = dsx[j] = y[j] = 0.f;
          }
          if (a.dskip) {
            const float total = row_sum(skip);
            if (tl == 15 && channel) a.part_d[at_sum + c] = total;
          }
        }
        const int each = (count + kScanWaves - 1) / kScanWaves;   // states of a wave's turn
        for (int turn = 0; turn < kScanWaves; ++turn) {
          for (int k = 0; k < each; ++k) {
            const int n = ((turn + wave) % kScanWaves) * each + k, at_c = n * kTile + cl;
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
              y[j] = fmaf(Cv[j], h, y[j]);
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
        if (sub + 1 == a.subs || p.c0 + kTile >= p.cend) {
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
        store_channels<kTile>(a.part_a + at_part, p, a.N, n0, count, th, tid);
        __syncthreads();
      }
      tid = fresh_thread();
      const Unit w = unit_of<kTile>(p, t0, 0, tid);
      Steps<T, kTile> steps;
      Gated<T, kTile> gated;
      float dx[8], ddt[8], dz[8];
      steps.load(a, p, t0, tid);
      gated.load(a, p, t0, tid);
      tile_store(t1, cl, tl, ds);   // in place of what only this lane has read
      tile_store(t2, cl, tl, dsx);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int at = tile_at(8 * w.u + k, w.t);
        ddt[k] = t1[at];
        dx[k] = t2[at];
      }
      __syncthreads();
      if (a.z) tile_store(t1, cl, tl, y);
      __syncthreads();
      if (w.live) {
        float x[8], raw[8], ev[8], z[8], step[8], skip[8];
        steps.x[0].get(x);
        steps.dt[0].get(raw);
        gated.dy[0].get(ev);
        if (a.z) gated.z[0].get(z);
        if (a.bias)
#pragma unroll
          for (int k = 0; k < 8; ++k) raw[k] += a.bias[w.c + k];
#pragma unroll
        for (int k = 0; k < 8; ++k) skip[k] = 0.f;
        if (a.skip)
#pragma unroll
          for (int k = 0; k < 8; ++k) skip[k] = a.skip[w.c + k];
#pragma unroll
        for (int k = 0; k < 8; ++k) ddt[k] = fmaf(x[k], dx[k], ddt[k]);
        if (a.softplus) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            step[k] = softplus(raw[k]);
            ddt[k] *= softplus_slope(raw[k], step[k]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) step[k] = raw[k];
        }
        if (a.z)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float g = sigmoid(z[k]), v = fmaf(skip[k], x[k], t1[tile_at(8 * w.u + k, w.t)]);
            dz[k] = ev[k] * v * (g * fmaf(z[k], 1.f - g, 1.f));
            ev[k] *= z[k] * g;
          }
#pragma unroll
        for (int k = 0; k < 8; ++k) dx[k] = fmaf(step[k], dx[k], skip[k] * ev[k]);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) dx[k] = ddt[k] = dz[k] = 0.f;
      }
      if (w.t < a.L - t0 && w.c < p.cend) {
        put_row<T>(a.dx, a.dxs, p, t0, w, dx);
        put_row<T>(a.ddt, a.ddts, p, t0, w, ddt);
        if (a.z) put_row<T>(a.dz, a.dzs, p, t0, w, dz);
      }
      if (a.dbias) {
        float v[8], total = 0.f;
        put_unit(t2, w, ddt);
        __syncthreads();
        tile_load(t2, cl, tl, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) total += v[j];
        total = row_sum(total);
        if (tl == 15 && channel) a.part_s[at_sum + c] = total;
      }
      __syncthreads();
    }
  }
}

// dB and dC: over the workgroups of a group of channels.
constexpr int kLowThreads = 256;
template <typename T> __global__ __launch_bounds__(kLowThreads) void k_scan_low(Scan a, int tiles) {
  const int64_t GN = (int64_t)a.G * a.N, per = (int64_t)a.L * GN;
  const int64_t i = (int64_t)blockIdx.x * kLowThreads + threadIdx.x;
  if (i >= per) return;
  const int b = blockIdx.y;
  const int t = (int)(i / GN), gn = (int)(i - t * GN), g = gn / a.N, n = gn - g * a.N;
  const float *part = blockIdx.z ? a.part_c : a.part_b;
  float sum = 0.f;
  if (t < clamped_length(a.lengths, b, a.L))
#pragma unroll 8
    for (int k = 0; k < tiles; ++k) sum += part[((int64_t)k * a.B + b) * per + i];
  const Rows &r = blockIdx.z ? a.dcs : a.dbs;
  static_cast<T *>(blockIdx.z ? a.dc : a.db)[b * r.b + g * r.h + t * r.t + n] = from_f32<T>(sum);
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
hipError_t launch_tiles(K kernel, const Scan &a, int width, size_t lds, hipStream_t st) {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  const int tiles = a.G * ((a.D / a.G + width - 1) / width);
  kernel<<<dim3((unsigned)(tiles * a.nseg), a.B), kScanThreads, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_backward_parts(const Scan &a, Dt dt, hipStream_t st) {
  const size_t lds = sizeof(float) * (W * kTok + 2 * kStates * kTok + 3 * kStates * W);
  return dt == Dt::BF16 ? launch_tiles(k_scan_parts<bf16>, a, W, lds, st)
                        : launch_tiles(k_scan_parts<float>, a, W, lds, st);
}

hipError_t launch_scan_backward(const Scan &a, Dt dt, hipStream_t st) {
  const size_t lds = sizeof(float) * (2 * kTile * kTok + 4 * kStates * kTok + 3 * kStates * kTile);
  return dt == Dt::BF16 ? launch_tiles(k_scan_backward<bf16>, a, kTile * a.subs, lds, st)
                        : launch_tiles(k_scan_backward<float>, a, kTile * a.subs, lds, st);
}

hipError_t launch_scan_backward_sums(const Scan &a, Dt dt, hipStream_t st) {
  const int64_t low = (int64_t)a.L * a.G * a.N;
  if (low > 0) {
    const int tiles = (a.D / a.G + kTile * a.subs - 1) / (kTile * a.subs);
    const dim3 grid((unsigned)((low + kLowThreads - 1) / kLowThreads), a.B, 2);
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
