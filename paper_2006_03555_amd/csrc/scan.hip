// scan.hip - selective state space scan over a sequence, forward: per channel d and state n
//
//   s_t = softplus(dt_t + bias_d),  h_t = exp(s_t A_dn) h_{t-1} + s_t x_t B_t[n],
//   y_t = (sum_n C_t[n] h_t[n] + skip_d x_t) silu(z_t)
//
// Bound by the vector unit: each (token, channel, state) takes a product and an exponential
// (two issue slots), the input's product, the recurrence once inside the lane and once from
// its true state, and the output's sum; B and C are read from LDS for two channels at a time.
// Nothing of size tokens x channels x states leaves the registers.
#include "scan_common.hpp"

namespace favor {
namespace {

// Channels per lane: a workgroup's 8 waves take 32 * kCh channels.
template <int kCh> constexpr int kWide = 4 * kScanWaves * kCh;

// One (chunk, n) step of kCh channels: a = 2^(s A), S and P of the lane, the row's scan.
// kOut: y += C h; h of the row's last lane goes back to `carry`.
template <int kCh, bool kOut> struct StateIn {   // what a step reads from LDS
  float B[8], C[8], A[kCh], h[kCh];

  __device__ __forceinline__ void load(const float *b, const float *c, const float *A2, const float *carry, int tl) {
    lane_load(b, tl, B);
    if (kOut) lane_load(c, tl, C);
#pragma unroll
    for (int i = 0; i < kCh; ++i) {
      A[i] = A2[4 * i];
      h[i] = carry[4 * i];
    }
  }
};
template <int kCh, bool kOut>
__device__ __forceinline__ void forward_state(const float (&s)[kCh][8], const float (&sx)[kCh][8],
                                              const float (&ssum)[kCh], const StateIn<kCh, kOut> &in,
                                              float *carry, int tl, float (&y)[kCh][8]) {
  float a[kCh][8], bx[kCh][8], S[kCh], P[kCh], h[kCh];
#pragma unroll
  for (int i = 0; i < kCh; ++i) {
    const float A = in.A[i];
    h[i] = in.h[i];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      a[i][j] = exp2_hw(s[i][j] * A);
      bx[i][j] = sx[i][j] * in.B[j];
    }
    S[i] = tl == 0 ? h[i] : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) S[i] = fmaf(a[i][j], S[i], bx[i][j]);
    P[i] = exp2_hw(ssum[i] * A);
  }
  if constexpr (kCh == 2) row_scan2<false>(S[0], P[0], h[0], S[1], P[1], h[1]);
  else row_scan<false>(S[0], P[0], h[0]);
#pragma unroll
  for (int i = 0; i < kCh; ++i) {
    if constexpr (kOut) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[i] = fmaf(a[i][j], h[i], bx[i][j]);
        y[i][j] = fmaf(in.C[j], h[i], y[i][j]);
      }
    }
    if (tl == 15) carry[4 * i] = S[i];
  }
}

// kOut: the rows y and the state after the last token. Otherwise the sums of the segments.
template <typename T, int kCh, bool kOut>
__global__ __launch_bounds__(kScanThreads, kOut && kCh == 2 ? 4 : 6) void k_scan(Scan a) {
  constexpr int W = kWide<kCh>;
  extern __shared__ __align__(16) float lds[];
  float *tile = lds, *tb = tile + W * kTok, *tc = tb + kStates * kTok;
  const int padded = (a.N + kStates - 1) / kStates * kStates;
  float *tA = tc + (kOut ? kStates * kTok : 0), *th = tA + padded * W;
  const ScanPlace p = scan_place(a, W);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, tl = lane % 16;
  const int cl = 4 * kCh * wave + lane / 16;   // this lane's first channel; the next is 4 on
  const int64_t DN = (int64_t)a.D * a.N, at_part = ((int64_t)p.b * a.nseg + p.seg) * DN;
  const float *h0 = nullptr;
  if (kOut && a.nseg > 1) h0 = a.part + at_part;
  else if (kOut && a.h_in) h0 = a.h_in + p.b * DN;
  for (int n0 = 0; n0 < a.N; n0 += kStates) {
    load_channels<W>(a.A, p, a.N, n0, min(kStates, a.N - n0), kLog2e, tA + n0 * W, threadIdx.x);
    load_channels<W>(h0, p, a.N, n0, min(kStates, a.N - n0), 1.f, th + n0 * W, threadIdx.x);
  }
  float seg_steps[kCh] = {};
  const int first = p.seg * a.chunks, last = min(first + a.chunks, (a.L + kTok - 1) / kTok);
  for (int chunk = first; chunk < last; ++chunk) {
    const int64_t t0 = (int64_t)chunk * kTok;
    const bool some = t0 < p.n;
    if (!some && !kOut) break;
    int tid = fresh_thread();
    if (some) {
      float s[kCh][8], sx[kCh][8], ssum[kCh], y[kCh][8];
      States<T> low_b, low_c;
      {
        // everything is requested at once; the tile holds the steps, then s x, then y
        Steps<T, W> steps;
        float in[kLoads<W>][8], own[kLoads<W>][8];
        steps.load(a, p, t0, tid);
        low_b.load(a.b, a.bs, p, t0, 0, min(kStates, a.N), tid);
        if (kOut) low_c.load(a.c, a.cs, p, t0, 0, min(kStates, a.N), tid);
#pragma unroll
        for (int i = 0; i < kLoads<W>; ++i) steps.template get<true>(a, unit_of<W>(p, t0, i, tid), i, own[i], in[i]);
        __syncthreads();   // the last chunk's rows have been read
#pragma unroll
        for (int i = 0; i < kLoads<W>; ++i) put_unit(tile, unit_of<W>(p, t0, i, tid), own[i]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kCh; ++i) tile_load(tile, cl + 4 * i, tl, s[i]);
        low_b.put(tb, p, t0, min(kStates, a.N), tid);
        if (kOut) low_c.put(tc, p, t0, min(kStates, a.N), tid);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLoads<W>; ++i) put_unit(tile, unit_of<W>(p, t0, i, tid), in[i]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kCh; ++i) {
          tile_load(tile, cl + 4 * i, tl, sx[i]);
          ssum[i] = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            ssum[i] += s[i][j];
            y[i][j] = 0.f;
          }
          if (!kOut) seg_steps[i] += ssum[i];
        }
      }
      for (int n0 = 0; n0 < a.N; n0 += kStates) {
        const int count = min(kStates, a.N - n0);
        if (n0) {
          tid = fresh_thread();
          low_b.load(a.b, a.bs, p, t0, n0, count, tid);
          if (kOut) low_c.load(a.c, a.cs, p, t0, n0, count, tid);
          __syncthreads();   // the last states' B and C have been read
          low_b.put(tb, p, t0, count, tid);
          if (kOut) low_c.put(tc, p, t0, count, tid);
          __syncthreads();
        }
        for (int n = 0; n < count; ++n) {
          const int at = (n0 + n) * W + cl;
          StateIn<kCh, kOut> in;
          in.load(tb + n * kTok, tc + n * kTok, tA + at, th + at, tl);
          forward_state<kCh, kOut>(s, sx, ssum, in, th + at, tl, y);
        }
      }
      if (kOut) {
#pragma unroll
        for (int i = 0; i < kCh; ++i) tile_store(tile, cl + 4 * i, tl, y[i]);
      }
    }
    RowVec<T, 8> rx[kLoads<W>], rz[kLoads<W>];
    tid = fresh_thread();
    if (kOut && some) {
#pragma unroll
      for (int i = 0; i < kLoads<W>; ++i) {
        const Unit w = unit_of<W>(p, t0, i, tid);
        if (a.skip) rx[i] = get_row<T>(a.x, a.xs, p, t0, w);
        if (a.z) rz[i] = get_row<T>(a.z, a.zs, p, t0, w);
      }
    }
    if (!kOut) continue;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLoads<W>; ++i) {
      const Unit w = unit_of<W>(p, t0, i, tid);
      if (w.t >= a.L - t0 || w.c >= p.cend) continue;
      float y[8], v[8];
      if (w.live) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = tile[tile_at(8 * w.u + k, w.t)];
        if (a.skip) {
          rx[i].get(v);
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = fmaf(a.skip[w.c + k], v[k], y[k]);
        }
        if (a.z) {
          rz[i].get(v);
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] *= v[k] * sigmoid(v[k]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = 0.f;
      }
      put_row<T>(a.y, a.ys, p, t0, w, y);
    }
  }
  __syncthreads();
  float *end = nullptr;
  if (!kOut) end = a.part + at_part;
  else if (a.h_out && p.seg == a.nseg - 1) end = a.h_out + p.b * DN;
  if (end)
    for (int n0 = 0; n0 < a.N; n0 += kStates)
      store_channels<W>(end, p, a.N, n0, min(kStates, a.N - n0), th + n0 * W, threadIdx.x);
  if (!kOut) {
#pragma unroll
    for (int i = 0; i < kCh; ++i) {
      const float total = row_sum(seg_steps[i]);
      const int c = p.c0 + cl + 4 * i;
      if (tl == 15 && c < p.cend) a.steps[((int64_t)p.b * a.nseg + p.seg) * a.D + c] = total;
    }
  }
}

// One thread per (sequence, channel, state): the states before each segment from the
// segments' sums; kRight: behind each segment, from the last.
constexpr int kPrefixThreads = 256;
template <bool kRight>
__device__ __forceinline__ void chain(const Scan &a, float *part, float h, float A2, int64_t at, int64_t at_s) {
  const int64_t DN = (int64_t)a.D * a.N;
  constexpr int kAhead = 8;
  for (int i = 0; i < a.nseg; i += kAhead) {
    float S[kAhead], s[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i + j >= a.nseg) break;
      const int k = kRight ? a.nseg - 1 - i - j : i + j;
      S[j] = part[at + k * DN];
      s[j] = a.steps[at_s + (int64_t)k * a.D];
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i + j >= a.nseg) break;
      const int k = kRight ? a.nseg - 1 - i - j : i + j;
      part[at + k * DN] = h;
      h = fmaf(exp2_hw(s[j] * A2), h, S[j]);
    }
  }
  if (kRight) {
    if (a.dh_in) a.dh_in[at - (int64_t)blockIdx.y * (a.nseg - 1) * DN] = h;
  }
}

template <bool kBackward> __global__ __launch_bounds__(kPrefixThreads) void k_scan_prefix(Scan a) {
  const int64_t DN = (int64_t)a.D * a.N, i = (int64_t)blockIdx.x * kPrefixThreads + threadIdx.x;
  if (i >= DN) return;
  const int b = blockIdx.y;
  const float A2 = kLog2e * a.A[i];
  const int64_t at = (int64_t)b * a.nseg * DN + i, at_s = (int64_t)b * a.nseg * a.D + i / a.N;
  if (kBackward && blockIdx.z) chain<true>(a, a.part_r, a.dh_out ? a.dh_out[b * DN + i] : 0.f, A2, at, at_s);
  else chain<false>(a, a.part, a.h_in ? a.h_in[b * DN + i] : 0.f, A2, at, at_s);
}

template <typename T, int kCh, bool kOut> hipError_t launch_as(const Scan &a, hipStream_t st) {
  constexpr int W = kWide<kCh>;
  const size_t lds = sizeof(float) * (W * kTok + (kOut ? 2 : 1) * kStates * kTok +
                                     2 * (size_t)((a.N + kStates - 1) / kStates * kStates) * W);
  const auto kernel = k_scan<T, kCh, kOut>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int tiles = a.G * ((a.D / a.G + W - 1) / W);
  const int segments = kOut ? a.nseg : a.nseg - 1;   // nothing follows the last segment's sums
  kernel<<<dim3((unsigned)(tiles * segments), a.B), kScanThreads, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan(const Scan &a, Dt dt, int tile, hipStream_t st) {
  if (dt == Dt::F32) return launch_as<float, 1, true>(a, st);
  return tile == kWide<2> ? launch_as<bf16, 2, true>(a, st) : launch_as<bf16, 1, true>(a, st);
}

hipError_t launch_scan_sums(const Scan &a, Dt dt, hipStream_t st) {
  return dt == Dt::BF16 ? launch_as<bf16, 1, false>(a, st) : launch_as<float, 1, false>(a, st);
}

hipError_t launch_scan_prefix(const Scan &a, bool backward, hipStream_t st) {
  const unsigned blocks = (unsigned)(((int64_t)a.D * a.N + kPrefixThreads - 1) / kPrefixThreads);
  if (backward) k_scan_prefix<true><<<dim3(blocks, a.B, 2), kPrefixThreads, 0, st>>>(a);
  else k_scan_prefix<false><<<dim3(blocks, a.B), kPrefixThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace favor
