// scan.hip - selective state space scan over a sequence, forward: per channel d and state n
//
//   s_t = softplus(dt_t + bias_d),  h_t = exp(s_t A_dn) h_{t-1} + s_t x_t B_t[n],
//   y_t = (sum_n C_t[n] h_t[n] + skip_d x_t) silu(z_t)
//
// Bound by the vector unit: each (token, channel, state) takes a product and an exponential
// (two issue slots), the input's product, the recurrence once inside the lane and once from
// its true state, and the output's sum: seven slots, and 10.6 as counted with the row's scan and
// the rows' way through LDS (the segments' sums, without an output: 8.7). Nothing of size tokens
// x channels x states leaves the registers. B4 L4096 D2048 N16 in bf16 (one segment): 225 to 264
// us, 2.0 to 2.4 T state steps/s; B1 L65536 D2048: sums of 63 of its 64 segments 505 us, prefix 13,
// then 749 us, 2.9 T/s.
#include "scan_common.hpp"

namespace favor {
namespace {

constexpr int W = 4 * kScanWaves;   // channels of a workgroup

// What a step of one state reads from LDS.
template <bool kOut> struct StateIn {
  float B[8], C[8], A, h;

  __device__ __forceinline__ void load(const float *b, const float *c, const float *A2, const float *carry, int tl) {
    lane_load(b, tl, B);
    if (kOut) lane_load(c, tl, C);
    A = *A2;
    h = *carry;
  }
};
// K states side by side: a = 2^(s A), S and P of the lane, the row's scan. kOut: y += C h; h of
// the row's last lane goes back to carry.
template <int K, bool kOut>
__device__ __forceinline__ void forward_states(const float (&s)[8], const float (&sx)[8], float ssum,
                                               const StateIn<kOut> (&in)[K], float *carry, int tl, float (&y)[8]) {
  float a[K][8], bx[K][8], S[K], P[K], h[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    h[k] = in[k].h;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      a[k][j] = exp2_hw(s[j] * in[k].A);
      bx[k][j] = sx[j] * in[k].B[j];
    }
    S[k] = tl == 0 ? h[k] : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) S[k] = fmaf(a[k][j], S[k], bx[k][j]);
    P[k] = exp2_hw(ssum * in[k].A);
  }
  if constexpr (K == 2) row_scan2<false>(S[0], P[0], h[0], S[1], P[1], h[1]);
  else row_scan(S[0], P[0], h[0]);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if constexpr (kOut) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[k] = fmaf(a[k][j], h[k], bx[k][j]);
        y[j] = fmaf(in[k].C[j], h[k], y[j]);
      }
    }
    if (tl == 15) carry[k * W] = S[k];
  }
}

// kOut: the rows y and the state after the last token. Otherwise the sums of the segments.
// kAhead, for calls of one segment in bf16, whose few workgroups a compute unit does not overlap:
// a chunk's rows are requested before the states of the one before are taken, two states go side
// by side, and y has a tile of its own, so that the next rows need not wait for its readers. Whole
// calls with it and without: B4 L4096 D2048 N16 230 and 239 us, B4 L2048 D2048 N64 370 and 391 (with
// four workgroups to a unit the registers cost more than it gains: B16 L1024 D4096 N16 357 and 340).
// In fp32, whose rows take twice the registers, it would spill and lose everywhere (B4 L4096 D2048
// N16 292 and 267, B1 L128 D512 N16 10.8 and 10.3), and so would segments' workgroups, of which
// three share a unit (745 and 726 at B1 L65536 D2048).
template <typename T, bool kOut, bool kAhead> struct ScanLds {
  static constexpr int kRaw = kPairTiles<T> * W * kTok;
  static constexpr int kRows = kRaw + (kAhead ? W * kTok : 0);   // else y takes the place of x and dt
  static constexpr int kLow = (kOut ? 2 : 1) * kStates * kTok;
  static size_t bytes(const Scan &a) {
    const int padded = ((kOut ? a.N : a.sum_states) + kStates - 1) / kStates * kStates;
    return sizeof(float) * (kRows + kLow + 2 * (size_t)padded * W);
  }
};
template <typename T, bool kOut, bool kAhead>
__global__ __launch_bounds__(kScanThreads, kAhead ? 4 : 6) void k_scan(Scan a) {
  constexpr int K = kAhead ? 2 : 1;
  using Lds = ScanLds<T, kOut, kAhead>;
  extern __shared__ __align__(16) float lds[];
  float *tile = lds, *ty = kAhead ? tile + Lds::kRaw : tile;
  float *tb = tile + Lds::kRows, *tc = tb + kStates * kTok;
  // the states of this workgroup; those of a chunk's pass are n0 to n0 + count - 1
  const int first_n = kOut ? 0 : blockIdx.z * a.sum_states, end_n = kOut ? a.N : min(first_n + a.sum_states, a.N);
  const int padded = (end_n - first_n + kStates - 1) / kStates * kStates;
  float *tA = tb + Lds::kLow, *th = tA + padded * W;
  const ScanPlace p = scan_place(a, W);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, tl = lane % 16;
  const int cl = 4 * wave + lane / 16, c = min(p.c0 + cl, p.cend - 1);   // this lane's channel
  const int64_t DN = (int64_t)a.D * a.N, at_part = ((int64_t)p.b * a.nseg + p.seg) * DN;
  const float *h0 = nullptr;
  if (kOut && a.nseg > 1) h0 = a.part + at_part;
  else if (kOut && a.h_in) h0 = a.h_in + p.b * DN;
  for (int n0 = first_n; n0 < end_n; n0 += kStates) {
    const int count = min(kStates, end_n - n0), at = (n0 - first_n) * W;
    load_channels<W>(a.A, p, a.N, n0, count, kLog2e, tA + at, threadIdx.x);
    load_channels<W>(h0, p, a.N, n0, count, 1.f, th + at, threadIdx.x);
  }
  const float bias = a.bias ? a.bias[c] : 0.f, skip = kOut && a.skip ? a.skip[c] : 0.f;
  float seg_steps = 0.f;
  const int first = p.seg * a.chunks, last = min(first + a.chunks, (a.L + kTok - 1) / kTok);
  const int end = min(last, (p.n + kTok - 1) / kTok);   // of the chunks that have tokens
  static_assert(kLoads<W> == 1, "one unit of a thread");
  RowVec<T, 8> rx, rdt, rz;
  States<T> low_b, low_c;
  const auto request = [&](int chunk, int tid) {
    const int64_t t0 = (int64_t)chunk * kTok;
    const Unit w = unit_of<W>(p, t0, 0, tid);
    rx = get_row<T>(a.x, a.xs, p, t0, w);
    rdt = get_row<T>(a.dt, a.dts, p, t0, w);
    low_b.load(a.b, a.bs, p, t0, first_n, min(kStates, end_n - first_n), tid);
    if (kOut) low_c.load(a.c, a.cs, p, t0, first_n, min(kStates, end_n - first_n), tid);
  };
  if (kAhead && first < end) request(first, fresh_thread());
  for (int chunk = first; chunk < end; ++chunk) {
    const int64_t t0 = (int64_t)chunk * kTok;
    int tid = fresh_thread();
    if (!kAhead) {
      request(chunk, tid);
      if (chunk > first) __syncthreads();   // the last chunk's rows have been read
    }
    put_pair<W>(tile, unit_of<W>(p, t0, 0, tid), rx, rdt);
    low_b.put(tb, p, t0, min(kStates, end_n - first_n), tid);
    if (kOut) low_c.put(tc, p, t0, min(kStates, end_n - first_n), tid);
    __syncthreads();
    tid = fresh_thread();
    if (kAhead) {
      if (kOut)   // x stands in where there is no z
        rz = get_row<T>(a.z ? a.z : a.x, a.z ? a.zs : a.xs, p, t0, unit_of<W>(p, t0, 0, tid));
      request(min(chunk + 1, end - 1), tid);
    }
    float s[8], sx[8], ssum, y[8] = {};
    get_pair<T, W>(tile, cl, tl, sx, s);
    ssum = lane_steps(a, lane_left(p, t0, tl), bias, s, sx);
#pragma unroll
    for (int j = 0; j < 8; ++j) sx[j] *= s[j];
    if (!kOut) seg_steps += ssum;
    for (int n0 = first_n; n0 < end_n; n0 += kStates) {
      const int count = min(kStates, end_n - n0);
      if (n0 > first_n) {
        tid = fresh_thread();
        States<T> more_b, more_c;
        more_b.load(a.b, a.bs, p, t0, n0, count, tid);
        if (kOut) more_c.load(a.c, a.cs, p, t0, n0, count, tid);
        __syncthreads();   // the last states' B and C have been read
        more_b.put(tb, p, t0, count, tid);
        if (kOut) more_c.put(tc, p, t0, count, tid);
        __syncthreads();
      }
      for (int n = 0; n < count; n += K) {   // a state behind the last is zeros
        const int at = (n0 - first_n + n) * W + cl;
        StateIn<kOut> in[K];
#pragma unroll
        for (int k = 0; k < K; ++k)
          in[k].load(tb + (n + k) * kTok, tc + (n + k) * kTok, tA + at + k * W, th + at + k * W, tl);
        forward_states<K, kOut>(s, sx, ssum, in, th + at, tl, y);
      }
    }
    if constexpr (!kOut) continue;
    if (a.skip) {
      float x[8], dt[8];
      get_pair<T, W>(tile, cl, tl, x, dt);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = fmaf(skip, x[j], y[j]);
    }
    tile_store(ty, cl, tl, y);   // in place of what only this lane reads
    tid = fresh_thread();
    const Unit w = unit_of<W>(p, t0, 0, tid);
    if (!kAhead && a.z) rz = get_row<T>(a.z, a.zs, p, t0, w);
    __syncthreads();
    if (w.t >= a.L - t0 || w.c >= p.cend) continue;
    float v[8], o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = ty[tile_at(8 * w.u + k, w.t)];
    if (a.z) {
      rz.get(v);
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] *= v[k] * sigmoid(v[k]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = w.live ? o[k] : 0.f;
    put_row<T>(a.y, a.ys, p, t0, w, o);
  }
  if (kOut)   // rows behind the sequence
    for (int chunk = max(first, end); chunk < last; ++chunk) {
      const int64_t t0 = (int64_t)chunk * kTok;
      const Unit w = unit_of<W>(p, t0, 0, threadIdx.x);
      const float none[8] = {};
      if (w.t < a.L - t0 && w.c < p.cend) put_row<T>(a.y, a.ys, p, t0, w, none);
    }
  __syncthreads();
  float *to = nullptr;
  if (!kOut) to = a.part + at_part;
  else if (a.h_out && p.seg == a.nseg - 1) to = a.h_out + p.b * DN;
  if (to)
    for (int n0 = first_n; n0 < end_n; n0 += kStates)
      store_channels<W>(to, p, a.N, n0, min(kStates, end_n - n0), th + (n0 - first_n) * W, threadIdx.x);
  if (!kOut && first_n == 0) {
    const float total = row_sum(seg_steps);
    if (tl == 15 && p.c0 + cl < p.cend) a.steps[((int64_t)p.b * a.nseg + p.seg) * a.D + c] = total;
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
      const float e = exp2_hw(0.5f * s[j] * A2);   // a growing segment may pass e^88, and h be 0
      h = h == 0.f ? S[j] : fmaf(e, e * h, S[j]);
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

template <typename T, bool kOut, bool kAhead> hipError_t launch_as(const Scan &a, hipStream_t st) {
  const size_t lds = ScanLds<T, kOut, kAhead>::bytes(a);
  const auto kernel = k_scan<T, kOut, kAhead>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int tiles = a.G * ((a.D / a.G + W - 1) / W);
  const int segments = kOut ? a.nseg : a.nseg - 1;   // nothing follows the last segment's sums
  const int parts = kOut ? 1 : (a.N + a.sum_states - 1) / a.sum_states;
  kernel<<<dim3((unsigned)(tiles * segments), a.B, parts), kScanThreads, lds, st>>>(a);
  return hipGetLastError();
}
template <typename T> hipError_t launch_rows(const Scan &a, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (a.nseg == 1) return launch_as<T, true, true>(a, st);
  return launch_as<T, true, false>(a, st);
}

}  // namespace

hipError_t launch_scan(const Scan &a, Dt dt, hipStream_t st) {
  return dt == Dt::BF16 ? launch_rows<bf16>(a, st) : launch_rows<float>(a, st);
}

hipError_t launch_scan_sums(const Scan &a, Dt dt, hipStream_t st) {
  return dt == Dt::BF16 ? launch_as<bf16, false, false>(a, st) : launch_as<float, false, false>(a, st);
}

hipError_t launch_scan_prefix(const Scan &a, bool backward, hipStream_t st) {
  const unsigned blocks = (unsigned)(((int64_t)a.D * a.N + kPrefixThreads - 1) / kPrefixThreads);
  if (backward) k_scan_prefix<true><<<dim3(blocks, a.B, 2), kPrefixThreads, 0, st>>>(a);
  else k_scan_prefix<false><<<dim3(blocks, a.B), kPrefixThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace favor
