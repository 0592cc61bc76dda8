// conv.hip - short causal convolution, one filter of `width` taps per channel, with an
// optional bias and SiLU:
//
//   u_t = bias + sum_j w[j] x_{t - W + 1 + j},   y_t = u_t or u_t sigmoid(u_t)
//   g_t = dy_t (dy/du)(u_t),  dx_t = sum_j w[j] g_{t + W - 1 - j},
//   dw[j] = sum_t g_t x_{t - W + 1 + j},  dbias = sum_t g_t
//
// Bound by the bytes: an input is read once and an output written once, with 2 W operations
// between them. A thread owns 16 bytes of neighbouring channels and a run of tokens, so the
// window of the last W - 1 inputs moves through its registers, and only the run's W - 1 first
// inputs are read twice. Everything is fp32 between load and store. 4 x 4096 x 4096 in bf16 with
// four taps: 70 us forward (268 MB: 3.8 TB/s), 88 backward (403 MB: 4.6 TB/s) and 5 for the sums.
#include "recurrent.hpp"
#include "vec_rows.hpp"

namespace favor {
namespace {

constexpr int kConvThreads = 256;
// Rows in flight; 8 against 4: 70.6 against 73.3 us (4 x 4096 x 4096 bf16, 4 taps)
constexpr int kAhead = 8;

// Token t of one sequence: x for t >= 0, the carried inputs before it.
template <typename T, int V>
__device__ __forceinline__ void input_row(RowVec<T, V> &r, const T *x, int64_t stride,
                                          const T *state, int64_t D, int W, int t, int n) {
  if (t >= n) r.zero();
  else if (t >= 0) r.load(x + t * stride);
  else if (state) r.load(state + (W - 1 + t) * D);
  else r.zero();
}

template <typename T, int W, int V>
__global__ __launch_bounds__(kConvThreads) void k_conv(Conv a) {
  const int units = a.D / V;
  const int64_t id = (int64_t)blockIdx.x * kConvThreads + threadIdx.x;
  const int run = (int)(id / units), unit = (int)(id - (int64_t)run * units);
  const int t0 = run * a.run, b = blockIdx.y;
  if (t0 >= max(a.L, 1)) return;
  const int c = unit * V;
  const int n = clamped_length(a.lengths, b, a.L);
  const T *x = static_cast<const T *>(a.x) + b * a.xs.b + c;
  T *y = static_cast<T *>(a.y) + b * a.ys.b + c;
  const T *state =
      a.state_in ? static_cast<const T *>(a.state_in) + (int64_t)b * (W - 1) * a.D + c : nullptr;
  float w[V][W], bias[V], win[W - 1][V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int j = 0; j < W; ++j) w[i][j] = a.w[(int64_t)(c + i) * W + j];
    bias[i] = a.bias ? a.bias[c + i] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < W - 1; ++i) {
    RowVec<T, V> r;
    input_row<T, V>(r, x, a.xs.t, state, a.D, W, t0 - (W - 1) + i, n);
    r.get(win[i]);
  }
  if (run == 0 && a.state_out) {
    // the inputs after the last token; all are read before the first is written, since
    // state_out may be state_in (whose readers are all in run 0: a run has W - 1 tokens)
    RowVec<T, V> r[W - 1];
    T *so = static_cast<T *>(a.state_out) + (int64_t)b * (W - 1) * a.D + c;
#pragma unroll
    for (int i = 0; i < W - 1; ++i)
      input_row<T, V>(r[i], x, a.xs.t, state, a.D, W, n - (W - 1) + i, n);
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      float v[V];
      r[i].get(v);
      store_row<V>(so + (int64_t)i * a.D, v);
    }
  }
  // kAhead rows at a time, the next ones requested before: two sets of registers in turn, and
  // requests without conditions (a row behind the last asks for the last one).
  const int t1 = min(t0 + a.run, a.L), last = min(n, t1) - 1;
  using Raw = RowVec<T, V>[kAhead];
  const auto request = [&](Raw &r, int t) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) r[i].load(x + min(t + i, last) * a.xs.t);
  };
  const auto rows = [&](const Raw &r, int t) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (t + i >= t1) break;
      float v[V], u[V];
      r[i].get(v);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        u[k] = bias[k];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) u[k] = fmaf(w[k][j], win[j][k], u[k]);
        u[k] = fmaf(w[k][W - 1], v[k], u[k]);
        if (a.silu) u[k] *= sigmoid(u[k]);
        if (t + i > last) u[k] = 0.f;
      }
      store_row<V>(y + (t + i) * a.ys.t, u);
#pragma unroll
      for (int k = 0; k < V; ++k) {
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) win[j][k] = win[j + 1][k];
        win[W - 2][k] = v[k];
      }
    }
  };
  int t = t0;
  if (last >= t0) {
    Raw even, odd;
    request(even, t);
    for (; t <= last; t += 2 * kAhead) {
      request(odd, t + kAhead);
      rows(even, t);
      request(even, t + 2 * kAhead);
      rows(odd, t + kAhead);
    }
  }
  const float none[V] = {};   // rows behind the sequence
  for (; t < t1; ++t) store_row<V>(y + t * a.ys.t, none);
}

// A workgroup takes `units_wide` neighbouring units by 256 / units_wide runs, and sums the
// filters' gradients of its runs in LDS.
constexpr int kBackWide = 16;
template <typename T> constexpr int back_vec(int W) {
  return sizeof(T) == 2 && W <= 4 ? 8 : 4;   // more taps of more channels spill
}
constexpr int kBackAhead = 2;   // rows in flight, of two tensors

template <typename T, int W, int V>
__global__ __launch_bounds__(kConvThreads) void k_conv_backward(Conv a, int wide, int tiles) {
  __shared__ float sums[(W + 1) * V][kConvThreads + 1];
  const int units = a.D / V, tid = threadIdx.x;
  const int tile = blockIdx.x % tiles, block = blockIdx.x / tiles;
  const int unit = tile * wide + tid % wide;
  const int high = kConvThreads / wide;
  const int b = blockIdx.y;
  const int run = block * high + tid / wide;
  const int64_t t0w = (int64_t)run * a.run;
  const bool live = unit < units && t0w < max(a.L, 1);
  float dw[W][V], db[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    db[k] = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j][k] = 0.f;
  }
  if (live) {
    const int t0 = (int)t0w, c = unit * V;
    const int n = clamped_length(a.lengths, b, a.L);
    const T *x = static_cast<const T *>(a.x) + b * a.xs.b + c;
    const T *dy = static_cast<const T *>(a.dy) + b * a.dys.b + c;
    T *dx = static_cast<T *>(a.dx) + b * a.dxs.b + c;
    const int64_t at_state = (int64_t)b * (W - 1) * a.D + c;
    const T *state = a.state_in ? static_cast<const T *>(a.state_in) + at_state : nullptr;
    const T *dso = a.dstate_out ? static_cast<const T *>(a.dstate_out) + at_state : nullptr;
    T *dsi = a.dstate_in ? static_cast<T *>(a.dstate_in) + at_state : nullptr;
    float w[W][V], bias[V], win[W][V], g[W][V];   // g[j]: of token t - W + 1 + j
#pragma unroll
    for (int k = 0; k < V; ++k) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        w[j][k] = a.w[(int64_t)(c + k) * W + j];
        g[j][k] = 0.f;
      }
      bias[k] = a.bias ? a.bias[c + k] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      RowVec<T, V> r;
      input_row<T, V>(r, x, a.xs.t, state, a.D, W, t0 - (W - 1) + i, n);
      r.get(win[i + 1]);
    }
    // dx of token s needs g up to s + W - 1: the run's last tokens read W - 1 rows past it
    const int end = min(t0 + a.run, a.L) + W - 1, last = min(n, end) - 1;
    struct Raw {
      RowVec<T, V> x[kBackAhead], d[kBackAhead];
    };
    const auto request = [&](Raw &r, int t) {   // as forward
#pragma unroll
      for (int i = 0; i < kBackAhead; ++i) {
        const int at = min(t + i, last);
        r.x[i].load(x + at * a.xs.t);
        r.d[i].load(dy + at * a.dys.t);
      }
    };
    const auto rows = [&](const Raw &r, int t) {
#pragma unroll
      for (int i = 0; i < kBackAhead; ++i) {
        const int tt = t + i;
        if (tt >= end) break;
        float d[V], o[V];
        r.d[i].get(d);
#pragma unroll
        for (int k = 0; k < V; ++k) {
#pragma unroll
          for (int j = 0; j < W - 1; ++j) {
            win[j][k] = win[j + 1][k];
            g[j][k] = g[j + 1][k];
          }
        }
        r.x[i].get(win[W - 1]);
        const bool inside = tt <= last && tt < n, own = inside && tt < t0 + a.run;
#pragma unroll
        for (int k = 0; k < V; ++k) {
          if (a.silu) {
            float u = bias[k];
#pragma unroll
            for (int j = 0; j < W; ++j) u = fmaf(w[j][k], win[j][k], u);
            const float s = sigmoid(u);
            d[k] *= s * fmaf(u, 1.f - s, 1.f);
          }
          g[W - 1][k] = inside ? d[k] : 0.f;
          if (own) {
            db[k] += d[k];
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][k] = fmaf(d[k], win[j][k], dw[j][k]);
          }
          o[k] = 0.f;
#pragma unroll
          for (int j = 0; j < W; ++j) o[k] = fmaf(w[W - 1 - j][k], g[j][k], o[k]);
        }
        const int s = tt - (W - 1);   // dx of this token is complete
        if (s < t0 && (run > 0 || !dsi)) continue;
        if (dso && s < n && s >= n - (W - 1)) {
          RowVec<T, V> q;
          float v[V];
          q.load(dso + (int64_t)(s - n + W - 1) * a.D);
          q.get(v);
#pragma unroll
          for (int k = 0; k < V; ++k) o[k] += v[k];
        }
        if (s >= 0) {
          if (s >= n) {
#pragma unroll
            for (int k = 0; k < V; ++k) o[k] = 0.f;
          }
          store_row<V>(dx + s * a.dxs.t, o);
        } else {
          store_row<V>(dsi + (int64_t)(s + W - 1) * a.D, o);
        }
      }
    };
    if (last >= t0) {
      Raw even, odd;
      request(even, t0);
      for (int t = t0; t < end; t += 2 * kBackAhead) {
        request(odd, t + kBackAhead);
        rows(even, t);
        request(even, t + 2 * kBackAhead);
        rows(odd, t + kBackAhead);
      }
    } else {   // no token of the sequence: zeros, and the states' gradients
      Raw none;
#pragma unroll
      for (int i = 0; i < kBackAhead; ++i) {
        none.x[i].zero();
        none.d[i].zero();
      }
      for (int t = t0; t < end; t += kBackAhead) rows(none, t);
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) {
#pragma unroll
    for (int j = 0; j < W; ++j) sums[j * V + k][tid] = dw[j][k];
    sums[W * V + k][tid] = db[k];
  }
  __syncthreads();
  const int64_t row = (int64_t)b * (gridDim.x / tiles) + block;
  for (int i = tid; i < wide * (W + 1) * V; i += kConvThreads) {
    const int j = i / (wide * V), ck = i - j * wide * V;   // tap, channel of the tile
    const int u = ck / V, k = ck - u * V;
    const int c = (tile * wide + u) * V + k;
    if (c >= a.D) continue;
    float s = 0.f;
    for (int r = 0; r < high; ++r) s += sums[j * V + k][r * wide + u];
    a.part[(row * (W + 1) + j) * a.D + c] = s;
  }
}

// Sums of part's rows: 64 columns by 16 row lanes of a workgroup, joined in a fixed order.
constexpr int kSumCols = 64, kSumLanes = 16;
__global__ __launch_bounds__(kSumCols *kSumLanes) void k_conv_sums(Conv a, int rows) {
  __shared__ float part[kSumLanes][kSumCols];
  const int64_t cols = (int64_t)(a.width + 1) * a.D;
  const int64_t col = (int64_t)blockIdx.x * kSumCols + threadIdx.x % kSumCols;
  const int lane = threadIdx.x / kSumCols;
  float s = 0.f;
  if (col < cols && a.part)
#pragma unroll 8
    for (int r = lane; r < rows; r += kSumLanes) s += a.part[r * cols + col];
  part[lane][threadIdx.x % kSumCols] = s;
  __syncthreads();
  if (lane || col >= cols) return;
  for (int i = 1; i < kSumLanes; ++i) s += part[i][threadIdx.x];
  const int j = (int)(col / a.D), c = (int)(col - (int64_t)j * a.D);
  if (j < a.width) a.dw[(int64_t)c * a.width + j] = s;
  else if (a.dbias) a.dbias[c] = s;
}

// One token of B sequences, the last inputs in a pool: bound by the launch and one round of
// loads (one sequence of 2048 channels: 4.5 us). A thread owns four channels of one sequence.
template <typename T>
__global__ __launch_bounds__(kConvThreads) void k_conv_step(Conv a) {
  __shared__ int next;
  constexpr int V = 4;
  const int W = a.width, c = (blockIdx.x * kConvThreads + threadIdx.x) * V;
  const int first = blockIdx.y;
  for (int b = first; b < a.B;) {
    int slot = b, after = a.B;
    if (a.slots) {
      slot = a.slots[b];
      if (slot >= 0 && slot < a.n_slots) {
        after = next_turn<kConvThreads>(a.slots, a.B, b, first, slot, &next);
        if (after < 0) return;
      }
    }
    const bool live = slot >= 0 && slot < a.n_slots;   // others have no state: y = 0
    if (c < a.D) {
      float u[V] = {0.f, 0.f, 0.f, 0.f}, v[V];
      if (live) {
        T *state = static_cast<T *>(a.state_out) + (int64_t)slot * (W - 1) * a.D + c;
        RowVec<T, V> r, rx;
        rx.load(static_cast<const T *>(a.x) + b * a.xs.b + c);
        if (a.bias)
#pragma unroll
          for (int k = 0; k < V; ++k) u[k] = a.bias[c + k];
        for (int j = 0; j < W; ++j) {
          if (j < W - 1) r.load(state + (int64_t)j * a.D);
          else r = rx;
          r.get(v);
#pragma unroll
          for (int k = 0; k < V; ++k) u[k] = fmaf(a.w[(int64_t)(c + k) * W + j], v[k], u[k]);
          if (j > 0) store_row<V>(state + (int64_t)(j - 1) * a.D, v);
        }
        if (a.silu)
#pragma unroll
          for (int k = 0; k < V; ++k) u[k] *= sigmoid(u[k]);
      }
      store_row<V>(static_cast<T *>(a.y) + b * a.ys.b + c, u);
    }
    b = after;
  }
}

template <typename T, int W>
hipError_t launch_w(const Conv &a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const int64_t runs = a.L > 0 ? (a.L + a.run - 1) / a.run : 1;
  const int64_t threads = runs * (a.D / V);
  const dim3 grid((unsigned)((threads + kConvThreads - 1) / kConvThreads), a.B);
  k_conv<T, W, V><<<grid, kConvThreads, 0, st>>>(a);
  return hipGetLastError();
}

struct BackCut {
  int wide, tiles, run, blocks;   // units of a workgroup, tiles of units, tokens of a run
};

// Each run reads W - 1 rows more than its own, so it is long, unless that leaves too few
// workgroups: 4 x 4096 x 4096 with four taps takes 89 us at 64 tokens (512 workgroups),
// 96 at 32 and 112 at 16.
constexpr int kBackBlocks = 512;
BackCut back_cut(int B, int L, int units) {
  BackCut c{1, 0, 128, 1};
  while (c.wide < kBackWide && c.wide < units) c.wide *= 2;
  c.tiles = (units + c.wide - 1) / c.wide;
  do {
    c.run /= 2;
    const int tokens = c.run * (kConvThreads / c.wide);
    c.blocks = L > 0 ? (L + tokens - 1) / tokens : 1;
  } while (c.run > 16 && (int64_t)B * c.tiles * c.blocks < kBackBlocks);
  return c;
}

template <typename T, int W>
hipError_t launch_back_w(const Conv &a, hipStream_t st) {
  constexpr int V = back_vec<T>(W);
  const BackCut c = back_cut(a.B, a.L, a.D / V);
  Conv run = a;
  run.run = c.run;
  k_conv_backward<T, W, V>
      <<<dim3(c.tiles * c.blocks, a.B), kConvThreads, 0, st>>>(run, c.wide, c.tiles);
  return hipGetLastError();
}

}  // namespace

int64_t conv_part_rows(int B, int L, int D, int width, Dt dt) {
  const int V = dt == Dt::BF16 ? back_vec<bf16>(width) : back_vec<float>(width);
  return (int64_t)B * back_cut(B, L, D / V).blocks;
}

#define FAVOR_BY_WIDTH(fn)                                           \
  switch (a.width) {                                                 \
    case 2: return dt == Dt::BF16 ? fn<bf16, 2>(a, st) : fn<float, 2>(a, st); \
    case 3: return dt == Dt::BF16 ? fn<bf16, 3>(a, st) : fn<float, 3>(a, st); \
    case 4: return dt == Dt::BF16 ? fn<bf16, 4>(a, st) : fn<float, 4>(a, st); \
    case 5: return dt == Dt::BF16 ? fn<bf16, 5>(a, st) : fn<float, 5>(a, st); \
    case 6: return dt == Dt::BF16 ? fn<bf16, 6>(a, st) : fn<float, 6>(a, st); \
    case 7: return dt == Dt::BF16 ? fn<bf16, 7>(a, st) : fn<float, 7>(a, st); \
    case 8: return dt == Dt::BF16 ? fn<bf16, 8>(a, st) : fn<float, 8>(a, st); \
  }                                                                  \
  return hipErrorInvalidValue;

hipError_t launch_conv(const Conv &a, Dt dt, hipStream_t st) { FAVOR_BY_WIDTH(launch_w) }
hipError_t launch_conv_backward(const Conv &a, Dt dt, hipStream_t st) {
  FAVOR_BY_WIDTH(launch_back_w)
}

hipError_t launch_conv_sums(const Conv &a, int rows, hipStream_t st) {
  const int64_t cols = (int64_t)(a.width + 1) * a.D;
  k_conv_sums<<<(unsigned)((cols + kSumCols - 1) / kSumCols), kSumCols * kSumLanes, 0, st>>>(a, rows);
  return hipGetLastError();
}

hipError_t launch_conv_step(const Conv &a, Dt dt, hipStream_t st) {
  const dim3 grid((a.D / 4 + kConvThreads - 1) / kConvThreads, a.B);
  if (dt == Dt::BF16) k_conv_step<bf16><<<grid, kConvThreads, 0, st>>>(a);
  else k_conv_step<float><<<grid, kConvThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace favor
