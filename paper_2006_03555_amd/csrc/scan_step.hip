// scan_step.hip - one token of the selective scan for B sequences whose states stay in a pool:
//
//   h <- exp(s A) h + s x B,  y = (C h + skip x) silu(z)      h [D][N] fp32, in place
//
// Bound by the states' bytes: each is read and written once (8 N bytes per channel), and A (4
// N) comes from the caches. kLanes neighbouring lanes share a channel and take kVec of its
// states at a time, so the state moves whole; their parts of y are joined by lane exchanges.
#include "recurrent.hpp"
#include "vec_rows.hpp"

namespace favor {
namespace {

constexpr int kStepThreads = 256;

template <int kVec> struct Floats;
template <> struct Floats<4> { using type = f32x4; };
template <> struct Floats<1> { typedef float type __attribute__((ext_vector_type(1))); };

template <typename T, int kVec>
__global__ __launch_bounds__(kStepThreads) void k_scan_step(Scan a, int lanes) {
  using V = typename Floats<kVec>::type;
  __shared__ int next;
  const int tid = threadIdx.x, unit0 = tid % lanes, units = a.N / kVec;
  const int d = blockIdx.x * (kStepThreads / lanes) + tid / lanes;
  const int first = blockIdx.y;
  const bool channel = d < a.D;
  const int dc = channel ? d : a.D - 1, g = dc / (a.D / a.G);
  for (int b = first; b < a.B;) {
    int slot = b, after = a.B;
    if (a.slots) {
      slot = a.slots[b];
      if (slot >= 0 && slot < a.n_slots) {
        after = next_turn<kStepThreads>(a.slots, a.B, b, first, slot, &next);
        if (after < 0) return;
      }
    }
    float y = 0.f;
    if (slot >= 0 && slot < a.n_slots) {   // others have no state: y = 0
      const float x = to_f32(static_cast<const T *>(a.x)[b * a.xs.b + dc]);
      float s = to_f32(static_cast<const T *>(a.dt)[b * a.dts.b + dc]);
      if (a.bias) s += a.bias[dc];
      if (a.softplus) s = softplus(s);
      const float sx = s * x;
      const T *B = static_cast<const T *>(a.b) + b * a.bs.b + g * a.bs.h;
      const T *C = static_cast<const T *>(a.c) + b * a.cs.b + g * a.cs.h;
      V *hp = reinterpret_cast<V *>(a.h_out + ((int64_t)slot * a.D + dc) * a.N);
      const V *Ap = reinterpret_cast<const V *>(a.A + (int64_t)dc * a.N);
      for (int i = unit0; i < units; i += lanes) {
        V h = hp[i];
        const V A = Ap[i];
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          h[k] = fmaf(exp2_hw(s * (kLog2e * A[k])), h[k], sx * to_f32(B[i * kVec + k]));
          y = fmaf(to_f32(C[i * kVec + k]), h[k], y);
        }
        if (channel) hp[i] = h;
      }
      for (int m = 1; m < lanes; m *= 2) y += __shfl_xor(y, m);
      if (a.skip) y = fmaf(a.skip[dc], x, y);
      if (a.z) {
        const float z = to_f32(static_cast<const T *>(a.z)[b * a.zs.b + dc]);
        y *= z * sigmoid(z);
      }
    }
    if (channel && unit0 == 0) static_cast<T *>(a.y)[b * a.ys.b + dc] = from_f32<T>(y);
    b = after;
  }
}

template <typename T, int kVec> hipError_t launch_v(const Scan &a, hipStream_t st) {
  int lanes = 1;
  while (lanes < 64 && lanes < a.N / kVec) lanes *= 2;
  const int per = kStepThreads / lanes;
  k_scan_step<T, kVec><<<dim3((a.D + per - 1) / per, a.B), kStepThreads, 0, st>>>(a, lanes);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_step(const Scan &a, Dt dt, hipStream_t st) {
  // a channel's states start at a multiple of 16 bytes where N is one of four
  if (a.N % 4 == 0) return dt == Dt::BF16 ? launch_v<bf16, 4>(a, st) : launch_v<float, 4>(a, st);
  return dt == Dt::BF16 ? launch_v<bf16, 1>(a, st) : launch_v<float, 1>(a, st);
}

}  // namespace favor
