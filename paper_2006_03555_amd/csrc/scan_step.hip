// scan_step.hip - one token of the selective scan for B sequences whose states stay in a pool:
//
//   h <- exp(s A) h + s x B,  y = (C h + skip x) silu(z)      h [D][N] fp32, in place
//
// Bound by the states' bytes, each read and written once (8 N bytes per channel), and nearly
// as much by what is done once per lane: softplus, silu and the turns. Neighbouring lanes
// share a channel, kVec states times kUnits each, so the state moves whole; their parts of y
// are joined by lane exchanges. 48 sequences x 4096 channels x 16 states, bf16, in a pool:
// 9.2 us (26.8 MB: 2.9 TB/s) with two units of four to a lane, 11.3 with one (twice the lanes
// that form softplus and silu) and 11.2 with four (a wave's load then takes 16 bytes of every
// 64); 12.9 with one and the loads behind the turns.
#include "recurrent.hpp"
#include "vec_rows.hpp"

namespace favor {
namespace {

constexpr int kStepThreads = 256;

template <int kVec> struct Floats;
template <> struct Floats<4> { using type = f32x4; };
template <> struct Floats<1> { typedef float type __attribute__((ext_vector_type(1))); };

template <typename T, int kVec, int kUnits>
__global__ __launch_bounds__(kStepThreads) void k_scan_step(Scan a, int lanes) {
  using V = typename Floats<kVec>::type;
  __shared__ int next;
  const int tid = threadIdx.x, unit0 = tid % lanes, units = a.N / kVec;
  const int d = blockIdx.x * (kStepThreads / lanes) + tid / lanes;
  const int first = blockIdx.y;
  const bool channel = d < a.D;
  const int dc = channel ? d : a.D - 1, g = dc / (a.D / a.G);
  // B and C begin at any element
  typedef T Low __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
  struct Unit {
    V h, A;
    Low B, C;
  };
  const float *A = a.A + (int64_t)dc * a.N;
  for (int b = first; b < a.B;) {
    const int slot = a.slots ? a.slots[b] : b;
    const bool live = slot >= 0 && slot < a.n_slots;   // others have no state: y = 0
    float *h = a.h_out + ((int64_t)slot * a.D + dc) * a.N;
    const T *B = static_cast<const T *>(a.b) + b * a.bs.b + g * a.bs.h;
    const T *C = static_cast<const T *>(a.c) + b * a.cs.b + g * a.cs.h;
    const auto request = [&](Unit &u, int i) {   // where there is no state A stands in
      const int at = i < units ? i * kVec : 0;
      u.h = *reinterpret_cast<const V *>((live ? h : A) + at);
      u.A = *reinterpret_cast<const V *>(A + at);
      u.B = *reinterpret_cast<const Low *>(B + at);
      u.C = *reinterpret_cast<const Low *>(C + at);
    };
    // everything is asked for before the turns are known: the sequences that share a place are
    // all this workgroup's, or it returns without a write
    Unit us[kUnits];
#pragma unroll
    for (int j = 0; j < kUnits; ++j) request(us[j], unit0 + j * lanes);
    const float x = to_f32(static_cast<const T *>(a.x)[b * a.xs.b + dc]);
    float s = to_f32(static_cast<const T *>(a.dt)[b * a.dts.b + dc]);
    const float bias = a.bias ? a.bias[dc] : 0.f, skip = a.skip ? a.skip[dc] : 0.f;
    const float z = a.z ? to_f32(static_cast<const T *>(a.z)[b * a.zs.b + dc]) : 0.f;
    int after = a.B;
    if (a.slots && live) {
      after = next_turn<kStepThreads>(a.slots, a.B, b, first, slot, &next);
      if (after < 0) return;
    }
    float y = 0.f;
    if (live) {
      s += bias;
      if (a.softplus) s = softplus(s);
      const float sx = s * x;
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
        const int i = unit0 + j * lanes;
        if (i >= units) break;
        Unit &u = us[j];
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          u.h[k] = fmaf(exp2_hw(s * (kLog2e * u.A[k])), u.h[k], sx * to_f32(u.B[k]));
          y = fmaf(to_f32(u.C[k]), u.h[k], y);
        }
        if (channel) *reinterpret_cast<V *>(h + i * kVec) = u.h;
      }
      for (int m = 1; m < lanes; m *= 2) y += __shfl_xor(y, m);
      y = fmaf(skip, x, y);
      if (a.z) y *= z * sigmoid(z);
    }
    if (channel && unit0 == 0) static_cast<T *>(a.y)[b * a.ys.b + dc] = from_f32<T>(y);
    b = after;
  }
}

template <typename T, int kVec, int kUnits> hipError_t launch_v(const Scan &a, hipStream_t st) {
  int lanes = 1;
  while (lanes * kUnits * kVec < a.N) lanes *= 2;
  const int per = kStepThreads / lanes;
  k_scan_step<T, kVec, kUnits>
      <<<dim3((a.D + per - 1) / per, a.B), kStepThreads, 0, st>>>(a, lanes);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_step(const Scan &a, Dt dt, hipStream_t st) {
  // a channel's states start at a multiple of 16 bytes where N is one of four
  if (a.N % 4 == 0)
    return dt == Dt::BF16 ? launch_v<bf16, 4, 2>(a, st) : launch_v<float, 4, 2>(a, st);
  return dt == Dt::BF16 ? launch_v<bf16, 1, 4>(a, st) : launch_v<float, 1, 4>(a, st);
}

}  // namespace favor
