// vec_rows.hpp - V contiguous elements of a row as floats, and the turns of sequences that
// share a place in a pool (device code).
#pragma once

#include "favor_common.hpp"

namespace favor {

template <typename T, int V> struct RowVec;   // raw registers of V elements
template <> struct RowVec<bf16, 8> {
  uint4 r;
  __device__ __forceinline__ void load(const bf16 *p) { r = *reinterpret_cast<const uint4 *>(p); }
  __device__ __forceinline__ void zero() { r = uint4{0, 0, 0, 0}; }
  __device__ __forceinline__ void get(float *v) const {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
template <> struct RowVec<bf16, 4> {
  uint2 r;
  __device__ __forceinline__ void load(const bf16 *p) { r = *reinterpret_cast<const uint2 *>(p); }
  __device__ __forceinline__ void zero() { r = uint2{0, 0}; }
  __device__ __forceinline__ void get(float *v) const {
    v[0] = __uint_as_float(r.x << 16);
    v[1] = __uint_as_float(r.x & 0xffff0000u);
    v[2] = __uint_as_float(r.y << 16);
    v[3] = __uint_as_float(r.y & 0xffff0000u);
  }
};
template <> struct RowVec<float, 4> {
  float4 r;
  __device__ __forceinline__ void load(const float *p) { r = *reinterpret_cast<const float4 *>(p); }
  __device__ __forceinline__ void zero() { r = float4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void get(float *v) const {
    v[0] = r.x;
    v[1] = r.y;
    v[2] = r.z;
    v[3] = r.w;
  }
};
template <> struct RowVec<float, 8> {
  float4 r[2];
  __device__ __forceinline__ void load(const float *p) {
    r[0] = reinterpret_cast<const float4 *>(p)[0];
    r[1] = reinterpret_cast<const float4 *>(p)[1];
  }
  __device__ __forceinline__ void zero() { r[0] = r[1] = float4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void get(float *v) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v[4 * i] = r[i].x;
      v[4 * i + 1] = r[i].y;
      v[4 * i + 2] = r[i].z;
      v[4 * i + 3] = r[i].w;
    }
  }
};

template <int V, typename T> __device__ __forceinline__ void store_row(T *p, const float *v) {
  if constexpr (V == 8) store8(p, f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]});
  else store4(p, f32x4{v[0], v[1], v[2], v[3]});
}

__device__ __forceinline__ int clamped_length(const int32_t *lengths, int b, int L) {
  return lengths ? min(max(lengths[b], 0), L) : L;
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 2^x and 1/x by the hardware's instructions (within 1 ulp; results below 2^-126 are 0).
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_hw(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float sigmoid(float x) { return rcp_hw(1.f + exp2_hw(-kLog2e * x)); }

// max(x, 0) + log(1 + e), e = exp(-|x|). With u = 1 + e as rounded, log(1 + e) is log(u) + (what
// the rounding left of e) / u, and u is 1 where that matters; so as e falls it is as precise as e
// itself, whose exponent's rounding is |x| 2^-24 of it (80 units at x = -80). 0 at -Inf; a NaN comes
// through e.
__device__ __forceinline__ float softplus(float x) {
  const float e = exp2_hw(-kLog2e * fabsf(x));
  const float u = 1.f + e;
  const float over = __builtin_amdgcn_fmed3f(x, 0.f, INFINITY);   // max(x, 0)
  return over + fmaf(kLn2, __builtin_amdgcn_logf(u), e - (u - 1.f));
}
// softplus' slope at x, of which s is softplus(x): e^x / (1 + e^x) = e^(x - s), within |x - s| 2^-24.
__device__ __forceinline__ float softplus_slope(float x, float s) { return exp2_hw(kLog2e * (x - s)); }

// Sequences that hold the same place of a pool take their turns in order, all in the first
// one's workgroup. Returns the sequence that follows b at its place (B: none), or -1 where b
// is `first`, the workgroup's own, and an earlier sequence has the place. For whole
// workgroups; `next` is one word of LDS.
template <int kThreads>
__device__ __forceinline__ int next_turn(const int32_t *slots, int B, int b, int first, int slot,
                                         int *next) {
  bool other = false, earlier = false;
  int mine = B;
  for (int i = threadIdx.x; i < B; i += kThreads)
    if (i != b && slots[i] == slot) {
      other = true;
      earlier |= i < b && b == first;
      if (i > b) mine = min(mine, i);
    }
  if (!__syncthreads_or(other)) return B;
  if (__syncthreads_or(earlier)) return -1;
  if (threadIdx.x == 0) *next = B;
  __syncthreads();
  if (mine < B) atomicMin(next, mine);
  __syncthreads();
  const int n = *next;
  __syncthreads();
  return n;
}

}  // namespace favor
