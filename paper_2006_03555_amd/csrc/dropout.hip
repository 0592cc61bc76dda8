// dropout.hip - y = residual + [bits >= threshold] x scale, the mask from a counter-based
// generator and never stored: the gradient's pass draws it again.
//
// Element n takes the 16 bits n % 8 of Philox4x32-10 (Salmon et al., SC'11) at counter
// n / 8, so that one call serves a thread's eight elements, a 16-byte unit in bf16. The share
// dropped is threshold / 2^16 and the scale is its own reciprocal, so the expectation is
// exact.
//
// Bound by the bytes: 16384 x 2048 bf16 elements take 30 us with a residual and 21 without
// when repeated on the same rows (6.8 and 6.4 TB/s, the memory-side cache's help), 64 us both
// on new rows (5.3 TB/s; a copy on this card: 4.95). With 32 bits per element 66 us.
#include "decay.hpp"
#include "favor_common.hpp"

namespace favor {
namespace {

constexpr int kDropThreads = 256;

__device__ __forceinline__ void philox4x32(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)c[0] * 0xD2511F53u, p1 = (uint64_t)c[2] * 0xCD9E8D57u;
    c[0] = (uint32_t)(p1 >> 32) ^ c[1] ^ k0;
    c[1] = (uint32_t)p1;
    c[2] = (uint32_t)(p0 >> 32) ^ c[3] ^ k1;
    c[3] = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

template <typename T>
__global__ __launch_bounds__(kDropThreads) void k_dropout(Dropout a) {
  const uint64_t seed = a.rng ? a.rng[0] : a.seed, offset = a.rng ? a.rng[1] : a.offset;
  const int64_t calls = (a.n + 7) / 8;
  const T *x = static_cast<const T *>(a.x), *res = static_cast<const T *>(a.residual);
  T *y = static_cast<T *>(a.y);
  for (int64_t i = (int64_t)blockIdx.x * kDropThreads + threadIdx.x; i < calls;
       i += (int64_t)gridDim.x * kDropThreads) {
    const int m = (int)min((int64_t)8, a.n - 8 * i);
    float v[8], r[8];
    if (m == 8) {
      load8_f32(x + 8 * i, v);
      if (res) load8_f32(res + 8 * i, r);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = j < m ? to_f32(x[8 * i + j]) : 0.f;
        r[j] = j < m && res ? to_f32(res[8 * i + j]) : 0.f;
      }
    }
    uint32_t w[4] = {(uint32_t)i, (uint32_t)((uint64_t)i >> 32), (uint32_t)offset,
                     (uint32_t)(offset >> 32)};
    philox4x32(w, (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t bits = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu;
      v[j] = bits >= a.threshold ? v[j] * a.scale : 0.f;   // a dropped NaN is gone
      if (res) v[j] += r[j];
    }
    if (m == 8) {
      store8(y + 8 * i, f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]});
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < m) y[8 * i + j] = from_f32<T>(v[j]);
    }
  }
}

}  // namespace

hipError_t launch_dropout(const Dropout &a, Dt dt, hipStream_t st) {
  const int64_t calls = (a.n + 7) / 8;
  const int64_t groups = (calls + kDropThreads - 1) / kDropThreads;
  const int grid = (int)(groups < 8192 ? groups : 8192);
  if (dt == Dt::BF16) k_dropout<bf16><<<grid, kDropThreads, 0, st>>>(a);
  else k_dropout<float><<<grid, kDropThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace favor
