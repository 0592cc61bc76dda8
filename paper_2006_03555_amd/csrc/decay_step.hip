// decay_step.hip - one token of linear attention with a decay per head (decay.hip's
// recurrence as it stands), for B sequences whose states stay in a pool:
//
//   S <- a S + k v^T,   o = c q^T S     S [dk][dv] fp32, in place
//
// Bound by the states' bytes: each is read and written once (8 dk dv bytes per head, 128
// KB at 128 x 128) and everything else is small. A workgroup takes one (sequence, head);
// a thread owns four value columns of every n-th row, so the state moves in 16-byte
// units, whole rows at a time; the threads' parts of o are summed in a fixed order.
// 1024 sequences x 16 heads at 128 x 128 (2.1 GB) take 412 us, 5.2 TB/s (a copy on this card:
// 4.95). 48 sequences (101 MB) repeated on the same states, which then stay in the memory-side
// cache, take 16.6 us, 6.1 TB/s, and 18.4 us, 5.5 TB/s, where new ones come from call to
// call. One sequence of 8 heads takes 4.0 us in a graph (traced alone 4.9), most of it the
// launch and one round of loads.
#include "decay.hpp"
#include "favor_common.hpp"

namespace favor {
namespace {

constexpr int kStepThreads = 256;
constexpr int kMaxD = 256;

template <typename T>
__global__ __launch_bounds__(kStepThreads) void k_decay_step(DecayStep a) {
  __shared__ float qk[2][kMaxD];
  __shared__ __align__(16) f32x4 part[kStepThreads];
  __shared__ int next;
  const int h = blockIdx.x % a.H;
  const int tid = threadIdx.x;
  const int units = a.dv / 4, groups = kStepThreads / units;
  const int unit = tid % units, group = tid / units;
  // a as two floats: one's rounding, the same at every token, would add up over a long memory
  // (8192 tokens: states up to 1.3e-4 off instead of 1.5e-5 at most; 48 sequences 18.4 us
  // instead of 18.2)
  const double decay = exp((double)a.log_decay[h]);
  const float lam = (float)decay, low = lam < INFINITY ? (float)(decay - lam) : 0.f;
  for (int b = blockIdx.x / a.H; b < a.B;) {
    // sequences that share a place take their turns in order, by the first one's
    // workgroup: find an earlier one (this workgroup has nothing to do) and the next
    int slot = b, after = a.B;
    if (a.slots) {
      slot = a.slots[b];
      __syncthreads();
      if (tid == 0) next = a.B;
      __syncthreads();
      if (slot >= 0 && slot < a.n_slots) {
        int mine = a.B;
        bool earlier = false;
        for (int i = tid; i < a.B; i += kStepThreads)
          if (a.slots[i] == slot) {
            if (i > b) mine = min(mine, i);
            earlier |= i < b && b == (int)(blockIdx.x / a.H);
          }
        if (mine < a.B) atomicMin(&next, mine);
        if (__syncthreads_or(earlier)) return;
        after = next;
      }
    }
    const bool live = slot >= 0 && slot < a.n_slots;   // others have no state: o = 0
    for (int i = tid; i < a.dk; i += kStepThreads) {
      qk[0][i] = to_f32(static_cast<const T *>(a.q)[b * a.qs.b + h * a.qs.h + i]);
      qk[1][i] = to_f32(static_cast<const T *>(a.k)[b * a.ks.b + h * a.ks.h + i]);
    }
    __syncthreads();
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    if (live && group < groups) {
      const T *vp = static_cast<const T *>(a.v) + b * a.vs.b + h * a.vs.h + 4 * unit;
      f32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = to_f32(vp[j]);
      f32x4 *sp = reinterpret_cast<f32x4 *>(a.state + ((size_t)slot * a.H + h) * a.dk * a.dv) + unit;
#pragma unroll 8
      for (int r = group; r < a.dk; r += groups) {
        f32x4 s = sp[(size_t)r * units];
        const float kr = qk[1][r], qr = qk[0][r];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[j] = fmaf(s[j], lam, fmaf(s[j], low, kr * v[j]));
          o[j] = fmaf(qr, s[j], o[j]);
        }
        sp[(size_t)r * units] = s;
      }
    }
    part[tid] = o;
    __syncthreads();
    if (tid < units) {
      for (int i = 1; i < groups; ++i) {
        const f32x4 p = part[i * units + tid];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += p[j];
      }
      T *op = static_cast<T *>(a.o) + b * a.os.b + h * a.os.h + 4 * tid;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] *= a.scale;
      store4(op, o);
    }
    b = after;
  }
}

}  // namespace

hipError_t launch_decay_step(const DecayStep &a, Dt dt, hipStream_t st) {
  if (dt == Dt::BF16) k_decay_step<bf16><<<a.B * a.H, kStepThreads, 0, st>>>(a);
  else k_decay_step<float><<<a.B * a.H, kStepThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace favor
