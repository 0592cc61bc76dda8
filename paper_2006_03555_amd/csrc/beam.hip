// beam.hip - beam search's step: the best n of an entry's K V continuations, and the states of
// a pool moved behind the beams they belong to.
//
//   score(k, v) = scores[k] + x[k][v] - log sum_u exp x[k][u]
//
// Selection is bound by reading the logits once. A wave streams one piece of a row: running
// maximum and sum of exponentials per lane, and the piece's best n as 64-bit keys (the logit's
// order, then the lower token), one per lane. What is not above the worst kept key needs one
// comparison; the first tile, which has nothing to compare with, takes the least of n group
// maxima as its bound. A second launch joins the pieces of each beam and the beams of each
// entry. A lane's tokens and the order of its sums depend on the row's length alone, so equal
// rows have equal scores wherever they lie in memory. Scores are compared in 64 bits.
#include "recurrent.hpp"
#include "vec_rows.hpp"

namespace favor {
namespace {

constexpr int kMaxN = 64;
constexpr int kCandidates = 256;   // of one tile, before it is taken in parts
constexpr int kPieceWaves = 4;

// Whole numbers in the order of the floats (-0 as 0); 0 is below every one of them.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t key_of(float x, int token) {
  return (uint64_t)ordered(x) << 32 | (uint32_t)~token;
}
__device__ __forceinline__ uint64_t read_lane(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
// Orders a wave's LDS accesses against its own later ones.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The n best keys of a wave: lane r has the r-th (0: none).
struct WaveBest {
  uint64_t *list, *sorted;   // LDS of this wave: kCandidates + kMaxN, kMaxN
  uint64_t top = 0, last = 0;
  int n;

  // Joins `count` <= kCandidates keys, all other than those kept and unlike, from `list`.
  __device__ __forceinline__ void join(int count) {
    const int lane = threadIdx.x % 64;
    const int have = __popcll(__ballot(top != 0));
    if (top) list[count + lane] = top;
    wave_fence();
    const int total = count + have;
    for (int i0 = 0; i0 < total; i0 += 64) {
      const int i = i0 + lane;
      const uint64_t mine = i < total ? list[i] : 0;
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < total; ++j) rank += list[j] > mine;
      if (i < total && rank < n) sorted[rank] = mine;
    }
    wave_fence();
    top = lane < min(n, total) ? sorted[lane] : 0;
    wave_fence();
    last = read_lane(top, n - 1);
  }
  // One key per lane (0: none).
  __device__ __forceinline__ void push(uint64_t key) {
    const bool better = key > last;
    const uint64_t who = __ballot(better);
    if (!who) return;
    if (better) list[__popcll(who & ((1ull << (threadIdx.x % 64)) - 1))] = key;
    join(__popcll(who));
  }
};

template <typename T> __device__ __forceinline__ void load_logits(const T *p, float *x) {
  RowVec<T, 8> r;   // rows start anywhere: the hardware takes any alignment
  __builtin_memcpy(&r, p, sizeof(r));
  r.get(x);
}

template <typename T, int E>
__global__ __launch_bounds__(64 * kPieceWaves) void k_beam_pieces(BeamSelect a) {
  __shared__ uint64_t lists[kPieceWaves][kCandidates + 2 * kMaxN];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int64_t id = (int64_t)blockIdx.x * kPieceWaves + wave;
  const int row = (int)(id / a.pieces), piece = (int)(id - (int64_t)row * a.pieces);
  if (row >= a.B * a.K || (a.ended && a.ended[row])) return;
  const T *x0 = static_cast<const T *>(a.logits) + row / a.K * a.ls.b + row % a.K * a.ls.h;
  const int begin = piece * a.piece_len, end = min(begin + a.piece_len, a.V);
  WaveBest best;
  best.list = lists[wave];
  best.sorted = lists[wave] + kCandidates + kMaxN;
  best.n = a.n;
  float m = -INFINITY, sum = 0.f;
  for (int64_t t0 = begin; t0 < end; t0 += 64 * E) {
    float x[E];
    const bool whole = t0 + 64 * E <= end;
#pragma unroll
    for (int v = 0; v < E / 8; ++v) {
      const int64_t t = t0 + 512 * v + 8 * lane;
      if (whole) load_logits(x0 + t, x + 8 * v);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) x[8 * v + i] = t + i < end ? to_f32(x0[t + i]) : -INFINITY;
    }
    float most = x[0];
#pragma unroll
    for (int i = 1; i < E; ++i) most = fmaxf(most, x[i]);
    // a piece of -Inf alone has the sum 0, one with a NaN or +Inf the sum NaN
    const float higher = fmaxf(m, most), ref = higher == -INFINITY ? 0.f : higher;
    sum *= exp2_hw((m - ref) * kLog2e);
#pragma unroll
    for (int i = 0; i < E; ++i) sum += exp2_hw((x[i] - ref) * kLog2e);
    m = higher;
    float bound = best.last ? unordered((uint32_t)(best.last >> 32)) : -INFINITY;
    if (t0 == begin) {
      int groups = 1;
      while (groups < a.n) groups *= 2;
      bound = most;
      for (int d = groups; d < 64; d *= 2) bound = fmaxf(bound, __shfl_xor(bound, d));
      for (int d = 1; d < groups; d *= 2) bound = fminf(bound, __shfl_xor(bound, d));
    }
    if (!__ballot(most >= bound)) continue;
    int count = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int token = (int)(t0 + 512 * (i / 8) + 8 * lane + i % 8);
      const bool in = x[i] >= bound && (whole || token < end);
      const uint64_t who = __ballot(in);
      if (!who) continue;
      const int at = count + __popcll(who & ((1ull << lane) - 1));
      if (in && at < kCandidates) best.list[at] = key_of(x[i], token);
      count += __popcll(who);
    }
    if (count <= kCandidates) {
      if (count) best.join(count);
    } else {   // a row of many equal or rising logits
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int token = (int)(t0 + 512 * (i / 8) + 8 * lane + i % 8);
        best.push(whole || token < end ? key_of(x[i], token) : 0);
      }
    }
  }
  float top = m;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  double total = (double)sum * exp2_hw((m - (top == -INFINITY ? 0.f : top)) * kLog2e);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d);
  if (lane == 0) a.stats[id] = float2{top, (float)total};
  if (lane < a.n) a.keys[id * a.n + lane] = best.top;
}

// A workgroup per entry: a wave joins the pieces of a beam, then each candidate finds its rank
// among all beams' (in a sorted list by halving).
constexpr int kMergeWaves = 8;
__global__ __launch_bounds__(64 * kMergeWaves) void k_beam_merge(BeamSelect a) {
  __shared__ uint64_t lists[kMergeWaves][kCandidates + 2 * kMaxN];
  extern __shared__ double score[];   // [K][n], best first
  int *token = reinterpret_cast<int *>(score + a.K * a.n), *count = token + a.K * a.n;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, b = blockIdx.x, n = a.n;
  for (int k = wave; k < a.K; k += kMergeWaves) {
    const int64_t row = (int64_t)b * a.K + k;
    const double own = a.scores[row];
    if (a.ended && a.ended[row]) {
      if (lane == 0) {
        score[k * n] = own;
        token[k * n] = a.end_token;
        count[k] = own - own == 0.0;   // finite
      }
      continue;
    }
    const float2 st = lane < a.pieces ? a.stats[row * a.pieces + lane] : float2{-INFINITY, 0.f};
    float top = st.x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    double sum = (double)st.y * exp2_hw((st.x - (top == -INFINITY ? 0.f : top)) * kLog2e);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    const double rest = log(sum);   // of the log-sum, beyond the maximum, which may be huge
    WaveBest best;
    best.list = lists[wave];
    best.sorted = lists[wave] + kCandidates + kMaxN;
    best.n = n;
    const int keys = a.pieces * n;
    for (int i = lane; i - lane < keys; i += 64)
      best.push(i < keys ? a.keys[row * keys + i] : 0);
    const float x = unordered((uint32_t)(best.top >> 32));
    const double s = own + (((double)x - top) - rest);
    const bool offered = best.top && s - s == 0.0;
    if (offered) {
      score[k * n + lane] = s;
      token[k * n + lane] = (int)~(uint32_t)best.top;
    }
    const int c = __popcll(__ballot(offered));   // the first c: scores fall
    if (lane == 0) count[k] = c;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.K * n; i += 64 * kMergeWaves) {
    const int k = i / n, r = i - k * n;
    if (r >= count[k]) continue;
    const double s = score[i];
    int rank = r;
    for (int o = 0; o < a.K; ++o) {
      if (o == k) continue;
      int lo = 0, hi = count[o];   // those before: higher, or as high of an earlier beam
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        const double v = score[o * n + mid];
        if (v > s || (v == s && o < k)) lo = mid + 1;
        else hi = mid;
      }
      rank += lo;
    }
    if (rank >= n) continue;
    a.out_scores[b * n + rank] = (float)s;
    a.parent[b * n + rank] = k;
    a.token[b * n + rank] = token[i];
  }
  int total = 0;
  for (int k = 0; k < a.K; ++k) total += count[k];
  for (int i = total + threadIdx.x; i < n; i += 64 * kMergeWaves) {   // too few to choose from
    a.out_scores[b * n + i] = -INFINITY;
    a.parent[b * n + i] = 0;
    a.token[b * n + i] = max(a.end_token, 0);
  }
}

// Copies of the states of beams with more than one child. The first child takes its parent's
// place; the others, in order, take the places of beams without children, in order. So a
// state that is read stays as it is, and no two copies write one place. Bound by the bytes of
// the states that are copied. Each wave works the whole plan of its entry out anew: K <= 64
// parents are one load and a few ballots.
constexpr int kCopyThreads = 256;
__global__ __launch_bounds__(kCopyThreads) void k_beam_reorder(BeamReorder a) {
  const int lane = threadIdx.x % 64, j = blockIdx.y % a.K, b = blockIdx.y / a.K;
  int parent = -1;
  if (lane < a.K) {
    parent = a.parent[(int64_t)b * a.K + lane];
    if (parent < 0 || parent >= a.K) parent = -1;   // continues nothing
  }
  const int mine = __builtin_amdgcn_readlane(parent, j);
  const uint64_t same = __ballot(parent == mine) & ((1ull << j) - 1);
  const int base = b * a.K;
  const bool keeps = mine >= 0 && !same;   // the first child
  if (keeps && blockIdx.x) return;
  int place;
  if (keeps) {
    place = mine;
  } else {
    // this beam is the `extra`-th without a place, and takes that one of the free ones
    uint64_t used = 0;
    int extra = 0;
    for (int i = 0; i < a.K; ++i) {
      const int p = __builtin_amdgcn_readlane(parent, i);
      const bool first = p >= 0 && !(used >> p & 1);
      if (first) used |= 1ull << p;
      else if (i < j) ++extra;
    }
    place = 0;
    for (int i = 0; i < a.K; ++i)
      if (!(used >> i & 1) && extra-- == 0) place = i;
  }
  const int to = a.slots ? a.slots[base + place] : base + place;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.new_slots[base + j] = to;
  if (keeps || mine < 0 || !a.n_pools) return;
  int lo = 0, hi = a.n_pools;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.first[mid] <= (int)blockIdx.x) lo = mid;
    else hi = mid;
  }
  const int from = a.slots ? a.slots[base + mine] : base + mine;
  const int n_slots = a.pool[lo].n_slots, units = a.pool[lo].units;
  if (from < 0 || from >= n_slots || to < 0 || to >= n_slots) return;
  const int64_t u0 = (int64_t)(blockIdx.x - a.first[lo]) * kBeamPieceUnits;
  const int count = (int)min((int64_t)kBeamPieceUnits, units - u0);
  const float4 *src = a.pool[lo].data + (int64_t)from * units + u0;
  float4 *dst = a.pool[lo].data + (int64_t)to * units + u0;
  int i = threadIdx.x;
  for (; i + 3 * kCopyThreads < count; i += 4 * kCopyThreads) {
    float4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = src[i + k * kCopyThreads];
#pragma unroll
    for (int k = 0; k < 4; ++k) dst[i + k * kCopyThreads] = v[k];
  }
  for (; i < count; i += kCopyThreads) dst[i] = src[i];
}

template <typename T> hipError_t launch_pieces_as(const BeamSelect &a, hipStream_t st) {
  const int64_t waves = (int64_t)a.B * a.K * a.pieces;
  const unsigned blocks = (unsigned)((waves + kPieceWaves - 1) / kPieceWaves);
  if (a.piece_len >= 2048) k_beam_pieces<T, 32><<<blocks, 64 * kPieceWaves, 0, st>>>(a);
  else k_beam_pieces<T, 8><<<blocks, 64 * kPieceWaves, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_beam_pieces(const BeamSelect &a, Dt dt, hipStream_t st) {
  return dt == Dt::BF16 ? launch_pieces_as<bf16>(a, st) : launch_pieces_as<float>(a, st);
}

hipError_t launch_beam_merge(const BeamSelect &a, hipStream_t st) {
  const size_t lds = (size_t)a.K * a.n * (sizeof(double) + sizeof(int)) + a.K * sizeof(int);
  if (lds > 32768) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(k_beam_merge),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  k_beam_merge<<<a.B, 64 * kMergeWaves, lds, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const BeamReorder &a, hipStream_t st) {
  const int pieces = a.n_pools ? a.first[a.n_pools] : 0;
  k_beam_reorder<<<dim3(pieces > 0 ? pieces : 1, a.B * a.K), kCopyThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace favor
