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
// entry. A lane's tokens and the order of its sums depend on V and the number of rows alone, so
// in one call equal rows have equal scores wherever they lie in memory (a batch of another size
// may cut rows into other pieces, and round their sums otherwise). Scores are compared in 64 bits.
// 32 entries of 8 beams of 131072 logits in bf16, a quarter of them ended: 21 us (2.5 TB/s) and 8
// for the merge; 4 beams of 50001 in fp32: 5.1 and 5.7, all latency. Masked logits cost no more than
// others: 32 x 8 x 131072 with both launches 29 us, 22 with all but 16 of a row at -Inf, 32 at the
// type's lowest value.
#include <cfloat>

#include "recurrent.hpp"
#include "vec_rows.hpp"

namespace favor {
namespace {

constexpr int kMaxN = 64;
constexpr int kCandidates = 256;   // of one tile, before it is taken in parts
constexpr int kPieceWaves = 4;
constexpr int kFew = 12;           // candidates that are put in one by one

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
// The wave's number as a scalar: what follows from it is the same in all lanes.
__device__ __forceinline__ int uniform_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }
// The lanes of `who` before this one.
__device__ __forceinline__ int before(uint64_t who) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
}
// Orders a wave's LDS accesses against its own later ones.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The largest of three, without the care for signalling NaNs.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// v of the lane and of its partner at distance kDistance, in either order, where blocks of
// kDistance lanes hold one value each (a mirror then is as good as an exchange).
template <int kDistance> __device__ __forceinline__ void partners(uint32_t v, uint32_t &a, uint32_t &b) {
  if constexpr (kDistance >= 16) {
    const auto r = kDistance == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false)
                                   : __builtin_amdgcn_permlane32_swap(v, v, false, false);
    a = r[0];
    b = r[1];
  } else {
    constexpr int kControl = kDistance == 1 ? 0xb1 : kDistance == 2 ? 0x4e : kDistance == 4 ? 0x141 : 0x140;
    a = v;
    b = __builtin_amdgcn_update_dpp(0, v, kControl, 0xf, 0xf, true);
  }
}
template <int kDistance, typename F> __device__ __forceinline__ float with_partner(float v, F &&f) {
  uint32_t a, b;
  partners<kDistance>(__float_as_uint(v), a, b);
  return f(__uint_as_float(a), __uint_as_float(b));
}
template <int kDistance> __device__ __forceinline__ double add_partner(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  uint32_t a0, b0, a1, b1;
  partners<kDistance>((uint32_t)u, a0, b0);
  partners<kDistance>((uint32_t)(u >> 32), a1, b1);
  return __builtin_bit_cast(double, (uint64_t)a1 << 32 | a0) + __builtin_bit_cast(double, (uint64_t)b1 << 32 | b0);
}
// Over the wave, step by step: f(distance, own, partner's).
template <typename F> __device__ __forceinline__ float over_wave(float v, F &&f) {
  v = with_partner<1>(v, [&](float a, float b) { return f(1, a, b); });
  v = with_partner<2>(v, [&](float a, float b) { return f(2, a, b); });
  v = with_partner<4>(v, [&](float a, float b) { return f(4, a, b); });
  v = with_partner<8>(v, [&](float a, float b) { return f(8, a, b); });
  v = with_partner<16>(v, [&](float a, float b) { return f(16, a, b); });
  return with_partner<32>(v, [&](float a, float b) { return f(32, a, b); });
}
__device__ __forceinline__ float wave_max(float v) {
  return over_wave(v, [](int, float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ double wave_sum(double v) {
  return add_partner<32>(add_partner<16>(add_partner<8>(add_partner<4>(add_partner<2>(add_partner<1>(v))))));
}
// Maxima whose product with log2 e is rounded by at most 64: 2 to what that leaves is in range.
// Past them (a mask of -1e10 or of the type's lowest value) the maximum is taken off before the
// product; neighbouring floats are 64 or more apart there, so all but the maximum itself adds
// nothing.
constexpr float kScaled = 0x1p30f;
__device__ __forceinline__ float scaled_to(float m) { return fminf(fmaxf(m, -kScaled), kScaled); }
__device__ __forceinline__ float scaled(float m) { return scaled_to(m) * kLog2e; }
__device__ __forceinline__ bool past_scaled(float m) {   // and finite
  constexpr uint32_t from = 2 * 0x4e800000u + 1, to = 2 * 0x7f800000u;   // by twice the bits of 2^30, of Inf
  return 2 * __float_as_uint(m) - from < to - from;
}

// The n best keys of a wave: lane r has the r-th (0: none).
struct WaveBest {
  uint64_t *list, *sorted;   // LDS of this wave: kCandidates + kMaxN + 8, kMaxN
  uint64_t top = 0, last = 0;
  int n;

  // Joins `count` <= kCandidates keys, all other than those kept and unlike, from `list`.
  __device__ __forceinline__ void join(int count) {
    const int lane = threadIdx.x % 64;
    const int have = __popcll(__ballot(top != 0));
    const int total = count + have;
    if (top) list[count + lane] = top;
    if (lane < 8) list[total + lane] = 0;   // whole groups of eight are read below
    wave_fence();
    for (int i0 = 0; i0 < total; i0 += 64) {
      const int i = i0 + lane;
      const uint64_t mine = i < total ? list[i] : 0;
      int rank = 0;
      for (int j = 0; j < total; j += 8)
#pragma unroll
        for (int k = 0; k < 8; ++k) rank += list[j + k] > mine;
      if (i < total && rank < n) sorted[rank] = mine;
    }
    wave_fence();
    top = lane < min(n, total) ? sorted[lane] : 0;
    wave_fence();
    last = read_lane(top, n - 1);
  }
  // One key, the same in all lanes: those behind it move on by a lane.
  __device__ __forceinline__ void insert(uint64_t key) {
    if (key <= last) return;
    const int rank = __popcll(__ballot(top > key)), lane = threadIdx.x % 64;
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)top, 0x138, 0xf, 0xf, false);   // wave_shr:1
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(top >> 32), 0x138, 0xf, 0xf, false);
    if (lane > rank) top = (uint64_t)hi << 32 | lo;
    if (lane == rank) top = key;
    if (lane >= n) top = 0;
    last = read_lane(top, n - 1);
  }
  // One key per lane (0: none).
  __device__ __forceinline__ void push(uint64_t key) {
    const bool better = key > last;
    const uint64_t who = __ballot(better);
    if (!who) return;
    if (better) list[before(who)] = key;
    join(__popcll(who));
  }
};

// E logits per lane and tile; the next tile is requested before this one is looked at.
template <typename T, int E>
__global__ __launch_bounds__(64 * kPieceWaves) void k_beam_pieces(BeamSelect a) {
  __shared__ uint64_t lists[kPieceWaves][kCandidates + 2 * kMaxN + 8];
  constexpr int kTile = 64 * E;
  const int wave = uniform_wave(), lane = threadIdx.x % 64;
  const int of_row = (a.pieces + kPieceWaves - 1) / kPieceWaves;
  const int row = blockIdx.x / of_row, piece = blockIdx.x % of_row * kPieceWaves + wave;
  if (piece >= a.pieces || (a.ended && a.ended[row])) return;
  const int64_t id = (int64_t)row * a.pieces + piece;
  const int begin = piece * a.piece_len, left = min(a.piece_len, a.V - begin);
  const T *x0 = static_cast<const T *>(a.logits) + row / a.K * a.ls.b + row % a.K * a.ls.h + begin + 8 * lane;
  WaveBest best;
  best.list = lists[wave];
  best.sorted = lists[wave] + kCandidates + kMaxN + 8;
  best.n = a.n;
  // sum of 2^(x log2 e - c), c = m log2 e as rounded: one fused multiply-add before each
  // exponential. A NaN makes the sum one, +Inf makes it infinite.
  float m = -INFINITY, c = -INFINITY, sum = 0.f;
  const auto look = [&](const float (&x)[E], int t0) {   // a tile's values, -Inf behind the piece
    float most = max3(x[0], x[1], x[2]);
#pragma unroll
    for (int i = 3; i + 1 < E; i += 2) most = max3(most, x[i], x[i + 1]);
    most = max3(most, x[E - 1], x[E - 1]);
    const float was = m;
    m = max3(m, most, most);
    const float now = scaled(m);
    if (!__ballot(past_scaled(m))) {
      sum *= exp2_hw(c - now);
#pragma unroll
      for (int i = 0; i < E; ++i) sum += exp2_hw(fmaf(x[i], kLog2e, -now));
      c = now;
    } else {
      const bool past = past_scaled(m);
      sum *= exp2_hw(past ? (was - m) * kLog2e : c - now);
#pragma unroll
      for (int i = 0; i < E; ++i) sum += exp2_hw(past ? (x[i] - m) * kLog2e : fmaf(x[i], kLog2e, -now));
      c = past ? -INFINITY : now;   // nothing beside a maximum that is not past it
    }
    // what a candidate reaches: more than the worst kept logit (an equal one of a later token comes
    // behind it), and a finite one (a mask of -Inf is never offered)
    float bound = best.last ? unordered((uint32_t)(best.last >> 32) + 1) : -FLT_MAX;
    if (t0 == 0) {
      int group = 64;   // lanes of one of n groups or more
      while (64 / group < a.n) group /= 2;
      bound = over_wave(most, [&](int d, float u, float v) { return d < group ? fmaxf(u, v) : fminf(u, v); });
      bound = fmaxf(bound, -FLT_MAX);
    }
    if (!__ballot(most >= bound)) return;
    int count = 0;
    const int t1 = begin + t0 + 8 * lane;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const bool in = x[i] >= bound;   // (tokens behind the piece are -Inf)
      const uint64_t who = __ballot(in);
      if (!who) continue;
      const int at = count + before(who);
      if (in && at < kCandidates) best.list[at] = key_of(x[i], t1 + 512 * (i / 8) + i % 8);
      count += __popcll(who);
    }
    if (count <= kFew) {
      wave_fence();
      for (int i = 0; i < count; ++i) best.insert(best.list[i]);
      wave_fence();
    } else if (count <= kCandidates) {
      best.join(count);
    } else {   // a row of many equal or rising logits
      for (int i = 0; i < E; ++i) {
        const int t = t0 + 512 * (i / 8) + i % 8;
        const float v = 8 * lane + t < left ? to_f32(x0[t]) : -INFINITY;
        best.push(v >= bound ? key_of(v, begin + 8 * lane + t) : 0);
      }
    }
  };
  // Whole tiles, the next one requested before this one is looked at (two sets of registers in
  // turn, and requests without conditions: the last ones ask for a tile once more; a copy or a
  // choice would wait for them). Rows start anywhere: any alignment will do.
  using Raw = RowVec<T, 8>[E / 8];
  const auto request = [&](Raw &to, int t0) {
    const T *p = x0 + min(t0, left - kTile);
#pragma unroll
    for (int v = 0; v < E / 8; ++v) __builtin_memcpy(&to[v], p + 512 * v, sizeof(to[v]));
  };
  const auto take = [&](const Raw &from, int t0) {
    float x[E];
#pragma unroll
    for (int v = 0; v < E / 8; ++v) from[v].get(x + 8 * v);
    look(x, t0);
  };
  int t0 = 0;
  if (left >= kTile) {
    Raw even, odd;
    request(even, 0);
    for (;;) {
      request(odd, t0 + kTile);
      take(even, t0);
      if ((t0 += kTile) + kTile > left) break;
      request(even, t0 + kTile);
      take(odd, t0);
      if ((t0 += kTile) + kTile > left) break;
    }
  }
  if (t0 < left) {
    float x[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int t = t0 + 512 * (i / 8) + i % 8;
      x[i] = 8 * lane + t < left ? to_f32(x0[t]) : -INFINITY;
    }
    look(x, t0);
  }
  const float top = wave_max(m);
  // what c's rounding left is in it
  sum *= exp2_hw(past_scaled(m) ? (m - top) * kLog2e : fmaf(-fmaxf(top, -kScaled), kLog2e, c));
  const double total = wave_sum(sum);
  if (lane == 0) a.stats[id] = float2{top, (float)total};
  if (lane < a.n) a.keys[id * a.n + lane] = best.top;
}

// A workgroup per entry: a wave joins the pieces of a beam, then each candidate finds its rank
// among all beams' (in a sorted list by halving).
constexpr int kMergeWaves = 8, kEarly = 8;
__global__ __launch_bounds__(64 * kMergeWaves) void k_beam_merge(BeamSelect a) {
  __shared__ uint64_t lists[kMergeWaves][kCandidates + 2 * kMaxN + 8];
  extern __shared__ double score[];   // [K][n], best first
  int *token = reinterpret_cast<int *>(score + a.K * a.n), *count = token + a.K * a.n;
  const int wave = uniform_wave(), lane = threadIdx.x % 64, b = blockIdx.x, n = a.n;
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
    // all that is small is requested at once: the pieces' statistics, their r-th keys, and as many
    // of the keys as most calls have
    const int keys = a.pieces * n, r = (n + a.pieces - 1) / a.pieces;
    const uint64_t *of_row = a.keys + row * keys;
    const float2 of_piece = a.stats[row * a.pieces + min(lane, a.pieces - 1)];
    const uint64_t rth = of_row[min(lane, a.pieces - 1) * n + r - 1];
    uint64_t early[kEarly];
#pragma unroll
    for (int j = 0; j < kEarly; ++j) early[j] = of_row[min(64 * j + lane, keys - 1)];
    const float2 st = lane < a.pieces ? of_piece : float2{-INFINITY, 0.f};
    const float top = wave_max(st.x);
    const double sum = wave_sum((double)st.y * exp2_hw((st.x - (top == -INFINITY ? 0.f : top)) * kLog2e));
    const double rest = log(sum);   // of the log-sum, beyond the maximum, which may be huge
    WaveBest best;
    best.list = lists[wave];
    best.sorted = lists[wave] + kCandidates + kMaxN + 8;
    best.n = n;
    // the k-th best of the pieces' r-th keys has r k >= n keys not below it: only those are joined
    WaveBest column = best;
    column.n = (n + r - 1) / r;
    column.push(lane < a.pieces ? rth : 0);
    const uint64_t bound = column.last ? column.last : 1;
    int held = 0;
    const auto take = [&](uint64_t key, int i0) {   // keys i0 .. i0 + 63 of the row
      const bool good = i0 + lane < keys && key >= bound;
      const uint64_t who = __ballot(good);
      if (good) best.list[held + before(who)] = key;
      held += __popcll(who);
      if (held <= kCandidates - 64 && i0 + 64 < keys) return;
      if (held) best.join(held);
      held = 0;
    };
#pragma unroll
    for (int j = 0; j < kEarly; ++j)
      if (64 * j < keys) take(early[j], 64 * j);
    for (int i0 = 64 * kEarly; i0 < keys; i0 += 64) take(of_row[min(i0 + lane, keys - 1)], i0);
    const float x = unordered((uint32_t)(best.top >> 32));
    const double s = own + (((double)x - top) - rest);
    const bool offered = best.top && fabsf((float)s) < INFINITY;   // as it is returned
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
// the states that are copied: 8 entries of 8 beams, 24 layers of 143 KB, 24 copies of each (165
// MB) 39 us, 4.2 TB/s. Each wave works the whole plan of its entry out anew: K <= 64 parents are
// one load and a few ballots.
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
  const f32x4 *src = static_cast<const f32x4 *>(a.pool[lo].data) + (int64_t)from * units + u0;
  f32x4 *dst = static_cast<f32x4 *>(a.pool[lo].data) + (int64_t)to * units + u0;
  int i = threadIdx.x;
  for (; i + 3 * kCopyThreads < count; i += 4 * kCopyThreads) {
    f32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = src[i + k * kCopyThreads];
#pragma unroll
    for (int k = 0; k < 4; ++k) dst[i + k * kCopyThreads] = v[k];
  }
  for (; i < count; i += kCopyThreads) dst[i] = src[i];
}

template <typename T> hipError_t launch_pieces_as(const BeamSelect &a, hipStream_t st) {
  const unsigned blocks = (unsigned)(a.B * a.K * ((a.pieces + kPieceWaves - 1) / kPieceWaves));
  if (a.piece_len >= 1024) k_beam_pieces<T, 16><<<blocks, 64 * kPieceWaves, 0, st>>>(a);
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
