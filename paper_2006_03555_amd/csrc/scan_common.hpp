// scan_common.hpp - what the selective scan's forward and backward kernels share: tiles of
// kScanTokens tokens in LDS, channel by channel, and the scan over the lanes of a row.
//
// A wave takes four channels side by side, 16 lanes each, and a lane 8 neighbouring tokens of
// its channel. Inside a lane the recurrence h_t = a_t h_{t-1} + b_t runs token by token; across
// the 16 lanes of a row its steps (P, S): h -> P h + S are joined in four rounds of row shifts,
// one fused multiply-add and one product each.
#pragma once

#include <type_traits>

#include "recurrent.hpp"
#include "vec_rows.hpp"

namespace favor {

constexpr int kTok = kScanTokens;   // tokens of a chunk: 16 lanes of 8
constexpr int kScanWaves = 8;
constexpr int kScanThreads = 64 * kScanWaves;
constexpr int kStates = kScanStates;

// Place of token t in a row of kTok: the first halves of the lanes' eight tokens, then the second
// halves, so that the 16 lanes of a row read 16 bytes each from all the banks at once.
__device__ __forceinline__ int token_at(int t) { return (t >> 3 << 2) + (t & 3) + ((t & 4) << 4); }
// Place of (channel of the tile, token) in a [channels][kTok] tile: the lanes' places change by
// the channel's eight, so that eight columns written side by side meet different banks.
__device__ __forceinline__ int tile_at(int c, int t) { return c * kTok + token_at(t ^ ((c >> 3 & 15) << 3)); }
// The eight tokens of a lane (`lane` of the row, as in the tile at 0), to and from registers.
__device__ __forceinline__ void lane_load(const float *row, int lane, float *v) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(row + 4 * lane);
  const f32x4 b = *reinterpret_cast<const f32x4 *>(row + 4 * lane + 64);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
__device__ __forceinline__ void lane_store(float *row, int lane, const float *v) {
  *reinterpret_cast<f32x4 *>(row + 4 * lane) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4 *>(row + 4 * lane + 64) = f32x4{v[4], v[5], v[6], v[7]};
}
// The same of channel c of a tile.
__device__ __forceinline__ void tile_load(const float *tile, int c, int tl, float *v) {
  lane_load(tile + c * kTok, tl ^ (c >> 3 & 15), v);
}
__device__ __forceinline__ void tile_store(float *tile, int c, int tl, const float *v) {
  lane_store(tile + c * kTok, tl ^ (c >> 3 & 15), v);
}

// The state h before each lane's tokens: on entry h holds, in every lane, the state before
// the row, S = P h + (the sum over the lane's own tokens) in its first lane (the last, where
// it runs from the right) and the sum alone in the others; on return h is the state before
// the lane and S the one behind it. P is used up. kRight: rows run from their last lane.
//
// The hardware wants two instructions between a register's write and its use by another lane.
#define FAVOR_SCAN2(shift)                                          \
  "v_fmac_f32_dpp %0, %0, %1 " shift " row_mask:0xf bank_mask:0xf\n" \
  "v_fmac_f32_dpp %3, %3, %4 " shift " row_mask:0xf bank_mask:0xf\n" \
  "v_mul_f32_dpp %1, %1, %1 " shift " row_mask:0xf bank_mask:0xf\n"  \
  "v_mul_f32_dpp %4, %4, %4 " shift " row_mask:0xf bank_mask:0xf\n"
#define FAVOR_SCAN2_ALL(dir)                                          \
  "s_nop 1\n" FAVOR_SCAN2(dir ":1") FAVOR_SCAN2(dir ":2") FAVOR_SCAN2(dir ":4") \
  "v_fmac_f32_dpp %0, %0, %1 " dir ":8 row_mask:0xf bank_mask:0xf\n"  \
  "v_fmac_f32_dpp %3, %3, %4 " dir ":8 row_mask:0xf bank_mask:0xf\n"  \
  "s_nop 1\n"                                                         \
  "v_mov_b32_dpp %2, %0 " dir ":1 row_mask:0xf bank_mask:0xf\n"       \
  "v_mov_b32_dpp %5, %3 " dir ":1 row_mask:0xf bank_mask:0xf\n"
template <bool kRight>
__device__ __forceinline__ void row_scan2(float &S0, float &P0, float &h0, float &S1, float &P1,
                                          float &h1) {
  if constexpr (kRight)
    asm(FAVOR_SCAN2_ALL("row_shl")
        : "+v"(S0), "+v"(P0), "+v"(h0), "+v"(S1), "+v"(P1), "+v"(h1));
  else
    asm(FAVOR_SCAN2_ALL("row_shr")
        : "+v"(S0), "+v"(P0), "+v"(h0), "+v"(S1), "+v"(P1), "+v"(h1));
}
#define FAVOR_SCAN1(n)                                                   \
  "v_fmac_f32_dpp %0, %0, %1 row_shr:" n " row_mask:0xf bank_mask:0xf\n" \
  "v_mul_f32_dpp %1, %1, %1 row_shr:" n " row_mask:0xf bank_mask:0xf\n"  \
  "s_nop 1\n"
__device__ __forceinline__ void row_scan(float &S, float &P, float &h) {   // from the left
  asm("s_nop 1\n" FAVOR_SCAN1("1") FAVOR_SCAN1("2") FAVOR_SCAN1("4")
      "v_fmac_f32_dpp %0, %0, %1 row_shr:8 row_mask:0xf bank_mask:0xf\n"
      "s_nop 1\n"
      "v_mov_b32_dpp %2, %0 row_shr:1 row_mask:0xf bank_mask:0xf\n"
      : "+v"(S), "+v"(P), "+v"(h));
}

// Both at once: S, P and h from the left, Q, P2 and q from the right.
__device__ __forceinline__ void row_scan_both(float &S, float &P, float &h, float &Q, float &P2, float &q) {
#define FAVOR_SCAN_BOTH(n)                                            \
  "v_fmac_f32_dpp %0, %0, %1 row_shr:" n " row_mask:0xf bank_mask:0xf\n" \
  "v_fmac_f32_dpp %3, %3, %4 row_shl:" n " row_mask:0xf bank_mask:0xf\n"
#define FAVOR_SCAN_BOTH_P(n)                                          \
  "v_mul_f32_dpp %1, %1, %1 row_shr:" n " row_mask:0xf bank_mask:0xf\n" \
  "v_mul_f32_dpp %4, %4, %4 row_shl:" n " row_mask:0xf bank_mask:0xf\n"
  asm("s_nop 1\n" FAVOR_SCAN_BOTH("1") FAVOR_SCAN_BOTH_P("1") FAVOR_SCAN_BOTH("2") FAVOR_SCAN_BOTH_P("2")
          FAVOR_SCAN_BOTH("4") FAVOR_SCAN_BOTH_P("4") FAVOR_SCAN_BOTH("8")
      "s_nop 1\n"
      "v_mov_b32_dpp %2, %0 row_shr:1 row_mask:0xf bank_mask:0xf\n"
      "v_mov_b32_dpp %5, %3 row_shl:1 row_mask:0xf bank_mask:0xf\n"
      : "+v"(S), "+v"(P), "+v"(h), "+v"(Q), "+v"(P2), "+v"(q));
}

// The sum over the 16 lanes of a row, in its last lane.
__device__ __forceinline__ float row_sum(float v) {
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x111, 0xf, 0xf, true));
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x112, 0xf, 0xf, true));
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x114, 0xf, 0xf, true));
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x118, 0xf, 0xf, true));
  return v;
}

// Where a workgroup works: a tile of channels inside one group, a segment, a sequence.
struct ScanPlace {
  int b, seg, g, tile, c0, cend, n;
};
__device__ __forceinline__ int group_tiles(const Scan &a, int width) {
  return (a.D / a.G + width - 1) / width;
}
__device__ __forceinline__ ScanPlace scan_place(const Scan &a, int width) {
  ScanPlace p;
  const int of_group = group_tiles(a, width), tiles = a.G * of_group, dg = a.D / a.G;
  p.b = blockIdx.y;
  p.seg = blockIdx.x / tiles;
  const int i = blockIdx.x - p.seg * tiles;
  p.seg += a.seg0;
  p.g = i / of_group;
  p.tile = i - p.g * of_group;
  p.c0 = p.g * dg + p.tile * width;
  p.cend = (p.g + 1) * dg;
  p.n = clamped_length(a.lengths, p.b, a.L);
  return p;
}

// The thread's number, as a value that each use forms its addresses from anew: kept over a whole
// loop they would take the registers that the scan needs.
__device__ __forceinline__ int fresh_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// What a thread loads of a tile of kWidth channels: kLoads units of eight channels of one token.
template <int kWidth> constexpr int kLoads = kTok * kWidth / 8 / kScanThreads;
struct Unit {
  int u, t, c;   // unit, token of the chunk, channel
  int tl, cl;    // the same where they are inside the sequence and the group, else others that are
  bool live;     // they are
};
template <int kWidth>
__device__ __forceinline__ Unit unit_of(const ScanPlace &p, int64_t t0, int i, int tid) {
  const int k = tid + i * kScanThreads;
  Unit w;
  w.u = k % (kWidth / 8);
  w.t = k / (kWidth / 8);
  w.c = p.c0 + 8 * w.u;
  const int left = (int)min((int64_t)kTok, p.n - t0);
  w.live = w.t < left && w.c < p.cend;
  w.tl = min(w.t, left - 1);
  w.cl = w.c < p.cend ? w.c : p.c0;
  return w;
}
// Loads ask for valid rows whether they are wanted or not (a chunk that is read has a token): a
// condition around each would wait for one before the next is requested.
// Rows of one chunk: a uniform base and 32-bit byte offsets (tokens are at most 2^25 bytes apart),
// which the loads take as they are.
template <typename T>
__device__ __forceinline__ T *chunk_rows(T *base, const Rows &r, const ScanPlace &p, int64_t t0) {
  return base + p.b * r.b + t0 * r.t;
}
template <typename T> __device__ __forceinline__ T *at_byte(T *base, uint32_t offset) {
  using Byte = std::conditional_t<std::is_const_v<T>, const char, char>;
  return reinterpret_cast<T *>(reinterpret_cast<Byte *>(base) + offset);
}
template <typename T> __device__ __forceinline__ uint32_t row_bytes(const Rows &r, int t, int c) {
  return (uint32_t)sizeof(T) * ((uint32_t)t * (uint32_t)r.t + (uint32_t)c);
}
template <typename T>
__device__ __forceinline__ RowVec<T, 8> get_row(const void *base, const Rows &r, const ScanPlace &p, int64_t t0,
                                                const Unit &w) {
  RowVec<T, 8> v;
  v.load(at_byte(chunk_rows(static_cast<const T *>(base), r, p, t0), row_bytes<T>(r, w.tl, w.cl)));
  return v;
}
template <typename T>
__device__ __forceinline__ T *row_out(void *base, const Rows &r, const ScanPlace &p, int64_t t0, const Unit &w) {
  return at_byte(chunk_rows(static_cast<T *>(base), r, p, t0), row_bytes<T>(r, w.t, w.c));
}
template <typename T>
__device__ __forceinline__ void put_row(void *base, const Rows &r, const ScanPlace &p, int64_t t0, const Unit &w,
                                        const float *v) {
  store_row<8>(row_out<T>(base, r, p, t0, w), v);
}
__device__ __forceinline__ void put_unit(float *tile, const Unit &w, const float *v) {
#pragma unroll
  for (int k = 0; k < 8; ++k) tile[tile_at(8 * w.u + k, w.t)] = v[k];
}

// Two rows of a tile on their way from memory to lanes (x and dt, dy and z): in bf16 both in one
// word, else a tile each.
template <typename T> constexpr int kPairTiles = sizeof(T) == 2 ? 1 : 2;
template <int kWidth>
__device__ __forceinline__ void put_pair(float *tile, const Unit &w, const RowVec<bf16, 8> &v0, const RowVec<bf16, 8> &v1) {
  const uint32_t a[4] = {v0.r.x, v0.r.y, v0.r.z, v0.r.w}, b[4] = {v1.r.x, v1.r.y, v1.r.z, v1.r.w};
#pragma unroll
  for (int k = 0; k < 8; ++k)   // the low or the high halves of two words
    tile[tile_at(8 * w.u + k, w.t)] = __uint_as_float(
        __builtin_amdgcn_perm(b[k / 2], a[k / 2], k % 2 ? 0x07060302u : 0x05040100u));
}
template <int kWidth>
__device__ __forceinline__ void put_pair(float *tile, const Unit &w, const RowVec<float, 8> &v0, const RowVec<float, 8> &v1) {
  float v[8];
  v0.get(v);
  put_unit(tile, w, v);
  v1.get(v);
  put_unit(tile + kWidth * kTok, w, v);
}
template <typename T, int kWidth>
__device__ __forceinline__ void get_pair(const float *tile, int c, int tl, float (&v0)[8], float (&v1)[8]) {
  tile_load(tile, c, tl, v0);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t both = __float_as_uint(v0[j]);
      v0[j] = __uint_as_float(both << 16);
      v1[j] = __uint_as_float(both & 0xffff0000u);
    }
  } else {
    tile_load(tile + kWidth * kTok, c, tl, v1);
  }
}
// How many of a lane's eight tokens are inside the sequence (8 or more: all).
__device__ __forceinline__ int lane_left(const ScanPlace &p, int64_t t0, int tl) {
  return (int)min((int64_t)kTok, p.n - t0) - 8 * tl;
}
// A lane's steps from its dt, and their sum; steps and x are zeros from token `left` on.
__device__ __forceinline__ float lane_steps(const Scan &a, int left, float bias, float (&s)[8], float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] += bias;
  if (a.softplus)
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = softplus(s[j]);
  if (left < 8)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= left) s[j] = x[j] = 0.f;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum += s[j];
  return sum;
}

// [states][kTok] tile of B or C: states n0 .., zeros behind the sequence. A thread keeps its
// state and takes every 32nd token.
template <typename T> struct States {
  static constexpr int kStep = kScanThreads / kStates, kEach = kTok / kStep;
  T v[kEach];

  __device__ __forceinline__ void load(const void *src, const Rows &r, const ScanPlace &p, int64_t t0, int n0,
                                       int count, int tid) {
    const T *base = chunk_rows(static_cast<const T *>(src), r, p, t0) + p.g * r.h + n0;
    const int left = (int)min((int64_t)kTok, p.n - t0);
    const uint32_t first = (uint32_t)(tid / kStates) * (uint32_t)r.t, last = (uint32_t)(left - 1) * (uint32_t)r.t;
    const uint32_t n = min(tid % kStates, count - 1);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      v[i] = *at_byte(base, (uint32_t)sizeof(T) * (min(first + i * kStep * (uint32_t)r.t, last) + n));
  }
  __device__ __forceinline__ void put(float *tile, const ScanPlace &p, int64_t t0, int count, int tid) const {
    static_assert(kStep % 8 == 0, "places of tokens kStep apart");
    const int n = tid % kStates, t1 = tid / kStates;
    const int left = n < count ? (int)min((int64_t)kTok, p.n - t0) : 0;
    float *to = tile + n * kTok + token_at(t1);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      to[token_at(i * kStep)] = t1 + i * kStep < left ? to_f32(v[i]) : 0.f;
  }
};

// The tile's channels, states n0 .. n0 + count - 1 (at most kStates), of a [D][N] array (null:
// zeros), to and from [kStates][kWidth] in LDS; states behind them are zeros.
template <int kWidth>
__device__ __forceinline__ void load_channels(const float *src, const ScanPlace &p, int N, int n0, int count,
                                              float scale, float *dst, int tid) {
#pragma unroll
  for (int i = 0; i < kWidth * kStates / kScanThreads; ++i) {
    const int k = tid + i * kScanThreads, c = k / kStates, n = k % kStates;
    float v = 0.f;
    if (src) v = src[(int64_t)min(p.c0 + c, p.cend - 1) * N + n0 + min(n, count - 1)];
    dst[n * kWidth + c] = n < count ? scale * v : 0.f;
  }
}
template <int kWidth>
__device__ __forceinline__ void store_channels(float *dst, const ScanPlace &p, int N, int n0, int count,
                                               const float *src, int tid) {
#pragma unroll
  for (int i = 0; i < kWidth * kStates / kScanThreads; ++i) {
    const int k = tid + i * kScanThreads, c = k / kStates, n = k % kStates;
    if (n < count && p.c0 + c < p.cend) dst[(int64_t)(p.c0 + c) * N + n0 + n] = src[n * kWidth + c];
  }
}

}  // namespace favor
