// scan_common.hpp - what the selective scan's forward and backward kernels share: tiles of
// kScanTokens tokens in LDS, channel by channel, and the scan over the lanes of a row.
//
// A wave takes four channels side by side, 16 lanes each, and a lane 8 neighbouring tokens of
// its channel. Inside a lane the recurrence h_t = a_t h_{t-1} + b_t runs token by token; across
// the 16 lanes of a row its steps (P, S): h -> P h + S are joined in four rounds of row shifts,
// one fused multiply-add and one product each.
#pragma once

#include "recurrent.hpp"
#include "vec_rows.hpp"

namespace favor {

constexpr int kTok = kScanTokens;   // tokens of a chunk: 16 lanes of 8
constexpr int kLaneTok = 8;
constexpr int kScanWaves = 8;
constexpr int kScanThreads = 64 * kScanWaves;
constexpr int kStates = 16;         // states of one pass over a chunk

// Place of (channel of the tile, token) in a [channels][kTok] tile: groups of four (fp32) or
// eight (bf16) tokens change places by channel, so that a row's eight channels, written as
// eight columns, meet different banks. A lane's eight tokens stay together.
template <typename T> __device__ __forceinline__ int tile_at(int c, int t) {
  if constexpr (sizeof(T) == 2) return c * kTok + ((((t >> 3) ^ (c >> 3)) & 15) << 3) + (t & 7);
  else return c * kTok + ((((t >> 2) ^ (c >> 3 << 1)) & 31) << 2) + (t & 3);
}
template <typename T> __device__ __forceinline__ void lane_tokens(const T *tile, int c, int tl, float *v) {
  RowVec<T, 8> r;
  r.load(tile + tile_at<T>(c, kLaneTok * tl));
  r.get(v);
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
#define FAVOR_SCAN1(shift)                                                     \
  "v_fmac_f32_dpp %0, %0, %1 " shift " row_mask:0xf bank_mask:0xf\n"            \
  "v_mul_f32_dpp %1, %1, %1 " shift " row_mask:0xf bank_mask:0xf\n"             \
  "s_nop 1\n"
#define FAVOR_SCAN1_ALL(dir)                                                   \
  "s_nop 1\n" FAVOR_SCAN1(dir ":1") FAVOR_SCAN1(dir ":2") FAVOR_SCAN1(dir ":4") \
  "v_fmac_f32_dpp %0, %0, %1 " dir ":8 row_mask:0xf bank_mask:0xf\n"           \
  "s_nop 1\n"                                                                  \
  "v_mov_b32_dpp %2, %0 " dir ":1 row_mask:0xf bank_mask:0xf\n"
template <bool kRight>
__device__ __forceinline__ void row_scan(float &S, float &P, float &h) {
  if constexpr (kRight) asm(FAVOR_SCAN1_ALL("row_shl") : "+v"(S), "+v"(P), "+v"(h));
  else asm(FAVOR_SCAN1_ALL("row_shr") : "+v"(S), "+v"(P), "+v"(h));
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
  p.g = i / of_group;
  p.tile = i - p.g * of_group;
  p.c0 = p.g * dg + p.tile * width;
  p.cend = (p.g + 1) * dg;
  p.n = clamped_length(a.lengths, p.b, a.L);
  return p;
}

// Steps s = softplus(dt + bias) of eight channels of one token.
template <typename T>
__device__ __forceinline__ void steps_of(const Scan &a, const RowVec<T, 8> &raw, int c, float *s) {
  raw.get(s);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (a.bias) s[k] += a.bias[c + k];
    if (a.softplus) s[k] = softplus(s[k]);
  }
}

// s and x of the tile's tokens t0 .. (zeros behind the sequence and the group).
template <typename T, int kWidth, typename X>
__device__ __forceinline__ void load_steps(const Scan &a, const ScanPlace &p, int64_t t0, float *ts, X *tx) {
  constexpr int units = kWidth / 8;
#pragma unroll
  for (int i = threadIdx.x; i < kTok * units; i += kScanThreads) {
    const int u = i % units, t = i / units, c = p.c0 + 8 * u;
    float s[8], x[8];
    if (t0 + t < p.n && c < p.cend) {
      RowVec<T, 8> rx, rd;
      rx.load(static_cast<const T *>(a.x) + p.b * a.xs.b + (t0 + t) * a.xs.t + c);
      rd.load(static_cast<const T *>(a.dt) + p.b * a.dts.b + (t0 + t) * a.dts.t + c);
      steps_of<T>(a, rd, c, s);
      rx.get(x);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] = x[k] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      ts[tile_at<float>(8 * u + k, t)] = s[k];
      tx[tile_at<X>(8 * u + k, t)] = from_f32<X>(x[k]);
    }
  }
}

// [states][kTok] tile of B or C (src of type T): states n0 .., zeros behind the sequence.
template <typename T>
__device__ __forceinline__ void load_states(const void *src, const Rows &r, const ScanPlace &p, int64_t t0,
                                            int n0, int count, float *tile) {
  const T *base = static_cast<const T *>(src) + p.b * r.b + p.g * r.h + n0;
  for (int i = threadIdx.x; i < kTok * kStates; i += kScanThreads) {
    const int n = i % kStates, t = i / kStates;
    float v = 0.f;
    if (n < count && t0 + t < p.n) v = to_f32(base[(t0 + t) * r.t + n]);
    tile[n * kTok + t] = v;
  }
}

__device__ __forceinline__ void load8(const float *p, float *v) {
  const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
__device__ __forceinline__ void store8_lds(float *p, const float *v) {
  reinterpret_cast<f32x4 *>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
  reinterpret_cast<f32x4 *>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
}

// The tile's channels, states n0 .. n0 + count - 1, of a [D][N] array (null: zeros), to and
// from [count][kWidth] in LDS.
template <int kWidth>
__device__ __forceinline__ void load_channels(const float *src, const ScanPlace &p, int N, int n0, int count,
                                              float scale, float *dst) {
  for (int i = threadIdx.x; i < kWidth * count; i += kScanThreads) {
    const int c = i / count, n = i - c * count;
    dst[n * kWidth + c] = src && p.c0 + c < p.cend ? scale * src[(int64_t)(p.c0 + c) * N + n0 + n] : 0.f;
  }
}
template <int kWidth>
__device__ __forceinline__ void store_channels(float *dst, const ScanPlace &p, int N, int n0, int count,
                                               const float *src) {
  for (int i = threadIdx.x; i < kWidth * count; i += kScanThreads) {
    const int c = i / count, n = i - c * count;
    if (p.c0 + c < p.cend) dst[(int64_t)(p.c0 + c) * N + n0 + n] = src[n * kWidth + c];
  }
}

}  // namespace favor
