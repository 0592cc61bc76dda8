// decay.hip - linear attention with a decay per head, in chunks of 64 tokens.
//
//   S_t = a S_{t-1} + k_t v_t^T,   o_t = c q_t^T S_t,   a = exp(log_decay of the head)
//
// A workgroup takes one (batch, head), a slice of the value columns and one segment of
// the sequence, and carries X = S (kd x slice, fp32, in matrix-core accumulators) over
// the segment's chunks. Of one chunk with rows i, j in [0, 64):
//   O   = (Q K^T o D) V + diag(a^(i + 1)) Q X     D_ij = a^(i - j) for j <= i, else 0
//   X  <- a^64 X + K^T diag(a^(63 - j)) V
// Every power has an exponent >= 0 and comes from a table, so a decay of 0 and one of 1
// are the same code and nothing overflows that the formula does not.
//
// The products are taken transposed, so that no accumulator has to change lanes: two
// adjacent tiles of X (rows k, columns v) are in chained order the A operand of
// O^T = X^T Q^T, and those of P^T = K Q^T (rows j, columns i) the B operand of V^T P^T.
// Only V^T and K^T need a transpose; bf16 tiles get it from the LDS transpose read. Each
// wave holds all of X's rows for 16 or 32 value columns; P^T is shared out over the waves
// and passes through LDS.
//
// Precision (bf16): X, and all sums, are fp32. The weighted values diag(a^(..)) V enter
// K^T V as three bf16 terms (24 bits: exact) where the call returns X, which is then as exact
// as fp32 inputs would make it. Where X only feeds outputs, two terms do: they leave at most
// 2^-16 of each product (2.6e-6 of X by its norm; 65536 x 16 heads of 128 x 128 in 380
// instead of 407 us, a training step of 4 x 4096 x 16 in 364 instead of 401). X in Q X and
// the pair weights in P V are two terms each, in every call: what they leave, 2^-16, is far
// below the output's own rounding, so that a row is as near as a rounded one can be, whatever
// batch it is in. With one term, 2^-8 off, errors by norm are 1.4 times a correctly rounded
// output's and those of single rows, whose few weights do not average out, up to 2.1 times;
// the same calls then take 358 and 328 us.
//
// Bound: the bytes, and at 128 x 128 in bf16 the power that the arithmetic takes. 512 segments
// of 2048 rows (65536 x 16 heads, 1.07 GB) take 250 us (4.3 TB/s), but 302 in the first tens
// of calls of a run, while the clock settles; 512 heads x 2048 rows 254. At 64 x 64 the scan moves 4.6 TB/s, at 256 x 64 4.5. fp32 is bound by a
// chunk's chain of products: 256 heads x 1024 rows of 128 x 128 (0.54 GB) 337 us. Calls of few
// heads read K and V twice, once for the segments' sums.
#include "decay.hpp"
#include "tile_common.hpp"

namespace favor {
namespace {

constexpr int kChunkT = 64;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// An LDS tile of 64 rows and W columns, in granules of four elements. Granule c of a row
// lies at place c ^ f(row), so that both ways of reading it meet each of the 64 banks once:
//   RowReader:   16 rows at two granules (bf16, 8 bytes each) or at one (fp32, 16 bytes)
//   TransReader: eight rows by four granules (bf16), or one column of four rows by four
//                granules (fp32)
// bf16 pairs of granules stay together, so staging writes 16 bytes.
template <typename T, int W>
struct Tile {
  static __device__ __forceinline__ int f(int row) {
    if (sizeof(T) == 4) return row & 15;
    return W == 64 ? (((row >> 1) & 3) << 2) | (((row >> 3) & 1) << 1)
                   : ((row & 7) << 2) | (((row >> 3) & 1) << 1);
  }
  static __device__ __forceinline__ int at(int row, int granule) {
    return row * W + 4 * (granule ^ f(row));
  }
  // granules the swizzle stays within: what lies above is a constant offset
  static constexpr int kSpan = sizeof(T) == 4 || W == 64 ? 16 : 32;
  static constexpr int kGranule = 4 * (int)sizeof(T);
  static constexpr int kRow = W * (int)sizeof(T);
};

// LDS addresses as integers. A tile starts at a multiple of 256 bytes, so that a swizzled
// place is a lane's own address with a constant exclusive-ored in: one register per way of
// reading instead of one per place.
using lds_t = uint32_t;
__device__ __forceinline__ lds_t lds_of(const void *p) {
  return (lds_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// Operand fragments of a tile's rows 16 b .. + 15 over columns 32 p .. + 31, chained order.
template <typename T, int W>
struct RowReader {
  using L = Tile<T, W>;
  lds_t base;
  __device__ __forceinline__ explicit RowReader(lds_t tile) {
    const int r = lane_id() & 15, g = lane_id() >> 4;
    base = tile + r * L::kRow + (g ^ L::f(r)) * L::kGranule;
  }
  __device__ __forceinline__ typename Mma<T>::frag operator()(int b, int p) const {
    typedef T quad __attribute__((ext_vector_type(4)));
    // volatile: loads of two fragments are not to be merged into one wide load, whose
    // halves would then have to be moved
    using ldsq = const volatile __attribute__((address_space(3))) quad;
    const int over = (8 * p & ~(L::kSpan - 1)) * L::kGranule + 16 * b * L::kRow;
    const int in = (8 * p & (L::kSpan - 1)) * L::kGranule;
    const quad lo = *(ldsq *)((base ^ in) + over);
    const quad hi = *(ldsq *)((base ^ (in + 4 * L::kGranule)) + over);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// Operand fragments of a tile's transpose: 16 columns over rows 32 m .. + 31, chained order.
// The columns are the granules c0, c0 + STEP, c0 + 2 STEP and c0 + 3 STEP, c0 having none of
// STEP's multiples' bits.
template <typename T, int W, int STEP>
struct TransReader {
  using L = Tile<T, W>;
  lds_t base;
  __device__ __forceinline__ explicit TransReader(lds_t tile) {
    const int c = lane_id() & 15, g = lane_id() >> 4;
    if constexpr (sizeof(T) == 2) {
      const int row = 4 * g + (c >> 2);
      base = tile + row * L::kRow + ((STEP * (c & 3)) ^ L::f(row)) * L::kGranule;
    } else {
      base = tile + 4 * g * L::kRow + ((STEP * (c >> 2)) ^ L::f(4 * g)) * L::kGranule + 4 * (c & 3);
    }
  }
  __device__ __forceinline__ typename Mma<T>::frag operator()(int c0, int m) const {
    const int over = (c0 & ~(L::kSpan - 1)) * L::kGranule + 32 * m * L::kRow;
    const int in = (c0 & (L::kSpan - 1)) * L::kGranule;
    if constexpr (sizeof(T) == 2) {
      using lds4 = __attribute__((address_space(3))) s16x4;
      const lds_t p = (base ^ in) + over;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p + 16 * L::kRow));
      struct Two { s16x4 a, b; };
      return __builtin_bit_cast(bf16x8, Two{lo, hi});
    } else {
      using ldsf = const __attribute__((address_space(3))) float;
      f32x8 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // f(4 g + i) = f(4 g) ^ i
        const lds_t p = (base ^ (in ^ i * L::kGranule)) + over + i * L::kRow;
        x[i] = *(ldsf *)p;
        x[4 + i] = *(ldsf *)(p + 16 * L::kRow);
      }
      return x;
    }
  }
};

// Eight fp32 values as N operand fragments whose sum they are: each term rounded, and what
// it leaves (exact) passed on. The dot product of a pair of terms with (-1, 0) or (0, -1)
// takes one term from its value without unpacking it.
// (These come from the arguments: the compiler writes (-1, 0) as an immediate that the
// instruction takes for the float -1.)
template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&f)[N],
                                       const uint32_t (&minus)[2]) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 first = __builtin_bit_cast(bf16x2, minus[0]);
  const bf16x2 second = __builtin_bit_cast(bf16x2, minus[1]);
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const bf16x2 t = {(bf16)r[i], (bf16)r[i + 1]};
      f[n][i] = t[0];
      f[n][i + 1] = t[1];
      if (n + 1 < N) {
        r[i] = __builtin_amdgcn_fdot2_f32_bf16(t, first, r[i], false);
        r[i + 1] = __builtin_amdgcn_fdot2_f32_bf16(t, second, r[i + 1], false);
      }
    }
}
template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], f32x8 (&f)[N], const uint32_t (&)[2]) {
  static_assert(N == 1, "fp32 operands are whole");
#pragma unroll
  for (int i = 0; i < 8; ++i) f[0][i] = x[i];
}
// Terms of the weighted values: all of them where X leaves the call.
template <typename T> constexpr int sum_terms(bool whole) {
  return sizeof(T) == 4 ? 1 : whole ? 3 : 2;
}

// The wave's number, as a scalar.
__device__ __forceinline__ int wave_id() {
  return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

// The value of lane 0, as a scalar.
__device__ __forceinline__ float uniform(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}

// a^64 for chunk after chunk as single floats whose products stay right: what the products
// so far lack (relative to a^(64 c)) goes into the next one. (One float's own rounding
// would be raised to the number of chunks: 128 of them put X off by 4e-6; a second float
// for its error costs one more operation on every element of X.)
struct Carry {
  float one, lack, inv;   // a^64 rounded, what the rounding left relative to it, 1 / one
  float err;              // (a^(64 c) / product) - 1
  // several: whether there will be a second chunk
  __device__ __forceinline__ Carry(float g, bool several)
      : one(0.f), lack(0.f), inv(0.f), err(0.f) {
    if (!several) {
      one = uniform(expf(g * kChunkT));
      return;
    }
    const double d = exp((double)g * kChunkT);
    one = uniform((float)d);
    const bool plain = one > 1e-30f && one < 1e30f;
    inv = uniform(plain ? 1.f / one : 0.f);
    lack = uniform(plain ? (float)((d - one) / d) : 0.f);
  }
  __device__ __forceinline__ float next() {
    err += lack;
    const float f = fmaf(one, err, one);
    err -= (f - one) * inv;
    return f;
  }
};

// What a workgroup works on.
struct Item {
  int bh, b, h, slice, seg;
  int len;    // tokens of the sequence
  int first;  // the segment's first row (in the scan's order)
  int n;      // its tokens
};

// The scan of a workgroup: scans that run together take turns, so that those that read the
// same rows read them at about the same time.
__device__ __forceinline__ const DecayScan &scan_of(const DecayPass &pass, int &id) {
  const int r = pass.n > 1 ? id % pass.n : 0;
  id = pass.n > 1 ? id / pass.n : id;
  return pass.scan[r];
}

__device__ __forceinline__ Item item_of(const DecayScan &a, int id, int nslice, int nseg) {
  Item it;
  it.slice = id % nslice;
  id /= nslice;
  it.seg = id % nseg;
  it.bh = id / nseg;
  it.b = it.bh / a.H;
  it.h = it.bh % a.H;
  it.len = a.lengths ? min(max(a.lengths[it.b], 0), a.L) : a.L;
  it.first = it.seg * a.seg_len;
  it.n = min(max(it.len - it.first, 0), a.seg_len);
  return it;
}
// The segment of the sequence's last token: it ends with X_n.
__device__ __forceinline__ int last_seg(const DecayScan &a, int len) {
  return len == 0 ? 0 : (len - 1) / a.seg_len;
}

// Rows of a chunk in global memory, reached through a buffer descriptor at the chunk's
// lowest row: a lane's 32-bit offset is formed once, rows further on are a scalar offset,
// and an offset of kOutside reads zeros or writes nothing. (Token strides are at most 2^25
// bytes, so that the 64 rows lie below it.)
constexpr uint32_t kOutside = 1u << 31;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk_rows(const void *x, const Rows &s,
                                                             const Item &it, int col,
                                                             bool reverse, int first) {
  const T *base = static_cast<const T *>(x) + it.b * s.b + it.h * s.h + col +
                  (reverse ? it.len - kChunkT - first : first) * s.t;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(base), 0, kOutside, 0x00020000);
}

// A chunk's rows on their way from global memory to an LDS tile: 16-byte units, zero past
// the chunk's n rows and the tensor's `width` columns. A thread keeps to one column; its
// rows are kRows apart.
template <typename T, int W, int NT>
struct Staged {
  static constexpr int kPer = 16 / (int)sizeof(T);
  static constexpr int kUnits = W / kPer;
  static constexpr int kRows = NT / kUnits;
  static constexpr int N = kChunkT / kRows;
  static_assert(NT % kUnits == 0 && kChunkT % kRows == 0, "whole passes");
  u32x4 r[N];
  uint32_t off;
  __device__ __forceinline__ void start(const Rows &s, bool reverse, int width) {
    const int row = threadIdx.x / kUnits, col = threadIdx.x % kUnits * kPer;
    off = ((reverse ? kRows - 1 - row : row) * (uint32_t)s.t + col) * (uint32_t)sizeof(T);
    if (col >= width) off = kOutside;
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t x, const Rows &s, bool reverse,
                                       int n) {
    const int row = threadIdx.x / kUnits;
    const uint32_t step = kRows * (uint32_t)s.t * (uint32_t)sizeof(T);
#pragma unroll
    for (int k = 0; k < N; ++k)
      r[k] = __builtin_amdgcn_raw_buffer_load_b128(
          x, row < n - k * kRows ? off : kOutside, (reverse ? N - 1 - k : k) * step, 0);
  }
  __device__ __forceinline__ void store(T *tile) const {
    const int row = threadIdx.x / kUnits, granule = threadIdx.x % kUnits * (kPer / 4);
#pragma unroll
    for (int k = 0; k < N; ++k)
      *reinterpret_cast<u32x4 *>(tile + Tile<T, W>::at(row + k * kRows, granule)) = r[k];
  }
};

// a^e for e = 0 .. 64, and the weights made of them.
struct Powers {
  float a[kChunkT + 1];
  f32x4 sum[kChunkT / 4];     // sum_scale a^(n - shift - j) of a chunk's n tokens, 0 behind them
  float row[kChunkT];         // row_scale a^(i + shift)
  float pair[kChunkT + 16];   // pair_scale a^(e) at e + 16, 0 for e < 0
};
// a^e = exp(g e) to about one rounding: g e as a sum of two floats, 0^0 = 1. (0 and Inf, past
// the range on either side, stay: the second float may be NaN there.)
__device__ __forceinline__ float power(float g, int e) {
  const float x = g * (float)e, low = fmaf(g, (float)e, -x);
  const float y = expf(x);
  return e == 0 ? 1.f : y > 0.f && y < INFINITY ? fmaf(y, low, y) : y;
}
__device__ __forceinline__ void fill_powers(Powers &p, float g) {
  if (threadIdx.x <= kChunkT) p.a[threadIdx.x] = power(g, threadIdx.x);
}
// The weights of a chunk's tokens in its sum (after fill_powers and a barrier).
__device__ __forceinline__ void fill_sum(Powers &p, int n, int shift, float scale) {
  if (threadIdx.x < kChunkT) {
    const int e = n - shift - (int)threadIdx.x;
    reinterpret_cast<float *>(p.sum)[threadIdx.x] = e >= 0 ? p.a[max(e, 0)] * scale : 0.f;
  }
}
// The weights of rows and pairs (likewise).
__device__ __forceinline__ void fill_rows(Powers &p, const DecayScan &a) {
  if (threadIdx.x < kChunkT) {
    p.row[threadIdx.x] = p.a[threadIdx.x + a.shift] * a.row_scale;
    p.pair[threadIdx.x + 16] = p.a[threadIdx.x] * a.pair_scale;
  } else if (threadIdx.x < kChunkT + 16) {
    p.pair[threadIdx.x - kChunkT] = 0.f;
  }
}

// A lane's 4 NCT consecutive columns of an output row, rounded to T. (No scalar offset: the
// compiler takes it that a 16-byte store with one needs no wait before its data registers
// are written again, and lanes 12 .. 15 then stored what came next.)
template <typename T, int NCT>
__device__ __forceinline__ void put_row(__amdgpu_buffer_rsrc_t x, uint32_t off,
                                        const f32x4 (&v)[NCT]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v[ct]), x, off + 16 * ct,
                                             0, 0);
  } else if constexpr (NCT == 2) {
    __builtin_amdgcn_raw_buffer_store_b128(
        __builtin_bit_cast(u32x4, Mma<bf16>::pack(v[0], v[1])), x, off, 0, 0);
  } else {
    bf16x4 b;
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = (bf16)v[0][j];
    __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, b), x, off, 0, 0);
  }
}

// X's tiles of one wave: [k rows / 16][its value columns / 16][a lane's four k rows].
template <int KD, int NCT>
struct State {
  float x[KD / 16][NCT][4];
};
// Column c (0 .. 15) of a wave's tile ct among the wave's value columns: with two tiles, a
// lane's accumulator rows of both are eight consecutive columns.
template <int NCT>
__device__ __forceinline__ int value_col(int ct, int c) {
  return NCT == 2 ? perm_col(ct, c) : c;
}
__device__ __forceinline__ void put(float (&x)[4], f32x4 v) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = v[j];
}
__device__ __forceinline__ f32x4 get(const float (&x)[4]) { return f32x4{x[0], x[1], x[2], x[3]}; }

// X before a segment; until the prefix pass, the sums of the segment in front of it.
__device__ __forceinline__ float *part_of(const DecayScan &a, int bh, int seg) {
  return a.part + ((size_t)bh * a.nseg + seg) * (a.kd * a.vd);
}

// X of one head in memory ([kd][vd], or transposed): four k rows of one column at a time.
// Null has no rows: it reads as zeros.
struct StateRows {
  __amdgpu_buffer_rsrc_t rows;
  int kd, vd;
  bool x_t;
  __device__ __forceinline__ StateRows(const DecayScan &a, const float *p)
      : rows(__builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(p), 0, kOutside, 0x00020000)),
        kd(p ? a.kd : 0), vd(a.vd), x_t(a.x_t) {}
  __device__ __forceinline__ uint32_t at(int kc, int vc) const {
    return vc < vd && kc < kd ? 4 * (uint32_t)(x_t ? vc * kd + kc : kc * vd + vc) : kOutside;
  }
  __device__ __forceinline__ void read(float (&x)[4], int kc, int vc) const {
    const uint32_t off = at(kc, vc);
    if (x_t) {
      put(x, __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, off, 0, 0)));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rows, off, 4 * j * vd, 0));
    }
  }
  __device__ __forceinline__ void write(const float (&x)[4], int kc, int vc) const {
    const uint32_t off = at(kc, vc);
    if (x_t) {
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, get(x)), rows, off, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[j]), rows, off, 4 * j * vd, 0);
    }
  }
};

template <int KD, int NW, int NCT>
__device__ __forceinline__ void load_state(const DecayScan &a, const Item &it,
                                           State<KD, NCT> &s) {
  const int l = lane_id(), w0 = 16 * NCT * (NW * it.slice + wave_id());
  // With several segments X_0 too comes from the workspace: the caller's may already hold
  // X_n, where they are the same.
  const float *p = a.x_in ? a.x_in + (size_t)it.bh * (a.kd * a.vd) : nullptr;
  if (a.nseg > 1 && (it.seg > 0 || p)) p = part_of(a, it.bh, it.seg);
  const StateRows rows(a, p);
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb) {
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
      rows.read(s.x[nb][ct], 16 * nb + 4 * (l >> 4), w0 + value_col<NCT>(ct, l & 15));
  }
}

template <int KD, int NW, int NCT>
__device__ __forceinline__ void store_state(const DecayScan &a, const Item &it, float *p,
                                            const State<KD, NCT> &s) {
  const int l = lane_id(), w0 = 16 * NCT * (NW * it.slice + wave_id());
  const StateRows rows(a, p);
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb) {
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
      rows.write(s.x[nb][ct], 16 * nb + 4 * (l >> 4), w0 + value_col<NCT>(ct, l & 15));
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The wave's value columns of a chunk, transposed: tokens in chained order.
template <typename T, int VS, int NCT>
__device__ __forceinline__ void load_values(lds_t Vs, typename Mma<T>::frag (&vt)[NCT][2]) {
  const TransReader<T, VS, NCT> values(Vs);
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int m = 0; m < 2; ++m) vt[ct][m] = values(4 * NCT * wave_id() + ct, m);
}

// diag(pw.sum) V in N operand terms.
template <typename T, int NCT, int N>
__device__ __forceinline__ void weigh_values(
    typename Mma<T>::frag (&vw)[2][NCT][N],
    const typename Mma<T>::frag (&vt)[NCT][2], const Powers &pw, const uint32_t (&minus)[2]) {
  const int g = lane_id() >> 4;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const f32x4 w0 = pw.sum[8 * m + g], w1 = pw.sum[8 * m + 4 + g];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = to_f32(vt[ct][m][i]) * w0[i];
        x[4 + i] = to_f32(vt[ct][m][4 + i]) * w1[i];
      }
      split8<N>(x, vw[m][ct], minus);
    }
  }
}

// X <- carry X + K^T (diag(pw.sum) V).
template <typename T, int KD, int NCT, int N>
__device__ __forceinline__ void update_state(
    State<KD, NCT> &s, lds_t Ks, const typename Mma<T>::frag (&vw)[2][NCT][N],
    float carry) {
  using P = Mma<T>;
  const TransReader<T, KD, 1> keys(Ks);
  // The chunk's sum starts from zero and joins X in one rounded step: the bf16 matrix
  // core cuts off what its accumulator cannot hold, always downwards, which over the
  // chunks of a long memory (8192 positive terms, a = 1) put X off by 6e-6.
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb) {
    f32x4 u[NCT];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) u[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const auto kt = keys(4 * nb, m);
#pragma unroll
      for (int t = N - 1; t >= 0; --t)
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) u[ct] = P::mma(kt, vw[m][ct][t], u[ct]);
    }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s.x[nb][ct][j] = fmaf(s.x[nb][ct][j], carry, u[ct][j]);
    // as many tiles' operands at a time as registers are left for (fp32, 256 heads x 1024 rows
    // of 128 x 128: eight 351 us and a backward pass of 700, two 337 and 657)
    constexpr int kGroup = NCT == 2 || sizeof(T) == 4 ? 2 : 8;
    if (nb % kGroup == kGroup - 1) __builtin_amdgcn_sched_barrier(0);
  }
}

// Wave priority by the chunk's number, lower as it rises (from 3 to 0, over and over): of two
// workgroups on a compute unit the one behind goes first. With equal priorities the older
// one always does, ends early and leaves the other alone (512 heads x 2048 rows of
// 128 x 128: 269 us, with this 254; at 64 x 64 253 and 231). Scans that run together read the
// same rows when they happen to keep pace and are better left alone: a training step of
// 4 x 4096 x 16 heads 364 us, with turns 373.
__device__ __forceinline__ void take_turns(int chunk) {
  switch (chunk & 3) {
    case 0: __builtin_amdgcn_s_setprio(3); break;
    case 1: __builtin_amdgcn_s_setprio(2); break;
    case 2: __builtin_amdgcn_s_setprio(1); break;
    default: __builtin_amdgcn_s_setprio(0);
  }
}

// The sums of one segment of 64 * chunks tokens, from X = 0. Bound by the bytes of K and V:
// those of 65536 x 16 heads of 128 x 128 (550 MB with the sums) in 111 us, 5.0 TB/s.
template <typename T, int KD, int NW, int NCT, bool WHOLE>
__global__ __launch_bounds__(64 * NW, 2) void k_decay_sums(DecayPass pass) {
  constexpr int NT = 64 * NW, VS = 16 * NW * NCT;
  // two buffers where two workgroups still share the unit: one barrier per chunk then
  constexpr int NB = sizeof(T) == 2 && KD <= 128 ? 2 : 1;
  __shared__ __align__(256) T Ks[NB][kChunkT * KD];
  __shared__ __align__(256) T Vs[NB][kChunkT * VS];
  __shared__ Powers pw;
  int id = xcd_item(blockIdx.x, gridDim.x);
  const DecayScan &a = scan_of(pass, id);
  const Item it = item_of(a, id, (a.vd + VS - 1) / VS, a.nseg - 1);
  if (it.seg >= last_seg(a, it.len)) return;   // X_n comes from the scan
  const int v0 = VS * it.slice;
  Staged<T, KD, NT> kr;
  Staged<T, VS, NT> vr;
  kr.start(a.ks, a.reverse, a.kd);
  vr.start(a.vs, a.reverse, a.vd - v0);
  const auto fetch = [&](int c) {
    const int r = it.first + c;
    kr.load(chunk_rows<T>(a.k, a.ks, it, 0, a.reverse, r), a.ks, a.reverse, kChunkT);
    vr.load(chunk_rows<T>(a.v, a.vs, it, v0, a.reverse, r), a.vs, a.reverse, kChunkT);
  };
  fetch(0);
  fill_powers(pw, a.log_decay[it.h]);
  __syncthreads();
  fill_sum(pw, kChunkT, a.shift, a.sum_scale);
  State<KD, NCT> s;
#pragma unroll
  for (int nb = 0; nb < KD / 16; ++nb)
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) put(s.x[nb][ct], f32x4{0.f, 0.f, 0.f, 0.f});
  Carry carry(a.log_decay[it.h], it.n > kChunkT);
  for (int c = 0; c < it.n; c += kChunkT) {
    take_turns(c / kChunkT);
    const int buf = NB == 2 ? (c / kChunkT) & 1 : 0;
    kr.store(Ks[buf]);
    vr.store(Vs[buf]);
    __syncthreads();
    if (c + kChunkT < it.n) fetch(c + kChunkT);
    typename Mma<T>::frag vt[NCT][2];
    const lds_t zero = c & a.zero;
    load_values<T, VS, NCT>(lds_of(Vs[buf]) + zero, vt);
    typename Mma<T>::frag vw[2][NCT][sum_terms<T>(WHOLE)];
    weigh_values<T>(vw, vt, pw, a.minus);
    update_state<T>(s, lds_of(Ks[buf]) + zero, vw, carry.next());
    if (NB == 1) __syncthreads();
  }
  store_state<KD, NW, NCT>(a, it, part_of(a, it.bh, it.seg + 1), s);
}

// part of a head's segments: X_0, then X before segment s + 1 = a^seg_len (X before s) + sums
// of s, four elements per thread. Bound by the bytes: 16 heads x 32 states of 128 x 128 read
// and written (67 MB) in 14 us, 4.8 TB/s. (Two elements per thread and twice as many loads
// ahead: calls 1 to 5 us longer.)
__global__ __launch_bounds__(256) void k_decay_prefix(DecayPass pass) {
  int id = blockIdx.y;
  const DecayScan &a = scan_of(pass, id);
  const int e = blockIdx.x * 256 + threadIdx.x, n = a.kd * a.vd / 4;
  const Item it = item_of(a, id, 1, 1);
  const int last = last_seg(a, it.len);
  if (e >= n) return;
  f32x4 x{0.f, 0.f, 0.f, 0.f};
  if (a.x_in) x = reinterpret_cast<const f32x4 *>(a.x_in)[(size_t)it.bh * n + e];
  // a^seg_len, which meets X once per segment, as two floats and a power of two: where it
  // is past fp32's range, its product with X need not be (2^400 takes any X but 0 past it)
  const double t = (double)a.log_decay[it.h] * a.seg_len * 1.4426950408889634074;
  const int two = t > -400. ? t < 400. ? (int)floor(t) : 400 : -400;
  const double d = exp2((t < 400. || t != t ? t : 400.) - two);
  const float hi = (float)d, lo = (float)(d - hi);
  f32x4 *p = reinterpret_cast<f32x4 *>(part_of(a, it.bh, 0)) + e;
  *p = x;
  p += n;
  constexpr int kAhead = 16;   // loads in flight
  for (int s = 0; s < last; s += kAhead, p += kAhead * n) {
    f32x4 u[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (s + k < last) u[k] = p[k * n];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (s + k < last) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float y = ldexpf(x[j], two);
          x[j] = fmaf(y, hi, fmaf(y, lo, u[k][j]));
        }
        p[k * n] = x;
      }
  }
}

// Terms of the pair weights and of X (see above).
template <typename T> constexpr int kRowTerms = sizeof(T) == 2 ? 2 : 1;

// The first terms of four pair weights. They keep within bf16's range, so that a weight past
// it ends as Inf, not as Inf - Inf.
__device__ __forceinline__ f32x4 first_term(f32x4 x) {
  f32x4 t;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    t[j] = to_f32((bf16)__builtin_amdgcn_fmed3f(x[j], -0x1.fep127f, 0x1.fep127f));
  return t;
}

// Waves per SIMD that the register budget of the scan is set for.
constexpr int scan_waves(int elt, int KD, int NCT) {
  return elt == 2 && KD <= 128 && NCT == 1 ? 4 : KD == 256 && elt == 4 ? 1 : 2;
}

template <typename T, int KD, int NW, int NCT, bool WHOLE>
__global__ __launch_bounds__(64 * NW, scan_waves(sizeof(T), KD, NCT)) void k_decay_scan(DecayPass pass) {
  using P = Mma<T>;
  using frag = typename P::frag;
  constexpr int NT = 64 * NW, VS = 16 * NW * NCT, NP = KD / 32, TERMS = kRowTerms<T>;
  __shared__ __align__(256) T Qs[kChunkT * KD];
  __shared__ __align__(256) T Ks[kChunkT * KD];
  __shared__ __align__(256) T Vs[kChunkT * VS];
  // the pair weights as B operands: rows 16 i .. + 15, tokens 32 m .. + 31 in fragment
  // first(i) + m. Second terms behind the first ones; at 256 k columns, where that would
  // leave no room for a second workgroup on the unit, in the values' place once they are read
  // (512 heads x 2048 rows of 256 x 64: 298 us instead of 407).
  constexpr bool kTight = TERMS == 2 && KD == 256;
  static_assert(!kTight || sizeof(Vs) >= 6 * 64 * sizeof(frag), "room for the second terms");
  __shared__ __align__(16) frag Ps[kTight ? 1 : TERMS][6 * 64];
  const auto pairs_of = [&](int term) {
    return kTight && term == 1 ? reinterpret_cast<frag *>(Vs) : Ps[term];
  };
  __shared__ Powers pw;
  const auto first = [](int i) { return (i >= 1) + (i >= 2) + 2 * (i >= 3); };
  int id = xcd_item(blockIdx.x, gridDim.x);
  const DecayScan &a = scan_of(pass, id);
  const Item it = item_of(a, id, (a.vd + VS - 1) / VS, a.nseg);
  const int w = wave_id(), l = lane_id(), g = l >> 4, c16 = l & 15;
  const int v0 = VS * it.slice;
  Staged<T, KD, NT> qr, kr;
  Staged<T, VS, NT> vr;
  qr.start(a.qs, a.reverse, a.kd);
  kr.start(a.ks, a.reverse, a.kd);
  vr.start(a.vs, a.reverse, a.vd - v0);
  const auto fetch_q = [&](int c) {
    qr.load(chunk_rows<T>(a.q, a.qs, it, 0, a.reverse, it.first + c), a.qs, a.reverse, it.n - c);
  };
  const auto fetch = [&](int c) {
    const int r = it.first + c, n = it.n - c;
    kr.load(chunk_rows<T>(a.k, a.ks, it, 0, a.reverse, r), a.ks, a.reverse, n);
    vr.load(chunk_rows<T>(a.v, a.vs, it, v0, a.reverse, r), a.vs, a.reverse, n);
  };
  if (it.n > 0) {
    fetch_q(0);
    fetch(0);
  }
  State<KD, NCT> s;
  load_state<KD, NW, NCT>(a, it, s);
  fill_powers(pw, a.log_decay[it.h]);
#pragma unroll
  for (int t = 0; t < (kTight ? 1 : TERMS); ++t)
    for (int i = threadIdx.x; i < 6 * 64; i += NT) Ps[t][i] = P::splat(0.f);   // j > i stays 0
  __syncthreads();
  fill_rows(pw, a);
  // a lane's outputs: row c16 of a block (in reversed order from the chunk's last block
  // down), 4 NCT columns
  const int vc = 16 * NCT * w + 4 * NCT * g;
  const uint32_t ostep = (a.reverse ? -16u : 16u) * (uint32_t)a.os.t * (uint32_t)sizeof(T);
  const uint32_t ooff = ((a.reverse ? kChunkT - 1 - c16 : c16) * (uint32_t)a.os.t + vc) *
                  (uint32_t)sizeof(T);
  Carry carry(a.log_decay[it.h], it.n > kChunkT);
  for (int c = 0; c < it.n; c += kChunkT) {
    if (pass.n == 1) take_turns(c / kChunkT);
    const int n = min(kChunkT, it.n - c);
    qr.store(Qs);
    kr.store(Ks);
    vr.store(Vs);
    if (c == 0 || n < kChunkT) fill_sum(pw, n, a.shift, a.sum_scale);
    __syncthreads();
    // At 256 k columns the next queries wait until the pairs' operands leave registers free.
    // (Their fetch has no condition, which would keep the old rows in registers until then;
    // behind the last chunk it reads nothing.)
    constexpr bool kLateQ = KD == 256;
    if (kLateQ || c + kChunkT < it.n) {
      if (!kLateQ) fetch_q(c + kChunkT);
      fetch(c + kChunkT);
    }

    const lds_t zero = c & a.zero;
    const RowReader<T, KD> queries(lds_of(Qs) + zero), keys(lds_of(Ks) + zero);

    // D o K Q^T, the ten 16 x 16 tiles with j <= i shared out over the waves
    const auto pairs = [&] {
      for (int t = w; t < 10; t += NW) {
        const int ib = (t >= 1) + (t >= 3) + (t >= 6), jb = t - ib * (ib + 1) / 2;
        const int e = 16 * (ib - jb) + c16 - 4 * g;
        float wt[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) wt[j] = pw.pair[16 + e - j];
        f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          x = P::mma(keys(jb, p), queries(ib, p), x);
          if (p % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // not all operands at once
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = e >= j ? x[j] * wt[j] : 0.f;   // (an Inf of j > i goes)
        const auto put = [&](int term, int half, f32x4 y) {
          store4(reinterpret_cast<T *>(pairs_of(term) + (first(ib) + (jb >> 1)) * 64 + l) + 4 * half, y);
        };
        if constexpr (TERMS == 1) {
          put(0, jb & 1, x);
        } else {
          const f32x4 x0 = first_term(x);
          put(0, jb & 1, x0);
          put(1, jb & 1, x - x0);
          if (kTight && ib == jb && !(jb & 1)) put(1, 1, f32x4{0.f, 0.f, 0.f, 0.f});   // j > i
        }
      }
    };
    if (!kTight) pairs();

    // X^T Q^T
    f32x4 o[4][NCT];
#pragma unroll
    for (int ib = 0; ib < 4; ++ib)
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) o[ib][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      frag xf[NCT][TERMS];
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] = s.x[2 * p][ct][j];
          x[4 + j] = s.x[2 * p + 1][ct][j];
        }
        split8(x, xf[ct], a.minus);
      }
#pragma unroll
      for (int ib = 0; ib < 4; ++ib) {
        const frag qf = queries(ib, p);
#pragma unroll
        for (int u = TERMS - 1; u >= 0; --u)
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) o[ib][ct] = P::mma(xf[ct][u], qf, o[ib][ct]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (kLateQ && !kTight) fetch_q(c + kChunkT);
#pragma unroll
    for (int ib = 0; ib < 4; ++ib) {
      const float f = pw.row[16 * ib + c16];
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[ib][ct][j] *= f;
    }
    frag vt[NCT][2], vw[2][NCT][sum_terms<T>(WHOLE)];
    load_values<T, VS, NCT>(lds_of(Vs) + zero, vt);
    __syncthreads();
    if (kTight) {
      pairs();
      fetch_q(c + kChunkT);   // (in front of the pairs, spilled: a tenth more)
      __syncthreads();
    }

    // + V^T (D o K Q^T)
    const auto rows = chunk_rows<T>(a.o, a.os, it, v0, a.reverse, it.first + c);
#pragma unroll
    for (int ib = 0; ib < 4; ++ib) {
#pragma unroll
      for (int m = 0; m <= ib / 2; ++m) {
#pragma unroll
        for (int u = TERMS - 1; u >= 0; --u) {
          const frag pf = pairs_of(u)[(first(ib) + m) * 64 + l];
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) o[ib][ct] = P::mma(vt[ct][m], pf, o[ib][ct]);
        }
      }
      put_row<T, NCT>(rows, c16 < n - 16 * ib && vc < a.vd - v0 ? ooff + zero + ib * ostep : kOutside,
                      o[ib]);
    }
    weigh_values<T>(vw, vt, pw, a.minus);
    update_state<T>(s, lds_of(Ks) + zero, vw, n == kChunkT ? carry.next() : pw.a[n]);
    __syncthreads();
  }

  if (a.x_out && it.seg == last_seg(a, it.len))
    store_state<KD, NW, NCT>(a, it, a.x_out + (size_t)it.bh * (a.kd * a.vd), s);
  // the rows of the segment past the sequence's end
  const int end = min(a.L, it.first + a.seg_len);
  constexpr int kPer = 16 / (int)sizeof(T), kUnits = VS / kPer;
  for (int r = it.first + it.n + threadIdx.x / kUnits; r < end; r += NT / kUnits) {
    const int col = v0 + threadIdx.x % kUnits * kPer;
    if (col < a.vd)
      *reinterpret_cast<u32x4 *>(static_cast<T *>(a.o) + it.b * a.os.b + it.h * a.os.h +
                                 r * a.os.t + col) = u32x4{0, 0, 0, 0};
  }
}

template <typename T, int KD, int NW, int NCT, bool WHOLE>
hipError_t launch(const DecayPass &pass, bool sums, hipStream_t st) {
  const DecayScan &a = pass.scan[0];
  const int heads = pass.n * a.BH * ((a.vd + a.slice - 1) / a.slice);
  if (sums)
    k_decay_sums<T, KD, NW * NCT, 1, WHOLE><<<heads * (a.nseg - 1), 64 * NW * NCT, 0, st>>>(pass);
  else
    k_decay_scan<T, KD, NW, NCT, WHOLE><<<heads * a.nseg, 64 * NW, 0, st>>>(pass);
  return hipGetLastError();
}

// fp32 inputs keep one value tile per wave, in twice as many waves: their operands take
// twice the registers. So do the sums, which have registers to spare: two buffers and eight
// waves against one and four, padded prompts of 6 x 1999 rows 97 to 100 -> 94 to 98 us.
template <typename T, bool WHOLE>
hipError_t dispatch(const DecayPass &p, bool sums, hipStream_t st) {
  constexpr int NW = sizeof(T) == 2 ? 4 : 8, NCT = 8 / NW;
  const int kd = p.scan[0].kd;
  const bool wide = p.scan[0].slice == 128;
  if (kd <= 64)
    return wide ? launch<T, 64, NW, NCT, WHOLE>(p, sums, st)
                : launch<T, 64, 4, 1, WHOLE>(p, sums, st);
  if (kd <= 128)
    return wide ? launch<T, 128, NW, NCT, WHOLE>(p, sums, st)
                : launch<T, 128, 4, 1, WHOLE>(p, sums, st);
  return launch<T, 256, 4, 1, WHOLE>(p, sums, st);
}
hipError_t dispatch(const DecayPass &p, Dt dt, bool sums, hipStream_t st) {
  if (dt == Dt::F32) return dispatch<float, true>(p, sums, st);
  for (int i = 0; i < p.n; ++i)
    if (p.scan[i].x_out) return dispatch<bf16, true>(p, sums, st);
  return dispatch<bf16, false>(p, sums, st);
}

}  // namespace

hipError_t launch_decay_sums(const DecayPass &p, Dt dt, hipStream_t st) {
  return dispatch(p, dt, true, st);
}
hipError_t launch_decay_prefix(const DecayPass &p, hipStream_t st) {
  const int n = p.scan[0].kd * p.scan[0].vd / 4;
  k_decay_prefix<<<dim3((n + 255) / 256, p.n * p.scan[0].BH), 256, 0, st>>>(p);
  return hipGetLastError();
}
hipError_t launch_decay_scan(const DecayPass &p, Dt dt, hipStream_t st) {
  return dispatch(p, dt, false, st);
}

}  // namespace favor
