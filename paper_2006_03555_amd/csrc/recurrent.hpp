// recurrent.hpp - launchers of the short convolution, the selective scan and the beam
// search's step (internal to libfavor; conv.hip, scan.hip, scan_backward.hip, scan_step.hip,
// beam.hip; called from recurrent_api.cpp).
#pragma once

#include "decay.hpp"

namespace favor {

// Short causal convolution over [B][L][D] rows of contiguous channels.
struct Conv {
  const void *x;
  const float *w, *bias;    // [D][width], [D] or null
  const int32_t *lengths;   // [B] or null
  const void *state_in;     // [B][width - 1][D] (the last inputs before x), or null for zeros
  void *state_out;          // those after it, or null
  void *y;
  Rows xs, ys;              // h unused
  int B, L, D, width, silu;
  int run;                  // tokens of one thread, at least width - 1
  // backward
  const void *dy, *dstate_out;
  void *dx, *dstate_in;
  float *dw, *dbias;
  float *part;              // [conv_part_rows][width + 1][D]
  Rows dys, dxs;
  // single tokens: state_out is the pool [n_slots][width - 1][D]
  const int32_t *slots;
  int n_slots;
};
hipError_t launch_conv(const Conv &a, Dt dt, hipStream_t st);
int64_t conv_part_rows(int B, int L, int D, int width, Dt dt);
hipError_t launch_conv_backward(const Conv &a, Dt dt, hipStream_t st);
// Sums over the rows of part [rows][width + 1][D] (null: zeros), to dw and dbias.
hipError_t launch_conv_sums(const Conv &a, int rows, hipStream_t st);
hipError_t launch_conv_step(const Conv &a, Dt dt, hipStream_t st);

// Selective scan: h = exp(s A) h + s x B, y = (C h + D x) silu(z), s = softplus(dt + bias).
// x, dt, z, y are [B][L][D] rows, B and C [B][L][G][N] (Rows: h is the group).
struct Scan {
  const void *x, *dt, *b, *c, *z;   // z nullable
  const float *A;                   // [D][N]
  const float *skip, *bias;         // [D], nullable
  const int32_t *lengths;
  const float *h_in;                // [B][D][N], or null for zeros
  float *h_out;
  void *y;
  Rows xs, dts, bs, cs, zs, ys;
  int B, L, D, N, G, softplus;
  int chunks, nseg;                 // chunks of kScanTokens tokens in one segment; segments
  int seg0;                         // the first segment of this launch
  int sum_states;                   // states of a workgroup of the segments' sums (of kScanStates)
  int subs;                         // backward: tiles of one workgroup
  // nseg > 1: the states before each segment [B][nseg][D][N] (first: the segments' sums) and
  // the segments' sums of s [B][nseg][D]
  float *part, *steps;
  // backward: segments are single chunks
  const void *dy;
  const float *dh_out;
  float *dh_in;
  void *dx, *ddt, *db, *dc, *dz;
  float *dA, *dskip, *dbias;
  float *part_r;                    // as part, for the gradient of the state, from the right
  float *part_a;                    // [B][nseg][D][N] sums of dA
  float *part_d, *part_s;           // [B][nseg][D] sums of dskip and of ddt
  float *part_b, *part_c;           // [workgroups of a group's channels][B][L][G][N]
  Rows dys, dxs, ddts, dbs, dcs, dzs;
  // single tokens: h_out is the pool [n_slots][D][N]
  const int32_t *slots;
  int n_slots;
};
constexpr int kScanTokens = 128;     // of one chunk
constexpr int kScanStates = 16;      // of one pass over a chunk
constexpr int kScanBackTile = 32;    // channels of one tile of the backward pass
// Workgroups of one launch over chunks (of rows of B and C): a launch takes less than 2^32 threads,
// so what is longer takes several launches (turns).
constexpr int kScanBlocks = 1 << 20, kLowBlocks = 1 << 16;
// The sums of the segments but the last, in part and steps; backward, where a segment is one
// chunk: of all of them, and in part_r too.
hipError_t launch_scan_sums(const Scan &a, Dt dt, hipStream_t st);
hipError_t launch_scan_backward_parts(const Scan &a, Dt dt, hipStream_t st);
// part (part_r): from sums to the states before (behind) each segment; backward: dh_in.
hipError_t launch_scan_prefix(const Scan &a, bool backward, hipStream_t st);
hipError_t launch_scan(const Scan &a, Dt dt, hipStream_t st);
hipError_t launch_scan_backward(const Scan &a, Dt dt, hipStream_t st);
// dB and dC, dA, dskip and dbias from their parts.
hipError_t launch_scan_backward_sums(const Scan &a, Dt dt, hipStream_t st);
hipError_t launch_scan_step(const Scan &a, Dt dt, hipStream_t st);

// Beam search's choice among K V continuations of each of B entries.
struct BeamSelect {
  const void *logits;
  Rows ls;                   // (batch, beam); t unused
  const float *scores;       // [B][K]
  const uint8_t *ended;      // [B][K] or null
  int B, K, V, n, end_token;
  int pieces, piece_len;     // of a row
  float2 *stats;             // [B K][pieces]: maximum, sum of exp(x - maximum)
  uint64_t *keys;            // [B K][pieces][n], best first; 0: none
  float *out_scores;         // [B][n]
  int32_t *parent, *token;   // [B][n]
};
hipError_t launch_beam_pieces(const BeamSelect &a, Dt dt, hipStream_t st);
hipError_t launch_beam_merge(const BeamSelect &a, hipStream_t st);

constexpr int kBeamPools = 64;       // pools of one launch
// 16-byte units that one workgroup copies; 8 x 8 beams, 24 layers 43 us with 2048, 45 with 4096
constexpr int kBeamPieceUnits = 2048;
constexpr int kBeamPieces = 1 << 23;   // of one launch (its threads are less than 2^32)
struct BeamReorder {
  const int32_t *parent, *slots;   // [B][K]; slots nullable
  int32_t *new_slots;
  int B, K, n_pools;
  struct { void *data; int32_t units, n_slots; } pool[kBeamPools];   // units of 16 bytes per slot
  int first[kBeamPools + 1];       // the first of a pool's pieces
};
hipError_t launch_beam_reorder(const BeamReorder &a, hipStream_t st);

}  // namespace favor
