// decay.hpp - launchers of the decayed linear attention and the dropout (internal to
// libfavor; decay.hip, decay_step.hip, dropout.hip; called from decay_api.cpp).
#pragma once

#include "kernels.hpp"

namespace favor {

// Element strides of a [B][H][L][d] tensor whose rows are contiguous.
struct Rows {
  int64_t b, h, t;
};

// One scan over a sequence per (batch, head), in one of two time orders (r = the row's
// place in the scan's order, a = the head's decay, n = the sequence's length):
//   o_r = row_scale a^(r + shift) q_r X_0 + pair_scale sum_{s <= r} a^(r - s) (q_r . k_s) v_s
//   X_n = a^n X_0 + sum_s sum_scale a^(n - shift - s) k_s v_s^T
// The forward pass is (q, k, v) with shift 1, X the state after the last token; dQ is
// (dout, V, K) on the transposed state; dV is (K, Q, dout) and dK (V, dout, Q) in
// reversed order with shift 0, X the state's gradient with its decay applied. X_0, X_n
// and part may be transposed ([vd][kd]), so that scans on X and on X^T share them.
struct DecayScan {
  const void *q, *k, *v;   // kd, kd and vd columns
  void *o;                 // vd columns
  Rows qs, ks, vs, os;
  const float *log_decay;  // [H]
  const int32_t *lengths;  // [B], or null: every sequence has L tokens
  const float *x_in;       // X_0 [BH][kd][vd], or null for zeros
  float *x_out;            // X_n, or null
  float *part;             // nseg > 1: [BH][nseg][X], X before each segment (first their sums)
  int x_t;                 // x_in, x_out and part hold [vd][kd]
  int BH, H, L, kd, vd;
  int seg_len, nseg;       // segments of seg_len rows (a multiple of 64)
  int slice;               // columns of v that one workgroup takes: 64, or 128 (kd <= 128)
  int reverse, shift;
  float pair_scale, row_scale, sum_scale;
  int zero = 0;   // the loops' addresses depend on it: they are formed anew, not kept
  uint32_t minus[2] = {0x0000bf80u, 0xbf800000u};   // bf16 pairs (-1, 0) and (0, -1)
};

// Scans launched together: the same kd, vd, slices, heads and segments. At most three.
struct DecayPass {
  DecayScan scan[3];
  int n;
};

// The sums of every segment but the last, in part.
hipError_t launch_decay_sums(const DecayPass &p, Dt dt, hipStream_t st);
// part: from each segment's sums to X before the segment that follows it.
hipError_t launch_decay_prefix(const DecayPass &p, hipStream_t st);
// The rows, each segment from the X before it.
hipError_t launch_decay_scan(const DecayPass &p, Dt dt, hipStream_t st);

// One token of B sequences on the states [n_slots][H][dk][dv], in place.
struct DecayStep {
  const void *q, *k, *v;
  void *o;
  Rows qs, ks, vs, os;     // t unused
  const float *log_decay;
  const int32_t *slots;    // [B] places of the sequences' states, or null: b
  float *state;
  int n_slots;
  int B, H, dk, dv;
  float scale;
};
hipError_t launch_decay_step(const DecayStep &a, Dt dt, hipStream_t st);

struct Dropout {
  const void *x, *residual;   // residual nullable
  void *y;
  int64_t n;
  uint32_t threshold;         // of 2^16: an element stays if its 16 bits are not below
  float scale;                // of the elements that stay
  uint64_t seed, offset;
  const uint64_t *rng;        // {seed, offset} in device memory, or null
};
hipError_t launch_dropout(const Dropout &a, Dt dt, hipStream_t st);

}  // namespace favor
