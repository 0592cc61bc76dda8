// decay_api.cpp - the C ABI of the decayed linear attention and the dropout: argument
// validation, workspace sizing, launch planning and dispatch. As in favor_api.cpp,
// validation is plain host code that touches no device.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "../../include/favor.h"
#include "decay.hpp"

namespace {

using favor::DecayScan;
using favor::Rows;

favor_status fail(favor_status st, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return favor::report(st, buf);
}
favor_status ok() { return favor::report(FAVOR_OK, ""); }

#define FAVOR_TRY(expr)                \
  do {                                 \
    favor_status st__ = (expr);        \
    if (st__ != FAVOR_OK) return st__; \
  } while (0)

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The integer in an enum-typed field (a C caller may store any int there).
int raw_enum(const void *p) {
  int v;
  std::memcpy(&v, p, sizeof v);
  return v;
}

favor_status check_ptr(const void *p, const char *name, bool needed, size_t align = 16) {
  if (!needed) return FAVOR_OK;
  if (!p) return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s is NULL", name);
  if (!aligned(p, align))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s is not %zu-byte aligned", name, align);
  return FAVOR_OK;
}
favor_status check_optional(const void *p, const char *name, size_t align = 16) {
  return check_ptr(p, name, p != nullptr, align);
}

// An output that is written while an input of the same size is read: the two may be one
// where `same` says so (each element is then read first), and must not overlap otherwise.
favor_status check_apart(const void *out, const char *name, const void *in, const char *other,
                         int64_t bytes, bool same) {
  if (!out || !in || (out == in && same)) return FAVOR_OK;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out), b = reinterpret_cast<uintptr_t>(in);
  if ((a > b ? a - b : b - a) >= (uint64_t)bytes) return FAVOR_OK;
  return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s overlaps %s", name, other);
}
int64_t state_bytes(const favor_decay_desc *g) {
  return (int64_t)sizeof(float) * g->B * g->H * g->dk * g->dv;
}

favor_status device_result(hipError_t e, const char *what) {
  if (e != hipSuccess) return fail(FAVOR_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

constexpr int kMaxL = 1 << 30;
constexpr int64_t kMaxStride = (int64_t)1 << 46;   // element offsets stay within 64 bits
// the kernels reach a chunk's 64 rows by 32-bit offsets
constexpr int64_t kMaxTokenBytes = 1 << 25;
enum Op { kOpForward = 0, kOpBackward = 1, kOpStep = 2 };

struct Tensor {
  const char *name;
  const favor_strides *s;
  int d;
  bool out;
};

// Strides of one tensor; dimensions of size 1 or less have none.
favor_status check_strides(const favor_decay_desc *g, const Tensor &t, int op) {
  const int64_t size[3] = {g->B, g->H, op == kOpStep ? 1 : g->L};
  const int64_t stride[3] = {t.s->batch, t.s->head, t.s->token};
  const int unit = raw_enum(&g->dtype) == FAVOR_BF16 ? 8 : 4;
  if (!stride[0] && !stride[1] && !stride[2]) return FAVOR_OK;   // contiguous
  int64_t reach = 0;
  for (int i = 0; i < 3; ++i) {
    if (size[i] <= 1) continue;
    if (stride[i] < 0)
      return fail(FAVOR_ERR_INVALID_ARGUMENT, "a stride of %s is negative", t.name);
    if (stride[i] % unit != 0)
      return fail(FAVOR_ERR_INVALID_ARGUMENT,
                  "strides of %s must be multiples of 16 bytes (%d elements)", t.name, unit);
    if (i == 2 && stride[i] > kMaxTokenBytes / (16 / unit))
      return fail(FAVOR_ERR_UNSUPPORTED, "the token stride of %s exceeds 2^25 bytes", t.name);
    if (stride[i] > kMaxStride / (size[i] - 1) || (reach += stride[i] * (size[i] - 1)) > kMaxStride)
      return fail(FAVOR_ERR_UNSUPPORTED, "%s reaches past 2^46 elements", t.name);
  }
  if (!t.out) return FAVOR_OK;
  // rows written must not share elements: taken by stride, each dimension steps over
  // everything inside it
  int at[3] = {0, 1, 2};
  std::sort(at, at + 3, [&](int i, int j) { return stride[i] < stride[j]; });
  int64_t inner = t.d;
  for (int i : at) {
    if (size[i] <= 1) continue;
    if (stride[i] < inner)
      return fail(FAVOR_ERR_INVALID_ARGUMENT, "rows of %s overlap", t.name);
    inner += stride[i] * (size[i] - 1);
  }
  return FAVOR_OK;
}

favor_status validate(const favor_decay_desc *g, int op) {
  if (!g) return fail(FAVOR_ERR_INVALID_ARGUMENT, "descriptor is NULL");
  if (op < kOpForward || op > kOpStep)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "unknown operation %d", op);
  if (g->B < 0 || g->H < 0 || g->L < 0)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "negative size B=%d H=%d L=%d", g->B, g->H, g->L);
  if (g->dk <= 0 || g->dv <= 0)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "dk=%d and dv=%d must be positive", g->dk, g->dv);
  const int dt = raw_enum(&g->dtype);
  if (dt != FAVOR_F32 && dt != FAVOR_BF16)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "unknown dtype %d", dt);
  if (!std::isfinite(g->scale))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "scale must be finite");
  if (g->L > kMaxL) return fail(FAVOR_ERR_UNSUPPORTED, "L=%d exceeds 2^30", g->L);
  if (g->dk % 8 != 0 || g->dv % 8 != 0 || g->dk > 256 || g->dv > 256)
    return fail(FAVOR_ERR_UNSUPPORTED,
                "dk=%d dv=%d not supported (multiples of 8, at most 256)", g->dk, g->dv);
  const long long bh = (long long)g->B * g->H;
  if (bh > 65535) return fail(FAVOR_ERR_UNSUPPORTED, "B*H=%lld exceeds 65535", bh);
  const Tensor ts[] = {{"Q", &g->q, g->dk, false},      {"K", &g->k, g->dk, false},
                       {"V", &g->v, g->dv, false},      {"out", &g->out, g->dv, op != kOpBackward},
                       {"dout", &g->grad_out, g->dv, false}, {"dQ", &g->grad_q, g->dk, true},
                       {"dK", &g->grad_k, g->dk, true}, {"dV", &g->grad_v, g->dv, true}};
  for (int i = 0; i < 8; ++i) {
    if (i == 3 ? op == kOpBackward : i > 3 && op != kOpBackward) continue;
    FAVOR_TRY(check_strides(g, ts[i], op));
  }
  return FAVOR_OK;
}

Rows rows_of(const favor_decay_desc *g, const favor_strides &s, int d) {
  if (!s.batch && !s.head && !s.token)
    return {(int64_t)g->H * g->L * d, (int64_t)g->L * d, d};
  return {g->B > 1 ? s.batch : 0, g->H > 1 ? s.head : 0, g->L > 1 ? s.token : 0};
}

favor::Dt dt_of(const favor_decay_desc *g) {
  return raw_enum(&g->dtype) == FAVOR_BF16 ? favor::Dt::BF16 : favor::Dt::F32;
}

// How a scan with kd k columns and vd value columns is cut: its value columns into slices,
// one per workgroup, and its rows into segments. A call of several segments runs a pass
// for their sums and one that chains them first, so K and V are read twice.
struct Cut {
  int slice;
  int seg_len, nseg;
};

// Whole calls in us (one to eight chunks of 64 rows per segment; a chunk takes a workgroup
// that has a compute unit for itself 3 us at 64 x 64 bf16, 4.5 at 128 x 128, 6 and 9 in fp32):
//   Long sequences: segments for 512 workgroups, two on each of the 256 compute units, as
//   long as they have 256 rows.
//   Shorter ones: as many segments as it takes for 256 workgroups, of one chunk at least,
//   from four chunks on. B1 H8, with 256-row segments / with this: bf16 64 x 64 L512
//   25.3 / 14.2, L4096 28.1 / 23.8; 128 x 128 L1024 34.3 / 24.7; fp32 128 x 128 L512
//   59.1 / 25.5, L4096 88.9 / 62.2. For 512 workgroups instead: bf16 64 x 64 L4096 29.0,
//   fp32 128 x 128 L2048 43.0 -> 49.5. Two chunks apart: bf16 64 x 64 L128 10.0 / 13.4.
//   Slices of 64 value columns for wider values while the chunks are few: twice as many
//   workgroups, each with half the work per chunk and the pair weights to itself. B1 H8
//   128 x 128, slices of 128 / 64: bf16 L128 17.3 / 12.7, L4096 38.8 / 39.7, B2 H16 L8192
//   117 / 130; fp32 L2048 45.3 / 43.0, L4096 62.2 / 67.4. With more than 128 k columns X
//   leaves room for no more.
constexpr int kFullWorkgroups = 512, kMinRows = 256;
constexpr int kSomeWorkgroups = 256, kMinSplitTiles = 4;
constexpr int kNarrowTiles = 512, kNarrowTilesF32 = 256;

// scans: how many run together on g's heads.
Cut cut_of(const favor_decay_desc *g, int kd, int vd, int scans) {
  const int tiles = std::max(1, (g->L + 63) / 64);
  const int heads = g->B * g->H * scans;
  const bool few = (long long)heads * tiles * ((vd + 127) / 128) <=
                   (raw_enum(&g->dtype) == FAVOR_BF16 ? kNarrowTiles : kNarrowTilesF32);
  Cut c;
  c.slice = kd > 128 || vd <= 64 || few ? 64 : 128;
  const int have = heads * ((vd + c.slice - 1) / c.slice);
  const int full = std::min(kFullWorkgroups / have, tiles / (kMinRows / 64));
  const int some = tiles < kMinSplitTiles ? 1 : std::min(kSomeWorkgroups / have, tiles);
  const int want = std::max(1, std::max(full, some));
  const int per = (tiles + want - 1) / want;
  c.seg_len = 64 * per;
  c.nseg = (tiles + per - 1) / per;
  return c;
}

// The backward pass sums for two scans and then runs three; its segments are cut for two.
constexpr int kBackwardScans = 2;

// Floats of one scan's segment states.
size_t part_floats(const favor_decay_desc *g, int nseg) {
  return nseg > 1 ? (size_t)g->B * g->H * nseg * g->dk * g->dv : 0;
}

// Workspace: the segment states of the forward pass's scan, or of the backward pass's two
// (S for dQ, its gradient R for dK and dV). The backward scans on [dv][dk] and [dk][dv]
// share one plan.
size_t workspace_of(const favor_decay_desc *g, int op) {
  if ((long long)g->B * g->H == 0 || g->L == 0) return 0;
  return round_up(part_floats(g, cut_of(g, g->dk, g->dv, op == kOpBackward ? kBackwardScans : 1).nseg) * sizeof(float) * (op == kOpBackward ? 2 : 1), 256);
}

favor_status check_workspace(const void *ws, size_t bytes, size_t need) {
  if (need == 0) return FAVOR_OK;
  if (!ws) return fail(FAVOR_ERR_INVALID_ARGUMENT, "workspace is NULL");
  if (!aligned(ws, 256))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "workspace is not 256-byte aligned");
  if (bytes < need)
    return fail(FAVOR_ERR_WORKSPACE_TOO_SMALL, "workspace %zu bytes, need %zu", bytes, need);
  return FAVOR_OK;
}

// A scan of g: kd, vd (exchanged on the transposed state), its segments and the arguments
// that all have in common.
DecayScan scan_of(const favor_decay_desc *g, bool swapped, int scans, const float *log_decay,
                  const int32_t *lengths) {
  DecayScan a{};
  a.log_decay = log_decay;
  a.lengths = lengths;
  a.BH = g->B * g->H;
  a.H = g->H;
  a.L = g->L;
  a.kd = swapped ? g->dv : g->dk;
  a.vd = swapped ? g->dk : g->dv;
  a.x_t = swapped;
  const Cut c = cut_of(g, g->dk, g->dv, scans);
  a.seg_len = c.seg_len;
  a.nseg = c.nseg;
  a.slice = cut_of(g, a.kd, a.vd, scans).slice;
  a.pair_scale = g->scale;
  return a;
}

// Forward order: the scale on the rows; reversed: on the sums, so that X takes the
// gradient of a state as it is.
void forward_order(DecayScan &a, float scale) {
  a.shift = 1;
  a.row_scale = scale;
  a.sum_scale = 1.f;
}
void reversed_order(DecayScan &a, float scale) {
  a.reverse = 1;
  a.row_scale = 1.f;
  a.sum_scale = scale;
}

favor_status run_sums(const favor::DecayPass &p, favor::Dt dt, hipStream_t st, const char *what) {
  if (p.scan[0].nseg <= 1) return ok();
  hipError_t e;
  {
    favor::LaunchTimer t(favor::kKerDecaySums, st);
    e = favor::launch_decay_sums(p, dt, st);
  }
  if (e != hipSuccess) return device_result(e, what);
  favor::LaunchTimer t(favor::kKerDecayPrefix, st);
  return device_result(favor::launch_decay_prefix(p, st), what);
}

favor_status run_scan(const favor::DecayPass &p, favor::Dt dt, hipStream_t st, const char *what) {
  favor::LaunchTimer t(favor::kKerDecayScan, st);
  return device_result(favor::launch_decay_scan(p, dt, st), what);
}

}  // namespace

extern "C" {

favor_status favor_validate_decay_desc(const favor_decay_desc *g, int op) {
  FAVOR_TRY(validate(g, op));
  return ok();
}

size_t favor_decay_workspace_size(const favor_decay_desc *g, int backward) {
  const int op = backward ? kOpBackward : kOpForward;
  if (validate(g, op) != FAVOR_OK) return 0;
  return workspace_of(g, op);
}

favor_status favor_attn_decay(const favor_decay_desc *g, const void *Q, const void *K,
                              const void *V, const float *log_decay, const int32_t *lengths,
                              void *out, const float *state_in, float *state_out, void *ws,
                              size_t ws_bytes, hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpForward));
  const bool heads = (long long)g->B * g->H > 0, work = heads && g->L > 0;
  const void *ptrs[] = {Q, K, V, out};
  const char *names[] = {"Q", "K", "V", "out"};
  for (int i = 0; i < 4; ++i) FAVOR_TRY(check_ptr(ptrs[i], names[i], work));
  FAVOR_TRY(check_ptr(log_decay, "log_decay", heads, 4));
  FAVOR_TRY(check_optional(lengths, "lengths", 4));
  FAVOR_TRY(check_optional(state_in, "state_in"));
  FAVOR_TRY(check_optional(state_out, "state_out"));
  if (work && (out == Q || out == K || out == V))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "out must not be an input");
  FAVOR_TRY(check_apart(state_out, "state_out", state_in, "state_in", state_bytes(g), true));
  if (!heads || (!work && !state_out)) return ok();
  FAVOR_TRY(check_workspace(ws, ws_bytes, workspace_of(g, kOpForward)));
  favor::DecayPass p{};
  p.n = 1;
  DecayScan &a = p.scan[0];
  a = scan_of(g, false, 1, log_decay, lengths);
  a.q = Q;
  a.k = K;
  a.v = V;
  a.o = out;
  a.qs = rows_of(g, g->q, g->dk);
  a.ks = rows_of(g, g->k, g->dk);
  a.vs = rows_of(g, g->v, g->dv);
  a.os = rows_of(g, g->out, g->dv);
  a.x_in = state_in;
  a.x_out = state_out;
  a.part = static_cast<float *>(ws);
  forward_order(a, g->scale);
  FAVOR_TRY(run_sums(p, dt_of(g), stream, "favor_attn_decay segment sums"));
  return run_scan(p, dt_of(g), stream, "favor_attn_decay");
}

favor_status favor_attn_decay_backward(const favor_decay_desc *g, const void *Q, const void *K,
                                       const void *V, const float *log_decay,
                                       const int32_t *lengths, const float *state_in,
                                       const void *dout, const float *dstate_out, void *dQ,
                                       void *dK, void *dV, float *dstate_in, void *ws,
                                       size_t ws_bytes, hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpBackward));
  const bool heads = (long long)g->B * g->H > 0, work = heads && g->L > 0;
  const void *ptrs[] = {Q, K, V, dout, dQ, dK, dV};
  const char *names[] = {"Q", "K", "V", "dout", "dQ", "dK", "dV"};
  for (int i = 0; i < 7; ++i) FAVOR_TRY(check_ptr(ptrs[i], names[i], work));
  FAVOR_TRY(check_ptr(log_decay, "log_decay", heads, 4));
  FAVOR_TRY(check_optional(lengths, "lengths", 4));
  FAVOR_TRY(check_optional(state_in, "state_in"));
  FAVOR_TRY(check_optional(dstate_out, "dstate_out"));
  FAVOR_TRY(check_optional(dstate_in, "dstate_in"));
  if (work)
    for (int o = 4; o < 7; ++o)
      for (int i = 0; i < o; ++i)
        if (ptrs[o] == ptrs[i])
          return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s must not be %s", names[o], names[i]);
  FAVOR_TRY(check_apart(dstate_in, "dstate_in", dstate_out, "dstate_out", state_bytes(g), true));
  FAVOR_TRY(check_apart(dstate_in, "dstate_in", state_in, "state_in", state_bytes(g), false));
  if (!heads || (!work && !dstate_in)) return ok();
  FAVOR_TRY(check_workspace(ws, ws_bytes, workspace_of(g, kOpBackward)));
  const favor::Dt dt = dt_of(g);
  const Rows qs = rows_of(g, g->q, g->dk), ks = rows_of(g, g->k, g->dk),
             vs = rows_of(g, g->v, g->dv), ds = rows_of(g, g->grad_out, g->dv);
  // dQ: queries dout, keys V, values K, on S^T; dK: queries V, keys dout, values Q, on R^T;
  // dV: queries K, keys Q, values dout, on R
  DecayScan dq = scan_of(g, true, kBackwardScans, log_decay, lengths), dk = dq;
  DecayScan dv = scan_of(g, false, kBackwardScans, log_decay, lengths);
  dq.q = dk.k = dv.v = dout;
  dq.qs = dk.ks = dv.vs = ds;
  dq.k = dk.q = V;
  dq.ks = dk.qs = vs;
  dq.v = dv.q = K;
  dq.vs = dv.qs = ks;
  dk.v = dv.k = Q;
  dk.vs = dv.ks = qs;
  dq.o = dQ;
  dk.o = dK;
  dv.o = dV;
  dq.os = rows_of(g, g->grad_q, g->dk);
  dk.os = rows_of(g, g->grad_k, g->dk);
  dv.os = rows_of(g, g->grad_v, g->dv);
  dq.x_in = state_in;
  dk.x_in = dv.x_in = dstate_out;
  dv.x_out = dstate_in;
  dq.part = static_cast<float *>(ws);
  dk.part = dv.part = dq.part + part_floats(g, dq.nseg);
  forward_order(dq, g->scale);
  reversed_order(dk, g->scale);
  reversed_order(dv, g->scale);
  // S of the segments from (K, V) and R from (Q, dout), both [dk][dv]
  DecayScan s = dv;
  s.k = K;
  s.ks = ks;
  s.v = V;
  s.vs = vs;
  s.x_in = state_in;
  s.part = dq.part;
  s.reverse = 0;
  forward_order(s, g->scale);
  FAVOR_TRY(run_sums({{s, dv}, 2}, dt, stream, "favor_attn_decay_backward segment sums"));
  if (!work) return run_scan({{dv}, 1}, dt, stream, "favor_attn_decay_backward state gradient");
  // dV leaves the incoming state's gradient, where dK may still be reading the outgoing one's
  const bool apart = dstate_in && dstate_in == dstate_out && dv.nseg == 1;
  if (g->dk == g->dv && !apart)
    return run_scan({{dk, dv, dq}, 3}, dt, stream, "favor_attn_decay_backward gradients");
  FAVOR_TRY(run_scan({{dk, dq}, 2}, dt, stream, "favor_attn_decay_backward dK, dQ"));
  return run_scan({{dv}, 1}, dt, stream, "favor_attn_decay_backward dV");
}

favor_status favor_attn_decay_step(const favor_decay_desc *g, const void *Q, const void *K,
                                   const void *V, const float *log_decay, const int32_t *slots,
                                   int32_t n_slots, float *state, void *out,
                                   hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpStep));
  if (n_slots < 0) return fail(FAVOR_ERR_INVALID_ARGUMENT, "n_slots=%d is negative", n_slots);
  if (!slots && n_slots < g->B)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "%d sequences have only %d states", g->B, n_slots);
  const bool work = (long long)g->B * g->H > 0;
  const void *ptrs[] = {Q, K, V, out};
  const char *names[] = {"Q", "K", "V", "out"};
  for (int i = 0; i < 4; ++i) FAVOR_TRY(check_ptr(ptrs[i], names[i], work));
  FAVOR_TRY(check_ptr(state, "state", work && n_slots > 0));
  FAVOR_TRY(check_ptr(log_decay, "log_decay", work, 4));
  FAVOR_TRY(check_optional(slots, "slots", 4));
  if (work && (out == Q || out == K || out == V))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "out must not be an input");
  if (!work) return ok();
  favor_decay_desc one = *g;
  one.L = 1;
  favor::DecayStep a{};
  a.q = Q;
  a.k = K;
  a.v = V;
  a.o = out;
  a.qs = rows_of(&one, g->q, g->dk);
  a.ks = rows_of(&one, g->k, g->dk);
  a.vs = rows_of(&one, g->v, g->dv);
  a.os = rows_of(&one, g->out, g->dv);
  a.log_decay = log_decay;
  a.slots = slots;
  a.state = state;
  a.n_slots = n_slots;
  a.B = g->B;
  a.H = g->H;
  a.dk = g->dk;
  a.dv = g->dv;
  a.scale = g->scale;
  hipError_t e;
  {
    favor::LaunchTimer t(favor::kKerDecayStep, stream);
    e = favor::launch_decay_step(a, dt_of(g), stream);
  }
  return device_result(e, "favor_attn_decay_step");
}

favor_status favor_dropout(const void *x, const void *residual, void *y, int64_t n,
                           favor_dtype dtype, double p, uint64_t seed, uint64_t offset,
                           const uint64_t *rng, hipStream_t stream) {
  const int dt = raw_enum(&dtype);
  if (n < 0) return fail(FAVOR_ERR_INVALID_ARGUMENT, "n=%lld is negative", (long long)n);
  if (dt != FAVOR_F32 && dt != FAVOR_BF16)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "unknown dtype %d", dt);
  if (!(p >= 0.0 && p <= 1.0))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "p=%g is not between 0 and 1", p);
  if (n > ((int64_t)1 << 60)) return fail(FAVOR_ERR_UNSUPPORTED, "n exceeds 2^60");
  FAVOR_TRY(check_ptr(x, "x", n > 0));
  FAVOR_TRY(check_ptr(y, "y", n > 0));
  FAVOR_TRY(check_optional(residual, "residual"));
  FAVOR_TRY(check_optional(rng, "rng", 8));
  const int64_t bytes = n * (dt == FAVOR_BF16 ? 2 : 4);
  FAVOR_TRY(check_apart(y, "y", x, "x", bytes, true));
  FAVOR_TRY(check_apart(y, "y", residual, "residual", bytes, true));
  if (n == 0) return ok();
  favor::Dropout a{};
  a.x = x;
  a.residual = residual;
  a.y = y;
  a.n = n;
  a.threshold = (uint32_t)std::nearbyint(p * 65536.0);
  a.scale = a.threshold < 65536 ? (float)(65536.0 / (65536 - a.threshold)) : 0.f;
  a.seed = seed;
  a.offset = offset;
  a.rng = rng;
  hipError_t e;
  {
    favor::LaunchTimer t(favor::kKerDropout, stream);
    e = favor::launch_dropout(a, dt == FAVOR_BF16 ? favor::Dt::BF16 : favor::Dt::F32, stream);
  }
  return device_result(e, "favor_dropout");
}

}  // extern "C"
