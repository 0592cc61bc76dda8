// recurrent_api.cpp - the C ABI of the short convolution, the selective scan and the beam
// search's step: argument validation, workspace sizing, launch planning and dispatch. As in
// favor_api.cpp, validation is plain host code that touches no device.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/favor.h"
#include "host_checks.hpp"
#include "recurrent.hpp"

namespace {

using favor::Dt;
using favor::Rows;
using namespace favor::host;

enum Op { kOpForward = 0, kOpBackward = 1, kOpStep = 2 };
constexpr int kMaxD = 65536, kMaxB = 65535;
constexpr int64_t kMaxBlocks = 0x7fffffff;
constexpr int64_t kMaxRows = (int64_t)1 << 38;   // elements of one sequence
// the scan reaches a chunk's 128 rows by 32-bit offsets
constexpr int64_t kMaxTokenBytes = 1 << 25;

Dt dt_of(const favor_dtype &d) { return raw_enum(&d) == FAVOR_BF16 ? Dt::BF16 : Dt::F32; }
int bytes_of(const favor_dtype &d) { return dt_of(d) == Dt::BF16 ? 2 : 4; }

favor_status check_op(int op) {
  if (op < kOpForward || op > kOpStep)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "unknown operation %d", op);
  return FAVOR_OK;
}
favor_status check_dtype(const favor_dtype &d) {
  const int dt = raw_enum(&d);
  if (dt != FAVOR_F32 && dt != FAVOR_BF16)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "unknown dtype %d", dt);
  return FAVOR_OK;
}
// row: of the longest rows that a call has
favor_status check_sizes(int B, int L, int D, int64_t row) {
  if (B < 0 || L < 0) return fail(FAVOR_ERR_INVALID_ARGUMENT, "negative size B=%d L=%d", B, L);
  if (D <= 0) return fail(FAVOR_ERR_INVALID_ARGUMENT, "D=%d must be positive", D);
  if (L > kMaxL) return fail(FAVOR_ERR_UNSUPPORTED, "L=%d exceeds 2^30", L);
  if (B > kMaxB) return fail(FAVOR_ERR_UNSUPPORTED, "B=%d exceeds 65535", B);
  if (D > kMaxD) return fail(FAVOR_ERR_UNSUPPORTED, "D=%d exceeds 65536", D);
  if (B && L && row > kMaxStride / B / L)
    return fail(FAVOR_ERR_UNSUPPORTED, "B=%d L=%d rows of %lld reach past 2^46 elements", B, L,
                (long long)row);
  return FAVOR_OK;
}

struct Tensor {
  const char *name;
  const favor_strides *s;
  bool out, low;   // low: [B][L][groups][N]
};

Rows rows_of(const favor_strides &s, int B, int L, int G, int d) {
  if (!s.batch && !s.head && !s.token) return {(int64_t)L * G * d, d, (int64_t)G * d};
  return {B > 1 ? s.batch : 0, G > 1 ? s.head : 0, L > 1 ? s.token : 0};
}

// Pointers that a call needs where it has work, and outputs that must not be inputs.
favor_status check_all(const void *const *ptrs, const char *const *names, int n, int first_out,
                       bool work) {
  for (int i = 0; i < n; ++i) FAVOR_TRY(check_ptr(ptrs[i], names[i], work));
  if (work)
    for (int o = first_out; o < n; ++o)
      for (int i = 0; i < o; ++i)
        if (ptrs[o] == ptrs[i])
          return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s must not be %s", names[o], names[i]);
  return FAVOR_OK;
}

favor_status check_slots(const int32_t *slots, int n_slots, int B, const void *state, bool work) {
  if (n_slots < 0) return fail(FAVOR_ERR_INVALID_ARGUMENT, "n_slots=%d is negative", n_slots);
  if (!slots && n_slots < B)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "%d sequences have only %d states", B, n_slots);
  FAVOR_TRY(check_ptr(state, "state", work && n_slots > 0));
  return check_optional(slots, "slots", 4);
}

// ------------------------------------------------------------------ convolution
// Tokens of one thread: the W - 1 inputs before its run are read again, so long runs read
// less, and short ones fill the card: 2048 threads on each of the 256 compute units.
int conv_run(const favor_conv_desc *g) {
  const int64_t threads = (int64_t)g->B * (g->D * bytes_of(g->dtype) / 16) * g->L;
  for (int run = 32; run > 8; run /= 2)
    if (threads / run >= 256 * 2048) return run;
  return 8;
}

int64_t part_rows(const favor_conv_desc *g) {
  return favor::conv_part_rows(g->B, g->L, g->D, g->width, dt_of(g->dtype));
}

favor_status validate(const favor_conv_desc *g, int op) {
  if (!g) return fail(FAVOR_ERR_INVALID_ARGUMENT, "descriptor is NULL");
  FAVOR_TRY(check_op(op));
  FAVOR_TRY(check_dtype(g->dtype));
  FAVOR_TRY(check_sizes(g->B, g->L, g->D, g->D));
  if (g->width <= 0) return fail(FAVOR_ERR_INVALID_ARGUMENT, "width=%d must be positive", g->width);
  if (g->width < 2 || g->width > 8)
    return fail(FAVOR_ERR_UNSUPPORTED, "width=%d not supported (2 to 8)", g->width);
  if (g->D % 8) return fail(FAVOR_ERR_UNSUPPORTED, "D=%d is not a multiple of 8", g->D);
  const Tensor ts[] = {{"x", &g->x, false, false}, {"y", &g->y, true, false},
                       {"dy", &g->grad_y, false, false}, {"dx", &g->grad_x, true, false}};
  for (int i = 0; i < 4; ++i) {
    if (i == 1 ? op == kOpBackward : i > 1 && op != kOpBackward) continue;
    const int64_t size[3] = {g->B, 1, op == kOpStep ? 1 : g->L};
    FAVOR_TRY(check_rows(ts[i].name, *ts[i].s, size, g->D, 16 / bytes_of(g->dtype), 0, ts[i].out));
  }
  // what one launch takes: a thread has 8 tokens of 4 channels at least, 32 of them in a long call
  if (op != kOpStep && (int64_t)g->L * g->D > kMaxRows)
    return fail(FAVOR_ERR_UNSUPPORTED, "L=%d D=%d: a sequence of more than 2^38 elements", g->L, g->D);
  if (op == kOpBackward && part_rows(g) > kMaxBlocks)
    return fail(FAVOR_ERR_UNSUPPORTED, "B=%d L=%d D=%d is too large", g->B, g->L, g->D);
  return FAVOR_OK;
}

size_t workspace_of(const favor_conv_desc *g) {
  if (g->B == 0) return 0;
  return round_up((size_t)part_rows(g) * (g->width + 1) * g->D * sizeof(float), 256);
}

favor::Conv conv_of(const favor_conv_desc *g, int L, const void *x, const float *weight,
                    const float *bias, const int32_t *lengths) {
  favor::Conv a{};
  a.x = x;
  a.w = weight;
  a.bias = bias;
  a.lengths = lengths;
  a.xs = rows_of(g->x, g->B, L, 1, g->D);
  a.B = g->B;
  a.L = L;
  a.D = g->D;
  a.width = g->width;
  a.silu = g->silu != 0;
  a.run = conv_run(g);
  return a;
}

int64_t state_bytes(const favor_conv_desc *g) {
  return (int64_t)g->B * (g->width - 1) * g->D * bytes_of(g->dtype);
}

// ------------------------------------------------------------------ selective scan
int tiles_of(const favor_scan_desc *g, int tile) {
  return g->groups * ((g->D / g->groups + tile - 1) / tile);
}
int chunks_of(const favor_scan_desc *g) { return (g->L + favor::kScanTokens - 1) / favor::kScanTokens; }

favor_status validate(const favor_scan_desc *g, int op) {
  if (!g) return fail(FAVOR_ERR_INVALID_ARGUMENT, "descriptor is NULL");
  FAVOR_TRY(check_op(op));
  FAVOR_TRY(check_dtype(g->dtype));
  const int64_t low = (int64_t)g->groups * g->N;
  FAVOR_TRY(check_sizes(g->B, g->L, g->D, std::max<int64_t>(g->D, low)));
  if (g->N <= 0 || g->groups <= 0)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "N=%d and groups=%d must be positive", g->N, g->groups);
  if (g->D % g->groups)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "D=%d is not a multiple of groups=%d", g->D, g->groups);
  if (g->N > 256) return fail(FAVOR_ERR_UNSUPPORTED, "N=%d exceeds 256", g->N);
  if (g->D / g->groups % 8)
    return fail(FAVOR_ERR_UNSUPPORTED, "D / groups=%d is not a multiple of 8", g->D / g->groups);
  const Tensor ts[] = {{"x", &g->x, false, false},        {"dt", &g->dt, false, false},
                       {"B", &g->b, false, true},         {"C", &g->c, false, true},
                       {"z", &g->z, false, false},        {"y", &g->y, true, false},
                       {"dy", &g->grad_y, false, false},  {"dx", &g->grad_x, true, false},
                       {"ddt", &g->grad_dt, true, false}, {"dB", &g->grad_b, true, true},
                       {"dC", &g->grad_c, true, true},    {"dz", &g->grad_z, true, false}};
  for (int i = 0; i < 12; ++i) {
    if (i == 5 ? op == kOpBackward : i > 5 && op != kOpBackward) continue;
    const int64_t size[3] = {g->B, ts[i].low ? g->groups : 1, op == kOpStep ? 1 : g->L};
    FAVOR_TRY(check_rows(ts[i].name, *ts[i].s, size, ts[i].low ? g->N : g->D,
                         ts[i].low ? 1 : 16 / bytes_of(g->dtype), kMaxTokenBytes / bytes_of(g->dtype),
                         ts[i].out));
  }
  // counts that the kernels hold in 32 bits
  if (op != kOpStep && (int64_t)g->L * g->D > kMaxRows)
    return fail(FAVOR_ERR_UNSUPPORTED, "L=%d D=%d: a sequence of more than 2^38 elements", g->L, g->D);
  if (op != kOpStep && (int64_t)g->B * chunks_of(g) > kMaxBlocks)
    return fail(FAVOR_ERR_UNSUPPORTED, "B=%d L=%d is too large", g->B, g->L);
  return FAVOR_OK;
}

// How a forward call is cut into segments of whole chunks. A call of several segments takes the
// sums of all but the last first, so their steps and decays are computed twice. Whole calls in
// us, bf16, N = 16:
//   One segment while its workgroups of 32 channels fill the 256 compute units, as long as
//   there are 240 of them: B4 L4096 D2048 (256) 230, in two segments 285, in eight 274 (fp32 267,
//   314, 300); B8 374, 493, 534.
//   Fewer: segments for 4096 workgroups. For 1024 / 2048 / 4096 / 8192 of them B1 L65536 D2048 1181
//   / 1127 / 1110 / 1107, B2 L4096 156 / 150 / 145 / 145, B1 L8192 D2048 N64 fp32 540 / 540 / 546 /
//   546. B1 L4096 83 in 32 segments and 219 in one, B3 L4096 (192) 216 in 16 and 221 in one (fp32
//   229 and 263), but B6 L1999 D1000 N24 fp32 (192) 192 in 16 and 184 in one.
//   One segment too where three passes over a chunk (16 states each) or fewer are all of it: two
//   more launches cost as much. B1 L256 D512 16.4 in one, 22.0 in two; B2 L384 D2048 23.4, in three
//   28.0; B1 L384 D512 22.8, in three 22.3; B1 L512 D512 29.5, in four 22.4; N64 fp32 L256 D2048
//   50.1, in two 40.7.
struct ScanCut {
  int chunks, nseg;
};
constexpr int kOneSegment = 240, kSegmentBlocks = 4096, kFewPasses = 3;
ScanCut cut_of(const favor_scan_desc *g) {
  ScanCut c;
  const int chunks = std::max(chunks_of(g), 1);
  const int64_t blocks = std::max<int64_t>(1, (int64_t)g->B * tiles_of(g, 32));
  const int passes = chunks * ((g->N + favor::kScanStates - 1) / favor::kScanStates);
  const int64_t want = blocks >= kOneSegment || passes <= kFewPasses ? 1 : kSegmentBlocks / blocks;
  c.chunks = (int)((chunks + want - 1) / want);
  c.nseg = (chunks + c.chunks - 1) / c.chunks;
  return c;
}

// States that one workgroup of the chunks' sums takes in the backward pass: a pass' 16 while that
// leaves few workgroups, else all of them, which read the rows once. Whole calls in us, by 16 / all:
// B2 L777 D512 N64 fp32 (224 workgroups of all) 121 / 130, B1 L300 D512 N48 (48) 78 / 91; B6 L1999
// D1000 N24 fp32 (3000 or so) 489 / 474. Forward, where only half as much comes with the rows, 16 are
// never slower: B1 L4096 D2048 N64 262 / 286, B6 L1999 D1000 N24 fp32 190 / 194.
constexpr int kSumBlocks = 1024;
int sum_states_of(const favor_scan_desc *g) {
  return (int64_t)g->B * tiles_of(g, favor::kScanBackTile) * chunks_of(g) < kSumBlocks ? favor::kScanStates : g->N;
}

// Tiles that one workgroup of the backward pass takes one after the other: their sums of dB and dC
// stay in LDS, and the workspace is as many times smaller. Whole calls in us with 1 / 2 / 4 tiles,
// bf16: B4 L4096 D2048 N16 831 / 830 / 783, B2 L4096 D4096 N8 646 / 608 / 584; with too few
// workgroups B1 L1024 D2048 82 / 89 / 124.
int subs_of(const favor_scan_desc *g) {
  if (g->N > 16) return 1;   // dB and dC of more states do not stay in LDS
  const int64_t rows = (int64_t)g->B * chunks_of(g);
  for (int subs = 4; subs > 1; subs /= 2)
    if (rows * tiles_of(g, subs * favor::kScanBackTile) >= 1024) return subs;
  return 1;
}

// Parts of a workspace, each 256-byte aligned.
struct Carver {
  char *base;
  size_t used = 0;
  float *floats(size_t n) {
    float *p = base ? reinterpret_cast<float *>(base + used) : nullptr;
    used += round_up(n * sizeof(float), 256);
    return p;
  }
};

size_t carve_forward(const favor_scan_desc *g, const ScanCut &c, void *ws, favor::Scan *a) {
  if (c.nseg <= 1) return 0;
  Carver w{static_cast<char *>(ws)};
  const size_t BD = (size_t)g->B * c.nseg * g->D;
  a->part = w.floats(BD * g->N);
  a->steps = w.floats(BD);
  return w.used;
}

size_t carve_backward(const favor_scan_desc *g, void *ws, favor::Scan *a) {
  Carver w{static_cast<char *>(ws)};
  const size_t BD = (size_t)g->B * chunks_of(g) * g->D;
  const size_t low = (size_t)(tiles_of(g, subs_of(g) * favor::kScanBackTile) / g->groups) * g->B *
                     g->L * g->groups * g->N;
  a->part = w.floats(BD * g->N);
  a->part_r = w.floats(BD * g->N);
  a->part_a = w.floats(BD * g->N);
  a->steps = w.floats(BD);
  a->part_d = w.floats(BD);
  a->part_s = w.floats(BD);
  a->part_b = w.floats(low);
  a->part_c = w.floats(low);
  return w.used;
}

size_t workspace_of(const favor_scan_desc *g, int op) {
  if (g->B == 0 || g->L == 0) return 0;
  favor::Scan a{};
  return op == kOpBackward ? carve_backward(g, nullptr, &a) : carve_forward(g, cut_of(g), nullptr, &a);
}

favor::Scan scan_of(const favor_scan_desc *g, int L, const void *x, const void *dt, const float *A,
                    const void *Bm, const void *C, const float *skip, const void *z,
                    const float *dt_bias, const int32_t *lengths) {
  favor::Scan a{};
  a.x = x;
  a.dt = dt;
  a.A = A;
  a.b = Bm;
  a.c = C;
  a.skip = skip;
  a.z = z;
  a.bias = dt_bias;
  a.lengths = lengths;
  a.B = g->B;
  a.L = L;
  a.D = g->D;
  a.N = g->N;
  a.G = g->groups;
  a.softplus = g->softplus != 0;
  a.xs = rows_of(g->x, g->B, L, 1, g->D);
  a.dts = rows_of(g->dt, g->B, L, 1, g->D);
  a.zs = rows_of(g->z, g->B, L, 1, g->D);
  a.ys = rows_of(g->y, g->B, L, 1, g->D);
  a.bs = rows_of(g->b, g->B, L, g->groups, g->N);
  a.cs = rows_of(g->c, g->B, L, g->groups, g->N);
  return a;
}

favor_status check_params(const float *A, const float *skip, const float *dt_bias, int N, bool any) {
  FAVOR_TRY(check_ptr(A, "A", any, N % 4 ? 4 : 16));
  FAVOR_TRY(check_optional(skip, "skip", 4));
  return check_optional(dt_bias, "dt_bias", 4);
}

int64_t state_bytes(const favor_scan_desc *g) {
  return (int64_t)sizeof(float) * g->B * g->D * g->N;
}

// ------------------------------------------------------------------ beams
favor_status validate(const favor_beam_desc *g) {
  if (!g) return fail(FAVOR_ERR_INVALID_ARGUMENT, "descriptor is NULL");
  FAVOR_TRY(check_dtype(g->dtype));
  if (g->B < 0) return fail(FAVOR_ERR_INVALID_ARGUMENT, "negative size B=%d", g->B);
  if (g->K <= 0 || g->V <= 0 || g->n <= 0)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "K=%d V=%d n=%d must be positive", g->K, g->V, g->n);
  if (g->end_token >= g->V)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "end_token=%d is not below V=%d", g->end_token, g->V);
  if (g->batch_stride < 0 || g->beam_stride < 0)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "a stride of logits is negative");
  if (g->K > 64 || g->n > 64)
    return fail(FAVOR_ERR_UNSUPPORTED, "K=%d n=%d not supported (at most 64)", g->K, g->n);
  if (g->V > kMaxL) return fail(FAVOR_ERR_UNSUPPORTED, "V=%d exceeds 2^30", g->V);
  if ((int64_t)g->B * g->K > 65535)
    return fail(FAVOR_ERR_UNSUPPORTED, "B*K=%lld exceeds 65535", (long long)g->B * g->K);
  if (g->batch_stride > kMaxStride / std::max(1, g->B) || g->beam_stride > kMaxStride / g->K)
    return fail(FAVOR_ERR_UNSUPPORTED, "logits reaches past 2^46 elements");
  return FAVOR_OK;
}

// No byte of one is the other's; their sizes may pass 64 bits together.
bool apart(const favor_beam_pool &a, const favor_beam_pool &b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.data), y = reinterpret_cast<uintptr_t>(b.data);
  const favor_beam_pool &lower = x < y ? a : b;
  if (x == y || !lower.bytes_per_slot) return x != y;
  return (x < y ? y - x : x - y) / (uint64_t)lower.bytes_per_slot >= (uint64_t)lower.n_slots;
}

// Pieces of a row, one wave each: 16 waves for each of the 256 compute units, of 512 tokens at
// least, and no more than one per lane of the wave that joins them.
void cut_row(const favor_beam_desc *g, int *pieces, int *len) {
  const int64_t rows = std::max<int64_t>(1, (int64_t)g->B * g->K);
  const int64_t want = std::min<int64_t>(64, std::max<int64_t>(1, (4096 + rows - 1) / rows));
  const int64_t each = (((int64_t)g->V + want - 1) / want + 511) / 512 * 512;
  *len = (int)each;
  *pieces = (int)((g->V + each - 1) / each);
}

size_t workspace_of(const favor_beam_desc *g, size_t *keys_at) {
  int pieces, len;
  cut_row(g, &pieces, &len);
  const size_t rows = (size_t)g->B * g->K * pieces;
  *keys_at = round_up(rows * sizeof(float2), 256);
  return rows ? *keys_at + round_up(rows * g->n * sizeof(uint64_t), 256) : 0;
}

}  // namespace

extern "C" {

favor_status favor_validate_conv_desc(const favor_conv_desc *g, int op) {
  FAVOR_TRY(validate(g, op));
  return ok();
}
favor_status favor_validate_scan_desc(const favor_scan_desc *g, int op) {
  FAVOR_TRY(validate(g, op));
  return ok();
}

favor_status favor_validate_beam_desc(const favor_beam_desc *g) {
  FAVOR_TRY(validate(g));
  return ok();
}

size_t favor_conv_workspace_size(const favor_conv_desc *g) {
  return validate(g, kOpBackward) == FAVOR_OK ? workspace_of(g) : 0;
}
size_t favor_scan_workspace_size(const favor_scan_desc *g, int backward) {
  const int op = backward ? kOpBackward : kOpForward;
  return validate(g, op) == FAVOR_OK ? workspace_of(g, op) : 0;
}
size_t favor_beam_workspace_size(const favor_beam_desc *g) {
  size_t keys;
  return validate(g) == FAVOR_OK ? workspace_of(g, &keys) : 0;
}

favor_status favor_conv(const favor_conv_desc *g, const void *x, const float *weight,
                        const float *bias, const int32_t *lengths, void *y, const void *state_in,
                        void *state_out, hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpForward));
  const bool any = g->B > 0, work = any && g->L > 0;
  const void *ptrs[] = {x, y};
  const char *names[] = {"x", "y"};
  FAVOR_TRY(check_all(ptrs, names, 2, 1, work));
  FAVOR_TRY(check_ptr(weight, "weight", any, 4));
  FAVOR_TRY(check_optional(bias, "bias", 4));
  FAVOR_TRY(check_optional(lengths, "lengths", 4));
  FAVOR_TRY(check_optional(state_in, "state_in"));
  FAVOR_TRY(check_optional(state_out, "state_out"));
  FAVOR_TRY(check_apart(state_out, "state_out", state_in, "state_in", state_bytes(g), true));
  if (!any || (!work && !state_out)) return ok();
  favor::Conv a = conv_of(g, g->L, x, weight, bias, lengths);
  a.y = y;
  a.ys = rows_of(g->y, g->B, g->L, 1, g->D);
  a.state_in = state_in;
  a.state_out = state_out;
  hipError_t e;
  {
    favor::LaunchTimer t(favor::kKerConv, stream);
    e = favor::launch_conv(a, dt_of(g->dtype), stream);
  }
  return device_result(e, "favor_conv");
}

favor_status favor_conv_backward(const favor_conv_desc *g, const void *x, const float *weight,
                                 const float *bias, const int32_t *lengths, const void *state_in,
                                 const void *dy, const void *dstate_out, void *dx, float *dweight,
                                 float *dbias, void *dstate_in, void *ws, size_t ws_bytes,
                                 hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpBackward));
  const bool any = g->B > 0, work = any && g->L > 0;
  const void *ptrs[] = {x, dy, dx};
  const char *names[] = {"x", "dy", "dx"};
  FAVOR_TRY(check_all(ptrs, names, 3, 2, work));
  FAVOR_TRY(check_ptr(weight, "weight", any, 4));
  FAVOR_TRY(check_ptr(dweight, "dweight", any || dweight, 4));
  FAVOR_TRY(check_optional(bias, "bias", 4));
  FAVOR_TRY(check_optional(dbias, "dbias", 4));
  FAVOR_TRY(check_optional(lengths, "lengths", 4));
  FAVOR_TRY(check_optional(state_in, "state_in"));
  FAVOR_TRY(check_optional(dstate_out, "dstate_out"));
  FAVOR_TRY(check_optional(dstate_in, "dstate_in"));
  FAVOR_TRY(check_apart(dstate_in, "dstate_in", state_in, "state_in", state_bytes(g), false));
  FAVOR_TRY(check_apart(dstate_in, "dstate_in", dstate_out, "dstate_out", state_bytes(g), false));
  const int64_t params = (int64_t)sizeof(float) * g->D * g->width;
  FAVOR_TRY(check_apart(dweight, "dweight", weight, "weight", params, false));
  if (!any && !dweight) return ok();
  FAVOR_TRY(check_workspace(ws, ws_bytes, workspace_of(g)));
  favor::Conv a = conv_of(g, g->L, x, weight, bias, lengths);
  a.state_in = state_in;
  a.dy = dy;
  a.dys = rows_of(g->grad_y, g->B, g->L, 1, g->D);
  a.dstate_out = dstate_out;
  a.dx = dx;
  a.dxs = rows_of(g->grad_x, g->B, g->L, 1, g->D);
  a.dstate_in = dstate_in;
  a.dw = dweight;
  a.dbias = dbias;
  a.part = any ? static_cast<float *>(ws) : nullptr;   // of no sequence: zeros
  const Dt dt = dt_of(g->dtype);
  hipError_t e = hipSuccess;
  if (any) {
    favor::LaunchTimer t(favor::kKerConvBwd, stream);
    e = favor::launch_conv_backward(a, dt, stream);
  }
  if (e != hipSuccess) return device_result(e, "favor_conv_backward");
  favor::LaunchTimer t(favor::kKerColumnSums, stream);
  return device_result(favor::launch_conv_sums(a, any ? (int)part_rows(g) : 1, stream),
                       "favor_conv_backward sums");
}

favor_status favor_conv_step(const favor_conv_desc *g, const void *x, const float *weight,
                             const float *bias, const int32_t *slots, int32_t n_slots, void *state,
                             void *y, hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpStep));
  const bool work = g->B > 0;
  const void *ptrs[] = {x, y};
  const char *names[] = {"x", "y"};
  FAVOR_TRY(check_all(ptrs, names, 2, 1, work));
  FAVOR_TRY(check_ptr(weight, "weight", work, 4));
  FAVOR_TRY(check_optional(bias, "bias", 4));
  FAVOR_TRY(check_slots(slots, n_slots, g->B, state, work));
  if (!work) return ok();
  favor::Conv a = conv_of(g, 1, x, weight, bias, nullptr);
  a.y = y;
  a.ys = rows_of(g->y, g->B, 1, 1, g->D);
  a.state_out = state;
  a.slots = slots;
  a.n_slots = n_slots;
  hipError_t e;
  {
    favor::LaunchTimer t(favor::kKerConvStep, stream);
    e = favor::launch_conv_step(a, dt_of(g->dtype), stream);
  }
  return device_result(e, "favor_conv_step");
}

favor_status favor_selective_scan(const favor_scan_desc *g, const void *x, const void *dt,
                                  const float *A, const void *Bm, const void *C, const float *skip,
                                  const void *z, const float *dt_bias, const int32_t *lengths,
                                  void *y, const float *state_in, float *state_out, void *ws,
                                  size_t ws_bytes, hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpForward));
  const bool any = g->B > 0, work = any && g->L > 0;
  const void *ptrs[] = {x, dt, y};
  const char *names[] = {"x", "dt", "y"};
  FAVOR_TRY(check_all(ptrs, names, 3, 2, work));
  const int elt = bytes_of(g->dtype);
  FAVOR_TRY(check_ptr(Bm, "B", work, elt));
  FAVOR_TRY(check_ptr(C, "C", work, elt));
  FAVOR_TRY(check_optional(z, "z"));
  if (work && (y == Bm || y == C || y == z))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "y must not be an input");
  FAVOR_TRY(check_params(A, skip, dt_bias, g->N, any));
  FAVOR_TRY(check_optional(lengths, "lengths", 4));
  FAVOR_TRY(check_optional(state_in, "state_in"));
  FAVOR_TRY(check_optional(state_out, "state_out"));
  FAVOR_TRY(check_apart(state_out, "state_out", state_in, "state_in", state_bytes(g), true));
  if (!any || (!work && !state_out)) return ok();
  FAVOR_TRY(check_workspace(ws, ws_bytes, workspace_of(g, kOpForward)));
  const ScanCut c = cut_of(g);
  favor::Scan a = scan_of(g, g->L, x, dt, A, Bm, C, skip, z, dt_bias, lengths);
  carve_forward(g, c, ws, &a);
  a.y = y;
  a.h_in = state_in;
  a.h_out = state_out;
  a.chunks = c.chunks;
  a.nseg = c.nseg;
  a.sum_states = favor::kScanStates;
  const Dt type = dt_of(g->dtype);
  if (c.nseg > 1) {
    hipError_t e;
    {
      favor::LaunchTimer t(favor::kKerScanSums, stream);
      e = favor::launch_scan_sums(a, type, stream);
    }
    if (e != hipSuccess) return device_result(e, "favor_selective_scan segment sums");
    favor::LaunchTimer t(favor::kKerScanPrefix, stream);
    e = favor::launch_scan_prefix(a, false, stream);
    if (e != hipSuccess) return device_result(e, "favor_selective_scan segment states");
  }
  favor::LaunchTimer t(favor::kKerScan, stream);
  return device_result(favor::launch_scan(a, type, stream), "favor_selective_scan");
}

favor_status favor_selective_scan_backward(
    const favor_scan_desc *g, const void *x, const void *dt, const float *A, const void *Bm,
    const void *C, const float *skip, const void *z, const float *dt_bias, const int32_t *lengths,
    const float *state_in, const void *dy, const float *dstate_out, void *dx, void *ddt, float *dA,
    void *dB, void *dC, float *dskip, void *dz, float *ddt_bias, float *dstate_in, void *ws,
    size_t ws_bytes, hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpBackward));
  const bool any = g->B > 0, work = any && g->L > 0;
  const void *ptrs[] = {x, dt, dy, dx, ddt};
  const char *names[] = {"x", "dt", "dy", "dx", "ddt"};
  FAVOR_TRY(check_all(ptrs, names, 5, 3, work));
  const int elt = bytes_of(g->dtype);
  const void *low[] = {Bm, C, dB, dC};
  const char *low_names[] = {"B", "C", "dB", "dC"};
  for (int i = 0; i < 4; ++i) FAVOR_TRY(check_ptr(low[i], low_names[i], work, elt));
  FAVOR_TRY(check_optional(z, "z"));
  FAVOR_TRY(check_ptr(dz, "dz", work && z));
  if (work) {
    const void *ins[] = {x, dt, dy, Bm, C, z}, *outs[] = {dx, ddt, dB, dC, z ? dz : nullptr};
    const char *out_names[] = {"dx", "ddt", "dB", "dC", "dz"};
    for (int o = 0; o < 5; ++o) {
      if (!outs[o]) continue;
      for (const void *i : ins)
        if (outs[o] == i)
          return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s must not be an input", out_names[o]);
      for (int i = 0; i < o; ++i)
        if (outs[o] == outs[i])
          return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s must not be %s", out_names[o], out_names[i]);
    }
  }
  FAVOR_TRY(check_params(A, skip, dt_bias, g->N, any));
  FAVOR_TRY(check_ptr(dA, "dA", any || dA, 4));
  FAVOR_TRY(check_ptr(dskip, "dskip", skip && (any || dskip), 4));
  FAVOR_TRY(check_ptr(ddt_bias, "ddt_bias", dt_bias && (any || ddt_bias), 4));
  FAVOR_TRY(check_optional(lengths, "lengths", 4));
  FAVOR_TRY(check_optional(state_in, "state_in"));
  FAVOR_TRY(check_optional(dstate_out, "dstate_out"));
  FAVOR_TRY(check_optional(dstate_in, "dstate_in"));
  FAVOR_TRY(check_apart(dstate_in, "dstate_in", dstate_out, "dstate_out", state_bytes(g), true));
  FAVOR_TRY(check_apart(dstate_in, "dstate_in", state_in, "state_in", state_bytes(g), false));
  FAVOR_TRY(check_apart(dA, "dA", A, "A", (int64_t)sizeof(float) * g->D * g->N, false));
  if (!any && !dA) return ok();
  FAVOR_TRY(check_workspace(ws, ws_bytes, workspace_of(g, kOpBackward)));
  favor::Scan a = scan_of(g, g->L, x, dt, A, Bm, C, skip, z, dt_bias, lengths);
  if (work) carve_backward(g, ws, &a);
  a.h_in = state_in;
  a.chunks = 1;
  a.nseg = any ? chunks_of(g) : 0;
  if (!any) a.B = 1, a.L = 0;   // no sequence: as one without tokens, the parameters' gradients are zeros
  a.sum_states = sum_states_of(g);
  a.subs = subs_of(g);
  a.dy = dy;
  a.dh_out = dstate_out;
  a.dh_in = dstate_in;
  a.dx = dx;
  a.ddt = ddt;
  a.dA = dA;
  a.db = dB;
  a.dc = dC;
  a.dskip = skip ? dskip : nullptr;
  a.dz = dz;
  a.dbias = dt_bias ? ddt_bias : nullptr;
  a.dys = rows_of(g->grad_y, g->B, g->L, 1, g->D);
  a.dxs = rows_of(g->grad_x, g->B, g->L, 1, g->D);
  a.ddts = rows_of(g->grad_dt, g->B, g->L, 1, g->D);
  a.dzs = rows_of(g->grad_z, g->B, g->L, 1, g->D);
  a.dbs = rows_of(g->grad_b, g->B, g->L, g->groups, g->N);
  a.dcs = rows_of(g->grad_c, g->B, g->L, g->groups, g->N);
  const Dt type = dt_of(g->dtype);
  hipError_t e = hipSuccess;
  if (work) {
    favor::LaunchTimer t(favor::kKerScanSums, stream);
    e = favor::launch_scan_backward_parts(a, type, stream);
  }
  if (e != hipSuccess) return device_result(e, "favor_selective_scan_backward chunk sums");
  if (any && (work || dstate_in)) {
    favor::LaunchTimer t(favor::kKerScanPrefix, stream);
    e = favor::launch_scan_prefix(a, true, stream);
  }
  if (e != hipSuccess) return device_result(e, "favor_selective_scan_backward chunk states");
  if (work) {
    favor::LaunchTimer t(favor::kKerScanBwd, stream);
    e = favor::launch_scan_backward(a, type, stream);
  }
  if (e != hipSuccess) return device_result(e, "favor_selective_scan_backward gradients");
  favor::LaunchTimer t(favor::kKerColumnSums, stream);
  return device_result(favor::launch_scan_backward_sums(a, type, stream),
                       "favor_selective_scan_backward sums");
}

favor_status favor_selective_scan_step(const favor_scan_desc *g, const void *x, const void *dt,
                                       const float *A, const void *Bm, const void *C,
                                       const float *skip, const void *z, const float *dt_bias,
                                       const int32_t *slots, int32_t n_slots, float *state, void *y,
                                       hipStream_t stream) {
  FAVOR_TRY(validate(g, kOpStep));
  const bool work = g->B > 0;
  const void *ptrs[] = {x, dt, y};
  const char *names[] = {"x", "dt", "y"};
  FAVOR_TRY(check_all(ptrs, names, 3, 2, work));
  const int elt = bytes_of(g->dtype);
  FAVOR_TRY(check_ptr(Bm, "B", work, elt));
  FAVOR_TRY(check_ptr(C, "C", work, elt));
  FAVOR_TRY(check_optional(z, "z"));
  if (work && (y == Bm || y == C || y == z))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "y must not be an input");
  FAVOR_TRY(check_params(A, skip, dt_bias, g->N, work));
  FAVOR_TRY(check_slots(slots, n_slots, g->B, state, work));
  if (!work) return ok();
  favor::Scan a = scan_of(g, 1, x, dt, A, Bm, C, skip, z, dt_bias, nullptr);
  a.y = y;
  a.h_out = state;
  a.slots = slots;
  a.n_slots = n_slots;
  hipError_t e;
  {
    favor::LaunchTimer t(favor::kKerScanStep, stream);
    e = favor::launch_scan_step(a, dt_of(g->dtype), stream);
  }
  return device_result(e, "favor_selective_scan_step");
}

favor_status favor_beam_select(const favor_beam_desc *g, const void *logits, const float *scores,
                               const uint8_t *ended, float *out_scores, int32_t *parent,
                               int32_t *token, void *ws, size_t ws_bytes, hipStream_t stream) {
  FAVOR_TRY(validate(g));
  const bool work = g->B > 0;
  if (ended && g->end_token < 0)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "ended without an end_token");
  FAVOR_TRY(check_ptr(logits, "logits", work, bytes_of(g->dtype)));
  FAVOR_TRY(check_ptr(scores, "scores", work, 4));
  FAVOR_TRY(check_ptr(out_scores, "out_scores", work, 4));
  FAVOR_TRY(check_ptr(parent, "parent", work, 4));
  FAVOR_TRY(check_ptr(token, "token", work, 4));
  // entries are written while others' scores and ended are read
  const int64_t outs = (int64_t)4 * g->B * g->n, ins = (int64_t)g->B * g->K;
  const void *out[] = {out_scores, parent, token};
  const char *names[] = {"out_scores", "parent", "token"};
  for (int i = 0; i < 3; ++i) {
    FAVOR_TRY(check_disjoint(out[i], names[i], outs, scores, "scores", 4 * ins));
    FAVOR_TRY(check_disjoint(out[i], names[i], outs, ended, "ended", ins));
    for (int j = 0; j < i; ++j)
      FAVOR_TRY(check_disjoint(out[i], names[i], outs, out[j], names[j], outs));
  }
  if (!work) return ok();
  size_t keys_at;
  FAVOR_TRY(check_workspace(ws, ws_bytes, workspace_of(g, &keys_at)));
  favor::BeamSelect a{};
  a.logits = logits;
  const bool whole = !g->batch_stride && !g->beam_stride;
  a.ls = {whole ? (int64_t)g->K * g->V : g->batch_stride, whole ? g->V : g->beam_stride, 0};
  a.scores = scores;
  a.ended = ended;
  a.B = g->B;
  a.K = g->K;
  a.V = g->V;
  a.n = g->n;
  a.end_token = g->end_token;
  cut_row(g, &a.pieces, &a.piece_len);
  a.stats = static_cast<float2 *>(ws);
  a.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(ws) + keys_at);
  a.out_scores = out_scores;
  a.parent = parent;
  a.token = token;
  hipError_t e;
  {
    favor::LaunchTimer t(favor::kKerBeamPieces, stream);
    e = favor::launch_beam_pieces(a, dt_of(g->dtype), stream);
  }
  if (e != hipSuccess) return device_result(e, "favor_beam_select pieces");
  favor::LaunchTimer t(favor::kKerBeamMerge, stream);
  return device_result(favor::launch_beam_merge(a, stream), "favor_beam_select");
}

favor_status favor_beam_reorder(int32_t B, int32_t K, const int32_t *parent, const int32_t *slots,
                                int32_t *new_slots, const favor_beam_pool *pools, int32_t n_pools,
                                hipStream_t stream) {
  if (B < 0 || K < 0 || n_pools < 0)
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "negative size B=%d K=%d n_pools=%d", B, K, n_pools);
  if (K > 64) return fail(FAVOR_ERR_UNSUPPORTED, "K=%d not supported (at most 64)", K);
  if ((int64_t)B * K > 65535)
    return fail(FAVOR_ERR_UNSUPPORTED, "B*K=%lld exceeds 65535", (long long)B * K);
  const bool work = (int64_t)B * K > 0;
  FAVOR_TRY(check_ptr(parent, "parent", work, 4));
  FAVOR_TRY(check_ptr(new_slots, "new_slots", work, 4));
  FAVOR_TRY(check_optional(slots, "slots", 4));
  const int64_t bytes = (int64_t)4 * B * K;
  FAVOR_TRY(check_apart(new_slots, "new_slots", slots, "slots", bytes, false));
  FAVOR_TRY(check_apart(new_slots, "new_slots", parent, "parent", bytes, false));
  if (n_pools > 0 && !pools) return fail(FAVOR_ERR_INVALID_ARGUMENT, "pools is NULL");
  for (int i = 0; i < n_pools; ++i) {
    const favor_beam_pool &p = pools[i];
    if (p.n_slots < 0 || p.bytes_per_slot < 0)
      return fail(FAVOR_ERR_INVALID_ARGUMENT, "pool %d has a negative size", i);
    if (p.bytes_per_slot % 16 || p.bytes_per_slot > (int64_t)1 << 34)
      return fail(FAVOR_ERR_UNSUPPORTED,
                  "pool %d: %lld bytes per slot (multiples of 16, at most 2^34)", i,
                  (long long)p.bytes_per_slot);
    FAVOR_TRY(check_ptr(p.data, "a pool", work && p.n_slots > 0 && p.bytes_per_slot > 0));
    for (int j = 0; j < i; ++j)
      if (p.data && pools[j].data && !apart(p, pools[j]))
        return fail(FAVOR_ERR_INVALID_ARGUMENT, "pools %d and %d are one or overlap", j, i);
  }
  if (!work) return ok();
  for (int first = 0; first == 0 || first < n_pools;) {
    favor::BeamReorder a{};
    a.parent = parent;
    a.slots = slots;
    a.new_slots = new_slots;
    a.B = B;
    a.K = K;
    while (a.n_pools < favor::kBeamPools && first + a.n_pools < n_pools) {
      const favor_beam_pool &p = pools[first + a.n_pools];
      const int64_t units = p.bytes_per_slot / 16;
      const int pieces = (int)((units + favor::kBeamPieceUnits - 1) / favor::kBeamPieceUnits);
      const int i = a.n_pools;
      if (i && a.first[i] + pieces > favor::kBeamPieces) break;   // the next launch's
      a.pool[i] = {p.data, (int32_t)units, p.n_slots};
      a.first[i + 1] = a.first[i] + pieces;
      a.n_pools = i + 1;
    }
    first += std::max(1, a.n_pools);
    hipError_t e;
    {
      favor::LaunchTimer t(favor::kKerBeamReorder, stream);
      e = favor::launch_beam_reorder(a, stream);
    }
    if (e != hipSuccess) return device_result(e, "favor_beam_reorder");
  }
  return ok();
}

}  // extern "C"
