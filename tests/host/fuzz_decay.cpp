// fuzz_decay.cpp - seeded fuzzer of the host layer of the decayed linear attention and the
// dropout (decay_api.cpp), built like fuzz_desc.cpp under address and undefined-behaviour
// sanitizers; the launchers of these operators are stood in for here. For random
// descriptors, strides, pointers and workspace sizes it checks that
//   * nothing crashes or overflows (the sanitizers abort on any finding);
//   * a call that returns an error launched nothing, and left a message;
//   * every launch has consistent arguments: segments that cover the sequence once, states
//     inside the workspace, grids and 32-bit row offsets within their limits.
// Usage: fuzz_decay SEED ITERATIONS
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>

#include "../../include/favor.h"
#include "../../paper_2006_03555_amd/csrc/decay.hpp"

namespace {

uint64_t g_state;
uint64_t next() {   // splitmix64
  uint64_t z = (g_state += 0x9E3779B97F4A7C15ull);
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
template <typename T, size_t N>
T pick(const T (&a)[N]) { return a[next() % N]; }
bool coin(int pct) { return (int)(next() % 100) < pct; }

int launches = 0;
const char *ws_at = nullptr;   // the call's workspace
size_t ws_size = 0;

void require(bool ok, const char *what) {
  if (!ok) {
    std::fprintf(stderr, "inconsistent launch arguments: %s\n", what);
    std::abort();
  }
}

void pass_ok(const favor::DecayPass &p, favor::Dt dt, bool sums) {
  ++launches;
  require(p.n >= 1 && p.n <= 3, "one to three scans");
  const favor::DecayScan &f = p.scan[0];
  for (int i = 0; i < p.n; ++i) {
    const favor::DecayScan &a = p.scan[i];
    require(a.BH > 0 && a.H > 0 && a.BH % a.H == 0, "B*H a positive multiple of H");
    require(a.kd == f.kd && a.vd == f.vd && a.slice == f.slice && a.BH == f.BH &&
                a.seg_len == f.seg_len && a.nseg == f.nseg, "scans of one shape");
    require(a.kd > 0 && a.kd <= 256 && a.vd > 0 && a.vd <= 256, "columns");
    require(a.slice == 64 || (a.slice == 128 && a.kd <= 128), "slices");
    require(a.seg_len > 0 && a.seg_len % 64 == 0 && a.nseg > 0, "segments of whole chunks");
    require((long long)a.seg_len * a.nseg >= a.L && (long long)a.seg_len * (a.nseg - 1) <= a.L,
            "segments cover L once");
    require(a.nseg == 1 || (long long)a.seg_len * (a.nseg - 1) < a.L, "no empty segment");
    require(a.log_decay, "decays");
    const long long grid = (long long)p.n * a.BH * ((a.vd + a.slice - 1) / a.slice) * a.nseg;
    require(grid < INT_MAX / 512, "grid");
    if (sums) require(a.nseg > 1, "sums of segments");
    if (a.nseg > 1) {
      require((long long)p.n * a.BH <= 65535, "prefix grid");
      const char *at = reinterpret_cast<const char *>(a.part);
      require(at >= ws_at && at + sizeof(float) * a.BH * a.nseg * a.kd * a.vd <= ws_at + ws_size,
              "states inside the workspace");
    }
    const int elt = dt == favor::Dt::BF16 ? 2 : 4;
    const favor::Rows rows[] = {a.qs, a.ks, a.vs, a.os};
    for (const auto &r : rows)
      require(r.t >= 0 && 63 * r.t * elt + 256 * elt <= (1ll << 31), "32-bit offsets in a chunk");
  }
}

}  // namespace

namespace favor {
hipError_t launch_decay_sums(const DecayPass &p, Dt dt, hipStream_t) {
  pass_ok(p, dt, true);
  return hipSuccess;
}
hipError_t launch_decay_prefix(const DecayPass &p, hipStream_t) {
  pass_ok(p, Dt::BF16, true);   // (reads no rows)
  return hipSuccess;
}
hipError_t launch_decay_scan(const DecayPass &p, Dt dt, hipStream_t) {
  pass_ok(p, dt, false);
  return hipSuccess;
}
hipError_t launch_decay_step(const DecayStep &a, Dt, hipStream_t) {
  ++launches;
  require(a.B > 0 && a.H > 0 && (long long)a.B * a.H <= 65535, "step grid");
  require(a.dk > 0 && a.dk <= 256 && a.dv > 0 && a.dv <= 256 && a.dv % 4 == 0, "step columns");
  require(a.n_slots >= 0 && (a.slots || a.n_slots >= a.B), "places");
  return hipSuccess;
}
hipError_t launch_dropout(const Dropout &a, Dt, hipStream_t) {
  ++launches;
  require(a.n > 0 && a.threshold <= 65536, "dropout");
  require(a.threshold == 65536 ? a.scale == 0.f : a.scale >= 1.f && a.scale <= 65536.f, "scale");
  return hipSuccess;
}
}  // namespace favor

namespace {

int fails = 0;
void check(bool ok, const char *what, long iter) {
  if (!ok) {
    std::fprintf(stderr, "iteration %ld: %s (%s)\n", iter, what, favor_last_error());
    ++fails;
  }
}

favor_strides random_strides(const favor_decay_desc &g, int d) {
  favor_strides s{0, 0, 0};
  if (coin(50)) return s;
  const int64_t H = g.H, L = g.L;
  if (coin(70)) {   // a usual layout, perhaps wider than its rows
    const int64_t w = d + 8 * (int64_t)(next() % 3);
    if (coin(50)) s = {(int64_t)((uint64_t)H * (uint64_t)L * (uint64_t)w), (int64_t)((uint64_t)L * (uint64_t)w), w};
    else s = {(int64_t)((uint64_t)H * (uint64_t)L * (uint64_t)w), w, (int64_t)((uint64_t)H * (uint64_t)w)};
    if (coin(20)) s.batch = 0;
    if (coin(20)) s.head = 0;
    return s;
  }
  const int64_t odd[] = {0, 8, 4, -8, 64, 1 << 23, (1 << 24), 1ll << 40, INT64_MAX, INT64_MIN, 1};
  return {pick(odd), pick(odd), pick(odd)};
}

favor_decay_desc random_desc() {
  favor_decay_desc g;
  std::memset(&g, 0, sizeof g);
  if (coin(10)) {   // raw garbage in every field
    uint32_t w[sizeof(g) / 4];
    for (auto &x : w) x = (uint32_t)next();
    std::memcpy(&g, w, sizeof g);
    return g;
  }
  const int32_t Bs[] = {0, 1, 2, 3, 8, 100, 65535, -1, INT_MAX, INT_MIN};
  const int32_t Hs[] = {1, 2, 8, 16, 64, 0, 65535, -1, INT_MAX};
  const int32_t Ls[] = {0, 1, 63, 64, 65, 257, 1999, 8192, 65536, 1 << 24, 1 << 30,
                        (1 << 30) + 1, INT_MAX, -1, INT_MIN};
  const int32_t ds[] = {8, 64, 64, 72, 128, 128, 136, 256, 248, 0, -8, 4, 264, INT_MAX};
  const float fs[] = {1.f, 0.125f, 0.f, -1.f, std::numeric_limits<float>::infinity(),
                      std::numeric_limits<float>::quiet_NaN()};
  const int dts[] = {FAVOR_F32, FAVOR_BF16, FAVOR_BF16, 2, -1};
  g.B = coin(85) ? (int32_t)(1 + next() % 4) : pick(Bs);
  g.H = coin(70) ? (int32_t)(1 + next() % 16) : pick(Hs);
  g.L = coin(60) ? (int32_t)(next() % 5000) : pick(Ls);
  g.dk = coin(80) ? (int32_t)(8 * (1 + next() % 32)) : pick(ds);
  g.dv = coin(80) ? (int32_t)(8 * (1 + next() % 32)) : pick(ds);
  const int dt = coin(90) ? (int)(next() % 2 ? FAVOR_F32 : FAVOR_BF16) : pick(dts);
  std::memcpy(&g.dtype, &dt, sizeof dt);
  g.scale = coin(90) ? 0.125f : pick(fs);
  g.q = random_strides(g, g.dk);
  g.k = random_strides(g, g.dk);
  g.v = random_strides(g, g.dv);
  g.out = random_strides(g, g.dv);
  g.grad_out = random_strides(g, g.dv);
  g.grad_q = random_strides(g, g.dk);
  g.grad_k = random_strides(g, g.dk);
  g.grad_v = random_strides(g, g.dv);
  return g;
}

// An address that is never followed; each far from the others.
template <typename T>
T *address(int i, int null_pct) {
  if (coin(null_pct)) return nullptr;
  uintptr_t p = (uintptr_t)(i + 1) << 50;
  if (coin(2)) p += 8;
  return reinterpret_cast<T *>(p);
}

}  // namespace

int main(int argc, char **argv) {
  g_state = argc > 1 ? std::strtoull(argv[1], nullptr, 10) : 1;
  const long iters = argc > 2 ? std::atol(argv[2]) : 20000;
  long ran = 0;
  for (long it = 0; it < iters; ++it) {
    const favor_decay_desc g = random_desc();
    const int op = (int)(next() % 4);
    const bool valid = op < 3 && favor_validate_decay_desc(&g, op) == FAVOR_OK;
    const size_t need = op < 2 ? favor_decay_workspace_size(&g, op) : 0;
    check(need == 0 || valid, "a workspace for an invalid descriptor", it);
    check(need % 256 == 0, "workspace size", it);
    launches = 0;
    const bool enough = coin(90);
    ws_size = enough ? need : need - (need ? 256 : 0);
    char *ws = reinterpret_cast<char *>((uintptr_t)1 << 58);
    ws_at = ws;
    const int np = coin(80) ? 0 : 10;
    const void *q = address<void>(0, np), *k = address<void>(1, np), *v = address<void>(2, np);
    const float *ld = address<float>(3, np);
    const int32_t *len = address<int32_t>(4, 50);
    const float *s0 = address<float>(5, 50);
    float *s1 = coin(20) ? const_cast<float *>(s0) : address<float>(6, 50);
    void *o = address<void>(7, np);
    favor_status st;
    if (op == 0) {
      st = favor_attn_decay(&g, q, k, v, ld, len, o, s0, s1, ws, ws_size, nullptr);
    } else if (op == 1) {
      const float *d1 = address<float>(8, 50);
      float *d0 = coin(20) ? const_cast<float *>(d1) : coin(10) ? const_cast<float *>(s0)
                                                                : address<float>(9, 50);
      st = favor_attn_decay_backward(&g, q, k, v, ld, len, s0, o, d1, address<void>(10, np),
                                     address<void>(11, np), address<void>(12, np), d0, ws, ws_size,
                                     nullptr);
    } else if (op == 2) {
      const int32_t ns[] = {0, 1, 4, 100, -1, INT_MAX};
      st = favor_attn_decay_step(&g, q, k, v, ld, len, pick(ns), s1, o, nullptr);
    } else {
      const double ps[] = {0.0, 0.1, 0.5, 1.0, 1.0 - 1e-9, -0.1, 2.0,
                           std::numeric_limits<double>::quiet_NaN()};
      const int64_t ns[] = {0, 1, 7, 1000, 1ll << 40, (1ll << 60) + 1, -1, INT64_MAX, INT64_MIN};
      const favor_dtype dt = coin(50) ? FAVOR_F32 : FAVOR_BF16;   // by value: a valid one
      st = favor_dropout(q, coin(50) ? nullptr : k, coin(30) ? const_cast<void *>(q) : o,
                         pick(ns), dt, pick(ps), next(), next(), nullptr, nullptr);
    }
    if (st != FAVOR_OK) {
      check(launches == 0, "an error after a launch", it);
      check(favor_last_error()[0] != 0, "an error without a message", it);
      check(valid || op == 3 || st != FAVOR_ERR_WORKSPACE_TOO_SMALL, "order of checks", it);
    } else {
      check(valid || op == 3, "an invalid descriptor was taken", it);
      ran += launches > 0;
    }
  }
  std::printf("%ld calls, %ld with launches, %d failures\n", iters, ran, fails);
  return fails != 0 || ran < iters / 20;
}
