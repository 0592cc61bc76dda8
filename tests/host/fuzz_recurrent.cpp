// fuzz_recurrent.cpp - seeded fuzzer of the host layer of the short convolution, the selective
// scan and the beam search's step (recurrent_api.cpp), built like fuzz_desc.cpp under address
// and undefined-behaviour sanitizers; the launchers of these operators are stood in for here.
// For random descriptors, strides, pointers and workspace sizes it checks that
//   * nothing crashes or overflows (the sanitizers abort on any finding);
//   * a call that returns an error launched nothing, and left a message;
//   * every launch has consistent arguments: segments that cover the sequence once, parts
//     inside the workspace, grids within their limits.
// Usage: fuzz_recurrent SEED ITERATIONS
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../include/favor.h"
#include "../../paper_2006_03555_amd/csrc/recurrent.hpp"

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

void inside(const void *p, long long count, int size, const char *what) {
  const char *at = static_cast<const char *>(p);
  require(count >= 0 && at >= ws_at && at + count * size <= ws_at + ws_size, what);
}

void conv_ok(const favor::Conv &a) {
  ++launches;
  require(a.B > 0 && a.B <= 65535 && a.D > 0 && a.D % 8 == 0, "convolution sizes");
  require(a.width >= 2 && a.width <= 8 && a.run >= a.width - 1, "runs hold the taps");
  require(((long long)a.L / a.run + 1) * (a.D / 4) / 256 < INT_MAX, "grid");
}

long long wide_tiles(const favor::Scan &a, int tile) {
  return (long long)a.G * ((a.D / a.G + tile - 1) / tile);
}

void scan_ok(const favor::Scan &a) {
  ++launches;
  require(a.B > 0 && a.B <= 65535 && a.G > 0 && a.D % a.G == 0 && a.D / a.G % 8 == 0, "channels");
  require(a.N > 0 && a.N <= 256, "states");
}

void segments_ok(const favor::Scan &a, bool part) {
  const long long per = (long long)a.chunks * favor::kScanTokens;
  require(a.chunks > 0 && a.nseg > 0 && per * a.nseg >= a.L, "segments cover L");
  require(a.nseg == 1 || per * (a.nseg - 1) < a.L, "no empty segment");
  if (!part) return;
  inside(a.part, (long long)a.B * a.nseg * a.D * a.N, 4, "states inside the workspace");
  inside(a.steps, (long long)a.B * a.nseg * a.D, 4, "steps inside the workspace");
}

void backward_ok(const favor::Scan &a) {
  const long long BD = (long long)a.B * a.nseg * a.D, low = (long long)a.B * a.L * a.G * a.N;
  require(a.chunks == 1 && (a.subs == 1 || a.subs == 2 || a.subs == 4), "chunks and tiles");
  inside(a.part_r, BD * a.N, 4, "part_r");
  inside(a.part_a, BD * a.N, 4, "part_a");
  inside(a.part_d, BD, 4, "part_d");
  inside(a.part_s, BD, 4, "part_s");
  const long long parts = wide_tiles(a, a.subs * favor::kScanBackTile) / a.G;
  inside(a.part_b, parts * low, 4, "part_b");
  inside(a.part_c, parts * low, 4, "part_c");
  // all of them, one after the other
  const float *at[] = {a.part, a.part_r, a.part_a, a.steps, a.part_d, a.part_s, a.part_b, a.part_c};
  const long long n[] = {BD * a.N, BD * a.N, BD * a.N, BD, BD, BD, parts * low};
  for (int i = 0; i < 7; ++i) require(at[i] + n[i] <= at[i + 1], "parts lie apart");
  require(wide_tiles(a, favor::kScanBackTile) * a.nseg < INT_MAX, "grid");
}

}  // namespace

namespace favor {
hipError_t launch_conv(const Conv &a, Dt, hipStream_t) {
  conv_ok(a);
  return hipSuccess;
}
int64_t conv_part_rows(int B, int L, int, int, Dt) { return (int64_t)B * (L / 1024 + 1); }
hipError_t launch_conv_backward(const Conv &a, Dt dt, hipStream_t) {
  conv_ok(a);
  inside(a.part, (long long)conv_part_rows(a.B, a.L, a.D, a.width, dt) * (a.width + 1) * a.D, 4,
         "filters' gradients inside the workspace");
  return hipSuccess;
}
hipError_t launch_conv_sums(const Conv &a, int rows, hipStream_t) {
  ++launches;
  require(rows > 0 && a.dw, "rows to sum");
  return hipSuccess;
}
hipError_t launch_conv_step(const Conv &a, Dt, hipStream_t) {
  conv_ok(a);
  require(a.n_slots >= 0 && (a.slots || a.n_slots >= a.B), "places");
  return hipSuccess;
}
hipError_t launch_scan_sums(const Scan &a, Dt, hipStream_t) {
  scan_ok(a);
  require(a.nseg > 1, "sums of segments");
  segments_ok(a, true);
  return hipSuccess;
}
hipError_t launch_scan_backward_parts(const Scan &a, Dt, hipStream_t) {
  scan_ok(a);
  segments_ok(a, true);
  backward_ok(a);
  return hipSuccess;
}
hipError_t launch_scan_prefix(const Scan &a, bool backward, hipStream_t) {
  scan_ok(a);
  if (a.nseg) segments_ok(a, true);
  else require(backward && a.L == 0, "segments");
  return hipSuccess;
}
hipError_t launch_scan(const Scan &a, Dt, hipStream_t) {
  scan_ok(a);
  if (a.L) segments_ok(a, a.nseg > 1);
  require(wide_tiles(a, 32) * a.nseg < INT_MAX, "grid");
  return hipSuccess;
}
hipError_t launch_scan_backward(const Scan &a, Dt, hipStream_t) {
  scan_ok(a);
  backward_ok(a);
  return hipSuccess;
}
hipError_t launch_scan_backward_sums(const Scan &a, Dt, hipStream_t) {
  scan_ok(a);
  require(a.dA, "gradients");
  return hipSuccess;
}
hipError_t launch_scan_step(const Scan &a, Dt, hipStream_t) {
  scan_ok(a);
  require(a.n_slots >= 0 && (a.slots || a.n_slots >= a.B), "places");
  return hipSuccess;
}
hipError_t launch_beam_pieces(const BeamSelect &a, Dt, hipStream_t) {
  ++launches;
  require(a.B > 0 && a.K > 0 && a.K <= 64 && a.n > 0 && a.n <= 64 && a.V > 0, "beams");
  require(a.pieces > 0 && a.pieces <= 64 && a.piece_len % 512 == 0, "pieces");
  require((long long)a.pieces * a.piece_len >= a.V &&
              (long long)(a.pieces - 1) * a.piece_len < a.V, "pieces cover the row once");
  const long long rows = (long long)a.B * a.K * a.pieces;
  inside(a.stats, rows, 8, "statistics");
  inside(a.keys, rows * a.n, 8, "keys");
  require(reinterpret_cast<const char *>(a.stats + rows) <= reinterpret_cast<const char *>(a.keys),
          "apart");
  require(!a.ended || a.end_token >= 0, "the end's token");
  return hipSuccess;
}
hipError_t launch_beam_merge(const BeamSelect &, hipStream_t) {
  ++launches;
  return hipSuccess;
}
hipError_t launch_beam_reorder(const BeamReorder &a, hipStream_t) {
  ++launches;
  require(a.B > 0 && a.K > 0 && a.K <= 64 && (long long)a.B * a.K <= 65535, "beams");
  require(a.n_pools >= 0 && a.n_pools <= kBeamPools && a.first[0] == 0, "pools");
  for (int i = 0; i < a.n_pools; ++i) {
    const long long n = a.first[i + 1] - (long long)a.first[i], units = a.pool[i].units;
    require(n >= 0 && n * kBeamPieceUnits >= units && (n - 1) * kBeamPieceUnits < units,
            "pieces cover a state once");
  }
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

favor_strides random_strides(int64_t L, int64_t rows, int64_t d) {
  favor_strides s{0, 0, 0};
  if (coin(50)) return s;
  if (coin(70)) {   // a usual layout, perhaps wider than its rows
    const uint64_t w = (uint64_t)d + 8 * (next() % 3), t = w * (uint64_t)rows;
    s = {(int64_t)((uint64_t)L * t), (int64_t)w, (int64_t)t};
    if (coin(20)) s.batch = 0;
    if (coin(10)) s.token = 0;
    return s;
  }
  const int64_t odd[] = {0, 8, 4, -8, 64, 1 << 23, (1 << 24), 1ll << 40, INT64_MAX, INT64_MIN, 1};
  return {pick(odd), pick(odd), pick(odd)};
}

const int32_t kOddB[] = {0, 1, 2, 100, 65535, 65536, -1, INT_MAX, INT_MIN};
const int32_t kOddL[] = {0, 1, 127, 128, 129, 8192, 65536, 1 << 24, 1 << 30, (1 << 30) + 1,
                         INT_MAX, -1, INT_MIN};
const int32_t kOddD[] = {8, 64, 72, 65536, 65544, 4, 0, -8, INT_MAX};

template <typename T> bool garbage(T *g) {   // in every field
  std::memset(g, 0, sizeof *g);
  if (!coin(10)) return false;
  uint32_t w[sizeof(T) / 4];
  for (auto &x : w) x = (uint32_t)next();
  std::memcpy(g, w, sizeof *g);
  return true;
}

template <typename T> void type_of(T *g) {
  const int dts[] = {FAVOR_F32, FAVOR_BF16, 2, -1};
  const int dt = coin(90) ? (int)(next() % 2 ? FAVOR_F32 : FAVOR_BF16) : pick(dts);
  std::memcpy(&g->dtype, &dt, sizeof dt);
}

favor_conv_desc conv_desc() {
  favor_conv_desc g;
  if (garbage(&g)) return g;
  g.B = coin(85) ? (int32_t)(1 + next() % 6) : pick(kOddB);
  g.L = coin(60) ? (int32_t)(next() % 5000) : pick(kOddL);
  g.D = coin(80) ? (int32_t)(8 * (1 + next() % 600)) : pick(kOddD);
  g.width = coin(90) ? (int32_t)(2 + next() % 7) : (int32_t)next();
  g.silu = (int32_t)(next() % 2);
  type_of(&g);
  for (favor_strides *s : {&g.x, &g.y, &g.grad_y, &g.grad_x}) *s = random_strides(g.L, 1, g.D);
  return g;
}

favor_scan_desc scan_desc() {
  favor_scan_desc g;
  if (garbage(&g)) return g;
  g.B = coin(85) ? (int32_t)(1 + next() % 40) : pick(kOddB);
  g.L = coin(60) ? (int32_t)(next() % 5000) : pick(kOddL);
  g.D = coin(80) ? (int32_t)(8 * (1 + next() % 600)) : pick(kOddD);
  g.N = coin(85) ? (int32_t)(1 + next() % 256) : pick(kOddD);
  g.groups = coin(80) ? 1 : (int32_t)(next() % 5);
  g.softplus = (int32_t)(next() % 2);
  type_of(&g);
  for (favor_strides *s : {&g.x, &g.dt, &g.z, &g.y, &g.grad_y, &g.grad_x, &g.grad_dt, &g.grad_z})
    *s = random_strides(g.L, 1, g.D);
  for (favor_strides *s : {&g.b, &g.c, &g.grad_b, &g.grad_c})
    *s = random_strides(g.L, g.groups, g.N);
  return g;
}

favor_beam_desc beam_desc() {
  favor_beam_desc g;
  if (garbage(&g)) return g;
  const int32_t few[] = {1, 4, 64, 65, 0, -1, INT_MAX};
  g.B = coin(85) ? (int32_t)(1 + next() % 100) : pick(kOddB);
  g.K = coin(85) ? (int32_t)(1 + next() % 64) : pick(few);
  g.n = coin(85) ? (int32_t)(1 + next() % 64) : pick(few);
  g.V = coin(80) ? (int32_t)(1 + next() % 200000) : pick(kOddL);
  g.end_token = coin(50) ? -1 : (int32_t)(next() % 1000);
  type_of(&g);
  if (coin(50)) {
    const favor_strides s = random_strides(g.K, 1, g.V);
    g.batch_stride = s.batch;
    g.beam_stride = s.token;
  }
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
    const int kind = (int)(next() % 4), op = (int)(next() % 3);
    const favor_conv_desc c = conv_desc();
    const favor_scan_desc s = scan_desc();
    const favor_beam_desc b = beam_desc();
    bool valid = true;
    size_t need = 0;
    if (kind == 0) {
      valid = favor_validate_conv_desc(&c, op) == FAVOR_OK;
      need = op == 1 ? favor_conv_workspace_size(&c) : 0;
    } else if (kind == 1) {
      valid = favor_validate_scan_desc(&s, op) == FAVOR_OK;
      need = op < 2 ? favor_scan_workspace_size(&s, op) : 0;
    } else if (kind == 2) {
      valid = favor_validate_beam_desc(&b) == FAVOR_OK;
      need = favor_beam_workspace_size(&b);
    }
    check(need == 0 || valid, "a workspace for an invalid descriptor", it);
    check(need % 256 == 0, "workspace size", it);
    launches = 0;
    ws_size = coin(90) ? need : need - (need ? 256 : 0);
    char *ws = reinterpret_cast<char *>((uintptr_t)1 << 58);
    ws_at = ws;
    const int np = coin(80) ? 0 : 10;
    void *p[16];
    for (int i = 0; i < 16; ++i) p[i] = address<void>(i, np);
    if (coin(10)) p[next() % 16] = p[next() % 16];
    const auto f = [&](int i) { return static_cast<float *>(p[i]); };
    const auto maybe = [&](int i) { return coin(50) ? nullptr : f(i); };
    const int32_t *len = address<int32_t>(16, 50);
    const int32_t ns[] = {0, 1, 6, 100, -1, INT_MAX};
    favor_status st;
    if (kind == 0 && op == 0) {
      st = favor_conv(&c, p[0], f(1), maybe(2), len, p[3], maybe(4), maybe(5), nullptr);
    } else if (kind == 0 && op == 1) {
      st = favor_conv_backward(&c, p[0], f(1), maybe(2), len, maybe(3), p[4], maybe(5), p[6], f(7),
                               maybe(8), maybe(9), ws, ws_size, nullptr);
    } else if (kind == 0) {
      st = favor_conv_step(&c, p[0], f(1), maybe(2), len, pick(ns), p[3], p[4], nullptr);
    } else if (kind == 1 && op == 0) {
      st = favor_selective_scan(&s, p[0], p[1], f(2), p[3], p[4], maybe(5), maybe(6), maybe(7), len,
                                p[8], maybe(9), maybe(10), ws, ws_size, nullptr);
    } else if (kind == 1 && op == 1) {
      float *const z = maybe(6);
      st = favor_selective_scan_backward(&s, p[0], p[1], f(2), p[3], p[4], maybe(5), z, maybe(7),
                                         len, maybe(8), p[9], maybe(10), p[11], p[12], f(13), p[14],
                                         p[15], address<float>(17, np), address<float>(18, np),
                                         address<float>(19, np), address<float>(20, 50), ws,
                                         ws_size, nullptr);
    } else if (kind == 1) {
      st = favor_selective_scan_step(&s, p[0], p[1], f(2), p[3], p[4], maybe(5), maybe(6), maybe(7),
                                     len, pick(ns), f(8), p[9], nullptr);
    } else if (kind == 2) {
      st = favor_beam_select(&b, p[0], f(1), reinterpret_cast<uint8_t *>(maybe(2)), f(3),
                             reinterpret_cast<int32_t *>(p[4]), reinterpret_cast<int32_t *>(p[5]),
                             ws, ws_size, nullptr);
    } else {
      favor_beam_pool pools[70];
      const int n = coin(90) ? (int)(next() % 6) : (int)(next() % 70);
      for (int i = 0; i < n; ++i) {
        const int64_t sizes[] = {0, 16, 1 << 17, 1ll << 34, (1ll << 34) + 16, 24, -16, INT64_MAX};
        pools[i] = {address<void>(30 + i, coin(90) ? 0 : np),
                    coin(90) ? (int64_t)(16 * (next() % 100000)) : pick(sizes), pick(ns)};
      }
      valid = true;
      st = favor_beam_reorder(coin(90) ? (int32_t)(next() % 50) : pick(kOddB),
                              coin(90) ? (int32_t)(next() % 65) : pick(kOddD),
                              reinterpret_cast<int32_t *>(p[0]), len,
                              reinterpret_cast<int32_t *>(p[1]), pools, coin(98) ? n : -1, nullptr);
    }
    if (st != FAVOR_OK) {
      check(launches == 0, "an error after a launch", it);
      check(favor_last_error()[0] != 0, "an error without a message", it);
      check(valid || st != FAVOR_ERR_WORKSPACE_TOO_SMALL, "order of checks", it);
    } else {
      check(valid, "an invalid descriptor was taken", it);
      ran += launches > 0;
    }
  }
  std::printf("%ld calls, %ld with launches, %d failures\n", iters, ran, fails);
  return fails != 0 || ran < iters / 20;
}
