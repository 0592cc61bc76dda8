// reorder_launches.cpp - the launches that favor_beam_reorder makes of many and of huge pools: each
// of less than 2^32 threads, and together every pool once, in order. Built with g++ like
// fuzz_recurrent.cpp; the other launchers of recurrent_api.cpp are never reached.
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../include/favor.h"
#include "../../paper_2006_03555_amd/csrc/recurrent.hpp"

static std::vector<favor::BeamReorder> seen;

namespace favor {
hipError_t launch_beam_reorder(const BeamReorder &a, hipStream_t) {
  seen.push_back(a);
  return hipSuccess;
}
}  // namespace favor

static int run(int n, int64_t bytes) {
  std::vector<favor_beam_pool> pools(n);
  for (int i = 0; i < n; ++i)
    pools[i] = {reinterpret_cast<void *>((uintptr_t)(i + 1) << 48), i % 7 == 3 ? 0 : bytes, 4};
  seen.clear();
  int32_t *const p = reinterpret_cast<int32_t *>((uintptr_t)1 << 40), *const q = p + 1024;
  if (favor_beam_reorder(2, 2, p, nullptr, q, pools.data(), n, nullptr) != FAVOR_OK) return 1;
  int at = 0;
  for (const favor::BeamReorder &a : seen) {
    if ((int64_t)a.first[a.n_pools] * 256 >= (int64_t)1 << 32) return 2;
    for (int i = 0; i < a.n_pools; ++i, ++at) {
      if (at >= n || a.pool[i].data != pools[at].data) return 3;
      const int64_t pieces = a.first[i + 1] - a.first[i];
      if (a.pool[i].units != pools[at].bytes_per_slot / 16) return 4;
      if (pieces != (a.pool[i].units + favor::kBeamPieceUnits - 1) / favor::kBeamPieceUnits) return 5;
    }
  }
  if (at != n || (n == 0 && seen.size() != 1)) return 6;
  std::printf("%d pools of %lld bytes: %d launches\n", n, (long long)bytes, (int)seen.size());
  return 0;
}

int main() {
  const struct { int n; int64_t bytes; } calls[] = {{0, 0}, {1, 16}, {64, 1 << 20}, {65, 1 << 20}, {131, 64},
                                                    {1, (int64_t)1 << 34}, {64, (int64_t)1 << 34},
                                                    {200, (int64_t)1 << 34}, {16, (int64_t)1 << 34}};
  for (const auto &c : calls)
    if (const int e = run(c.n, c.bytes)) {
      std::printf("%d pools of %lld bytes: failure %d (%s)\n", c.n, (long long)c.bytes, e, favor_last_error());
      return 1;
    }
  return 0;
}
