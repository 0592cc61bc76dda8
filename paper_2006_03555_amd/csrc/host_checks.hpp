// host_checks.hpp - argument checks that the C entry points share: plain host code that
// touches no device (internal to libfavor).
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "../../include/favor.h"
#include "kernels.hpp"

namespace favor {
namespace host {

inline favor_status fail(favor_status st, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return report(st, buf);
}
inline favor_status ok() { return report(FAVOR_OK, ""); }

#define FAVOR_TRY(expr)                \
  do {                                 \
    favor_status st__ = (expr);        \
    if (st__ != FAVOR_OK) return st__; \
  } while (0)

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The integer in an enum-typed field (a C caller may store any int there).
inline int raw_enum(const void *p) {
  int v;
  std::memcpy(&v, p, sizeof v);
  return v;
}

inline favor_status check_ptr(const void *p, const char *name, bool needed, size_t align = 16) {
  if (!needed) return FAVOR_OK;
  if (!p) return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s is NULL", name);
  if (!aligned(p, align))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s is not %zu-byte aligned", name, align);
  return FAVOR_OK;
}
inline favor_status check_optional(const void *p, const char *name, size_t align = 16) {
  return check_ptr(p, name, p != nullptr, align);
}

// An output that is written while an input of the same size is read: the two may be one
// where `same` says so (each element is then read first), and must not overlap otherwise.
inline favor_status check_apart(const void *out, const char *name, const void *in,
                                const char *other, int64_t bytes, bool same) {
  if (!out || !in || (out == in && same)) return FAVOR_OK;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out), b = reinterpret_cast<uintptr_t>(in);
  if ((a > b ? a - b : b - a) >= (uint64_t)bytes) return FAVOR_OK;
  return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s overlaps %s", name, other);
}

// The same of an output and an input of any sizes.
inline favor_status check_disjoint(const void *out, const char *name, int64_t out_bytes,
                                   const void *in, const char *other, int64_t in_bytes) {
  if (!out || !in) return FAVOR_OK;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out), b = reinterpret_cast<uintptr_t>(in);
  if (a >= b ? a - b >= (uint64_t)in_bytes : b - a >= (uint64_t)out_bytes) return FAVOR_OK;
  return fail(FAVOR_ERR_INVALID_ARGUMENT, "%s overlaps %s", name, other);
}

inline favor_status device_result(hipError_t e, const char *what) {
  if (e != hipSuccess) return fail(FAVOR_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

inline favor_status check_workspace(const void *ws, size_t bytes, size_t need) {
  if (need == 0) return FAVOR_OK;
  if (!ws) return fail(FAVOR_ERR_INVALID_ARGUMENT, "workspace is NULL");
  if (!aligned(ws, 256))
    return fail(FAVOR_ERR_INVALID_ARGUMENT, "workspace is not 256-byte aligned");
  if (bytes < need)
    return fail(FAVOR_ERR_WORKSPACE_TOO_SMALL, "workspace %zu bytes, need %zu", bytes, need);
  return FAVOR_OK;
}

constexpr int kMaxL = 1 << 30;
constexpr int64_t kMaxStride = (int64_t)1 << 46;   // element offsets stay within 64 bits

// Rows of d contiguous elements, by stride in three dimensions of the given sizes (those of
// size 1 or less have no stride; three zeros mean the contiguous layout). unit: what the
// strides must be multiples of; reach: the largest stride of the last dimension (0: any).
// Rows of an output must not share elements.
inline favor_status check_rows(const char *name, const favor_strides &s, const int64_t (&size)[3],
                               int d, int unit, int64_t reach_last, bool out) {
  const int64_t stride[3] = {s.batch, s.head, s.token};
  if (!stride[0] && !stride[1] && !stride[2]) return FAVOR_OK;
  int64_t reach = 0;
  for (int i = 0; i < 3; ++i) {
    if (size[i] <= 1) continue;
    if (stride[i] < 0)
      return fail(FAVOR_ERR_INVALID_ARGUMENT, "a stride of %s is negative", name);
    if (stride[i] % unit != 0)
      return fail(FAVOR_ERR_INVALID_ARGUMENT,
                  "strides of %s must be multiples of 16 bytes (%d elements)", name, unit);
    if (i == 2 && reach_last && stride[i] > reach_last)
      return fail(FAVOR_ERR_UNSUPPORTED, "the token stride of %s exceeds 2^25 bytes", name);
    if (stride[i] > kMaxStride / (size[i] - 1) || (reach += stride[i] * (size[i] - 1)) > kMaxStride)
      return fail(FAVOR_ERR_UNSUPPORTED, "%s reaches past 2^46 elements", name);
  }
  if (!out) return FAVOR_OK;
  // taken by stride, each dimension steps over everything inside it
  int at[3] = {0, 1, 2};
  std::sort(at, at + 3, [&](int i, int j) { return stride[i] < stride[j]; });
  int64_t inner = d;
  for (int i : at) {
    if (size[i] <= 1) continue;
    if (stride[i] < inner)
      return fail(FAVOR_ERR_INVALID_ARGUMENT, "rows of %s overlap", name);
    inner += stride[i] * (size[i] - 1);
  }
  return FAVOR_OK;
}

}  // namespace host
}  // namespace favor
