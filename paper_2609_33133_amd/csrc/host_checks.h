// What the C entry points' host sides share: errors, checks of arguments, the
// launch hook around a kernel (internal to libaugtree).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include <cstdio>
#include <exception>

#include "internal.h"

namespace augtree {

template <class... A>
inline int fail(int status, const char* fmt, A... a) {
  char buf[512];
  std::snprintf(buf, sizeof(buf), fmt, a...);
  return fail_status(status, buf);
}

inline int hip_ok(hipError_t e, const char* what) {
  return e == hipSuccess ? AUGTREE_OK : fail(AUGTREE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Calls the launch hook around one kernel launch.
struct Hook {
  const char* role;
  hipStream_t stream;
  Hook(const char* r, hipStream_t s) : role(r), stream(s) { launch_hook(role, 0, stream); }
  ~Hook() { launch_hook(role, 1, stream); }
};

// No C++ exception crosses the ABI (the tables are vectors).
template <class F>
inline int guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "host allocation failed: %s", e.what());
  }
}

inline int check_ptr(const void* p, const char* name, bool required, size_t align = 16) {
  if (!p) return required ? fail(AUGTREE_ERR_INVALID_ARGUMENT, "null pointer: %s", name) : AUGTREE_OK;
  if (reinterpret_cast<uintptr_t>(p) % align)
    return fail(AUGTREE_ERR_MISALIGNED, "pointer %s is not %d-byte aligned", name, (int)align);
  return AUGTREE_OK;
}

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline size_t align_up(size_t n) { return (n + 255) / 256 * 256; }

inline int check_ws(const void* ws, size_t have, size_t need) {
  if (!ws || have < need)
    return fail(AUGTREE_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? have : (size_t)0, need);
  return check_ptr(ws, "ws", true, 256);
}

struct Named {
  const void* p;
  const char* name;
};

inline int check_all(const Named* v, int n, bool required) {
  for (int i = 0; i < n; ++i)
    if (int st = check_ptr(v[i].p, v[i].name, required)) return st;
  return AUGTREE_OK;
}

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && na && nb && x < y + nb && y < x + na;
}

// A tensor of a call, for the check that outputs are apart from all else. An `in_place` output may be an `in_place`
// input itself.
struct Span {
  const void* p;
  size_t bytes;
  const char* name;
  bool in_place = false;
};

inline int check_apart(const Span* in, int n_in, const Span* out, int n_out) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (overlap(out[i].p, out[i].bytes, in[j].p, in[j].bytes) &&
          !(out[i].in_place && in[j].in_place && out[i].p == in[j].p))
        return fail(AUGTREE_ERR_INVALID_ARGUMENT, "%s overlaps %s", out[i].name, in[j].name);
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
        return fail(AUGTREE_ERR_INVALID_ARGUMENT, "%s overlaps %s", out[i].name, out[j].name);
  }
  return AUGTREE_OK;
}

}  // namespace augtree
