// What the C entry points share: the detail of the last failure, argument checks, workspace slabs.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstddef>
#include <cstdint>
#include <cstdio>

#include "../../include/shadowkv.h"

namespace skv {

inline thread_local char g_err[512] = "";

inline void set_err(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
}

inline int fail_inval(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return SHADOWKV_EINVAL;
}

inline int fail_hip(const char* what, hipError_t e) {
  set_err("%s: %s", what, hipGetErrorString(e));
  return SHADOWKV_EHIP;
}

constexpr size_t kAlign = 256;
inline size_t up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_workspace(void* ws, size_t have, size_t need) {
  if (!ws) { set_err("workspace is NULL"); return SHADOWKV_EWORKSPACE; }
  if (reinterpret_cast<uintptr_t>(ws) % kAlign) { set_err("workspace must be 256-byte aligned"); return SHADOWKV_EWORKSPACE; }
  if (have < need) { set_err("workspace too small: %zu bytes given, %zu needed", have, need); return SHADOWKV_EWORKSPACE; }
  return SHADOWKV_OK;
}

// memory that an argument covers (p may be NULL: none)
struct Bytes {
  const void* p;
  size_t n;
};
inline bool meet(const Bytes& a, const Bytes& b) {
  const char *x = static_cast<const char*>(a.p), *y = static_cast<const char*>(b.p);
  return x && y && a.n && b.n && x < y + b.n && y < x + a.n;
}

}  // namespace skv
