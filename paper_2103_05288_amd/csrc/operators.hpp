// What the operators outside the fusion patterns (decoder.cpp, step.cpp) share on the host: refusals, sizes, entering an
// operator, enqueueing a kernel, the boundary of a C function.
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <stdexcept>

#include "disc_internal.hpp"

namespace disc {

constexpr int64_t kNonTemporalBytes = 64 << 20;   // from here on past the caches, as the fused patterns
constexpr int64_t kMostElements = (int64_t)1 << 60;
constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 1;     // of one launch, by axis; calls of more tokens are several launches

inline int refuse(disc_ctx* c, int code, const char* what) { return context_fail(c, code, what); }
inline int refuse(disc_ctx* c, int code, const char* what, long long got) {
  char buf[160];
  snprintf(buf, sizeof buf, "%s (got %lld)", what, got);
  return context_fail(c, code, buf);
}

// a * b of two sizes, or -1 where that is more than any memory holds
inline int64_t times(int64_t a, int64_t b) {
  if (a < 0 || b < 0) return -1;
  if (a == 0 || b == 0) return 0;
  return a > kMostElements / b ? -1 : a * b;
}

// rows [tokens][heads] of `d` elements: every stride is a size, and the extent fits
inline bool strides_ok(int64_t tokens, int64_t token, int64_t heads, int64_t head, int64_t d) {
  if (token < 0 || head < 0) return false;
  const int64_t a = times(tokens - 1, token), b = times(heads - 1, head);
  return a >= 0 && b >= 0 && a + b + d <= kMostElements;
}
// ... and no two of them overlap
inline bool rows_apart(int64_t tokens, int64_t token, int64_t heads, int64_t head, int64_t d) {
  if (tokens <= 1) return heads <= 1 || head >= d;
  if (heads <= 1) return token >= d;
  return (head >= d && token >= (heads - 1) * head + d) || (token >= d && head >= (tokens - 1) * token + d);
}
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

inline Operator* get_operator(disc_ctx* c, int32_t id, Operator::Kind kind) {
  auto& all = *context_operators(c);
  if (id < 0 || id >= (int)all.size() || all[id]->kind != kind) return nullptr;
  return all[id].get();
}

// The context's device is the current one while kernels are enqueued (the default stream is the current device's).
struct OnDevice {
  int before = -1;
  bool ok = true;
  explicit OnDevice(int device) {
    int now = -1;
    ok = hipGetDevice(&now) == hipSuccess;
    if (ok && now != device) {
      ok = hipSetDevice(device) == hipSuccess;
      before = now;
    }
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

inline int enqueue(disc_ctx* c, void* fn, uint64_t blocks, uint32_t y, uint32_t threads, const void* args, size_t size, void* stream) {
  void* extra[] = {HIP_LAUNCH_PARAM_BUFFER_POINTER, const_cast<void*>(args), HIP_LAUNCH_PARAM_BUFFER_SIZE, &size, HIP_LAUNCH_PARAM_END};
  const hipError_t e = hipModuleLaunchKernel((hipFunction_t)fn, (uint32_t)blocks, y, 1, threads, 1, 1, 0, (hipStream_t)stream, nullptr, extra);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    char buf[128];
    snprintf(buf, sizeof buf, "hipModuleLaunchKernel: %s", hipGetErrorString(e));
    return context_fail(c, DISC_ERR_HIP, buf);
  }
  return DISC_OK;
}
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Compiles the operator and enters it, or finds the one that was made of the same description.  `measured`: the kernel
// whose blocks a CU are asked for.
inline int enter(disc_ctx* c, std::unique_ptr<Operator> o, const std::string& macros, const char* header, const char* const* names, int n, int measured, int32_t* id_out) {
  auto& all = *context_operators(c);
  for (size_t i = 0; i < all.size(); ++i)
    if (all[i]->key == o->key) {
      *id_out = (int32_t)i;
      return DISC_OK;
    }
  o->code = macros;
  for (const auto& other : all)   // (compiled for another registration already, whose numbers are arguments of the kernels)
    if (other->code == macros) {
      o->module = other->module;
      std::copy(std::begin(other->fn), std::end(other->fn), o->fn);
      o->resident = other->resident;
      *id_out = (int32_t)all.size();
      all.push_back(std::move(o));
      return DISC_OK;
    }
  std::vector<char> code;
  const int rc = context_compile(c, macros + header, &code);
  if (rc) return rc;
  all.reserve(all.size() + 1);
  const int device = context_device(c);
  if (device >= 0) {
    OnDevice on(device);
    if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
    hipModule_t m = nullptr;
    if (hipModuleLoadData(&m, code.data()) != hipSuccess) {
      (void)hipGetLastError();
      return refuse(c, DISC_ERR_HIP, "hipModuleLoadData failed");
    }
    o->module = m;
    o->owns_module = true;
    for (int i = 0; i < n; ++i) {
      hipFunction_t f = nullptr;
      if (hipModuleGetFunction(&f, m, names[i]) != hipSuccess) {
        (void)hipGetLastError();
        (void)hipModuleUnload(m);
        return refuse(c, DISC_ERR_HIP, "hipModuleGetFunction failed");
      }
      o->fn[i] = f;
    }
    int blocks = 0;
    if (hipModuleOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, (hipFunction_t)o->fn[measured], 256, 0) == hipSuccess && blocks > 0)
      o->resident = blocks;
    else
      (void)hipGetLastError();
  }
  *id_out = (int32_t)all.size();
  all.push_back(std::move(o));
  return DISC_OK;
}

inline std::string text(const char* format, double x) {
  char buf[64];
  snprintf(buf, sizeof buf, format, x);
  return buf;
}

inline int fail_inside(disc_ctx* c, const char* what) noexcept {
  char buf[160];
  snprintf(buf, sizeof buf, "internal error: %s", what);
  if (c) context_fail(c, DISC_ERR_INTERNAL, buf);
  return DISC_ERR_INTERNAL;
}

// Nothing leaves a C function by exception.
template <class F>
inline int guarded(disc_ctx* c, F f) noexcept {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail_inside(c, "out of host memory");
  } catch (const std::exception& e) {
    return fail_inside(c, e.what());
  } catch (...) {
    return fail_inside(c, "unknown exception");
  }
}

}  // namespace disc
