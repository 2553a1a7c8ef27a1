// What the C entry points share: the error message, argument checks and the
// carving of caller-owned buffers.  Defined in moe_api.cpp.
#pragma once

#include <hip/hip_runtime.h>

#include <initializer_list>
#include <utility>

#include "moe.h"

namespace moe {

// Sets the thread's error message and returns `code`; clears it.
int fail(int code, const char* fmt, ...);
int ok();
int hip_status(hipError_t e, const char* where);

int check_dims(const moe_dims* d);
int check_experts_dims(const moe_experts_dims* d);
int check_ptrs(std::initializer_list<std::pair<const char*, const void*>> ps);

// Sequential carve-up of a buffer into 256-byte aligned regions.
struct Carve {
  char* base;
  size_t off = 0;
  explicit Carve(void* b) : base(static_cast<char*>(b)) {}
  template <typename T>
  T* take(size_t count) {
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += (count * sizeof(T) + 255) / 256 * 256;
    return p;
  }
};

}  // namespace moe
