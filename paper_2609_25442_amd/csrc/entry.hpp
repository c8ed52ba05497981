// What the library's C entries share: the calling thread's error message, the
// guard that turns exceptions into codes, and the checks of device pointers.
#ifndef WB_ENTRY_HPP
#define WB_ENTRY_HPP

#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <new>
#include <string>

#include "wb_internal.hpp"

namespace wb {

extern thread_local std::string g_error;

inline int set_error(int code, const std::string& msg) {
  g_error = msg;
  return code;
}

template <class F>
int guarded(F&& f) {
  try {
    g_error.clear();
    return f();
  } catch (const wb::Error& e) {
    return set_error(e.code, e.what());
  } catch (const std::bad_alloc&) {
    return set_error(WB_ENOMEM, "host allocation failed");
  } catch (const std::exception& e) {
    return set_error(WB_EINVAL, e.what());
  }
}

inline int hip_fail(hipError_t e, const char* what) {
  return set_error(WB_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

// The device allocation of the pointer checked last in one call: the tensors
// of a rank mostly share a few allocations, and each query of the runtime
// takes about as long as a launch. Never kept past the call.
struct KnownRange {
  uintptr_t begin = 0, end = 0;
};

// Refuse a pointer the GPU cannot address (pageable host memory, or an
// address the runtime does not know) and one whose device allocation is
// smaller than what the kernels will touch. Pinned host memory is accepted;
// the runtime does not size it. what() names the pointer.
template <class What>
int check_extent_as(const void* p, int64_t bytes, What&& what, int align = 16, KnownRange* known = nullptr) {
  if (!p) return set_error(WB_EINVAL, what() + " is null");
  if (reinterpret_cast<uintptr_t>(p) % align != 0)
    return set_error(WB_EINVAL, what() + " is not " + std::to_string(align) + "-byte aligned");
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  auto fits = [&](uintptr_t end) -> int {
    if (at + uint64_t(bytes) > end)
      return set_error(WB_EINVAL, what() + " is smaller than the plan needs (" + std::to_string(bytes) + " bytes)");
    return WB_OK;
  };
  if (known && at >= known->begin && at < known->end) return fits(known->end);
  hipPointerAttribute_t attr;
  if (hipPointerGetAttributes(&attr, p) != hipSuccess) {
    (void)hipGetLastError();
    return set_error(WB_EINVAL, what() + " is not memory the GPU can address (device or pinned host)");
  }
  if (attr.type == hipMemoryTypeUnregistered)
    return set_error(WB_EINVAL, what() + " is pageable host memory: the kernels need device or pinned host memory");
  hipDeviceptr_t base = nullptr;
  size_t size = 0;
  if (hipMemGetAddressRange(&base, &size, const_cast<void*>(p)) != hipSuccess) {
    (void)hipGetLastError();
    return WB_OK;
  }
  const uintptr_t begin = reinterpret_cast<uintptr_t>(base);
  if (known && at >= begin) *known = KnownRange{begin, begin + size};
  return fits(begin + size);
}

inline int check_extent(const void* p, int64_t bytes, const char* what, int align = 16) {
  return check_extent_as(p, bytes, [&] { return std::string(what); }, align);
}

}  // namespace wb

#endif
