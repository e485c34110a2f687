// What the operators of an expert-parallel layer share (moe.hip, act.hip):
// their element types, and the host side of an entry point on device arrays.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <exception>
#include <string>

#include "device.h"
#include "netsim.h"

namespace netsim_ops {

using bf16 = __bf16;
using f16 = _Float16;

inline int64_t type_size(int32_t type) { return type == NETSIM_F32 ? 4 : 2; }
inline bool type_ok(int32_t type) { return type == NETSIM_F32 || type == NETSIM_BF16 || type == NETSIM_F16; }

inline netsim_status fail(netsim_status code, const char* what, const char* why) {
  netsim_host::set_thread_error((std::string(what) + ": " + why).c_str());
  return code;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return a > 0 ? (a - 1) / b + 1 : 0; }

// Whether p may be read as elements of `size` bytes.
inline bool aligned(const void* p, int64_t size) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)size == 0; }

// Makes `device` current for one call and puts the caller's back afterwards.
class OnDevice {
 public:
  explicit OnDevice(int32_t device) {
    err_ = hipGetDevice(&before_);
    if (err_ == hipSuccess && before_ != device) {
      err_ = hipSetDevice(device);
      moved_ = err_ == hipSuccess;
    }
  }
  ~OnDevice() {
    if (moved_) (void)hipSetDevice(before_);
  }
  hipError_t error() const { return err_; }

 private:
  int before_ = 0;
  bool moved_ = false;
  hipError_t err_ = hipSuccess;
};

// Runs an entry point's body; nothing it throws crosses the C boundary.
template <class F>
netsim_status entry(const char* what, int32_t device, F&& body) {
  try {
    if (device < 0 || device >= 64) return fail(NETSIM_E_INVALID, what, "bad device");
    return body();
  } catch (const std::exception&) {
    return NETSIM_E_NOMEM;
  }
}

// The launches of an entry point, on `device`: `go` enqueues them.
template <class F>
netsim_status launch(const char* what, int32_t device, F&& go) {
  OnDevice on(device);
  hipError_t e = on.error();
  if (e == hipSuccess) {
    go();
    e = hipGetLastError();
  }
  return e == hipSuccess ? NETSIM_OK : fail(NETSIM_E_DEVICE, what, hipGetErrorString(e));
}

// A grid of 2^32 threads or more is cut short by the runtime, without an error:
// work over `count` items goes in launches of at most `most`.
template <class F>
void in_launches(int64_t count, int64_t most, F&& go) {
  for (int64_t first = 0; first < count; first += most) go(first, count - first < most ? count - first : most);
}

// Calls f with a value of the element type `type` names.
template <class F>
void with_type(int32_t type, F&& f) {
  if (type == NETSIM_F32)
    f(float{});
  else if (type == NETSIM_BF16)
    f(bf16{});
  else
    f(f16{});
}

}  // namespace netsim_ops
