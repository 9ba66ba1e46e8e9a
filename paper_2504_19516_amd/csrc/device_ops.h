// What the operators on device data share: element types, the checks of a call's stream, launches.
#pragma once
#include <tuple>

#include "common.h"
#include "sts.h"

namespace sts {

typedef _Float16 f16;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

void record_hip_error(hipError_t e);          // what sts_last_hip_error() reports (engine.hip)

constexpr int OP_PAGE = 16;                    // tokens of a page
constexpr int OP_MAX_REQUESTS = 4096;          // requests of a batch: their lengths are scanned in one workgroup's LDS

// 16 bytes of T
template <typename T> struct Vec16;
template <> struct Vec16<float> { typedef f32x4 type; };
template <> struct Vec16<bf16> { typedef bf16x8 type; };
template <> struct Vec16<f16> { typedef f16x8 type; };
template <typename T> using vec16 = typename Vec16<T>::type;

// The device of a call is its stream's: it is made the current one for the launches, and the caller's comes back at the end.
class OnStreamDevice {
 public:
  explicit OnStreamDevice(hipStream_t s) {
    // the null stream and the runtime's other two reserved handles belong to the current device
    if (reinterpret_cast<uintptr_t>(s) <= 2) return;
    hipDevice_t dev = 0;
    if ((err_ = hipStreamGetDevice(s, &dev)) != hipSuccess || (err_ = hipGetDevice(&before_)) != hipSuccess) return;
    if (dev != before_ && (err_ = hipSetDevice(dev)) == hipSuccess) moved_ = true;
  }
  ~OnStreamDevice() { if (moved_) (void)hipSetDevice(before_); }
  OnStreamDevice(const OnStreamDevice&) = delete;
  OnStreamDevice& operator=(const OnStreamDevice&) = delete;
  hipError_t error() const { return err_; }

 private:
  hipError_t err_ = hipSuccess;
  int before_ = 0;
  bool moved_ = false;
};

// Launch that reports its own error and not one that an earlier call of the thread left behind.
template <typename... P, typename... A>
hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t s, const A&... args) {
  std::tuple<P...> values{args...};
  return std::apply([&](auto&... v) {
    void* ptrs[] = {static_cast<void*>(&v)...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, lds, s);
  }, values);
}

inline int op_result(hipError_t e) {
  if (e == hipSuccess) return STS_OK;
  record_hip_error(e);
  return STS_EHIP;
}

inline size_t dtype_bytes(int dtype) { return dtype == STS_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace sts
