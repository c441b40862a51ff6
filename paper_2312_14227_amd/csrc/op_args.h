// What the stand-alone operators of the C ABI check and set up in front of their launches.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "et.h"

namespace et_op {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t type_size(int32_t dtype) { return dtype == ET_BF16 ? 2 : 4; }
inline bool type_ok(int32_t dtype) { return dtype == ET_F32 || dtype == ET_BF16; }

// The launches of a call go to the device of its stream, whichever device is current (kernels and device limits are looked up for the current one)
struct OnDeviceOf {
  int before = -1;
  bool ok = true, switched = false;
  int dev = -1;
  explicit OnDeviceOf(hipStream_t s) {
    ok = hipGetDevice(&before) == hipSuccess;
    dev = before;
    if (!ok || !s) return;
    hipDevice_t d;
    if (hipStreamGetDevice(s, &d) != hipSuccess) { ok = false; return; }
    dev = (int)d;
    if (dev != before) ok = switched = hipSetDevice(dev) == hipSuccess;
  }
  ~OnDeviceOf() {
    if (switched) (void)hipSetDevice(before);
  }
};

inline int device_cus(int dev) {
  int n = 0;
  return hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0 ? n : 256;
}

// A matrix of `rows` rows: bytes from the first to behind the last, of a row, from a row to the next
struct Span {
  uintptr_t begin, end, width, step;
  Span(const void* p, int64_t rows, int64_t cols, int64_t stride, size_t size)
      : begin(reinterpret_cast<uintptr_t>(p)), end(begin + (size_t)((rows - 1) * stride + cols) * size), width((size_t)cols * size), step((size_t)stride * size) {}
  // Whether two have a byte in common, if they are as many bytes from row to row apart: rows may lie beside each other's.  Otherwise whether what they reach over does
  bool meets(const Span& o) const {
    if (begin >= o.end || o.begin >= end) return false;
    if (step != o.step || step == 0) return true;
    const uintptr_t at = o.begin >= begin ? (o.begin - begin) % step : (step - (begin - o.begin) % step) % step;   // where o's rows begin, counted from the beginning of these
    return at < width || at + o.width > step;
  }
};

// The losses, without and with their launches (row_loss.hip); launches: how many (nullable)
int policy_loss(int32_t rows, int32_t classes, const void* logits, int32_t dtype, int64_t stride, const int32_t* label, const et_policy* p, void* grad, int32_t grad_dtype,
                int64_t grad_stride, void* ws, size_t ws_bytes, hipStream_t s, float* loss, bool check_only, int* launches);
int preference_loss(int32_t rows, int32_t pairs, int32_t classes, const void* logits, int32_t dtype, int64_t stride, const int32_t* label, const et_preference* p, void* grad,
                    int32_t grad_dtype, int64_t grad_stride, void* ws, size_t ws_bytes, hipStream_t s, float* loss, bool check_only, int* launches);

}  // namespace et_op
