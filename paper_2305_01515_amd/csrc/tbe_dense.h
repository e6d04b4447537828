// Shared by the operators beside the embedding path (scan, bias, AdamW): element types, 16-byte pieces, host-side checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tbe.h"

namespace tbe {

// Error without a handle of the embedding path: the text is what tbe_last_error(NULL) returns (tbe_api.hip).
int report(int code, const char *text) noexcept;

// HIP keeps an error until it is read: the next call's look after its launch must not find it again.
inline int report_hip(hipError_t e) noexcept {
  (void)hipGetLastError();
  return report(e == hipErrorOutOfMemory ? TBE_ENOMEM : TBE_EHIP, hipGetErrorString(e));
}

// what every handle of these operators holds
struct DenseBase {
  int device = 0;
};

// TBE_OK if the handle is there and its GPU is current
inline int check_handle(const DenseBase *s) noexcept {
  if (!s) return report(TBE_EINVAL, "null handle");
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return report_hip(e);
  if (dev != s->device) return report(TBE_EORDER, "the current GPU is not the one the handle was created on");
  return TBE_OK;
}

inline int check_launch() noexcept {
  hipError_t e = hipGetLastError();
  return e == hipSuccess ? TBE_OK : report_hip(e);
}

// workgroups of so many threads that a launch takes at most: a grid has fewer than 2^32 work-items
constexpr int64_t most_groups(int threads) { return (int64_t)0xFFFFFFFF / threads; }

inline int elem_bytes(int dtype) { return dtype == TBE_FP32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == TBE_FP32 || dtype == TBE_FP16 || dtype == TBE_BF16; }

template <int DT> struct Elem;
template <> struct Elem<TBE_FP32> { using type = float; };
template <> struct Elem<TBE_FP16> { using type = _Float16; };
template <> struct Elem<TBE_BF16> { using type = __bf16; };

// V elements of type E, moved as one
template <class E, int V> struct alignas(sizeof(E) * V) Pack { E e[V]; };

}  // namespace tbe
