// Element types and host helpers shared by the training-step operators (mist_embed.hip, mist_step.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "mist.h"

namespace mist {

__attribute__((visibility("hidden"))) mist_status lib_fail(mist_status code, const char* msg) noexcept;  // sets the thread's error

inline mist_status hip_failed(hipError_t e, const char* what) noexcept {
  char text[256];
  snprintf(text, sizeof text, "%s: %s", what, hipGetErrorString(e));
  return lib_fail(MIST_E_DEVICE, text);
}

// Storage types.  Conversions to 16 bits round to nearest even and keep NaN.
template <int TYPE>
struct Elem;
template <>
struct Elem<MIST_F32> {
  using type = float;
};
template <>
struct Elem<MIST_BF16> {
  using type = __bf16;
};
template <>
struct Elem<MIST_F16> {
  using type = _Float16;
};

// N consecutive values, read and written by instructions of up to 16 bytes.  They need only their element's
// alignment (the device's global memory instructions take any), so that shards take the same path.  Rows of the
// embedding have to be whole vectors too.
template <class T, int N>
struct Vec {
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

inline int64_t type_bytes(int32_t type) { return type == MIST_F32 ? 4 : 2; }
inline bool type_ok(int32_t type) { return type == MIST_F32 || type == MIST_BF16 || type == MIST_F16; }

// f(Elem<A>{}, Elem<B>{}) for the pair of types (a, b).
template <class F>
void with_type(int32_t a, F&& f) {
  if (a == MIST_F32) f(Elem<MIST_F32>{});
  else if (a == MIST_BF16) f(Elem<MIST_BF16>{});
  else f(Elem<MIST_F16>{});
}
template <class F>
void with_types(int32_t a, int32_t b, F&& f) {
  with_type(a, [&](auto x) { with_type(b, [&](auto y) { f(x, y); }); });
}

}  // namespace mist
