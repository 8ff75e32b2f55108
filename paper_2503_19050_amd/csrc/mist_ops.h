// Element types, vectors, lane exchanges and host helpers shared by the operators of a training step, its last stage and a layer
// (mist_embed.hip, mist_step.hip, mist_token.hip, mist_block.hip, mist_kept.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
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

typedef float Float8 __attribute__((ext_vector_type(8)));

// Eight columns of a row.  The columns at its end, and lanes past it, are read from the row's last eight values, in bounds and without
// a branch, and moved down when they are used: read value by value they would be waited for eight times (residual and norm of
// 65536 x 2559 bf16: 513 us so, 330 by one access).
// WHOLE: every lane has all eight.
template <bool WHOLE = false>
struct Eight {
  int col, left;  // left: columns there are from col on, none where <= 0
  int at, shift;  // the columns read, and how far they are to be moved down (8: nothing is left)
  bool narrow;    // the row has less than eight
  __device__ __forceinline__ Eight() {}
  __device__ __forceinline__ Eight(int column, int width) : col(column), left(width - column), narrow(width < 8) {
    at = narrow ? 0 : min(col, width - 8);
    shift = narrow ? 0 : min(col - at, 8);
  }
};

// As they are stored: 4 registers of 16-bit values.
template <class T>
using Raw8 = T __attribute__((ext_vector_type(8)));
template <class T, bool WHOLE>
__device__ __forceinline__ Raw8<T> load_raw8(const T* row, const Eight<WHOLE>& c) {
  if (WHOLE) return *(const typename Vec<T, 8>::type*)(row + c.col);
  if (!c.narrow) return *(const typename Vec<T, 8>::type*)(row + c.at);
  Raw8<T> x = (T)0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < c.left) x[k] = row[c.col + k];
  return x;
}
// Moved down, with zeros for what is not there.
template <class T, bool WHOLE>
__device__ __forceinline__ Raw8<T> settled(Raw8<T> x, const Eight<WHOLE>& c) {
  if (WHOLE) return x;
  typedef uint32_t Words __attribute__((ext_vector_type(sizeof(Raw8<T>) / 4)));
  constexpr int kWords = sizeof(Raw8<T>) / 4, kPer = 4 / sizeof(T);
  if (c.shift) {
    Words w = __builtin_bit_cast(Words, x);
#pragma unroll
    for (int step = 8; step >= kPer; step /= 2) {
#pragma unroll
      for (int k = 0; k < kWords; ++k) w[k] = !(c.shift & step) ? w[k] : k + step / kPer < kWords ? w[k + step / kPer] : 0u;
    }
    if (kPer == 2) {
#pragma unroll
      for (int k = 0; k < kWords; ++k) w[k] = !(c.shift & 1) ? w[k] : k + 1 < kWords ? w[k] >> 16 | w[k + 1] << 16 : w[k] >> 16;
    }
    x = __builtin_bit_cast(Raw8<T>, w);
  }
  return x;
}
template <class T, bool WHOLE>
__device__ __forceinline__ Float8 wide8(Raw8<T> x, const Eight<WHOLE>& c) {
  return __builtin_convertvector(settled<T>(x, c), Float8);
}
template <class T, bool WHOLE>
__device__ __forceinline__ Float8 load8(const T* row, const Eight<WHOLE>& c) {
  return wide8<T>(load_raw8(row, c), c);
}
template <class T, bool WHOLE>
__device__ __forceinline__ void store8(T* row, const Eight<WHOLE>& c, Float8 x) {
  if (WHOLE || c.left >= 8) {
    *(typename Vec<T, 8>::type*)(row + c.col) = __builtin_convertvector(x, typename Vec<T, 8>::type);
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < c.left) row[c.col + k] = (T)x[k];
}

// Sum, or largest, over a wave; every lane has the result.  Exchanges within 16 lanes are operands of the additions
// themselves, those of halves and quarters of the wave two instructions: no trip through shared memory.
template <int CTRL>
__device__ __forceinline__ uint32_t lanes(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ __forceinline__ float lanes(float x) {
  return __uint_as_float(lanes<CTRL>(__float_as_uint(x)));
}
// The largest of 16 neighbouring lanes, as unsigned numbers.
__device__ __forceinline__ uint32_t most_of_16(uint32_t x) {
  x = max(x, lanes<0xB1>(x));   // pairs
  x = max(x, lanes<0x4E>(x));   // fours
  x = max(x, lanes<0x141>(x));  // eights: mirrored
  return max(x, lanes<0x140>(x));
}
template <class J>
__device__ __forceinline__ float join_pairs_of_16(float x, J join) {
  const auto q = __builtin_amdgcn_permlane16_swap((unsigned)__float_as_int(x), (unsigned)__float_as_int(x), false, false);
  return join(__int_as_float((int)q[0]), __int_as_float((int)q[1]));
}
template <class J>
__device__ __forceinline__ float join_pairs_of_32(float x, J join) {
  const auto h = __builtin_amdgcn_permlane32_swap((unsigned)__float_as_int(x), (unsigned)__float_as_int(x), false, false);
  return join(__int_as_float((int)h[0]), __int_as_float((int)h[1]));
}
// Over groups of LANES (16, 32 or 64) neighbouring lanes.
template <int LANES = 64, class J>
__device__ __forceinline__ float wave_join(float x, J join) {
  x = join(x, lanes<0xB1>(x));   // pairs
  x = join(x, lanes<0x4E>(x));   // fours
  x = join(x, lanes<0x141>(x));  // eights: mirrored
  x = join(x, lanes<0x140>(x));  // sixteens: mirrored
  if (LANES >= 32) x = join_pairs_of_16(x, join);
  if (LANES >= 64) x = join_pairs_of_32(x, join);
  return x;
}
template <int LANES = 64>
__device__ __forceinline__ float wave_sum(float x) {
  return wave_join<LANES>(x, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float x) {
  return wave_join(x, [](float a, float b) { return fmaxf(a, b); });
}

// exp(x) by the base-2 instruction: off by 2^-24 |x| from the product and 1 ulp from the instruction.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// The addresses of rows of width elements, for checks of what shares memory.
struct Range {
  uintptr_t lo, hi;
};
inline Range range_of(const void* p, int64_t rows, int64_t stride, int64_t width, int64_t bytes) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  if (!p || rows <= 0 || width <= 0) return Range{lo, lo};
  const unsigned __int128 n = ((unsigned __int128)(rows - 1) * (uint64_t)stride + (uint64_t)width) * (uint64_t)bytes;
  return Range{lo, n > UINTPTR_MAX - lo ? UINTPTR_MAX : lo + (uintptr_t)n};
}
inline bool overlap(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi; }

// Whether two sets of rows share memory: their ranges do, unless both lie beside each other in rows of one stride (the
// halves of a product's output).
struct Rows {
  const void* p;
  int64_t rows, stride, width, bytes;  // bytes: of an element
};
inline bool overlap(const Rows& a, const Rows& b) {
  if (!overlap(range_of(a.p, a.rows, a.stride, a.width, a.bytes), range_of(b.p, b.rows, b.stride, b.width, b.bytes))) return false;
  const int64_t step = a.stride * a.bytes, wa = a.width * a.bytes, wb = b.width * b.bytes;
  if (a.rows <= 1 || b.rows <= 1 || step != b.stride * b.bytes || wa > step || wb > step) return true;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p), m = (uintptr_t)step;
  const int64_t off = (int64_t)(y >= x ? (y - x) % m : (m - (x - y) % m) % m);
  return off < wa || off + wb > step;
}

// A tensor of a call, by its addresses (Range or Rows).
template <class R>
struct Use {
  R at;
  bool out;
};
inline Range span_of(const Range& x) { return x; }
inline Range span_of(const Rows& x) { return range_of(x.p, x.rows, x.stride, x.width, x.bytes); }
// Whether an output of the first list shares memory with another tensor of it, or one of the first list with one of the second where
// either is an output.
template <class R, size_t N, size_t M>
bool shared(const Use<R> (&all)[N], const Use<R> (&others)[M]) {
  Range a[N], b[M];
  for (size_t i = 0; i < N; ++i) a[i] = span_of(all[i].at);
  for (size_t i = 0; i < M; ++i) b[i] = span_of(others[i].at);
  auto meet = [](const Use<R>& x, Range p, const Use<R>& y, Range q) {
    return (x.out || y.out) && p.lo != p.hi && q.lo != q.hi && overlap(p, q) && overlap(x.at, y.at);
  };
  for (size_t i = 0; i < N; ++i) {
    for (size_t k = 0; k < i; ++k)
      if (meet(all[i], a[i], all[k], a[k])) return true;
    for (size_t k = 0; k < M; ++k)
      if (meet(all[i], a[i], others[k], b[k])) return true;
  }
  return false;
}
template <class R, size_t N>
bool shared(const Use<R> (&all)[N]) {
  return shared<R>(all, {Use<R>{R{}, false}});
}

inline bool is_aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

constexpr int64_t kMostStride = (int64_t)1 << 40;
inline bool stride_ok(int64_t x) { return x >= 0 && x <= kMostStride; }

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
