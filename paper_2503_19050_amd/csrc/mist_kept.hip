// Tensors kept in 8 bits, and the MLP's activation with its inputs kept so.
//
// A group of 128 values is held by 16 neighbouring lanes, eight values each; its largest magnitude goes around them by four exchanges.
// Scales are powers of two: products with them are exact, so that a value's only rounding is the one to a
// whole multiple, and loaded values are exact in bf16.  Everything is one pass of a few operations a byte: bound by memory.
// Measured on one MI355X, where a large copy reads and writes 4.9 TB/s: store of 65536 x 8192 bf16 319 us, 5.0 TB/s, of 32768 x 8192 fp32 229, 5.9;
// load to bf16 275, 5.9; silu with a gate, 8192 x 13824 bf16, 166 us, 5.4 TB/s, its gradient 160, 5.7; gelu, 65536 x 10240, 645 and 641, 5.2.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mist_ops.h"

using mist::fast_exp;
using mist::Float8;
using mist::hip_failed;
using mist::lib_fail;
using mist::load8;
using mist::store8;

namespace {

constexpr int kThreads = 256;
constexpr int kLanes = MIST_KEPT_GROUP / 8;        // of a group
constexpr int64_t kMostBlocks = (int64_t)1 << 22;  // a grid stays below 2^32 threads; kernels loop

typedef int8_t Byte8 __attribute__((ext_vector_type(8)));

// Eight columns of a row: work of one lane.
struct Place {
  int64_t row;
  int32_t group;
  mist::Eight<> c;
};

struct Shape {
  int64_t rows;
  int32_t width, groups;
};

// f(place) for every lane of every group; the 16 lanes of a group come together.
template <class F>
__device__ __forceinline__ void each_place(const Shape& s, F&& f) {
  const uint32_t per_row = (uint32_t)s.groups * kLanes;  // below 2^28
  const int64_t total = s.rows * per_row;
  for (int64_t block = (int64_t)blockIdx.x * kThreads; block < total; block += (int64_t)gridDim.x * kThreads) {
    int64_t row = block / per_row;
    uint32_t at = (uint32_t)(block - row * per_row) + threadIdx.x;
    const uint32_t more = at / per_row;
    row += more;
    at -= more * per_row;
    if (row >= s.rows) continue;  // whole groups of lanes
    f(Place{row, (int32_t)(at / kLanes), mist::Eight<>((int)(at * 8), s.width)});
  }
}

// The byte of a group from its largest magnitude's bits: inf and NaN are the largest, as unsigned numbers.
__device__ __forceinline__ uint32_t byte_of(uint32_t most) {
  if (most >= 0x7F800000u) return 255;
  // exponent of the least power of two e with most <= 127 * 2^e = 1.984375 * 2^(e + 6): a mantissa past that carries
  const int32_t e = (int32_t)((most + 0x1FFFFu) >> 23) - 6;
  return (uint32_t)min(max(e, 1), 248);
}

// One lane's part of storing a group: all 16 lanes call it.
__device__ __forceinline__ void store_group(const Shape& s, const Place& p, Float8 x, const mist_kept& k) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  static_assert(kLanes == 16, "a group is a row of lanes");
  most = mist::most_of_16(most);
  const uint32_t byte = byte_of(most);
  const float inverse = byte == 255 ? 0.0f : __uint_as_float((254 - byte) << 23);
  Byte8 q;
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = byte == 255 ? 0 : (int8_t)(int)fminf(fmaxf(rintf(x[i] * inverse), -127.0f), 127.0f);
  *(Byte8*)(k.values + (p.row * s.groups + p.group) * MIST_KEPT_GROUP + p.c.col % MIST_KEPT_GROUP) = q;
  if (p.c.col % MIST_KEPT_GROUP == 0) k.exponents[p.row * s.groups + p.group] = (uint8_t)byte;
}

// The byte 255 gives an infinite factor of zeros: NaN.
__device__ __forceinline__ Float8 load_group(const Shape& s, const Place& p, const mist_kept& k) {
  const float step = __uint_as_float((uint32_t)k.exponents[p.row * s.groups + p.group] << 23);
  const Byte8 q = *(const Byte8*)(k.values + (p.row * s.groups + p.group) * MIST_KEPT_GROUP + p.c.col % MIST_KEPT_GROUP);
  return __builtin_convertvector(q, Float8) * step;
}

// f16's largest value is kept as one past it.
template <class T>
__device__ __forceinline__ Float8 in_range(Float8 x) {
  if (sizeof(T) == 2 && !__is_same(T, __bf16)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] > 65504.0f ? 65504.0f : x[i] < -65504.0f ? -65504.0f : x[i];
  }
  return x;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_store(Shape s, const T* x, int64_t stride, mist_kept k) {
  each_place(s, [&](const Place& p) { store_group(s, p, load8(x + p.row * stride, p.c), k); });
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_load(Shape s, mist_kept k, T* x, int64_t stride) {
  each_place(s, [&](const Place& p) { store8(x + p.row * stride, p.c, in_range<T>(load_group(s, p, k))); });
}

// The activation and its derivative.  With e = exp(-z) and p = 1 / (1 + e), 1 - p is e p, without the difference's loss; where e is
// infinite p and a are 0.
struct Act {
  float a, slope;
};
constexpr float kFinite = 3e38f;
template <int KIND>
__device__ __forceinline__ Act act(float x) {
  if (KIND == MIST_ACT_SILU) {
    const float e = fast_exp(-x), p = __builtin_amdgcn_rcpf(1.0f + e), a = x * p;
    return Act{a, fmaf(a, fminf(e, kFinite) * p, p)};
  }
  // 1/2 (1 + tanh z) = 1 / (1 + exp(-2 z)); past 13 it is 0 or 1 in fp32, and the cube stays finite
  constexpr float k = 1.5957691216057308f;  // 2 sqrt(2 / pi)
  const float w = fminf(fmaxf(x, -13.0f), 13.0f), w2 = w * w;
  const float e = fast_exp(-k * w * fmaf(0.044715f, w2, 1.0f)), p = __builtin_amdgcn_rcpf(1.0f + e), a = x * p;
  return Act{a, fmaf(a, fminf(e, kFinite) * p * (k * fmaf(0.134145f, w2, 1.0f)), p)};
}

struct Strides {
  int64_t up, gate, out, again;
};

template <class T, int KIND, bool GATE>
__global__ __launch_bounds__(kThreads) void k_act(Shape s, Strides st, const T* up, const T* gate, T* out, mist_kept up8, mist_kept gate8) {
  each_place(s, [&](const Place& p) {
    const Float8 u = load8(up + p.row * st.up, p.c);
    Float8 g, y;
    if (GATE) g = load8(gate + p.row * st.gate, p.c);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = GATE ? act<KIND>(g[i]).a * u[i] : act<KIND>(u[i]).a;
    if (up8.values) store_group(s, p, u, up8);
    if (GATE && gate8.values) store_group(s, p, g, gate8);
    store8(out + p.row * st.out, p.c, y);
  });
}

template <class T, int KIND, bool GATE>
__global__ __launch_bounds__(kThreads) void k_act_back(Shape s, Strides st, mist_kept up8, mist_kept gate8, const T* dout, T* dup, T* dgate, T* again) {
  each_place(s, [&](const Place& p) {
    const Float8 d = load8(dout + p.row * st.out, p.c), u = in_range<T>(load_group(s, p, up8));
    Float8 g, y, du, dg;
    if (GATE) g = in_range<T>(load_group(s, p, gate8));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Act f = act<KIND>(GATE ? g[i] : u[i]);
      y[i] = GATE ? f.a * u[i] : f.a;
      du[i] = d[i] * (GATE ? f.a : f.slope);
      if (GATE) dg[i] = d[i] * u[i] * f.slope;
    }
    store8(dup + p.row * st.up, p.c, du);
    if (GATE) store8(dgate + p.row * st.gate, p.c, dg);
    if (again) store8(again + p.row * st.again, p.c, y);
  });
}

bool shape_ok(int64_t rows, int64_t width, const char** why) {
  *why = rows < 0 || rows > INT32_MAX || width < 1 || width > INT32_MAX ? "rows must be in 0..2^31-1, width in 1..2^31-1"
         : rows * ((width + MIST_KEPT_GROUP - 1) / MIST_KEPT_GROUP) >= (int64_t)1 << 40 ? "too many values (2^40 groups)" : nullptr;
  return !*why;
}
Shape shape_of(int64_t rows, int64_t width) { return Shape{rows, (int32_t)width, (int32_t)((width + MIST_KEPT_GROUP - 1) / MIST_KEPT_GROUP)}; }

// A tensor of the call; `like`: the input whose place an output may take.
struct Tensor {
  const void* p;
  int64_t stride;
  bool out;
  const void* like[2];
};

mist::Rows rows_of(const Shape& s, const Tensor& t, int32_t type) { return mist::Rows{t.p, s.rows, t.stride, s.width, mist::type_bytes(type)}; }
mist::Range range_of(const Shape& s, const Tensor& t, int32_t type) { return mist::range_of(t.p, s.rows, t.stride, s.width, mist::type_bytes(type)); }
mist::Range values_of(const Shape& s, const mist_kept* k) {
  return mist::range_of(k->values, s.rows, (int64_t)s.groups * MIST_KEPT_GROUP, (int64_t)s.groups * MIST_KEPT_GROUP, 1);
}
mist::Range exponents_of(const Shape& s, const mist_kept* k) { return mist::range_of(k->exponents, s.rows, s.groups, s.groups, 1); }

mist_status check_tensors(const Shape& s, int32_t type, std::initializer_list<Tensor> ts, std::initializer_list<const mist_kept*> ks, bool ks_out) {
  for (const Tensor& t : ts) {
    if (!mist::stride_ok(t.stride)) return lib_fail(MIST_E_INVALID, "kept activations: strides must be in 0..2^40");
    if (!mist::is_aligned(t.p, (size_t)mist::type_bytes(type))) return lib_fail(MIST_E_INVALID, "kept activations: a buffer is not aligned to its elements");
    if (!t.p || !t.out) continue;
    if (s.rows > 1 && t.stride < s.width) return lib_fail(MIST_E_INVALID, "kept activations: rows of an output overlap");
    for (const Tensor& o : ts) {
      if (&o == &t || !o.p) continue;
      const bool same = !o.out && o.p == t.p && (s.rows <= 1 || o.stride == t.stride) && (o.p == t.like[0] || o.p == t.like[1]);
      if (!same && mist::overlap(rows_of(s, t, type), rows_of(s, o, type)))
        return lib_fail(MIST_E_INVALID, "kept activations: an output overlaps another tensor");
    }
  }
  for (auto it = ks.begin(); it != ks.end(); ++it) {
    const mist_kept* k = *it;
    if (!k) continue;
    if (s.rows && (!k->values || !k->exponents)) return lib_fail(MIST_E_INVALID, "kept activations: null buffer");
    if (!mist::is_aligned(k->values, 16)) return lib_fail(MIST_E_INVALID, "kept activations: values are not aligned to 16");
    for (const Tensor& t : ts)
      if ((t.out || ks_out) && t.p && (mist::overlap(range_of(s, t, type), values_of(s, k)) || mist::overlap(range_of(s, t, type), exponents_of(s, k))))
        return lib_fail(MIST_E_INVALID, "kept activations: values or exponents overlap a tensor");
    if (!ks_out) continue;
    if (mist::overlap(values_of(s, k), exponents_of(s, k))) return lib_fail(MIST_E_INVALID, "kept activations: values and exponents overlap");
    for (auto o = ks.begin(); o != it; ++o)
      if (*o && (mist::overlap(values_of(s, k), values_of(s, *o)) || mist::overlap(values_of(s, k), exponents_of(s, *o)) || mist::overlap(exponents_of(s, k), exponents_of(s, *o))))
        return lib_fail(MIST_E_INVALID, "kept activations: two of them overlap");
  }
  return MIST_OK;
}

unsigned blocks_of(const Shape& s) {
  return (unsigned)std::min<int64_t>((s.rows * s.groups * kLanes + kThreads - 1) / kThreads, kMostBlocks);
}

mist_status check(const mist_kept_desc* d) {
  if (!d) return lib_fail(MIST_E_INVALID, "kept activations: null descriptor");
  const char* why;
  if (!shape_ok(d->rows, d->width, &why)) return lib_fail(MIST_E_INVALID, why);
  if (!mist::type_ok(d->type)) return lib_fail(MIST_E_INVALID, "kept activations: unknown element type");
  return MIST_OK;
}

mist_status check(const mist_act_desc* d) {
  if (!d) return lib_fail(MIST_E_INVALID, "activation: null descriptor");
  const char* why;
  if (!shape_ok(d->rows, d->width, &why)) return lib_fail(MIST_E_INVALID, why);
  if (!mist::type_ok(d->type)) return lib_fail(MIST_E_INVALID, "activation: unknown element type");
  if (d->kind != MIST_ACT_SILU && d->kind != MIST_ACT_GELU) return lib_fail(MIST_E_INVALID, "activation: unknown kind");
  return MIST_OK;
}

// f(type, kind, gated)
template <class F>
void with_act(const mist_act_desc* d, bool gated, F&& f) {
  mist::with_type(d->type, [&](auto x) {
    auto kind = [&](auto k) {
      if (gated) f(x, k, std::true_type{});
      else f(x, k, std::false_type{});
    };
    if (d->kind == MIST_ACT_SILU) kind(std::integral_constant<int, MIST_ACT_SILU>{});
    else kind(std::integral_constant<int, MIST_ACT_GELU>{});
  });
}

mist_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, what);
}

}  // namespace

extern "C" {

mist_status mist_kept_store(const mist_kept_desc* d, const void* x, int8_t* values, uint8_t* exponents, void* stream) {
  if (const mist_status st = check(d)) return st;
  const Shape s = shape_of(d->rows, d->width);
  if (s.rows && !x) return lib_fail(MIST_E_INVALID, "kept activations: null buffer");
  const mist_kept k{values, exponents};
  if (const mist_status st = check_tensors(s, d->type, {{x, d->stride, false, {}}}, {&k}, true)) return st;
  if (s.rows == 0) return MIST_OK;
  mist::with_type(d->type, [&](auto e) {
    using T = typename decltype(e)::type;
    hipLaunchKernelGGL((k_store<T>), dim3(blocks_of(s)), dim3(kThreads), 0, (hipStream_t)stream, s, (const T*)x, d->stride, k);
  });
  return launched("kept activations");
}

mist_status mist_kept_load(const mist_kept_desc* d, const int8_t* values, const uint8_t* exponents, void* x, void* stream) {
  if (const mist_status st = check(d)) return st;
  const Shape s = shape_of(d->rows, d->width);
  if (s.rows && !x) return lib_fail(MIST_E_INVALID, "kept activations: null buffer");
  const mist_kept k{const_cast<int8_t*>(values), const_cast<uint8_t*>(exponents)};
  if (const mist_status st = check_tensors(s, d->type, {{x, d->stride, true, {}}}, {&k}, false)) return st;
  if (s.rows == 0) return MIST_OK;
  mist::with_type(d->type, [&](auto e) {
    using T = typename decltype(e)::type;
    hipLaunchKernelGGL((k_load<T>), dim3(blocks_of(s)), dim3(kThreads), 0, (hipStream_t)stream, s, k, (T*)x, d->stride);
  });
  return launched("kept activations");
}

mist_status mist_act_forward(const mist_act_desc* d, const void* up, const void* gate, void* out, const mist_kept* up8, const mist_kept* gate8,
                             void* stream) {
  if (const mist_status st = check(d)) return st;
  const Shape s = shape_of(d->rows, d->width);
  if (gate8 && !gate) return lib_fail(MIST_E_INVALID, "activation: a gate to keep that is not there");
  if (s.rows && (!up || !out)) return lib_fail(MIST_E_INVALID, "activation: null buffer");
  if (const mist_status st = check_tensors(s, d->type, {{up, d->up_stride, false, {}}, {gate, d->gate_stride, false, {}}, {out, d->out_stride, true, {up, gate}}},
                                           {up8, gate8}, true))
    return st;
  if (s.rows == 0) return MIST_OK;
  const mist_kept none{};
  with_act(d, gate != nullptr, [&](auto e, auto kind, auto gated) {
    using T = typename decltype(e)::type;
    hipLaunchKernelGGL((k_act<T, kind.value, gated.value>), dim3(blocks_of(s)), dim3(kThreads), 0, (hipStream_t)stream, s,
                       Strides{d->up_stride, d->gate_stride, d->out_stride, 0}, (const T*)up, (const T*)gate, (T*)out, up8 ? *up8 : none, gate8 ? *gate8 : none);
  });
  return launched("activation");
}

mist_status mist_act_backward(const mist_act_desc* d, const mist_kept* up8, const mist_kept* gate8, const void* dout, void* dup, void* dgate, void* again,
                              void* stream) {
  if (const mist_status st = check(d)) return st;
  const Shape s = shape_of(d->rows, d->width);
  if (!up8 || (s.rows && (!dout || !dup || (gate8 && !dgate)))) return lib_fail(MIST_E_INVALID, "activation's gradient: null buffer");
  if (!gate8 && dgate) return lib_fail(MIST_E_INVALID, "activation's gradient: of a gate that is not there");
  if (const mist_status st = check_tensors(s, d->type, {{dout, d->out_stride, false, {}}, {dup, d->up_stride, true, {dout, nullptr}},
                                                        {dgate, d->gate_stride, true, {dout, nullptr}}, {again, d->again_stride, true, {}}},
                                           {up8, gate8}, false))
    return st;
  if (s.rows == 0) return MIST_OK;
  const mist_kept none{};
  with_act(d, gate8 != nullptr, [&](auto e, auto kind, auto gated) {
    using T = typename decltype(e)::type;
    hipLaunchKernelGGL((k_act_back<T, kind.value, gated.value>), dim3(blocks_of(s)), dim3(kThreads), 0, (hipStream_t)stream, s,
                       Strides{d->up_stride, d->gate_stride, d->out_stride, d->again_stride}, *up8, gate8 ? *gate8 : none, (const T*)dout, (T*)dup, (T*)dgate,
                       (T*)again);
  });
  return launched("activation's gradient");
}

}  // extern "C"
