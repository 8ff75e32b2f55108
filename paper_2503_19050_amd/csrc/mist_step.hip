// Lists of tensors, the global gradient norm, clipping and the Adam step.
//
// Each is one pass over its values, a few operations a byte: bound by memory.  A list's tensors are cut into
// pieces of 4096 elements, one block each (on one card, blocks that take pieces in turn measured 3650 us where these
// take 3410, pieces of 2048 or 8192 elements 3515 and 3500: Adam step of 629 million parameters).  Measured on one
// MI355X, where a large copy reads and writes 4.9 TB/s:
//   norm   302 million fp32  200 us, 6.1 TB/s;  629 million bf16  212 us, 6.0 TB/s
//   clip   302 million fp32 to bf16  294 us, 6.2 TB/s (its reads partly from the cache)
//   Adam   629 million, bf16 gradients and weights  3156 us, 5.6 TB/s;  39.7 million in f16, one element
//          off alignment  222 us, 5.3 TB/s
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "mist_ops.h"

using mist::hip_failed;
using mist::lib_fail;
using mist::Vec;

namespace {

constexpr int kThreads = 256;
constexpr int kTotalThreads = 1024;
constexpr int64_t kChunk = 4096;     // elements a block takes at a time, of one tensor
constexpr int64_t kMostPieces = (int64_t)1 << 28;
constexpr uint32_t kGridX = 1 << 22;  // blocks along x, so that a dimension has less than 2^32 threads
constexpr int kNormBlocks = 2048;    // partial results of the norm, at most

// A block's piece of work: elements [part * kChunk, ...) of a tensor.
struct Piece {
  int32_t tensor, part;
};

// The tables as kernels see them.
struct List {
  const uint64_t* ptr;    // [n] addresses
  const int64_t* size;    // [n] elements
  const Piece* piece;     // [n_pieces]
};

}  // namespace

struct mist_tensors {
  int device = 0;
  int32_t type = 0;
  std::vector<int64_t> size;
  int64_t n_pieces = 0;
  bool overlaps = false;  // a value is in two of the tensors
  List list{};
  void* block = nullptr;  // the device tables
  mist_allocator alloc{};
  bool own_alloc = false;
};

namespace {

struct Span {
  uint64_t ptr;
  int64_t begin, end;  // elements
};

// The block's number counted from the last of `blocks`; negative past the first.
__device__ __forceinline__ int64_t block_from_last(int64_t blocks) {
  return blocks - 1 - ((int64_t)blockIdx.y * gridDim.x + blockIdx.x);
}

__device__ __forceinline__ Span span_of(const List& l, const Piece p) {
  const int64_t begin = (int64_t)p.part * kChunk, size = l.size[p.tensor];
  return Span{l.ptr[p.tensor], begin, begin + kChunk < size ? begin + kChunk : size};
}

// Sum, or largest with NaN above everything, over a block; the result is in thread 0.
template <bool MAX>
__device__ __forceinline__ double join(double a, double b) {
  if (!MAX) return a + b;
  return a > b || a != a ? a : b;
}
template <bool MAX, int THREADS>
__device__ double block_join(double x) {
  __shared__ double part[THREADS / 64];
  for (int d = 32; d; d >>= 1) x = join<MAX>(x, __shfl_down(x, d));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
  __syncthreads();
  x = part[0];
  for (int k = 1; k < THREADS / 64; ++k) x = join<MAX>(x, part[k]);
  return x;
}

__device__ void finish(const mist_clip_desc& c, mist_step_record* r, double total) {
  const double scale = fabs((double)c.grad_scale);
  const double norm = scale * (c.kind == MIST_NORM_L2 ? sqrt(total) : total);
  r->norm = (float)norm;
  const bool fine = r->norm < HUGE_VALF;  // of the norm as it is reported; false for NaN
  r->coef = fine ? (float)(c.grad_scale * (norm > c.max_norm ? c.max_norm / norm : 1.0)) : c.grad_scale;
  r->applied = fine;
  r->step += fine;
  r->skipped += !fine;
}

// Reads only: pieces in turn, four loads of 16 bytes a thread in flight; the next piece's table entries are
// read ahead.  The blocks' results are joined by a launch of their own: letting the last block to arrive do
// it in this one takes a release of the XCD's cache from every block, which measured 85 us more on 302
// million fp32 gradients (224 us) where the launch takes 5.
template <class G, bool MAX>
__global__ __launch_bounds__(kThreads) void k_norm(List l, int64_t n_pieces, double* __restrict__ part) {
  constexpr int kV = 16 / sizeof(G), kLoads = 4;
  typedef typename Vec<G, kV>::type V;
  double sum = 0.0;
  auto add = [&](G g) {
    const double x = (double)(float)g;
    sum = MAX ? join<true>(sum, fabs(x)) : fma(x, x, sum);
  };
  int64_t k = blockIdx.x;
  Span s = k < n_pieces ? span_of(l, l.piece[k]) : Span{};
  for (; k < n_pieces; k += gridDim.x) {
    const G* g = (const G*)s.ptr + s.begin;
    const int n = (int)(s.end - s.begin), vectors = n / kV;
    if (k + gridDim.x < n_pieces) s = span_of(l, l.piece[k + gridDim.x]);
    for (int i0 = 0; i0 < vectors; i0 += kThreads * kLoads) {
      V x[kLoads];
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int i = i0 + j * kThreads + threadIdx.x;
        x[j] = i < vectors ? *(const V*)(g + i * kV) : V{};
      }
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int c = 0; c < kV; ++c) add(x[j][c]);
    }
    if (const int i = vectors * kV + threadIdx.x; i < n) add(g[i]);
  }
  sum = block_join<MAX, kThreads>(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// One block: joins the results in order.
template <bool MAX>
__global__ __launch_bounds__(kTotalThreads) void k_total(const double* __restrict__ part, int32_t n, mist_clip_desc c, int32_t accumulate,
                                                         int32_t do_finish, mist_step_record* r) {
  double x = 0.0;
#pragma unroll 2
  for (int32_t k = threadIdx.x; k < n; k += kTotalThreads) x = join<MAX>(x, part[k]);
  x = block_join<MAX, kTotalThreads>(x);
  if (threadIdx.x) return;
  if (accumulate) x = join<MAX>(r->total, x);
  r->total = x;
  if (do_finish) finish(c, r, x);
}

__global__ void k_finish(mist_clip_desc c, mist_step_record* r) { finish(c, r, r->total); }

// Pieces from the last to the first: what the norm has read last is still in the cache.  Two blocks a piece
// (302 million fp32 gradients to bf16: 486 us with the norm, 507 with one, 515 with blocks that loop).
constexpr int kClipBlocks = 2;

template <class G, class O>
__global__ __launch_bounds__(kThreads) void k_clip(List g, List out, int64_t n_pieces, const mist_step_record* __restrict__ r) {
  constexpr int kV = sizeof(G) == 2 && sizeof(O) == 2 ? 8 : 4, kLoads = 2;
  typedef typename Vec<G, kV>::type VG;
  typedef typename Vec<O, kV>::type VO;
  typedef typename Vec<float, kV>::type VF;
  const int64_t block = block_from_last(n_pieces * kClipBlocks);
  if (block < 0) return;
  const Piece p = g.piece[block / kClipBlocks];
  Span s = span_of(g, p);
  s.begin += block % kClipBlocks * (kChunk / kClipBlocks);
  s.end = min(s.end, s.begin + kChunk / kClipBlocks);
  if (s.begin >= s.end) return;
  const float coef = r->applied ? r->coef : 1.0f;
  const G* x = (const G*)s.ptr + s.begin;
  O* y = (O*)out.ptr[p.tensor] + s.begin;
  const int n = (int)(s.end - s.begin), vectors = n / kV;
  for (int i0 = 0; i0 < vectors; i0 += kThreads * kLoads) {
    VG v[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = i0 + j * kThreads + threadIdx.x;
      if (i < vectors) v[j] = *(const VG*)(x + i * kV);
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = i0 + j * kThreads + threadIdx.x;
      if (i < vectors) __builtin_nontemporal_store(__builtin_convertvector(coef * __builtin_convertvector(v[j], VF), VO), (VO*)(y + i * kV));
    }
  }
  if (const int i = vectors * kV + threadIdx.x; i < n) y[i] = (O)(coef * (float)x[i]);
}

// A beta in two fp32 terms, hi + lo.  One alone is off by up to 2^-25, which for a slow average (beta near 1) is a part
// of 1 - beta: 0.1 % at 0.99999, all of it at 1 - 1e-8.  hi is below beta and lo above 0 (unless beta is 0), so
// that an infinite average stays infinite.
struct Decay {
  float hi, lo;
};

Decay decay_of(double beta) {
  if (!(beta > 0.0)) return Decay{0.0f, 0.0f};
  float hi = (float)beta;
  if ((double)hi >= beta) hi = std::nextafterf(hi, 0.0f);
  return Decay{hi, (float)(beta - (double)hi)};
}

struct AdamArgs {
  List p, m, v, g, w;
  double beta1, beta2;
  Decay b1, b2;
  float one_b1, one_b2, lr, decay, eps;
};

__device__ double power(double x, int64_t n) {
  double y = 1.0;
  for (; n > 0; n >>= 1, x *= x)
    if (n & 1) y *= x;
  return y;
}

struct AdamScalars {
  float coef, ibc1, ibc2;
};

__device__ __forceinline__ void adam_one(const AdamArgs& a, const AdamScalars& c, float g, float& p, float& m, float& v) {
  const float x = c.coef * g;
  m = fmaf(a.b1.hi, m, fmaf(a.b1.lo, m, a.one_b1 * x));
  v = fmaf(a.b2.hi, v, fmaf(a.b2.lo, v, a.one_b2 * x * x));
  // the decay joins the update: a factor 1 - lr * weight_decay next to 1 holds a small product in few bits or none
  p = fmaf(-a.lr, fmaf(a.decay, p, m * c.ibc1 / (sqrtf(v * c.ibc2) + a.eps)), p);
  asm("" : "+v"(p));  // the weights are the stored p rounded, not the sum rounded once to 16 bits
}

// Pieces from the last to the first, as the clipping takes them.
template <class G, class W, bool WEIGHTS>
__global__ __launch_bounds__(kThreads) void k_adam(AdamArgs a, int64_t n_pieces, const mist_step_record* __restrict__ r) {
  constexpr int kV = 4, kLoads = 4;
  typedef typename Vec<G, kV>::type VG;
  typedef typename Vec<W, kV>::type VW;
  typedef typename Vec<float, kV>::type VF;
  const int64_t block = block_from_last(n_pieces);
  if (block < 0 || !r->applied) return;
  const Piece piece = a.g.piece[block];
  const Span s = span_of(a.g, piece);
  const AdamScalars c{r->coef, (float)(1.0 / (1.0 - power(a.beta1, r->step))), (float)(1.0 / (1.0 - power(a.beta2, r->step)))};
  const G* g = (const G*)s.ptr + s.begin;
  float* p = (float*)a.p.ptr[piece.tensor] + s.begin;
  float* m = (float*)a.m.ptr[piece.tensor] + s.begin;
  float* v = (float*)a.v.ptr[piece.tensor] + s.begin;
  W* w = WEIGHTS ? (W*)a.w.ptr[piece.tensor] + s.begin : nullptr;
  const int n = (int)(s.end - s.begin), vectors = n / kV;
  for (int i0 = 0; i0 < vectors; i0 += kThreads * kLoads) {
    VG vg[kLoads];
    VF vp[kLoads], vm[kLoads], vv[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = i0 + j * kThreads + threadIdx.x;
      if (i < vectors) {
        vg[j] = *(const VG*)(g + i * kV);
        vp[j] = __builtin_nontemporal_load((const VF*)(p + i * kV));
        vm[j] = __builtin_nontemporal_load((const VF*)(m + i * kV));
        vv[j] = __builtin_nontemporal_load((const VF*)(v + i * kV));
      }
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = i0 + j * kThreads + threadIdx.x;
      if (i < vectors) {
#pragma unroll
        for (int k = 0; k < kV; ++k) {
          float pk = vp[j][k], mk = vm[j][k], vk = vv[j][k];
          adam_one(a, c, (float)vg[j][k], pk, mk, vk);
          vp[j][k] = pk, vm[j][k] = mk, vv[j][k] = vk;
        }
        __builtin_nontemporal_store(vp[j], (VF*)(p + i * kV));
        __builtin_nontemporal_store(vm[j], (VF*)(m + i * kV));
        __builtin_nontemporal_store(vv[j], (VF*)(v + i * kV));
        if (WEIGHTS) __builtin_nontemporal_store(__builtin_convertvector(vp[j], VW), (VW*)(w + i * kV));
      }
    }
  }
  if (const int i = vectors * kV + threadIdx.x; i < n) {
    adam_one(a, c, (float)g[i], p[i], m[i], v[i]);
    if (WEIGHTS) w[i] = (W)p[i];
  }
}

bool tensors_overlap(const void* const* ptrs, const int64_t* sizes, int64_t n, int64_t bytes) {
  std::vector<std::pair<uintptr_t, int64_t>> at;
  at.reserve((size_t)n);
  for (int64_t i = 0; i < n; ++i)
    if (sizes[i]) at.emplace_back(reinterpret_cast<uintptr_t>(ptrs[i]), sizes[i] * bytes);
  std::sort(at.begin(), at.end());
  for (size_t i = 1; i < at.size(); ++i)
    if (at[i].first - at[i - 1].first < (uint64_t)at[i - 1].second) return true;
  return false;
}

// Frees the tables and the list, on its device.  Nothing uses them any more.
void release(mist_tensors* T) {
  if (!T) return;
  int cur = 0;
  const bool known = hipGetDevice(&cur) == hipSuccess;
  if (known && cur != T->device) (void)hipSetDevice(T->device);
  if (T->block) {
    if (T->own_alloc) (void)hipFree(T->block);
    else T->alloc.free(T->block, T->alloc.ctx);
  }
  if (known && cur != T->device) (void)hipSetDevice(cur);
  delete T;
}

// Waits for the work of the list's device.
hipError_t wait_for(const mist_tensors* T) {
  int cur = 0;
  hipError_t e = hipGetDevice(&cur);
  if (e == hipSuccess && cur != T->device) e = hipSetDevice(T->device);
  if (e != hipSuccess) return e;
  e = hipDeviceSynchronize();
  if (e != hipSuccess) (void)hipGetLastError();
  if (cur != T->device) (void)hipSetDevice(cur);
  return e;
}

mist_status on_device(const mist_tensors* T, const char* what) {
  int dev = -1;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_failed(e, what);
  if (dev != T->device) return lib_fail(MIST_E_INVALID, "tensor list: another device is current than the list's");
  return MIST_OK;
}

mist_status like(const mist_tensors* a, const mist_tensors* b) {
  if (a == b) return MIST_OK;
  if (a->device != b->device) return lib_fail(MIST_E_INVALID, "tensor lists are on different devices");
  if (a->size != b->size) return lib_fail(MIST_E_INVALID, "tensor lists differ in count or sizes");
  return MIST_OK;
}

// A list that is written: two blocks would take a value that occurs twice, in any order.
mist_status written(const mist_tensors* T) {
  return T && T->overlaps ? lib_fail(MIST_E_INVALID, "tensor list: tensors that are written overlap") : MIST_OK;
}

bool clip_ok(const mist_clip_desc* c) {
  return (c->kind == MIST_NORM_L2 || c->kind == MIST_NORM_MAX) && std::isfinite(c->grad_scale) && c->grad_scale != 0.0f &&
         c->max_norm > 0.0;
}

bool aligned8(const void* p) { return reinterpret_cast<uintptr_t>(p) % 8 == 0; }

dim3 grid_of(int64_t blocks) {
  const uint32_t x = (uint32_t)std::min<int64_t>(blocks, kGridX);
  return dim3(x, (uint32_t)((blocks + x - 1) / x));
}

int32_t norm_blocks(const mist_tensors* g) { return (int32_t)std::min<int64_t>(g->n_pieces, kNormBlocks); }

}  // namespace

extern "C" {

mist_status mist_tensors_create(const void* const* ptrs, const int64_t* sizes, int64_t n, int32_t type,
                                const mist_allocator* alloc, mist_tensors** out) {
  if (!out) return lib_fail(MIST_E_INVALID, "tensor list: null argument");
  *out = nullptr;
  if (n < 0 || n > INT32_MAX || (n && (!ptrs || !sizes))) return lib_fail(MIST_E_INVALID, "tensor list: null argument or bad count");
  if (!mist::type_ok(type)) return lib_fail(MIST_E_INVALID, "tensor list: unknown element type");
  if (alloc && (!alloc->alloc || !alloc->free)) return lib_fail(MIST_E_INVALID, "tensor list: allocator without functions");
  const int64_t bytes = mist::type_bytes(type);
  int64_t pieces = 0;
  for (int64_t i = 0; i < n; ++i) {
    if (sizes[i] < 0 || sizes[i] > ((int64_t)1 << 42)) return lib_fail(MIST_E_INVALID, "tensor list: sizes must be in 0..2^42");
    if (sizes[i] && (!ptrs[i] || reinterpret_cast<uintptr_t>(ptrs[i]) % bytes))
      return lib_fail(MIST_E_INVALID, "tensor list: a tensor is null or not aligned to its elements");
    pieces += (sizes[i] + kChunk - 1) / kChunk;
    if (pieces > kMostPieces) return lib_fail(MIST_E_INVALID, "tensor list: too many elements (over about 2^40)");
  }
  mist_tensors* T = nullptr;
  try {
    T = new mist_tensors;
    T->type = type;
    T->size.assign(sizes, sizes + n);
    T->n_pieces = pieces;
    T->overlaps = tensors_overlap(ptrs, sizes, n, bytes);
    hipError_t e = hipGetDevice(&T->device);
    if (e == hipSuccess && pieces) {
      // one block: addresses, sizes, pieces (8 bytes each)
      std::vector<uint64_t> table((size_t)(2 * n + pieces));
      Piece* piece = reinterpret_cast<Piece*>(table.data() + 2 * n);
      for (int64_t i = 0; i < n; ++i) {
        table[(size_t)i] = (uint64_t)reinterpret_cast<uintptr_t>(ptrs[i]);
        table[(size_t)(n + i)] = (uint64_t)sizes[i];
        for (int64_t k = 0; k * kChunk < sizes[i]; ++k) *piece++ = Piece{(int32_t)i, (int32_t)k};
      }
      const size_t total = table.size() * 8;
      if (alloc) {
        T->alloc = *alloc;
        T->block = alloc->alloc(total, nullptr, alloc->ctx);
      } else {
        T->own_alloc = true;
        if (hipMalloc(&T->block, total) != hipSuccess) {
          (void)hipGetLastError();
          T->block = nullptr;
        }
      }
      if (!T->block) {
        release(T);
        return lib_fail(MIST_E_NOMEM, "tensor list: device memory");
      }
      // the copy is on the null stream; callers use other streams, so it is waited for
      e = hipMemcpy(T->block, table.data(), total, hipMemcpyHostToDevice);
      if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
      T->list = List{(const uint64_t*)T->block, (const int64_t*)T->block + n, (const Piece*)((const uint64_t*)T->block + 2 * n)};
    }
    if (e != hipSuccess) {
      release(T);
      return hip_failed(e, "tensor list");
    }
  } catch (...) {
    release(T);
    return lib_fail(MIST_E_NOMEM, "tensor list: host memory");
  }
  *out = T;
  return MIST_OK;
}

mist_status mist_tensors_destroy(mist_tensors* T) {
  if (T && T->block) {
    const hipError_t e = wait_for(T);
    if (e != hipSuccess) return hip_failed(e, "tensor list: its work cannot be waited for");
  }
  release(T);
  return MIST_OK;
}

mist_status mist_norm_workspace(const mist_tensors* g, size_t* bytes) {
  if (!g || !bytes) return lib_fail(MIST_E_INVALID, "gradient norm: null argument");
  *bytes = (size_t)norm_blocks(g) * 8;
  return MIST_OK;
}

mist_status mist_grad_norm(const mist_tensors* g, const mist_clip_desc* c, int32_t accumulate, int32_t do_finish,
                           mist_step_record* record, void* workspace, size_t workspace_bytes, void* stream) {
  if (!g || !c || !record) return lib_fail(MIST_E_INVALID, "gradient norm: null argument");
  if (!clip_ok(c)) return lib_fail(MIST_E_INVALID, "gradient norm: unknown kind, or grad_scale or max_norm out of range");
  if (accumulate != 0 && accumulate != 1) return lib_fail(MIST_E_INVALID, "gradient norm: accumulate must be 0 or 1");
  if (do_finish != 0 && do_finish != 1) return lib_fail(MIST_E_INVALID, "gradient norm: finish must be 0 or 1");
  const int32_t blocks = norm_blocks(g);
  if (blocks && !workspace) return lib_fail(MIST_E_INVALID, "gradient norm: null workspace");
  if (workspace_bytes < (size_t)blocks * 8) return lib_fail(MIST_E_RANGE, "gradient norm: workspace too small");
  if (!aligned8(workspace) || !aligned8(record)) return lib_fail(MIST_E_INVALID, "gradient norm: workspace or record not aligned to 8");
  if (const mist_status st = on_device(g, "gradient norm")) return st;
  const hipStream_t st = (hipStream_t)stream;
  const bool max = c->kind == MIST_NORM_MAX;
  double* part = (double*)workspace;
  mist::with_type(g->type, [&](auto x) {
    using G = typename decltype(x)::type;
    const auto kernel = max ? k_norm<G, true> : k_norm<G, false>;
    if (blocks) hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, st, g->list, g->n_pieces, part);
  });
  hipLaunchKernelGGL(max ? k_total<true> : k_total<false>, dim3(1), dim3(kTotalThreads), 0, st, part, blocks, *c, accumulate, do_finish,
                     record);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "gradient norm");
}

mist_status mist_grad_finish(const mist_clip_desc* c, mist_step_record* record, void* stream) {
  if (!c || !record) return lib_fail(MIST_E_INVALID, "gradient norm: null argument");
  if (!clip_ok(c)) return lib_fail(MIST_E_INVALID, "gradient norm: unknown kind, or grad_scale or max_norm out of range");
  if (!aligned8(record)) return lib_fail(MIST_E_INVALID, "gradient norm: record not aligned to 8");
  hipLaunchKernelGGL(k_finish, dim3(1), dim3(1), 0, (hipStream_t)stream, *c, record);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "gradient norm");
}

mist_status mist_grad_clip(const mist_tensors* g, const mist_step_record* record, const mist_tensors* out, void* stream) {
  if (!g || !record || !out) return lib_fail(MIST_E_INVALID, "clipping: null argument");
  if (!aligned8(record)) return lib_fail(MIST_E_INVALID, "clipping: record not aligned to 8");
  if (const mist_status st = like(g, out)) return st;
  if (const mist_status st = written(out)) return st;
  if (const mist_status st = on_device(g, "clipping")) return st;
  if (!g->n_pieces) return MIST_OK;
  mist::with_types(g->type, out->type, [&](auto x, auto y) {
    using G = typename decltype(x)::type;
    using O = typename decltype(y)::type;
    hipLaunchKernelGGL((k_clip<G, O>), grid_of(g->n_pieces * kClipBlocks), dim3(kThreads), 0, (hipStream_t)stream, g->list, out->list,
                       g->n_pieces, record);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "clipping");
}

mist_status mist_adam_step(const mist_tensors* p, const mist_tensors* m, const mist_tensors* v, const mist_tensors* g,
                           const mist_tensors* w, const mist_step_record* record, const mist_adam_desc* a, void* stream) {
  if (!p || !m || !v || !g || !record || !a) return lib_fail(MIST_E_INVALID, "Adam step: null argument");
  if (!aligned8(record)) return lib_fail(MIST_E_INVALID, "Adam step: record not aligned to 8");
  if (p->type != MIST_F32 || m->type != MIST_F32 || v->type != MIST_F32)
    return lib_fail(MIST_E_INVALID, "Adam step: master weights, m and v must be MIST_F32");
  if (p == m || p == v || m == v || p == g || m == g || v == g || (w && (w == p || w == m || w == v || w == g)))
    return lib_fail(MIST_E_INVALID, "Adam step: the lists must be distinct");
  if (!(a->lr >= 0.0 && std::isfinite((float)a->lr)) || !(a->beta1 >= 0.0 && a->beta1 < 1.0) || !(a->beta2 >= 0.0 && a->beta2 < 1.0) ||
      !((float)a->eps > 0.0f && std::isfinite((float)a->eps)) || !(a->weight_decay >= 0.0 && std::isfinite((float)a->weight_decay)))
    return lib_fail(MIST_E_INVALID, "Adam step: lr, beta, eps or weight_decay out of range");
  for (const mist_tensors* t : {p, m, v, w ? w : g})
    if (const mist_status st = like(g, t)) return st;
  for (const mist_tensors* t : {p, m, v, w})
    if (const mist_status st = written(t)) return st;
  if (const mist_status st = on_device(g, "Adam step")) return st;
  if (!g->n_pieces) return MIST_OK;
  AdamArgs k{p->list, m->list, v->list, g->list, w ? w->list : List{}, a->beta1, a->beta2,
             decay_of(a->beta1), decay_of(a->beta2), (float)(1.0 - a->beta1), (float)(1.0 - a->beta2),
             (float)a->lr, (float)a->weight_decay, (float)a->eps};
  const dim3 grid = grid_of(g->n_pieces), block(kThreads);
  mist::with_types(g->type, w ? w->type : MIST_F32, [&](auto x, auto y) {
    using G = typename decltype(x)::type;
    using W = typename decltype(y)::type;
    if (w) hipLaunchKernelGGL((k_adam<G, W, true>), grid, block, 0, (hipStream_t)stream, k, g->n_pieces, record);
    else if constexpr (sizeof(W) == 4) hipLaunchKernelGGL((k_adam<G, W, false>), grid, block, 0, (hipStream_t)stream, k, g->n_pieces, record);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "Adam step");
}

}  // extern "C"
