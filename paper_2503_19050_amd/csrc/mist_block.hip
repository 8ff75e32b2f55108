// The residual around a block, the norms before and after it, and their gradients.
//
// A row is held in the registers of its block, eight consecutive columns a thread, from its one reading to its one writing;
// the norms' sums go over the waves through shared memory.  A block takes rows of a part in turn and keeps the weights,
// and in the backward pass the weights' gradients, of its columns in registers.  The parts' gradients are joined by a second launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "mist_ops.h"

using mist::Float8;
using mist::hip_failed;
using mist::lib_fail;
using mist::load8;
using mist::store8;
using mist::wave_sum;

namespace {

constexpr int kMostWaves = 16;
constexpr int64_t kMostTokens = (int64_t)1 << 30;
constexpr int64_t kMostBlocks = 4096;  // of the forward pass; they take rows in turn
constexpr int64_t kParts = 1024;       // of the backward pass, about
constexpr int64_t kPartRows = 8;       // a part has at least, where there are as many
constexpr int kSlots = 5;              // gradients summed over tokens
constexpr int kJoinThreads = 1024;

struct BlockArgs {
  int64_t n, seq, hidden, x_stride, block_stride, y_stride, h_stride, gate_stride;
  int32_t layer, weight_type;
  float eps, res_scale, block_scale, inv_hidden;
  const void *weight, *bias, *post_weight, *post_bias, *gate;
};

__device__ __forceinline__ Float8 load_weight(const void* p, int32_t type, int64_t col, int64_t left) {
  if (type == MIST_F32) return load8((const float*)p + col, left);
  if (type == MIST_BF16) return load8((const __bf16*)p + col, left);
  return load8((const _Float16*)p + col, left);
}
__device__ __forceinline__ void store_weight(void* p, int32_t type, int64_t at, float x, int32_t accumulate) {
  if (type == MIST_F32) ((float*)p)[at] = accumulate ? ((float*)p)[at] + x : x;
  else if (type == MIST_BF16) ((__bf16*)p)[at] = (__bf16)(accumulate ? (float)((__bf16*)p)[at] + x : x);
  else ((_Float16*)p)[at] = (_Float16)(accumulate ? (float)((_Float16*)p)[at] + x : x);
}

__device__ __forceinline__ float sum8(Float8 x) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }
__device__ __forceinline__ Float8 masked(Float8 x, int64_t left) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k >= left) x[k] = 0.0f;
  return x;
}

// Sums over the block.  Two buffers in turn: a wave writes one only after every wave has read its last values.
struct Join {
  float2* part;  // [2][kMostWaves]
  int waves, turn;
  __device__ __forceinline__ float2 sum(float a, float b) {
    a = wave_sum(a);
    b = wave_sum(b);
    if (waves == 1) return float2{a, b};
    float2* p = part + turn * kMostWaves;
    turn ^= 1;
    if (threadIdx.x % 64 == 0) p[threadIdx.x / 64] = float2{a, b};
    __syncthreads();
    float2 s = p[0];
    for (int k = 1; k < waves; ++k) s.x += p[k].x, s.y += p[k].y;
    return s;
  }
};

struct Moments {
  float mean, r;
};
// The variance is of the distances from the mean, not a difference of squares.
template <int U>
__device__ __forceinline__ Moments moments(const BlockArgs& a, Join& join, const Float8* x, const int* left) {
  float mean = 0.0f, s = 0.0f;
  if (a.layer) {
#pragma unroll
    for (int u = 0; u < U; ++u) s += sum8(x[u]);
    mean = join.sum(s, 0.0f).x * a.inv_hidden;
    s = 0.0f;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Float8 d = masked(x[u] - mean, left[u]);
    s += sum8(d * d);
  }
  return Moments{mean, 1.0f / sqrtf(join.sum(s, 0.0f).x * a.inv_hidden + a.eps)};
}

template <int U>
struct Columns {
  int col[U], left[U];
  __device__ __forceinline__ explicit Columns(const BlockArgs& a) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      col[u] = (u * (int)blockDim.x + (int)threadIdx.x) * 8;
      left[u] = (int)a.hidden - col[u];  // none where <= 0
    }
  }
};
template <int U, class F>
__device__ __forceinline__ void each(F&& f) {
#pragma unroll
  for (int u = 0; u < U; ++u) f(u);
}

template <class A, class R, int U>
__global__ __launch_bounds__(kMostWaves * 64) void k_forward(BlockArgs a, const R* x, const A* block, R* y, A* h, float* stats) {
  __shared__ float2 part[2 * kMostWaves];
  Join join{part, (int)blockDim.x / 64, 0};
  const Columns<U> c(a);
  Float8 w[U] = {}, wb[U] = {}, pw[U] = {}, pb[U] = {}, gate[U];
  each<U>([&](int u) {
    if (a.weight) w[u] = load_weight(a.weight, a.weight_type, c.col[u], c.left[u]);
    if (a.bias) wb[u] = load_weight(a.bias, a.weight_type, c.col[u], c.left[u]);
    if (a.post_weight) pw[u] = load_weight(a.post_weight, a.weight_type, c.col[u], c.left[u]);
    if (a.post_bias) pb[u] = load_weight(a.post_bias, a.weight_type, c.col[u], c.left[u]);
    gate[u] = 1.0f;
    if (a.gate && !a.gate_stride) gate[u] = load_weight(a.gate, a.weight_type, c.col[u], c.left[u]);
  });
  for (int64_t t = blockIdx.x; t < a.n; t += gridDim.x) {
    Float8 v[U];
    each<U>([&](int u) { v[u] = load8(x + t * a.x_stride + c.col[u], c.left[u]); });
    Moments before{0.0f, 1.0f}, after{0.0f, 1.0f};
    if (block) {
      Float8 b[U];
      each<U>([&](int u) {
        b[u] = load8(block + t * a.block_stride + c.col[u], c.left[u]);
        if (a.gate_stride) gate[u] = load_weight(a.gate, a.weight_type, t / a.seq * a.gate_stride + c.col[u], c.left[u]);
      });
      if (a.post_weight) {
        before = moments<U>(a, join, b, c.left);
        each<U>([&](int u) { b[u] = (b[u] - before.mean) * before.r * pw[u] + pb[u]; });
      }
      each<U>([&](int u) {
        v[u] = a.res_scale * v[u] + a.block_scale * (b[u] * gate[u]);
        store8(y + t * a.y_stride + c.col[u], c.left[u], v[u]);
        // the norm is of y as it is stored
        v[u] = masked(__builtin_convertvector(__builtin_convertvector(v[u], typename mist::Vec<R, 8>::type), Float8), c.left[u]);
      });
    }
    if (h) {
      after = moments<U>(a, join, v, c.left);
      each<U>([&](int u) { store8(h + t * a.h_stride + c.col[u], c.left[u], (v[u] - after.mean) * after.r * w[u] + wb[u]); });
    }
    if (threadIdx.x == 0) *(float4*)(stats + t * 4) = float4{before.mean, before.r, after.mean, after.r};
  }
}

// How the backward pass cuts the tokens: parts of `seqs` whole sequences each, or (seqs = 1) `pieces` parts a sequence of `rows`
// tokens.  Without a gate of their own the sequences are one.
struct Parts {
  int64_t batch, seq, seqs, pieces, rows, n;
};

struct BackArgs {
  BlockArgs a;
  Parts parts;
  int64_t dh_stride, dy_stride, dx_stride, dblock_stride, dgate_stride;
  float* slot[kSlots];  // [parts][hidden] each: dweight, dbias, dpost_weight, dpost_bias, dgate; null: not wanted
  void* dgate;          // where whole sequences are a part's: its gradient is written at their end
  int32_t accumulate;
};

template <class A, class R, int U, bool MORE>
__global__ __launch_bounds__(kMostWaves * 64) void k_backward(BackArgs k, const R* y, const A* block, const float* stats, const A* dh, const R* dy,
                                                              R* dx, A* dblock) {
  __shared__ float2 shared[2 * kMostWaves];
  const BlockArgs& a = k.a;
  Join join{shared, (int)blockDim.x / 64, 0};
  const Columns<U> c(a);
  Float8 w[U] = {}, pw[U] = {}, pb[U] = {}, gate[U];
  Float8 sw[U] = {}, sb[U] = {}, spw[U] = {}, spb[U] = {}, sg[U] = {};
  each<U>([&](int u) {
    if (a.weight) w[u] = load_weight(a.weight, a.weight_type, c.col[u], c.left[u]);
    if (MORE && a.post_weight) pw[u] = load_weight(a.post_weight, a.weight_type, c.col[u], c.left[u]);
    if (MORE && a.post_bias) pb[u] = load_weight(a.post_bias, a.weight_type, c.col[u], c.left[u]);
    gate[u] = 1.0f;
    if (MORE && a.gate && !a.gate_stride) gate[u] = load_weight(a.gate, a.weight_type, c.col[u], c.left[u]);
  });
  const int64_t part = blockIdx.x, first = part / k.parts.pieces * k.parts.seqs, row0 = part % k.parts.pieces * k.parts.rows;
  for (int64_t s = first; s < min(first + k.parts.seqs, k.parts.batch); ++s) {
    if (MORE && a.gate_stride) each<U>([&](int u) { gate[u] = load_weight(a.gate, a.weight_type, s * a.gate_stride + c.col[u], c.left[u]); });
    for (int64_t r = row0; r < min(row0 + k.parts.rows, k.parts.seq); ++r) {
      const int64_t t = s * k.parts.seq + r;
      const float4 st = *(const float4*)(stats + t * 4);
      Float8 d[U], b[U];
      each<U>([&](int u) { d[u] = dy ? load8(dy + t * k.dy_stride + c.col[u], c.left[u]) : Float8{}; });
      if (block) each<U>([&](int u) { b[u] = load8(block + t * a.block_stride + c.col[u], c.left[u]); });
      if (dh) {
        Float8 g[U], n[U];
        float p = 0.0f, q = 0.0f;
        each<U>([&](int u) {
          g[u] = load8(dh + t * k.dh_stride + c.col[u], c.left[u]);
          n[u] = (load8(y + t * a.y_stride + c.col[u], c.left[u]) - st.z) * st.w;
          sb[u] += g[u];
          sw[u] += g[u] * n[u];
          g[u] *= w[u];
          p += sum8(g[u]);
          q += sum8(g[u] * n[u]);
        });
        const float2 m = join.sum(p, q);
        const float mean = a.layer ? m.x * a.inv_hidden : 0.0f, along = m.y * a.inv_hidden;
        each<U>([&](int u) { d[u] += st.w * (g[u] - mean - n[u] * along); });
      }
      if (dx) each<U>([&](int u) { store8(dx + t * k.dx_stride + c.col[u], c.left[u], a.res_scale * d[u]); });
      if (block) {
        each<U>([&](int u) { d[u] *= a.block_scale; });
        if (MORE) {
          if (a.post_weight) {
            float p = 0.0f, q = 0.0f;
            each<U>([&](int u) {
              b[u] = masked((b[u] - st.x) * st.y, c.left[u]);
              sg[u] += d[u] * (b[u] * pw[u] + pb[u]);
              d[u] = masked(d[u] * gate[u], c.left[u]);
              spb[u] += d[u];
              spw[u] += d[u] * b[u];
              d[u] *= pw[u];
              p += sum8(d[u]);
              q += sum8(d[u] * b[u]);
            });
            const float2 m = join.sum(p, q);
            const float mean = a.layer ? m.x * a.inv_hidden : 0.0f, along = m.y * a.inv_hidden;
            each<U>([&](int u) { d[u] = st.y * (d[u] - mean - b[u] * along); });
          } else {
            each<U>([&](int u) {
              sg[u] += d[u] * b[u];
              d[u] *= gate[u];
            });
          }
        }
        if (dblock) each<U>([&](int u) { store8(dblock + t * k.dblock_stride + c.col[u], c.left[u], d[u]); });
      }
    }
    if (MORE && k.dgate) {
      each<U>([&](int u) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < c.left[u]) store_weight(k.dgate, a.weight_type, s * k.dgate_stride + c.col[u] + i, sg[u][i], k.accumulate);
        sg[u] = 0.0f;
      });
    }
  }
  each<U>([&](int u) {
    const int64_t at = part * a.hidden + c.col[u];
    if (k.slot[0]) store8(k.slot[0] + at, c.left[u], sw[u]);
    if (k.slot[1]) store8(k.slot[1] + at, c.left[u], sb[u]);
    if (MORE && k.slot[2]) store8(k.slot[2] + at, c.left[u], spw[u]);
    if (MORE && k.slot[3]) store8(k.slot[3] + at, c.left[u], spb[u]);
    if (MORE && k.slot[4]) store8(k.slot[4] + at, c.left[u], sg[u]);
  });
}

// The parts' sums, in order: parts[i * count .. ) of `count` rows give row i of out.  One wave's 64 columns a block, 16 shares of the rows.
struct JoinJob {
  const float* part;
  void* out;
  int64_t count, rows, stride;  // parts a row of out, rows of out and their stride
};
struct JoinArgs {
  JoinJob job[kSlots];
  int64_t hidden;
  int32_t type, accumulate;
};
__global__ __launch_bounds__(kJoinThreads) void k_join_parts(JoinArgs k) {
  constexpr int kShares = kJoinThreads / 64;
  __shared__ float share[kShares][64];
  const JoinJob j = k.job[blockIdx.y];
  const int lane = threadIdx.x % 64, mine = threadIdx.x / 64;
  const int64_t columns = (k.hidden + 63) / 64, per = (j.count + kShares - 1) / kShares;
  for (int64_t i = blockIdx.x; i < columns * j.rows; i += gridDim.x) {
    const int64_t row = i / columns, col = i % columns * 64 + lane;
    float s = 0.0f;
    if (col < k.hidden) {
      const float* p = j.part + (row * j.count) * k.hidden + col;
      const int64_t end = min(j.count, (mine + 1) * per);
#pragma unroll 8
      for (int64_t r = mine * per; r < end; ++r) s += p[r * k.hidden];
    }
    __syncthreads();
    share[mine][lane] = s;
    __syncthreads();
    if (mine == 0 && col < k.hidden) {
      for (int w = 1; w < kShares; ++w) s += share[w][lane];
      store_weight(j.out, k.type, row * j.stride + col, s, k.accumulate);
    }
  }
}

mist_status check(const mist_block_desc* d) {
  if (!d) return lib_fail(MIST_E_INVALID, "block norm: null descriptor");
  if (d->batch < 0 || d->seq < 0 || d->batch > INT32_MAX || d->seq > INT32_MAX || (d->batch && d->seq >= kMostTokens / d->batch + (kMostTokens % d->batch != 0)))
    return lib_fail(MIST_E_INVALID, "block norm: batch and seq must be >= 0 with fewer than 2^30 tokens");
  if (d->hidden < 1 || d->hidden > MIST_BLOCK_MAX_HIDDEN) return lib_fail(MIST_E_INVALID, "block norm: hidden must be in 1..16384");
  if (d->kind != MIST_BLOCK_RMS && d->kind != MIST_BLOCK_LAYER) return lib_fail(MIST_E_INVALID, "block norm: unknown kind");
  if (!mist::type_ok(d->type) || !mist::type_ok(d->res_type) || !mist::type_ok(d->weight_type))
    return lib_fail(MIST_E_INVALID, "block norm: unknown element type");
  if (d->res_type != d->type && d->res_type != MIST_F32)
    return lib_fail(MIST_E_INVALID, "block norm: the residual must be of the block's type or fp32");
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps) || !std::isfinite(d->res_scale) || !std::isfinite(d->block_scale))
    return lib_fail(MIST_E_INVALID, "block norm: eps must be >= 0, scales finite");
  for (int64_t x : {d->x_stride, d->block_stride, d->y_stride, d->h_stride, d->gate_stride})
    if (!mist::stride_ok(x)) return lib_fail(MIST_E_INVALID, "block norm: strides must be in 0..2^40");
  return MIST_OK;
}

// A tensor of the call, for the checks of alignment and of what shares memory.
struct Tensor {
  const void* p;
  int64_t stride;
  int32_t type;
  bool out;
  const void* may_be[2];  // inputs whose place it may take
};

mist_status check_tensors(const mist_block_desc* d, std::initializer_list<Tensor> ts) {
  const int64_t n = d->batch * d->seq;
  for (const Tensor& t : ts) {
    const int64_t bytes = mist::type_bytes(t.type);
    if (!mist::is_aligned(t.p, (size_t)bytes)) return lib_fail(MIST_E_INVALID, "block norm: a buffer is not aligned to its elements");
    if (!t.p || !t.out) continue;
    if (n > 1 && t.stride < d->hidden) return lib_fail(MIST_E_INVALID, "block norm: rows of an output overlap");
    for (const Tensor& o : ts) {
      if (&o == &t || !o.p) continue;
      const bool same = o.p == t.p && (n == 1 || o.stride == t.stride) && o.type == t.type && (o.p == t.may_be[0] || o.p == t.may_be[1]) && !o.out;
      if (!same && mist::overlap(mist::Rows{t.p, n, t.stride, d->hidden, bytes}, mist::Rows{o.p, n, o.stride, d->hidden, mist::type_bytes(o.type)}))
        return lib_fail(MIST_E_INVALID, "block norm: an output overlaps another tensor");
    }
  }
  return MIST_OK;
}

BlockArgs args(const mist_block_desc* d, const void* weight, const void* bias, const void* post_weight, const void* post_bias, const void* gate) {
  return BlockArgs{d->batch * d->seq, std::max<int64_t>(d->seq, 1), d->hidden, d->x_stride, d->block_stride, d->y_stride, d->h_stride,
                   gate && d->batch > 1 ? d->gate_stride : 0, d->kind == MIST_BLOCK_LAYER, d->weight_type, d->eps, d->res_scale, d->block_scale,
                   (float)(1.0 / (double)d->hidden), weight, bias, post_weight, post_bias, gate};
}

bool weights_ok(const mist_block_desc* d, std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!mist::is_aligned(p, (size_t)mist::type_bytes(d->weight_type))) return false;
  return true;
}

int units(int64_t hidden) { return hidden > kMostWaves * 512 ? 2 : 1; }
unsigned threads(int64_t hidden) { return (unsigned)((hidden + units(hidden) * 512 - 1) / (units(hidden) * 512) * 64); }

// f(activation type, residual type, columns a thread / 8)
template <class F>
void with_kernel(const mist_block_desc* d, F&& f) {
  mist::with_type(d->type, [&](auto x) {
    using A = typename decltype(x)::type;
    auto run = [&](auto r) {
      using R = typename decltype(r)::type;
      if (units(d->hidden) == 2) f(A{}, R{}, std::integral_constant<int, 2>{});
      else f(A{}, R{}, std::integral_constant<int, 1>{});
    };
    if (d->res_type == d->type) run(x);
    else run(mist::Elem<MIST_F32>{});
  });
}

mist_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, what);
}

Parts parts_of(const mist_block_desc* d, bool by_sequence) {
  Parts p{};
  p.batch = by_sequence ? d->batch : 1;
  p.seq = by_sequence ? d->seq : d->batch * d->seq;
  if (!p.batch || !p.seq) return p;
  p.pieces = std::clamp<int64_t>(kParts / p.batch, 1, (p.seq + kPartRows - 1) / kPartRows);
  p.rows = (p.seq + p.pieces - 1) / p.pieces;
  p.pieces = (p.seq + p.rows - 1) / p.rows;
  p.seqs = p.pieces > 1 ? 1 : std::max<int64_t>((p.batch + kParts - 1) / kParts, std::min<int64_t>((kPartRows + p.seq - 1) / p.seq, p.batch));
  p.n = (p.batch + p.seqs - 1) / p.seqs * p.pieces;
  return p;
}

struct Plan {
  Parts parts;
  size_t bytes;
  bool wanted[kSlots], direct;  // direct: gates' gradients need no parts
};
Plan plan_of(const mist_block_desc* d, const mist_block_grads* g) {
  Plan p{};
  const bool by_sequence = d->gate_stride && d->batch > 1;
  p.parts = parts_of(d, by_sequence);
  const void* out[kSlots] = {g->dweight, g->dbias, g->dpost_weight, g->dpost_bias, g->dgate};
  p.direct = by_sequence && p.parts.pieces == 1;
  for (int i = 0; i < kSlots; ++i) {
    p.wanted[i] = out[i] && !(i == 4 && p.direct);
    if (p.wanted[i]) p.bytes += (size_t)p.parts.n * d->hidden * 4 + 256;
  }
  return p;
}

mist_status check_grads(const mist_block_desc* d, const mist_block_grads* g) {
  if (const mist_status st = check(d)) return st;
  if (!g) return lib_fail(MIST_E_INVALID, "block norm's gradient: null descriptor");
  if (g->accumulate != 0 && g->accumulate != 1) return lib_fail(MIST_E_INVALID, "block norm's gradient: accumulate must be 0 or 1");
  for (int64_t x : {g->dh_stride, g->dy_stride, g->dx_stride, g->dblock_stride, g->dgate_stride})
    if (!mist::stride_ok(x)) return lib_fail(MIST_E_INVALID, "block norm: strides must be in 0..2^40");
  if (g->dgate && d->gate_stride && d->batch > 1 && g->dgate_stride < d->hidden)
    return lib_fail(MIST_E_INVALID, "block norm's gradient: rows of the gates' gradient overlap");
  return MIST_OK;
}

}  // namespace

extern "C" {

mist_status mist_block_forward(const mist_block_desc* d, const void* x, const void* block, const void* weight, const void* bias,
                               const void* post_weight, const void* post_bias, const void* gate, void* y, void* h, float* stats, void* stream) {
  if (const mist_status st = check(d)) return st;
  if ((bias && !weight) || (post_bias && !post_weight)) return lib_fail(MIST_E_INVALID, "block norm: a bias without its weight");
  const BlockArgs a = args(d, weight, bias, post_weight, post_bias, gate);
  if (a.n == 0) return MIST_OK;
  if (!block && (y || post_weight || gate || d->res_scale != 1.0f)) return lib_fail(MIST_E_INVALID, "block norm: without a block y is x");
  if (!block && !weight) return lib_fail(MIST_E_INVALID, "block norm: neither a block nor a norm");
  if (!x || !stats || (block && !y) || (weight && !h) || (h && !weight)) return lib_fail(MIST_E_INVALID, "block norm: null buffer, or h without its weight");
  if (!mist::is_aligned(stats, 16) || !weights_ok(d, {weight, bias, post_weight, post_bias, gate}))
    return lib_fail(MIST_E_INVALID, "block norm: a buffer is not aligned to its elements, or stats to 16");
  if (const mist_status st = check_tensors(d, {{x, d->x_stride, d->res_type, false, {}}, {block, d->block_stride, d->type, false, {}},
                                               {y, d->y_stride, d->res_type, true, {x, block}}, {h, d->h_stride, d->type, true, {}}}))
    return st;
  with_kernel(d, [&](auto e, auto f, auto u) {
    using A = decltype(e);
    using R = decltype(f);
    hipLaunchKernelGGL((k_forward<A, R, u.value>), dim3((unsigned)std::min<int64_t>(a.n, kMostBlocks)), dim3(threads(d->hidden)), 0, (hipStream_t)stream, a,
                       (const R*)x, (const A*)block, (R*)y, (A*)h, stats);
  });
  return launched("block norm");
}

mist_status mist_block_workspace(const mist_block_desc* d, const mist_block_grads* g, size_t* bytes) {
  if (!bytes) return lib_fail(MIST_E_INVALID, "block norm's gradient: null argument");
  if (const mist_status st = check_grads(d, g)) return st;
  *bytes = plan_of(d, g).bytes;
  return MIST_OK;
}

mist_status mist_block_backward(const mist_block_desc* d, const void* y, const void* block, const float* stats, const void* weight,
                                const void* post_weight, const void* post_bias, const void* gate, const mist_block_grads* g, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (const mist_status st = check_grads(d, g)) return st;
  const bool any = d->batch && d->seq;
  if (any && !block && (post_weight || gate || g->dblock || d->res_scale != 1.0f)) return lib_fail(MIST_E_INVALID, "block norm's gradient: without a block y is x");
  if (post_bias && !post_weight) return lib_fail(MIST_E_INVALID, "block norm's gradient: a bias without its weight");
  if (any && ((!weight && (g->dweight || g->dbias)) || (!post_weight && (g->dpost_weight || g->dpost_bias)) || (!gate && g->dgate)))
    return lib_fail(MIST_E_INVALID, "block norm's gradient: of a weight, bias or gate that is not there");
  BlockArgs a = args(d, weight, nullptr, post_weight, post_bias, gate);
  Plan p = plan_of(d, g);
  if (!any && g->accumulate) return MIST_OK;
  if (any && (!stats || (weight && (!y || !g->dh)) || (!weight && g->dh) || (!g->dh && !g->dy)))
    return lib_fail(MIST_E_INVALID, "block norm's gradient: null buffer, or dh without its weight");
  if (!mist::is_aligned(stats, 16) || !mist::is_aligned(workspace, 256) ||
      !weights_ok(d, {weight, post_weight, post_bias, gate, g->dweight, g->dbias, g->dpost_weight, g->dpost_bias, g->dgate}))
    return lib_fail(MIST_E_INVALID, "block norm's gradient: a buffer is not aligned to its elements, stats to 16 or the workspace to 256");
  if (p.bytes && !workspace) return lib_fail(MIST_E_INVALID, "block norm's gradient: null workspace");
  if (workspace_bytes < p.bytes) return lib_fail(MIST_E_RANGE, "block norm's gradient: workspace too small");
  if (const mist_status st = check_tensors(d, {{y, d->y_stride, d->res_type, false, {}}, {block, d->block_stride, d->type, false, {}},
                                               {g->dh, g->dh_stride, d->type, false, {}}, {g->dy, g->dy_stride, d->res_type, false, {}},
                                               {g->dx, g->dx_stride, d->res_type, true, {g->dy, nullptr}},
                                               {g->dblock, g->dblock_stride, d->type, true, {g->dh, block}}}))
    return st;
  BackArgs k{};
  k.a = a;
  k.parts = p.parts;
  k.dh_stride = g->dh_stride, k.dy_stride = g->dy_stride, k.dx_stride = g->dx_stride, k.dblock_stride = g->dblock_stride;
  k.dgate_stride = g->dgate_stride;
  k.dgate = p.direct ? g->dgate : nullptr;
  k.accumulate = g->accumulate;
  JoinArgs j{};
  j.hidden = d->hidden, j.type = d->weight_type, j.accumulate = g->accumulate;
  void* out[kSlots] = {g->dweight, g->dbias, g->dpost_weight, g->dpost_bias, g->dgate};
  int jobs = 0;
  char* ws = (char*)workspace;
  int64_t most = 0;
  for (int i = 0; i < kSlots; ++i) {
    if (!p.wanted[i]) continue;
    k.slot[i] = (float*)ws;
    const bool gates = i == 4 && a.gate_stride;
    j.job[jobs++] = JoinJob{k.slot[i], out[i], gates ? p.parts.pieces : p.parts.n, gates ? d->batch : 1, gates ? g->dgate_stride : 0};
    most = std::max(most, (d->hidden + 63) / 64 * j.job[jobs - 1].rows);
    ws += ((size_t)p.parts.n * d->hidden * 4 + 255) / 256 * 256;
  }
  const hipStream_t st = (hipStream_t)stream;
  if (any) {
    with_kernel(d, [&](auto e, auto f, auto u) {
      using A = decltype(e);
      using R = decltype(f);
      const auto kernel = post_weight || gate ? k_backward<A, R, u.value, true> : k_backward<A, R, u.value, false>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)p.parts.n), dim3(threads(d->hidden)), 0, st, k, (const R*)y, (const A*)block, stats, (const A*)g->dh,
                         (const R*)g->dy, (R*)g->dx, (A*)g->dblock);
    });
  }
  if (jobs) hipLaunchKernelGGL(k_join_parts, dim3((unsigned)std::min<int64_t>(most, 65536), (unsigned)jobs), dim3(kJoinThreads), 0, st, j);
  return launched("block norm's gradient");
}

}  // extern "C"
