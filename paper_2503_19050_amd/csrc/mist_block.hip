// The residual around a block, the norms before and after it, and their gradients.
//
// A row is held in the registers of its block, eight consecutive columns a thread, from its one reading to its one writing;
// the norms' sums go over the waves through shared memory.  A block takes rows of a part in turn and keeps the weights,
// and in the backward pass the weights' gradients, of its columns in registers.  The parts' gradients are joined by a second launch.
// Bound by memory; what it takes is enough rows in flight, so the next row is read ahead and registers decide.  Measured on one MI355X, where
// a large copy reads and writes 4.9 TB/s, forward and backward: 65536 x 2560 bf16 268 and 364 us (5.0 and 4.6 TB/s), 65536 x 5120
// 536 and 675 (5.0, 5.0), 32768 x 8192 398-441 and 528 (4.9-5.4, 5.1), 65536 x 512 45 and 82 (5.9, 4.1), 65536 x 2559 326 and 541
// (4.1, 3.1), 32768 x 4096 with a norm before and gates by sequence 231 and 324 (4.7, 5.0).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mist_ops.h"

using mist::Eight;
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
constexpr int64_t kPartRows = 4;       // a part has at least, where there are as many
constexpr int64_t kMostRows = 512;     // added one after another in fp32, as long as kMostParts parts are enough
constexpr int64_t kMostParts = 4096;
constexpr int kSlots = 5;              // gradients summed over tokens
constexpr int kJoinThreads = 1024;

struct BlockArgs {
  int64_t n, seq, hidden, x_stride, block_stride, y_stride, h_stride, gate_stride;
  int32_t layer, weight_type;
  float eps, res_scale, block_scale, inv_hidden;
  const void *weight, *bias, *post_weight, *post_bias, *gate;
};

template <bool WHOLE>
__device__ __forceinline__ Float8 load_weight(const void* p, int32_t type, int64_t row, const Eight<WHOLE>& c) {
  if (type == MIST_F32) return load8((const float*)p + row, c);
  if (type == MIST_BF16) return load8((const __bf16*)p + row, c);
  return load8((const _Float16*)p + row, c);
}
__device__ __forceinline__ void store_weight(void* p, int32_t type, int64_t at, float x, int32_t accumulate) {
  if (type == MIST_F32) ((float*)p)[at] = accumulate ? ((float*)p)[at] + x : x;
  else if (type == MIST_BF16) ((__bf16*)p)[at] = (__bf16)(accumulate ? (float)((__bf16*)p)[at] + x : x);
  else ((_Float16*)p)[at] = (_Float16)(accumulate ? (float)((_Float16*)p)[at] + x : x);
}

__device__ __forceinline__ float sum8(Float8 x) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }
template <bool WHOLE>
__device__ __forceinline__ Float8 masked(Float8 x, const Eight<WHOLE>& c) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (!WHOLE && k >= c.left) x[k] = 0.0f;
  return x;
}

// The sum over the rows that lie beside each other in a wave.
template <int L>
__device__ __forceinline__ Float8 over_rows(Float8 x) {
  if (L < 64) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (L == 16) x[k] = mist::join_pairs_of_16(x[k], [](float p, float q) { return p + q; });
      x[k] = mist::join_pairs_of_32(x[k], [](float p, float q) { return p + q; });
    }
  }
  return x;
}

// Sums over a row's lanes: L of a wave (16 or 32: rows of up to 128 or 256 columns lie beside each other in it), or all waves of the block.
// Waves meet in two places in turn: one writes a place only after every wave has read its last values.
template <int L>
struct Join {
  float2* part;   // [2][kMostWaves]
  float2* count;  // [kMostWaves]: columns of each wave, and one over them
  int waves, turn;
  template <int U>
  __device__ __forceinline__ void count_columns(const BlockArgs& a) {
    if (!a.layer || L < 64 || waves == 1) return;
    if ((int)threadIdx.x < waves) {
      int n = 0;
      for (int u = 0; u < U; ++u) n += min(max((int)a.hidden - (u * (int)blockDim.x + (int)threadIdx.x * 64) * 8, 0), 512);
      count[threadIdx.x] = float2{(float)n, 1.0f / (float)n};
    }
    __syncthreads();
  }
  __device__ __forceinline__ const float2* meet(float a, float b) {
    float2* p = part + turn * kMostWaves;
    turn ^= 1;
    if (threadIdx.x % 64 == 0) p[threadIdx.x / 64] = float2{a, b};
    __syncthreads();
    return p;
  }
  __device__ __forceinline__ float2 sum(float a, float b) {
    a = wave_sum<L>(a);
    b = wave_sum<L>(b);
    if (L < 64 || waves == 1) return float2{a, b};
    const float2 s = of_waves(meet(a, b));
    return float2{wave_sum<16>(s.x), wave_sum<16>(s.y)};
  }
  // a wave's value for each of 16 lanes, in every 16 lanes; zeros past the last wave
  __device__ __forceinline__ float2 of_waves(const float2* p) const {
    const int k = (int)threadIdx.x % 16;
    return k < waves ? p[k] : float2{0.0f, 0.0f};
  }
};

// A thread's columns.
template <int U, int L, bool WHOLE>
struct Columns {
  Eight<WHOLE> e[U];
  __device__ __forceinline__ explicit Columns(const BlockArgs& a) {
    const int lane = L < 64 ? (int)threadIdx.x % L : (int)threadIdx.x, all = L < 64 ? L : (int)blockDim.x;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      e[u] = Eight<WHOLE>((u * all + lane) * 8, (int)a.hidden);
    }
  }
};
template <int U, class F>
__device__ __forceinline__ void each(F&& f) {
#pragma unroll
  for (int u = 0; u < U; ++u) f(u);
}

// A thread's values of a weight, `none` without one: in registers, or read where they are used by rows of more than 8192 columns.
template <int U, int L, bool WHOLE>
struct Weights {
  const void* p;
  const Columns<U, L, WHOLE>& c;
  int32_t type;
  float none;
  Float8 held;
  __device__ __forceinline__ Weights(const BlockArgs& a, const void* weight, const Columns<U, L, WHOLE>& columns, float without)
      : p(weight), c(columns), type(a.weight_type), none(without) {
    if (U == 1) held = read(0);
  }
  __device__ __forceinline__ Float8 read(int u) const { return p ? load_weight(p, type, 0, c.e[u]) : Float8(none); }
  __device__ __forceinline__ Float8 operator()(int u) const { return U == 1 ? held : read(u); }
};

struct Moments {
  float mean, r;
};
// The variance is of the distances from the mean, not a difference of squares: of each wave's values from that wave's mean, and of
// the waves' means, so that the waves meet once.
template <int U, int L, bool WHOLE>
__device__ __forceinline__ Moments moments(const BlockArgs& a, Join<L>& join, const Columns<U, L, WHOLE>& c, const Float8* x) {
  float s = 0.0f, q = 0.0f;
  if (!a.layer) {
    each<U>([&](int u) { s += sum8(x[u] * x[u]); });
    return Moments{0.0f, 1.0f / sqrtf(join.sum(s, 0.0f).x * a.inv_hidden + a.eps)};
  }
  each<U>([&](int u) { s += sum8(x[u]); });
  s = wave_sum<L>(s);
  const bool alone = L < 64 || join.waves == 1;
  const float near = s * (alone ? a.inv_hidden : join.count[threadIdx.x / 64].y);
  each<U>([&](int u) {
    const Float8 d = masked(x[u] - near, c.e[u]);
    q += sum8(d * d);
  });
  q = wave_sum<L>(q);
  float mean = near;
  if (!alone) {
    const float2 p = join.of_waves(join.meet(s, q)), n = join.of_waves(join.count);
    mean = wave_sum<16>(p.x) * a.inv_hidden;
    const float d = p.x * n.y - mean;
    q = wave_sum<16>(fmaf(n.x * d, d, p.y));
  }
  return Moments{mean, 1.0f / sqrtf(q * a.inv_hidden + a.eps)};
}

// Rows of one reading, before they are converted.
template <class A, class R, int U>
struct Input {
  mist::Raw8<R> x[U];
  mist::Raw8<A> b[U];
};

// Waves of a kernel's largest block.  Kernels for rows of up to ten waves (eight with a norm before or a gate) are built apart from those
// for wider ones, which have 128 registers at most; rows beside each other are one wave's.
constexpr int narrow_waves(bool more) { return more ? 8 : 10; }
constexpr int most_waves(int u, int l, bool wide, bool more) { return l < 64 ? 1 : u == 1 && !wide ? narrow_waves(more) : kMostWaves; }

// The next row is read before the sums of this one are waited for, where the registers are there.
// MORE: a norm before, or a gate.
template <class A, class R, int U, int L, bool WIDE, bool WHOLE, bool MORE>
__global__ __launch_bounds__(most_waves(U, L, WIDE, MORE) * 64) void k_forward(BlockArgs a, const R* x, const A* block, R* y, A* h, float* stats, int32_t of_sum) {
  constexpr int kRows = 64 / L;  // of a block at a time
  __shared__ float2 part[3 * kMostWaves];
  Join<L> join{part, part + 2 * kMostWaves, (int)blockDim.x / 64, 0};
  join.template count_columns<U>(a);
  const Columns<U, L, WHOLE> c(a);
  const Weights<U, L, WHOLE> w(a, a.weight, c, 1.0f), wb(a, a.bias, c, 0.0f), pw(a, MORE ? a.post_weight : nullptr, c, 1.0f), pb(a, MORE ? a.post_bias : nullptr, c, 0.0f);
  const Weights<U, L, WHOLE> shared_gate(a, !MORE || a.gate_stride ? nullptr : a.gate, c, 1.0f);
  const int sub = L < 64 ? (int)threadIdx.x / L : 0;
  auto read = [&](int64_t t0) {
    const int64_t t = min(t0 + sub, a.n - 1);
    Input<A, R, U> in;
    each<U>([&](int u) {
      in.x[u] = mist::load_raw8(x + t * a.x_stride, c.e[u]);
      if (block) in.b[u] = mist::load_raw8(block + t * a.block_stride, c.e[u]);
    });
    return in;
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  Input<A, R, U> in;
  if (U == 1) in = read((int64_t)blockIdx.x * kRows);
  for (int64_t t0 = (int64_t)blockIdx.x * kRows; t0 < a.n; t0 += step) {
    const int64_t t = t0 + sub;
    const bool there = L == 64 || t < a.n;
    Input<A, R, U> now;
    if constexpr (U == 1) {
      now = in;
      if (t0 + step < a.n) in = read(t0 + step);
    } else {
      now = read(t0);
    }
    Float8 v[U];
    each<U>([&](int u) { v[u] = mist::wide8<R>(now.x[u], c.e[u]); });
    Moments before{0.0f, 1.0f}, after{0.0f, 1.0f};
    if (block) {
      Float8 b[U];
      each<U>([&](int u) {
        b[u] = mist::wide8<A>(now.b[u], c.e[u]);
      });
      const int64_t gate_row = MORE && a.gate_stride ? min(t, a.n - 1) / a.seq * a.gate_stride : 0;
      if (MORE && a.post_weight) {
        before = moments<U, L, WHOLE>(a, join, c, b);
        each<U>([&](int u) { b[u] = (b[u] - before.mean) * before.r * pw(u) + pb(u); });
      }
      each<U>([&](int u) {
        if (MORE) b[u] *= a.gate_stride ? load_weight(a.gate, a.weight_type, gate_row, c.e[u]) : shared_gate(u);
        v[u] = a.res_scale * v[u] + a.block_scale * b[u];
        if (there) store8(y + t * a.y_stride, c.e[u], v[u]);
        // of y as it is stored: formed again from it, h has the same bits
        if (!of_sum) v[u] = __builtin_convertvector(__builtin_convertvector(v[u], mist::Raw8<R>), Float8);
        v[u] = masked(v[u], c.e[u]);
      });
    }
    if (h) {
      after = moments<U, L, WHOLE>(a, join, c, v);
      if (there) each<U>([&](int u) { store8(h + t * a.h_stride, c.e[u], (v[u] - after.mean) * after.r * w(u) + wb(u)); });
    }
    if (there && c.e[0].col == 0) *(float4*)(stats + t * 4) = float4{before.mean, before.r, after.mean, after.r};
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

// Waves a SIMD of the backward pass without a norm before or a gate.  Five, with a few registers spilled, are worth it to blocks of several
// waves and 16-bit rows (65536 x 2560: 377 us, 438 with four), not to single waves (65536 x 512: 75 and 66) or fp32 (1000 x 1024: 11.8 and 9.3).
constexpr int back_waves(int u, int l, bool wide, size_t res_bytes) { return u == 1 && l == 64 && !wide && res_bytes == 2 ? 5 : 4; }

template <class A, class R, int U>
struct BackInput {
  mist::Raw8<R> y[U], dy[U];
  mist::Raw8<A> b[U], dh[U];
  float4 st;
};

// With e the gradient of gate v (v = n post_weight + post_bias) over a sequence's tokens, the sums of e and of e n are all
// that the gradients of gate, post_weight and post_bias need: two sums a column for three.
template <class A, class R, int U, int L, bool WIDE, bool WHOLE, bool MORE>
__global__ __launch_bounds__(most_waves(U, L, WIDE, MORE) * 64, MORE && !WIDE ? L == 64 ? 3 : 2 : back_waves(U, L, WIDE, sizeof(R))) void k_backward(BackArgs k, const R* y, const A* block, const float* stats, const A* dh, const R* dy, R* dx,
                                                                          A* dblock) {
  constexpr bool kAhead = U == 1 && !(MORE && WIDE);
  constexpr int kRows = 64 / L;
  __shared__ float2 shared[2 * kMostWaves];
  const BlockArgs& a = k.a;
  Join<L> join{shared, nullptr, (int)blockDim.x / 64, 0};
  const Columns<U, L, WHOLE> c(a);
  const Weights<U, L, WHOLE> w(a, a.weight, c, 1.0f);
  Float8 gp[U];  // gate post_weight
  Float8 sw[U] = {}, sb[U] = {}, sen[U], se[U];
  auto post_weight = [&](int u) { return a.post_weight ? load_weight(a.post_weight, a.weight_type, 0, c.e[u]) : Float8(1.0f); };
  auto gate = [&](int u, int64_t s) { return a.gate ? load_weight(a.gate, a.weight_type, s * a.gate_stride, c.e[u]) : Float8(1.0f); };
  const int sub = L < 64 ? (int)threadIdx.x / L : 0;
  const int64_t part = blockIdx.x, first = part / k.parts.pieces * k.parts.seqs, row0 = part % k.parts.pieces * k.parts.rows;
  const int64_t last = min(first + k.parts.seqs, k.parts.batch), row1 = min(row0 + k.parts.rows, k.parts.seq);
  auto read = [&](int64_t s, int64_t r0) {
    const int64_t t = s * k.parts.seq + min(r0 + sub, row1 - 1);
    BackInput<A, R, U> in;
    each<U>([&](int u) {
      if (dh) in.dh[u] = mist::load_raw8(dh + t * k.dh_stride, c.e[u]);
      if (dh) in.y[u] = mist::load_raw8(y + t * a.y_stride, c.e[u]);
      if (dy) in.dy[u] = mist::load_raw8(dy + t * k.dy_stride, c.e[u]);
      if (MORE && block) in.b[u] = mist::load_raw8(block + t * a.block_stride, c.e[u]);
    });
    in.st = *(const float4*)(stats + t * 4);
    return in;
  };
  BackInput<A, R, U> in;
  if (kAhead) in = read(first, row0);
  for (int64_t s = first; s < last; ++s) {
    each<U>([&](int u) {
      if (MORE) gp[u] = gate(u, s) * post_weight(u);
      sen[u] = se[u] = 0.0f;
    });
    for (int64_t r0 = row0; r0 < row1; r0 += kRows) {
      const int64_t t = s * k.parts.seq + r0 + sub;
      const bool there = L == 64 || r0 + sub < row1;
      if (!kAhead) in = read(s, r0);
      const float4 st = in.st;
      Float8 d[U], g[U], n[U], b[U];
      each<U>([&](int u) {
        d[u] = dy ? mist::wide8<R>(in.dy[u], c.e[u]) : Float8(0.0f);
        if (dh) g[u] = mist::wide8<A>(in.dh[u], c.e[u]);
        if (dh) n[u] = (mist::wide8<R>(in.y[u], c.e[u]) - st.z) * st.w;
        if (MORE && block) b[u] = masked((mist::wide8<A>(in.b[u], c.e[u]) - st.x) * st.y, c.e[u]);
      });
      if (kAhead) {  // in the registers that have just been read
        if (r0 + kRows < row1) in = read(s, r0 + kRows);
        else if (s + 1 < last) in = read(s + 1, row0);
      }
      if (dh) {
        float p = 0.0f, q = 0.0f;
        each<U>([&](int u) {
          if (there) {
            sb[u] += g[u];
            sw[u] += g[u] * n[u];
          }
          g[u] *= w(u);
          p += sum8(g[u]);
          q += sum8(masked(g[u] * n[u], c.e[u]));
        });
        const float2 m = join.sum(p, q);
        const float mean = a.layer ? m.x * a.inv_hidden : 0.0f, along = m.y * a.inv_hidden;
        each<U>([&](int u) { d[u] += st.w * (g[u] - mean - n[u] * along); });
      }
      if (dx && there) each<U>([&](int u) { store8(dx + t * k.dx_stride, c.e[u], a.res_scale * d[u]); });
      if (block) {
        each<U>([&](int u) { d[u] *= a.block_scale; });
        if (MORE) {
          each<U>([&](int u) {
            if (there) {
              se[u] += d[u];
              sen[u] += d[u] * b[u];
            }
            d[u] = masked(d[u] * gp[u], c.e[u]);
          });
          if (a.post_weight) {
            float p = 0.0f, q = 0.0f;
            each<U>([&](int u) {
              p += sum8(d[u]);
              q += sum8(d[u] * b[u]);
            });
            const float2 m = join.sum(p, q);
            const float mean = a.layer ? m.x * a.inv_hidden : 0.0f, along = m.y * a.inv_hidden;
            each<U>([&](int u) { d[u] = st.y * (d[u] - mean - b[u] * along); });
          }
        }
        if (dblock && there) each<U>([&](int u) { store8(dblock + t * k.dblock_stride, c.e[u], d[u]); });
      }
    }
    if (MORE) {
      each<U>([&](int u) {
        se[u] = over_rows<L>(se[u]);
        sen[u] = over_rows<L>(sen[u]);
        if (sub) return;
        const Float8 g = gate(u, s);
        const int64_t at = part * a.hidden;
        auto add = [&](float* p, Float8 x) {  // the part's sum over its sequences
          if (s > first) x += load8(p + at, c.e[u]);
          store8(p + at, c.e[u], x);
        };
        if (k.slot[2]) add(k.slot[2], g * sen[u]);
        if (k.slot[3]) add(k.slot[3], g * se[u]);
        if (!k.slot[4] && !k.dgate) return;
        Float8 x = sen[u];
        if (a.post_weight) x *= post_weight(u);
        if (a.post_bias) x += load_weight(a.post_bias, a.weight_type, 0, c.e[u]) * se[u];
        if (k.slot[4]) add(k.slot[4], x);
        if (!k.dgate) return;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < c.e[u].left) store_weight(k.dgate, a.weight_type, s * k.dgate_stride + c.e[u].col + i, x[i], k.accumulate);
      });
    }
  }
  each<U>([&](int u) {
    const int64_t at = part * a.hidden;
    sw[u] = over_rows<L>(sw[u]);
    sb[u] = over_rows<L>(sb[u]);
    if (k.slot[0] && !sub) store8(k.slot[0] + at, c.e[u], sw[u]);
    if (k.slot[1] && !sub) store8(k.slot[1] + at, c.e[u], sb[u]);
  });
}

// The parts' sums, in an order that goes by their number: parts [i * count, (i + 1) * count) give row i of out.  A block
// takes 64 columns in 16 shares of the parts, or, of many parts, 32 columns (a cache line) in 32 shares.
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
__host__ __device__ __forceinline__ int join_columns(const JoinJob& j) { return j.count >= 256 ? 32 : 64; }

__global__ __launch_bounds__(kJoinThreads) void k_join_parts(JoinArgs k) {
  constexpr int kWaves = kJoinThreads / 64;
  __shared__ float share[kWaves][64];
  const JoinJob j = k.job[blockIdx.y];
  const int width = join_columns(j), lane = (int)threadIdx.x % width, mine = (int)threadIdx.x / width, shares = kJoinThreads / width;
  const int64_t columns = (k.hidden + width - 1) / width;
  for (int64_t i = blockIdx.x; i < columns * j.rows; i += gridDim.x) {
    const int64_t row = i / columns, col = i % columns * width + lane;
    float s = 0.0f;
    if (col < k.hidden) {
      const float* p = j.part + row * j.count * k.hidden + col;
#pragma unroll 8
      for (int64_t r = mine; r < j.count; r += shares) s += p[r * k.hidden];
    }
    auto sum = [](float a, float b) { return a + b; };
    if (width == 32) s = mist::join_pairs_of_32(s, sum);  // the shares of a wave
    __syncthreads();
    share[threadIdx.x / 64][threadIdx.x % 64] = s;
    __syncthreads();
    if (mine == 0 && col < k.hidden) {
      s = 0.0f;
      for (int w = 0; w < kWaves; ++w) s += share[w][lane];
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
  if (d->of_sum != 0 && d->of_sum != 1) return lib_fail(MIST_E_INVALID, "block norm: of_sum must be 0 or 1");
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

// A vector of n values, and rows of the residual's or the block's type, for the checks of the call's other tensors.
mist::Use<mist::Rows> vector(const void* p, int64_t n, int64_t bytes, bool out) { return {mist::Rows{p, 1, 0, n, bytes}, out}; }
mist::Use<mist::Rows> rows(const mist_block_desc* d, const void* p, int64_t stride, int32_t type, bool out) {
  return {mist::Rows{p, d->batch * d->seq, stride, d->hidden, mist::type_bytes(type)}, out};
}
// gates by sequence, or one for all
mist::Use<mist::Rows> gates(const mist_block_desc* d, const void* p, int64_t stride, bool out) {
  const bool by_sequence = d->gate_stride && d->batch != 1;
  return {mist::Rows{p, by_sequence ? d->batch : 1, by_sequence ? stride : 0, d->hidden, mist::type_bytes(d->weight_type)}, out};
}
mist_status not_shared(bool shared) { return shared ? lib_fail(MIST_E_INVALID, "block norm: an output or the workspace overlaps another tensor") : MIST_OK; }

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

int lanes(int64_t hidden) { return hidden <= 128 ? 16 : hidden <= 256 ? 32 : 64; }
int units(int64_t hidden) { return hidden > kMostWaves * 512 ? 2 : 1; }
unsigned threads(int64_t hidden) { return (unsigned)((hidden + units(hidden) * 512 - 1) / (units(hidden) * 512) * 64); }

// f(activation type, residual type, columns a thread / 8, lanes a row, a wide row, whole waves)
template <class F>
void with_kernel(const mist_block_desc* d, bool more, F&& f) {
  mist::with_type(d->type, [&](auto x) {
    using A = typename decltype(x)::type;
    auto run = [&](auto r) {
      using R = typename decltype(r)::type;
      using One = std::integral_constant<int, 1>;
      using Wave = std::integral_constant<int, 64>;
      using No = std::false_type;
      const auto wave = [&](auto whole) {  // rows of whole waves are the common ones; the others' code has their ends to hold and to mask
        if (threads(d->hidden) > (unsigned)narrow_waves(more) * 64) f(A{}, R{}, One{}, Wave{}, std::true_type{}, whole);
        else f(A{}, R{}, One{}, Wave{}, No{}, whole);
      };
      if (units(d->hidden) == 2) f(A{}, R{}, std::integral_constant<int, 2>{}, Wave{}, std::true_type{}, No{});
      else if (lanes(d->hidden) == 32) f(A{}, R{}, One{}, std::integral_constant<int, 32>{}, No{}, No{});
      else if (lanes(d->hidden) == 16) f(A{}, R{}, One{}, std::integral_constant<int, 16>{}, No{}, No{});
      else if (d->hidden % 512 == 0) wave(std::true_type{});
      else wave(No{});
    };
    if (d->res_type == d->type) run(x);
    else run(mist::Elem<MIST_F32>{});
  });
}

mist_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, what);
}

// Waves of the backward pass that a CU holds: one round of blocks of the same work (two to four rounds took 0-5 % more), or as many rounds as
// keep the sums' chains short.
int64_t resident_waves(const mist_block_desc* d, int64_t waves, bool more) {
  const bool wide = waves == 1 || waves > narrow_waves(more);
  return more && !wide ? 12 : more ? 16 : 4 * back_waves(units(d->hidden), lanes(d->hidden), wide, (size_t)mist::type_bytes(d->res_type));
}

Parts parts_of(const mist_block_desc* d, bool by_sequence, bool more) {
  Parts p{};
  p.batch = by_sequence ? d->batch : 1;
  p.seq = by_sequence ? d->seq : d->batch * d->seq;
  if (!p.batch || !p.seq) return p;
  const int64_t waves = threads(d->hidden) / 64, round = 256 * std::max<int64_t>(1, resident_waves(d, waves, more) / waves), least = kPartRows * 64 / lanes(d->hidden);
  const int64_t parts = round * std::clamp<int64_t>((p.batch * p.seq + round * kMostRows - 1) / (round * kMostRows), 1, std::max<int64_t>(1, kMostParts / round));
  p.pieces = std::clamp<int64_t>(parts / p.batch, 1, (p.seq + least - 1) / least);
  p.rows = (p.seq + p.pieces - 1) / p.pieces;
  p.pieces = (p.seq + p.rows - 1) / p.rows;
  p.seqs = p.pieces > 1 ? 1 : std::max<int64_t>((p.batch + parts - 1) / parts, std::min<int64_t>((least + p.seq - 1) / p.seq, p.batch));
  p.n = (p.batch + p.seqs - 1) / p.seqs * p.pieces;
  return p;
}

struct Plan {
  Parts parts;
  size_t bytes;
  bool wanted[kSlots], direct;  // direct: gates' gradients need no parts
};
// more: a norm before or a gate, as the kernel has it, whether or not their gradients are wanted.
Plan plan_of(const mist_block_desc* d, const mist_block_grads* g, bool more) {
  Plan p{};
  const bool by_sequence = d->gate_stride && d->batch > 1;
  p.parts = parts_of(d, by_sequence, more);
  const void* out[kSlots] = {g->dweight, g->dbias, g->dpost_weight, g->dpost_bias, g->dgate};
  p.direct = by_sequence && p.parts.pieces == 1;
  for (int i = 0; i < kSlots; ++i) {
    p.wanted[i] = out[i] && !(i == 4 && p.direct);
    if (p.wanted[i]) p.bytes += (size_t)p.parts.n * d->hidden * 4 + 256;
  }
  return p;
}

// The query does not see whether there is a norm before or a gate, unless their gradients are wanted: enough for both.
size_t scratch_of(const mist_block_desc* d, const mist_block_grads* g) {
  const size_t more = plan_of(d, g, true).bytes;
  return g->dpost_weight || g->dpost_bias || g->dgate ? more : std::max(more, plan_of(d, g, false).bytes);
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
  const int64_t wide = mist::type_bytes(d->weight_type);
  if (const mist_status st = not_shared(mist::shared<mist::Rows>(
          {vector(stats, a.n * 4, 4, true), vector(weight, d->hidden, wide, false), vector(bias, d->hidden, wide, false), vector(post_weight, d->hidden, wide, false),
           vector(post_bias, d->hidden, wide, false), gates(d, gate, d->gate_stride, false)},
          {rows(d, x, d->x_stride, d->res_type, false), rows(d, block, d->block_stride, d->type, false), rows(d, y, d->y_stride, d->res_type, true),
           rows(d, h, d->h_stride, d->type, true)})))
    return st;
  with_kernel(d, post_weight || gate, [&](auto e, auto f, auto u, auto l, auto wide, auto whole) {
    using A = decltype(e);
    using R = decltype(f);
    constexpr bool kWide = l.value == 64;  // its registers are the same for all
    const auto kernel = post_weight || gate ? k_forward<A, R, u.value, l.value, kWide, whole.value, true> : k_forward<A, R, u.value, l.value, kWide, whole.value, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>((a.n * l.value + 63) / 64, kMostBlocks)), dim3(threads(d->hidden)), 0, (hipStream_t)stream, a,
                       (const R*)x, (const A*)block, (R*)y, (A*)h, stats, d->of_sum);
  });
  return launched("block norm");
}

mist_status mist_block_workspace(const mist_block_desc* d, const mist_block_grads* g, size_t* bytes) {
  if (!bytes) return lib_fail(MIST_E_INVALID, "block norm's gradient: null argument");
  if (const mist_status st = check_grads(d, g)) return st;
  *bytes = scratch_of(d, g);
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
  const Plan p = plan_of(d, g, post_weight || gate);
  const size_t need = scratch_of(d, g);
  if (!any && g->accumulate) return MIST_OK;
  if (any && (!stats || (weight && (!y || !g->dh)) || (!weight && g->dh) || (!g->dh && !g->dy)))
    return lib_fail(MIST_E_INVALID, "block norm's gradient: null buffer, or dh without its weight");
  if (!mist::is_aligned(stats, 16) || !mist::is_aligned(workspace, 256) ||
      !weights_ok(d, {weight, post_weight, post_bias, gate, g->dweight, g->dbias, g->dpost_weight, g->dpost_bias, g->dgate}))
    return lib_fail(MIST_E_INVALID, "block norm's gradient: a buffer is not aligned to its elements, stats to 16 or the workspace to 256");
  if (need && !workspace) return lib_fail(MIST_E_INVALID, "block norm's gradient: null workspace");
  if (workspace_bytes < need) return lib_fail(MIST_E_RANGE, "block norm's gradient: workspace too small");
  if (const mist_status st = check_tensors(d, {{y, d->y_stride, d->res_type, false, {}}, {block, d->block_stride, d->type, false, {}},
                                               {g->dh, g->dh_stride, d->type, false, {}}, {g->dy, g->dy_stride, d->res_type, false, {}},
                                               {g->dx, g->dx_stride, d->res_type, true, {g->dy, nullptr}},
                                               {g->dblock, g->dblock_stride, d->type, true, {g->dh, block}}}))
    return st;
  const int64_t wide = mist::type_bytes(d->weight_type);
  if (const mist_status st = not_shared(mist::shared<mist::Rows>(
          {vector(stats, a.n * 4, 4, false), vector(weight, d->hidden, wide, false), vector(post_weight, d->hidden, wide, false), vector(post_bias, d->hidden, wide, false),
           gates(d, gate, d->gate_stride, false), vector(g->dweight, d->hidden, wide, true), vector(g->dbias, d->hidden, wide, true),
           vector(g->dpost_weight, d->hidden, wide, true), vector(g->dpost_bias, d->hidden, wide, true), gates(d, g->dgate, g->dgate_stride, true),
           vector(workspace, (int64_t)p.bytes, 1, true)},
          {rows(d, y, d->y_stride, d->res_type, false), rows(d, block, d->block_stride, d->type, false), rows(d, g->dh, g->dh_stride, d->type, false),
           rows(d, g->dy, g->dy_stride, d->res_type, false), rows(d, g->dx, g->dx_stride, d->res_type, true), rows(d, g->dblock, g->dblock_stride, d->type, true)})))
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
    const bool gates = i == 4 && d->gate_stride && d->batch != 1;  // a row for each sequence
    if (gates && !d->batch) continue;
    j.job[jobs++] = JoinJob{k.slot[i], out[i], gates ? p.parts.pieces : p.parts.n, gates ? d->batch : 1, gates ? g->dgate_stride : 0};
    most = std::max(most, (d->hidden + join_columns(j.job[jobs - 1]) - 1) / join_columns(j.job[jobs - 1]) * j.job[jobs - 1].rows);
    ws += ((size_t)p.parts.n * d->hidden * 4 + 255) / 256 * 256;
  }
  if (!any && !jobs) return MIST_OK;
  const hipStream_t st = (hipStream_t)stream;
  if (any) {
    with_kernel(d, post_weight || gate, [&](auto e, auto f, auto u, auto l, auto wide, auto whole) {
      using A = decltype(e);
      using R = decltype(f);
      const auto kernel = post_weight || gate          ? k_backward<A, R, u.value, l.value, wide.value, whole.value, true>
                          : threads(d->hidden) == 64 && l.value == 64 ? k_backward<A, R, u.value, l.value, true, whole.value, false>
                                                                      : k_backward<A, R, u.value, l.value, wide.value, whole.value, false>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)p.parts.n), dim3(threads(d->hidden)), 0, st, k, (const R*)y, (const A*)block, stats, (const A*)g->dh,
                         (const R*)g->dy, (R*)g->dx, (A*)g->dblock);
    });
  }
  if (jobs) hipLaunchKernelGGL(k_join_parts, dim3((unsigned)std::min<int64_t>(most, 65536), (unsigned)jobs), dim3(kJoinThreads), 0, st, j);
  return launched("block norm's gradient");
}

}  // extern "C"
