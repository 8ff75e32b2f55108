// Token log probabilities, entropies and alternatives, their gradient, and the loss of a training microbatch.
//
// z = scale * logits is never stored.  A row's largest logit comes first, and exponentials are of the scaled distance from it, not of a
// difference of scaled values: the distance is exact for 16-bit logits and never above 0, so that every exponential is at most 1, however large
// the logits are (a fused product less a rounded largest one is off by up to half a step of that: past any exponential from 2^31 on).  A row stays in the registers of its block from its one reading to the
// last pass over it (of 16-bit values up to 65536, of fp32 32768; longer ones by chunks, whose sums are rescaled); the loss writes the
// gradient from there.  Measured on one MI355X, where a large copy reads and writes 4.9 TB/s:
//   loss        32768 x 50257 bf16  1265 us, 5.2 TB/s: memory
//   gradient    8192 x 50257 bf16   306 us, 5.4 TB/s: memory
//   statistics  8192 x 32000 fp32   171 us, 6.1 TB/s: memory;  8192 x 50256 bf16  158 us, 5.2 TB/s: vector instructions, 12.0 a
//               logit (a conversion and the maximum, then a conversion, the exponential and five more)
//   with 8 alternatives  16376 x 50257 bf16  461-470 us
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mist_ops.h"

using mist::fast_exp;
using mist::hip_failed;
using mist::lib_fail;
using mist::wave_max;
using mist::wave_sum;

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostTokens = (int64_t)1 << 30;
constexpr float kLowest = -3.4028234663852886e38f;  // finite
constexpr float kLow = -1000.0f;  // of a logarithm, beside an exponential that is 0 there: 0 * kLow is 0 where 0 * -inf is not
constexpr int64_t kMostBlocks = (int64_t)1 << 20;  // a grid stays below 2^32 threads; kernels loop

struct TokenArgs {
  int64_t rows, vocab_begin, ids_stride, logits_batch_stride, logits_stride, grad_batch_stride, grad_stride;
  uint32_t seq;  // at least 1
  int32_t n, ids_bytes, top;  // n: tokens
  float scale, pre, rest;  // log2(e) scale = pre * rest, with pre a power of two: 1 unless a scale is past 2^64 either way
};

__device__ __forceinline__ int64_t offset_of(const TokenArgs& a, int32_t t, int64_t batch_stride, int64_t stride) {
  const uint32_t b = (uint32_t)t / a.seq;
  return b * batch_stride + ((uint32_t)t - b * a.seq) * stride;
}
__device__ __forceinline__ int64_t target_of(const TokenArgs& a, const void* targets, int32_t t) {
  const int64_t at = offset_of(a, t, a.ids_stride, 1);
  return a.ids_bytes == 4 ? ((const int32_t*)targets)[at] : ((const int64_t*)targets)[at];
}
__device__ __forceinline__ int64_t logits_offset(const TokenArgs& a, int32_t t) { return offset_of(a, t, a.logits_batch_stride, a.logits_stride); }
__device__ __forceinline__ int64_t grad_offset(const TokenArgs& a, int32_t t) { return offset_of(a, t, a.grad_batch_stride, a.grad_stride); }

// Unsigned numbers in the order of the logits: -0 as 0, NaN above everything.  -inf, which is no alternative, is 0.
constexpr uint32_t kNanRank = 0xFFFFFFFEu;  // no key is all ones
__device__ __forceinline__ uint32_t rank_of(float x) {
  if (x != x) return kNanRank;
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b == 0xFF800000u ? 0u : b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_rank(uint32_t r) {
  if (r == kNanRank) return __builtin_nanf("");
  if (r == 0) return -HUGE_VALF;
  return __uint_as_float(r >> 31 ? r & 0x7FFFFFFFu : ~r);
}
// Distinct keys of alternatives: larger logits first, the lower id first among equals.
__device__ __forceinline__ uint64_t key_of(uint32_t rank, uint32_t id) { return (uint64_t)rank << 32 | (uint32_t)~id; }

template <int L = 64>
__device__ __forceinline__ uint64_t wave_max_key(uint64_t x) {
#pragma unroll
  for (int d = L / 2; d; d >>= 1) {
    const uint64_t y = (uint64_t)__shfl_xor((int)(x >> 32), d) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)x, d);
    x = y > x ? y : x;
  }
  return x;
}

// What a row's results are formed from: stats of the row or of all ranks.
struct Stats {
  float m, s, u, z;
};
__device__ __forceinline__ bool nothing(const Stats& x) { return x.m == -HUGE_VALF && x.s == 0.0f; }  // all masked out
__device__ __forceinline__ float lse_of(const Stats& x) { return nothing(x) ? x.m : x.m + logf(x.s); }
__device__ __forceinline__ float entropy_of(const Stats& x) { return nothing(x) ? 0.0f : logf(x.s) - x.u / x.s; }
__device__ __forceinline__ float logp_of(float z, float lse, int64_t target) {
  return target < 0 ? 0.0f : z == -HUGE_VALF && !(lse != lse) ? z : z - lse;
}

// A block's sums and largest values: joined over its waves through two places in turn, so that a wave writes one only after
// every wave has read its last values.
template <int WAVES>
struct Join {
  float2 (*part)[WAVES];
  int turn;
  __device__ __forceinline__ void put(float a, float b) {
    float2* p = part[turn];
    turn ^= 1;
    if (threadIdx.x % 64 == 0) p[threadIdx.x / 64] = float2{a, b};
    __syncthreads();
  }
  __device__ __forceinline__ float2 sum(float a, float b) {
    a = wave_sum(a);
    b = wave_sum(b);
    if (WAVES == 1) return float2{a, b};
    const float2* p = part[turn];
    put(a, b);
    float2 s = p[0];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) s.x += p[k].x, s.y += p[k].y;
    return s;
  }
  __device__ __forceinline__ float2 most_and_least(float2 x) {
    if (WAVES == 1) return x;
    const float2* p = part[turn];
    put(x.x, x.y);
    x = p[0];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) x = float2{fmaxf(x.x, p[k].x), fminf(x.y, p[k].y)};
    return x;
  }
};

// A chunk of a row in the registers of its block: vectors of 16 bytes at whole multiples of 16 in memory, N a thread, in turn
// over the threads, and what lies before the first and after the last, one value a thread.  (50257 16-bit values a row, most off
// alignment: 163 us for 8192 aligned rows, 221 with vectors from the row's first value on.)  What is not there is -inf.  The
// values stay in their type between the passes over them (the empty assembly keeps the compiler from holding them converted, which takes
// twice the registers of 16-bit values).
typedef uint32_t Raw __attribute__((ext_vector_type(4)));

template <class T, int THREADS, int N, bool ALIGN = true>
struct Chunk {
  static constexpr int kV = 16 / sizeof(T), kAll = THREADS * N * kV;
  typedef T V __attribute__((ext_vector_type(kV)));
  typedef typename mist::Vec<T, kV>::type Anywhere;
  Raw v[N];
  float odd;
  int n, head;  // values, and those before the first vector

  __device__ __forceinline__ int place(int j) const {
    int at = threadIdx.x;
    asm("" : "+v"(at));  // formed anew where it is used, rather than N of them held
    return head + (j * THREADS + at) * kV;
  }
  __device__ __forceinline__ int tail() const { return n - (n - head) % kV; }  // past the last vector
  // of the odd value; n or more: none
  __device__ __forceinline__ int odd_place() const { return odd_place((int)threadIdx.x); }
  __device__ __forceinline__ int odd_place(int t) const { return t < head ? t : tail() + t - head; }
  __device__ __forceinline__ bool any(int j) const { return head + (j * THREADS + 1) * kV <= n; }  // the j-th vector of some thread
  __device__ __forceinline__ void load(const T* x, int count, bool read = true) {
    n = count;
    head = !ALIGN ? 0 : min(n, (int)(-(reinterpret_cast<uintptr_t>(x) / sizeof(T)) % kV));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      V r = (T)-HUGE_VALF;
      const int at = place(j);
      if (read && at + kV <= n) r = *(const std::conditional_t<ALIGN, V, Anywhere>*)(x + (uint32_t)at);
      v[j] = __builtin_bit_cast(Raw, r);
    }
    odd = read && odd_place() < n ? (float)x[odd_place()] : -HUGE_VALF;
  }
  // f(value); vectors that no thread has are passed over
  template <class F>
  __device__ __forceinline__ void each_of(int j, F&& f) {
    asm("" : "+v"(v[j]));
    const V r = __builtin_bit_cast(V, v[j]);
#pragma unroll
    for (int k = 0; k < kV; ++k) f((float)r[k]);
  }
  template <class F>
  __device__ __forceinline__ void each(F&& f) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (any(j)) each_of(j, f);
    f(odd);
  }
  // The largest value, and those of eight groups of vectors.
  static constexpr int kPer = N / 8, kGroup = kPer * kV;  // vectors and values of a group
  __device__ __forceinline__ float largest(float (&group)[8]) {
    float low = odd == odd ? odd : -HUGE_VALF;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      group[i] = -HUGE_VALF;
#pragma unroll
      for (int j = i * kPer; j < (i + 1) * kPer; ++j)
        if (any(j)) each_of(j, [&](float x) { group[i] = fmaxf(group[i], x); });
      low = fmaxf(low, group[i]);
    }
    return low;
  }
  // the place of a group's k-th value in a thread
  __device__ __forceinline__ int group_place(int i, int thread, int k) const { return head + ((i * kPer + k / kV) * THREADS + thread) * kV + k % kV; }
  // y = f(value)
  template <class F>
  __device__ __forceinline__ void store(T* y, F&& f) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int at = place(j);
      if (at + kV > n) continue;
      asm("" : "+v"(v[j]));
      const V r = __builtin_bit_cast(V, v[j]);
      V q;
#pragma unroll
      for (int k = 0; k < kV; ++k) q[k] = (T)f((float)r[k]);
      *(Anywhere*)(y + (uint32_t)at) = q;
    }
    if (odd_place() < n) y[odd_place()] = (T)f(odd);
  }
  // whether this thread holds a place
  __device__ __forceinline__ bool mine(int at) const {
    const int t = threadIdx.x;
    return at < head ? at == t : at >= tail() ? at - tail() + head == t : (at - head) / kV % THREADS == t;
  }
};

// Alternatives.  At least q = ceil(top / waves) lanes of each wave have a value of at least the wave's q-th largest lane
// maximum, so the least of these over the waves bounds a row's top-th largest value from below.  The few groups of a thread's values
// that reach it are listed (and all of a thread with a NaN), and the block then looks through them together, from the cache: a wave that
// looks through its own registers takes as many instructions for one lane's group as for all lanes' (8 alternatives of 8192
// rows of 50257 16-bit values: 254 us so, 237 by the list).  A candidate's place is the number of larger ones.  Where a list
// is too short (equal values in many places) the largest are taken one by one, with a pass each.
constexpr int kCandidates = 512;

struct Top {
  uint64_t list[kCandidates];
  uint64_t best[MIST_TOKEN_MAX_TOP];  // of the chunks before, in order; 0: none
  uint64_t part[8];
  uint32_t group[kCandidates];        // group << 16 | thread; 8: the odd value
  int count, groups;
};

// The wave's q-th largest value (or less, where several are equal to it).
__device__ __forceinline__ float wave_bound(float x, int q) {
  if (q > 6) {  // by the number of larger lanes: 64 steps that do not wait for each other
    int larger = 0;
#pragma unroll
    for (int k = 0; k < 64; ++k) larger += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), k)) > x;
    return -wave_max(larger < q ? -x : -HUGE_VALF);
  }
  float bound = -HUGE_VALF;
  for (int k = 0; k < q; ++k) {
    bound = wave_max(x);
    if (bound == -HUGE_VALF) break;
    if ((int)threadIdx.x % 64 == __ffsll((unsigned long long)__ballot(x == bound)) - 1) x = -HUGE_VALF;
  }
  return bound;
}

__device__ __forceinline__ void add_group(Top& t, int i) {
  const int at = atomicAdd(&t.groups, 1);
  if (at < kCandidates) t.group[at] = (uint32_t)i << 16 | threadIdx.x;
}
// bound is finite or +inf: what is masked out is below it
template <class C>
__device__ __forceinline__ void list_groups(const C& c, const float (&group)[8], bool nan, float bound, Top& t) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (nan || group[i] >= bound) add_group(t, i);
  if (!(c.odd < bound)) add_group(t, 8);
}
// The listed groups' values from bound on with keys above least join the candidates, each once: a group's places past the last
// vector are others' odd values.  Between two barriers.
template <int THREADS, class C, class T>
__device__ __forceinline__ void list_candidates(const C& c, const T* x, uint32_t base, float bound, uint64_t least, Top& t) {
  for (int i = threadIdx.x; i < min(t.groups, kCandidates) * C::kGroup; i += THREADS) {
    const uint32_t g = t.group[i / C::kGroup];
    const int k = i % C::kGroup, thread = (int)(g & 0xFFFF), which = (int)(g >> 16);
    const int at = which < 8 ? c.group_place(which, thread, k) : c.odd_place(thread) + (k ? c.n : 0);
    const float v = at < (which < 8 ? c.tail() : c.n) ? (float)x[at] : -HUGE_VALF;
    if (v < bound) continue;
    const uint64_t key = key_of(rank_of(v), base + (uint32_t)at);
    if (key <= least) continue;
    const int to = atomicAdd(&t.count, 1);
    if (to < kCandidates) t.list[to] = key;
  }
}

// f(place, key) of the `top` largest of a chunk's candidates (those of the whole block are listed) and of the chunks
// before; places without one are left out.  All threads come; x, n: the chunk, where the list was too short.
template <int THREADS, class T, class F>
__device__ __forceinline__ void take_top(const T* x, int n, uint32_t base, int top, Top& t, F&& f) {
  const int tid = threadIdx.x;
  int count = t.count;
  if (count > kCandidates || t.groups > kCandidates) {
    __syncthreads();
    uint64_t last = ~0ull;
    count = 0;
    for (int k = 0; k < top; ++k) {
      uint64_t best = 0;
      for (int at = tid; at < n; at += THREADS) {
        const uint32_t rank = rank_of((float)x[at]);
        const uint64_t key = rank ? key_of(rank, base + (uint32_t)at) : 0;
        if (key > best && key < last) best = key;
      }
      best = wave_max_key(best);
      if (THREADS > 64) {
        if (tid % 64 == 0) t.part[tid / 64] = best;
        __syncthreads();
        for (int w = 0; w < THREADS / 64; ++w) best = std::max(best, t.part[w]);
      }
      if (tid == 0) t.list[k] = best;
      __syncthreads();
      if (!best) break;
      last = best;
      ++count;
    }
  }
  const int before = base ? top : 0;
  if (count + before <= 64) {  // one wave, by its registers
    if (tid >= 64) return;
    const uint64_t key = tid < count ? t.list[tid] : tid < count + before ? t.best[tid - count] : 0;
    int larger = 0;
    for (int k = 0; k < count + before; ++k) {
      const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), k) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)key, k);
      larger += other > key;
    }
    if (key && larger < top) f(larger, key);
    return;
  }
  for (int i = tid; i < count + before; i += THREADS) {
    const uint64_t key = i < count ? t.list[i] : t.best[i - count];
    int larger = 0;
    for (int k = 0; k < count; ++k) larger += t.list[k] > key;
    for (int k = 0; k < before; ++k) larger += t.best[k] > key;
    if (key && larger < top) f(larger, key);
  }
}

// The exponent of 2 of exp(z - max z): the distance from the largest logit, times log2(e) scale.  from: pre times that logit; 0 where
// nothing is visible (the exponentials are 0, of -inf, not NaN), +inf where the largest z is: all of the row becomes NaN.
__device__ __forceinline__ float start_of(const TokenArgs& a, float most) {
  const float m = most * a.scale;
  return m == -HUGE_VALF ? 0.0f : m == HUGE_VALF ? m : most * a.pre;
}
__device__ __forceinline__ float below(const TokenArgs& a, float x, float from) { return fmaf(x, a.pre, -from) * a.rest; }

// A row's gradient, p (c0 + c1 log p) + [j = target] up with scale in the factors.  One without factors is zeros, whatever the
// logits are: they are not looked at.  z is rounded before lse, which is none below it, is subtracted: p is at most 1.
struct Slope {
  float lse, c0, c1, up;
};
__device__ __forceinline__ bool flat(const Slope& g) { return g.c0 == 0.0f && g.c1 == 0.0f && g.up == 0.0f; }
__device__ __forceinline__ Slope slope_of(float lse, float scale, float dlogp, float dentropy, float entropy) {
  if (lse == -HUGE_VALF) return Slope{0.0f, 0.0f, 0.0f, 0.0f};
  return Slope{lse, scale * (dentropy != 0.0f ? -dlogp - dentropy * entropy : -dlogp), scale * -dentropy, scale * dlogp};
}
__device__ __forceinline__ float slope_at(const Slope& g, float x, float scale) {
  const float z = x * scale, l = z - g.lse, p = fast_exp(l);
  return p * fmaf(g.c1, fmaxf(l, kLow), g.c0);
}

struct RowOut {
  float *stats, *logp, *lse, *entropy;
  int32_t* top_ids;
  float* top_logp;
  const float* weights;
  float weight;
};

// A row a block: its results, with alternatives, or logp and the gradient.
enum Mode { kStats, kTop, kLoss };

template <class T, int THREADS, int N, Mode MODE>
__global__ __launch_bounds__(THREADS, N == 8 ? MODE == kTop ? 5 : 8 : 4) void k_row(TokenArgs a, const T* logits, const void* targets, RowOut o, T* dlogits) {
  using C = Chunk<T, THREADS, N>;
  __shared__ float2 part[2][THREADS / 64];
  __shared__ std::conditional_t<MODE == kTop, Top, int> top;
  Join<THREADS / 64> join{part, 0};
  for (int32_t t = blockIdx.x; t < a.n; t += gridDim.x) {
    const T* x = logits + logits_offset(a, t);
    const int64_t target = targets ? target_of(a, targets, t) : -1, at = target < 0 ? -1 : target - a.vocab_begin;
    const bool here = at >= 0 && at < a.rows;
    const float xt = here ? (float)x[at] : -HUGE_VALF;
    Stats r{-HUGE_VALF, 0.0f, 0.0f, here ? xt * a.scale : -HUGE_VALF};
    if constexpr (MODE == kTop) {
      if (threadIdx.x == 0) top.count = top.groups = 0;
      if (threadIdx.x < (unsigned)a.top) {
        top.best[threadIdx.x] = 0;
        o.top_ids[(int64_t)t * a.top + threadIdx.x] = -1;
        o.top_logp[(int64_t)t * a.top + threadIdx.x] = -HUGE_VALF;
      }
      if (THREADS == 64) __syncthreads();  // larger blocks meet in their joins
    }
    C c;
    float s = 0.0f, u = 0.0f, bound = 0.0f;  // u: in units of log(2)
    float most = -HUGE_VALF, from = 0.0f;
    for (int64_t base = 0; base < a.rows; base += C::kAll) {
      const int n = (int)min((int64_t)C::kAll, a.rows - base);
      c.load(x + base, n);
      float group[8];
      const float low = c.largest(group);
      float2 w = {wave_max(low), 0.0f};
      if (MODE == kTop) w.y = wave_bound(low, (a.top + THREADS / 64 - 1) / (THREADS / 64));
      w = join.most_and_least(w);
      const float start = start_of(a, fmaxf(most, w.x));
      if (base) {
        // where nothing was visible s and u are 0
        const float d = most * a.scale == -HUGE_VALF ? 0.0f : (from - start) * a.rest, f = __builtin_amdgcn_exp2f(d);
        u = f * fmaf(fmaxf(d, kLow), s, u);  // d may be near fp32's end, and f 0
        s *= f;
      }
      most = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(fmaxf(most, w.x))));  // the block's, in a scalar register
      from = start;
      c.each([&](float v) {
        const float d = below(a, v, from), e = __builtin_amdgcn_exp2f(d);
        s += e;
        if (MODE != kLoss) u = fmaf(e, fmaxf(d, kLow), u);  // a NaN comes with e
      });
      if constexpr (MODE == kTop) {
        bound = fmaxf(w.y, kLowest);
        list_groups(c, group, s != s, bound, top);
        if (base + C::kAll < a.rows) {  // more chunks
          uint64_t mine[2] = {0, 0};
          int place[2] = {-1, -1}, k = 0;
          __syncthreads();
          list_candidates<THREADS>(c, x + base, (uint32_t)base, bound, base ? top.best[a.top - 1] : 0, top);
          __syncthreads();
          take_top<THREADS>(x + base, n, (uint32_t)base, a.top, top, [&](int at, uint64_t key) { place[k & 1] = at, mine[k++ & 1] = key; });
          __syncthreads();
          if (threadIdx.x == 0) top.count = top.groups = 0;
          for (int i = 0; i < 2; ++i)
            if (place[i] >= 0) top.best[place[i]] = mine[i];
          __syncthreads();
        }
      }
    }
    const float2 su = join.sum(s, u);
    r.m = most * a.scale, r.s = su.x, r.u = su.y * 0.693147180559945309f;
    const float l = lse_of(r);
    if (threadIdx.x == 0) {
      if (MODE == kLoss) {
        o.logp[t] = logp_of(r.z, l, target);
      } else if (o.stats) {
        *(float4*)(o.stats + (int64_t)t * 4) = float4{r.m, r.s, r.u, r.z};
      } else {
        o.lse[t] = l;
        if (o.logp) o.logp[t] = logp_of(r.z, l, target);
        if (o.entropy) o.entropy[t] = entropy_of(r);
      }
    }
    if constexpr (MODE == kLoss) {
      // the exponentials over their sum: no rounding of lse comes into p
      const Slope g = slope_of(l, a.scale, target < 0 ? 0.0f : -(o.weights ? o.weight * o.weights[t] : o.weight), 0.0f, 0.0f);
      const bool zero = flat(g);
      const float share = g.c0 / r.s;
      T* y = dlogits + grad_offset(a, t);
      // the last chunk is still here; the others are read again
      const int64_t final = (a.rows - 1) / C::kAll * C::kAll;
      for (int64_t base = final; base >= 0; base -= C::kAll) {
        const int n = (int)min((int64_t)C::kAll, a.rows - base);
        if (base != final) c.load(x + base, n);
        c.store(y + base, [&](float v) { return zero ? 0.0f : __builtin_amdgcn_exp2f(below(a, v, from)) * share; });
        const int64_t k = at - base;
        if (here && k >= 0 && k < n && c.mine((int)k)) y[at] = (T)(zero ? 0.0f : fmaf(__builtin_amdgcn_exp2f(below(a, xt, from)), share, g.up));
      }
    } else if constexpr (MODE == kTop) {
      if (THREADS == 64) __syncthreads();  // else the sums' join was the barrier after the last group
      const int64_t base = (a.rows - 1) / C::kAll * C::kAll;
      list_candidates<THREADS>(c, x + base, (uint32_t)base, bound, base ? top.best[a.top - 1] : 0, top);
      __syncthreads();
      take_top<THREADS>(x + base, (int)(a.rows - base), (uint32_t)base, a.top, top, [&](int at, uint64_t key) {
        const float z = of_rank((uint32_t)(key >> 32)) * a.scale;
        o.top_ids[(int64_t)t * a.top + at] = (int32_t)(~(uint32_t)key + (uint32_t)a.vocab_begin);
        o.top_logp[(int64_t)t * a.top + at] = o.stats || z == -HUGE_VALF ? z : z - l;  // a finite logit whose z is past fp32
      });
      if (t + (int32_t)gridDim.x < a.n) __syncthreads();
    }
  }
}

// L lanes a token: 16 where that many ranks are all (8 ranks of 32768 tokens: 15 us with 64 lanes a token, 6.5 with 16).
template <int L>
__global__ __launch_bounds__(kThreads) void k_join(TokenArgs a, int32_t ranks, const float* stats, const int32_t* ids, const float* zs,
                                                   const void* targets, float* logp, float* lse, float* entropy, int32_t* out_ids,
                                                   float* out_logp) {
  const int lane = threadIdx.x % L;
  const auto most = [](float x) { return mist::wave_join<L>(x, [](float p, float q) { return fmaxf(p, q); }); };
  for (int64_t t = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L; t < a.n; t += (int64_t)gridDim.x * (kThreads / L)) {
    Stats r{-HUGE_VALF, 0.0f, 0.0f, -HUGE_VALF};
    for (int32_t k = lane; k < ranks; k += L) {
      const float4 x = *(const float4*)(stats + ((int64_t)k * a.n + t) * 4);
      r.m = fmaxf(r.m, x.x);
      r.z = fmaxf(r.z, x.w);
    }
    r.m = most(r.m);
    r.z = most(r.z);
    const float from = r.m == -HUGE_VALF ? 0.0f : r.m;
    for (int32_t k = lane; k < ranks; k += L) {
      const float4 x = *(const float4*)(stats + ((int64_t)k * a.n + t) * 4);
      const float d = x.x - from, f = expf(d);
      r.s = fmaf(f, x.y, r.s);
      r.u += f * fmaf(fmaxf(d, kLow), x.y, x.z);
    }
    r.s = wave_sum<L>(r.s);
    r.u = wave_sum<L>(r.u);
    const float l = lse_of(r);
    const int64_t target = targets ? target_of(a, targets, (int32_t)t) : -1;
    if (lane == 0) {
      lse[t] = l;
      if (logp) logp[t] = logp_of(r.z, l, target);
      if (entropy) entropy[t] = entropy_of(r);
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
      uint64_t best = 0;
      for (int64_t j = lane; j < (int64_t)ranks * a.top; j += L) {
        const int64_t at = (j / a.top * a.n + t) * a.top + j % a.top;
        const int32_t id = ids[at];
        const uint32_t rank = rank_of(zs[at]);
        const uint64_t key = id >= 0 ? key_of(rank, (uint32_t)id) : 0;  // a finite logit whose z is past fp32 is one too: rank 0
        if (key > best && key < last) best = key;
      }
      last = best = wave_max_key<L>(best);
      if (lane == 0) {
        const uint32_t rank = (uint32_t)(best >> 32);
        out_ids[t * a.top + k] = best ? (int32_t)~(uint32_t)best : -1;
        out_logp[t * a.top + k] = rank ? of_rank(rank) - l : -HUGE_VALF;
      }
    }
  }
}

// One pass: a block takes a slab of a row.
constexpr int kGradVectors = 2;

template <class T>
__global__ __launch_bounds__(kThreads) void k_grad(TokenArgs a, int32_t slabs, const T* logits, const void* targets, const float* lse, const float* dlogp,
                                                   const float* entropy, const float* dentropy, T* dlogits) {
  using C = Chunk<T, kThreads, kGradVectors, false>;
  for (int64_t i = blockIdx.x; i < (int64_t)a.n * slabs; i += gridDim.x) {
    const int32_t t = (int32_t)(i / slabs);
    const int64_t base = i % slabs * C::kAll;
    const int n = (int)min((int64_t)C::kAll, a.rows - base);
    const int64_t target = dlogp ? target_of(a, targets, t) : -1, at = target < 0 ? -1 : target - a.vocab_begin - base;
    const Slope g = slope_of(lse[t], a.scale, target >= 0 ? dlogp[t] : 0.0f, dentropy ? dentropy[t] : 0.0f, dentropy ? entropy[t] : 0.0f);
    const bool zero = flat(g), here = at >= 0 && at < n;
    const T* x = logits + logits_offset(a, t) + base;
    T* y = dlogits + grad_offset(a, t) + base;
    C c;
    c.load(x, n, !zero);
    const bool owner = here && c.mine((int)at);
    const float xt = owner && !zero ? (float)x[at] : 0.0f;
    c.store(y, [&](float v) { return zero ? 0.0f : slope_at(g, v, a.scale); });
    if (owner && !zero) y[at] = (T)(slope_at(g, xt, a.scale) + g.up);
  }
}

// f(threads, vectors a thread): the smallest block that holds a row in its registers; the largest takes longer ones by chunks.
template <class T, class F>
void with_block(int64_t rows, F&& f) {
  constexpr int kN = 8, kWave = 64 * kN * 16 / (int)sizeof(T);
  if (rows <= kWave) f(std::integral_constant<int, 64>{}, std::integral_constant<int, kN>{});
  else if (rows <= 4 * kWave) f(std::integral_constant<int, 256>{}, std::integral_constant<int, kN>{});
  else if (rows <= 8 * kWave) f(std::integral_constant<int, 512>{}, std::integral_constant<int, kN>{});
  else f(std::integral_constant<int, 512>{}, std::integral_constant<int, 2 * kN>{});
}

mist_status check(const mist_token_desc* d) {
  if (!d) return lib_fail(MIST_E_INVALID, "token log probabilities: null descriptor");
  if (d->batch < 0 || d->seq < 0 || d->batch > INT32_MAX || d->seq > INT32_MAX || (d->batch && d->seq >= kMostTokens / d->batch + (kMostTokens % d->batch != 0)))
    return lib_fail(MIST_E_INVALID, "token log probabilities: batch and seq must be >= 0 with fewer than 2^30 tokens");
  if (d->ids_bytes != 4 && d->ids_bytes != 8) return lib_fail(MIST_E_INVALID, "token log probabilities: targets must be of 4 or 8 bytes");
  if (d->top < 0 || d->top > MIST_TOKEN_MAX_TOP) return lib_fail(MIST_E_INVALID, "token log probabilities: top must be in 0..64");
  if (!mist::stride_ok(d->ids_stride)) return lib_fail(MIST_E_INVALID, "token log probabilities: strides must be in 0..2^40");
  return MIST_OK;
}

mist_status check_logits(const mist_token_desc* d) {
  if (const mist_status st = check(d)) return st;
  if (d->rows < 1 || d->rows > INT32_MAX - 1) return lib_fail(MIST_E_INVALID, "token log probabilities: rows must be in 1..2^31-2");
  if (d->vocab_begin < 0 || d->vocab_begin > INT32_MAX || d->vocab_begin + d->rows > INT32_MAX)
    return lib_fail(MIST_E_INVALID, "token log probabilities: ids must be below 2^31");
  if (!mist::type_ok(d->type)) return lib_fail(MIST_E_INVALID, "token log probabilities: unknown element type");
  if (!std::isfinite(d->scale) || d->scale <= 0.0f) return lib_fail(MIST_E_INVALID, "token log probabilities: scale must be finite and > 0");
  if (!mist::stride_ok(d->logits_batch_stride) || !mist::stride_ok(d->logits_stride))
    return lib_fail(MIST_E_INVALID, "token log probabilities: strides must be in 0..2^40");
  return MIST_OK;
}

mist::Range rows_range(const mist_token_desc* d, const void* p, int64_t batch_stride, int64_t stride) {
  const int64_t bytes = mist::type_bytes(d->type);
  const mist::Range one = mist::range_of(p, d->seq, stride, d->rows, bytes);
  const mist::Range all = mist::range_of(p, d->batch, batch_stride, 1, bytes);
  const uintptr_t more = all.hi - all.lo - bytes, last = one.hi - one.lo;  // to the last sequence, and of it
  return mist::Range{all.lo, last > UINTPTR_MAX - all.lo - more ? UINTPTR_MAX : all.lo + more + last};
}

mist_status check_grad(const mist_token_desc* d, const void* logits, const void* dlogits) {
  const int64_t B = d->batch, S = d->seq, bs = d->grad_batch_stride, s = d->grad_stride, w = d->rows;
  if (!mist::stride_ok(bs) || !mist::stride_ok(s)) return lib_fail(MIST_E_INVALID, "token log probabilities: strides must be in 0..2^40");
  const bool by_batch = (S == 1 || s >= w) && (B == 1 || (__int128)bs >= (__int128)(S - 1) * s + w);
  const bool by_pos = (B == 1 || bs >= w) && (S == 1 || (__int128)s >= (__int128)(B - 1) * bs + w);
  if (!by_batch && !by_pos) return lib_fail(MIST_E_INVALID, "token log probabilities: rows of the gradient overlap");
  const bool same = dlogits == logits && (B == 1 || bs == d->logits_batch_stride) && (S == 1 || s == d->logits_stride);
  if (!same && mist::overlap(rows_range(d, logits, d->logits_batch_stride, d->logits_stride), rows_range(d, dlogits, bs, s)))
    return lib_fail(MIST_E_INVALID, "token log probabilities: the gradient overlaps the logits");
  return MIST_OK;
}

TokenArgs args(const mist_token_desc* d) {
  const float pre = d->scale > 0x1p64f ? 0x1p64f : d->scale < 0x1p-64f ? 0x1p-64f : 1.0f;
  return TokenArgs{d->rows, d->vocab_begin, d->ids_stride, d->logits_batch_stride, d->logits_stride,
                   d->grad_batch_stride, d->grad_stride, (uint32_t)std::max<int64_t>(d->seq, 1), (int32_t)(d->batch * d->seq), d->ids_bytes, d->top, d->scale,
                   pre, (float)(1.44269504088896341 * d->scale / pre)};
}

// The addresses of n values of 4 bytes (2^50 bytes at most: more than there are on any device), and of the targets.
mist::Range values(const void* p, int64_t n) { return mist::range_of(p, 1, 0, std::min<int64_t>(n, (int64_t)1 << 48), 4); }
mist::Range targets_range(const mist_token_desc* d, const void* p) { return mist::range_of(p, d->batch, d->ids_stride, d->seq, d->ids_bytes); }
mist::Range logits_range(const mist_token_desc* d, const void* p) { return rows_range(d, p, d->logits_batch_stride, d->logits_stride); }
mist::Range grad_range(const mist_token_desc* d, const void* p) { return rows_range(d, p, d->grad_batch_stride, d->grad_stride); }
mist_status not_shared(bool shared) { return shared ? lib_fail(MIST_E_INVALID, "token log probabilities: an output overlaps another tensor") : MIST_OK; }

bool floats_ok(std::initializer_list<const float*> ps) {
  for (const float* p : ps)
    if (!mist::is_aligned(p, 4)) return false;
  return true;
}

mist_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, what);
}

mist_status forward(const mist_token_desc* d, const void* logits, const void* targets, float* stats, float* logp, float* lse, float* entropy,
                    int32_t* top_ids, float* top_logp, void* stream) {
  const TokenArgs a = args(d);
  if (a.n == 0) return MIST_OK;
  if (!logits || (!targets && (logp || stats)) || (!stats && !lse) || (d->top && (!top_ids || !top_logp)))
    return lib_fail(MIST_E_INVALID, "token log probabilities: null buffer");
  if (!mist::is_aligned(logits, mist::type_bytes(d->type)) || !mist::is_aligned(targets, d->ids_bytes) || !mist::is_aligned(stats, 16) ||
      !mist::is_aligned(top_ids, 4) || !floats_ok({logp, lse, entropy, top_logp}))
    return lib_fail(MIST_E_INVALID, "token log probabilities: a buffer is not aligned to its elements, or stats to 16");
  const int64_t n = a.n;
  if (const mist_status st = not_shared(mist::shared<mist::Range>({{logits_range(d, logits), false}, {targets_range(d, targets), false}, {values(stats, n * 4), true},
                                                                   {values(logp, n), true}, {values(lse, n), true}, {values(entropy, n), true},
                                                                   {values(top_ids, n * a.top), true}, {values(top_logp, n * a.top), true}})))
    return st;
  const unsigned blocks = (unsigned)std::min<int64_t>(a.n, kMostBlocks);
  mist::with_type(d->type, [&](auto x) {
    using T = typename decltype(x)::type;
    with_block<T>(d->rows, [&](auto threads, auto vectors) {
      const auto kernel = a.top ? k_row<T, threads.value, vectors.value, kTop> : k_row<T, threads.value, vectors.value, kStats>;
      hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads.value), 0, (hipStream_t)stream, a, (const T*)logits, targets,
                         RowOut{stats, logp, lse, entropy, top_ids, top_logp, nullptr, 0.0f}, (T*)nullptr);
    });
  });
  return launched("token log probabilities");
}

}  // namespace

extern "C" {

mist_status mist_token_logprob(const mist_token_desc* d, const void* logits, const void* targets, float* logp, float* lse, float* entropy,
                               int32_t* top_ids, float* top_logp, void* stream) {
  if (const mist_status st = check_logits(d)) return st;
  if (d->vocab_begin) return lib_fail(MIST_E_INVALID, "token log probabilities: a shard gives a part (vocab_begin must be 0)");
  if (d->batch && d->seq && !lse) return lib_fail(MIST_E_INVALID, "token log probabilities: null buffer");
  return forward(d, logits, targets, nullptr, logp, lse, entropy, top_ids, top_logp, stream);
}

mist_status mist_token_part(const mist_token_desc* d, const void* logits, const void* targets, float* stats, int32_t* top_ids, float* top_z,
                            void* stream) {
  if (const mist_status st = check_logits(d)) return st;
  if (d->batch && d->seq && !stats) return lib_fail(MIST_E_INVALID, "token log probabilities: null buffer");
  return forward(d, logits, targets, stats, nullptr, nullptr, nullptr, top_ids, top_z, stream);
}

mist_status mist_token_join(const mist_token_desc* d, int32_t ranks, const float* stats, const int32_t* top_ids, const float* top_z,
                            const void* targets, float* logp, float* lse, float* entropy, int32_t* out_ids, float* out_logp, void* stream) {
  if (const mist_status st = check(d)) return st;
  if (ranks < 1 || ranks > 65536) return lib_fail(MIST_E_INVALID, "token log probabilities: ranks must be in 1..65536");
  const TokenArgs a = args(d);
  if (a.n == 0) return MIST_OK;
  if (!stats || !lse || (logp && !targets) || (d->top && (!top_ids || !top_z || !out_ids || !out_logp)))
    return lib_fail(MIST_E_INVALID, "token log probabilities: null buffer");
  if (!mist::is_aligned(stats, 16) || !mist::is_aligned(targets, d->ids_bytes) || !mist::is_aligned(top_ids, 4) || !mist::is_aligned(out_ids, 4) ||
      !floats_ok({top_z, logp, lse, entropy, out_logp}))
    return lib_fail(MIST_E_INVALID, "token log probabilities: a buffer is not aligned to its elements, or stats to 16");
  const int64_t n = a.n, most = n * a.top;
  if (const mist_status st = not_shared(mist::shared<mist::Range>({{values(stats, ranks * n * 4), false}, {values(top_ids, ranks * most), false}, {values(top_z, ranks * most), false},
                                                                   {targets_range(d, targets), false}, {values(logp, n), true}, {values(lse, n), true},
                                                                   {values(entropy, n), true}, {values(out_ids, most), true}, {values(out_logp, most), true}})))
    return st;
  const int lanes = (int64_t)ranks * std::max(1, a.top) <= 16 ? 16 : 64, tokens = kThreads / lanes;
  const int64_t blocks = std::min<int64_t>((a.n + tokens - 1) / tokens, kMostBlocks);
  hipLaunchKernelGGL(lanes == 16 ? k_join<16> : k_join<64>, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, ranks, stats, top_ids, top_z, targets, logp, lse,
                     entropy, out_ids, out_logp);
  return launched("token log probabilities");
}

mist_status mist_token_grad(const mist_token_desc* d, const void* logits, const void* targets, const float* lse, const float* dlogp,
                            const float* entropy, const float* dentropy, void* dlogits, void* stream) {
  if (const mist_status st = check_logits(d)) return st;
  const TokenArgs a = args(d);
  if (a.n == 0) return MIST_OK;
  if (!logits || !lse || !dlogits || (dlogp && !targets) || (dentropy && !entropy))
    return lib_fail(MIST_E_INVALID, "token log probabilities: null buffer");
  const size_t bytes = (size_t)mist::type_bytes(d->type);
  if (!mist::is_aligned(logits, bytes) || !mist::is_aligned(dlogits, bytes) || !mist::is_aligned(targets, d->ids_bytes) ||
      !floats_ok({lse, dlogp, entropy, dentropy}))
    return lib_fail(MIST_E_INVALID, "token log probabilities: a buffer is not aligned to its elements");
  if (const mist_status st = check_grad(d, logits, dlogits)) return st;
  const int64_t n = a.n;
  if (const mist_status st = not_shared(mist::shared<mist::Range>({{grad_range(d, dlogits), true}, {targets_range(d, targets), false}, {values(lse, n), false},
                                                                   {values(dlogp, n), false}, {values(entropy, n), false}, {values(dentropy, n), false}})))
    return st;
  mist::with_type(d->type, [&](auto x) {
    using T = typename decltype(x)::type;
    constexpr int kSlab = Chunk<T, kThreads, kGradVectors, false>::kAll;
    const int32_t slabs = (int32_t)((d->rows + kSlab - 1) / kSlab);
    const unsigned blocks = (unsigned)std::min<int64_t>((int64_t)a.n * slabs, kMostBlocks);
    hipLaunchKernelGGL((k_grad<T>), dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, a, slabs, (const T*)logits, targets, lse, dlogp, entropy, dentropy,
                       (T*)dlogits);
  });
  return launched("token log probabilities' gradient");
}

mist_status mist_token_loss(const mist_token_desc* d, const void* logits, const void* targets, const float* weights, float weight, float* logp,
                            void* dlogits, void* stream) {
  if (const mist_status st = check_logits(d)) return st;
  if (d->vocab_begin) return lib_fail(MIST_E_INVALID, "token loss: needs the whole vocabulary (vocab_begin must be 0)");
  if (!std::isfinite(weight)) return lib_fail(MIST_E_INVALID, "token loss: weight must be finite");
  const TokenArgs a = args(d);
  if (a.n == 0) return MIST_OK;
  if (!logits || !targets || !logp || !dlogits) return lib_fail(MIST_E_INVALID, "token loss: null buffer");
  const size_t bytes = (size_t)mist::type_bytes(d->type);
  if (!mist::is_aligned(logits, bytes) || !mist::is_aligned(dlogits, bytes) || !mist::is_aligned(targets, d->ids_bytes) || !floats_ok({weights, logp}))
    return lib_fail(MIST_E_INVALID, "token loss: a buffer is not aligned to its elements");
  if (const mist_status st = check_grad(d, logits, dlogits)) return st;
  const int64_t n = a.n;
  if (const mist_status st = not_shared(mist::shared<mist::Range>({{grad_range(d, dlogits), true}, {targets_range(d, targets), false}, {values(weights, n), false}, {values(logp, n), true}}) ||
                                        mist::shared<mist::Range>({{values(logp, n), true}, {logits_range(d, logits), false}})))
    return st;
  const unsigned blocks = (unsigned)std::min<int64_t>(a.n, kMostBlocks);
  mist::with_type(d->type, [&](auto x) {
    using T = typename decltype(x)::type;
    with_block<T>(d->rows, [&](auto threads, auto vectors) {
      hipLaunchKernelGGL((k_row<T, threads.value, vectors.value, kLoss>), dim3(blocks), dim3(threads.value), 0, (hipStream_t)stream, a, (const T*)logits, targets,
                         RowOut{nullptr, logp, nullptr, nullptr, nullptr, nullptr, weights, weight}, (T*)dlogits);
    });
  });
  return launched("token loss");
}

}  // extern "C"
