// Token log probabilities, entropies and alternatives, their gradient, and the loss of a training microbatch.
//
// z = scale * logits is never stored: scale z - m is one fused multiply-add.  A row's largest logit comes first, so that every
// exponential is at most 1 and a row needs no rescaling.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "mist_ops.h"

using mist::fast_exp;
using mist::hip_failed;
using mist::lib_fail;
using mist::wave_max;
using mist::wave_sum;

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostTokens = (int64_t)1 << 30;
constexpr float kLow = -1000.0f;  // of a logarithm, beside an exponential that is 0 there: 0 * kLow is 0 where 0 * -inf is not
constexpr int64_t kMostBlocks = (int64_t)1 << 20;  // a grid stays below 2^32 threads; kernels loop

struct TokenArgs {
  int64_t seq, rows, vocab_begin, ids_stride, logits_batch_stride, logits_stride, grad_batch_stride, grad_stride;
  int32_t n, ids_bytes, top;  // n: tokens
  float scale;
};

__device__ __forceinline__ int64_t target_of(const TokenArgs& a, const void* targets, int32_t t) {
  const int64_t at = t / a.seq * a.ids_stride + t % a.seq;
  return a.ids_bytes == 4 ? ((const int32_t*)targets)[at] : ((const int64_t*)targets)[at];
}
__device__ __forceinline__ int64_t logits_offset(const TokenArgs& a, int32_t t) {
  return t / a.seq * a.logits_batch_stride + t % a.seq * a.logits_stride;
}
__device__ __forceinline__ int64_t grad_offset(const TokenArgs& a, int32_t t) {
  return t / a.seq * a.grad_batch_stride + t % a.seq * a.grad_stride;
}

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

__device__ __forceinline__ uint64_t wave_max_key(uint64_t x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
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

template <class F, class J>
__device__ __forceinline__ float block_join(float x, F wave, J join) {
  __shared__ float part[kThreads / 64];
  x = wave(x);
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
  __syncthreads();
  x = part[0];
  for (int k = 1; k < kThreads / 64; ++k) x = join(x, part[k]);
  return x;
}
__device__ __forceinline__ float block_sum(float x) { return block_join(x, [](float v) { return wave_sum(v); }, [](float p, float q) { return p + q; }); }
__device__ __forceinline__ float block_max(float x) { return block_join(x, [](float v) { return wave_max(v); }, [](float p, float q) { return fmaxf(p, q); }); }

// m, s and u of a row; every thread has them.
template <class T>
__device__ Stats row_stats(const TokenArgs& a, const T* x) {
  float m = -HUGE_VALF;
  for (int64_t j = threadIdx.x; j < a.rows; j += kThreads) m = fmaxf(m, (float)x[j]);
  m = block_max(m) * a.scale;
  const float from = m == -HUGE_VALF ? 0.0f : m;  // nothing is visible: exponentials of -inf, not of NaN
  float s = 0.0f, u = 0.0f;
  for (int64_t j = threadIdx.x; j < a.rows; j += kThreads) {
    const float d = fmaf((float)x[j], a.scale, -from), e = fast_exp(d);
    s += e;
    u = fmaf(e, fmaxf(d, kLow), u);  // a NaN comes with e
  }
  return Stats{m, block_sum(s), block_sum(u), 0.0f};
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_logprob(TokenArgs a, const T* logits, const void* targets, float* stats, float* logp, float* lse,
                                                      float* entropy, int32_t* top_ids, float* top_logp) {
  __shared__ uint64_t part[kThreads / 64];
  for (int32_t t = blockIdx.x; t < a.n; t += gridDim.x) {
    const T* x = logits + logits_offset(a, t);
    Stats r = row_stats(a, x);
    const int64_t target = targets ? target_of(a, targets, t) : -1, at = target - a.vocab_begin;
    r.z = target >= 0 && at >= 0 && at < a.rows ? (float)x[at] * a.scale : -HUGE_VALF;
    const float l = lse_of(r);
    if (threadIdx.x == 0) {
      if (stats) {
        *(float4*)(stats + (int64_t)t * 4) = float4{r.m, r.s, r.u, r.z};
      } else {
        lse[t] = l;
        if (logp) logp[t] = logp_of(r.z, l, target);
        if (entropy) entropy[t] = entropy_of(r);
      }
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
      uint64_t best = 0;
      for (int64_t j = threadIdx.x; j < a.rows; j += kThreads) {
        const uint32_t rank = rank_of((float)x[j]);
        const uint64_t key = rank ? key_of(rank, (uint32_t)j) : 0;
        if (key > best && key < last) best = key;
      }
      best = wave_max_key(best);
      __syncthreads();
      if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = best;
      __syncthreads();
      for (int w = 0; w < kThreads / 64; ++w) best = std::max(best, part[w]);
      last = best;
      if (threadIdx.x == 0) {
        const float z = of_rank((uint32_t)(best >> 32)) * a.scale;
        top_ids[(int64_t)t * a.top + k] = best ? (int32_t)(~(uint32_t)best + (uint32_t)a.vocab_begin) : -1;
        top_logp[(int64_t)t * a.top + k] = !best ? -HUGE_VALF : stats ? z : z - l;
      }
    }
  }
}

// One wave a token.
__global__ __launch_bounds__(kThreads) void k_join(TokenArgs a, int32_t ranks, const float* stats, const int32_t* ids, const float* zs,
                                                   const void* targets, float* logp, float* lse, float* entropy, int32_t* out_ids,
                                                   float* out_logp) {
  const int lane = threadIdx.x % 64;
  for (int64_t t = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64; t < a.n; t += (int64_t)gridDim.x * (kThreads / 64)) {
    Stats r{-HUGE_VALF, 0.0f, 0.0f, -HUGE_VALF};
    for (int32_t k = lane; k < ranks; k += 64) {
      const float4 x = *(const float4*)(stats + ((int64_t)k * a.n + t) * 4);
      r.m = fmaxf(r.m, x.x);
      r.z = fmaxf(r.z, x.w);
    }
    r.m = wave_max(r.m);
    r.z = wave_max(r.z);
    const float from = r.m == -HUGE_VALF ? 0.0f : r.m;
    for (int32_t k = lane; k < ranks; k += 64) {
      const float4 x = *(const float4*)(stats + ((int64_t)k * a.n + t) * 4);
      const float d = x.x - from, f = expf(d);
      r.s = fmaf(f, x.y, r.s);
      r.u += f * fmaf(fmaxf(d, kLow), x.y, x.z);
    }
    r.s = wave_sum(r.s);
    r.u = wave_sum(r.u);
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
      for (int64_t j = lane; j < (int64_t)ranks * a.top; j += 64) {
        const int64_t at = (j / a.top * a.n + t) * a.top + j % a.top;
        const int32_t id = ids[at];
        const uint32_t rank = rank_of(zs[at]);
        const uint64_t key = id >= 0 && rank ? key_of(rank, (uint32_t)id) : 0;
        if (key > best && key < last) best = key;
      }
      last = best = wave_max_key(best);
      if (lane == 0) {
        out_ids[t * a.top + k] = best ? (int32_t)~(uint32_t)best : -1;
        out_logp[t * a.top + k] = best ? of_rank((uint32_t)(best >> 32)) - l : -HUGE_VALF;
      }
    }
  }
}

// A row's gradient, p (c0 + c1 log p) + [j = target] up with scale in the factors.  One without factors is zeros, whatever the
// logits are: they are not looked at.
struct Slope {
  float lse, c0, c1, up;
};
__device__ __forceinline__ bool flat(const Slope& g) { return g.c0 == 0.0f && g.c1 == 0.0f && g.up == 0.0f; }
__device__ __forceinline__ Slope slope_of(float lse, float scale, float dlogp, float dentropy, float entropy) {
  if (lse == -HUGE_VALF) return Slope{0.0f, 0.0f, 0.0f, 0.0f};
  return Slope{lse, scale * (dentropy != 0.0f ? -dlogp - dentropy * entropy : -dlogp), scale * -dentropy, scale * dlogp};
}
__device__ __forceinline__ float slope_at(const Slope& g, float x, float scale) {
  const float l = fmaf(x, scale, -g.lse), p = fast_exp(l);
  return p * fmaf(g.c1, fmaxf(l, kLow), g.c0);
}

template <class T>
__device__ void write_slope(const TokenArgs& a, const Slope& g, const T* x, T* y, int64_t at) {
  const bool zero = flat(g);
  for (int64_t j = threadIdx.x; j < a.rows; j += kThreads) {
    float d = zero ? 0.0f : slope_at(g, (float)x[j], a.scale);
    if (j == at) d += g.up;
    y[j] = (T)d;
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_grad(TokenArgs a, const T* logits, const void* targets, const float* lse, const float* dlogp,
                                                   const float* entropy, const float* dentropy, T* dlogits) {
  for (int32_t t = blockIdx.x; t < a.n; t += gridDim.x) {
    const int64_t target = dlogp ? target_of(a, targets, t) : -1;
    const Slope g = slope_of(lse[t], a.scale, target >= 0 ? dlogp[t] : 0.0f, dentropy ? dentropy[t] : 0.0f, dentropy ? entropy[t] : 0.0f);
    write_slope(a, g, logits + logits_offset(a, t), dlogits + grad_offset(a, t), target < 0 ? -1 : target - a.vocab_begin);
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_loss(TokenArgs a, const T* logits, const void* targets, const float* weights, float weight, float* logp,
                                                   T* dlogits) {
  for (int32_t t = blockIdx.x; t < a.n; t += gridDim.x) {
    const T* x = logits + logits_offset(a, t);
    const int64_t target = target_of(a, targets, t);
    Stats r = row_stats(a, x);
    r.z = target >= 0 && target < a.rows ? (float)x[target] * a.scale : -HUGE_VALF;
    __syncthreads();  // the gradient may overwrite the target's logit
    const float l = lse_of(r);
    if (threadIdx.x == 0) logp[t] = logp_of(r.z, l, target);
    const Slope g = slope_of(l, a.scale, target < 0 ? 0.0f : -(weights ? weight * weights[t] : weight), 0.0f, 0.0f);
    write_slope(a, g, x, dlogits + grad_offset(a, t), target);
  }
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
  return TokenArgs{std::max<int64_t>(d->seq, 1), d->rows, d->vocab_begin, d->ids_stride, d->logits_batch_stride, d->logits_stride,
                   d->grad_batch_stride, d->grad_stride, (int32_t)(d->batch * d->seq), d->ids_bytes, d->top, d->scale};
}

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
  const unsigned blocks = (unsigned)std::min<int64_t>(a.n, kMostBlocks);
  mist::with_type(d->type, [&](auto x) {
    using T = typename decltype(x)::type;
    hipLaunchKernelGGL((k_logprob<T>), dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const T*)logits, targets, stats, logp, lse,
                       entropy, top_ids, top_logp);
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
  const int64_t blocks = std::min<int64_t>((a.n + kThreads / 64 - 1) / (kThreads / 64), kMostBlocks);
  hipLaunchKernelGGL(k_join, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a, ranks, stats, top_ids, top_z, targets, logp, lse,
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
  const unsigned blocks = (unsigned)std::min<int64_t>(a.n, kMostBlocks);
  mist::with_type(d->type, [&](auto x) {
    using T = typename decltype(x)::type;
    hipLaunchKernelGGL((k_grad<T>), dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const T*)logits, targets, lse, dlogp, entropy, dentropy,
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
  const unsigned blocks = (unsigned)std::min<int64_t>(a.n, kMostBlocks);
  mist::with_type(d->type, [&](auto x) {
    using T = typename decltype(x)::type;
    hipLaunchKernelGGL((k_loss<T>), dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, a, (const T*)logits, targets, weights, weight, logp,
                       (T*)dlogits);
  });
  return launched("token loss");
}

}  // extern "C"
