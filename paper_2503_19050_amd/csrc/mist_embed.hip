// The first stage's embedding, a vocabulary-parallel table with learned positions, and its gradient.
#include <hip/hip_runtime.h>

#include <cmath>

#include "mist_ops.h"

namespace {

using mist::hip_failed;
using mist::lib_fail;

constexpr int kThreads = 256;

struct EmbedArgs {
  int64_t batch, seq, hidden, rows, begin;
  int64_t ids_stride, act_batch_stride, act_stride, table_stride, pos_stride;
  int32_t ids_bytes;
  float scale;
};

// Row of the shard that token (b, s) finds, or -1.
__device__ __forceinline__ int32_t token_row(const EmbedArgs& a, const void* ids, int64_t b, int64_t s) {
  const int64_t at = b * a.ids_stride + s;
  const int64_t id = a.ids_bytes == 4 ? (int64_t)((const int32_t*)ids)[at] : ((const int64_t*)ids)[at];
  return id >= a.begin && id - a.begin < a.rows ? (int32_t)(id - a.begin) : -1;
}

// One block a token.
template <class A, class W>
__global__ __launch_bounds__(kThreads) void k_embed(EmbedArgs a, const void* __restrict__ ids, const W* __restrict__ table,
                                                    const W* __restrict__ pos, A* __restrict__ out) {
  const int64_t b = blockIdx.x / a.seq, s = blockIdx.x % a.seq;
  const int32_t row = token_row(a, ids, b, s);
  for (int64_t c = threadIdx.x; c < a.hidden; c += kThreads) {
    float x = row >= 0 ? a.scale * (float)table[row * a.table_stride + c] : 0.0f;
    if (pos) x += (float)pos[s * a.pos_stride + c];
    out[b * a.act_batch_stride + s * a.act_stride + c] = (A)x;
  }
}

// Place of each token in the order by (row, token): the number of tokens before it in that order.
// Tokens of no row are left out.
__global__ __launch_bounds__(kThreads) void k_rank(EmbedArgs a, const void* __restrict__ ids, int32_t n,
                                                   int32_t* __restrict__ token, int32_t* __restrict__ row_of) {
  const int32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const int32_t row = token_row(a, ids, i / a.seq, i % a.seq);
  int32_t place = 0, kept = 0;
  for (int32_t j = 0; j < n; ++j) {
    const int32_t other = token_row(a, ids, j / a.seq, j % a.seq);
    place += other >= 0 && (other < row || (other == row && j < i));
    kept += other >= 0;
  }
  if (row >= 0) {
    token[place] = i;
    row_of[place] = row;
  }
  if (i >= kept) row_of[i] = INT32_MAX;  // places that no token takes
}

// One block a table row: finds its tokens and adds them up in order.
template <class A, class W>
__global__ __launch_bounds__(kThreads) void k_dtable(EmbedArgs a, const A* __restrict__ grad, int32_t n,
                                                     const int32_t* __restrict__ token, const int32_t* __restrict__ row_of,
                                                     W* __restrict__ dtable, int32_t accumulate) {
  const int32_t row = blockIdx.x;
  int32_t lo = 0, hi = n;  // first place of a row not below this one
  while (lo < hi) {
    const int32_t mid = (lo + hi) / 2;
    if (row_of[mid] < row) lo = mid + 1;
    else hi = mid;
  }
  if (accumulate && (lo == n || row_of[lo] != row)) return;
  for (int64_t c = threadIdx.x; c < a.hidden; c += kThreads) {
    float sum = 0.0f;
    for (int32_t k = lo; k < n && row_of[k] == row; ++k) {
      const int64_t i = token[k];
      sum += (float)grad[i / a.seq * a.act_batch_stride + i % a.seq * a.act_stride + c];
    }
    W* d = dtable + row * a.table_stride + c;
    *d = (W)(accumulate ? (float)*d + a.scale * sum : a.scale * sum);
  }
}

// One block a position.
template <class A, class W>
__global__ __launch_bounds__(kThreads) void k_dpos(EmbedArgs a, const A* __restrict__ grad, W* __restrict__ dpos,
                                                   int32_t accumulate) {
  const int64_t s = blockIdx.x;
  for (int64_t c = threadIdx.x; c < a.hidden; c += kThreads) {
    float sum = 0.0f;
    for (int64_t b = 0; b < a.batch; ++b) sum += (float)grad[b * a.act_batch_stride + s * a.act_stride + c];
    W* d = dpos + s * a.pos_stride + c;
    *d = (W)(accumulate ? (float)*d + sum : sum);
  }
}

mist_status check(const mist_embed_desc* d, bool out) {
  if (!d) return lib_fail(MIST_E_INVALID, "embedding: null descriptor");
  if (d->batch < 0 || d->seq < 0 || (d->batch && d->seq > INT32_MAX / d->batch))
    return lib_fail(MIST_E_INVALID, "embedding: batch and seq must be >= 0 with fewer than 2^31 tokens");
  if (d->hidden < 1 || d->hidden > (1 << 24)) return lib_fail(MIST_E_INVALID, "embedding: hidden must be in 1..2^24");
  if (d->rows < 1 || d->rows > INT32_MAX - 1) return lib_fail(MIST_E_INVALID, "embedding: rows must be in 1..2^31-2");
  if (d->vocab_begin < 0 || d->vocab_begin > INT32_MAX)
    return lib_fail(MIST_E_INVALID, "embedding: vocab_begin must be in [0, 2^31)");
  if (d->ids_bytes != 4 && d->ids_bytes != 8) return lib_fail(MIST_E_INVALID, "embedding: ids must be of 4 or 8 bytes");
  if (!mist::type_ok(d->act_type) || !mist::type_ok(d->table_type))
    return lib_fail(MIST_E_INVALID, "embedding: unknown element type");
  if (!std::isfinite(d->scale)) return lib_fail(MIST_E_INVALID, "embedding: scale must be finite");
  const int64_t most = (int64_t)1 << 40;  // products of strides with their counts stay below 2^63
  for (int64_t x : {d->ids_stride, d->act_batch_stride, d->act_stride, d->table_stride, d->pos_stride})
    if (x < 0 || x > most) return lib_fail(MIST_E_INVALID, "embedding: strides must be in 0..2^40");
  if (d->table_stride < d->hidden && d->rows > 1)
    return lib_fail(MIST_E_INVALID, "embedding: rows of the table overlap (table_stride < hidden)");
  if (out && d->batch && d->seq) {
    const int64_t h = d->hidden, B = d->batch, S = d->seq, bs = d->act_batch_stride, s = d->act_stride;
    const bool by_batch = (S == 1 || s >= h) && (B == 1 || (__int128)bs >= (__int128)(S - 1) * s + h);
    const bool by_pos = (B == 1 || bs >= h) && (S == 1 || (__int128)s >= (__int128)(B - 1) * bs + h);
    if (!by_batch && !by_pos) return lib_fail(MIST_E_INVALID, "embedding: positions of the output overlap");
  }
  return MIST_OK;
}

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

EmbedArgs args(const mist_embed_desc* d) {
  return EmbedArgs{d->batch, d->seq, d->hidden, d->rows, d->vocab_begin, d->ids_stride, d->act_batch_stride,
                   d->act_stride, d->table_stride, d->pos_stride, d->ids_bytes, d->scale};
}

}  // namespace

extern "C" {

mist_status mist_embed_forward(const mist_embed_desc* d, const void* ids, const void* table, const void* pos, void* out,
                               void* stream) {
  if (const mist_status st = check(d, true)) return st;
  const int64_t n = d->batch * d->seq;
  if (n == 0) return MIST_OK;
  if (!ids || !table || !out) return lib_fail(MIST_E_INVALID, "embedding: null buffer");
  if (pos && d->seq > 1 && d->pos_stride < d->hidden)
    return lib_fail(MIST_E_INVALID, "embedding: rows of the positions overlap (pos_stride < hidden)");
  if (!aligned(ids, d->ids_bytes) || !aligned(out, mist::type_bytes(d->act_type)) ||
      !aligned(table, mist::type_bytes(d->table_type)) || !aligned(pos, mist::type_bytes(d->table_type)))
    return lib_fail(MIST_E_INVALID, "embedding: a buffer is not aligned to its elements");
  const EmbedArgs a = args(d);
  mist::with_types(d->act_type, d->table_type, [&](auto x, auto w) {
    using A = typename decltype(x)::type;
    using W = typename decltype(w)::type;
    hipLaunchKernelGGL((k_embed<A, W>), dim3((unsigned)n), dim3(kThreads), 0, (hipStream_t)stream, a, ids, (const W*)table,
                       (const W*)pos, (A*)out);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "embedding");
}

mist_status mist_embed_workspace(const mist_embed_desc* d, size_t* bytes) {
  if (!bytes) return lib_fail(MIST_E_INVALID, "embedding: null argument");
  if (const mist_status st = check(d, false)) return st;
  *bytes = (size_t)(d->batch * d->seq) * 8;
  return MIST_OK;
}

mist_status mist_embed_backward(const mist_embed_desc* d, const void* ids, const void* grad, void* dtable, void* dpos,
                                int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  if (const mist_status st = mist_embed_workspace(d, &need)) return st;
  if (accumulate != 0 && accumulate != 1) return lib_fail(MIST_E_INVALID, "embedding: accumulate must be 0 or 1");
  const int64_t n = d->batch * d->seq;
  if (!dtable || (n && (!ids || !grad))) return lib_fail(MIST_E_INVALID, "embedding: null buffer");
  if (need && !workspace) return lib_fail(MIST_E_INVALID, "embedding: null workspace");
  if (workspace_bytes < need) return lib_fail(MIST_E_RANGE, "embedding: workspace too small");
  if (dpos && d->seq > 1 && d->pos_stride < d->hidden)
    return lib_fail(MIST_E_INVALID, "embedding: rows of the positions overlap (pos_stride < hidden)");
  if (!aligned(ids, d->ids_bytes) || !aligned(grad, mist::type_bytes(d->act_type)) ||
      !aligned(dtable, mist::type_bytes(d->table_type)) || !aligned(dpos, mist::type_bytes(d->table_type)) ||
      !aligned(workspace, 256))
    return lib_fail(MIST_E_INVALID, "embedding: a buffer is not aligned to its elements, or the workspace to 256");
  const EmbedArgs a = args(d);
  const hipStream_t st = (hipStream_t)stream;
  int32_t* token = (int32_t*)workspace;
  int32_t* row_of = token + n;
  if (n) hipLaunchKernelGGL(k_rank, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, a, ids, (int32_t)n, token, row_of);
  mist::with_types(d->act_type, d->table_type, [&](auto x, auto w) {
    using A = typename decltype(x)::type;
    using W = typename decltype(w)::type;
    hipLaunchKernelGGL((k_dtable<A, W>), dim3((unsigned)d->rows), dim3(kThreads), 0, st, a, (const A*)grad, (int32_t)n, token,
                       row_of, (W*)dtable, accumulate);
    if (dpos && d->seq)
      hipLaunchKernelGGL((k_dpos<A, W>), dim3((unsigned)d->seq), dim3(kThreads), 0, st, a, (const A*)grad, (W*)dpos, accumulate);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "embedding gradient");
}

}  // extern "C"
