// The first stage's embedding, a vocabulary-parallel table with learned positions, and its gradient.
//
// Both are bound by memory.  The lookup gathers rows and writes activations.  The gradient orders the
// tokens by row (stable, so that a row's terms are added in token order whatever ran first), sums each
// row's terms in fp32 registers and writes the row once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "mist_ops.h"

namespace {

using mist::hip_failed;
using mist::lib_fail;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kVec = 8;             // values of a lane
constexpr int kSlab = 64 * kVec;    // columns of a wave
constexpr int64_t kMostTokens = (int64_t)1 << 30;  // places past the last token stay below 2^31
constexpr int kChunk = 64;          // ordered tokens of a wave, one a lane

struct EmbedArgs {
  int64_t batch, seq, hidden, rows, begin;
  int64_t ids_stride, act_batch_stride, act_stride, table_stride, pos_stride;
  int32_t ids_bytes;
  float scale;
  int32_t n;      // tokens
  int32_t slabs;  // column slabs
};

// An ordered token: its row (args.rows: no row of the shard) and its index b * seq + s.
struct Entry {
  uint32_t row, token;
};

typedef float Float8 __attribute__((ext_vector_type(8), aligned(16)));

// Eight values of one lane.  VEC: consecutive, 16 bytes a load; otherwise 64 columns apart, one by one
// (for rows that are not aligned to 16 bytes, or of a size that is no multiple of 8).
template <bool VEC>
__device__ __forceinline__ int64_t first_col(int32_t slab) {
  const int lane = threadIdx.x % 64;
  return (int64_t)slab * kSlab + (VEC ? lane * kVec : lane);
}

template <class T, bool VEC>
struct Lane8 {
  typedef T type __attribute__((ext_vector_type(8), aligned(16)));
  type v;
  __device__ __forceinline__ void load(const T* row, int64_t col, int64_t hidden) {
    if (VEC) {
      v = col < hidden ? *(const type*)(row + col) : type{};
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] = col + 64 * k < hidden ? row[col + 64 * k] : (T)0.0f;
    }
  }
  __device__ __forceinline__ Float8 get() const { return __builtin_convertvector(v, Float8); }
  static __device__ __forceinline__ void store(T* row, int64_t col, int64_t hidden, Float8 x) {
    const type y = __builtin_convertvector(x, type);
    if (VEC) {
      if (col < hidden) *(type*)(row + col) = y;
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k)
        if (col + 64 * k < hidden) row[col + 64 * k] = y[k];
    }
  }
};

__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

__device__ __forceinline__ int32_t wave_index() {
  return __builtin_amdgcn_readfirstlane((int32_t)(blockIdx.x * kWaves + threadIdx.x / 64));
}

// Row of the shard that token (b, s) finds; args.rows if none.
__device__ __forceinline__ uint32_t token_row(const EmbedArgs& a, const void* ids, uint32_t token) {
  const uint32_t b = token / (uint32_t)a.seq, s = token % (uint32_t)a.seq;
  const int64_t at = b * a.ids_stride + s;
  const int64_t id = a.ids_bytes == 4 ? (int64_t)((const int32_t*)ids)[at] : ((const int64_t*)ids)[at];
  return id >= a.begin && id - a.begin < a.rows ? (uint32_t)(id - a.begin) : (uint32_t)a.rows;
}

__device__ __forceinline__ int64_t act_offset(const EmbedArgs& a, uint32_t token) {
  return token / (uint32_t)a.seq * a.act_batch_stride + token % (uint32_t)a.seq * a.act_stride;
}

// ---- lookup ----------------------------------------------------------------------------------------
// A wave takes `per_wave` (at most 64) tokens and one slab of columns, kAhead rows in flight.  With
// positions the tokens are taken position by position, so that the batch shares a position's row in
// the cache.
constexpr int kAhead = 8;

template <class A, class W, bool VEC, bool POS>
__global__ __launch_bounds__(kThreads) void k_embed(EmbedArgs a, int32_t per_wave, const void* __restrict__ ids,
                                                    const W* __restrict__ table, const W* __restrict__ pos, A* __restrict__ out) {
  const int64_t wave = wave_index();
  const int32_t slab = (int32_t)(wave % a.slabs);
  const int64_t first = wave / a.slabs * per_wave;
  if (first >= a.n) return;
  const int32_t count = (int32_t)(a.n - first < per_wave ? a.n - first : per_wave);
  const int lane = threadIdx.x % 64;
  uint32_t token = (uint32_t)first + (lane < count ? lane : 0);
  if (POS) token = token % (uint32_t)a.batch * (uint32_t)a.seq + token / (uint32_t)a.batch;
  const uint32_t row = token_row(a, ids, token);
  const int64_t row_at = row < a.rows ? row * a.table_stride : -1;
  const int64_t out_at = act_offset(a, token);
  const uint32_t s = token % (uint32_t)a.seq;
  const int64_t col = first_col<VEC>(slab);
  for (int k0 = 0; k0 < count; k0 += kAhead) {
    Lane8<W, VEC> x[kAhead], p[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k0 + k < count) {
        const int64_t at = lane_value(row_at, k0 + k);
        if (at >= 0) x[k].load(table + at, col, a.hidden);
        else x[k].v = {};
        if (POS) p[k].load(pos + lane_value(s, k0 + k) * a.pos_stride, col, a.hidden);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k0 + k < count) {
        Float8 y = a.scale * x[k].get();
        if (POS) y += p[k].get();
        Lane8<A, VEC>::store(out + lane_value(out_at, k0 + k), col, a.hidden, y);
      }
    }
  }
}

// ---- order of the tokens ---------------------------------------------------------------------------
// Short inputs: a token's place is the number of tokens before it by (row, token), counted directly;
// one launch.  A block places 16 tokens against all of them, 16 lanes a token.
constexpr int32_t kCounted = 8192;   // tokens up to which places are counted
constexpr int kPlaced = 16;

__global__ __launch_bounds__(kThreads) void k_place(EmbedArgs a, const void* __restrict__ ids, Entry* __restrict__ out) {
  __shared__ uint32_t row[kCounted];
  for (int32_t i = threadIdx.x; i < a.n; i += kThreads) row[i] = token_row(a, ids, i);
  __syncthreads();
  const int32_t i = blockIdx.x * kPlaced + threadIdx.x / 16;
  const uint32_t mine = row[i < a.n ? i : 0];
  int32_t place = 0;
  for (int32_t j = threadIdx.x % 16; j < a.n; j += 16) place += row[j] < mine || (row[j] == mine && j < i);
  for (int d = 8; d; d >>= 1) place += __shfl_xor(place, d);
  if (threadIdx.x % 16 == 0 && i < a.n) out[place] = Entry{mine, (uint32_t)i};
}

// Long inputs: radix order, least significant digit first, each pass stable.  A pass counts the digits
// of every tile, then moves each tile's tokens to their digits' places; a tile's waves take consecutive
// tokens, a wave's lanes find their equals with one ballot a digit bit.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMaxTiles = 128;
constexpr int kMaxDigits = 512;      // 9 bits

struct SortArgs {
  const Entry* in;    // nullptr: the tokens themselves
  Entry* out;
  int32_t* hist;      // [tiles][digits]
  int32_t n, tile, tiles, shift, bits;
};

__device__ __forceinline__ Entry sort_entry(const EmbedArgs& a, const SortArgs& s, const void* ids, int32_t i) {
  return s.in ? s.in[i] : Entry{token_row(a, ids, i), (uint32_t)i};
}

__global__ __launch_bounds__(kSortThreads) void k_digits(EmbedArgs a, SortArgs s, const void* __restrict__ ids) {
  __shared__ int32_t count[kMaxDigits];
  const int32_t digits = 1 << s.bits;
  for (int32_t d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
  __syncthreads();
  const int32_t end = min(s.n, ((int32_t)blockIdx.x + 1) * s.tile);
  for (int32_t i = blockIdx.x * s.tile + threadIdx.x; i < end; i += kSortThreads)
    atomicAdd(&count[sort_entry(a, s, ids, i).row >> s.shift & (digits - 1)], 1);
  __syncthreads();
  for (int32_t d = threadIdx.x; d < digits; d += kSortThreads) s.hist[blockIdx.x * digits + d] = count[d];
}

// Lanes of the wave whose digit is this lane's (live: those that have one).
__device__ __forceinline__ uint64_t equals(uint32_t digit, int bits, bool live) {
  uint64_t m = __ballot(live);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    m &= digit >> b & 1 ? set : ~set;
  }
  return m;
}

__global__ __launch_bounds__(kSortThreads) void k_move(EmbedArgs a, SortArgs s, const void* __restrict__ ids) {
  __shared__ int32_t at[kSortWaves][kMaxDigits];  // counts, then places
  __shared__ int32_t scan[kMaxDigits], before[kMaxDigits];
  const int32_t digits = 1 << s.bits, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  for (int32_t d = threadIdx.x; d < kSortWaves * kMaxDigits; d += kSortThreads) (&at[0][0])[d] = 0;
  // digit d: its tokens in all tiles, and in the tiles before this one
  if ((int32_t)threadIdx.x < digits) {
    int32_t total = 0, mine = 0;
    for (int32_t t = 0; t < s.tiles; ++t) {
      const int32_t c = s.hist[t * digits + threadIdx.x];
      total += c;
      mine += t < (int32_t)blockIdx.x ? c : 0;
    }
    scan[threadIdx.x] = total;
    before[threadIdx.x] = mine;
  }
  __syncthreads();
  for (int32_t d = 1; d < digits; d <<= 1) {
    const int32_t x = (int32_t)threadIdx.x < digits && (int32_t)threadIdx.x >= d ? scan[threadIdx.x - d] : 0;
    __syncthreads();
    if ((int32_t)threadIdx.x < digits) scan[threadIdx.x] += x;
    __syncthreads();
  }
  const int32_t per_wave = s.tile / kSortWaves;   // a multiple of 64
  const int32_t begin = blockIdx.x * s.tile + wave * per_wave, end = min(s.n, begin + per_wave);
  for (int32_t i0 = begin; i0 < end; i0 += 64) {
    const bool live = i0 + lane < end;
    const Entry e = sort_entry(a, s, ids, live ? i0 + lane : begin);
    const uint32_t digit = e.row >> s.shift & (digits - 1);
    const uint64_t m = equals(digit, s.bits, live);
    if (live && (m & ((1ull << lane) - 1)) == 0) at[wave][digit] += __popcll(m);
    __builtin_amdgcn_wave_barrier();  // the next round's lanes read what this one's wrote
  }
  __syncthreads();
  if ((int32_t)threadIdx.x < digits) {
    int32_t sum = (threadIdx.x ? scan[threadIdx.x - 1] : 0) + before[threadIdx.x];
    for (int w = 0; w < kSortWaves; ++w) {
      const int32_t c = at[w][threadIdx.x];
      at[w][threadIdx.x] = sum;
      sum += c;
    }
  }
  __syncthreads();
  for (int32_t i0 = begin; i0 < end; i0 += 64) {
    const bool live = i0 + lane < end;
    const Entry e = sort_entry(a, s, ids, live ? i0 + lane : begin);
    const uint32_t digit = e.row >> s.shift & (digits - 1);
    const uint64_t m = equals(digit, s.bits, live);
    const int32_t before_me = __popcll(m & ((1ull << lane) - 1));
    const int32_t place = at[wave][digit];
    if (live) s.out[place + before_me] = e;
    __builtin_amdgcn_wave_barrier();
    if (live && before_me == 0) at[wave][digit] = place + __popcll(m);
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- sums of the rows ------------------------------------------------------------------------------
// A wave takes a chunk of 64 ordered tokens and a slab of columns, and adds up runs of equal rows in
// registers.  A run that crosses one chunk boundary is finished by the chunk where it begins.  A run that
// touches three chunks or more is long: each chunk leaves its piece in `part`, slot 1 the chunk where
// the run begins and slot 0 the others, and k_join adds the pieces in order.
struct RowArgs {
  const Entry* order;
  float* part;          // [chunks][2][slabs][kSlab], in lane order
  int32_t chunks;
  int32_t accumulate;
  int64_t sum_waves;    // waves that sum chunks; the rest, one a row, clear rows without a token
};

__device__ __forceinline__ uint32_t row_at(const RowArgs& r, const EmbedArgs& a, int64_t i) {
  return i >= 0 && i < a.n ? r.order[i].row : (uint32_t)a.rows;
}

template <class A, class W, bool VEC>
struct RowSum {
  const EmbedArgs& a;
  const RowArgs& r;
  const A* grad;
  W* dtable;
  int32_t chunk, slab;
  int64_t col;
  Float8 acc = {};
  static constexpr int kGroup = sizeof(A) == 2 ? 8 : 4;

  __device__ __forceinline__ void part_out(int slot) {
    float* p = r.part + (((int64_t)chunk * 2 + slot) * a.slabs + slab) * kSlab + threadIdx.x % 64 * kVec;
    *(Float8*)p = acc;
  }

  // Tokens [from, to) of the 64 whose rows and offsets the lanes hold.  `next` is the row after the last
  // lane's.  slot >= 0: the range is one piece of a long run.
  __device__ __forceinline__ void take(uint32_t row, int64_t offset, int from, int to, uint32_t next, int slot) {
    for (int k0 = from; k0 < to; k0 += kGroup) {
      Lane8<A, VEC> x[kGroup];
      Lane8<W, VEC> old[kGroup];
      bool ends[kGroup];
      uint32_t mine[kGroup];
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        if (k0 + k < to) {
          mine[k] = lane_value(row, k0 + k);
          ends[k] = slot < 0 && mine[k] != (k0 + k < 63 ? lane_value(row, k0 + k + 1) : next);
          x[k].load(grad + lane_value(offset, k0 + k), col, a.hidden);
          if (r.accumulate && ends[k]) old[k].load(dtable + mine[k] * a.table_stride, col, a.hidden);
        }
      }
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        if (k0 + k < to) {
          acc += x[k].get();
          if (ends[k]) {
            Float8 y = a.scale * acc;
            if (r.accumulate) y += old[k].get();
            Lane8<W, VEC>::store(dtable + mine[k] * a.table_stride, col, a.hidden, y);
            acc = Float8{};
          }
        }
      }
    }
    if (slot >= 0) {
      part_out(slot);
      acc = Float8{};
    }
  }

  __device__ __forceinline__ void run() {
    const int64_t base = (int64_t)chunk * kChunk;
    const int lane = threadIdx.x % 64;
    const uint32_t none = (uint32_t)a.rows;
    const bool in0 = base + lane < a.n, in1 = base + 64 + lane < a.n;
    const Entry e0 = in0 ? r.order[base + lane] : Entry{none, 0}, e1 = in1 ? r.order[base + 64 + lane] : Entry{none, 0};
    const uint32_t first = lane_value(e0.row, 0), last = lane_value(e0.row, 63), after = lane_value(e1.row, 0);
    if (first == none) return;
    const uint32_t before = row_at(r, a, base - 1);
    const int64_t off0 = act_offset(a, e0.token);
    const int valid = __popcll(__ballot(e0.row != none));
    int from = 0;
    if (chunk > 0 && before == first) {  // the first run began earlier
      const int lead = __popcll(__ballot(e0.row == first));
      const bool short_run = row_at(r, a, base - 65) != first && after != first;
      if (!short_run) take(e0.row, off0, 0, lead, none, 0);
      from = lead;
    }
    if (from == valid) return;
    const bool goes_on = last != none && after == last;  // the last run begins here and crosses the boundary
    if (!goes_on) {
      take(e0.row, off0, from, valid, after, -1);
      return;
    }
    const int tail = 64 - __popcll(__ballot(e0.row == last));  // where it begins
    if (row_at(r, a, base + 128) != last) {
      take(e0.row, off0, from, 64, after, -1);
      const int more = __popcll(__ballot(e1.row == last));
      take(e1.row, act_offset(a, e1.token), 0, more, none, -1);
    } else {
      take(e0.row, off0, from, tail, after, -1);
      take(e0.row, off0, tail, 64, after, 1);
    }
  }
};

// Whether a token has the row: a search with 64 probes a step.
__device__ __forceinline__ bool has_token(const RowArgs& r, int32_t n, uint32_t row) {
  const int lane = threadIdx.x % 64;
  int32_t lo = 0, hi = n;   // the first place of a row not below is in [lo, hi]
  while (hi - lo > 63) {
    const int32_t step = (hi - lo + 63) / 64;
    const int32_t at = lo + lane * step;
    const int below = __popcll(__ballot(at < hi && r.order[at < hi ? at : lo].row < row));
    if (below == 0) return r.order[lo].row == row;
    hi = min(hi, lo + below * step);
    lo = lo + (below - 1) * step + 1;
  }
  const int32_t at = lo + lane;
  return __ballot(at < n && r.order[at < n ? at : 0].row == row) != 0;
}

template <class A, class W, bool VEC>
__global__ __launch_bounds__(kThreads) void k_rows(EmbedArgs a, RowArgs r, const A* __restrict__ grad, W* __restrict__ dtable) {
  const int64_t waves = (int64_t)gridDim.x * kWaves, all = r.sum_waves + (r.accumulate ? 0 : a.rows);
  for (int64_t w = wave_index(); w < all; w += waves) {
    if (w < r.sum_waves) {
      const int32_t chunk = (int32_t)(w / a.slabs), slab = (int32_t)(w % a.slabs);
      RowSum<A, W, VEC> s{a, r, grad, dtable, chunk, slab, first_col<VEC>(slab)};
      s.run();
    } else {
      const uint32_t row = (uint32_t)(w - r.sum_waves);
      if (a.n && has_token(r, a.n, row)) continue;
      for (int32_t slab = 0; slab < a.slabs; ++slab)
        Lane8<W, VEC>::store(dtable + row * a.table_stride, first_col<VEC>(slab), a.hidden, Float8{});
    }
  }
}

// Long runs that begin in the block's chunks: the waves add up a quarter of the pieces each, in
// order, and the quarters are added in order.
constexpr int kJoinChunks = 16;

template <class W, bool VEC>
__global__ __launch_bounds__(kThreads) void k_join(EmbedArgs a, RowArgs r, W* __restrict__ dtable) {
  __shared__ Float8 quarter[kWaves][64];
  const int32_t slab = (int32_t)(blockIdx.x % a.slabs), wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int32_t first = (int32_t)(blockIdx.x / a.slabs) * kJoinChunks;
  for (int32_t c = first; c < first + kJoinChunks && c < r.chunks; ++c) {
    const int64_t base = (int64_t)c * kChunk;
    const uint32_t row = row_at(r, a, base + 63);
    if (row == (uint32_t)a.rows || row_at(r, a, base - 1) == row || row_at(r, a, base + 64) != row || row_at(r, a, base + 128) != row)
      continue;
    int32_t end = c + 2;  // the run's chunks are [c, end)
    for (;;) {
      const uint64_t in = __ballot(row_at(r, a, (int64_t)(end + lane) * kChunk) == row);
      end += in == ~0ull ? 64 : __ffsll((unsigned long long)~in) - 1;
      if (in != ~0ull) break;
    }
    const int32_t pieces = end - c, share = (pieces + kWaves - 1) / kWaves;
    Float8 acc = {};
    const int32_t to = min(pieces, (wave + 1) * share);
#pragma unroll 4
    for (int32_t k = wave * share; k < to; ++k)
      acc += *(const Float8*)(r.part + (((int64_t)(c + k) * 2 + (k == 0)) * a.slabs + slab) * kSlab + lane * kVec);
    quarter[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
      for (int w = 1; w < kWaves; ++w) acc += quarter[w][lane];
      const int64_t col = first_col<VEC>(slab);
      W* d = dtable + row * a.table_stride;
      Float8 y = a.scale * acc;
      if (r.accumulate) {
        Lane8<W, VEC> old;
        old.load(d, col, a.hidden);
        y += old.get();
      }
      Lane8<W, VEC>::store(d, col, a.hidden, y);
    }
    __syncthreads();
  }
}

// A wave takes a position and a slab, and adds up the batch.
template <class A, class W, bool VEC>
__global__ __launch_bounds__(kThreads) void k_dpos(EmbedArgs a, const A* __restrict__ grad, W* __restrict__ dpos,
                                                   int32_t accumulate) {
  const int64_t waves = (int64_t)gridDim.x * kWaves, all = a.seq * a.slabs;
  for (int64_t w = wave_index(); w < all; w += waves) {
    const int64_t s = w / a.slabs, col = first_col<VEC>((int32_t)(w % a.slabs));
    Float8 acc = {};
    for (int64_t b0 = 0; b0 < a.batch; b0 += kAhead) {
      Lane8<A, VEC> x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (b0 + k < a.batch) x[k].load(grad + (b0 + k) * a.act_batch_stride + s * a.act_stride, col, a.hidden);
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (b0 + k < a.batch) acc += x[k].get();
    }
    W* d = dpos + s * a.pos_stride;
    if (accumulate) {
      Lane8<W, VEC> old;
      old.load(d, col, a.hidden);
      acc += old.get();
    }
    Lane8<W, VEC>::store(d, col, a.hidden, acc);
  }
}

// ---- host ------------------------------------------------------------------------------------------
mist_status check(const mist_embed_desc* d, bool out) {
  if (!d) return lib_fail(MIST_E_INVALID, "embedding: null descriptor");
  if (d->batch < 0 || d->seq < 0 || d->batch > INT32_MAX || d->seq > INT32_MAX || (d->batch && d->seq >= kMostTokens / d->batch + (kMostTokens % d->batch != 0)))
    return lib_fail(MIST_E_INVALID, "embedding: batch and seq must be >= 0 with fewer than 2^30 tokens");
  if (d->hidden < 1 || d->hidden > (1 << 24)) return lib_fail(MIST_E_INVALID, "embedding: hidden must be in 1..2^24");
  if (d->rows < 1 || d->rows > INT32_MAX - 1) return lib_fail(MIST_E_INVALID, "embedding: rows must be in 1..2^31-2");
  if (d->vocab_begin < 0 || d->vocab_begin > INT32_MAX)
    return lib_fail(MIST_E_INVALID, "embedding: vocab_begin must be in [0, 2^31)");
  if (d->ids_bytes != 4 && d->ids_bytes != 8) return lib_fail(MIST_E_INVALID, "embedding: ids must be of 4 or 8 bytes");
  if (!mist::type_ok(d->act_type) || !mist::type_ok(d->table_type))
    return lib_fail(MIST_E_INVALID, "embedding: unknown element type");
  if (!std::isfinite(d->scale)) return lib_fail(MIST_E_INVALID, "embedding: scale must be finite");
  const int64_t most = (int64_t)1 << 40;  // products of strides with their counts need not fit, addresses in use do
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
                   d->act_stride, d->table_stride, d->pos_stride, d->ids_bytes, d->scale,
                   (int32_t)(d->batch * d->seq), (int32_t)((d->hidden + kSlab - 1) / kSlab)};
}

// Whether every lane's eight values are one aligned piece of 16 bytes (32 in fp32).
bool vectors(const mist_embed_desc* d, const void* act, const void* table, const void* pos) {
  return d->hidden % kVec == 0 && (d->batch == 1 || d->act_batch_stride % kVec == 0) && (d->seq == 1 || d->act_stride % kVec == 0) &&
         (d->rows == 1 || d->table_stride % kVec == 0) && (!pos || d->seq == 1 || d->pos_stride % kVec == 0) && aligned(act, 16) &&
         aligned(table, 16) && aligned(pos, 16);
}

template <class F>
void with_bool(bool b, F&& f) {
  if (b) f(std::true_type{});
  else f(std::false_type{});
}

// Blocks for a number of waves, capped so that a grid stays below 2^32 threads (kernels loop).
unsigned blocks_of(int64_t waves) { return (unsigned)std::min<int64_t>((waves + kWaves - 1) / kWaves, 1 << 23); }

// Places in the workspace.
struct Scratch {
  int64_t chunks;
  size_t order, other, hist, part, bytes;
};
Scratch scratch(const EmbedArgs& a) {
  Scratch s{};
  s.chunks = ((int64_t)a.n + kChunk - 1) / kChunk;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) / 256 * 256;
    return was;
  };
  s.order = take((size_t)a.n * sizeof(Entry));
  if (a.n > kCounted) {
    s.other = take((size_t)a.n * sizeof(Entry));
    s.hist = take((size_t)kMaxTiles * kMaxDigits * 4);
  }
  s.part = take(a.n > 2 * kChunk ? (size_t)s.chunks * 2 * a.slabs * kSlab * 4 : 0);
  s.bytes = at;
  return s;
}

void order_tokens(const EmbedArgs& a, const void* ids, const Scratch& s, char* ws, hipStream_t st) {
  Entry* order = (Entry*)(ws + s.order);
  if (a.n <= kCounted) {
    hipLaunchKernelGGL(k_place, dim3((unsigned)((a.n + kPlaced - 1) / kPlaced)), dim3(kThreads), 0, st, a, ids, order);
    return;
  }
  int bits = 1;  // of the largest key, rows
  while (a.rows >> bits) ++bits;
  const int passes = (bits + 8) / 9;
  SortArgs p{};
  p.hist = (int32_t*)(ws + s.hist);
  p.n = a.n;
  const int64_t tile = ((int64_t)a.n + kMaxTiles - 1) / kMaxTiles;
  p.tile = (int32_t)((tile + kSortThreads - 1) / kSortThreads * kSortThreads);
  p.tiles = (int32_t)(((int64_t)a.n + p.tile - 1) / p.tile);
  p.bits = (bits + passes - 1) / passes;
  Entry* buf[2] = {order, (Entry*)(ws + s.other)};
  for (int k = 0; k < passes; ++k) {
    p.out = buf[(passes - 1 - k) % 2];  // the last pass ends in `order`
    p.shift = k * p.bits;
    hipLaunchKernelGGL(k_digits, dim3(p.tiles), dim3(kSortThreads), 0, st, a, p, ids);
    hipLaunchKernelGGL(k_move, dim3(p.tiles), dim3(kSortThreads), 0, st, a, p, ids);
    p.in = p.out;
  }
}

}  // namespace

extern "C" {

mist_status mist_embed_forward(const mist_embed_desc* d, const void* ids, const void* table, const void* pos, void* out,
                               void* stream) {
  if (const mist_status st = check(d, true)) return st;
  if (d->batch == 0 || d->seq == 0) return MIST_OK;
  if (!ids || !table || !out) return lib_fail(MIST_E_INVALID, "embedding: null buffer");
  if (pos && d->seq > 1 && d->pos_stride < d->hidden)
    return lib_fail(MIST_E_INVALID, "embedding: rows of the positions overlap (pos_stride < hidden)");
  if (!aligned(ids, d->ids_bytes) || !aligned(out, mist::type_bytes(d->act_type)) ||
      !aligned(table, mist::type_bytes(d->table_type)) || !aligned(pos, mist::type_bytes(d->table_type)))
    return lib_fail(MIST_E_INVALID, "embedding: a buffer is not aligned to its elements");
  const EmbedArgs a = args(d);
  // enough tokens a wave to keep several rows in flight, few enough to fill the device
  int64_t per_wave = std::clamp<int64_t>((int64_t)a.n * a.slabs / 8192, 1, 64);
  const int64_t waves = (a.n + per_wave - 1) / per_wave * a.slabs;
  if (waves > (int64_t)kWaves << 23) return lib_fail(MIST_E_INVALID, "embedding: too many values for one call");
  mist::with_types(d->act_type, d->table_type, [&](auto x, auto w) {
    using A = typename decltype(x)::type;
    using W = typename decltype(w)::type;
    with_bool(vectors(d, out, table, pos), [&](auto vec) {
      with_bool(pos != nullptr, [&](auto with_pos) {
        hipLaunchKernelGGL((k_embed<A, W, vec.value, with_pos.value>), dim3(blocks_of(waves)), dim3(kThreads), 0, (hipStream_t)stream, a,
                           (int32_t)per_wave, ids, (const W*)table, (const W*)pos, (A*)out);
      });
    });
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "embedding");
}

mist_status mist_embed_workspace(const mist_embed_desc* d, size_t* bytes) {
  if (!bytes) return lib_fail(MIST_E_INVALID, "embedding: null argument");
  if (const mist_status st = check(d, false)) return st;
  *bytes = scratch(args(d)).bytes;
  return MIST_OK;
}

mist_status mist_embed_backward(const mist_embed_desc* d, const void* ids, const void* grad, void* dtable, void* dpos,
                                int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (const mist_status st = check(d, false)) return st;
  if (accumulate != 0 && accumulate != 1) return lib_fail(MIST_E_INVALID, "embedding: accumulate must be 0 or 1");
  const EmbedArgs a = args(d);
  const Scratch s = scratch(a);
  if (!dtable || (a.n && (!ids || !grad))) return lib_fail(MIST_E_INVALID, "embedding: null buffer");
  if (s.bytes && !workspace) return lib_fail(MIST_E_INVALID, "embedding: null workspace");
  if (workspace_bytes < s.bytes) return lib_fail(MIST_E_RANGE, "embedding: workspace too small");
  if (dpos && d->seq > 1 && d->pos_stride < d->hidden)
    return lib_fail(MIST_E_INVALID, "embedding: rows of the positions overlap (pos_stride < hidden)");
  if (!aligned(ids, d->ids_bytes) || !aligned(grad, mist::type_bytes(d->act_type)) ||
      !aligned(dtable, mist::type_bytes(d->table_type)) || !aligned(dpos, mist::type_bytes(d->table_type)) ||
      !aligned(workspace, 256))
    return lib_fail(MIST_E_INVALID, "embedding: a buffer is not aligned to its elements, or the workspace to 256");
  const int64_t join_blocks = (s.chunks + kJoinChunks - 1) / kJoinChunks * a.slabs;
  if (join_blocks > 1 << 23) return lib_fail(MIST_E_INVALID, "embedding: too many values for one call");
  const hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  if (a.n) order_tokens(a, ids, s, ws, st);
  const RowArgs r{(const Entry*)(ws + s.order), (float*)(ws + s.part), (int32_t)s.chunks, accumulate, s.chunks * a.slabs};
  mist::with_types(d->act_type, d->table_type, [&](auto x, auto w) {
    using A = typename decltype(x)::type;
    using W = typename decltype(w)::type;
    with_bool(vectors(d, grad, dtable, dpos), [&](auto vec) {
      const int64_t waves = r.sum_waves + (accumulate ? 0 : a.rows);
      if (waves)
        hipLaunchKernelGGL((k_rows<A, W, vec.value>), dim3(blocks_of(waves)), dim3(kThreads), 0, st, a, r, (const A*)grad, (W*)dtable);
      if (a.n > 2 * kChunk)
        hipLaunchKernelGGL((k_join<W, vec.value>), dim3((unsigned)join_blocks), dim3(kThreads), 0, st, a, r, (W*)dtable);
      if (dpos && d->seq)
        hipLaunchKernelGGL((k_dpos<A, W, vec.value>), dim3(blocks_of(a.seq * a.slabs)), dim3(kThreads), 0, st, a, (const A*)grad, (W*)dpos,
                           accumulate);
    });
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "embedding gradient");
}

}  // extern "C"
