// The first stage's embedding, a vocabulary-parallel table with learned positions, and its gradient.
//
// out[b, s] = scale * W[id] + P[s];  dW[v] = scale * sum of dout[b, s] over the tokens of row v;  dP[s] = sum over b.
// One operation a value or two: both are bound by memory, and short inputs by launches (about 4 us each).
//
// The lookup gathers rows and writes activations, a wave a slab of 512 columns of a few tokens.  The gradient
// orders the tokens by row (stable, so that a row's terms are added in token order whatever ran first), sums
// each row's terms in fp32 registers and writes the row once: no atomics on values.  Measured on one MI355X
// (16-bit values; a large copy reads and writes 4.9 TB/s, a fill writes 6.8):
//   lookup    65536 tokens of 2560 columns with positions  93 us, 336 MB written and 205 MB read: 5.7 TB/s
//             32768 of 8192 in a shard of 4000 rows         81 us, 537 MB written and 80 MB read: 7.6 TB/s
//   gradient  65536 of 2560, 50257 rows, with positions   188 us: order with the positions' sums 4 x 23 us
//             (335 MB read), rows 98 us (339 MB read, 262 MB written), long runs 6.5 us.  The gradient is read twice,
//             once by position and once by row: 5 TB/s over the call
//             131072 of 8192, 32000 rows                  443 us: order 27 us, rows 405 us (1617 MB read, 549 MB
//             written: 5.3 TB/s), long runs 13 us
//             4095 of 4096 added to fp32                   30 us: order 7 us, rows 19 us, long runs 5 us
//             256 of 512 in fp32, 2048 rows                9.1 us, one launch
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "mist_ops.h"

namespace {

using mist::hip_failed;
using mist::lib_fail;
using mist::Vec;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kVec = 8;             // values of a lane
constexpr int kSlab = 64 * kVec;    // columns of a wave
constexpr int kJoinRuns = 128;      // long runs joined at a time
constexpr int64_t kCache = (int64_t)256 << 20;  // the memory-side cache
constexpr int64_t kHeld = 86000000;             // of rows that a lookup reaches, see k_embed
constexpr int64_t kMostTokens = (int64_t)1 << 30;  // places past the last token stay below 2^31
constexpr int kMaxChunk = 64;       // ordered tokens of a wave, one a lane, at most

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

typedef Vec<float, kVec>::type Float8;

// Which eight columns of a slab a lane holds:
//   kWide   eight in a row: one access of 16 bytes (both types of 16 bits, hidden a multiple of 8)
//   kSplit  two fours 256 apart: accesses of 16 bytes for fp32, 8 for 16 bits (hidden a multiple of 4).  Eight in
//           a row would leave every other 16 bytes of a store to a second instruction: 2.4 TB/s where this
//           reaches 5.3 (64365 tokens, 5440 columns)
//   kOdd    one by one, 64 apart (any hidden)
// Columns past the row are read as the row's last ones, so that loads need no branch, and not written.
enum Layout { kWide, kSplit, kOdd };

template <int L>
struct Cols {
  static constexpr int kRun = L == kWide ? 8 : L == kSplit ? 4 : 1, kRuns = kVec / kRun;
  int32_t first, hidden;
  __device__ __forceinline__ Cols(int32_t slab, int64_t h)
      : first(slab * kSlab + (int32_t)(threadIdx.x % 64) * kRun), hidden((int32_t)h) {}
  __device__ __forceinline__ bool in(int k) const { return first + 64 * kRun * k < hidden; }
  // Run k of a row of T.  The offset is a 32-bit one to a uniform address, which takes no registers of its own.
  template <class T>
  __device__ __forceinline__ T* at(T* row, int k) const {
    const uint32_t offset = (uint32_t)min(first + 64 * kRun * k, hidden - kRun) * (uint32_t)sizeof(T);
    return (T*)((uintptr_t)row + offset);
  }
};

// ONCE: not wanted again soon, so that it does not displace what is (rows of the table, the
// gradient between its two uses).
template <class T, int L>
struct Lane8 {
  static constexpr int kRun = Cols<L>::kRun, kRuns = Cols<L>::kRuns;
  typedef typename Vec<T, kRun>::type Run;
  Run v[kRuns];
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const T* row, const Cols<L>& c) {
#pragma unroll
    for (int k = 0; k < kRuns; ++k) {
      const Run* p = (const Run*)c.at(row, k);
      v[k] = ONCE ? __builtin_nontemporal_load(p) : *p;
    }
  }
  __device__ __forceinline__ Float8 get() const {
    Float8 x;
#pragma unroll
    for (int k = 0; k < kVec; ++k) x[k] = (float)v[k / kRun][k % kRun];
    return x;
  }
  template <bool ONCE = false>
  static __device__ __forceinline__ void store(T* row, const Cols<L>& c, Float8 x) {
#pragma unroll
    for (int k = 0; k < kRuns; ++k) {
      Run y;
#pragma unroll
      for (int i = 0; i < kRun; ++i) y[i] = (T)x[k * kRun + i];
      if (!c.in(k)) continue;
      if (ONCE) __builtin_nontemporal_store(y, (Run*)c.at(row, k));
      else *(Run*)c.at(row, k) = y;
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
  const int64_t at = a.ids_stride == a.seq ? token : token / (uint32_t)a.seq * a.ids_stride + token % (uint32_t)a.seq;
  const int64_t id = a.ids_bytes == 4 ? (int64_t)((const int32_t*)ids)[at] : ((const int64_t*)ids)[at];
  return id >= a.begin && id - a.begin < a.rows ? (uint32_t)(id - a.begin) : (uint32_t)a.rows;
}

__device__ __forceinline__ int64_t act_offset(const EmbedArgs& a, uint32_t token) {
  return token / (uint32_t)a.seq * a.act_batch_stride + token % (uint32_t)a.seq * a.act_stride;
}

// ---- lookup ----------------------------------------------------------------------------------------
// A wave takes `per_wave` (at most kAhead) tokens and one slab of columns, all rows in flight: 4 (32768 tokens
// of 8192 columns: 88 us; 8 tokens 98, 16 102), or 16 with positions (65536 of 2560: 94 us; 8 tokens 99,
// 4 106).  These are in 16 bits; fp32 tables and odd widths hold 256 registers with 16 (fp32 189 us for the 172 of a copy).
// With positions the tokens are taken position by position, so that a wave reads a position's row once for
// its part of the batch.
// by_slab: the blocks take the slabs in turn, so that with 2, 4, 8 or 16 slabs an XCD (blocks are dealt to the 8 in
// turn) sees few columns, and its L2 holds more of the table's rows.  That gains 4 to 17 % while the rows that the
// tokens reach take at most kHeld bytes, and loses up to 30 % past it, where the longer strides between accesses
// cost more.  Both ways, text's tokens, 16 bits (us by slab / in order, by megabytes of rows reached): 65536 tokens of 4096
// columns 76: 93 / 110, 81: 101 / 110, 86: 119 / 109, 94: 135 / 117; 65536 of 8192 75: 179 / 195, 87: 192 / 193, 97: 245 / 208;
// 65536 of 2048 69: 57 / 62; 32768 of 8192 in a shard of 4000 rows 82 / 89.  In fp32 the sides change at 90 to 100.  With 32 slabs
// there is nothing to gain (16384 of 16384: 95 / 94).
template <bool POS>
constexpr int kAhead = POS ? 16 : 4;

template <class A, class W, int L, bool POS>
__global__ __launch_bounds__(kThreads) void k_embed(EmbedArgs a, int32_t per_wave, bool by_slab, int32_t group0, const void* __restrict__ ids,
                                                    const W* __restrict__ table, const W* __restrict__ pos, A* __restrict__ out) {
  const uint32_t slabs = (uint32_t)a.slabs, wave = (uint32_t)wave_index();
  const int32_t slab = (int32_t)(by_slab ? blockIdx.x % slabs : wave % slabs);
  const int64_t first = (int64_t)(group0 + (by_slab ? blockIdx.x / slabs * kWaves + wave % kWaves : wave / slabs)) * per_wave;
  if (first >= a.n) return;
  const int32_t count = (int32_t)(a.n - first < per_wave ? a.n - first : per_wave);
  const int lane = threadIdx.x % 64;
  uint32_t token = (uint32_t)first + (lane < count ? lane : 0);
  if (POS) token = token % (uint32_t)a.batch * (uint32_t)a.seq + token / (uint32_t)a.batch;
  const uint32_t row = token_row(a, ids, token);
  const int64_t row_at = row < a.rows ? row * a.table_stride : -1;
  const int64_t out_at = act_offset(a, token);
  const uint32_t s = token % (uint32_t)a.seq;
  const Cols<L> col(slab, a.hidden);
  Lane8<W, L> x[kAhead<POS>], p[kAhead<POS>];
#pragma unroll
  for (int k = 0; k < kAhead<POS>; ++k) {
    if (k < count) {
      const int64_t at = lane_value(row_at, k);
      if (at >= 0) x[k].load(table + at, col);
      else x[k] = {};
      if (POS && (k == 0 || lane_value(s, k) != lane_value(s, k - 1))) p[k].load(pos + lane_value(s, k) * a.pos_stride, col);
    }
  }
  Float8 at_s = {};
#pragma unroll
  for (int k = 0; k < kAhead<POS>; ++k) {
    if (k < count) {
      Float8 y = a.scale * x[k].get();
      if (POS) {
        if (k == 0 || lane_value(s, k) != lane_value(s, k - 1)) at_s = p[k].get();
        y += at_s;
      }
      Lane8<A, L>::template store<true>(out + lane_value(out_at, k), col, y);
    }
  }
}

// ---- sums of the positions -------------------------------------------------------------------------
// A wave takes a position and a slab, and adds up the batch.  The work is spread over the launches that order
// the tokens, which leave most of the device idle: `block` of `blocks` more blocks takes the items [begin, end).
// The reads reach 3.6 to 3.9 TB/s (32 x 2048 tokens of 2560 columns, 16 bits): a launch's share is 160 blocks beside the 64
// that order, fewer than the CUs.  More loads at once, several positions a wave, or several waves a position measured the same or
// worse there; a batch far larger than the sequence leaves few waves.
template <int L>
constexpr int kPosAhead = L == kOdd ? 2 : 8;  // one by one, eight take more registers than a block of 1024 threads has

// The batch is summed in parts of 64, the rows' largest piece, so that a term meets 64 + batch / 64 roundings and
// not batch: one sum over 2^20 sequences lost 0.7 % of terms whose last bits it did not hold.
constexpr int64_t kPosPart = 64;

template <class A, class W>
struct PosArgs {
  const A* grad;
  W* dpos;
  int64_t begin, end;  // of seq * slabs
  int32_t accumulate;
};

template <int L, class A, class W>
__device__ void sum_positions(const EmbedArgs& a, const PosArgs<A, W>& p, uint32_t block, uint32_t blocks) {
  const int32_t waves = blockDim.x / 64;
  int64_t item = p.begin + __builtin_amdgcn_readfirstlane((int32_t)(block * waves + threadIdx.x / 64));
  for (; item < p.end; item += (int64_t)blocks * waves) {
    const int64_t s = item / a.slabs;
    const Cols<L> col((int32_t)(item % a.slabs), a.hidden);
    Float8 acc = {}, done = {};
    for (int64_t b0 = 0; b0 < a.batch; b0 += kPosAhead<L>) {
      Lane8<A, L> x[kPosAhead<L>];
#pragma unroll
      for (int k = 0; k < kPosAhead<L>; ++k)
        if (b0 + k < a.batch) x[k].load(p.grad + (b0 + k) * a.act_batch_stride + s * a.act_stride, col);
#pragma unroll
      for (int k = 0; k < kPosAhead<L>; ++k)
        if (b0 + k < a.batch) acc += x[k].get();
      if ((b0 + kPosAhead<L>) % kPosPart == 0) {
        done += acc;
        acc = Float8{};
      }
    }
    acc += done;
    W* d = p.dpos + s * a.pos_stride;
    if (p.accumulate) {
      Lane8<W, L> old;
      old.load(d, col);
      acc += old.get();
    }
    Lane8<W, L>::store(d, col, acc);
  }
}

// ---- order of the tokens ---------------------------------------------------------------------------
// Short inputs: a token's place is the number of tokens before it by (row, token), counted directly;
// one launch.  A block's 16 waves place a token each against all of them.
constexpr int32_t kCounted = 8192;   // tokens up to which places are counted
constexpr int kPlaceThreads = 1024, kPlaced = kPlaceThreads / 64;

template <class A, class W, int L>
__global__ __launch_bounds__(kPlaceThreads) void k_place(EmbedArgs a, PosArgs<A, W> pos, const void* __restrict__ ids, Entry* __restrict__ out,
                                                         int32_t* __restrict__ longs) {
  const int32_t blocks = (a.n + kPlaced - 1) / kPlaced;
  if ((int32_t)blockIdx.x >= blocks) {
    sum_positions<L>(a, pos, blockIdx.x - blocks, gridDim.x - blocks);
    return;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *longs = 0;
  __shared__ uint4 rows[kCounted / 4];
  uint32_t* row = (uint32_t*)rows;
  const int32_t steps = (a.n + 255) / 256;   // of 64 lanes by 4 tokens
#pragma unroll 4
  for (int32_t i = threadIdx.x; i < steps * 256; i += kPlaceThreads) row[i] = i < a.n ? token_row(a, ids, i) : UINT32_MAX;
  __syncthreads();
  const int32_t i = blockIdx.x * kPlaced + threadIdx.x / 64, lane = threadIdx.x % 64;
  const uint32_t mine = row[i < a.n ? i : 0];
  int32_t place = 0;
#pragma unroll 4
  for (int32_t t = 0; t < steps; ++t) {
    const int32_t q = t * 64 + lane, j = q * 4;
    const uint4 r = rows[q];
    place += r.x < mine + (j < i);       // rows are below 2^31: r < mine, or equal and before
    place += r.y < mine + (j + 1 < i);
    place += r.z < mine + (j + 2 < i);
    place += r.w < mine + (j + 3 < i);
  }
  for (int d = 32; d; d >>= 1) place += __shfl_xor(place, d);
  if (lane == 0 && i < a.n) out[place] = Entry{mine, (uint32_t)i};
}

// Counting takes 7 us for 4095 tokens; four launches of the radix order 25 us and more.
//
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
  int32_t* longs;     // cleared
  int32_t n, tile, tiles, shift, bits;
};

__device__ __forceinline__ Entry sort_entry(const EmbedArgs& a, const SortArgs& s, const void* ids, int32_t i) {
  return s.in ? s.in[i] : Entry{token_row(a, ids, i), (uint32_t)i};
}

template <class A, class W, int L>
__global__ __launch_bounds__(kSortThreads) void k_digits(EmbedArgs a, SortArgs s, PosArgs<A, W> pos, const void* __restrict__ ids) {
  if ((int32_t)blockIdx.x >= s.tiles) {
    sum_positions<L>(a, pos, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    return;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *s.longs = 0;
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

template <class A, class W, int L>
__global__ __launch_bounds__(kSortThreads) void k_move(EmbedArgs a, SortArgs s, PosArgs<A, W> pos, const void* __restrict__ ids) {
  if ((int32_t)blockIdx.x >= s.tiles) {
    sum_positions<L>(a, pos, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    return;
  }
  __shared__ int32_t at[kSortWaves][kMaxDigits];  // counts, then places
  __shared__ int32_t total[kSortThreads], before[kSortThreads], wave_total[kMaxDigits / 64];
  const int32_t digits = 1 << s.bits, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  for (int32_t d = threadIdx.x; d < kSortWaves * kMaxDigits; d += kSortThreads) (&at[0][0])[d] = 0;
  // a digit's tokens in all tiles, and in the tiles before this one; 1024 / digits threads a digit
  {
    const int32_t d = threadIdx.x % digits, parts = kSortThreads / digits, share = (s.tiles + parts - 1) / parts;
    const int32_t t0 = threadIdx.x / digits * share, t1 = min(s.tiles, t0 + share);
    int32_t all = 0, mine = 0;
#pragma unroll 8
    for (int32_t t = t0; t < t1; ++t) {
      const int32_t c = s.hist[t * digits + d];
      all += c;
      mine += t < (int32_t)blockIdx.x ? c : 0;
    }
    total[threadIdx.x] = all;
    before[threadIdx.x] = mine;
  }
  __syncthreads();
  int32_t sum = 0, mine = 0, scan = 0;  // of digit threadIdx.x
  if ((int32_t)threadIdx.x < digits) {
    for (int32_t t = threadIdx.x; t < kSortThreads; t += digits) {
      sum += total[t];
      mine += before[t];
    }
  }
  scan = sum;
  for (int d = 1; d < 64; d <<= 1) {
    const int32_t x = __shfl_up(scan, d);
    scan += lane >= d ? x : 0;
  }
  if (lane == 63 && wave < kMaxDigits / 64) wave_total[wave] = scan;
  __syncthreads();
  for (int w = 0; w < wave && w < kMaxDigits / 64; ++w) scan += wave_total[w];
  const int32_t base = scan - sum + mine;  // place of the tile's first token of digit threadIdx.x
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
    int32_t place = base;
    for (int w = 0; w < kSortWaves; ++w) {
      const int32_t c = at[w][threadIdx.x];
      at[w][threadIdx.x] = place;
      place += c;
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
// A wave takes a chunk of up to 64 ordered tokens and a slab of columns, and adds up runs of equal rows in
// registers.  A run that crosses one chunk boundary is finished by the chunk where it begins.  A run that
// touches three chunks or more is long: each chunk leaves its piece in `part`, slot 1 the chunk where
// the run begins and slot 0 the others, and k_join adds the pieces in order.
struct RowArgs {
  const Entry* order;
  int32_t* longs;       // count of long runs, then the chunks where they begin, in any order
  float* part;          // [chunks][2][slabs][kSlab], in lane order
  int32_t chunk, chunks;  // tokens a chunk, a power of two; chunks
  int32_t accumulate;
  int64_t sum_waves;    // waves that sum chunks; the rest clear rows without a token
};

__device__ __forceinline__ uint32_t row_at(const RowArgs& r, const EmbedArgs& a, int64_t i) {
  return i >= 0 && i < a.n ? r.order[i].row : (uint32_t)a.rows;
}

template <class A, class W, int L, bool ONCE>
struct RowSum {
  const EmbedArgs& a;
  const RowArgs& r;
  const A* grad;
  W* dtable;
  int32_t chunk, slab;
  Cols<L> col;
  Float8 acc = {};
  static constexpr int kGroup = sizeof(A) == 2 ? 8 : 4;

  __device__ __forceinline__ void part_out(int slot) {
    float* p = r.part + (((int64_t)chunk * 2 + slot) * a.slabs + slab) * kSlab + threadIdx.x % 64 * kVec;
    *(Float8*)p = acc;
  }

  // Tokens [from, to) of the chunk whose rows and offsets the lanes hold.  `next` is the row after the last
  // lane's.  slot >= 0: the range is one piece of a long run.
  __device__ __forceinline__ void take(uint32_t row, int64_t offset, int from, int to, uint32_t next, int slot) {
    for (int k0 = from; k0 < to; k0 += kGroup) {
      Lane8<A, L> x[kGroup];
      Lane8<W, L> old[kGroup];
      bool ends[kGroup];
      uint32_t mine[kGroup];
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        if (k0 + k < to) {
          mine[k] = lane_value(row, k0 + k);
          ends[k] = slot < 0 && mine[k] != (k0 + k < r.chunk - 1 ? lane_value(row, k0 + k + 1) : next);
          x[k].template load<ONCE>(grad + lane_value(offset, k0 + k), col);
          if (r.accumulate && ends[k]) old[k].load(dtable + mine[k] * a.table_stride, col);
        }
      }
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        if (k0 + k < to) {
          acc += x[k].get();
          if (ends[k]) {
            Float8 y = a.scale * acc;
            W* d = dtable + mine[k] * a.table_stride;
            if (r.accumulate) Lane8<W, L>::store(d, col, y + old[k].get());
            else Lane8<W, L>::template store<true>(d, col, y);
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
    const int C = r.chunk, lane = threadIdx.x % 64;
    const int64_t base = (int64_t)chunk * C;
    const uint32_t none = (uint32_t)a.rows;
    const bool in0 = lane < C && base + lane < a.n, in1 = lane < C && base + C + lane < a.n;
    const Entry e0 = in0 ? r.order[base + lane] : Entry{none, 0}, e1 = in1 ? r.order[base + C + lane] : Entry{none, 0};
    const uint32_t first = lane_value(e0.row, 0), last = lane_value(e0.row, C - 1), after = lane_value(e1.row, 0);
    if (first == none) return;
    const uint32_t before = row_at(r, a, base - 1);
    const int64_t off0 = act_offset(a, e0.token);
    const int valid = __popcll(__ballot(e0.row != none));
    int from = 0;
    if (chunk > 0 && before == first) {  // the first run began earlier
      const int lead = __popcll(__ballot(e0.row == first));
      const bool short_run = row_at(r, a, base - 1 - C) != first && after != first;
      if (!short_run) take(e0.row, off0, 0, lead, none, 0);
      from = lead;
    }
    if (from == valid) return;
    const bool goes_on = last != none && after == last;  // the last run begins here and crosses the boundary
    if (!goes_on) {
      take(e0.row, off0, from, valid, after, -1);
      return;
    }
    const int tail = C - __popcll(__ballot(e0.row == last));  // where it begins
    if (row_at(r, a, base + 2 * C) != last) {
      take(e0.row, off0, from, C, after, -1);
      const int more = __popcll(__ballot(e1.row == last));
      take(e1.row, act_offset(a, e1.token), 0, more, none, -1);
    } else {
      take(e0.row, off0, from, tail, after, -1);
      take(e0.row, off0, tail, C, after, 1);
      if (slab == 0 && lane == 0) r.longs[1 + atomicAdd(r.longs, 1)] = chunk;
    }
  }
};

// Rows [first, first + kClear) without a token are cleared; a lane looks for each.  (131072 tokens of 8192 columns:
// 441 us with 2 or 4 rows a wave, 448 with 16, 447 with one; 65536 of 2560: 190, 191, 202.)
constexpr int kClear = 4;

template <class W, int L>
__device__ __forceinline__ void clear_rows(const EmbedArgs& a, const RowArgs& r, W* dtable, int64_t first) {
  const int lane = threadIdx.x % 64;
  const int64_t row = first + lane;
  bool found = lane >= kClear || row >= a.rows;
  if (!found) {
    int32_t lo = 0, hi = a.n;  // the first place of a row not below is in [lo, hi]
    while (lo < hi) {
      const int32_t mid = lo + (hi - lo) / 2;
      if (r.order[mid].row < row) lo = mid + 1;
      else hi = mid;
    }
    found = lo < a.n && r.order[lo].row == row;
  }
  for (uint64_t clear = ~__ballot(found); clear; clear &= clear - 1) {
    W* d = dtable + (first + __ffsll((unsigned long long)clear) - 1) * a.table_stride;
    for (int32_t slab = 0; slab < a.slabs; ++slab) Lane8<W, L>::template store<true>(d, Cols<L>(slab, a.hidden), Float8{});
  }
}

template <class A, class W, int L, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_rows(EmbedArgs a, RowArgs r, const A* __restrict__ grad, W* __restrict__ dtable) {
  const int64_t waves = (int64_t)gridDim.x * kWaves, all = r.sum_waves + (r.accumulate ? 0 : (a.rows + kClear - 1) / kClear);
  for (int64_t w = wave_index(); w < all; w += waves) {
    if (w < r.sum_waves) {
      const int32_t chunk = (int32_t)(w / a.slabs), slab = (int32_t)(w % a.slabs);
      RowSum<A, W, L, ONCE> s{a, r, grad, dtable, chunk, slab, Cols<L>(slab, a.hidden)};
      s.run();
    } else {
      clear_rows<W, L>(a, r, dtable, (w - r.sum_waves) * kClear);
    }
  }
}

// Long runs: a block takes a run and a slab, its waves add up a share of the pieces each, in order, and the
// shares are added in order.
template <class W, int L>
__global__ __launch_bounds__(kThreads) void k_join(EmbedArgs a, RowArgs r, W* __restrict__ dtable) {
  __shared__ Float8 shares[kWaves][64];
  const int32_t slab = (int32_t)(blockIdx.x % a.slabs), wave = threadIdx.x / 64, lane = threadIdx.x % 64, C = r.chunk;
  const Cols<L> col(slab, a.hidden);
  const int32_t runs = r.longs[0];
  for (int32_t i = (int32_t)(blockIdx.x / a.slabs); i < runs; i += (int32_t)(gridDim.x / a.slabs)) {
    const int32_t c = r.longs[1 + i];
    const uint32_t row = r.order[(int64_t)c * C + C - 1].row;
    int32_t end = c + 2;  // the run's chunks are [c, end)
    for (;;) {
      const uint64_t in = __ballot(row_at(r, a, (int64_t)(end + lane) * C) == row);
      end += in == ~0ull ? 64 : __ffsll((unsigned long long)~in) - 1;
      if (in != ~0ull) break;
    }
    const int32_t pieces = end - c, share = (pieces + kWaves - 1) / kWaves, to = min(pieces, (wave + 1) * share);
    Float8 acc = {};
#pragma unroll 8
    for (int32_t k = wave * share; k < to; ++k)
      acc += *(const Float8*)(r.part + (((int64_t)(c + k) * 2 + (k == 0)) * a.slabs + slab) * kSlab + lane * kVec);
    shares[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
      for (int w = 1; w < kWaves; ++w) acc += shares[w][lane];
      W* d = dtable + row * a.table_stride;
      Float8 y = a.scale * acc;
      if (r.accumulate) {
        Lane8<W, L> old;
        old.load(d, col);
        y += old.get();
      }
      Lane8<W, L>::store(d, col, y);
    }
    __syncthreads();
  }
}

// ---- short inputs ----------------------------------------------------------------------------------
// Everything in one launch, where launches are what takes the time.  A block takes a token and a slab; it finds
// the tokens of the same row with a ballot a wave, and goes on if its token is the first of them.  Each
// wave adds up its 64 tokens' terms in order and the waves' sums are added in order; up to kFew terms
// are left to the first wave.  Further blocks clear rows without a token, and sum positions.
// Against the three launches of the longer way (tokens added to 16 bits): 9 us for 14.4 up to about 9000 waves,
// 14.9 for 14.4 at 16384 (1024 tokens, 512 columns), 25 for 14.5 at 32768.
constexpr int32_t kShort = 1024;     // tokens, at most
constexpr int64_t kShortWaves = 16384;
constexpr int kFew = 8, kShortClear = 64;

template <class A, class W, int L>
__global__ __launch_bounds__(kShort) void k_short(EmbedArgs a, PosArgs<A, W> pos, const void* __restrict__ ids, const A* __restrict__ grad,
                                                  W* __restrict__ dtable, int32_t accumulate) {
  __shared__ Float8 shares[kShort / 64][64];
  __shared__ uint64_t same[kShort / 64];
  const int32_t sums = a.n * a.slabs, clears = accumulate ? 0 : (int32_t)((a.rows + kShortClear - 1) / kShortClear);
  const int32_t i0 = threadIdx.x, wave = __builtin_amdgcn_readfirstlane((int32_t)threadIdx.x / 64), lane = threadIdx.x % 64, waves = blockDim.x / 64;
  int64_t block = blockIdx.x;
  if (block >= sums + clears) {
    sum_positions<L>(a, pos, blockIdx.x - sums - clears, gridDim.x - sums - clears);
    return;
  }
  const uint32_t row = i0 < a.n ? token_row(a, ids, i0) : (uint32_t)a.rows;
  if (block >= sums) {
    uint8_t* seen = (uint8_t*)same;  // of kShortClear rows
    const int64_t first = (block - sums) * kShortClear;
    if (threadIdx.x < kShortClear) seen[threadIdx.x] = 0;
    __syncthreads();
    if (row >= first && row < first + kShortClear) seen[row - first] = 1;
    __syncthreads();
    for (int k = wave; k < kShortClear && first + k < a.rows; k += waves) {
      if (seen[k]) continue;
      for (int32_t slab = 0; slab < a.slabs; ++slab)
        Lane8<W, L>::template store<true>(dtable + (first + k) * a.table_stride, Cols<L>(slab, a.hidden), Float8{});
    }
    return;
  }
  const int32_t token = (int32_t)block / a.slabs, slab = (int32_t)block % a.slabs;
  const uint32_t mine = token_row(a, ids, token);
  if (mine == (uint32_t)a.rows) return;
  const uint64_t my = __ballot(row == mine);
  if (lane == 0) same[wave] = my;
  __syncthreads();
  int total = 0;
  for (int w = 0; w < waves; ++w) {
    const uint64_t m = same[w];
    if (m && w * 64 + __ffsll((unsigned long long)m) - 1 < token) return;  // not the first of the row
    total += __popcll(m);
  }
  const Cols<L> col(slab, a.hidden);
  Float8 acc = {};
  auto add = [&](uint64_t m, int32_t base) {
    while (m) {
      Lane8<A, L> x[kFew];
      const int count = __popcll(m);
#pragma unroll
      for (int k = 0; k < kFew; ++k) {
        if (k < count) {
          x[k].load(grad + act_offset(a, base + __ffsll((unsigned long long)m) - 1), col);
          m &= m - 1;
        }
      }
#pragma unroll
      for (int k = 0; k < kFew; ++k)
        if (k < count) acc += x[k].get();
    }
  };
  if (total <= kFew) {
    if (wave) return;
    for (int w = 0; w < waves; ++w) {
      const uint64_t m = same[w];
      add((uint64_t)__builtin_amdgcn_readfirstlane((int)(m >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)m), w * 64);
    }
  } else {
    add(my, wave * 64);
    shares[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < waves; ++w) acc += shares[w][lane];
  }
  W* d = dtable + mine * a.table_stride;
  Float8 y = a.scale * acc;
  if (accumulate) {
    Lane8<W, L> old;
    old.load(d, col);
    y += old.get();
  }
  Lane8<W, L>::store(d, col, y);
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

// Rows of a table that n tokens reach, as text has them (the k-th most frequent 1 / k as often as the first): the sum over k of
// 1 - (1 - p_k)^n with p_k = 1 / (k ln(rows + 1)), as an integral: rows (1 - e^-x) + rows x E1(x), x = n / (rows ln(rows + 1)).
// E1 from its series below 1 and the approximation 5.1.54 of Abramowitz and Stegun from there on.
double rows_reached(int64_t n, int64_t rows) {
  const double x = (double)n / ((double)rows * std::log((double)rows + 1.0));
  if (x >= 1.0) return (double)rows * (1.0 - std::exp(-x) * (1.0 - (x * (x + 2.334733) + 0.250621) / (x * (x + 3.330657) + 1.681534)));
  const double e1 = -0.57721566 - std::log(x) + x * (1.0 - x * (1.0 / 4 - x * (1.0 / 18 - x * (1.0 / 96 - x / 600))));
  return (double)rows * (x * e1 - std::expm1(-x));
}

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

EmbedArgs args(const mist_embed_desc* d) {
  return EmbedArgs{d->batch, d->seq, d->hidden, d->rows, d->vocab_begin, d->ids_stride, d->act_batch_stride,
                   d->act_stride, d->table_stride, d->pos_stride, d->ids_bytes, d->scale,
                   (int32_t)(d->batch * d->seq), (int32_t)((d->hidden + kSlab - 1) / kSlab)};
}

// f(the layout for the types and hidden).
template <class A, class W, class F>
void with_layout(int64_t hidden, F&& f) {
  if constexpr (sizeof(A) == 2 && sizeof(W) == 2) {
    if (hidden % 8 == 0) return f(std::integral_constant<int, kWide>{});
  }
  if (hidden % 4 == 0) f(std::integral_constant<int, kSplit>{});
  else f(std::integral_constant<int, kOdd>{});
}

// Blocks for a number of waves, capped so that a grid stays below 2^32 threads (kernels loop).
unsigned blocks_of(int64_t waves, int per_block) { return (unsigned)std::min<int64_t>((waves + per_block - 1) / per_block, 1 << 21); }

// Whether one launch does all (k_short): few tokens, and few waves to look through them.
bool is_short(const EmbedArgs& a) { return a.n <= kShort && (int64_t)a.n * a.slabs * ((a.n + 63) / 64) <= kShortWaves && a.rows <= 1 << 24; }

// Places in the workspace.
struct Scratch {
  int32_t chunk;
  int64_t chunks;
  size_t order, other, hist, longs, part, bytes;
};
Scratch scratch(const EmbedArgs& a) {
  Scratch s{};
  if (is_short(a)) return s;
  // Smaller chunks where there are too few waves to hide the gather's latency.
  s.chunk = kMaxChunk;
  while (s.chunk > 8 && ((int64_t)a.n + s.chunk - 1) / s.chunk * a.slabs < 2048) s.chunk /= 2;
  s.chunks = ((int64_t)a.n + s.chunk - 1) / s.chunk;
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
  s.longs = take((size_t)(s.chunks / 2 + 2) * 4);
  s.part = take(s.chunks > 2 ? (size_t)s.chunks * 2 * a.slabs * kSlab * 4 : 0);
  s.bytes = at;
  return s;
}

template <int L, class A, class W>
void order_tokens(const EmbedArgs& a, const void* ids, const Scratch& s, PosArgs<A, W> pos, char* ws, hipStream_t st) {
  Entry* order = (Entry*)(ws + s.order);
  const int64_t items = pos.dpos ? a.seq * a.slabs : 0;  // of the positions
  if (a.n <= kCounted) {
    pos.end = items;
    const dim3 grid((unsigned)((a.n + kPlaced - 1) / kPlaced) + blocks_of(items, kPlaced));
    if (grid.x) hipLaunchKernelGGL((k_place<A, W, L>), grid, dim3(kPlaceThreads), 0, st, a, pos, ids, order, (int32_t*)(ws + s.longs));
    return;
  }
  int bits = 1;  // of the largest key, rows
  while (a.rows >> bits) ++bits;
  const int passes = (bits + 8) / 9;
  SortArgs p{};
  p.hist = (int32_t*)(ws + s.hist);
  p.longs = (int32_t*)(ws + s.longs);
  p.n = a.n;
  const int64_t tile = ((int64_t)a.n + kMaxTiles - 1) / kMaxTiles;
  p.tile = (int32_t)((tile + kSortThreads - 1) / kSortThreads * kSortThreads);
  p.tiles = (int32_t)(((int64_t)a.n + p.tile - 1) / p.tile);
  p.bits = (bits + passes - 1) / passes;
  Entry* buf[2] = {order, (Entry*)(ws + s.other)};
  for (int k = 0; k < 2 * passes; ++k) {
    if (k % 2 == 0) {
      p.out = buf[(passes - 1 - k / 2) % 2];  // the last pass ends in `order`
      p.shift = k / 2 * p.bits;
    }
    pos.begin = items * k / (2 * passes);
    pos.end = items * (k + 1) / (2 * passes);
    const dim3 grid(p.tiles + blocks_of(pos.end - pos.begin, kSortWaves));
    if (k % 2 == 0) {
      hipLaunchKernelGGL((k_digits<A, W, L>), grid, dim3(kSortThreads), 0, st, a, p, pos, ids);
    } else {
      hipLaunchKernelGGL((k_move<A, W, L>), grid, dim3(kSortThreads), 0, st, a, p, pos, ids);
      p.in = p.out;
    }
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
  const int64_t per_wave = std::clamp<int64_t>((int64_t)a.n * a.slabs / 16384, 1, pos ? kAhead<true> : kAhead<false>);
  const int64_t row_bytes = a.hidden * mist::type_bytes(d->table_type);
  const bool by_slab = !pos && a.slabs > 1 && 16 % a.slabs == 0 && (a.rows * row_bytes <= kHeld || rows_reached(a.n, a.rows) * row_bytes <= kHeld);
  const int64_t groups = (a.n + per_wave - 1) / per_wave;
  // A launch's grid stays below 2^32 threads; whole blocks of groups, so that no group is in two launches.
  const int64_t most = ((int64_t)1 << 23) / a.slabs * kWaves;
  mist::with_types(d->act_type, d->table_type, [&](auto x, auto w) {
    using A = typename decltype(x)::type;
    using W = typename decltype(w)::type;
    with_layout<A, W>(d->hidden, [&](auto layout) {
      const auto kernel = pos ? k_embed<A, W, layout.value, true> : k_embed<A, W, layout.value, false>;
      for (int64_t group0 = 0; group0 < groups; group0 += most) {
        const int64_t count = std::min(most, groups - group0);
        const int64_t waves = (by_slab ? (count + kWaves - 1) / kWaves * kWaves : count) * a.slabs;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((waves + kWaves - 1) / kWaves)), dim3(kThreads), 0, (hipStream_t)stream, a,
                           (int32_t)per_wave, by_slab, (int32_t)group0, ids, (const W*)table, (const W*)pos, (A*)out);
      }
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
  const int64_t join_blocks = std::min<int64_t>(s.chunks / 2, kJoinRuns) * a.slabs;  // at most 2^7 2^15
  const hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  const RowArgs r{(const Entry*)(ws + s.order), (int32_t*)(ws + s.longs), (float*)(ws + s.part), s.chunk, (int32_t)s.chunks, accumulate, s.chunks * a.slabs};
  mist::with_types(d->act_type, d->table_type, [&](auto x, auto w) {
    using A = typename decltype(x)::type;
    using W = typename decltype(w)::type;
    const PosArgs<A, W> p{(const A*)grad, (W*)dpos, 0, 0, accumulate};
    with_layout<A, W>(d->hidden, [&](auto layout) {
      constexpr int L = layout.value;
      if (is_short(a)) {
        const int threads = std::max(256, (a.n + 63) / 64 * 64);
        const int64_t blocks = (int64_t)a.n * a.slabs + (accumulate ? 0 : (a.rows + kShortClear - 1) / kShortClear);
        PosArgs<A, W> all = p;
        all.end = dpos ? a.seq * a.slabs : 0;
        const dim3 grid((unsigned)(blocks + blocks_of(all.end, threads / 64)));
        if (grid.x) hipLaunchKernelGGL((k_short<A, W, L>), grid, dim3(threads), 0, st, a, all, ids, (const A*)grad, (W*)dtable, accumulate);
        return;
      }
      order_tokens<L>(a, ids, s, p, ws, st);
      const int64_t waves = r.sum_waves + (accumulate ? 0 : (a.rows + kClear - 1) / kClear);
      const bool once = a.n * a.hidden * (int64_t)sizeof(A) > kCache;
      const auto rows = once ? k_rows<A, W, L, true> : k_rows<A, W, L, false>;
      if (waves) hipLaunchKernelGGL(rows, dim3(blocks_of(waves, kWaves)), dim3(kThreads), 0, st, a, r, (const A*)grad, (W*)dtable);
      if (s.chunks > 2)
        hipLaunchKernelGGL((k_join<W, L>), dim3((unsigned)join_blocks), dim3(kThreads), 0, st, a, r, (W*)dtable);
    });
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MIST_OK : hip_failed(e, "embedding gradient");
}

}  // extern "C"
