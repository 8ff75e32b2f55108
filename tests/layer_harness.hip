// The host side of the loss, the norms around a block and the kept activations on the CPU: their sources compiled for the
// host alone, over a stand-in for the HIP runtime whose kernels only leave a record of their launch.  Each scenario exits with 0, or
// prints what differs.  Built and run by test_layer_harness.py.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <string>
#include <type_traits>
#include <vector>

#include "../paper_2503_19050_amd/csrc/mist_ops.h"

namespace token {  // the files have names of their own for the same things
#include "../paper_2503_19050_amd/csrc/mist_token.hip"
}
namespace kept {
#include "../paper_2503_19050_amd/csrc/mist_kept.hip"
}
#include "../paper_2503_19050_amd/csrc/mist_block.hip"

namespace {

int g_bad = 0, g_launches = 0;
dim3 g_grid, g_block;
bool g_back = false;  // the next launch is k_backward
BackArgs g_args;
dim3 g_parts;

void check(bool ok, const char* what) {
  if (!ok) {
    std::printf("%s\n", what);
    g_bad = 1;
  }
}

}  // namespace

namespace mist {
mist_status lib_fail(mist_status code, const char*) noexcept { return code; }
}  // namespace mist

extern "C" {
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "stand-in error"; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  g_grid = grid;
  g_block = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* st) {
  *grid = g_grid;
  *block = g_block;
  *shared = 0;
  *st = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  if (g_back) {
    std::memcpy((void*)&g_args, args[0], sizeof g_args);
    g_parts = grid;
    g_back = false;
  }
  ++g_launches;
  check((uint64_t)grid.x * block.x < 1ull << 32 && grid.x && grid.y && grid.y < 65536 && block.x <= 1024 && block.x % 64 == 0 && block.y == 1,
        "a launch of 2^32 threads or more, of none, or of part of a wave");
  return hipSuccess;
}
void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
void __hipUnregisterFatBinary(void**) {}
}

namespace {

// Addresses that nothing reads, 2^52 apart.
template <class T = void>
T* at(int k) {
  return reinterpret_cast<T*>((uintptr_t)k << 52);
}

// Every launch is one the device takes, from single tokens to the most that is allowed.
void grids() {
  const struct {
    int64_t batch, seq;
  } tokens[] = {{1, 1}, {3, 5}, {1, 70000}, {70000, 1}, {1 << 15, (1 << 15) - 1}, {(1 << 30) - 1, 1}, {1, (1 << 30) - 1}, {0, 7}, {7, 0}};
  for (const auto& t : tokens) {
    const bool any = t.batch && t.seq;
    for (int32_t type : {MIST_F32, MIST_BF16, MIST_F16}) {
      for (int64_t rows : {1ll, 4096ll, 4097ll, 50257ll, 70001ll, (1ll << 31) - 2}) {
        const int64_t n = t.batch * t.seq;
        if ((__int128)n * rows * 4 > (__int128)1 << 51 || t.seq * rows > mist::kMostStride) continue;
        for (int32_t top : {0, 64}) {
          const mist_token_desc d{t.batch, t.seq, rows, 0, t.seq, t.seq * rows, rows, t.seq * rows, rows, 8, type, top, 1.0f};
          g_launches = 0;
          check(mist_token_logprob(&d, at(1), at(2), at<float>(3), at<float>(4), at<float>(5), at<int32_t>(6), at<float>(7), nullptr) == MIST_OK, "log probabilities");
          check(mist_token_part(&d, at(1), at(2), at<float>(3), at<int32_t>(6), at<float>(7), nullptr) == MIST_OK, "a part");
          for (int32_t ranks : {1, 16, 65536})
            check(mist_token_join(&d, ranks, at<float>(1), at<int32_t>(2), at<float>(3), at(4), at<float>(5), at<float>(6), at<float>(7), at<int32_t>(8), at<float>(9), nullptr) == MIST_OK,
                  "parts joined");
          check(mist_token_grad(&d, at(1), at(2), at<float>(3), at<float>(4), at<float>(5), at<float>(6), at(7), nullptr) == MIST_OK, "a gradient");
          check(mist_token_loss(&d, at(1), at(2), at<float>(3), 1.0f, at<float>(4), at(1), nullptr) == MIST_OK, "a loss in place");
          check(g_launches == (any ? 7 : 0), "the number of launches");
        }
      }
      for (int64_t hidden : {1ll, 7ll, 128ll, 129ll, 257ll, 512ll, 5120ll, 5632ll, 8192ll, 8193ll, 16384ll})
        for (int64_t gate : {0ll, 16384ll}) {
          const mist_block_desc d{t.batch, t.seq, hidden, hidden, hidden, hidden, hidden, gate, MIST_BLOCK_LAYER, type, type == MIST_F32 ? MIST_F32 : gate ? MIST_F32 : type, type, 1e-5f, 1.0f, 1.0f};
          check(mist_block_forward(&d, at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), at(9), at<float>(10), nullptr) == MIST_OK, "a norm");
          const mist_block_grads g{at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), at(9), hidden, hidden, hidden, hidden, 16384, 0};
          size_t bytes = 0;
          check(mist_block_workspace(&d, &g, &bytes) == MIST_OK && bytes < 2ull << 30, "a norm's workspace");
          check(mist_block_backward(&d, at(10), at(11), at<float>(12), at(13), at(14), at(15), at(16), &g, at(17), bytes, nullptr) == MIST_OK, "a norm's gradient");
        }
    }
  }
  for (int64_t rows : {0ll, 1ll, 1000003ll, (1ll << 31) - 1})
    for (int64_t width : {1ll, 127ll, 128ll, 13824ll, 60000ll, (1ll << 31) - 1}) {
      const int64_t groups = (width + 127) / 128;
      const bool fits = rows * groups < 1ll << 40;
      const mist_kept_desc d{rows, width, width, MIST_BF16};
      const mist_act_desc c{rows, width, width, width, width, width, MIST_F32, MIST_ACT_GELU};
      const mist_kept u{at<int8_t>(2), at<uint8_t>(3)}, g{at<int8_t>(4), at<uint8_t>(5)};
      const mist_status want = fits ? MIST_OK : MIST_E_INVALID;
      check(mist_kept_store(&d, at(1), at<int8_t>(2), at<uint8_t>(3), nullptr) == want && mist_kept_load(&d, at<int8_t>(2), at<uint8_t>(3), at(1), nullptr) == want, "kept");
      check(mist_act_forward(&c, at(1), at(6), at(7), &u, &g, nullptr) == want && mist_act_backward(&c, &u, &g, at(1), at(6), at(7), at(8), nullptr) == want, "activations");
    }
}

// The backward pass's parts take every token once, and their sums lie in the workspace beside each other.
void parts() {
  for (int64_t batch : {1, 2, 3, 7, 64, 300, 6000})
    for (int64_t seq : {1, 2, 3, 5, 31, 64, 513, 4099})
      for (int64_t hidden : {24, 200, 512, 2560, 8192, 9000})
        for (int64_t gate : {0, 16384}) {
          if (batch * seq > 400000) continue;
          const mist_block_desc d{batch, seq, hidden, hidden, hidden, hidden, hidden, gate, MIST_BLOCK_RMS, MIST_BF16, MIST_BF16, MIST_F32, 1e-5f, 1.0f, 1.0f};
          const mist_block_grads g{at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), at(9), hidden, hidden, hidden, hidden, 16384, 0};
          size_t bytes = 0;
          check(mist_block_workspace(&d, &g, &bytes) == MIST_OK, "a workspace");
          g_back = true;
          char* ws = at<char>(17);
          check(mist_block_backward(&d, at(10), at(11), at<float>(12), at(13), at(14), at(15), at(16), &g, ws, bytes, nullptr) == MIST_OK, "a gradient");
          const Parts& p = g_args.parts;
          check(!g_back && p.n == (int64_t)g_parts.x && p.batch * p.seq == batch * seq, "the launch's parts");
          std::vector<uint8_t> taken((size_t)(batch * seq));
          for (int64_t part = 0; part < p.n; ++part) {
            const int64_t first = part / p.pieces * p.seqs, row0 = part % p.pieces * p.rows;
            check(first < p.batch && row0 < p.seq, "a part without tokens");
            for (int64_t s = first; s < std::min(first + p.seqs, p.batch); ++s)
              for (int64_t r = row0; r < std::min(row0 + p.rows, p.seq); ++r) ++taken[(size_t)(s * p.seq + r)];
          }
          check(std::all_of(taken.begin(), taken.end(), [](uint8_t k) { return k == 1; }), "a token that no part takes, or two");
          const char* end = ws;
          for (int i = 0; i < kSlots; ++i) {
            if (!g_args.slot[i]) continue;
            check((const char*)g_args.slot[i] >= end, "sums that overlap");
            end = (const char*)(g_args.slot[i] + p.n * hidden);
          }
          check(end <= ws + bytes, "sums past the workspace");
          check((g_args.slot[4] == nullptr) == (g_args.dgate != nullptr) && (!g_args.dgate || p.pieces == 1), "where the gates' gradients go");
        }
}

// What shares memory: rows beside each other at one stride do not, and no difference of addresses or strides overflows.
void ranges() {
  const struct {
    int64_t shift, rows, stride, width;
    bool want;
  } all[] = {{0, 5, 10, 5, true}, {5, 5, 10, 5, false}, {4, 5, 10, 5, true}, {6, 5, 10, 5, true}, {-5, 5, 10, 5, false}, {15, 5, 10, 5, false},
             {14, 5, 10, 5, true}, {5, 1, 10, 5, false}, {4, 1, 10, 5, true}, {45, 5, 10, 5, false}, {44, 5, 10, 5, true}, {3, 5, 4, 5, true},
             {1, (1ll << 31) - 1, 1ll << 40, 1, false}, {0, (1ll << 31) - 1, 1ll << 40, 1, true}};
  for (const auto& c : all) {
    char* p = reinterpret_cast<char*>((uintptr_t)1 << 40);
    const mist::Rows a{p, c.rows, c.stride, c.width, 2}, b{p + 2 * c.shift, c.rows, c.stride, c.width, 2};
    check(mist::overlap(a, b) == c.want && mist::overlap(b, a) == c.want, "whether rows share memory");
  }
  const mist::Range r = mist::range_of(reinterpret_cast<void*>(UINTPTR_MAX - 100), 1ll << 31, 1ll << 40, 5, 4);
  check(r.hi == UINTPTR_MAX, "a range past the last address");
}

}  // namespace

int main(int argc, char** argv) {
  const struct {
    const char* name;
    void (*run)();
  } all[] = {{"grids", grids}, {"parts", parts}, {"ranges", ranges}};
  for (const auto& s : all)
    if (argc == 2 && !std::strcmp(argv[1], s.name)) {
      s.run();
      return g_bad;
    }
  std::printf("no such scenario\n");
  return 2;
}
