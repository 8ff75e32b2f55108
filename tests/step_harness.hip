// The host side of the training-step operators on the CPU: mist_step.hip and mist_embed.hip themselves, compiled
// for the host alone, over a stand-in for the HIP runtime whose device memory is host memory and whose kernels
// only leave a record of their launch.  Each scenario exits with 0, or prints what differs.  Built and run by
// test_step_harness.py.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "../paper_2503_19050_amd/csrc/mist_ops.h"

namespace lookup {  // both files have names of their own for the same things
#include "../paper_2503_19050_amd/csrc/mist_embed.hip"
}
#include "../paper_2503_19050_amd/csrc/mist_step.hip"

namespace {

struct Launch {
  dim3 grid, block;
  lookup::EmbedArgs embed;   // k_embed's arguments, where the scenario launches only it
  int32_t per_wave, group0;
  bool by_slab;
};
std::vector<Launch> g_launches;
bool g_is_embed = false;
int g_device = 0, g_pending = 0;  // the current device; launches not yet waited for
int g_syncs_fail = 0;             // device synchronizations that fail from here on
long g_copies_left = -1, g_mallocs_left = -1, g_news_left = -1;  // calls that succeed before one fails (-1: none does)
int g_allocated = 0, g_freed_in_use = 0, g_freed_on = -1;
int g_bad = 0;
std::string g_error;
dim3 g_grid, g_block;

void check(bool ok, const char* what) {
  if (!ok) {
    std::printf("%s\n", what);
    g_bad = 1;
  }
}

void* take(size_t n, void*, void*) {
  if (g_mallocs_left >= 0 && g_mallocs_left-- == 0) return nullptr;
  ++g_allocated;
  return std::malloc(n);
}
void give(void* p, void*) {
  if (g_pending) ++g_freed_in_use;
  g_freed_on = g_device;
  --g_allocated;
  std::free(p);
}
const mist_allocator kAlloc{take, give, nullptr};

}  // namespace

void* operator new(size_t n) {
  if (g_news_left >= 0 && g_news_left-- == 0) throw std::bad_alloc();
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

namespace mist {
mist_status lib_fail(mist_status code, const char* msg) noexcept {
  const long news = g_news_left;
  g_news_left = -1;
  g_error = msg;
  g_news_left = news;
  return code;
}
}  // namespace mist

extern "C" {
hipError_t hipMalloc(void** p, size_t n) { return (*p = take(n, nullptr, nullptr)) ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void* p) {
  give(p, nullptr);
  return hipSuccess;
}
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) {
  if (g_copies_left >= 0 && g_copies_left-- == 0) return hipErrorUnknown;
  std::memcpy(d, s, n);
  return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipDeviceSynchronize() {
  if (g_syncs_fail) {
    --g_syncs_fail;
    return hipErrorStreamCaptureUnsupported;
  }
  g_pending = 0;
  return hipSuccess;
}
hipError_t hipGetDevice(int* d) {
  *d = g_device;
  return hipSuccess;
}
hipError_t hipSetDevice(int d) {
  g_device = d;
  return hipSuccess;
}
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
  Launch l{grid, block, {}, 0, 0, false};
  if (g_is_embed) {
    l.embed = *(const lookup::EmbedArgs*)args[0];
    l.per_wave = *(const int32_t*)args[1];
    l.by_slab = *(const bool*)args[2];
    l.group0 = *(const int32_t*)args[3];
  }
  g_launches.push_back(l);
  ++g_pending;
  check((uint64_t)grid.x * block.x < 1ull << 32 && (uint64_t)grid.y * block.y < 1ull << 32 && grid.x && grid.y && block.x <= 1024,
        "a launch of 2^32 threads or more, or of none");
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

float g_values[1 << 12];
mist_step_record g_record;
double g_workspace[MIST_NORM_WORKSPACE / 8];
const mist_clip_desc kClip{MIST_NORM_L2, 1.0f, 1.0};
const mist_adam_desc kAdam{0.1, 0.9, 0.99, 1e-8, 0.0};

mist_tensors* list(std::vector<const void*> at, std::vector<int64_t> sizes, int32_t type = MIST_F32, const mist_allocator* alloc = &kAlloc) {
  mist_tensors* T = nullptr;
  check(mist_tensors_create(at.data(), sizes.data(), (int64_t)at.size(), type, alloc, &T) == MIST_OK && T, "a list is refused");
  return T;
}
mist_tensors* part(int64_t first, int64_t n) { return list({g_values + first}, {n}); }

// Tables hold what was given, are freed on the list's device after its work, and the current device stays.
void lists() {
  for (const mist_allocator* alloc : {&kAlloc, (const mist_allocator*)nullptr}) {
    mist_tensors* T = list({g_values, nullptr, g_values + 5}, {3, 0, 4000}, MIST_F32, alloc);
    check(T->n_pieces == 2 && T->list.ptr[2] == (uint64_t)(uintptr_t)(g_values + 5) && T->list.size[2] == 4000, "the tables' addresses or sizes");
    check(T->list.piece[1].tensor == 2 && T->list.piece[1].part == 0, "the tables' pieces");
    check(mist_grad_norm(T, &kClip, 0, 1, &g_record, g_workspace, sizeof g_workspace, nullptr) == MIST_OK && g_launches.size() == 2, "the norm's launches");
    g_launches.clear();
    g_device = 3;
    check(mist_grad_norm(T, &kClip, 0, 1, &g_record, g_workspace, sizeof g_workspace, nullptr) == MIST_E_INVALID, "a call with another device current");
    check(mist_tensors_destroy(T) == MIST_OK && g_device == 3 && g_freed_on == 0 && !g_allocated && !g_freed_in_use, "the list's end");
    g_device = 0;
  }
  mist_tensors* T = list({nullptr, nullptr}, {0, 0});   // no table
  check(!g_allocated && mist_grad_norm(T, &kClip, 0, 1, &g_record, nullptr, 0, nullptr) == MIST_OK && g_launches.size() == 1, "an empty list's norm");
  check(mist_grad_clip(T, &g_record, T, nullptr) == MIST_OK && g_launches.size() == 1, "an empty list's clipping");
  check(mist_tensors_destroy(T) == MIST_OK, "an empty list's end");
}

// Whatever allocation or copy fails, there is no list, and what was allocated is freed once.
void failures() {
  const void* at[2] = {g_values, g_values + 2048};
  const int64_t sizes[2] = {2000, 1000};
  for (const mist_allocator* alloc : {&kAlloc, (const mist_allocator*)nullptr}) {
    for (long* left : {&g_news_left, &g_mallocs_left, &g_copies_left}) {
      bool done = false;
      for (long k = 0; k < 20 && !done; ++k) {
        *left = k;
        mist_tensors* T = (mist_tensors*)&g_record;
        const mist_status st = mist_tensors_create(at, sizes, 2, MIST_F32, alloc, &T);
        done = *left >= 0;
        *left = -1;
        check(st == MIST_OK ? T != nullptr : !T && !g_allocated && !g_error.empty(), "a failed list");
        if (!done) check(st == (left == &g_copies_left ? MIST_E_DEVICE : MIST_E_NOMEM), "a failed list's status");
        if (T) mist_tensors_destroy(T);
        check(!g_allocated, "memory left");
      }
      check(done, "a list that is never made");
    }
  }
}

// A wait that fails, as inside a capture, frees nothing: the list is there for another try.
void failing_wait() {
  for (const mist_allocator* alloc : {&kAlloc, (const mist_allocator*)nullptr}) {
    mist_tensors* T = list({g_values}, {5000}, MIST_BF16, alloc);
    mist_grad_norm(T, &kClip, 0, 1, &g_record, g_workspace, sizeof g_workspace, nullptr);
    g_syncs_fail = 2;
    g_device = 2;
    check(mist_tensors_destroy(T) == MIST_E_DEVICE && g_allocated == 1 && !g_freed_in_use && g_device == 2, "tables freed while in use");
    if (g_allocated != 1) return;
    check(mist_tensors_destroy(T) == MIST_E_DEVICE && g_allocated == 1, "tables freed while in use");
    check(mist_tensors_destroy(T) == MIST_OK && !g_allocated && !g_freed_in_use && g_device == 2, "a second try");
    g_device = 0;
  }
}

// Lists that are written hold no value twice; lists that are read may.
void overlaps() {
  mist_tensors *a = part(0, 100), *b = part(100, 100), *c = part(200, 100), *d = part(300, 100), *e = part(400, 100);
  auto clip = [&](mist_tensors* g, mist_tensors* out) { return mist_grad_clip(g, &g_record, out, nullptr); };
  auto adam = [&](mist_tensors* p, mist_tensors* m, mist_tensors* v, mist_tensors* g, mist_tensors* w) {
    return mist_adam_step(p, m, v, g, w, &g_record, &kAdam, nullptr);
  };
  check(clip(a, a) == MIST_OK && clip(a, b) == MIST_OK && adam(a, b, c, d, e) == MIST_OK, "lists apart");
  for (auto* T : {a, b, c, d, e}) mist_tensors_destroy(T);
  const std::vector<int64_t> sizes{100, 7, 0, 100};
  auto four = [&](int64_t first, int64_t second, int64_t fourth) {
    return list({g_values + first, g_values + second, nullptr, g_values + fourth}, sizes);
  };
  mist_tensors *p = four(700, 800, 807), *m = four(1000, 1200, 1100), *v = four(1607, 1500, 1507), *g = four(2000, 2300, 2400), *w = four(2707, 2700, 2807);
  check(clip(g, g) == MIST_OK && clip(g, p) == MIST_OK && adam(p, m, v, g, w) == MIST_OK && adam(p, m, v, g, nullptr) == MIST_OK, "tensors that touch");
  for (mist_tensors* bad : {four(3000, 3200, 3000), four(3000, 3099, 3200), four(3000, 3093, 3200), four(3106, 3100, 3300), four(3050, 3010, 3000)}) {
    const size_t launches = g_launches.size();
    check(clip(bad, bad) == MIST_E_INVALID && clip(g, bad) == MIST_E_INVALID, "clipping into values that occur twice");
    check(adam(bad, m, v, g, w) == MIST_E_INVALID && adam(p, bad, v, g, w) == MIST_E_INVALID && adam(p, m, bad, g, nullptr) == MIST_E_INVALID &&
              adam(p, m, v, g, bad) == MIST_E_INVALID, "a step of values that occur twice");
    check(g_launches.size() == launches, "a refused call's launches");
    check(clip(bad, g) == MIST_OK && adam(p, m, v, bad, w) == MIST_OK, "values that are read twice");
    mist_tensors_destroy(bad);
  }
  for (auto* T : {p, m, v, g, w}) mist_tensors_destroy(T);
}

// Long lists: every piece has a block.
void grids() {
  for (const int64_t n : {(int64_t)1, kChunk, kChunk + 1, kChunk * 2047, kChunk * (kGridX / 2) + 5, kChunk * kGridX - 1, kChunk * kGridX + 1}) {
    mist_tensors *g = list({(const void*)4096}, {n}, MIST_BF16), *p = list({(const void*)((int64_t)1 << 45)}, {n}, MIST_F32);
    g_launches.clear();
    check(mist_grad_clip(g, &g_record, p, nullptr) == MIST_OK && g_launches.size() == 1, "clipping of a long list");
    check((int64_t)g_launches[0].grid.x * g_launches[0].grid.y >= g->n_pieces * kClipBlocks, "pieces without a block");
    check(mist_grad_norm(g, &kClip, 0, 0, &g_record, g_workspace, sizeof g_workspace, nullptr) == MIST_OK && g_launches.size() == 3 &&
              g_launches[1].grid.x <= MIST_NORM_WORKSPACE / 8, "the norm of a long list");
    mist_tensors_destroy(g);
    mist_tensors_destroy(p);
  }
}

// Lookups: the launches' waves take every group of tokens and slab once.
void lookups() {
  g_is_embed = true;
  for (const int64_t n : {(int64_t)1, (int64_t)300, (int64_t)70000, (int64_t)1 << 27, ((int64_t)1 << 27) + 1, ((int64_t)1 << 30) - 1}) {
    for (const int64_t hidden : {(int64_t)1, (int64_t)512, (int64_t)513, (int64_t)1536, (int64_t)4096, (int64_t)1 << 24}) {
      if (hidden > 4096 && n > 70000) continue;  // more than any memory
      for (const bool pos : {false, true}) {
        for (const int64_t rows : {(int64_t)100, (int64_t)1 << 30}) {
          const mist_embed_desc d{1, n, hidden, rows, 0, n, 0, hidden, hidden, hidden, 8, MIST_BF16, MIST_BF16, 1.0f};
          g_launches.clear();
          check(mist_embed_forward(&d, (void*)4096, (void*)4096, pos ? (void*)4096 : nullptr, (void*)4096, nullptr) == MIST_OK, "a lookup is refused");
          int64_t next = 0, groups = 0;
          for (const Launch& l : g_launches) {
            const int64_t slabs = l.embed.slabs;
            groups = (n + l.per_wave - 1) / l.per_wave;
            check(l.group0 == next, "groups between two launches");
            const int64_t covered = l.by_slab ? l.grid.x / slabs * lookup::kWaves : l.grid.x * (int64_t)lookup::kWaves / slabs;
            check(!l.by_slab || l.grid.x % slabs == 0, "a slab's last block");
            const bool last = &l == &g_launches.back();
            check(last || l.grid.x * (int64_t)lookup::kWaves == covered * slabs, "a group in two launches");
            next += covered;
          }
          check(next >= groups && groups > 0, "groups that no launch takes");
          if (g_bad) return;
        }
      }
    }
  }
}

// Which lookups take the slabs in turn: by the rows that their tokens reach, from both sides of where it was measured.
void slab_order() {
  g_is_embed = true;
  for (const int64_t rows : {(int64_t)1, (int64_t)300, (int64_t)20000}) {
    for (const int64_t n : {(int64_t)1, (int64_t)5000, (int64_t)400000}) {
      double sum = 0.0;
      for (int64_t k = 1; k <= rows; ++k) sum += 1.0 - std::pow(1.0 - 1.0 / (double)k / std::log((double)rows + 1.0), (double)n);
      if (rows > 1) check(std::fabs(lookup::rows_reached(n, rows) - sum) < 0.03 * sum + 1.0, "the rows reached");
      check(lookup::rows_reached(n, rows) >= 0.0 && lookup::rows_reached(n, rows) <= (double)rows, "more rows than there are");
    }
  }
  const struct {
    int64_t n, hidden, rows;
    int32_t type;
    bool pos, want;
  } all[] = {{65536, 4096, 13671, MIST_BF16, false, true},  {65536, 4096, 24000, MIST_BF16, false, false}, {65536, 4096, 32000, MIST_F16, false, false},
             {16384, 4096, 32000, MIST_BF16, false, true},  {65536, 2048, 50257, MIST_BF16, false, true},  {32768, 8192, 4000, MIST_BF16, false, true},
             {65536, 8192, 4882, MIST_BF16, false, true},   {65536, 8192, 12000, MIST_BF16, false, false}, {65536, 2048, 15625, MIST_F32, false, true},
             {65536, 2048, 23437, MIST_F32, false, false},  {16384, 16384, 4000, MIST_BF16, false, false}, {65536, 512, 100, MIST_BF16, false, false},
             {65536, 2048, 50257, MIST_BF16, true, false},  {65536, 2560, 100, MIST_BF16, false, false},   {1, 1024, 1, MIST_BF16, false, true}};
  for (const auto& c : all) {
    const mist_embed_desc d{1, c.n, c.hidden, c.rows, 0, c.n, 0, c.hidden, c.hidden, c.hidden, 8, c.type, c.type, 1.0f};
    g_launches.clear();
    check(mist_embed_forward(&d, (void*)4096, (void*)4096, c.pos ? (void*)4096 : nullptr, (void*)4096, nullptr) == MIST_OK &&
              g_launches.size() == 1 && g_launches[0].by_slab == c.want, "which lookups take the slabs in turn");
  }
}

}  // namespace

int main(int argc, char** argv) {
  const struct {
    const char* name;
    void (*run)();
  } all[] = {{"lists", lists}, {"failures", failures}, {"failing_wait", failing_wait}, {"overlaps", overlaps}, {"grids", grids}, {"lookups", lookups}, {"slab_order", slab_order}};
  for (const auto& s : all)
    if (argc == 2 && !std::strcmp(argv[1], s.name)) {
      s.run();
      return g_bad;
    }
  std::printf("no such scenario\n");
  return 2;
}
