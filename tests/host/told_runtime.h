// A device runtime on host memory whose calls can be told to fail, for programs linked to the library: their
// symbols come before those of the runtime that the library is linked to.  No kernel runs; device memory is
// zero until something is copied there.
#pragma once
#include <cstdio>
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "spanq.h"

namespace {
int fail_in = -1;  // calls until one fails, -1: none does
int calls = 0;     // that could have failed
int live = 0;      // device allocations
constexpr int kError = 2;  // out of memory
int launch_error = 0;

int step() {
  ++calls;
  if (fail_in < 0) return 0;
  return fail_in-- == 0 ? kError : 0;
}
int make(void** p, size_t n) {
  const int e = step();
  if (e) return e;
  *p = std::calloc(1, n ? n : 1);
  ++live;
  return 0;
}
int drop(void* p) {
  if (p) --live;
  std::free(p);
  return 0;
}
}  // namespace

extern "C" {
int hipSetDevice(int) { return step(); }
int hipGetDevice(int* d) { return *d = 0; }
int hipDeviceGetAttribute(int* v, int, int) { return *v = 0; }
int hipDeviceGetDefaultMemPool(void** p, int) { *p = nullptr; return 0; }
int hipMemPoolSetAttribute(void*, int, void*) { return 0; }
int hipDeviceSynchronize() { return 0; }
int hipMalloc(void** p, size_t n) { return make(p, n); }
int hipFree(void* p) { return drop(p); }
int hipMallocAsync(void** p, size_t n, void*) { return make(p, n); }
int hipFreeAsync(void* p, void*) { return drop(p); }
int hipMemcpy(void* to, const void* from, size_t n, int) {
  std::memcpy(to, from, n);
  return 0;
}
int hipMemcpyAsync(void* to, const void* from, size_t n, int, void*) {
  const int e = step();
  if (!e) std::memcpy(to, from, n);
  return e;
}
int hipEventCreateWithFlags(void** e, unsigned) {
  *e = nullptr;
  const int r = step();
  if (!r) *e = std::malloc(1);
  return r;
}
int hipEventCreate(void** e) { return hipEventCreateWithFlags(e, 0); }
int hipEventDestroy(void* e) {
  std::free(e);
  return 0;
}
int hipEventRecord(void*, void*) { return step(); }
int hipEventSynchronize(void*) { return step(); }
int hipEventQuery(void*) { return 0; }
int hipStreamSynchronize(void*) { return step(); }
int hipStreamWaitEvent(void*, void*, unsigned) { return step(); }
int hipStreamIsCapturing(void*, int* s) { return *s = 0; }
int hipThreadExchangeStreamCaptureMode(int*) { return 0; }
int hipGetLastError() {
  const int e = launch_error;
  launch_error = 0;
  return e;
}
const char* hipGetErrorString(int) { return "told to fail"; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipGetSymbolAddress(void** p, const void*) {
  static char there[1 << 20];
  *p = there;
  return 0;
}
int __hipPushCallConfiguration(unsigned long long, unsigned, unsigned long long, unsigned, size_t, void*) { return 0; }
int __hipPopCallConfiguration(unsigned* grid, unsigned* block, size_t* lds, void** stream) {
  for (int i = 0; i < 3; ++i) grid[i] = block[i] = 1;
  *lds = 0;
  *stream = nullptr;
  return 0;
}
int hipLaunchKernel(const void*, unsigned long long, unsigned, unsigned long long, unsigned, void**, size_t, void*) {
  const int e = step();
  if (e) launch_error = e;
  return e;
}
int hipHostMalloc(void** p, size_t n, unsigned) { return make(p, n); }
int hipHostFree(void* p) { return drop(p); }
// the matrix product library, which is not told to do anything
int hipblasLtCreate(void** h) { return *h = nullptr, 0; }
int hipblasLtDestroy(void*) { return 0; }
int hipblasLtMatmulDescCreate(void** d, int, int) { return *d = nullptr, 0; }
int hipblasLtMatmulDescDestroy(void*) { return 0; }
int hipblasLtMatmulPreferenceCreate(void** p) { return *p = nullptr, 0; }
int hipblasLtMatmulPreferenceDestroy(void*) { return 0; }
int hipblasLtMatmulPreferenceSetAttribute(void*, int, const void*, size_t) { return 0; }
int hipblasLtMatrixLayoutCreate(void** l, int, uint64_t, uint64_t, int64_t) { return *l = nullptr, 0; }
int hipblasLtMatrixLayoutDestroy(void*) { return 0; }
int hipblasLtMatmulAlgoGetHeuristic(void*, void*, void*, void*, void*, void*, void*, int, void* result, int* found) {
  struct Result {  // an algorithm (24 bytes), its workspace, status and figures
    unsigned long long algo[3], workspace, rest[3];
  };
  *static_cast<Result*>(result) = Result{};
  *found = 1;
  return 0;
}
int hipblasLtMatmul(void*, void*, const void*, const void*, void*, const void*, void*, const void*, const void*, void*, void*,
                    void*, const void*, void*, size_t, void*) {
  return step() ? 7 : 0;
}
}

namespace {

#define CHECK(x)                                                                     \
  do {                                                                               \
    if (!(x)) {                                                                      \
      std::fprintf(stderr, "line %d: %s (%s)\n", __LINE__, #x, span_last_error());  \
      std::exit(1);                                                                  \
    }                                                                                \
  } while (0)

struct Seen {
  std::vector<int32_t> pages[2];
  int64_t free_pages, pinned, steps, tokens, decode_pages;
  bool operator==(const Seen& o) const {
    return pages[0] == o.pages[0] && pages[1] == o.pages[1] && free_pages == o.free_pages && pinned == o.pinned &&
           steps == o.steps && tokens == o.tokens && decode_pages == o.decode_pages;
  }
};

Seen look(span_pool* pool, span_plan_t* plan) {
  Seen s{};
  for (int q = 0; q < 2; ++q) {
    int32_t n = 0, hit = 0;
    s.pages[q].resize(64);
    CHECK(span_plan_block_table(plan, q, q == 0 ? 1 : 0, s.pages[q].data(), 64, &n, &hit) == SPAN_OK);
    s.pages[q].resize(n);
  }
  span_pool_info i{};
  CHECK(span_pool_get_info(pool, &i) == SPAN_OK);
  span_stats st{};
  CHECK(span_plan_stats(plan, &st) == SPAN_OK);
  s.free_pages = i.free_pages;
  s.pinned = i.pinned_pages;
  s.steps = st.decode_steps;
  s.tokens = st.decode_tokens;
  s.decode_pages = st.decode_pages;
  return s;
}

}  // namespace
