// Decode steps whose calls of the device runtime fail, one after another: nothing is appended, and the
// step can be planned again.  The runtime is this program's own, on host memory (its symbols come before
// the library's runtime), and no kernel runs.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "spanq.h"

namespace {
int fail_in = -1;  // calls until one fails, -1: none does
int calls = 0;     // that could have failed
int live = 0;      // device allocations
constexpr int kError = 2;  // out of memory

int step() {
  ++calls;
  if (fail_in < 0) return 0;
  return fail_in-- == 0 ? kError : 0;
}
int make(void** p, size_t n) {
  const int e = step();
  if (e) return e;
  *p = std::malloc(n ? n : 1);
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
int hipStreamSynchronize(void*) { return 0; }
int hipStreamWaitEvent(void*, void*, unsigned) { return step(); }
int hipStreamIsCapturing(void*, int* s) { return *s = 0; }
int hipThreadExchangeStreamCaptureMode(int*) { return 0; }
int hipGetLastError() { return 0; }
const char* hipGetErrorString(int) { return "told to fail"; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipGetSymbolAddress(void** p, const void*) {
  static char there[1 << 20];
  *p = there;
  return 0;
}
int hipLaunchKernel(const void*, unsigned long long, unsigned, unsigned long long, unsigned, void**, size_t, void*) { return 0; }
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

// Steps of one plan, each tried with every call of the runtime failing in turn before it is let through.
int run(int dtype, void* other_stream) {
  span_pool_config cfg{};
  cfg.num_layers = 1;
  cfg.num_q_heads = 2;
  cfg.num_kv_heads = 1;
  cfg.head_dim = 64;
  cfg.page_size = 16;
  cfg.num_pages = 64;
  cfg.dtype = dtype;
  cfg.rope_theta = 1e4f;
  cfg.device = 0;
  span_pool* pool = nullptr;
  CHECK(span_pool_create(&cfg, &pool) == SPAN_OK);
  std::vector<int32_t> tok(64);
  for (int i = 0; i < 64; ++i) tok[i] = i;
  span_tokens frag{tok.data(), 5, 20};
  span_query q[2] = {};
  q[0].prefix = span_tokens{tok.data(), 17, 0};
  q[0].frags = &frag;
  q[0].n_frags = 1;
  q[0].cross = span_tokens{tok.data() + 30, 13, 30};
  q[1].cross = span_tokens{tok.data() + 50, 3, 50};
  span_plan_t* plan = nullptr;
  CHECK(span_plan(pool, q, 2, nullptr, &plan) == SPAN_OK);
  const Seen first = look(pool, plan);
  int failed = 0;
  const int32_t steps[][2] = {{1, 40}, {30, 0}, {0, 2}, {5000 / 16, 1}, {2, 2}};
  for (const auto& n : steps) {
    const int64_t rows[2] = {0, 1000};
    for (int at = 0;; ++at) {
      const Seen before = look(pool, plan);
      fail_in = at;
      const int rc = span_plan_decode(plan, n, rows, at % 2 ? other_stream : nullptr);
      const bool hit = fail_in < 0;
      fail_in = -1;
      if (rc == SPAN_OK && !hit) break;
      if (rc == SPAN_OK) {  // a failure that the call can do without (a kept block's event)
        const int32_t back[2] = {n[0], n[1]};
        CHECK(span_plan_rewind(plan, back) == SPAN_OK);
        continue;
      }
      ++failed;
      CHECK(hit && std::strlen(span_last_error()) > 0);
      Seen now = look(pool, plan);
      // (steps that went through and were taken back stay in the totals)
      CHECK(now == before);
      char x[256];
      CHECK(span_decode_attend(plan, 0, x, x, x, x, nullptr) == SPAN_ESTATE);
    }
  }
  const Seen last = look(pool, plan);
  CHECK(last.pages[0].size() == (13 + 1 + 30 + 312 + 2 + 15) / 16 && last.pages[1].size() == (3 + 40 + 2 + 1 + 2 + 15) / 16);
  CHECK(span_plan_destroy(plan) == SPAN_OK);
  span_pool_info i{};
  CHECK(span_pool_get_info(pool, &i) == SPAN_OK && i.free_pages == 64);
  CHECK(span_pool_destroy(pool) == SPAN_OK);
  CHECK(!(first == last));
  return failed;
}

}  // namespace

int main() {
  static char stream;
  int failed = 0;
  for (int dtype : {SPAN_F32, SPAN_BF16}) failed += run(dtype, &stream);
  CHECK(failed > 40 && live == 0);
  std::printf("%d failures\nall checks passed\n", failed);
}
