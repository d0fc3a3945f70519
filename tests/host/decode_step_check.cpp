// Decode steps whose calls of the device runtime fail, one after another: nothing is appended, and the
// step can be planned again.
#include "told_runtime.h"

namespace {

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
  span_tokens frag{tok.data(), 5, 0, 20};
  span_query q[2] = {};
  q[0].prefix = span_tokens{tok.data(), 17, 0, 0};
  q[0].frags = &frag;
  q[0].n_frags = 1;
  q[0].cross = span_tokens{tok.data() + 30, 13, 0, 30};
  q[1].cross = span_tokens{tok.data() + 50, 3, 0, 50};
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
