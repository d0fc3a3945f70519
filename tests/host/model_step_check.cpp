// Calls of a decoder stack whose calls of the device runtime, or whose host allocations, fail one after
// another: every one ends with an error and no exception, a decode step that fails appends nothing, and what
// failed goes through when it is tried again.
#include <new>

#include "told_runtime.h"

namespace {
int throw_in = -1;  // host allocations until one fails, -1: none does
}

void* operator new(size_t n) {
  if (throw_in >= 0 && throw_in-- == 0) throw std::bad_alloc();
  void* p = std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

namespace {

bool same_pages(const Seen& a, const Seen& b) {
  return a.pages[0] == b.pages[0] && a.pages[1] == b.pages[1] && a.free_pages == b.free_pages && a.pinned == b.pinned;
}

// f() with every call of the runtime, then every host allocation failing in turn; the last one goes through.
// `undo` takes back a call that went through with a failure that it can do without.
template <class F, class U>
int each_failure(span_pool* pool, span_plan_t* plan, bool allocations, F f, U undo) {
  for (int at = 0, failed = 0;; ++at) {
    const Seen before = look(pool, plan);
    int& countdown = allocations ? throw_in : fail_in;
    countdown = at;
    const int rc = f();
    const bool hit = countdown < 0;
    countdown = -1;
    if (!hit) {
      CHECK(rc == SPAN_OK);
      return failed;
    }
    if (rc == SPAN_OK) {
      undo();
    } else {
      ++failed;
      CHECK(!allocations || rc == SPAN_ENOMEM);
      CHECK(same_pages(look(pool, plan), before));
    }
  }
}

}  // namespace

int main() {
  constexpr int kLayers = 2, kHidden = 64, kFfn = 128, kVocab = 64;
  span_pool_config cfg{};
  cfg.num_layers = kLayers;
  cfg.num_q_heads = 2;
  cfg.num_kv_heads = 1;
  cfg.head_dim = 64;
  cfg.page_size = 16;
  cfg.num_pages = 64;
  cfg.dtype = SPAN_BF16;
  cfg.rope_theta = 1e4f;
  cfg.device = 0;
  span_pool* pool = nullptr;
  CHECK(span_pool_create(&cfg, &pool) == SPAN_OK);
  static char weights[64] __attribute__((aligned(64)));  // (never read)
  const void* table[kLayers] = {weights, weights};
  span_model_config mc{};
  mc.num_layers = kLayers;
  mc.hidden = kHidden;
  mc.num_q_heads = 2;
  mc.num_kv_heads = 1;
  mc.head_dim = 64;
  mc.ffn = kFfn;
  mc.vocab = kVocab;
  mc.rms_eps = 1e-5f;
  mc.embed = mc.final_norm = mc.lm_head = weights;
  mc.attn_norm = mc.w_qkv = mc.w_o = mc.ffn_norm = mc.w_gate_up = mc.w_down = table;
  span_model* model = nullptr;
  CHECK(span_model_create(pool, &mc, &model) == SPAN_OK);
  span_model_adapters ad{};
  ad.n_adapters = 2;
  ad.max_rank = 8;
  ad.a_qkv = ad.b_qkv = ad.a_down = ad.b_down = table;
  CHECK(span_model_set_adapters(model, &ad) == SPAN_OK && span_model_set_qk_norm(model, table, nullptr) == SPAN_OK);

  std::vector<int32_t> tok(64);
  for (int i = 0; i < 64; ++i) tok[i] = i;
  span_tokens frag{tok.data(), 5, 0, 20};
  span_query q[2] = {};
  q[0].prefix = span_tokens{tok.data(), 17, 0, 0};
  q[0].frags = &frag;
  q[0].n_frags = 1;
  q[0].cross = span_tokens{tok.data() + 30, 13, 0, 30};
  q[1].cross = span_tokens{tok.data() + 50, 3, 0, 50};
  const int32_t ids[2] = {1, -1}, next[2] = {3, 5}, drafts[2][3] = {{1, 2, 3}, {4, 0, 0}}, n_drafts[2] = {3, 1};
  const float ua[2][3] = {}, us[2] = {0.5f, 0.5f}, heat[2] = {1.f, 0.f};
  const span_sampling sampling{&ua[0][0], us, heat, nullptr};

  int failed = 0;
  for (bool allocations : {false, true}) {
    span_plan_t* plan = nullptr;
    CHECK(span_plan(pool, q, 2, nullptr, &plan) == SPAN_OK && span_plan_set_adapters(plan, ids) == SPAN_OK);
    int32_t first[2], out[2][4], n_out[2];
    float lp[2][4];
    failed += each_failure(pool, plan, allocations, [&] {
      return span_model_forward(model, plan, tok.data(), 64, kLayers, nullptr, nullptr, first, nullptr);
    }, [] {});
    for (int again = 0; again < 3; ++again) {
      failed += each_failure(pool, plan, allocations, [&] { return span_model_decode(model, plan, next, nullptr, first, nullptr); },
                             [&] {
                               const int32_t back[2] = {1, 1};
                               CHECK(span_plan_rewind(plan, back) == SPAN_OK);
                             });
      failed += each_failure(pool, plan, allocations, [&] {
        return span_model_decode_drafts(model, plan, next, &drafts[0][0], n_drafts, 3, &sampling, &out[0][0], n_out, &lp[0][0],
                                        nullptr);
      }, [&] {
        const int32_t back[2] = {n_out[0], n_out[1]};
        CHECK(span_plan_rewind(plan, back) == SPAN_OK);
      });
      CHECK(n_out[0] == 1 && n_out[1] == 1);  // (no kernel ran: nothing was accepted)
    }
    const Seen last = look(pool, plan);
    CHECK(last.pages[0].size() == (13 + 6 + 15) / 16 && last.pages[1].size() == 1);
    CHECK(span_plan_destroy(plan) == SPAN_OK);
  }
  span_model* shared = model;

  // queries that share their cross rows have one activation for both: one adapter too
  q[1].cross = q[0].cross;
  for (int other : {-1, 1}) {
    span_plan_t* plan = nullptr;
    const int32_t both[2] = {1, other};
    CHECK(span_plan(pool, q, 2, nullptr, &plan) == SPAN_OK && span_plan_set_adapters(plan, both) == SPAN_OK);
    int32_t first[2];
    CHECK(span_model_forward(shared, plan, tok.data(), 64, kLayers, nullptr, nullptr, first, nullptr) ==
          (other == 1 ? SPAN_OK : SPAN_EINVAL));
    CHECK(span_plan_destroy(plan) == SPAN_OK);
  }
  CHECK(span_model_destroy(shared) == SPAN_OK);

  // products wider than the operator takes are refused when they are given, not in the middle of a forward
  mc.ffn = (1 << 19) + 8;
  CHECK(span_model_create(pool, &mc, &model) == SPAN_OK);
  CHECK(span_model_set_adapters(model, &ad) == SPAN_OK);  // (down: a long reduction)
  ad.a_gate_up = ad.b_gate_up = table;
  CHECK(span_model_set_adapters(model, &ad) == SPAN_EINVAL);
  CHECK(span_model_destroy(model) == SPAN_OK);
  CHECK(span_pool_destroy(pool) == SPAN_OK);
  CHECK(failed > 300 && live == 0);
  std::printf("%d failures\nall checks passed\n", failed);
}
