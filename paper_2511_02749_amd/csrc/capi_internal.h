// Internal entries shared by the C-ABI sources (not part of the public ABI).
#pragma once
#include <cstddef>
#include <cstdint>
#include <vector>

#include "../../include/spanq.h"

namespace spanq {

// span_plan's work.  With region == nullptr the plan's device data (work lists,
// scheduling counters, split-KV partials) come from a block the pool kept or the device's
// stream-ordered allocator, and the rotary table grows as needed.  With a region, they are placed
// in region[0, region_bytes) (256-byte aligned device memory of the pool's device)
// and nothing is allocated: SPAN_EINVAL if they do not fit or the table is too
// short, SPAN_ESTATE while another plan holds the device's region.  `who` names
// the entry point in error messages.
int plan_impl(span_pool* pool, const span_query* qs, int32_t nq, void* stream, span_plan_t** out,
              unsigned char* region, size_t region_bytes, const char* who);

// Device ordinal of a pool; -1 for a null or host-only pool.
int pool_device(const span_pool* pool);

// Record a failure for span_last_error and return its status.
int report(int code, const char* msg);

// The page index of a pool (host side).
const class PoolIndex* pool_index(const span_pool* pool);

// The pool a plan was made on.
span_pool* plan_pool(const span_plan_t* plan);

// Pool shape: {num_layers, num_q_heads, num_kv_heads, head_dim, dtype}.
void pool_shape(const span_pool* pool, int32_t out[5]);

// Caller row of each query's last cross token, -1 for a query without one.
void plan_last_cross_rows(const span_plan_t* plan, std::vector<int64_t>* rows);

// The adapter of each query's cross and decoded rows (span_plan_set_adapters), -1 for none;
// empty if the plan has none at all.  The cross rows of query q before any decode step
// are caller rows row0[q] .. row0[q] + n[q] - 1.
const std::vector<int32_t>& plan_adapters(const span_plan_t* plan);
void plan_cross_spans(const span_plan_t* plan, std::vector<int64_t>* row0, std::vector<int32_t>* n);

}  // namespace spanq
