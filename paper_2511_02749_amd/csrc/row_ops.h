// Launchers of the row operators (qk_norm.hip, adapters.hip, verify.hip).  Arguments are
// the public records, already checked (row_ops.cpp).
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/spanq.h"

namespace spanq {

hipError_t launch_qk_norm_rope(const span_qk_norm& a, hipStream_t s);

// What a call needs; _up_to: what it and every call of fewer rows or requests need.
size_t adapter_workspace_bytes(const span_adapter_call& a);
size_t adapter_workspace_up_to(const span_adapter_call& a);
// Why sizes of a call are refused, or null.
const char* check_adapter_sizes(const span_adapter_call& a);
hipError_t launch_adapter_apply(const span_adapter_call& a, hipStream_t s);

size_t verify_workspace_bytes(int64_t n_requests, int max_drafts, int vocab);
size_t verify_workspace_up_to(int64_t n_requests, int max_drafts, int vocab);
hipError_t launch_verify_drafts(const span_verify_call& a, hipStream_t s);

}  // namespace spanq
