// C-ABI of the row operators: every argument checked on the host before a launch.
#include <hip/hip_runtime.h>

#include <cmath>
#include <limits>
#include <string>

#include "capi_internal.h"
#include "hip_blocks.h"
#include "row_ops.h"

using namespace spanq;

// the binding packs these records byte by byte
static_assert(sizeof(span_qk_norm) == 176 && sizeof(span_adapter_call) == 152 && sizeof(span_verify_call) == 160,
              "public argument records");

namespace {

int bad(const char* who, const char* what) {
  return report(SPAN_EINVAL, (std::string(who) + ": " + what).c_str());
}

int done(const char* who, hipError_t e) {
  if (e == hipSuccess) return SPAN_OK;
  return report(SPAN_EHIP, (std::string(who) + ": " + hipGetErrorString(e)).c_str());
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

constexpr int64_t kMaxRows = std::numeric_limits<int32_t>::max();
constexpr int64_t kMaxWide = int64_t{1} << 20;  // features, columns and requests
constexpr int64_t kMaxStride = int64_t{1} << 23;  // of base and out: a work-group's rows in 32 bits

// One of q, k, v: its input, output, strides and gain.
const char* check_part(const void* in, const void* out, const void* gain, int64_t in_stride, int64_t out_stride,
                       int64_t width, int64_t vec, bool rows) {
  if (!in != !out) return "an input without its output, or an output without its input";
  if (!in) return nullptr;
  if (!aligned(in, 16) || !aligned(out, 16) || !aligned(gain, 16)) return "rows and gains must be 16-byte aligned";
  if (in_stride < width || out_stride < width || in_stride % vec != 0 || out_stride % vec != 0)
    return "strides must be multiples of 16 bytes and hold a row";
  if (in == out && (rows || in_stride != out_stride)) return "in place needs the same stride and no row list";
  return nullptr;
}

const char* check_verify_sizes(const span_verify_call& a) {
  if (a.n_requests < 0 || a.n_requests > kMaxWide) return "n_requests must lie in [0, 2^20]";
  if (a.max_drafts < 0 || a.max_drafts > SPAN_MAX_DRAFTS) return "max_drafts must lie in [0, SPAN_MAX_DRAFTS]";
  if (a.vocab < 1 || a.vocab > (1 << 24)) return "vocab must lie in [1, 2^24]";
  return nullptr;
}

}  // namespace

const char* spanq::check_adapter_sizes(const span_adapter_call& a) {
  if (a.n_rows < 0 || a.n_rows > kMaxRows) return "n_rows must lie in [0, 2^31)";
  if (a.in_features < 8 || a.in_features % 8 != 0 || a.in_features > kMaxWide)
    return "in_features must be a multiple of 8 in [8, 2^20]";
  if (a.max_rank < 8 || a.max_rank % 8 != 0 || a.max_rank > 128) return "max_rank must be a multiple of 8 in [8, 128]";
  if (a.n_parts < 1 || a.n_parts > 4) return "n_parts must lie in [1, 4]";
  int64_t n = 0;
  for (int p = 0; p < a.n_parts; ++p) {
    if (a.part_cols[p] < 8 || a.part_cols[p] % 8 != 0) return "part_cols must be positive multiples of 8";
    n += a.part_cols[p];
  }
  if (n > kMaxWide) return "the parts' columns must be at most 2^20 together";
  return nullptr;
}

extern "C" {

int span_qk_norm_rope(const span_qk_norm* args, void* stream) {
  const char* who = "span_qk_norm_rope";
  if (!args) return bad(who, "null argument");
  const span_qk_norm& a = *args;
  if (a.head_dim != 64 && a.head_dim != 128) return bad(who, "head_dim must be 64 or 128");
  if (a.dtype != SPAN_F32 && a.dtype != SPAN_BF16) return bad(who, "dtype must be SPAN_F32 or SPAN_BF16");
  if (a.n_rows < 0 || a.n_rows > kMaxRows || a.out_rows < 0 || a.out_rows > kMaxRows || (!a.rows && a.out_rows < a.n_rows))
    return bad(who, "n_rows and out_rows must lie in [0, 2^31), out_rows hold n_rows without a row list");
  if (a.num_q_heads < 0 || a.num_kv_heads < 0 || (a.q && a.num_q_heads < 1) || ((a.k || a.v) && a.num_kv_heads < 1) ||
      a.num_q_heads > 65536 || a.num_kv_heads > 65536)
    return bad(who, "bad head count");
  if (!(a.eps >= 0.f) || !std::isfinite(a.eps)) return bad(who, "eps must be finite and not negative");
  if (a.positions && (!(a.rope_theta > 0.f) || !std::isfinite(a.rope_theta))) return bad(who, "rope_theta must be positive");
  if (a.device < 0) return bad(who, "bad device");
  if (a.reserved != 0) return bad(who, "reserved must be 0");
  const int64_t vec = a.dtype == SPAN_BF16 ? 8 : 4;
  const int64_t wq = static_cast<int64_t>(a.num_q_heads) * a.head_dim, wk = static_cast<int64_t>(a.num_kv_heads) * a.head_dim;
  const char* what = check_part(a.q, a.q_out, a.q_gain, a.q_stride, a.q_out_stride, wq, vec, a.rows != nullptr);
  if (!what) what = check_part(a.k, a.k_out, a.k_gain, a.k_stride, a.k_out_stride, wk, vec, a.rows != nullptr);
  if (!what) what = check_part(a.v, a.v_out, nullptr, a.v_stride, a.v_out_stride, wk, vec, a.rows != nullptr);
  if (what) return bad(who, what);
  if (a.n_rows == 0 || (!a.q && !a.k && !a.v)) return SPAN_OK;
  const DeviceScope device(a.device);
  if (device.error() != hipSuccess) return done(who, device.error());  // (nothing runs on another one)
  return done(who, launch_qk_norm_rope(a, static_cast<hipStream_t>(stream)));
}

int span_adapter_workspace(const span_adapter_call* args, size_t* bytes) {
  const char* who = "span_adapter_workspace";
  if (!args || !bytes) return bad(who, "null argument");
  if (const char* what = check_adapter_sizes(*args)) return bad(who, what);
  *bytes = adapter_workspace_up_to(*args);
  return SPAN_OK;
}

int span_adapter_apply(const span_adapter_call* args, void* stream) {
  const char* who = "span_adapter_apply";
  if (!args) return bad(who, "null argument");
  const span_adapter_call& a = *args;
  if (const char* what = check_adapter_sizes(a)) return bad(who, what);
  if (a.n_adapters < 0) return bad(who, "n_adapters must not be negative");
  if (a.device < 0) return bad(who, "bad device");
  if (a.reserved != 0) return bad(who, "reserved must be 0");
  if (a.n_rows == 0) return SPAN_OK;
  int64_t n = 0;
  for (int p = 0; p < a.n_parts; ++p) n += a.part_cols[p];
  if (!a.x || !a.base || !a.out || !a.ids || (a.n_adapters > 0 && (!a.a || !a.b))) return bad(who, "null argument");
  if (!aligned(a.x, 16) || !aligned(a.base, 16) || !aligned(a.out, 16) || !aligned(a.a, 16) || !aligned(a.b, 16) ||
      !aligned(a.workspace, 16))
    return bad(who, "rows, weights and workspace must be 16-byte aligned");
  if (a.x_stride < a.in_features || a.base_stride < n || a.out_stride < n || a.x_stride % 8 != 0 ||
      a.base_stride % 8 != 0 || a.out_stride % 8 != 0 || a.base_stride > kMaxStride || a.out_stride > kMaxStride)
    return bad(who, "strides must be multiples of 8 and hold a row, base's and out's at most 2^23");
  if (a.base == a.out && a.base_stride != a.out_stride) return bad(who, "in place needs the same stride");
  if (a.workspace_bytes < adapter_workspace_bytes(a) || !a.workspace)
    return bad(who, "the workspace is smaller than span_adapter_workspace says");
  const DeviceScope device(a.device);
  if (device.error() != hipSuccess) return done(who, device.error());  // (nothing runs on another one)
  return done(who, launch_adapter_apply(a, static_cast<hipStream_t>(stream)));
}

int span_verify_workspace(const span_verify_call* args, size_t* bytes) {
  const char* who = "span_verify_workspace";
  if (!args || !bytes) return bad(who, "null argument");
  if (const char* what = check_verify_sizes(*args)) return bad(who, what);
  *bytes = verify_workspace_up_to(args->n_requests, args->max_drafts, args->vocab);
  return SPAN_OK;
}

int span_verify_drafts(const span_verify_call* args, void* stream) {
  const char* who = "span_verify_drafts";
  if (!args) return bad(who, "null argument");
  const span_verify_call& a = *args;
  if (const char* what = check_verify_sizes(a)) return bad(who, what);
  if (a.device < 0) return bad(who, "bad device");
  if (a.n_requests == 0) return SPAN_OK;
  if (!a.target_logits || !a.u_sample || !a.accepted || !a.tokens || (a.max_drafts > 0 && (!a.drafts || !a.u_accept)))
    return bad(who, "null argument");
  if (a.target_rows < 0 || a.target_stride < a.vocab || (a.draft_logits && (a.draft_rows < 0 || a.draft_stride < a.vocab)))
    return bad(who, "rows must not be negative, strides hold a row");
  if (!aligned(a.target_logits, 4) || !aligned(a.draft_logits, 4) || !aligned(a.workspace, 16))
    return bad(who, "logits must be 4-byte aligned, the workspace 16-byte");
  if (!a.workspace || a.workspace_bytes < verify_workspace_bytes(a.n_requests, a.max_drafts, a.vocab))
    return bad(who, "the workspace is smaller than span_verify_workspace says");
  const DeviceScope device(a.device);
  if (device.error() != hipSuccess) return done(who, device.error());  // (nothing runs on another one)
  return done(who, launch_verify_drafts(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
