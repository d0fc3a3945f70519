// Norms of queries and keys for each head, with the rotation in the same pass.
//
//   y = x / sqrt(mean_d(x^2) + eps) * gain          over the head_dim values of one head
//   (y_i, y_{i + d/2}) -> (y_i cos - y_{i+d/2} sin, y_{i+d/2} cos + y_i sin)
//   at angle  position * theta^(-2i/d)
//
// and the rows' way from one product's q|k|v rows to the caller's rows; values are copied.
// Bound: HBM, each element read once and written once, ~10 operations each.  8192 rows of 32 + 2 x 8
// heads of 128 with their rotation take 39 us, 5.2 TB/s, as fast as a copy; one row 3 us.
//
// A lane holds 16 bytes of the head's first half and the 16 bytes d/2 further on, so both
// members of a pair are in one lane, the sum of squares takes log2(lanes per head) lane
// exchanges, and every access is a 16-byte vector.  A work-group takes one row: it puts its
// cos and sin into LDS once (all heads share them), then walks the heads.  Angles are formed in 64
// bits, in turns, their cos and sin too: at position 120000 a 32-bit product would be off by 0.004
// radians, and an angle rounded to 32 bits moves a small cos or sin by many of its last bits.  Sums,
// norm and rotation are 32-bit; the only rounding to 16 bits is the result's.
#include <hip/hip_runtime.h>

#include <cmath>

#include "dev_common.h"
#include "grid.h"
#include "page_write.h"
#include "row_ops.h"

namespace spanq {
namespace {

constexpr int kThreads = 256;

struct QkArgs {
  span_qk_norm a;
  double log2_theta;
  int64_t row0;  // first row of the launch
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void qk_norm_kernel(const QkArgs g) {
  constexpr int E = Chunk16<T>::E;
  constexpr int H = D / 2;
  constexpr int L = H / E;  // lanes per head
  constexpr int G = kThreads / L;
  __shared__ float2 turn[H];
  const span_qk_norm& a = g.a;
  const int64_t row = g.row0 + blockIdx.x;
  const int64_t to = a.rows ? a.rows[row] : row;
  if (to < 0 || to >= a.out_rows) return;
  if (a.positions) {
    if (const int i = threadIdx.x; i < H) {
      const double inv = exp2(-2.0 * i / D * g.log2_theta) * 0.15915494309189533577;  // turns per position
      double t = static_cast<double>(a.positions[row]) * inv;
      t -= rint(t);
      double sn, cs;
      sincospi(2.0 * t, &sn, &cs);
      turn[i] = float2{static_cast<float>(cs), static_cast<float>(sn)};
    }
    __syncthreads();
  }
  const int nq = a.q ? a.num_q_heads : 0, nk = a.k ? a.num_kv_heads : 0, nv = a.v ? a.num_kv_heads : 0;
  const int heads = nq + nk + nv;
  const int c = threadIdx.x % L;
  for (int e = threadIdx.x / L; e < heads; e += G) {
    int h = e;
    const T* src;
    T* dst;
    const T* gain = nullptr;
    bool rotate = false;
    if (h < nq) {
      src = static_cast<const T*>(a.q) + row * a.q_stride;
      dst = static_cast<T*>(a.q_out) + to * a.q_out_stride;
      gain = static_cast<const T*>(a.q_gain);
      rotate = a.positions != nullptr;
    } else if (h < nq + nk) {
      h -= nq;
      src = static_cast<const T*>(a.k) + row * a.k_stride;
      dst = static_cast<T*>(a.k_out) + to * a.k_out_stride;
      gain = static_cast<const T*>(a.k_gain);
      rotate = a.positions != nullptr;
    } else {
      h -= nq + nk;
      src = static_cast<const T*>(a.v) + row * a.v_stride;
      dst = static_cast<T*>(a.v_out) + to * a.v_out_stride;
    }
    src += h * D + c * E;
    dst += h * D + c * E;
    Chunk16<T> x0 = load16(src), x1 = load16(src + H);
    if (gain || rotate) {
      float y0[E], y1[E];
#pragma unroll
      for (int u = 0; u < E; ++u) {
        y0[u] = to_f32(x0.x[u]);
        y1[u] = to_f32(x1.x[u]);
      }
      if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int u = 0; u < E; ++u) ss = fmaf(y0[u], y0[u], fmaf(y1[u], y1[u], ss));
#pragma unroll
        for (int off = L / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        const float scale = 1.0f / sqrtf(ss / static_cast<float>(D) + a.eps);
        const Chunk16<T> g0 = load16(gain + c * E), g1 = load16(gain + H + c * E);
#pragma unroll
        for (int u = 0; u < E; ++u) {
          y0[u] = y0[u] * scale * to_f32(g0.x[u]);
          y1[u] = y1[u] * scale * to_f32(g1.x[u]);
        }
      }
      if (rotate) {
#pragma unroll
        for (int u = 0; u < E; ++u) {
          const float2 t = turn[c * E + u];
          const float lo = y0[u] * t.x - y1[u] * t.y;
          y1[u] = y1[u] * t.x + y0[u] * t.y;
          y0[u] = lo;
        }
      }
#pragma unroll
      for (int u = 0; u < E; ++u) {
        x0.x[u] = from_f32<T>(y0[u]);
        x1.x[u] = from_f32<T>(y1[u]);
      }
    }
    store16(dst, x0);
    store16(dst + H, x1);
  }
}

template <typename T, int D>
hipError_t launch_d(const span_qk_norm& a, hipStream_t s) {
  QkArgs g{a, std::log2(static_cast<double>(a.rope_theta)), 0};
  return launch_in_slices(a.n_rows, kThreads, hipErrorInvalidValue, [&](int64_t first, int64_t count) {
    g.row0 = first;
    qk_norm_kernel<T, D><<<static_cast<unsigned>(count), kThreads, 0, s>>>(g);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_qk_norm_rope(const span_qk_norm& a, hipStream_t s) {
  if (a.dtype == SPAN_BF16) return a.head_dim == 128 ? launch_d<bf16_t, 128>(a, s) : launch_d<bf16_t, 64>(a, s);
  return a.head_dim == 128 ? launch_d<float, 128>(a, s) : launch_d<float, 64>(a, s);
}

}  // namespace spanq
