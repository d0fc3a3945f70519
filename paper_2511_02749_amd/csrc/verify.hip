// Verification of drafted tokens against the target's probabilities, from given random
// numbers; without drafts, a token sampled for each request.
//
//   p_j = softmax(x_j / T),  q_j = softmax(y_j / T) or 1 at the drafted token
//   draft j is kept if u_j q_j(d_j) < p_j(d_j), and every draft before it was
//   next token: the first i with  sum_{i' <= i} w_i' > u sum w,  w = max(p_a - q_a, 0) at the
//   first refused draft a (p_a where that is nothing), w = p_k after the last draft
//   T <= 0: a draft is kept if it is the argmax of x_j, the next token is the argmax of x_a
//
// Three launches (two where no draft has a distribution):
// 1. every row in chunks of kChunk logits, one work-group each: the chunk's largest logit, its
//    lowest id, and the sum of exp against it;
// 2. (draft logits) the chunks of the one row that decides a request: sums of max(p - q, 0);
// 3. one work-group per request: the chunk where the running sum passes u, then the token in
//    it, and the outputs.
// 2 and 3 form acceptance from the chunks' sums again, each work-group for itself (a few
// hundred numbers), rather than wait for another launch.
//
// Weights and sums are 64-bit: borders of the running sum over 10^5 tokens lie 10^-5 and
// less apart, where 32-bit sums, and their order, would choose another token every few
// thousand calls.  64-bit instructions run at the 32-bit rate here; the exponential is its
// Taylor series on [-ln 2 / 2, ln 2 / 2] to the 11th power (6e-15 relative).
//
// Bound: HBM, each logit read once (and the deciding row again, from the last-level cache),
// about 20 vector instructions per logit beside it.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "grid.h"
#include "row_ops.h"

namespace spanq {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;
constexpr int kPer = kChunk / kThreads;
constexpr int kPickThreads = 1024;
constexpr int kMaxDrafts = SPAN_MAX_DRAFTS;

struct Stat {
  double sum;  // of exp((x - max) / T) over the chunk
  float max;   // -inf: nothing in the chunk has weight
  int32_t arg;
};

struct Args {
  span_verify_call c;
  int chunks;
  int q0;          // first request of the launch
  Stat* target;    // [requests][drafts + 1][chunks]
  Stat* draft;     // [requests][drafts][chunks]
  double* left;    // [requests][chunks]: sums of max(p - q, 0)
};

// exp(t) for t <= 0; 0 below -700, and for a NaN.
__device__ __forceinline__ double exp_neg(double t) {
  if (!(t > -700.0)) return 0.0;
  const double k = rint(t * 1.4426950408889634074);  // t = k ln 2 + f
  const double f = fma(k, -0.69314718055994530942, t);
  double p = 1.0 / 39916800.0;
  p = fma(p, f, 1.0 / 3628800.0);
  p = fma(p, f, 1.0 / 362880.0);
  p = fma(p, f, 1.0 / 40320.0);
  p = fma(p, f, 1.0 / 5040.0);
  p = fma(p, f, 1.0 / 720.0);
  p = fma(p, f, 1.0 / 120.0);
  p = fma(p, f, 1.0 / 24.0);
  p = fma(p, f, 1.0 / 6.0);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.0);
  p = fma(p, f, 1.0);
  return ldexp(p, static_cast<int>(k));
}

// The weight of logit x against the largest one: 1 at it (an infinite one too), else
// exp((x - max) / T); 0 for -inf and NaN.
__device__ __forceinline__ double weight(float x, float max, double inv_t) {
  if (!(max > -INFINITY)) return 0.0;
  if (x == max) return 1.0;
  return exp_neg((static_cast<double>(x) - static_cast<double>(max)) * inv_t);
}

__device__ __forceinline__ void better(float& bv, int& bi, float v, int i) {
  if (v > bv || (v == bv && i < bi)) {
    bv = v;
    bi = i;
  }
}

__device__ __forceinline__ double shfl_xor_f64(double v, int off) { return __shfl_xor(v, off); }

struct Request {
  bool valid;    // its rows lie inside the logits
  int n_drafts;
  bool greedy;
  double inv_t;
  int64_t target_row, draft_row;
};

__device__ __forceinline__ Request request_of(const span_verify_call& c, int q) {
  Request r;
  const int k = c.max_drafts;
  r.n_drafts = c.n_drafts ? max(0, min(c.n_drafts[q], k)) : k;
  const float t = c.temperature ? c.temperature[q] : 1.f;
  r.greedy = !(t > 0.f);
  r.inv_t = r.greedy ? 1.0 : 1.0 / static_cast<double>(t);
  r.target_row = c.target_row0 ? c.target_row0[q] : static_cast<int64_t>(q) * (k + 1);
  r.draft_row = c.draft_row0 ? c.draft_row0[q] : static_cast<int64_t>(q) * k;
  r.valid = r.target_row >= 0 && r.target_row + r.n_drafts < c.target_rows &&
            (!c.draft_logits || r.n_drafts == 0 || (r.draft_row >= 0 && r.draft_row + r.n_drafts <= c.draft_rows));
  return r;
}

// ------------------------------------------------------------------ 1: chunks of every row
template <bool kVec>
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(const Args a) {
  __shared__ float s_max[kThreads / 64];
  __shared__ int s_arg[kThreads / 64];
  __shared__ double s_sum[kThreads / 64];
  const span_verify_call& c = a.c;
  const int q = a.q0 + static_cast<int>(blockIdx.z);
  const int k = c.max_drafts;
  const bool draft = static_cast<int>(blockIdx.y) > k;
  const int j = draft ? static_cast<int>(blockIdx.y) - k - 1 : static_cast<int>(blockIdx.y);
  const Request r = request_of(c, q);
  if (!r.valid || (draft ? j >= r.n_drafts || r.greedy : j > r.n_drafts)) return;
  const float* row = draft ? c.draft_logits + (r.draft_row + j) * c.draft_stride
                           : c.target_logits + (r.target_row + j) * c.target_stride;
  const int base = blockIdx.x * kChunk;
  float x[kPer];
  if constexpr (kVec) {
#pragma unroll
    for (int u = 0; u < kPer / 4; ++u) {
      const int i = base + 4 * (u * kThreads + static_cast<int>(threadIdx.x));
      if (i + 3 < c.vocab) {
        const float4 v = *reinterpret_cast<const float4*>(row + i);
        x[4 * u] = v.x;
        x[4 * u + 1] = v.y;
        x[4 * u + 2] = v.z;
        x[4 * u + 3] = v.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * u + e] = i + e < c.vocab ? row[i + e] : -INFINITY;
      }
    }
  } else {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = base + u * kThreads + static_cast<int>(threadIdx.x);
      x[u] = i < c.vocab ? row[i] : -INFINITY;
    }
  }
  float best = -INFINITY;
  int arg = INT32_MAX;
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int i = kVec ? base + 4 * ((u / 4) * kThreads + static_cast<int>(threadIdx.x)) + u % 4
                       : base + u * kThreads + static_cast<int>(threadIdx.x);
    if (x[u] > best) {  // ids rise: an equal later one keeps the lower id
      best = x[u];
      arg = i;
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) better(best, arg, __shfl_xor(best, off), __shfl_xor(arg, off));
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    s_max[wave] = best;
    s_arg[wave] = arg;
  }
  __syncthreads();
  best = s_max[0];
  arg = s_arg[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) better(best, arg, s_max[w], s_arg[w]);
  double sum = 0.0;
#pragma unroll
  for (int u = 0; u < kPer; ++u) sum += weight(x[u], best, r.inv_t);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += shfl_xor_f64(sum, off);
  if ((threadIdx.x & 63) == 0) s_sum[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) sum += s_sum[w];
    Stat* to = draft ? a.draft + (static_cast<int64_t>(q) * k + j) * a.chunks
                     : a.target + (static_cast<int64_t>(q) * (k + 1) + j) * a.chunks;
    to[blockIdx.x] = Stat{sum, best, arg};
  }
}

// A row's largest logit, its lowest id and its sum of weights, by one wave.
__device__ __forceinline__ Stat whole_row(const Stat* st, int chunks, double inv_t, int lane) {
  float best = -INFINITY;
  int arg = INT32_MAX;
  for (int i = lane; i < chunks; i += 64) better(best, arg, st[i].max, st[i].arg);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) better(best, arg, __shfl_xor(best, off), __shfl_xor(arg, off));
  double sum = 0.0;
  for (int i = lane; i < chunks; i += 64) sum += st[i].sum * weight(st[i].max, best, inv_t);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += shfl_xor_f64(sum, off);
  return Stat{sum, best, arg};
}

// What the work-groups of 2 and 3 need of a request's rows.
struct Verdict {
  Stat p[kMaxDrafts + 1], q[kMaxDrafts];
  int keep[kMaxDrafts];
};

// Acceptance of a request's drafts, by all waves of the work-group; returns the number
// kept.  p and q of `v` hold the rows' sums afterwards.
__device__ int accept(const Args& a, int q, const Request& r, Verdict& v, int waves) {
  const span_verify_call& c = a.c;
  const int k = c.max_drafts;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool dist = c.draft_logits && !r.greedy;
  for (int e = wave; e < r.n_drafts + 1 + (dist ? r.n_drafts : 0); e += waves) {
    if (e <= r.n_drafts) {
      const Stat s = whole_row(a.target + (static_cast<int64_t>(q) * (k + 1) + e) * a.chunks, a.chunks, r.inv_t, lane);
      if (lane == 0) v.p[e] = s;
    } else {
      const int j = e - r.n_drafts - 1;
      const Stat s = whole_row(a.draft + (static_cast<int64_t>(q) * k + j) * a.chunks, a.chunks, r.inv_t, lane);
      if (lane == 0) v.q[j] = s;
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j < r.n_drafts; j += blockDim.x) {
    const int d = c.drafts[static_cast<int64_t>(q) * k + j];
    bool keep = false;
    if (r.greedy) {
      keep = v.p[j].sum > 0.0 && d == v.p[j].arg;
    } else if (d >= 0 && d < c.vocab) {
      const float x = c.target_logits[(r.target_row + j) * c.target_stride + d];
      const double pd = v.p[j].sum > 0.0 ? weight(x, v.p[j].max, r.inv_t) / v.p[j].sum : 0.0;
      double qd = 1.0;
      if (dist) {
        const float y = c.draft_logits[(r.draft_row + j) * c.draft_stride + d];
        qd = v.q[j].sum > 0.0 ? weight(y, v.q[j].max, r.inv_t) / v.q[j].sum : 0.0;
      }
      keep = static_cast<double>(c.u_accept[static_cast<int64_t>(q) * k + j]) * qd < pd;
    }
    v.keep[j] = keep;
  }
  __syncthreads();
  int n = 0;
  while (n < r.n_drafts && v.keep[n]) ++n;
  return n;
}

// What the row that decides a request leaves of token i: max(p - q, 0), or p.
struct Left {
  const float* x;
  const float* y;  // the draft's logits, or null
  float pm, qm;
  double ps, qs, inv_t;  // 1 / sums
  int one_hot;           // the token taken out of p where the draft has no distribution, -1: none
  __device__ __forceinline__ double operator()(int i) const {
    double w = weight(x[i], pm, inv_t) * ps;
    if (y) w = fmax(w - weight(y[i], qm, inv_t) * qs, 0.0);
    return i == one_hot ? 0.0 : w;
  }
};

__device__ __forceinline__ double inverse(double s) { return s > 0.0 ? 1.0 / s : 0.0; }

__device__ __forceinline__ Left left_of(const Args& a, int q, const Request& r, const Verdict& v, int n, bool plain) {
  const span_verify_call& c = a.c;
  Left l{};
  l.x = c.target_logits + (r.target_row + n) * c.target_stride;
  l.pm = v.p[n].max;
  l.ps = inverse(v.p[n].sum);
  l.inv_t = r.inv_t;
  l.one_hot = -1;
  if (n < r.n_drafts && !plain) {
    if (c.draft_logits) {
      l.y = c.draft_logits + (r.draft_row + n) * c.draft_stride;
      l.qm = v.q[n].max;
      l.qs = inverse(v.q[n].sum);
    } else {
      const int d = c.drafts[static_cast<int64_t>(q) * c.max_drafts + n];
      l.one_hot = d >= 0 && d < c.vocab ? d : -1;
    }
  }
  return l;
}

// ------------------------------------------------------------------ 2: what the deciding row leaves
__global__ __launch_bounds__(kThreads) void verify_left_kernel(const Args a) {
  __shared__ Verdict v;
  __shared__ double s_sum[kThreads / 64];
  const span_verify_call& c = a.c;
  const int q = a.q0 + static_cast<int>(blockIdx.y);
  const Request r = request_of(c, q);
  if (!r.valid || r.greedy || r.n_drafts == 0) return;
  const int n = accept(a, q, r, v, kThreads / 64);
  if (n == r.n_drafts) return;  // after the last draft the chunks' own sums serve
  const Left l = left_of(a, q, r, v, n, false);
  double sum = 0.0;
  for (int u = 0; u < kPer; ++u) {
    const int i = blockIdx.x * kChunk + u * kThreads + static_cast<int>(threadIdx.x);
    if (i < c.vocab) sum += l(i);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += shfl_xor_f64(sum, off);
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) sum += s_sum[w];
    a.left[static_cast<int64_t>(q) * a.chunks + blockIdx.x] = sum;
  }
}

// Sum of v over the threads before this one, and over all of them.
__device__ __forceinline__ double scan_before(double v, double* total, double* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double inc = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double o = __shfl_up(inc, off);
    if (lane >= off) inc += o;
  }
  if (lane == 63) s_wave[wave] = inc;
  __syncthreads();
  double before = 0.0, all = 0.0;
  for (int w = 0; w < kPickThreads / 64; ++w) {
    if (w == wave) before = all;
    all += s_wave[w];
  }
  __syncthreads();
  *total = all;
  const double up = __shfl_up(inc, 1);
  return before + (lane > 0 ? up : 0.0);
}

// ------------------------------------------------------------------ 3: the token
__global__ __launch_bounds__(kPickThreads) void verify_pick_kernel(const Args a) {
  __shared__ Verdict v;
  __shared__ double s_wave[kPickThreads / 64];
  __shared__ int s_first, s_last;
  __shared__ double s_before;
  const span_verify_call& c = a.c;
  const int q = a.q0 + static_cast<int>(blockIdx.x);
  const int k = c.max_drafts;
  const Request r = request_of(c, q);
  int32_t* tokens = c.tokens + static_cast<int64_t>(q) * (k + 1);
  float* lps = c.logprobs ? c.logprobs + static_cast<int64_t>(q) * (k + 1) : nullptr;
  if (!r.valid) {
    for (int j = threadIdx.x; j <= k; j += kPickThreads) {
      tokens[j] = -1;
      if (lps) lps[j] = 0.f;
    }
    if (threadIdx.x == 0) c.accepted[q] = -1;
    return;
  }
  const int n = accept(a, q, r, v, kPickThreads / 64);
  int token = -1;
  if (r.greedy) {
    token = v.p[n].sum > 0.0 ? v.p[n].arg : -1;
  } else if (v.p[n].sum > 0.0) {
    const double u = static_cast<double>(c.u_sample[q]);
    const Stat* st = a.target + (static_cast<int64_t>(q) * (k + 1) + n) * a.chunks;
    bool plain = n == r.n_drafts;
    // chunk sums in order: the first chunk whose running sum passes u times the whole
    for (;;) {
      const Left l = left_of(a, q, r, v, n, plain);
      const double* left = !plain && l.y ? a.left + static_cast<int64_t>(q) * a.chunks : nullptr;
      double total = 0.0, run = 0.0;
      auto chunk_sum = [&](int i) -> double {
        if (left) return left[i];
        double s = st[i].sum * weight(st[i].max, l.pm, r.inv_t) * l.ps;
        if (l.one_hot >= 0 && l.one_hot / kChunk == i) {
          s -= weight(l.x[l.one_hot], l.pm, r.inv_t) * l.ps;
          s = s > 0.0 ? s : 0.0;
        }
        return s;
      };
      // the whole, then the chunk: kPickThreads chunks at a time
      for (int b = 0; b < a.chunks; b += kPickThreads) {
        const int i = b + static_cast<int>(threadIdx.x);
        double all;
        (void)scan_before(i < a.chunks ? chunk_sum(i) : 0.0, &all, s_wave);
        total += all;
      }
      if (!(total > 0.0) && !plain) {  // nothing left of p: p itself
        plain = true;
        continue;
      }
      const double target = u * total;
      if (threadIdx.x == 0) {
        s_first = INT32_MAX;
        s_last = -1;
      }
      __syncthreads();
      for (int b = 0; b < a.chunks; b += kPickThreads) {
        const int i = b + static_cast<int>(threadIdx.x);
        const double w = i < a.chunks ? chunk_sum(i) : 0.0;
        double all;
        const double before = run + scan_before(w, &all, s_wave);
        if (w > 0.0) {
          if (before + w > target) atomicMin(&s_first, i);
          atomicMax(&s_last, i);
        }
        run += all;
      }
      __syncthreads();
      const int chunk = s_first != INT32_MAX ? s_first : s_last;
      __syncthreads();
      run = 0.0;
      for (int b = 0; b < a.chunks; b += kPickThreads) {
        const int i = b + static_cast<int>(threadIdx.x);
        double all;
        const double before = run + scan_before(i < a.chunks ? chunk_sum(i) : 0.0, &all, s_wave);
        if (i == chunk) s_before = before;
        run += all;
      }
      if (threadIdx.x == 0) {
        s_first = INT32_MAX;
        s_last = -1;
      }
      __syncthreads();
      // the token in the chunk: each thread four tokens that follow one another
      constexpr int kEach = kChunk / kPickThreads;
      const int i0 = chunk * kChunk + static_cast<int>(threadIdx.x) * kEach;
      double w[kEach], mine = 0.0;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        w[e] = i0 + e < c.vocab ? l(i0 + e) : 0.0;
        mine += w[e];
      }
      double all;
      double at = s_before + scan_before(mine, &all, s_wave);
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        at += w[e];
        if (w[e] > 0.0) {
          if (at > target) atomicMin(&s_first, i0 + e);
          atomicMax(&s_last, i0 + e);
        }
      }
      __syncthreads();
      token = s_first != INT32_MAX ? s_first : s_last;
      break;
    }
  }
  for (int j = threadIdx.x; j <= k; j += kPickThreads) {
    int t = -1;
    if (j < n) t = c.drafts[static_cast<int64_t>(q) * k + j];
    if (j == n) t = token;
    tokens[j] = t;
    if (lps) {
      float lp = 0.f;
      if (t >= 0) {
        const float x = c.target_logits[(r.target_row + j) * c.target_stride + t];
        // a weight that is 1 (the largest logit) has no difference to scale
        const double d = x == v.p[j].max ? 0.0 : (static_cast<double>(x) - static_cast<double>(v.p[j].max)) * r.inv_t;
        lp = static_cast<float>(d - log(v.p[j].sum));
      }
      lps[j] = lp;
    }
  }
  if (threadIdx.x == 0) c.accepted[q] = n;
}

int chunks_of(int vocab) { return (vocab + kChunk - 1) / kChunk; }

}  // namespace

size_t verify_workspace_bytes(int64_t n, int max_drafts, int vocab) {
  const size_t ch = static_cast<size_t>(chunks_of(vocab)), nz = static_cast<size_t>(n), k = max_drafts;
  return nz * ch * ((2 * k + 1) * sizeof(Stat) + sizeof(double));
}

hipError_t launch_verify_drafts(const span_verify_call& c, hipStream_t s) {
  Args a{};
  a.c = c;
  a.chunks = chunks_of(c.vocab);
  const size_t n = static_cast<size_t>(c.n_requests), ch = static_cast<size_t>(a.chunks), k = c.max_drafts;
  a.target = static_cast<Stat*>(c.workspace);
  a.draft = a.target + n * (k + 1) * ch;
  a.left = reinterpret_cast<double*>(a.draft + n * k * ch);
  const bool vec = reinterpret_cast<uintptr_t>(c.target_logits) % 16 == 0 && c.target_stride % 4 == 0 &&
                   (!c.draft_logits || (reinterpret_cast<uintptr_t>(c.draft_logits) % 16 == 0 && c.draft_stride % 4 == 0));
  const unsigned rows = static_cast<unsigned>(c.max_drafts + 1 + (c.draft_logits ? c.max_drafts : 0));
  // requests on the grid's last dimension: as many at once as it takes
  const int64_t threads = std::max<int64_t>(static_cast<int64_t>(a.chunks) * rows * kThreads, int64_t{1} << 17);
  return launch_in_slices(c.n_requests, threads, hipErrorInvalidValue, [&](int64_t first, int64_t count) -> hipError_t {
    a.q0 = static_cast<int>(first);
    const unsigned nq = static_cast<unsigned>(count);
    if (vec) {
      verify_stats_kernel<true><<<dim3(a.chunks, rows, nq), kThreads, 0, s>>>(a);
    } else {
      verify_stats_kernel<false><<<dim3(a.chunks, rows, nq), kThreads, 0, s>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && c.draft_logits && c.max_drafts > 0) {
      verify_left_kernel<<<dim3(a.chunks, nq), kThreads, 0, s>>>(a);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    verify_pick_kernel<<<nq, kPickThreads, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace spanq
