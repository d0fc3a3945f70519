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
// 1. every row in chunks of kChunk logits (chunk_of), one wave each: the chunk's largest logit, its
//    lowest id, and the sum of exp against it;
// 2. (draft logits) the chunks of the one row that decides a request: sums of max(p - q, 0);
// 3. one work-group per request: the chunk where the running sum passes u, then the token in
//    it, and the outputs.
// 2 and 3 form acceptance from the chunks' sums again, each work-group for itself (a few
// hundred numbers), rather than wait for another launch.
//
// Weights and sums are 64-bit: borders of the running sum over 10^5 tokens lie 10^-5 and
// less apart, where 32-bit sums, and their order, would choose another token every few
// thousand calls.  64-bit instructions run at the 32-bit rate here; an exponential
// takes 17 of them.
//
// Bound: HBM, each logit read once (and the deciding row again, from the last-level cache),
// 17 vector instructions per logit beside it.  64 requests of 4 drafts with a distribution,
// 128256 tokens (295 MB): 56 us in 1 (5.3 TB/s), 18 in 2, 10 in 3.  The instructions still count: with
// three more for each exponential 64 and 24.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "grid.h"
#include "row_ops.h"

namespace spanq {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// A wave for each row of up to three drafts and their distributions.  Of 1024 / 512 / 256: one request of
// four drafts 7.4 / 6.5 / 7.2 us, 64 with distributions 10.3 / 10.2 / 12.4, 256 without drafts 7.5 / 6.8 / 6.9.
constexpr int kPickThreads = 512;
constexpr int kMaxDrafts = SPAN_MAX_DRAFTS;
constexpr double kLog2e = 1.4426950408889634074;

struct Stat {
  double sum;  // of the weights, relative to the chunk's own largest logit (scale_of)
  float max;   // -inf: nothing in the chunk has weight
  int32_t arg;
};

struct Args {
  span_verify_call c;
  int chunks;
  int q0;          // first request of the launch
  Stat* target;    // [requests][drafts + 1][chunks]
  Stat* draft;     // [requests][drafts][chunks]; without distributions, of each draft its own chunk alone:
                   // what target row j holds there without drafted token j
  double* left;    // [requests][chunks]: sums of max(p - q, 0)
};

// What weights are relative to: w(x) = 2^(x c - k), c = log2(e) / T, k the whole number next to c
// times the largest logit, so that x c - k is rounded once.  Where that logit is infinite, or c times
// it past 2^40, all the weight lies on the logits equal to it (others, 2^-24 of it away, weigh
// nothing); where it is -inf, there is none.
struct Scale {
  double c, k;
  float only;  // `hot`: the logit with all the weight, NaN if none has any
  bool hot;
};
__device__ __forceinline__ Scale scale_of(float max, double c) {
  const double at = static_cast<double>(max) * c;
  return Scale{c, rint(at), max > -INFINITY ? max : NAN, !(fabs(at) < 0x1p40)};
}

// 2^t of t = x c - k, c and k finite; 0 below 2^-1200, which -inf and NaN are taken to.
__device__ __forceinline__ double weight_at(float x, const Scale& s) {
  const double t = fmax(fma(static_cast<double>(x), s.c, -s.k), -1200.0);
  const double n = rint(t), f = t - n;
  // 2^f on [-1/2, 1/2], least relative error of a polynomial (Remez exchange): 1.36e-14
  double p = 1.0150337260976417e-07;
  p = fma(p, f, 1.3259405611204192e-06);
  p = fma(p, f, 1.5252984835578367e-05);
  p = fma(p, f, 1.5403434948081424e-04);
  p = fma(p, f, 1.3333557617609879e-03);
  p = fma(p, f, 9.6181291920672020e-03);
  p = fma(p, f, 5.5504108668685580e-02);
  p = fma(p, f, 2.4022650695649653e-01);
  p = fma(p, f, 6.9314718055987100e-01);
  p = fma(p, f, 1.0000000000000127);
  return ldexp(p, static_cast<int>(n));
}
__device__ __forceinline__ double weight(float x, const Scale& s) {
  return s.hot ? (x == s.only ? 1.0 : 0.0) : weight_at(x, s);
}

// Values of other lanes by vector instructions alone: DPP rotations inside a row of 16, and
// swaps of rows and of halves.
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xf, true);
}
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = dpp<kCtrl, kRows>(static_cast<uint32_t>(u));
  const uint64_t hi = dpp<kCtrl, kRows>(static_cast<uint32_t>(u >> 32));
  return __builtin_bit_cast(double, lo | hi << 32);
}
// v of all 64 lanes joined by f, which commutes: the same bits in every lane.
template <class F>
__device__ __forceinline__ uint32_t join32(uint32_t v, F f) {
  v = f(v, dpp<0x128>(v));  // row_ror:8, 4, 2, 1
  v = f(v, dpp<0x124>(v));
  v = f(v, dpp<0x122>(v));
  v = f(v, dpp<0x121>(v));
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = f(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(b[0], b[1]);
}
__device__ __forceinline__ float wave_max(float v) {
  return __uint_as_float(join32(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
__device__ __forceinline__ int wave_min(int v) {
  return static_cast<int>(join32(static_cast<uint32_t>(v), [](uint32_t a, uint32_t b) {
    return static_cast<uint32_t>(min(static_cast<int>(a), static_cast<int>(b)));
  }));
}
__device__ __forceinline__ double wave_sum(double v) {
  v += dpp<0x128>(v);
  v += dpp<0x124>(v);
  v += dpp<0x122>(v);
  v += dpp<0x121>(v);
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  auto lo = __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(u), static_cast<uint32_t>(u), false, false);
  auto hi = __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(u >> 32), static_cast<uint32_t>(u >> 32), false, false);
  auto pair = [](uint32_t l, uint32_t h) { return __builtin_bit_cast(double, static_cast<uint64_t>(h) << 32 | l); };
  v = pair(lo[0], hi[0]) + pair(lo[1], hi[1]);
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  lo = __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(w), static_cast<uint32_t>(w), false, false);
  hi = __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(w >> 32), static_cast<uint32_t>(w >> 32), false, false);
  return pair(lo[0], hi[0]) + pair(lo[1], hi[1]);
}
// Sum of v over this lane and those before it.
__device__ __forceinline__ double wave_scan(double v) {
  v += dpp<0x111>(v);       // row_shr:1, 2, 4, 8
  v += dpp<0x112>(v);
  v += dpp<0x114>(v);
  v += dpp<0x118>(v);
  v += dpp<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3
  v += dpp<0x143, 0xc>(v);  // row_bcast:31 into rows 2 and 3
  return v;
}

struct Request {
  bool valid;    // its rows lie inside the logits
  int n_drafts;
  bool greedy;
  double c;      // log2(e) / T
  int64_t target_row, draft_row;
};

__device__ __forceinline__ Request request_of(const span_verify_call& c, int q) {
  Request r;
  const int k = c.max_drafts;
  r.n_drafts = c.n_drafts ? max(0, min(c.n_drafts[q], k)) : k;
  const float t = c.temperature ? c.temperature[q] : 1.f;
  r.greedy = !(t > 0.f);
  r.c = r.greedy ? kLog2e : kLog2e / static_cast<double>(t);
  r.target_row = c.target_row0 ? c.target_row0[q] : static_cast<int64_t>(q) * (k + 1);
  r.draft_row = c.draft_row0 ? c.draft_row0[q] : static_cast<int64_t>(q) * k;
  r.valid = r.target_row >= 0 && r.target_row + r.n_drafts < c.target_rows &&
            (!c.draft_logits || r.n_drafts == 0 || (r.draft_row >= 0 && r.draft_row + r.n_drafts <= c.draft_rows));
  return r;
}

// A lane's kPer logits of a chunk, four at a time (a vector of 16 bytes from any multiple of
// four: rows of an odd vocabulary start anywhere); -inf past the vocabulary.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ int id_of(int base, int lane, int u) { return base + 4 * (64 * (u / 4) + lane) + u % 4; }

template <int kPer>
__device__ __forceinline__ void load_chunk(const float* __restrict__ row, int base, int lane, int vocab,
                                           float (&x)[kPer]) {
  if (base + 64 * kPer <= vocab) {
#pragma unroll
    for (int u = 0; u < kPer; u += 4) {
      const f32x4_any v = *reinterpret_cast<const f32x4_any*>(row + id_of(base, lane, u));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u + e] = v[e];
    }
  } else {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = id_of(base, lane, u);
      x[u] = i < vocab ? row[i] : -INFINITY;
    }
  }
}

// What a chunk's sum is in the row's scale; nothing where its largest weight would not be a normal
// number there, so that a chunk with a sum has a token with a weight.
__device__ __forceinline__ double in_row(const Stat& chunk, const Scale& row) {
  if (row.hot) return chunk.max == row.only ? chunk.sum : 0.0;
  const double octaves = rint(static_cast<double>(chunk.max) * row.c) - row.k;
  const double sum = octaves >= -1021.0 ? chunk.sum : 0.0;
  return ldexp(sum, static_cast<int>(fmax(octaves, -1021.0)));
}

// Largest of a wave's logits, -inf if none is a number.
template <int kPer>
__device__ __forceinline__ float chunk_max(const float (&x)[kPer]) {
  float best = x[0];
#pragma unroll
  for (int u = 1; u < kPer; ++u) best = fmaxf(best, x[u]);
  best = wave_max(best);
  return best > -INFINITY ? best : -INFINITY;
}
// Sum of a wave's weights.
template <int kPer>
__device__ __forceinline__ double chunk_sum(const float (&x)[kPer], const Scale& s) {
  double sum = 0.0;
  if (s.hot) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) sum += x[u] == s.only ? 1.0 : 0.0;
  } else {
#pragma unroll
    for (int u = 0; u < kPer; ++u) sum += weight_at(x[u], s);
  }
  return wave_sum(sum);
}

// ------------------------------------------------------------------ 1: chunks of every row
template <int kChunk>
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(const Args a) {
  constexpr int kPer = kChunk / 64;
  const span_verify_call& c = a.c;
  const int q = a.q0 + static_cast<int>(blockIdx.z);
  const int k = c.max_drafts;
  const bool draft = static_cast<int>(blockIdx.y) > k;
  const int j = draft ? static_cast<int>(blockIdx.y) - k - 1 : static_cast<int>(blockIdx.y);
  const int lane = threadIdx.x & 63;
  const int chunk = blockIdx.x * kWaves + (threadIdx.x >> 6);
  const Request r = request_of(c, q);
  if (chunk >= a.chunks || !r.valid || (draft ? j >= r.n_drafts || r.greedy : j > r.n_drafts)) return;
  const float* row = draft ? c.draft_logits + (r.draft_row + j) * c.draft_stride
                           : c.target_logits + (r.target_row + j) * c.target_stride;
  const int base = chunk * kChunk;
  int held = -1;  // drafted token j
  if (!draft && !c.draft_logits && !r.greedy && j < r.n_drafts) held = c.drafts[static_cast<int64_t>(q) * k + j];
  if (held >= c.vocab) held = -1;
  float x[kPer];
  load_chunk(row, base, lane, c.vocab, x);
  const float best = chunk_max(x);
  int arg = INT32_MAX;
  if (r.greedy) {
#pragma unroll
    for (int u = kPer - 1; u >= 0; --u)
      if (x[u] == best) arg = id_of(base, lane, u);  // a lane's ids rise with u
    arg = wave_min(arg);
  }
  const Scale s = scale_of(best, r.c);
  double sum;
  if (held >= base && held < base + kChunk) {
    // A refused draft without a distribution leaves the row without that token, which a difference
    // of sums would not tell from a rounding: its chunk is added up without it, the token last.
    const float token = row[held];
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (id_of(base, lane, u) == held) x[u] = -INFINITY;
    Stat rest{0.0, chunk_max(x), INT32_MAX};
    rest.sum = chunk_sum(x, scale_of(rest.max, r.c));
    sum = in_row(rest, s) + weight(token, s);
    if (lane == 0) a.draft[(static_cast<int64_t>(q) * k + j) * a.chunks + chunk] = rest;
  } else {
    sum = chunk_sum(x, s);
  }
  if (lane == 0) {
    Stat* to = draft ? a.draft + (static_cast<int64_t>(q) * k + j) * a.chunks
                     : a.target + (static_cast<int64_t>(q) * (k + 1) + j) * a.chunks;
    to[chunk] = Stat{sum, best, arg};
  }
}

// A row's largest logit, its lowest id (greedy requests) and its sum of weights, by one wave;
// *own: what the lane's chunk, the lane-th, adds to that sum.
__device__ __forceinline__ Stat whole_row(const Stat* st, int chunks, const Request& r, int lane, double* own) {
  Stat mine{0.0, -INFINITY, INT32_MAX};
  if (lane < chunks) mine = st[lane];
  float best = mine.max;
  for (int i = lane + 64; i < chunks; i += 64) best = fmaxf(best, st[i].max);
  best = wave_max(best);
  int arg = INT32_MAX;
  if (r.greedy) {
    arg = mine.max == best ? mine.arg : INT32_MAX;
    for (int i = lane + 64; i < chunks; i += 64)
      if (st[i].max == best) arg = min(arg, st[i].arg);
    arg = wave_min(arg);
  }
  const Scale s = scale_of(best, r.c);
  double sum = *own = in_row(mine, s);
  for (int i = lane + 64; i < chunks; i += 64) sum += in_row(st[i], s);
  return Stat{wave_sum(sum), best, arg};
}

// What the work-groups of 2 and 3 need of a request's rows.
struct Verdict {
  Stat p[kMaxDrafts + 1], q[kMaxDrafts];  // (q without distributions: what a draft's chunk holds without it)
  float x[kMaxDrafts];  // the drafted tokens' logits
  int d[kMaxDrafts], keep[kMaxDrafts];
};

// Acceptance of a request's drafts, by all waves of the work-group; returns the number
// kept.  p and q of `v` hold the rows' sums afterwards, chunk[j][i] (if given) what chunk i < 64
// adds to target row j's.
// kChunk: of the chunks, where v.q is to hold what they have without the drafts; 0: not asked for.
template <int kNW, int kChunk>
__device__ __forceinline__ int accept(const Args& a, int q, const Request& r, Verdict& v,
                                      double (*chunk)[64] = nullptr) {
  const span_verify_call& c = a.c;
  const int k = c.max_drafts;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool dist = c.draft_logits && !r.greedy;
  // the drafted tokens and their logits: asked for first, used last
  const int mine = static_cast<int>(threadIdx.x);
  int d = -1;
  float x = 0.f, y = 0.f, u = 0.f, rest_max = -INFINITY;
  double rest = 0.0;
  if (mine < r.n_drafts) {
    d = c.drafts[static_cast<int64_t>(q) * k + mine];
    u = c.u_accept[static_cast<int64_t>(q) * k + mine];
    if (d >= 0 && d < c.vocab) {
      x = c.target_logits[(r.target_row + mine) * c.target_stride + d];
      if (dist) y = c.draft_logits[(r.draft_row + mine) * c.draft_stride + d];
      if constexpr (kChunk > 0)
        if (!dist && !r.greedy) {
          const Stat& st = a.draft[(static_cast<int64_t>(q) * k + mine) * a.chunks + d / kChunk];
          rest = st.sum;
          rest_max = st.max;
        }
    }
  }
  for (int e = wave; e < r.n_drafts + 1 + (dist ? r.n_drafts : 0); e += kNW) {
    const bool of_p = e <= r.n_drafts;
    const int j = of_p ? e : e - r.n_drafts - 1;
    const Stat* st = of_p ? a.target + (static_cast<int64_t>(q) * (k + 1) + j) * a.chunks
                          : a.draft + (static_cast<int64_t>(q) * k + j) * a.chunks;
    double own;
    const Stat s = whole_row(st, a.chunks, r, lane, &own);
    if (lane == 0) (of_p ? v.p[j] : v.q[j]) = s;
    if (chunk && of_p) chunk[j][lane] = own;
  }
  __syncthreads();
  if (mine < r.n_drafts) {
    const int j = mine;
    bool keep = false;
    if (r.greedy) {
      keep = v.p[j].sum > 0.0 && d == v.p[j].arg;
    } else if (d >= 0 && d < c.vocab) {
      const double pd = v.p[j].sum > 0.0 ? weight(x, scale_of(v.p[j].max, r.c)) / v.p[j].sum : 0.0;
      double qd = 1.0;
      if (dist) qd = v.q[j].sum > 0.0 ? weight(y, scale_of(v.q[j].max, r.c)) / v.q[j].sum : 0.0;
      keep = static_cast<double>(u) * qd < pd;
    }
    v.keep[j] = keep;
    v.d[j] = d;
    v.x[j] = x;
    if constexpr (kChunk > 0)
      if (!dist) v.q[j] = Stat{rest, rest_max, INT32_MAX};
  }
  __syncthreads();
  int n = 0;
  while (n < r.n_drafts && v.keep[n]) ++n;
  return n;
}

// A row's sum of weights and its inverse, 0 and 0 if there are none.
struct Whole {
  double sum, inverse;
};
__device__ __forceinline__ Whole whole_of(double s) { return s > 0.0 ? Whole{s, 1.0 / s} : Whole{0.0, 0.0}; }

// max(p - q, 0) of two weights and their rows' sums.  Both quotients are rounded as divisions are, and before the
// difference: otherwise that of equal ones, or of two that are all of their rows, would be a rounding, not 0, and
// where p = q nothing may be left.
__device__ __forceinline__ double residue(double p, const Whole& ps, double q, const Whole& qs) {
  double a = p * ps.inverse, b = q * qs.inverse;
  a = fma(fma(-ps.sum, a, p), ps.inverse, a);
  b = fma(fma(-qs.sum, b, q), qs.inverse, b);
  return fmax(a - b, 0.0);
}

// What the row that decides a request leaves of a token: max(p - q, 0), or p.
struct Left {
  const float* x;
  const float* y;  // the draft's logits, or null
  Scale p, q;
  Whole ps, qs;
  int one_hot;    // the token taken out of p where the draft has no distribution, -1: none
  __device__ __forceinline__ double of(int i, float xi, float yi) const {
    if (y) return residue(weight(xi, p), ps, weight(yi, q), qs);
    return i == one_hot ? 0.0 : weight(xi, p) * ps.inverse;
  }
};

// At the first refused draft n, or (plain, or after the last draft) p_n itself.
__device__ __forceinline__ Left left_of(const Args& a, int q, const Request& r, const Verdict& v, int n, bool plain) {
  const span_verify_call& c = a.c;
  Left l{};
  l.x = c.target_logits + (r.target_row + n) * c.target_stride;
  l.p = scale_of(v.p[n].max, r.c);
  l.ps = whole_of(v.p[n].sum);
  l.one_hot = -1;
  if (n < r.n_drafts && !plain) {
    if (c.draft_logits) {
      l.y = c.draft_logits + (r.draft_row + n) * c.draft_stride;
      l.q = scale_of(v.q[n].max, r.c);
      l.qs = whole_of(v.q[n].sum);
    } else {
      const int d = v.d[n];
      l.one_hot = d >= 0 && d < c.vocab ? d : -1;
    }
  }
  return l;
}

// ------------------------------------------------------------------ 2: what the deciding row leaves
// All waves of 64 requests stand on the chip at once, so acceptance (5 us), their loads (66 MB) and
// two exponentials a token (7 us of instructions) follow one another: 18 us.  With eight waves a
// work-group the same, with 16 an eighth more; acceptance in a launch of its own costs what it saves.
template <int kChunk>
__global__ __launch_bounds__(kThreads) void verify_left_kernel(const Args a) {
  constexpr int kPer = kChunk / 64;
  __shared__ Verdict v;
  const span_verify_call& c = a.c;
  const int q = a.q0 + static_cast<int>(blockIdx.y);
  const int lane = threadIdx.x & 63;
  const Request r = request_of(c, q);
  if (!r.valid || r.greedy || r.n_drafts == 0) return;
  const int n = accept<kWaves, 0>(a, q, r, v);
  const int chunk = blockIdx.x * (kWaves) + (threadIdx.x >> 6);
  if (n == r.n_drafts || chunk >= a.chunks) return;  // after the last draft the chunks' own sums serve
  const Left l = left_of(a, q, r, v, n, false);
  const int base = chunk * kChunk;
  float x[kPer], y[kPer];
  load_chunk(l.x, base, lane, c.vocab, x);
  load_chunk(l.y, base, lane, c.vocab, y);
  double sum = 0.0;
  if (l.p.hot || l.q.hot) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) sum += l.of(-2, x[u], y[u]);
  } else {
#pragma unroll
    for (int u = 0; u < kPer; ++u) sum += residue(weight_at(x[u], l.p), l.ps, weight_at(y[u], l.q), l.qs);
  }
  sum = wave_sum(sum);
  if (lane == 0) a.left[static_cast<int64_t>(q) * a.chunks + chunk] = sum;
}

// ------------------------------------------------------------------ 3: the token
// 6.5 us for one request: four loads that need one another's results, and sums over a work-group.
template <int kChunk>
__global__ __launch_bounds__(kPickThreads) void verify_pick_kernel(const Args a) {
  constexpr int kPickWaves = kPickThreads / 64;
  constexpr int kEach = (kChunk + kPickThreads - 1) / kPickThreads;  // of the first threads, if there are too many
  __shared__ Verdict v;
  __shared__ double s_chunk[kMaxDrafts + 1][64];
  __shared__ double s_wave[kPickWaves];
  __shared__ int s_first, s_last;
  __shared__ float s_x;
  const span_verify_call& c = a.c;
  const int q = a.q0 + static_cast<int>(blockIdx.x);
  const int k = c.max_drafts;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Request r = request_of(c, q);
  int32_t* tokens = c.tokens + static_cast<int64_t>(q) * (k + 1);
  float* lps = c.logprobs ? c.logprobs + static_cast<int64_t>(q) * (k + 1) : nullptr;
  if (!r.valid) {
    if (static_cast<int>(threadIdx.x) <= k) {
      tokens[threadIdx.x] = -1;
      if (lps) lps[threadIdx.x] = 0.f;
    }
    if (threadIdx.x == 0) c.accepted[q] = -1;
    return;
  }
  if (threadIdx.x == 0) {
    s_first = INT32_MAX;
    s_last = -1;
  }
  const float u_sample = c.u_sample[q];
  const int n = accept<kPickWaves, kChunk>(a, q, r, v, s_chunk);  // (its barriers also publish s_first and s_last)
  int token = -1;
  if (!(v.p[n].sum > 0.0)) {
  } else if (r.greedy) {
    token = v.p[n].arg;
  } else {
    const Stat* st = a.target + (static_cast<int64_t>(q) * (k + 1) + n) * a.chunks;
    // Every wave finds the chunk for itself: the first one whose running sum passes u times
    // the whole, else the last with any weight.
    Left l = left_of(a, q, r, v, n, false);
    double aim = 0.0, before = 0.0;
    int chunk = -1;
    for (int attempt = 0; attempt < 2 && chunk < 0; ++attempt) {
      if (attempt == 1) l = left_of(a, q, r, v, n, true);  // nothing left of p: p itself
      auto chunk_sum = [&](int i) -> double {
        if (i >= a.chunks) return 0.0;
        if (l.y) return a.left[static_cast<int64_t>(q) * a.chunks + i];
        if (l.one_hot >= 0 && l.one_hot / kChunk == i) return in_row(v.q[n], l.p) * l.ps.inverse;
        return (i < 64 ? s_chunk[n][i] : in_row(st[i], l.p)) * l.ps.inverse;
      };
      const double own = chunk_sum(lane);  // all of them up to 64 chunks
      double total = 0.0;
      for (int b = 0; b < a.chunks; b += 64) total += wave_sum(b == 0 ? own : chunk_sum(b + lane));
      aim = static_cast<double>(u_sample) * total;
      double run = 0.0;
      for (int b = 0; b < a.chunks; b += 64) {
        const double w = b == 0 ? own : chunk_sum(b + lane);
        const double upto = run + wave_scan(w);
        const unsigned long long some = __ballot(w > 0.0), past = __ballot(w > 0.0 && upto > aim);
        // the first that passes; while none does, the last with weight
        const int at = past ? __ffsll(past) - 1 : some ? 63 - __clzll(some) : -1;
        if (at >= 0) {
          chunk = b + at;
          before = __shfl(upto, at) - __shfl(w, at);
        }
        if (past) break;
        run = __shfl(upto, 63);
      }
    }
    // the token in the chunk: each thread tokens that follow one another
    const int i0 = chunk * kChunk + static_cast<int>(threadIdx.x) * kEach;
    float x[kEach], y[kEach];
    double w[kEach], mine = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = min(i0 + e, c.vocab - 1);
      x[e] = l.x[i];
      y[e] = l.y ? l.y[i] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      w[e] = i0 + e < min(c.vocab, (chunk + 1) * kChunk) ? l.of(i0 + e, x[e], y[e]) : 0.0;
      mine += w[e];
    }
    const double upto = wave_scan(mine);
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    double at = before + upto - mine;
    for (int e = 0; e < wave; ++e) at += s_wave[e];
    int first = INT32_MAX, last = -1;
#pragma unroll
    for (int e = kEach - 1; e >= 0; --e)
      if (w[e] > 0.0) last = max(last, i0 + e);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      at += w[e];
      if (w[e] > 0.0 && at > aim) first = min(first, i0 + e);
    }
    if (first != INT32_MAX) atomicMin(&s_first, first);
    if (last >= 0) atomicMax(&s_last, last);
    __syncthreads();
    token = s_first != INT32_MAX ? s_first : s_last;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (i0 + e == token) s_x = x[e];
    __syncthreads();
  }
  const int j = static_cast<int>(threadIdx.x);
  if (j <= k) {
    const int t = j < n ? v.d[j] : j == n ? token : -1;
    tokens[j] = t;
    if (lps) {
      float lp = 0.f;
      if (t >= 0) {
        const float x = j < n ? v.x[j] : r.greedy ? v.p[n].max : s_x;
        const Scale s = scale_of(v.p[j].max, r.c);
        // (a logit with all the weight is relative to itself)
        const double d = s.hot ? 0.0 : fma(static_cast<double>(x), s.c, -s.k);
        lp = static_cast<float>(d * 0.69314718055994530942 - log(v.p[j].sum));
      }
      lps[j] = lp;
    }
  }
  if (threadIdx.x == 0) c.accepted[q] = n;
}

int64_t chunks_of(int vocab, int chunk) { return (vocab + chunk - 1) / chunk; }

// Logits of a chunk: the fewest of 512, 1024 and 2048 that leave a row at most 64 chunks, one for
// each lane that adds them up, and all rows at most 2^16.  Small chunks spread few logits over the chip,
// and are more to add up in 2 and 3.  Four drafts with a distribution, captured calls of 512 / 1024 / 2048 in us:
//   vocabulary 8000:    8 requests 15.2 / 16.7 / 20.1   64: 21.0 / 22.2 / 25.1   256: 34.2 / 33.4 / 35.9
//   vocabulary 32768:   8 requests 15.9 / 17.0 / 20.6   64: 32.3 / 31.5 / 32.2   256: 100 / 88 / 83
bool chunk_fits(int64_t requests, int max_drafts, int vocab, int chunk) {
  const int64_t n = chunks_of(vocab, chunk);
  return n <= 64 && requests * (2 * max_drafts + 1) * n <= 1 << 16;
}
int chunk_of(int64_t requests, int max_drafts, int vocab) {
  for (const int chunk : {512, 1024})
    if (chunk_fits(requests, max_drafts, vocab, chunk)) return chunk;
  return 2048;
}

// f(a chunk size as a type)
template <class F>
hipError_t with_chunk(int chunk, F f) {
  switch (chunk) {
    case 512: return f(std::integral_constant<int, 512>{});
    case 1024: return f(std::integral_constant<int, 1024>{});
    default: return f(std::integral_constant<int, 2048>{});
  }
}

}  // namespace

size_t verify_workspace_bytes(int64_t n, int max_drafts, int vocab) {
  const int64_t ch = chunks_of(vocab, chunk_of(n, max_drafts, vocab));
  return static_cast<size_t>(n * ch) * ((2 * static_cast<size_t>(max_drafts) + 1) * sizeof(Stat) + sizeof(double));
}

size_t verify_workspace_up_to(int64_t n, int max_drafts, int vocab) {
  size_t most = verify_workspace_bytes(n, max_drafts, vocab);
  for (const int chunk : {512, 1024}) {  // the most requests that take chunks so small
    const int64_t ch = chunks_of(vocab, chunk);
    if (ch <= 64) most = std::max(most, verify_workspace_bytes(std::min(n, (1 << 16) / (ch * (2 * max_drafts + 1))), max_drafts, vocab));
  }
  return most;
}

hipError_t launch_verify_drafts(const span_verify_call& c, hipStream_t s) {
  Args a{};
  a.c = c;
  const int chunk = chunk_of(c.n_requests, c.max_drafts, c.vocab);
  a.chunks = static_cast<int>(chunks_of(c.vocab, chunk));
  const size_t n = static_cast<size_t>(c.n_requests), ch = static_cast<size_t>(a.chunks), k = c.max_drafts;
  a.target = static_cast<Stat*>(c.workspace);
  a.draft = a.target + n * (k + 1) * ch;
  a.left = reinterpret_cast<double*>(a.draft + n * k * ch);
  const unsigned rows = static_cast<unsigned>(c.max_drafts + 1 + (c.draft_logits ? c.max_drafts : 0));
  // requests on the grid's last dimension: as many at once as it takes
  const int64_t threads = std::max<int64_t>((a.chunks + kWaves - 1) / kWaves * static_cast<int64_t>(rows) * kThreads, int64_t{1} << 17);
  return launch_in_slices(c.n_requests, threads, hipErrorInvalidValue, [&](int64_t first, int64_t count) -> hipError_t {
    a.q0 = static_cast<int>(first);
    const unsigned nq = static_cast<unsigned>(count);
    const unsigned groups = static_cast<unsigned>((a.chunks + kWaves - 1) / kWaves);
    return with_chunk(chunk, [&](auto size) -> hipError_t {
      constexpr int kChunk = decltype(size)::value;
      verify_stats_kernel<kChunk><<<dim3(groups, rows, nq), kThreads, 0, s>>>(a);
      hipError_t e = hipGetLastError();
      if (e == hipSuccess && c.draft_logits && c.max_drafts > 0) {
        verify_left_kernel<kChunk><<<dim3(groups, nq), kThreads, 0, s>>>(a);
        e = hipGetLastError();
      }
      if (e != hipSuccess) return e;
      verify_pick_kernel<kChunk><<<nq, kPickThreads, 0, s>>>(a);
      return hipGetLastError();
    });
  });
}

}  // namespace spanq
