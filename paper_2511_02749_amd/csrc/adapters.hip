// Low-rank adapters of many requests beside a shared projection:
//
//   out[i] = base[i] + scale[a] (x[i] A[a]^T) B[a]^T,   a = ids[i], rows without one copied
//
// Shrink: H = x A^T, sums of K products in fp32 split over a work-group's waves and over
// work-groups, each slice's partial in the workspace.  Expand: the partials summed in slice
// order, the product with B, scale and base added, rounded once.  For many rows of wide
// products the partials are summed once in between (finish); else expand does it as it goes.
//
// Few rows (a decode step): the rows of one adapter, up to 16 at a time,
// wherever they lie in the call, are one group, found from the ids by the work-groups
// themselves, so that each adapter's weights are read once.  Many rows (prefilled
// segments, large decode steps): a launch of its own orders the rows by adapter, and tiles of
// 64 ordered rows are worked once for each adapter that occurs in one, mostly one.  The ids
// stay on the device and may change between replays of a captured call.
//
// Matrix instructions 16x16x32, every operand 16 bytes of a row.  The second product's
// columns are dealt to its tiles so that a lane's results of all tiles are columns that
// follow one another, and base and out go as whole lines.  H enters it as three bf16 numbers
// that add up to it (24 significant bits): two of them side by side in the 32 deep reduction
// over the same 16 ranks, the third in an instruction of its own.
//
// Bound: HBM (x, base and out for many rows, A and B for few); 2 R (K P + N) operations a row.
// Decode steps are bound by the latency of their two launches and the loads in a row inside them.
//
// Times of calls are of captured ones, one after another over three sets of inputs; a kernel's alone is its
// median in a trace of such calls.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "dev_common.h"
#include "mfma_common.h"
#include "row_ops.h"

namespace spanq {
namespace {

using mfma::hi_bf16;
using mfma::lo_bf16;
using mfma::pack_bf16x2;

constexpr int kTile = 16;      // rows of a group, ranks of a block
constexpr int kParts = 3;      // bf16 numbers that hold a value of H: high, middle, low
constexpr int kFewRows = 256;  // at most, of the few-row form (few_rows)
// Work-groups over K at most.  Few rows, 16 for 8: 48 rows of K 14336 18.3 -> 18.1 us, but 200 rows of
// rank 128, whose partials are many, 33.3 -> 34.1.
constexpr int kFewSlices = 8;
constexpr int kManySlices = 16;
constexpr int kXcds = 8;
// Work-groups to which the adapters of a tile are dealt (2048 rows of 28672 columns in four segments: 76.2
// us with one, 73.4 with four; with eight, which are mostly empty, 1000 rows of 4096 columns 25.2 -> 28.1).
constexpr int kManyGroups = 4;
constexpr int kManyTiles = 4;  // 16-row tiles of a many-row work-group

// Shrink work-groups: waves (each with its own part of K), 16-row and 16-column tiles of H,
// and products of 32 values whose loads are in flight together (few rows: 16 KB a wave; with four
// waves and half the loads 200 rows of rank 128 take 37.0 us for 33.3, 48 rows of K 14336 the same 18.2).
struct FewShrink {
  static constexpr int kWaves = 2, kRows = 1, kCols = 1, kSteps = 8;
};
struct ManyShrink {
  static constexpr int kWaves = 4, kRows = kManyTiles, kCols = 4, kSteps = 2;
};

struct Shape {
  const bf16_t* x;
  const bf16_t* base;
  bf16_t* out;
  const int32_t* ids;
  const bf16_t* a;
  const bf16_t* b;
  const float* scale;
  const int32_t* ranks;
  float* part;   // [slices][rows][h_cols] fp32
  bf16_t* h;     // many rows: [rows][h_cols / 16][kParts][16]
  int2* order;   // many rows: {row, its adapter or -1}, each adapter's rows together; H lies in this order
  int64_t rows, x_stride, base_stride, out_stride;
  int K, R, n_adapters, n_parts;
  int N;         // columns of all parts
  int cols[4];   // columns of each part
  int rank_blocks, h_cols;  // ceil(R / 16); 16 * n_parts * rank_blocks
  int slices, k_slice;
  int run;  // tiles of 16 rows that an expand work-group of many rows takes
};

__device__ __forceinline__ int adapter_of(const Shape& s, int64_t row) {
  const int id = row < s.rows ? s.ids[row] : -1;
  return id >= 0 && id < s.n_adapters ? id : -1;
}

// (a scalar, so that what follows from it is one too)
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

__device__ __forceinline__ int rank_of(const Shape& s, int id) {
  return s.ranks ? max(0, min(s.ranks[id], s.R)) : s.R;
}

// The group that row j of few rows leads: rows of its adapter from j on, the first 16, if
// as many of them as make whole groups lie before j.  Fills rows[0 .. n) and returns n, 0 if
// j leads none.  Called by all threads; every wave finds it, wave 0 writes it.
__device__ __forceinline__ int few_group(const Shape& s, int j, int* aid, int* rows) {
  const int lane = threadIdx.x & 63;
  const int mine = adapter_of(s, j);
  *aid = mine;
  const int n_rows = static_cast<int>(s.rows);
  int id[kFewRows / 64];
#pragma unroll
  for (int b = 0; b < kFewRows / 64; ++b) id[b] = 64 * b < n_rows ? adapter_of(s, 64 * b + lane) : -1;
  int before = 0, n = 0;
#pragma unroll
  for (int b = 0; b < kFewRows / 64; ++b) {
    const int row = 64 * b + lane;
    const bool same = row < n_rows && id[b] == mine;
    before += __popcll(__ballot(same && row < j));
    const unsigned long long later = __ballot(same && row >= j);
    const int at = n + __popcll(later & ((1ull << lane) - 1));
    if (threadIdx.x < 64 && same && row >= j && at < kTile) rows[at] = row;
    n += __popcll(later);
  }
  __syncthreads();
  return before % kTile == 0 ? min(n, kTile) : 0;
}

// The adapters of 64 rows (lane i: row i), each with its rows as a mask: f(adapter, rows).
// Wave-uniform.
template <class F>
__device__ __forceinline__ void for_adapters(int id, unsigned long long live, F f) {
  while (live) {
    const int aid = __builtin_amdgcn_readlane(id, __ffsll(live) - 1);
    const unsigned long long mine = __ballot(id == aid) & live;
    f(aid, mine);
    live &= ~mine;
  }
}

__device__ __forceinline__ bf16x8_t as_frag(const uint4& v) { return __builtin_bit_cast(bf16x8_t, v); }

// The upper halves of two words, packed.
__device__ __forceinline__ uint32_t upper(uint32_t a, uint32_t b) { return a >> 16 | (b & 0xffff0000u); }

// Two floats as their parts, packed: the upper half of the float, of what that leaves, and of what
// is then left, 8 significant bits each, so that no more than 24 remain to be rounded (infinities
// and NaN are the first part's alone).
__device__ __forceinline__ void split3(float a, float b, uint32_t* part) {
  uint32_t u = __float_as_uint(a), v = __float_as_uint(b);
  part[0] = upper(u, v);
#pragma unroll
  for (int i = 1; i < kParts; ++i) {
    const float x = __uint_as_float(u), y = __uint_as_float(v);
    u = __float_as_uint(isfinite(x) ? x - hi_bf16(u) : 0.f);
    v = __float_as_uint(isfinite(y) ? y - hi_bf16(v) : 0.f);
    part[i] = upper(u, v);
  }
}

// Four sums of H as their parts, ranks 4 q .. of a block at h.
__device__ __forceinline__ void store_split(bf16_t* h, int q, const float4& sum) {
  uint32_t lo[kParts], hi[kParts];
  split3(sum.x, sum.y, lo);
  split3(sum.z, sum.w, hi);
#pragma unroll
  for (int i = 0; i < kParts; ++i) reinterpret_cast<uint2*>(h)[q + 4 * i] = uint2{lo[i], hi[i]};
}

// acc[j] + the product of 32 ranks' worth of H with the weights of tile j
template <int J>
__device__ __forceinline__ void multiply_h(const uint4& h, const uint4 (&w)[J], f32x4_t (&acc)[J]) {
#pragma unroll
  for (int j = 0; j < J; ++j)
    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(h), as_frag(w[j]), acc[j], 0, 0, 0);
}

// Eight weights, infinite ones and NaN replaced by 0.  An infinite weight times H is what it is times H's
// high part, which has H's sign and is 0 only where H is; a middle or low part may be 0 or of the
// other sign and would make it NaN.
__device__ __forceinline__ uint4 finite_of(const uint4& v) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
    if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
  }
  return uint4{w[0], w[1], w[2], w[3]};
}

// Is any result of the tiles infinite or NaN?  Wave-uniform.
template <int J>
__device__ __forceinline__ bool any_wild(const f32x4_t (&acc)[J]) {
  uint32_t most = 0;  // of the values' bits without their signs
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, __float_as_uint(fabsf(acc[j][i])));
  return __ballot(most >= 0x7f800000u) != 0;
}

__device__ __forceinline__ float4 operator+(const float4& a, const float4& b) {
  return float4{a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w};
}

// Many rows: their order, by adapter, rows without one last (adapters that are equal modulo
// the number of the others' buckets lie among each other, which costs time, nothing else).  One
// work-group counts each bucket's rows, adds the counts up and gives every row its place; which
// of a bucket's rows comes first may change from run to run, and no result depends on it.
// 777 rows 4.1 us, 2048 rows 4.8, 65536 rows 38 to 50: the latency of two passes.  Without it 2048 rows of 32 mixed
// adapters (rank 32, 4096 -> 28672) take 1002 us for 95, and rows in segments 4 us less.
constexpr int kOrderThreads = 1024;  // and buckets
__global__ __launch_bounds__(kOrderThreads) void adapter_order_kernel(const Shape s) {
  __shared__ int place[kOrderThreads];
  __shared__ int sums[kOrderThreads / 64];
  const int t = threadIdx.x, lane = t & 63, n = static_cast<int>(s.rows);
  // The next places of a row's bucket: where a wave's rows are all of one, as in a prefilled
  // segment, one lane takes them all.
  auto take = [&](int id) {
    const int bucket = id < 0 ? kOrderThreads - 1 : id % (kOrderThreads - 1);
    const int first = __builtin_amdgcn_readfirstlane(bucket);
    const unsigned long long all = __ballot(true);
    if (__ballot(bucket != first) != 0) return atomicAdd(&place[bucket], 1);
    const int before = __popcll(all & ((1ull << lane) - 1));
    int at = 0;
    if (before == 0) at = atomicAdd(&place[bucket], __popcll(all));
    return __builtin_amdgcn_readfirstlane(at) + before;
  };
  // f(row, its adapter) for the thread's rows, four ids asked for together
  auto each = [&](auto f) {
    constexpr int kAhead = 4;
    for (int i0 = t; i0 < n; i0 += kAhead * kOrderThreads) {
      int id[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) id[u] = adapter_of(s, i0 + u * kOrderThreads);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i0 + u * kOrderThreads < n) f(i0 + u * kOrderThreads, id[u]);
    }
  };
  place[t] = 0;
  __syncthreads();
  each([&](int, int id) { take(id); });
  __syncthreads();
  const int mine = place[t];
  int upto = mine;  // sum of the wave's buckets up to this one
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int v = __shfl_up(upto, d);
    upto += lane >= d ? v : 0;
  }
  if (lane == 63) sums[wave_id()] = upto;
  __syncthreads();
  int before = upto - mine;
  for (int w = 0; w < wave_id(); ++w) before += sums[w];
  place[t] = before;
  __syncthreads();
  each([&](int i, int id) { s.order[take(id)] = int2{i, id}; });
}

// H of one group (few) or of a tile of 64 ordered rows: one slice of K, C::kCols column tiles.
// 64 rows of 64 adapters, K 4096, rank 16 (8.4 MB of A): 5.0 us; 48 rows of 12, K 14336, rank 64 (22
// MB): 11.7 us, four rounds of loads one after another.  2048 rows, K 4096, 64 columns of H: 12.0 us.
template <bool kFew, class C>
__global__ __launch_bounds__(64 * C::kWaves) void adapter_shrink_kernel(const Shape s) {
  __shared__ float4 red[C::kWaves][C::kCols][16 * C::kRows][4];
  __shared__ int list[16 * C::kRows];  // rows of the call
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int col_groups = (s.h_cols / 16 + C::kCols - 1) / C::kCols;
  // Few rows: a work-group for each slice and column group of every row.  Many: units of a tile and a
  // slice are dealt to the XCDs, a unit's column groups one after another, so that x is fetched once,
  // and with eight or sixteen slices one XCD alone fetches a slice of A.  1387 rows, K 13224, 96 columns
  // of H: 33 us with five slices as they come, 23 with eight.
  const int unit = kFew ? blockIdx.x / col_groups : blockIdx.x / (kXcds * col_groups) * kXcds + blockIdx.x % kXcds;
  const int slice = kFew ? unit : unit % s.slices;
  const int ct0 = (kFew ? blockIdx.x : blockIdx.x / kXcds) % col_groups * C::kCols;
  const int64_t tile = kFew ? 0 : unit / s.slices;
  const int n_ct = min(C::kCols, s.h_cols / 16 - ct0);
  const int sub = s.k_slice / C::kWaves;
  const int k0 = slice * s.k_slice + wave * sub;
  const int k1 = min(s.K, k0 + sub);
  const int m = lane & 15, g = lane >> 4;
  // h_row(i): where H of row i of the group or tile goes
  auto work = [&](int aid, unsigned long long mine, auto h_row) {
    const int rank = rank_of(s, aid);
    // Rows outside the group and ranks past the adapter's are read as the group's first row and
    // rank: no result of theirs is used, and no load needs a branch.
    const int row1 = __ffsll(mine) - 1;
    const bf16_t* xp[C::kRows];
#pragma unroll
    for (int t = 0; t < C::kRows; ++t)
      xp[t] = s.x + list[(mine >> (16 * t + m)) & 1 ? 16 * t + m : row1] * s.x_stride + 8 * g;
    const bf16_t* ap[C::kCols];
#pragma unroll
    for (int c = 0; c < C::kCols; ++c) {
      const int ct = ct0 + min(c, n_ct - 1), p = ct / s.rank_blocks, r = (ct - p * s.rank_blocks) * 16 + m;
      ap[c] = s.a + ((static_cast<int64_t>(aid) * s.n_parts + p) * s.R + (r < rank ? r : 0)) * s.K + 8 * g;
    }
    f32x4_t acc[C::kRows][C::kCols] = {};
    uint4 xv[C::kRows][C::kSteps], wv[C::kCols][C::kSteps];
    auto multiply = [&] {
#pragma unroll
      for (int u = 0; u < C::kSteps; ++u)
#pragma unroll
        for (int t = 0; t < C::kRows; ++t)
#pragma unroll
          for (int c = 0; c < C::kCols; ++c)
            acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(wv[c][u]), as_frag(xv[t][u]), acc[t][c], 0, 0, 0);
    };
    int k = k0;
    for (; k + 32 * C::kSteps <= k1; k += 32 * C::kSteps) {
#pragma unroll
      for (int u = 0; u < C::kSteps; ++u) {
#pragma unroll
        for (int t = 0; t < C::kRows; ++t) xv[t][u] = *reinterpret_cast<const uint4*>(xp[t] + k + 32 * u);
#pragma unroll
        for (int c = 0; c < C::kCols; ++c) wv[c][u] = *reinterpret_cast<const uint4*>(ap[c] + k + 32 * u);
      }
      multiply();
    }
    if (k < k1) {  // the end of a K that is no multiple
#pragma unroll
      for (int u = 0; u < C::kSteps; ++u) {
        const bool in = k + 32 * u + 8 * g < k1;
#pragma unroll
        for (int t = 0; t < C::kRows; ++t) {
          xv[t][u] = uint4{0u, 0u, 0u, 0u};
          if (in) xv[t][u] = *reinterpret_cast<const uint4*>(xp[t] + k + 32 * u);
        }
#pragma unroll
        for (int c = 0; c < C::kCols; ++c) {
          wv[c][u] = uint4{0u, 0u, 0u, 0u};
          if (in) wv[c][u] = *reinterpret_cast<const uint4*>(ap[c] + k + 32 * u);
        }
      }
      multiply();
    }
    // A lane holds ranks 4 g .. of row m of each tile.  Stores of matrix instructions' results stand behind a
    // condition here (all four tiles stored: 1 us more for one): their wait is spelled out.
    asm volatile("s_nop 15" ::: "memory");
#pragma unroll
    for (int t = 0; t < C::kRows; ++t)
#pragma unroll
      for (int c = 0; c < C::kCols; ++c)
        if (c < n_ct) red[wave][c][16 * t + m][g] = __builtin_bit_cast(float4, acc[t][c]);
    __syncthreads();
    for (int e = threadIdx.x; e < n_ct * 64 * C::kRows; e += 64 * C::kWaves) {
      const int q = e & 3, row = (e >> 2) % (16 * C::kRows), c = e / (64 * C::kRows);
      if (!((mine >> row) & 1)) continue;
      float4 sum = red[0][c][row][q];
#pragma unroll
      for (int w = 1; w < C::kWaves; ++w) sum = sum + red[w][c][row][q];
      const int64_t to = h_row(row);
      const int r = (ct0 + c) % s.rank_blocks * 16 + 4 * q;  // past the rank H is zero
      sum = float4{r < rank ? sum.x : 0.f, r + 1 < rank ? sum.y : 0.f, r + 2 < rank ? sum.z : 0.f, r + 3 < rank ? sum.w : 0.f};
      if (!kFew && s.h && s.slices == 1)
        store_split(s.h + kParts * (to * s.h_cols + (ct0 + c) * 16), q, sum);
      else
        *reinterpret_cast<float4*>(s.part + (slice * s.rows + to) * s.h_cols + (ct0 + c) * 16 + 4 * q) = sum;
    }
    __syncthreads();
  };
  if constexpr (kFew) {
    int aid = 0;
    const int n = few_group(s, blockIdx.y, &aid, list);
    if (n > 0 && aid >= 0) work(aid, (1ull << n) - 1, [&](int i) -> int64_t { return list[i]; });
  } else {
    const int64_t row0 = tile * (16 * C::kRows);
    if (row0 >= s.rows) return;
    const int64_t row = row0 + lane;
    const unsigned long long live = __ballot(row < s.rows);
    const int2 at = row < s.rows ? s.order[row] : int2{0, -1};
    if (wave == 0) list[lane] = at.x;
    __syncthreads();
    // the tile's adapters are dealt to kManyGroups work-groups: where a tile holds the end of one
    // request and the start of the next, neither waits for the other
    int n = 0;
    for_adapters(at.y, live, [&](int aid, unsigned long long mine) {
      if (aid >= 0 && n++ % kManyGroups == static_cast<int>(blockIdx.z))
        work(aid, mine, [&](int i) -> int64_t { return row0 + i; });
    });
  }
}

// Many rows: the slices' partials of H added up, as their parts (2048 rows, 64 columns, 8
// slices: 5.0 us).
__global__ __launch_bounds__(256) void adapter_finish_kernel(const Shape s) {
  const int64_t plane = s.rows * s.h_cols / 4;  // in vectors of four
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (e >= plane) return;
  const float4* p = reinterpret_cast<const float4*>(s.part) + e;
  float4 v[kManySlices];
#pragma unroll
  for (int i = 0; i < kManySlices; ++i) v[i] = i < s.slices ? p[i * plane] : float4{0.f, 0.f, 0.f, 0.f};
  float4 sum = v[0];
#pragma unroll
  for (int i = 1; i < kManySlices; ++i) sum = sum + v[i];
  store_split(s.h + 16 * kParts * (e / 4), static_cast<int>(e & 3), sum);
}

// Zeroes elements n .. 7 of eight bf16 values.
__device__ __forceinline__ uint4 first_of(const uint4& v, int n) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n < 2 * i + 2) w[i] &= 0xffffu;
    if (n < 2 * i + 1) w[i] = 0u;
  }
  return uint4{w[0], w[1], w[2], w[3]};
}

constexpr int kExpandWaves = 4;

// The wave's columns of one part, n0 .. of `width`, and where they lie in all columns.
struct Cols {
  int part, n0, width, col0;
};

// J tiles of 16 columns: column m of tile j is column J m + j of the wave's, so that a lane's
// results are J columns that follow one another.
// kStream: base and out pass the caches by (a call of many rows reads and writes each of
// their lines once: 2048 rows of 28672 columns 74.3 -> 71.7 us, of 6144 at rank 128 68.4 -> 69.5).
template <int J, bool kStream>
struct Out {
  typedef uint32_t Vec __attribute__((ext_vector_type(J / 2)));
  // Ranks r0 .. r0 + 7 of tile j's weights, those past `rank` zero.  Columns past the part's
  // and ranks past R are read as its first ones: no result of theirs is used.
  static __device__ __forceinline__ uint4 weights(const Shape& s, const Cols& c, int aid, int j, int m, int r0,
                                                  int rank, bool whole) {
    const int col = c.n0 + J * m < c.width ? c.n0 + J * m + j : j;
    // (columns times rank stay below 2^28 bytes)
    const char* part = reinterpret_cast<const char*>(s.b + (static_cast<int64_t>(aid) * s.N + c.col0) * s.R);
    const uint4 v = *reinterpret_cast<const uint4*>(part + static_cast<uint32_t>(2 * (col * s.R + (r0 < s.R ? r0 : 0))));
    return whole ? v : first_of(v, rank - r0);
  }
  static __device__ __forceinline__ Vec base(const bf16_t* rows, int64_t stride, const Cols& c, int r, int m) {
    const Vec* p = reinterpret_cast<const Vec*>(rows + offset(r, stride, c.n0 + J * m < c.width ? c.n0 + J * m : 0));
    return kStream ? __builtin_nontemporal_load(p) : *p;
  }
  static __device__ __forceinline__ void store(bf16_t* rows, int64_t stride, const Cols& c, int r, int m, const Vec& v) {
    Vec* p = reinterpret_cast<Vec*>(rows + offset(r, stride, c.n0 + J * m));
    if (kStream)
      __builtin_nontemporal_store(v, p);
    else
      *p = v;
  }
  // (strides are at most 2^23: one 32 x 32 bit product)
  static __device__ __forceinline__ uint64_t offset(int r, int64_t stride, int col) {
    return static_cast<uint64_t>(static_cast<uint32_t>(r)) * static_cast<uint32_t>(stride) + static_cast<uint32_t>(col);
  }
  // base + scale * row i of the tiles' results
  static __device__ __forceinline__ Vec add(const Vec& base, const f32x4_t (&acc)[J], int i, float scale) {
    Vec v;
#pragma unroll
    for (int j = 0; j < J / 2; ++j)
      v[j] = pack_bf16x2(fmaf(scale, acc[2 * j][i], lo_bf16(base[j])), fmaf(scale, acc[2 * j + 1][i], hi_bf16(base[j])));
    return v;
  }
  // The tiles' results once more, where one is infinite or NaN: only H's high parts meet infinite weights.
  // h(rb, at): vector `at` of block rb of the lane's row of H.  With kPairs the low parts of two
  // blocks go together.  The steps are those of the first time, so that finite results keep their bits.
  // (The weights are fetched again: kept for this, they would cost registers that every call has to give.)
  template <bool kPairs, class F>
  static __device__ __forceinline__ void wild(const Shape& s, const Cols& c, int aid, int rank, int m, int g, F h,
                                              f32x4_t (&acc)[J]) {
#pragma unroll
    for (int j = 0; j < J; ++j) acc[j] = f32x4_t{};
    auto weight = [&](int rb, int j) { return weights(s, c, aid, j, m, 16 * rb + 8 * (g & 1), rank, false); };
    auto multiply = [](const uint4& h, const uint4& w, f32x4_t& sum) {
      sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(h), as_frag(w), sum, 0, 0, 0);
    };
    auto first = [&](int rb) {
      const uint4 part = h(rb, g);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint4 w = weight(rb, j), finite = finite_of(w);
        multiply(part, g < 2 ? w : finite, acc[j]);
      }
    };
#pragma unroll 1
    for (int rb = 0; 16 * rb < rank; rb += kPairs ? 2 : 1) {
      if constexpr (!kPairs) first(rb);
      const int mine = kPairs ? rb + (g >> 1) : rb;
      const uint4 low = kPairs || g < 2 ? h(mine, 4 + (g & 1)) : uint4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int j = 0; j < J; ++j) multiply(low, finite_of(weight(mine, j)), acc[j]);
      if constexpr (kPairs) {
        first(rb);
        if (16 * rb + 16 < rank) first(rb + 1);
      }
    }
  }
};

template <int J>
__device__ __forceinline__ Cols cols_of(const Shape& s, int block, int wave) {
  constexpr int kCols = 16 * J * kExpandWaves;
  Cols c{0, 0, 0, 0};
  for (; c.part < s.n_parts - 1; ++c.part) {
    const int nb = (s.cols[c.part] + kCols - 1) / kCols;
    if (block < nb) break;
    block -= nb;
    c.col0 += s.cols[c.part];
  }
  c.width = s.cols[c.part];
  c.n0 = block * kCols + wave * 16 * J;
  return c;
}

template <int J>
unsigned col_blocks(const Shape& s) {
  unsigned n = 0;
  for (int p = 0; p < s.n_parts; ++p) n += (s.cols[p] + 16 * J * kExpandWaves - 1) / (16 * J * kExpandWaves);
  return n;
}

// One group of few rows, or a tile of 16 ordered rows of a call that has too few for runs: 64
// columns a wave.  The slices' partials are added up on the way.  A tile's adapters are dealt to
// kManyGroups work-groups, as in shrink.  64 rows of 64 adapters, 4096 columns, rank 16 (8.4 MB of
// B): 7.6 us; 777 ordered rows of 2048 columns: 7.0.
// Waves a SIMD: five for few rows, three for a tile, which bounds the registers to 96 and 168; for `wild` the compiler
// would take more (one row 7.4 us for 7.1).
constexpr int kTileJ = 4;
template <bool kFew>
__global__ __launch_bounds__(64 * kExpandWaves, kFew ? 5 : 3) void adapter_expand_tile_kernel(const Shape s) {
  constexpr int J = kTileJ;
  using O = Out<J, false>;
  __shared__ int list[kTile];
  __shared__ __align__(16) uint2 hs[128 / 16][kTile][kParts][4];  // [block of ranks][row][part][four ranks]
  const int lane = threadIdx.x & 63;
  const int m = lane & 15, g = lane >> 4;
  const Cols cols = cols_of<J>(s, blockIdx.x, wave_id());
  const bool in_place = s.base == s.out && s.base_stride == s.out_stride;
  const int64_t row0 = static_cast<int64_t>(blockIdx.y) * kTile;  // (of the order)
  int aid = 0, count = 0;
  unsigned long long todo = 1;  // adapters of the tile that are this work-group's, as their first rows
  if constexpr (kFew) {
    count = few_group(s, blockIdx.y, &aid, list);
    if (count == 0 || (aid < 0 && in_place)) return;
  } else {
    count = static_cast<int>(min<int64_t>(kTile, s.rows - row0));
    const int2 at = lane < count ? s.order[row0 + lane] : int2{0, -1};
    aid = at.y;
    if (threadIdx.x < kTile) list[lane] = at.x;
    __syncthreads();
    todo = 0;
    int n = 0;
    for_adapters(aid, (1ull << count) - 1, [&](int id, unsigned long long mine) {
      if (n++ % kManyGroups == static_cast<int>(blockIdx.z) && !(id < 0 && in_place)) todo |= mine & -mine;
    });
    if (todo == 0) return;
  }
  const bool has_col = cols.n0 + J * m < cols.width;
  const bf16_t* base = s.base + cols.col0;
  bf16_t* out = s.out + cols.col0;
  // (rows past the group's are read as its last)
  typename O::Vec bv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) bv[i] = O::base(base, s.base_stride, cols, list[min(4 * g + i, count - 1)], m);
  auto put = [&](unsigned long long mine, auto value) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (has_col && ((mine >> (4 * g + i)) & 1)) O::store(out, s.out_stride, cols, list[4 * g + i], m, value(i));
  };
  // H of the rows, formed once and only if any has an adapter: eight slices' partials asked for
  // before the first is added
  bool formed = false;
  auto form = [&] {
    const int64_t plane = s.rows * s.h_cols;
    for (int e = threadIdx.x; e < kTile * 4 * s.rank_blocks; e += 64 * kExpandWaves) {
      const int q = e & 3, row = (e >> 2) & 15, rb = e >> 6;
      if (row < count) {
        const int64_t at = kFew ? list[row] : row0 + row;
        const float4* p = reinterpret_cast<const float4*>(s.part + at * s.h_cols + (cols.part * s.rank_blocks + rb) * 16) + q;
        float4 sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i0 = 0; i0 < (kFew ? kFewSlices : kManySlices); i0 += 8) {
          if (i0 >= s.slices) break;
          float4 v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = i0 + i < s.slices ? p[(i0 + i) * plane / 4] : float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 8; ++i) sum = sum + v[i];
        }
        store_split(reinterpret_cast<bf16_t*>(hs[rb][row]), q, sum);
      }
    }
    __syncthreads();
  };
  while (todo) {
    const int lead = __ffsll(todo) - 1;
    todo &= todo - 1;
    unsigned long long mine = (1ull << count) - 1;
    if constexpr (!kFew) {
      const int id = __builtin_amdgcn_readlane(aid, lead);
      mine = __ballot(lane < count && aid == id);
      if (id < 0) {
        put(mine, [&](int i) { return bv[i]; });
        continue;
      }
    } else if (aid < 0) {
      put(mine, [&](int i) { return bv[i]; });
      return;
    }
    const int id = kFew ? aid : __builtin_amdgcn_readlane(aid, lead);
    // the first block's weights, asked for before its rank is known
    uint4 wv[J];
#pragma unroll
    for (int j = 0; j < J; ++j) wv[j] = O::weights(s, cols, id, j, m, 8 * (g & 1), 0, true);
    const int rank = rank_of(s, id);
    const float scale = s.scale ? s.scale[id] : 1.f;
    if (!formed) form();
    formed = true;
    auto load_h = [&](int rb, int at) { return reinterpret_cast<const uint4*>(hs[rb][min(m, count - 1)])[at]; };
    f32x4_t acc[J] = {};
    for (int rb = 0; 16 * rb < rank; ++rb) {
      // of H, ranks 8 (g & 1) .. of the block: high (g < 2) or middle parts, then low ones or nothing
      const uint4 first = load_h(rb, g), low = g < 2 ? load_h(rb, 4 + g) : uint4{0u, 0u, 0u, 0u};
      if (16 * rb + 16 > rank) {
#pragma unroll
        for (int j = 0; j < J; ++j) wv[j] = first_of(wv[j], rank - 16 * rb - 8 * (g & 1));
      }
      uint4 next[J];
#pragma unroll
      for (int j = 0; j < J; ++j) next[j] = O::weights(s, cols, id, j, m, 16 * (rb + 1) + 8 * (g & 1), 0, true);
      multiply_h(first, wv, acc);
      multiply_h(low, wv, acc);
#pragma unroll
      for (int j = 0; j < J; ++j) wv[j] = next[j];
    }
    if (__builtin_expect(any_wild(acc), 0)) O::template wild<false>(s, cols, id, rank, m, g, load_h, acc);
    put(mine, [&](int i) { return O::add(bv[i], acc, i, scale); });
    if constexpr (kFew) return;
  }
}

// Many rows: 64 columns a wave, a run of tiles of 16 rows one after another.  The run's H lies in
// LDS, which the four waves read instead of each fetching it (2048 rows of 28672 columns: 7 us more with its three
// parts from memory); the next tile's base is on its way while a tile is worked, and the weights of
// all kKept blocks of ranks stay in registers while the adapter stays (2048 rows of 6144 columns, rank 128: 69.5 us
// in all).  2048 rows of 28672 columns, rank 32, move 235 MB in 55 us, 4.3 TB/s; were the
// weights asked for only once the rank is known, 6 us more.  Short runs (kShortRun) have a form with room for no
// more in LDS and registers (300 rows of 8200 columns, rank 128, 38.3 us for 40.8), and of small ranks take H with
// the base, from memory (192 rows of 28672 columns, 32 mixed adapters, 48.7 us for 50.5; rank 128 39.2 for 38.3).
constexpr int kManyJ = 4;
constexpr int kManyRun = 8;  // at most
constexpr int kShortRun = 2;
// (Two blocks kept: three waves a SIMD, at most 168 registers.  For `wild` the compiler would take 176: 2048 rows of
// 28672 columns 79 us for 74 in all, not captured.)
template <int kKept, int kRun>
__global__ __launch_bounds__(64 * kExpandWaves, kKept == 2 ? 3 : 1) void adapter_expand_many_kernel(const Shape s) {
  constexpr int J = kManyJ;
  using O = Out<J, true>;
  const int lane = threadIdx.x & 63;
  const int m = lane & 15, g = lane >> 4;
  constexpr int kThreads = 64 * kExpandWaves;
  constexpr int kVecs = 2 * kParts;            // of 16 bytes in a block of ranks
  constexpr int kRowVecs = kVecs * kKept + 1;  // (16 rows' reads fall on different banks)
  __shared__ int list[16 * kRun];  // rows of the call
  constexpr bool kLds = kRun > kShortRun || kKept > 2;
  __shared__ uint4 hs[kLds ? 16 * kRun * kRowVecs : 1];
  const Cols cols = cols_of<J>(s, blockIdx.x, wave_id());
  const bool in_place = s.base == s.out && s.base_stride == s.out_stride;
  const bool has_col = cols.n0 + J * m < cols.width;
  const int64_t row0 = static_cast<int64_t>(blockIdx.y) * (16 * s.run);
  const int n_rows = static_cast<int>(min<int64_t>(16 * s.run, s.rows - row0));
  int ids[(16 * kRun + 63) / 64], rows[(16 * kRun + 63) / 64];
#pragma unroll
  for (int i = 0; i < (16 * kRun + 63) / 64; ++i) {
    const int2 at = 64 * i + lane < n_rows ? s.order[row0 + 64 * i + lane] : int2{0, -1};
    rows[i] = at.x;
    ids[i] = at.y;
  }
  // The run's H, which all waves read, in LDS; asked for together with the rows.  Rows past the last and blocks
  // past the last hold parts of the last: no result of theirs is used, or they meet weights of zero.
  const uint4* h0 = reinterpret_cast<const uint4*>(s.h + kParts * (row0 * s.h_cols + cols.part * s.rank_blocks * 16));
  constexpr int kAll = kVecs * kKept * 16 * kRun, kEach = (kAll + kThreads - 1) / kThreads;
  uint4 hv[kEach];
#pragma unroll
  for (int u = 0; u < kEach && kLds; ++u) {
    const int e = u * kThreads + threadIdx.x, r = min(e / (kVecs * kKept), n_rows - 1);
    const int v = min(e % (kVecs * kKept), kVecs * s.rank_blocks - 1);
    hv[u] = h0[static_cast<uint32_t>(r * (kVecs * s.h_cols / 16) + v)];
  }
#pragma unroll
  for (int i = 0; i < (16 * kRun + 63) / 64; ++i)
    if (wave_id() == 0 && 64 * i + lane < n_rows) list[64 * i + lane] = rows[i];
#pragma unroll
  for (int u = 0; u < kEach && kLds; ++u) {
    const int e = u * kThreads + threadIdx.x;
    if (kAll % kThreads == 0 || e < kAll) hs[e / (kVecs * kKept) * kRowVecs + e % (kVecs * kKept)] = hv[u];
  }
  __syncthreads();
  if (cols.n0 >= cols.width) return;
  // vector `at` of block rb of row r of H
  auto load_h = [&](int r, int rb, int at) {
    if constexpr (kLds) return hs[r * kRowVecs + kVecs * rb + at];
    return h0[static_cast<uint32_t>(min(r, n_rows - 1) * (kVecs * s.h_cols / 16) + kVecs * min(rb, s.rank_blocks - 1) + at)];
  };
  const bf16_t* base = s.base + cols.col0;
  bf16_t* out = s.out + cols.col0;
  struct Ahead {
    typename O::Vec base[4];
    uint4 h[kLds ? 1 : kKept], low[kLds ? 1 : kKept / 2];
  };
  auto fetch = [&](int t, Ahead& a) {
    if constexpr (!kLds) {
#pragma unroll
      for (int k = 0; k < kKept; ++k) a.h[k] = load_h(16 * t + m, k, g);
#pragma unroll
      for (int k = 0; k < kKept; k += 2) a.low[k / 2] = load_h(16 * t + m, k + (g >> 1), 4 + (g & 1));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) a.base[i] = O::base(base, s.base_stride, cols, list[min(16 * t + 4 * g + i, n_rows - 1)], m);
  };
  uint4 wv[kKept][J];
  int kept = -1, rank = 0;
  float scale = 0.f;
  auto keep = [&](int aid) {
    kept = aid;
    rank = rank_of(s, aid);
    scale = s.scale ? s.scale[aid] : 1.f;
#pragma unroll
    for (int k = 0; k < kKept; ++k)
#pragma unroll
      for (int j = 0; j < J; ++j)
        wv[k][j] = O::weights(s, cols, aid, j, m, 16 * k + 8 * (g & 1), rank, true);
    if (rank < 16 * kKept) {
#pragma unroll
      for (int k = 0; k < kKept; ++k)
#pragma unroll
        for (int j = 0; j < J; ++j) wv[k][j] = first_of(wv[k][j], rank - 16 * k - 8 * (g & 1));
    }
  };
  // Of H, a lane's ranks 8 (g & 1) .. of a block: high (g < 2) or middle parts; of two blocks, the
  // first's (g < 2) or the second's low parts.
  auto multiply = [&](int t, const Ahead& a, f32x4_t (&acc)[J]) {
    auto h_of = [&](int k) { return kLds ? load_h(16 * t + m, k, g) : a.h[kLds ? 0 : k]; };
#pragma unroll
    for (int k = 0; k < kKept; k += 2) {
      if (16 * k >= rank) break;
      uint4 w[J];  // (past the rank they are zero, and low parts are finite)
#pragma unroll
      for (int j = 0; j < J; ++j) w[j] = g < 2 ? wv[k][j] : wv[k + 1][j];
      multiply_h(kLds ? load_h(16 * t + m, k + (g >> 1), 4 + (g & 1)) : a.low[kLds ? 0 : k / 2], w, acc);
      multiply_h(h_of(k), wv[k], acc);
      if (16 * k + 16 < rank) multiply_h(h_of(k + 1), wv[k + 1], acc);
    }
    if (__builtin_expect(any_wild(acc), 0))
      O::template wild<true>(s, cols, kept, rank, m, g, [&](int rb, int at) { return load_h(16 * t + m, rb, at); }, acc);
  };
  // The usual run, whole and of one adapter, in a loop without a condition on a load or
  // store: each would make the next wait for all of them, stores included.
  const int first = __builtin_amdgcn_readfirstlane(ids[0]);
  bool same = n_rows == 16 * s.run && cols.n0 + 16 * J <= cols.width && first >= 0;
#pragma unroll
  for (int i = 0; i < (16 * kRun + 63) / 64; ++i) same &= __ballot(64 * i + lane < n_rows && ids[i] != first) == 0;
  if (same) {
    Ahead now, ahead;
    fetch(0, ahead);
    keep(first);
    for (int t = 0; t < s.run; ++t) {
      now = ahead;
      fetch(t + 1, ahead);  // (of the last tile: the last row again)
      f32x4_t acc[J] = {};
      multiply(t, now, acc);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        O::store(out, s.out_stride, cols, list[16 * t + 4 * g + i], m, O::add(now.base[i], acc, i, scale));
    }
    return;
  }
  for (int t = 0; 16 * t < n_rows; ++t) {
    const int id = __shfl(ids[t / 4], 16 * (t % 4) + m);
    Ahead now;
    fetch(t, now);
    for_adapters(id, (1ull << min(16, n_rows - 16 * t)) - 1, [&](int aid, unsigned long long mine) {
      if (aid < 0 && in_place) return;
      f32x4_t acc[J] = {};
      if (aid >= 0) {
        if (aid != kept) keep(aid);
        multiply(t, now, acc);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (has_col && ((mine >> (4 * g + i)) & 1))
          O::store(out, s.out_stride, cols, list[16 * t + 4 * g + i], m, aid < 0 ? now.base[i] : O::add(now.base[i], acc, i, scale));
    });
  }
}

template <int kKept>
void launch_expand_many(const Shape& s, const dim3& grid, hipStream_t st) {
  if (s.run <= kShortRun)
    adapter_expand_many_kernel<kKept, kShortRun><<<grid, 64 * kExpandWaves, 0, st>>>(s);
  else
    adapter_expand_many_kernel<kKept, kManyRun><<<grid, 64 * kExpandWaves, 0, st>>>(s);
}

template <class C>
unsigned h_groups(const Shape& s) {
  return (s.h_cols / 16 + C::kCols - 1) / C::kCols;
}

// Rows up to which the few-row form serves.  It reads B again for each 16 rows of an adapter,
// the many-row form orders the rows first and gains by long runs.  K 4096, few / many in us, 1 adapter and 32 mixed
// ones:
//   N 4096, rank 16:   130 rows 16.3 / 13.4, 12.5 / 27.2   256 rows 20.2 / 13.8, 14.2 / 24.9
//   N 8192, rank 32:   192 rows 25.9 / 16.0, 21.1 / 34.1   N 12288: 29.8 / 18.4, 25.9 / 36.2
//   N 28672, rank 32:   96 rows 24.2 / 18.5, 36.8 / 50.4   192 rows 42.3 / 24.7, 47.0 / 48.9
// Mixed adapters lose more by the other form than one adapter does up to these rows, and a call does not say how many of
// its adapters occur; one adapter's rows by themselves, up to here, would be better off with the many-row form.
constexpr int kNarrow = 8192;
int few_rows(const Shape& s) { return s.N <= kNarrow ? kFewRows : kFewRows / 2; }

// Many rows, but too few for runs: their expand adds the slices' partials up itself, up to so
// many blocks of 16 ranks of them for a row, a launch less; every work-group across the columns does
// it again.  Itself / by a launch, us:
//   N 4096, rank 16:   257 rows 14.0 / 16.4, 384 rows of 32 mixed adapters 25.6 / 26.9
//   N 28672, rank 32:  130 rows 24.6 / 22.3, 32 mixed adapters 62.4 / 52.2
constexpr int kTilePartials = 32;

// `rows` rows of the call from `first` on; *bytes: of the workspace they need.
Shape shape_of(const span_adapter_call& c, int64_t first, int64_t rows, size_t* bytes) {
  Shape s{};
  s.x = static_cast<const bf16_t*>(c.x) + first * c.x_stride;
  s.base = static_cast<const bf16_t*>(c.base) + first * c.base_stride;
  s.out = static_cast<bf16_t*>(c.out) + first * c.out_stride;
  s.ids = c.ids + first;
  s.a = static_cast<const bf16_t*>(c.a);
  s.b = static_cast<const bf16_t*>(c.b);
  s.scale = c.scale;
  s.ranks = c.ranks;
  s.rows = rows;
  s.x_stride = c.x_stride;
  s.base_stride = c.base_stride;
  s.out_stride = c.out_stride;
  s.K = c.in_features;
  s.R = c.max_rank;
  s.n_adapters = c.n_adapters;
  s.n_parts = c.n_parts;
  for (int p = 0; p < c.n_parts; ++p) s.N += s.cols[p] = c.part_cols[p];
  s.rank_blocks = (s.R + 15) / 16;
  s.h_cols = 16 * s.n_parts * s.rank_blocks;
  // K slices: enough work-groups for the chip, and for many rows a multiple of the XCDs' number where K
  // allows it and partials are not too many (10000 rows: K 4096, 16 columns of H 90 us with eight, 107
  // with one; K 2048, 128 columns 160 and 131)
  const bool few = rows <= few_rows(s);
  const int unit = 32 * (few ? FewShrink::kSteps * FewShrink::kWaves : ManyShrink::kSteps * ManyShrink::kWaves);
  const int64_t most = (s.K + unit - 1) / unit;
  const int64_t tiles = (rows + 16 * kManyTiles - 1) / (16 * kManyTiles) * h_groups<ManyShrink>(s);
  const int64_t want = few ? kFewSlices : (tiles >= 256 ? 1 : tiles > 16 ? kXcds : kManySlices);
  const int64_t n = std::max<int64_t>(1, std::min(want, most));
  s.k_slice = static_cast<int>(((s.K + n - 1) / n + unit - 1) / unit * unit);
  s.slices = (s.K + s.k_slice - 1) / s.k_slice;
  // runs as long as leave three work-groups for a CU
  s.run = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kManyRun, (rows + 15) / 16 * col_blocks<kManyJ>(s) / 768)));
  const bool tile = few || (s.run == 1 && s.N <= kNarrow && s.slices * s.rank_blocks <= kTilePartials);
  const int64_t plane = rows * s.h_cols, planes = tile || s.slices > 1 ? s.slices : 0;
  s.part = static_cast<float*>(c.workspace);
  s.h = tile ? nullptr : reinterpret_cast<bf16_t*>(s.part + planes * plane);
  const int64_t sums = planes * plane * sizeof(float) + (tile ? 0 : kParts * plane * sizeof(bf16_t));
  s.order = few ? nullptr : reinterpret_cast<int2*>(static_cast<char*>(c.workspace) + sums);
  *bytes = sums + (few ? 0 : rows * sizeof(int2));
  return s;
}

}  // namespace

// Rows worked at once: grids stay below 2^32 threads (expand: at most 2^20 / 256 + 4 work-groups of
// 256 threads across, and down 2^16 / 128, as runs are whole where there are that many).
constexpr int64_t kRowsAtOnce = int64_t{1} << 16;

size_t adapter_workspace_bytes(const span_adapter_call& a) {
  size_t most = 0;
  // the last rows of a long call may be few, and split K further
  for (const int64_t n : {std::min(a.n_rows, kRowsAtOnce), a.n_rows % kRowsAtOnce}) {
    size_t bytes = 0;
    (void)shape_of(a, 0, n, &bytes);
    most = std::max(most, bytes);
  }
  return most;
}

size_t adapter_workspace_up_to(const span_adapter_call& a) {
  // the most rows of either form, and of each number of K slices, which falls with the tiles
  size_t most = adapter_workspace_bytes(a), bytes = 0;
  const auto of = [&](int64_t n) {
    (void)shape_of(a, 0, n, &bytes);
    most = std::max(most, bytes);
  };
  const int64_t n = std::min(a.n_rows, kRowsAtOnce);
  for (const int64_t few : {kFewRows / 2, kFewRows}) of(std::min<int64_t>(n, few));
  for (int64_t rows = 16 * kManyTiles; rows < n && rows <= 256 * 16 * kManyTiles; rows += 16 * kManyTiles) of(rows);
  return most;
}

hipError_t launch_adapter_apply(const span_adapter_call& a, hipStream_t st) {
  for (int64_t first = 0; first < a.n_rows; first += kRowsAtOnce) {
    size_t bytes = 0;
    const Shape s = shape_of(a, first, std::min(kRowsAtOnce, a.n_rows - first), &bytes);
    hipError_t e = hipSuccess;
    if (s.rows <= few_rows(s)) {
      const unsigned rows = static_cast<unsigned>(s.rows);
      adapter_shrink_kernel<true, FewShrink><<<dim3(s.slices * h_groups<FewShrink>(s), rows), 64 * FewShrink::kWaves, 0, st>>>(s);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      adapter_expand_tile_kernel<true><<<dim3(col_blocks<kTileJ>(s), rows), 64 * kExpandWaves, 0, st>>>(s);
    } else {
      const unsigned tiles = static_cast<unsigned>((s.rows + 16 * kManyTiles - 1) / (16 * kManyTiles));
      adapter_order_kernel<<<1, kOrderThreads, 0, st>>>(s);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      adapter_shrink_kernel<false, ManyShrink><<<dim3((tiles * s.slices + kXcds - 1) / kXcds * kXcds * h_groups<ManyShrink>(s), 1, kManyGroups), 64 * ManyShrink::kWaves, 0, st>>>(s);
      e = hipGetLastError();
      if (e == hipSuccess && s.h && s.slices > 1) {
        adapter_finish_kernel<<<static_cast<unsigned>((s.rows * s.h_cols / 4 + 255) / 256), 256, 0, st>>>(s);
        e = hipGetLastError();
      }
      if (e != hipSuccess) return e;
      const unsigned runs = static_cast<unsigned>((s.rows + 16 * s.run - 1) / (16 * s.run));
      const dim3 grid(col_blocks<kManyJ>(s), runs);
      if (s.h && s.rank_blocks <= 2)
        launch_expand_many<2>(s, grid, st);
      else if (s.h && s.rank_blocks <= 4)
        launch_expand_many<4>(s, grid, st);
      else if (s.h)
        launch_expand_many<8>(s, grid, st);
      else
        adapter_expand_tile_kernel<false><<<dim3(col_blocks<kTileJ>(s), runs, kManyGroups), 64 * kExpandWaves, 0, st>>>(s);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace spanq
