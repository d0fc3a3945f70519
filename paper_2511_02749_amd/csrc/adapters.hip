// Low-rank adapters of many requests beside a shared projection:
//
//   out[i] = base[i] + scale[a] (x[i] A[a]^T) B[a]^T,   a = ids[i], rows without one copied
//
// in two launches.  Shrink: H = x A^T, sums of K products in fp32 split over the work-group's
// waves (and over work-groups when there are few row tiles), partials in the workspace.
// Expand: the partials summed in slice order, the product with B, scale and base added,
// rounded once.
//
// Rows come in tiles of 16 in the caller's order, whatever their adapters: a tile is worked
// once for each adapter that occurs in it (the group of its first row, the leader), and
// only that group's rows are written.  So nothing is sorted, ids stay on the device and may
// change between replays of a captured call.  The few-row form puts the groups of a tile on the grid
// (a decode step has up to 16 adapters in a tile, all independent), the many-row form walks
// them (a prefilled tile mostly has one).
//
// Matrix instructions 16x16x32: the weights are the A operand, the rows the B operand, so
// that a lane ends with four consecutive columns of one row.  H goes into the second product
// as two bf16 numbers, high and low part (16 significant bits), side by side in the 32 deep
// reduction over the same 16 weights, which costs nothing: the instruction is 32 deep and a
// block of ranks 16.
//
// Bound: HBM (x, base and out for many rows, A and B for few); 2 R (K P + N) operations a row.
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

constexpr int kTile = 16;     // rows of a tile
constexpr int kShrinkWaves = 8;
constexpr int kGroupCols = 4;  // 16-column tiles of H that one shrink work-group forms
constexpr int kFewRows = 256;  // up to here the groups of a tile are on the grid

struct Shape {
  const bf16_t* x;
  const bf16_t* base;
  bf16_t* out;
  const int32_t* ids;
  const bf16_t* a;
  const bf16_t* b;
  const float* scale;
  const int32_t* ranks;
  float* h;  // [slices][rows][h_cols]
  int64_t rows, x_stride, base_stride, out_stride;
  int K, R, n_adapters, n_parts;
  int N;         // columns of all parts
  int cols[4];   // columns of each part
  int rank_blocks, h_cols;  // ceil(R / 16); 16 * n_parts * rank_blocks
  int slices, k_slice;
};

// The adapter of tile row `lane & 15`, -1 for none.
__device__ __forceinline__ int tile_id(const Shape& s, int64_t row0, int lane) {
  const int64_t row = row0 + (lane & 15);
  const int id = row < s.rows ? s.ids[row] : -1;
  return id >= 0 && id < s.n_adapters ? id : -1;
}

__device__ __forceinline__ int rank_of(const Shape& s, int id) {
  return s.ranks ? max(0, min(s.ranks[id], s.R)) : s.R;
}

// Groups of a tile: f(adapter, rows of the group as a mask) for the group that row j leads
// (j >= 0) or for every group (j < 0).  Wave-uniform.
template <class F>
__device__ __forceinline__ void for_groups(int id, unsigned live, int j, F f) {
  unsigned left = live;
  while (left) {
    const int first = j < 0 ? __ffs(left) - 1 : j;
    if (!((live >> first) & 1)) return;
    const int aid = __builtin_amdgcn_readlane(id, first);
    const unsigned mine = static_cast<unsigned>(__ballot(id == aid)) & live;
    if (j >= 0 && (mine & ((1u << j) - 1))) return;  // another row leads
    f(aid, mine);
    if (j >= 0) return;
    left &= ~mine;
  }
}

__device__ __forceinline__ bf16x8_t as_frag(const uint4& v) { return __builtin_bit_cast(bf16x8_t, v); }

// H partials of one tile, one slice of K and kGroupCols column tiles.
__global__ __launch_bounds__(64 * kShrinkWaves) void adapter_shrink_kernel(const Shape s, bool few) {
  __shared__ float4 red[kShrinkWaves][kGroupCols][kTile][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col_groups = (s.h_cols / 16 + kGroupCols - 1) / kGroupCols;
  const int slice = blockIdx.x / col_groups, ct0 = (blockIdx.x % col_groups) * kGroupCols;
  const int n_ct = min(kGroupCols, s.h_cols / 16 - ct0);
  const int64_t row0 = static_cast<int64_t>(blockIdx.y) * kTile;
  const int n_rows = static_cast<int>(min<int64_t>(kTile, s.rows - row0));
  const int id = tile_id(s, row0, lane);
  const int sub = s.k_slice / kShrinkWaves;  // a multiple of 64
  const int k0 = slice * s.k_slice + wave * sub;
  const int k1 = min(s.K, k0 + sub);
  const int m = lane & 15, g = lane >> 4;
  for_groups(id, (1u << n_rows) - 1, few ? static_cast<int>(blockIdx.z) : -1, [&](int aid, unsigned mine) {
    if (aid < 0) return;
    const int rank = rank_of(s, aid);
    const bool has_row = (mine >> m) & 1;
    const bf16_t* xp = s.x + (row0 + m) * s.x_stride;
    const bf16_t* ap[kGroupCols];
    bool has_w[kGroupCols];
#pragma unroll
    for (int c = 0; c < kGroupCols; ++c) {
      const int ct = ct0 + c, p = ct / s.rank_blocks, r = (ct - p * s.rank_blocks) * 16 + m;
      has_w[c] = c < n_ct && r < rank;
      ap[c] = s.a + ((static_cast<int64_t>(aid) * s.n_parts + p) * s.R + r) * s.K;
    }
    f32x4_t acc[kGroupCols] = {};
    for (int k = k0; k < k1; k += 64) {
      // lane group g covers k + 16 g .. + 15: the same order in both operands
      uint4 xv[2], wv[kGroupCols][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int kk = k + 16 * g + 8 * t;
        xv[t] = uint4{0u, 0u, 0u, 0u};
        if (has_row && kk < k1) xv[t] = *reinterpret_cast<const uint4*>(xp + kk);
#pragma unroll
        for (int c = 0; c < kGroupCols; ++c) {
          wv[c][t] = uint4{0u, 0u, 0u, 0u};
          if (has_w[c] && kk < k1) wv[c][t] = *reinterpret_cast<const uint4*>(ap[c] + kk);
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < kGroupCols; ++c)
          acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(wv[c][t]), as_frag(xv[t]), acc[c], 0, 0, 0);
    }
#pragma unroll
    for (int c = 0; c < kGroupCols; ++c)
      if (c < n_ct) red[wave][c][m][g] = __builtin_bit_cast(float4, acc[c]);
    __syncthreads();
    for (int e = threadIdx.x; e < n_ct * kTile * 4; e += 64 * kShrinkWaves) {
      const int q = e & 3, row = (e >> 2) & 15, c = e >> 6;
      if ((mine >> row) & 1) {
        float4 sum = red[0][c][row][q];
#pragma unroll
        for (int w = 1; w < kShrinkWaves; ++w) {
          const float4 v = red[w][c][row][q];
          sum.x += v.x;
          sum.y += v.y;
          sum.z += v.z;
          sum.w += v.w;
        }
        *reinterpret_cast<float4*>(s.h + (static_cast<int64_t>(slice) * s.rows + row0 + row) * s.h_cols +
                                   (ct0 + c) * 16 + 4 * q) = sum;
      }
    }
    __syncthreads();
  });
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
constexpr int kWaveCols = 64;

// Columns [256 b, 256 b + 256) of one part for one tile of rows (few) or `tiles` tiles.
__global__ __launch_bounds__(64 * kExpandWaves) void adapter_expand_kernel(const Shape s, bool few, int tiles) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m = lane & 15, g = lane >> 4;
  int block = blockIdx.x, part = 0, col0 = 0;
  for (; part < s.n_parts - 1; ++part) {
    const int nb = (s.cols[part] + kExpandWaves * kWaveCols - 1) / (kExpandWaves * kWaveCols);
    if (block < nb) break;
    block -= nb;
    col0 += s.cols[part];
  }
  const int width = s.cols[part];
  const int n0 = (block * kExpandWaves + wave) * kWaveCols;  // in the part
  if (n0 >= width) return;
  const bool in_place = s.base == s.out && s.base_stride == s.out_stride;
  for (int t = 0; t < tiles; ++t) {
    const int64_t row0 = (static_cast<int64_t>(blockIdx.y) * tiles + t) * kTile;
    if (row0 >= s.rows) break;
    const int n_rows = static_cast<int>(min<int64_t>(kTile, s.rows - row0));
    const int id = tile_id(s, row0, lane);
    const int64_t row = row0 + m;
    for_groups(id, (1u << n_rows) - 1, few ? static_cast<int>(blockIdx.z) : -1, [&](int aid, unsigned mine) {
      const bool has_row = (mine >> m) & 1;
      const int n = n0 + 16 * g;  // the lane's 16 columns of row m
      if (aid < 0 && in_place) return;
      uint4 bv[2] = {};
      const bf16_t* bp = s.base + row * s.base_stride + col0 + n;
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (has_row && n + 8 * u < width) bv[u] = reinterpret_cast<const uint4*>(bp)[u];
      f32x4_t acc[4] = {};
      float scale = 0.f;
      if (aid >= 0) {
        scale = s.scale ? s.scale[aid] : 1.f;
        const int rank = rank_of(s, aid);
        const float* hp = s.h + row * s.h_cols + part * s.rank_blocks * 16;
        const int64_t plane = s.rows * s.h_cols;
        for (int rb = 0; 16 * rb < rank; ++rb) {
          const int r0 = 16 * rb + 8 * (g & 1);
          const int n_r = min(8, rank - r0);
          float h[8] = {};
          if (has_row && n_r > 0) {
            for (int sl = 0; sl < s.slices; ++sl) {
              const float4* p4 = reinterpret_cast<const float4*>(hp + sl * plane + r0);
              const float4 u = p4[0], v = p4[1];
              h[0] += u.x;
              h[1] += u.y;
              h[2] += u.z;
              h[3] += u.w;
              h[4] += v.x;
              h[5] += v.y;
              h[6] += v.z;
              h[7] += v.w;
            }
          }
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = pack_bf16x2(h[2 * i], h[2 * i + 1]);
            if (g >= 2) {  // the low parts; none of a value that is not finite
              const float l0 = h[2 * i] - lo_bf16(w[i]), l1 = h[2 * i + 1] - hi_bf16(w[i]);
              w[i] = pack_bf16x2(isfinite(l0) ? l0 : 0.f, isfinite(l1) ? l1 : 0.f);
            }
          }
          const uint4 hv = first_of(uint4{w[0], w[1], w[2], w[3]}, n_r);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            // tile j's row m is column 16 (m / 4) + 4 j + m % 4: a lane's four results of
            // four tiles are 16 consecutive columns
            const int col = n0 + 16 * (m >> 2) + 4 * j + (m & 3);
            uint4 wv = uint4{0u, 0u, 0u, 0u};
            if (col < width && n_r > 0)
              wv = first_of(*reinterpret_cast<const uint4*>(
                                s.b + (static_cast<int64_t>(aid) * s.N + col0 + col) * s.R + r0), n_r);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(wv), as_frag(hv), acc[j], 0, 0, 0);
          }
        }
      }
      if (!has_row) return;
      bf16_t* op = s.out + row * s.out_stride + col0 + n;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (n + 8 * u >= width) break;
        if (aid < 0) {
          reinterpret_cast<uint4*>(op)[u] = bv[u];
          continue;
        }
        const uint32_t w[4] = {bv[u].x, bv[u].y, bv[u].z, bv[u].w};
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4_t& c = acc[2 * u + i / 2];
          o[i] = pack_bf16x2(fmaf(scale, c[2 * (i & 1)], lo_bf16(w[i])), fmaf(scale, c[2 * (i & 1) + 1], hi_bf16(w[i])));
        }
        reinterpret_cast<uint4*>(op)[u] = uint4{o[0], o[1], o[2], o[3]};
      }
    });
  }
}

Shape shape_of(const span_adapter_call& c, int64_t first, int64_t rows) {
  Shape s{};
  s.x = static_cast<const bf16_t*>(c.x) + first * c.x_stride;
  s.base = static_cast<const bf16_t*>(c.base) + first * c.base_stride;
  s.out = static_cast<bf16_t*>(c.out) + first * c.out_stride;
  s.ids = c.ids + first;
  s.a = static_cast<const bf16_t*>(c.a);
  s.b = static_cast<const bf16_t*>(c.b);
  s.scale = c.scale;
  s.ranks = c.ranks;
  s.h = static_cast<float*>(c.workspace);
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
  // K slices: few rows want more work-groups than there are tiles, many rows fill the chip by themselves.
  const int64_t tiles = (s.rows + kTile - 1) / kTile;
  const int64_t want = s.rows <= kFewRows ? 16 : 256 / std::max<int64_t>(1, tiles);
  const int unit = 64 * kShrinkWaves;
  const int most = (s.K + unit - 1) / unit;
  const int n = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(want, most)));
  s.k_slice = ((s.K + n - 1) / n + unit - 1) / unit * unit;
  s.slices = (s.K + s.k_slice - 1) / s.k_slice;
  return s;
}

}  // namespace

// Rows worked at once: grids stay below 2^32 threads (kMaxCols columns at 256 a work-group
// of 256, four row tiles each).
constexpr int64_t kRowsAtOnce = int64_t{1} << 17;

size_t adapter_workspace_bytes(const span_adapter_call& a) {
  size_t most = 0;
  // the last rows of a long call may be few, and split K further
  for (const int64_t n : {std::min(a.n_rows, kRowsAtOnce), a.n_rows % kRowsAtOnce}) {
    const Shape s = shape_of(a, 0, n);
    most = std::max(most, static_cast<size_t>(s.slices) * n * s.h_cols * sizeof(float));
  }
  return most;
}

hipError_t launch_adapter_apply(const span_adapter_call& a, hipStream_t st) {
  for (int64_t first = 0; first < a.n_rows; first += kRowsAtOnce) {
    const Shape s = shape_of(a, first, std::min(kRowsAtOnce, a.n_rows - first));
    const bool few = s.rows <= kFewRows;
    const unsigned tiles = static_cast<unsigned>((s.rows + kTile - 1) / kTile);
    const unsigned groups = few ? static_cast<unsigned>(std::min<int64_t>(kTile, s.rows)) : 1;
    const int col_groups = (s.h_cols / 16 + kGroupCols - 1) / kGroupCols;
    adapter_shrink_kernel<<<dim3(s.slices * col_groups, tiles, groups), 64 * kShrinkWaves, 0, st>>>(s, few);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    unsigned blocks = 0;
    for (int p = 0; p < s.n_parts; ++p)
      blocks += (s.cols[p] + kExpandWaves * kWaveCols - 1) / (kExpandWaves * kWaveCols);
    const unsigned per = few ? 1 : 4;
    adapter_expand_kernel<<<dim3(blocks, (tiles + per - 1) / per, groups), 64 * kExpandWaves, 0, st>>>(s, few, per);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace spanq
