// Matrix products on CUDA cores: fp32, and every layout that TMA cannot address.
//
// A block of 128 threads forms a 64 x 64 tile of C, 8 x 4 of it per thread, from 16 values of k at a time, staged in shared memory as fp32 and loaded
// one step ahead.  A thread's rows and columns are two runs, one in each half of the tile, so that its operands are wide loads without bank
// conflicts, and so that in a gated product (columns [0, 32) of the tile are those of B_0, the others the same columns of B_1) it holds g and u of
// the same elements.  Sums are fp32, by multiply-adds of two rows at a time.
//
// Where the tiles leave multiprocessors idle, the blocks of a cluster each take a part of k; the parts are added in the order of the ranks, so the sum is
// the same in every run.
//
// What bounds it: waits for shared memory and the rounds of blocks.  1024 x 1024 x 2816, both products 588 us, 30 TFLOP/s of 74; with tiles of 128 x 128, 8 x 8 a
// thread, 650 us (352 blocks of the gated product where 296 fit at once), with 32 values of k a step 621.  389 x 250 x 1021, backward, 74 us on the
// device: starts, meetings and ends of short sums.
#include <cooperative_groups.h>
#include <cuda_fp8.h>

#include <algorithm>

#include "f32x2.cuh"
#include "product_ops.h"

namespace muon {
namespace {

namespace cg = cooperative_groups;
constexpr int kMaxSplit = 8, kTile = 64, kHalf = kTile / 2, kThreads = 128, kBlocks = 4;       // kBlocks: on a multiprocessor; they cover one another's waits
constexpr int kColumns = 4, kH = kColumns / 2;           // of C per thread: 8 rows of kColumns, kH of them in each half of the tile
constexpr int kStep = 16, kLoads = kTile * kStep / kThreads;     // values of k; elements of an operand that a thread loads in a step
constexpr int kPitch = kTile + 4;                        // of a staged row: eight neighbouring k of four rows lie in 32 banks

struct SimtArgs {
  Product p[kMaxProducts];
  int32_t tile_begin[kMaxProducts];
  int32_t count, split;
};

template <int TYPE>
__device__ __forceinline__ float value_at(const void* p) {
  if constexpr (TYPE == kTypeFp32) return __ldg(static_cast<const float*>(p));
  if constexpr (TYPE == kTypeBf16) return __bfloat162float(*static_cast<const __nv_bfloat16*>(p));
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(__ldg(static_cast<const uint8_t*>(p)), __NV_E4M3)));
}
template <int TYPE> constexpr int kSizeOf = TYPE == kTypeFp32 ? 4 : TYPE == kTypeBf16 ? 2 : 1;

// Element (row, col) of a matrix as it lies in memory.
__device__ __forceinline__ float element_of(const Operand& o, int64_t row, int64_t col) {
  const char* p = static_cast<const char*>(o.data);
  const int64_t at = row * o.ld + col;
  if (o.type == kTypeFp32) return value_at<kTypeFp32>(p + at * 4);
  if (o.type == kTypeBf16) return value_at<kTypeBf16>(p + at * 2);
  return value_at<kTypeE4m3>(p + at) * scale_of(__ldg(o.scales + row / o.block_rows * o.lds + (col >> 7)));
}

// What a thread loads of an operand in every step: along the memory's rows, eight values of k (a sector of fp32) or all rows of the tile.
template <int TYPE>
struct Loader {
  static constexpr int kGroups = kStep / 8, kRowsApart = kThreads / 8, kApart = kThreads / kTile;
  // of the two halves of the tile, which are of one matrix or of two; in registers, for the launch's arguments are far away
  const char *lo, *hi;
  int64_t ld_lo, ld_hi;
  const Operand* blocks;        // 8 bits: the scales (one matrix)
  bool mn;
  int row_lo, row_hi, rows;     // of the operand: the first element's in each half of the tile
  int k;                        // of the first element, from the step's beginning on
  __device__ __forceinline__ void init(const Operand& first_half, const Operand& second_half, bool halves, int first, int rows_) {
    const Operand& second = halves ? second_half : first_half;
    lo = static_cast<const char*>(first_half.data);
    hi = static_cast<const char*>(second.data);
    ld_lo = first_half.ld;
    ld_hi = second.ld;
    blocks = &first_half;
    mn = first_half.mn_major != 0;
    rows = rows_;
    k = mn ? int(threadIdx.x) / kTile : int(threadIdx.x) % 8;
    row_lo = first + (mn ? int(threadIdx.x) % kTile : int(threadIdx.x) / 8);
    row_hi = halves ? row_lo : row_lo + kHalf;
  }
  __device__ __forceinline__ void load(int k0, int kdim, float (&v)[kLoads]) const {
    if (mn) {
      const bool in = row_lo < rows;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int kk = k0 + k + i * kApart;
        v[i] = 0.f;
        if (in && kk < kdim) v[i] = one(lo, ld_lo, kk, row_lo);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int group = i / kGroups, kk = k0 + k + 8 * (i % kGroups);
        const bool first = group * kRowsApart < kHalf;
        const int r = first ? row_lo + group * kRowsApart : row_hi + group * kRowsApart - kHalf;
        v[i] = 0.f;
        if (r < rows && kk < kdim) v[i] = one(first ? lo : hi, first ? ld_lo : ld_hi, r, kk);
      }
    }
  }
  __device__ __forceinline__ float one(const char* base, int64_t ld, int64_t r, int c) const {
    const float x = value_at<TYPE>(base + (r * ld + c) * kSizeOf<TYPE>);
    if constexpr (TYPE == kTypeE4m3) return x * scale_of(__ldg(blocks->scales + (blocks->block_rows == 1 ? r : r >> 7) * blocks->lds + (c >> 7)));
    return x;
  }
  __device__ __forceinline__ void stage(float (*s)[kPitch], const float (&v)[kLoads]) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (mn) s[int(threadIdx.x) / kTile + i * kApart][int(threadIdx.x) % kTile] = v[i];
      else s[int(threadIdx.x) % 8 + 8 * (i % kGroups)][int(threadIdx.x) / 8 + i / kGroups * kRowsApart] = v[i];
    }
  }
};

__device__ __forceinline__ void put(void* base, int type, int64_t at, float v) {
  if (type == kTypeFp32) static_cast<float*>(base)[at] = v;
  else static_cast<__nv_bfloat16*>(base)[at] = __float2bfloat16_rn(v);
}

// Two sums of a row of the tile, half a tile apart: g and u of a column, or two columns.
__device__ __forceinline__ void finish(const Product& p, const Activation& f, int64_t row, int n0, int c, float first, float second) {
  const Epilogue& e = p.e;
  if (row >= p.m) return;
  if (e.kind == kGated) {
    const int64_t col = n0 + c;
    if (col >= p.n) return;
    float a, slope;
    activate<false>(f, first, &a, &slope);
    put(e.c, e.type, row * e.ldc + col, a * second);
    if (e.gate) {
      put(e.gate, e.gate_up_type, row * e.ld_gate + col, first);
      put(e.up, e.gate_up_type, row * e.ld_up + col, second);
    }
    return;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t col = n0 + c + h * kHalf;
    if (col >= p.n) continue;
    const float v = h ? second : first;
    if (e.kind == kPlain) {
      put(e.c, e.type, row * e.ldc + col, v);
      continue;
    }
    const float g = element_of(e.in_gate, row, col), u = element_of(e.in_up, row, col);
    float a, slope;
    activate<false>(f, g, &a, &slope);
    put(e.gate, e.type, row * e.ld_gate + col, v * u * slope);
    put(e.up, e.type, row * e.ld_up + col, v * a);
    put(e.c, e.type, row * e.ldc + col, a * u);
  }
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads, kBlocks) product_kernel(const __grid_constant__ SimtArgs L) {
  __shared__ __align__(16) float stages[4][kStep][kPitch];    // two places for A, two for B
  const int block = int(blockIdx.x) / L.split, rank = int(blockIdx.x) % L.split;
  int which = 0;
  for (int i = 1; i < L.count; ++i)
    if (block >= L.tile_begin[i]) which = i;
  const Product& p = L.p[which];
  const bool gated = p.e.kind == kGated;
  const int tiles_m = (p.m + kTile - 1) / kTile, tile = block - L.tile_begin[which];
  const int m0 = tile % tiles_m * kTile, n0 = tile / tiles_m * (gated ? kHalf : kTile);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  uint64_t acc[4][kColumns] = {};                             // two rows each: 0, 1 and 2, 3 of the run in either half
  const int steps = (p.k + kStep - 1) / kStep, total = steps * p.segments;
  const int begin = int(int64_t(total) * rank / L.split), end = int(int64_t(total) * (rank + 1) / L.split);
  Loader<TYPE> la, lb;
  float va[kLoads], vb[kLoads];
  int segment = -1;
  auto load = [&](int t) {
    const int s = t >= steps ? 1 : 0;
    if (s != segment) {
      la.init(p.a[s], p.a[s], false, m0, p.m);
      lb.init(p.b[s], p.b[1], gated, n0, p.n);
      segment = s;
    }
    la.load((t - s * steps) * kStep, p.k, va);
    lb.load((t - s * steps) * kStep, p.k, vb);
  };
  auto keep = [&](int t) {
    la.stage(stages[t & 1], va);
    lb.stage(stages[2 + (t & 1)], vb);
  };
  if (end > begin) {
    load(begin);
    keep(begin);
  }
  __syncthreads();
  for (int t = begin; t < end; ++t) {
    if (t + 1 < end) load(t + 1);
    // the operands of a value of k are read while the one before is multiplied
    uint64_t a[2][4];
    float b[2][kColumns];
    auto fetch = [&](int k, int to) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(&stages[t & 1][k][half * kHalf + ty * 4]);
        a[to][half * 2] = x.x;
        a[to][half * 2 + 1] = x.y;
        const float* pb = &stages[2 + (t & 1)][k][half * kHalf + tx * kH];
        const float2 y = *reinterpret_cast<const float2*>(pb);
        b[to][half * 2] = y.x;
        b[to][half * 2 + 1] = y.y;
      }
    };
    fetch(0, 0);
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      if (k + 1 < kStep) fetch(k + 1, (k + 1) & 1);
#pragma unroll
      for (int j = 0; j < kColumns; ++j) {
        const uint64_t bb = twice(b[k & 1][j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = fma2(a[k & 1][i], bb, acc[i][j]);
      }
    }
    if (t + 1 < end) keep(t + 1);       // the other place, which every thread left before the last meeting
    __syncthreads();
  }
  const Activation f = activation_of(p.e.activation);
  auto row_of = [&](int i) { return (i / 2) * kHalf + ty * 4 + (i % 2) * 2; };      // the first of a pair's rows
  if (L.split > 1) {
    constexpr int kRow = kTile + 1;
    static_assert(kTile * kRow <= 4 * kStep * kPitch, "the sums take the place of the operands");
    float* sums = &stages[0][0][0];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kColumns; ++j) {
        const float2 pair = both(acc[i][j]);
        float* to = sums + row_of(i) * kRow + (j / kH) * kHalf + tx * kH + j % kH;
        to[0] = pair.x;
        to[kRow] = pair.y;
      }
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
#pragma unroll 2
    for (int i = rank * kThreads + int(threadIdx.x); i < kTile * kHalf; i += L.split * kThreads) {
      const int r = i / kHalf, c = i % kHalf;
      float first[kMaxSplit], second[kMaxSplit];
#pragma unroll
      for (int q = 0; q < kMaxSplit; ++q)
        if (q < L.split) {
          const float* from = cl.map_shared_rank(sums, unsigned(q)) + r * kRow + c;
          first[q] = from[0];
          second[q] = from[kHalf];
        }
      float x = first[0], y = second[0];
#pragma unroll
      for (int q = 1; q < kMaxSplit; ++q)
        if (q < L.split) {
          x += first[q];
          y += second[q];
        }
      finish(p, f, m0 + r, n0, c, x, y);
    }
    cl.sync();                        // a block's shared memory stays until its peers have read it
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < kH; ++j) {
      const float2 first = both(acc[i][j]), second = both(acc[i][kH + j]);
      finish(p, f, m0 + row_of(i), n0, tx * kH + j, first.x, second.x);
      finish(p, f, m0 + row_of(i) + 1, n0, tx * kH + j, first.y, second.y);
    }
}

template <int TYPE>
int launch(const SimtArgs& L, int64_t tiles, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(tiles * L.split), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(L.split);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, product_kernel<TYPE>, L) == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

}  // namespace

int launch_products_simt(const Product* list, int count, int siblings, int sms, cudaStream_t st) {
  SimtArgs L = {};
  int64_t tiles = 0, most = 0, steps = INT64_MAX;      // of all products, of one of them; of the shortest
  for (int i = 0; i < count; ++i) {
    const Product& p = list[i];
    if (p.m == 0 || p.n == 0) continue;
    const int64_t wide = p.e.kind == kGated ? kHalf : kTile, n = (int64_t(p.m) + kTile - 1) / kTile * ((p.n + wide - 1) / wide);
    L.p[L.count] = p;
    if (tiles > INT32_MAX) return MUON_ERR_UNSUPPORTED;
    L.tile_begin[L.count++] = int32_t(tiles);
    tiles += n;
    most = std::max(most, n);
    steps = std::min<int64_t>(steps, (int64_t(p.k) + kStep - 1) / kStep * p.segments);
  }
  if (L.count == 0) return 0;
  // A part of k is worth a block from four steps on.  `siblings` decides, not how many of them are in this launch: a gradient is the same, bit for bit,
  // whichever others are wanted.
  L.split = int(std::max<int64_t>(1, std::min<int64_t>({kMaxSplit, 3 * int64_t(sms) / (most * siblings), steps / 4})));
  if (tiles * L.split > INT32_MAX) return MUON_ERR_UNSUPPORTED;
  switch (list[0].a[0].type) {
    case kTypeFp32: return launch<kTypeFp32>(L, tiles, st);
    case kTypeBf16: return launch<kTypeBf16>(L, tiles, st);
    default: return launch<kTypeE4m3>(L, tiles, st);
  }
}

}  // namespace muon
