// Matrix products on CUDA cores: fp32, and every layout that TMA cannot address.
//
// A block of 256 threads forms a TILE x TILE tile of C, R x R of it per thread (R = TILE / 16), from 16 or 32 values of k at a time, staged in shared
// memory as fp32 and loaded one step ahead.  A thread's rows and columns are two runs, one in each half of the tile, so that its operands are
// two wide loads without bank conflicts, and so that in a gated product (columns [0, TILE/2) of the tile are those of B_0, the others
// the same columns of B_1) it holds g and u of the same elements.  Sums are fp32, by two-wide multiply-adds.
//
// Where 128 x 128 tiles would leave multiprocessors idle, the tiles are 64 x 64 and the blocks of a cluster each take a part of k; the parts are added
// in the order of the ranks, so the sum is the same in every run.
#include <cooperative_groups.h>
#include <cuda_fp8.h>

#include <algorithm>

#include "f32x2.cuh"
#include "product_ops.h"

namespace muon {
namespace {

namespace cg = cooperative_groups;
constexpr int kThreads = 256, kMaxSplit = 8;
// Values of k in a step.  The small tiles are latency-bound: twice as many in flight (32 instead of 16) halve the number of waits.
template <int TILE> constexpr int kStep = TILE == 64 ? 32 : 16;
template <int TILE> constexpr int kPitch = TILE == 64 ? 66 : 132;      // of a staged row: neighbouring k in other banks, rows aligned for the wide loads

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

// What a thread loads of an operand in every step.  Threads run along the memory's rows.
template <int TILE, int TYPE>
struct Loader {
  static constexpr int kStepK = kStep<TILE>, kLoads = TILE * kStepK / kThreads, kRowsApart = kThreads / kStepK;
  const Operand *lo, *hi;       // hi: of the second half of the tile, which is another matrix or the same
  bool mn;
  int row_lo, row_hi, rows;     // of the operand: the first element's in each half of the tile
  int k;                        // of the first element, from the step's beginning on
  __device__ __forceinline__ void init(const Operand& first_half, const Operand& second_half, bool halves, int first, int rows_) {
    lo = &first_half;
    hi = halves ? &second_half : &first_half;
    mn = lo->mn_major != 0;
    rows = rows_;
    k = mn ? int(threadIdx.x) / TILE : int(threadIdx.x) % kStepK;
    row_lo = first + (mn ? int(threadIdx.x) % TILE : int(threadIdx.x) / kStepK);
    row_hi = halves ? row_lo : row_lo + TILE / 2;
  }
  __device__ __forceinline__ void load(int k0, int kdim, float (&v)[kLoads]) const {
    if (mn) {                   // slot i is kThreads / TILE values of k further
      const bool in = row_lo < rows;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int kk = k0 + k + i * (kThreads / TILE);
        v[i] = 0.f;
        if (in && kk < kdim) v[i] = one(*lo, kk, row_lo);
      }
    } else {                    // slot i is kRowsApart rows further
      const bool in = k0 + k < kdim;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = (i < kLoads / 2 ? row_lo : row_hi) + (i % (kLoads / 2)) * kRowsApart;
        v[i] = 0.f;
        if (in && r < rows) v[i] = one(i < kLoads / 2 ? *lo : *hi, r, k0 + k);
      }
    }
  }
  static __device__ __forceinline__ float one(const Operand& m, int64_t r, int c) {
    const float x = value_at<TYPE>(static_cast<const char*>(m.data) + (r * m.ld + c) * kSizeOf<TYPE>);
    if constexpr (TYPE == kTypeE4m3) return x * scale_of(__ldg(m.scales + (m.block_rows == 1 ? r : r >> 7) * m.lds + (c >> 7)));
    return x;
  }
  __device__ __forceinline__ void stage(float (*s)[kPitch<TILE>], const float (&v)[kLoads]) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int idx = int(threadIdx.x) + i * kThreads;
      if (mn) s[idx / TILE][idx % TILE] = v[i];
      else s[idx % kStepK][idx / kStepK] = v[i];
    }
  }
};

__device__ __forceinline__ void put(void* base, int type, int64_t at, float v) {
  if (type == kTypeFp32) static_cast<float*>(base)[at] = v;
  else static_cast<__nv_bfloat16*>(base)[at] = __float2bfloat16_rn(v);
}

// Two sums of a row of the tile, half a tile apart: g and u of a column, or two columns.
template <int TILE>
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
    const int64_t col = n0 + c + h * (TILE / 2);
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

template <int TILE, int TYPE>
__global__ void __launch_bounds__(kThreads) product_kernel(const __grid_constant__ SimtArgs L) {
  constexpr int R = TILE / 16, H = R / 2, kStepK = kStep<TILE>;
  __shared__ __align__(16) float stages[4][kStepK][kPitch<TILE>];      // two places for A, two for B
  const int block = int(blockIdx.x) / L.split, rank = int(blockIdx.x) % L.split;
  int which = 0;
  for (int i = 1; i < L.count; ++i)
    if (block >= L.tile_begin[i]) which = i;
  const Product& p = L.p[which];
  const bool gated = p.e.kind == kGated;
  const int tiles_m = (p.m + TILE - 1) / TILE, tile = block - L.tile_begin[which];
  const int m0 = tile % tiles_m * TILE, n0 = tile / tiles_m * (gated ? TILE / 2 : TILE);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  uint64_t acc[R][H] = {};
  const int steps = (p.k + kStepK - 1) / kStepK, total = steps * p.segments;
  const int begin = int(int64_t(total) * rank / L.split), end = int(int64_t(total) * (rank + 1) / L.split);
  Loader<TILE, TYPE> la, lb;
  float va[decltype(la)::kLoads], vb[decltype(lb)::kLoads];
  int segment = -1;
  auto load = [&](int t) {
    const int s = t >= steps ? 1 : 0;
    if (s != segment) {
      la.init(p.a[s], p.a[s], false, m0, p.m);
      lb.init(p.b[s], p.b[1], gated, n0, p.n);
      segment = s;
    }
    la.load((t - s * steps) * kStepK, p.k, va);
    lb.load((t - s * steps) * kStepK, p.k, vb);
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
#pragma unroll
    for (int k = 0; k < kStepK; ++k) {
      float a[R];
      uint64_t b[H];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float* pa = &stages[t & 1][k][half * (TILE / 2) + ty * H];
        const float* pb = &stages[2 + (t & 1)][k][half * (TILE / 2) + tx * H];
        if constexpr (H == 4) {
          const float4 x = *reinterpret_cast<const float4*>(pa);
          a[half * 4] = x.x; a[half * 4 + 1] = x.y; a[half * 4 + 2] = x.z; a[half * 4 + 3] = x.w;
          const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(pb);
          b[half * 2] = y.x;
          b[half * 2 + 1] = y.y;
        } else {
          const float2 x = *reinterpret_cast<const float2*>(pa);
          a[half * 2] = x.x;
          a[half * 2 + 1] = x.y;
          b[half] = *reinterpret_cast<const uint64_t*>(pb);
        }
      }
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < H; ++j) acc[i][j] = fma2(twice(a[i]), b[j], acc[i][j]);
    }
    if (t + 1 < end) keep(t + 1);       // the other place, which every thread left before the last meeting
    __syncthreads();
  }
  const Activation f = activation_of(p.e.activation);
  auto row_of = [&](int i) { return (i / H) * (TILE / 2) + ty * H + i % H; };
  if constexpr (TILE == 64) {
    if (L.split > 1) {
      constexpr int kRow = TILE + 1;
      static_assert(TILE * kRow <= 4 * kStepK * kPitch<TILE>, "the sums take the place of the operands");
      float* sums = &stages[0][0][0];
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < H; ++j) {
          const float2 pair = both(acc[i][j]);
          float* to = sums + row_of(i) * kRow + (2 * j / H) * (TILE / 2) + tx * H + (2 * j) % H;
          to[0] = pair.x;
          to[1] = pair.y;
        }
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();
#pragma unroll 2
      for (int i = rank * kThreads + int(threadIdx.x); i < TILE * TILE / 2; i += L.split * kThreads) {
        const int r = i / (TILE / 2), c = i % (TILE / 2);
        float first[kMaxSplit], second[kMaxSplit];
#pragma unroll
        for (int q = 0; q < kMaxSplit; ++q)
          if (q < L.split) {
            const float* from = cl.map_shared_rank(sums, unsigned(q)) + r * kRow + c;
            first[q] = from[0];
            second[q] = from[TILE / 2];
          }
        float x = first[0], y = second[0];
#pragma unroll
        for (int q = 1; q < kMaxSplit; ++q)
          if (q < L.split) {
            x += first[q];
            y += second[q];
          }
        finish<TILE>(p, f, m0 + r, n0, c, x, y);
      }
      cl.sync();                        // a block's shared memory stays until its peers have read it
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    float v[R];
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const float2 pair = both(acc[i][j]);
      v[2 * j] = pair.x;
      v[2 * j + 1] = pair.y;
    }
#pragma unroll
    for (int j = 0; j < H; ++j) finish<TILE>(p, f, m0 + row_of(i), n0, tx * H + j, v[j], v[H + j]);
  }
}

template <int TILE, int TYPE>
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
  return cudaLaunchKernelEx(&cfg, product_kernel<TILE, TYPE>, L) == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

}  // namespace

int launch_products_simt(const Product* list, int count, int siblings, int sms, cudaStream_t st) {
  SimtArgs L = {};
  int64_t tiles[2] = {0, 0}, most[2] = {0, 0};      // of 64 and of 128: of all products, of one of them
  int64_t begin[2][kMaxProducts] = {}, steps = INT64_MAX;
  for (int i = 0; i < count; ++i) {
    const Product& p = list[i];
    if (p.m == 0 || p.n == 0) continue;
    L.p[L.count] = p;
    for (int s = 0; s < 2; ++s) {
      const int64_t tile = s ? 128 : 64, wide = p.e.kind == kGated ? tile / 2 : tile;
      begin[s][L.count] = tiles[s];
      const int64_t n = (p.m + tile - 1) / tile * ((p.n + wide - 1) / wide);
      tiles[s] += n;
      most[s] = std::max(most[s], n);
    }
    steps = std::min<int64_t>(steps, (int64_t(p.k) + kStep<64> - 1) / kStep<64> * p.segments);
    ++L.count;
  }
  if (L.count == 0) return 0;
  // A tile of 128 reads each operand half as often; with fewer of them than multiprocessors most of the device would stand still.
  const int large = most[1] * siblings >= sms ? 1 : 0;
  // Three blocks of the small tiles fit a multiprocessor; a part of k is worth a block from four steps on.  `siblings` decides, not how many of them
  // are in this launch: a gradient is the same, bit for bit, whichever others are wanted.
  L.split = large ? 1 : int(std::max<int64_t>(1, std::min<int64_t>({kMaxSplit, 3 * int64_t(sms) / (most[0] * siblings), steps / 4})));
  if (tiles[large] * L.split > INT32_MAX) return MUON_ERR_UNSUPPORTED;
  for (int i = 0; i < L.count; ++i) L.tile_begin[i] = int32_t(begin[large][i]);
  switch (list[0].a[0].type) {
    case kTypeFp32: return large ? launch<128, kTypeFp32>(L, tiles[1], st) : launch<64, kTypeFp32>(L, tiles[0], st);
    case kTypeBf16: return large ? launch<128, kTypeBf16>(L, tiles[1], st) : launch<64, kTypeBf16>(L, tiles[0], st);
    default: return large ? launch<128, kTypeE4m3>(L, tiles[1], st) : launch<64, kTypeE4m3>(L, tiles[0], st);
  }
}

}  // namespace muon
