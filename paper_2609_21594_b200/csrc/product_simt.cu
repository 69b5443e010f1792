// Matrix products on CUDA cores: fp32, and every layout that TMA cannot address.
//
// A block forms a TILE x TILE tile of C, 8 x 8 (TILE = 128, 256 threads) or 8 x 4 (64, 128 threads) of it per thread, from 8 or 32 values of k at a
// time, staged in shared memory as fp32 and loaded one step ahead.  A thread's rows and columns are two runs, one in each half of the tile, so
// that its operands are wide loads without bank conflicts, and so that in a gated product (columns [0, TILE/2) of the tile are those of B_0,
// the others the same columns of B_1) it holds g and u of the same elements.  Sums are fp32, by multiply-adds of two rows at a time.
//
// Where 128 x 128 tiles would leave multiprocessors idle, the tiles are 64 x 64 and the blocks of a cluster each take a part of k; the parts are added
// in the order of the ranks, so the sum is the same in every run.
//
// What bounds it: 1024 x 1024 x 2816, both products 650 us, 27 TFLOP/s of 74, the multiply-add pipe 59 % busy while blocks run, and 352 blocks of the
// gated product where 296 fit at once.  389 x 250 x 1021, backward, 77 us on the device: starts, meetings and ends of short sums.
#include <cooperative_groups.h>
#include <cuda_fp8.h>

#include <algorithm>

#include "f32x2.cuh"
#include "product_ops.h"

namespace muon {
namespace {

namespace cg = cooperative_groups;
constexpr int kMaxSplit = 8;
template <int TILE>
struct Tile {
  static constexpr int columns = TILE / 16, threads = TILE * TILE / (8 * columns);     // of C per thread: 8 rows of `columns`
  static constexpr int step = TILE == 64 ? 32 : 8;       // values of k; the small tiles wait more for memory, so that more is in flight there
  static constexpr int blocks = TILE == 64 ? 4 : 2;      // on a multiprocessor: what one waits for, the others cover
  static constexpr int pitch = TILE + 4;                 // of a staged row: eight neighbouring k of four rows lie in 32 banks
  static constexpr int loads = TILE * step / threads;    // elements of an operand that a thread loads in a step
};

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
template <int TILE, int TYPE>
struct Loader {
  using T = Tile<TILE>;
  static constexpr int kGroups = T::step / 8, kRowsApart = T::threads / 8, kApart = T::threads / TILE;
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
    k = mn ? int(threadIdx.x) / TILE : int(threadIdx.x) % 8;
    row_lo = first + (mn ? int(threadIdx.x) % TILE : int(threadIdx.x) / 8);
    row_hi = halves ? row_lo : row_lo + TILE / 2;
  }
  __device__ __forceinline__ void load(int k0, int kdim, float (&v)[T::loads]) const {
    if (mn) {
      const bool in = row_lo < rows;
#pragma unroll
      for (int i = 0; i < T::loads; ++i) {
        const int kk = k0 + k + i * kApart;
        v[i] = 0.f;
        if (in && kk < kdim) v[i] = one(lo, ld_lo, kk, row_lo);
      }
    } else {
#pragma unroll
      for (int i = 0; i < T::loads; ++i) {
        const int group = i / kGroups, kk = k0 + k + 8 * (i % kGroups);
        const bool first = group * kRowsApart < TILE / 2;
        const int r = first ? row_lo + group * kRowsApart : row_hi + group * kRowsApart - TILE / 2;
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
  __device__ __forceinline__ void stage(float (*s)[T::pitch], const float (&v)[T::loads]) const {
#pragma unroll
    for (int i = 0; i < T::loads; ++i) {
      if (mn) s[int(threadIdx.x) / TILE + i * kApart][int(threadIdx.x) % TILE] = v[i];
      else s[int(threadIdx.x) % 8 + 8 * (i % kGroups)][int(threadIdx.x) / 8 + i / kGroups * kRowsApart] = v[i];
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
__global__ void __launch_bounds__(Tile<TILE>::threads, Tile<TILE>::blocks) product_kernel(const __grid_constant__ SimtArgs L) {
  using T = Tile<TILE>;
  constexpr int N = T::columns, H = N / 2;                        // columns of a thread, and those in each half of the tile
  __shared__ __align__(16) float stages[4][T::step][T::pitch];    // two places for A, two for B
  const int block = int(blockIdx.x) / L.split, rank = int(blockIdx.x) % L.split;
  int which = 0;
  for (int i = 1; i < L.count; ++i)
    if (block >= L.tile_begin[i]) which = i;
  const Product& p = L.p[which];
  const bool gated = p.e.kind == kGated;
  const int tiles_m = (p.m + TILE - 1) / TILE, tile = block - L.tile_begin[which];
  const int m0 = tile % tiles_m * TILE, n0 = tile / tiles_m * (gated ? TILE / 2 : TILE);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  uint64_t acc[4][N] = {};                                        // two rows each: 0, 1 and 2, 3 of the run in either half
  const int steps = (p.k + T::step - 1) / T::step, total = steps * p.segments;
  const int begin = int(int64_t(total) * rank / L.split), end = int(int64_t(total) * (rank + 1) / L.split);
  Loader<TILE, TYPE> la, lb;
  float va[T::loads], vb[T::loads];
  int segment = -1;
  auto load = [&](int t) {
    const int s = t >= steps ? 1 : 0;
    if (s != segment) {
      la.init(p.a[s], p.a[s], false, m0, p.m);
      lb.init(p.b[s], p.b[1], gated, n0, p.n);
      segment = s;
    }
    la.load((t - s * steps) * T::step, p.k, va);
    lb.load((t - s * steps) * T::step, p.k, vb);
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
    float b[2][N];
    auto fetch = [&](int k, int to) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(&stages[t & 1][k][half * (TILE / 2) + ty * 4]);
        a[to][half * 2] = x.x;
        a[to][half * 2 + 1] = x.y;
        const float* pb = &stages[2 + (t & 1)][k][half * (TILE / 2) + tx * H];
        if constexpr (H == 4) {
          const float4 y = *reinterpret_cast<const float4*>(pb);
          b[to][half * 4] = y.x; b[to][half * 4 + 1] = y.y; b[to][half * 4 + 2] = y.z; b[to][half * 4 + 3] = y.w;
        } else {
          const float2 y = *reinterpret_cast<const float2*>(pb);
          b[to][half * 2] = y.x;
          b[to][half * 2 + 1] = y.y;
        }
      }
    };
    fetch(0, 0);
#pragma unroll 8
    for (int k = 0; k < T::step; ++k) {
      if (k + 1 < T::step) fetch(k + 1, (k + 1) & 1);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const uint64_t bb = twice(b[k & 1][j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = fma2(a[k & 1][i], bb, acc[i][j]);
      }
    }
    if (t + 1 < end) keep(t + 1);       // the other place, which every thread left before the last meeting
    __syncthreads();
  }
  const Activation f = activation_of(p.e.activation);
  auto row_of = [&](int i) { return (i / 2) * (TILE / 2) + ty * 4 + (i % 2) * 2; };      // the first of a pair's rows
  if constexpr (TILE == 64) {
    if (L.split > 1) {
      constexpr int kRow = TILE + 1;
      static_assert(TILE * kRow <= 4 * T::step * T::pitch, "the sums take the place of the operands");
      float* sums = &stages[0][0][0];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float2 pair = both(acc[i][j]);
          float* to = sums + row_of(i) * kRow + (j / H) * (TILE / 2) + tx * H + j % H;
          to[0] = pair.x;
          to[kRow] = pair.y;
        }
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();
#pragma unroll 2
      for (int i = rank * T::threads + int(threadIdx.x); i < TILE * TILE / 2; i += L.split * T::threads) {
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
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const float2 first = both(acc[i][j]), second = both(acc[i][H + j]);
      finish<TILE>(p, f, m0 + row_of(i), n0, tx * H + j, first.x, second.x);
      finish<TILE>(p, f, m0 + row_of(i) + 1, n0, tx * H + j, first.y, second.y);
    }
}

template <int TILE, int TYPE>
int launch(const SimtArgs& L, int64_t tiles, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(tiles * L.split), 1, 1);
  cfg.blockDim = dim3(Tile<TILE>::threads, 1, 1);
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
    steps = std::min<int64_t>(steps, (int64_t(p.k) + Tile<64>::step - 1) / Tile<64>::step * p.segments);
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
