// Matrix products on CUDA cores: fp32, and every layout that TMA cannot address.
//
// A block of 256 threads forms a TILE x TILE tile of C, R x R of it per thread (R = TILE / 16), from 16 values of k at a time, staged in shared
// memory as fp32 and loaded one step ahead.  A thread's rows and columns are two runs, one in each half of the tile, so that its operands are
// two wide loads without bank conflicts, and so that in a gated product (columns [0, TILE/2) of the tile are those of B_0, the others
// the same columns of B_1) it holds g and u of the same elements.  Sums are fp32, by two-wide multiply-adds.
#include <cuda_fp8.h>

#include "f32x2.cuh"
#include "product_ops.h"

namespace muon {
namespace {

constexpr int kThreads = 256, kStep = 16;

// Element (row, col) of the matrix as it lies in memory.
template <int TYPE>
__device__ __forceinline__ float element(const Operand& o, int64_t row, int64_t col) {
  if constexpr (TYPE == kTypeFp32) return __ldg(static_cast<const float*>(o.data) + row * o.ld + col);
  if constexpr (TYPE == kTypeBf16) return __bfloat162float(static_cast<const __nv_bfloat16*>(o.data)[row * o.ld + col]);
  const __half_raw h = __nv_cvt_fp8_to_halfraw(static_cast<const uint8_t*>(o.data)[row * o.ld + col], __NV_E4M3);
  return __half2float(__half(h)) * scale_of(__ldg(o.scales + row / o.block_rows * o.lds + (col >> 7)));
}
__device__ __forceinline__ float element_of(const Operand& o, int64_t row, int64_t col) {
  return o.type == kTypeFp32 ? element<kTypeFp32>(o, row, col) : o.type == kTypeBf16 ? element<kTypeBf16>(o, row, col) : element<kTypeE4m3>(o, row, col);
}

// A step of an operand: TILE rows of it from `first` on, k from k0 on.  Threads run along the memory's rows.
template <int TILE, int TYPE, bool MN>
__device__ __forceinline__ void load_step(const Operand& lo, const Operand& hi, bool halves, int first, int rows, int k0, int k, float (&v)[TILE / 16]) {
#pragma unroll
  for (int i = 0; i < TILE / 16; ++i) {
    const int idx = int(threadIdx.x) + i * kThreads;
    const int kk = MN ? idx / TILE : idx % kStep, r = MN ? idx % TILE : idx / kStep;
    const bool second = halves && r >= TILE / 2;
    const int64_t row = first + (second ? r - TILE / 2 : r);
    const bool in = row < rows && k0 + kk < k && (!halves || row < first + TILE / 2);
    const Operand& o = second ? hi : lo;
    v[i] = in ? (MN ? element<TYPE>(o, k0 + kk, row) : element<TYPE>(o, row, k0 + kk)) : 0.f;
  }
}
template <int TILE>
__device__ __forceinline__ void load_step(const Operand& lo, const Operand& hi, bool halves, int first, int rows, int k0, int k, float (&v)[TILE / 16]) {
  auto with = [&](auto type) {
    if (lo.mn_major) load_step<TILE, decltype(type)::value, true>(lo, hi, halves, first, rows, k0, k, v);
    else load_step<TILE, decltype(type)::value, false>(lo, hi, halves, first, rows, k0, k, v);
  };
  if (lo.type == kTypeFp32) with(std::integral_constant<int, kTypeFp32>());
  else if (lo.type == kTypeBf16) with(std::integral_constant<int, kTypeBf16>());
  else with(std::integral_constant<int, kTypeE4m3>());
}
template <int TILE>
__device__ __forceinline__ void stage(float (*s)[TILE + 4], bool mn, const float (&v)[TILE / 16]) {
#pragma unroll
  for (int i = 0; i < TILE / 16; ++i) {
    const int idx = int(threadIdx.x) + i * kThreads;
    if (mn) s[idx / TILE][idx % TILE] = v[i];
    else s[idx % kStep][idx / kStep] = v[i];
  }
}

__device__ __forceinline__ void put(void* base, int type, int64_t at, float v) {
  if (type == kTypeFp32) static_cast<float*>(base)[at] = v;
  else static_cast<__nv_bfloat16*>(base)[at] = __float2bfloat16_rn(v);
}

template <int TILE>
__global__ void __launch_bounds__(kThreads) product_kernel(const __grid_constant__ Product p) {
  constexpr int R = TILE / 16, H = R / 2;
  __shared__ __align__(16) float sa[2][kStep][TILE + 4], sb[2][kStep][TILE + 4];
  const bool gated = p.e.kind == kGated;
  const int cols = gated ? TILE / 2 : TILE;
  const int tiles_m = (p.m + TILE - 1) / TILE;
  const int m0 = int(blockIdx.x % unsigned(tiles_m)) * TILE, n0 = int(blockIdx.x / unsigned(tiles_m)) * cols;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  uint64_t acc[R][H] = {};
  const int steps = (p.k + kStep - 1) / kStep, total = steps * p.segments;
  float va[R], vb[R];
  auto load = [&](int t) {
    const int s = t >= steps ? 1 : 0, k0 = (t - s * steps) * kStep;
    load_step<TILE>(p.a[s], p.a[s], false, m0, p.m, k0, p.k, va);
    load_step<TILE>(p.b[s], p.b[1], gated, n0, p.n, k0, p.k, vb);
  };
  auto keep = [&](int t) {
    const int s = t >= steps ? 1 : 0;
    stage<TILE>(sa[t & 1], p.a[s].mn_major != 0, va);
    stage<TILE>(sb[t & 1], p.b[s].mn_major != 0, vb);
  };
  if (total > 0) {
    load(0);
    keep(0);
  }
  __syncthreads();
  for (int t = 0; t < total; ++t) {
    if (t + 1 < total) load(t + 1);
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      float a[R];
      uint64_t b[H];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float* pa = &sa[t & 1][k][half * (TILE / 2) + ty * H];
        const float* pb = &sb[t & 1][k][half * (TILE / 2) + tx * H];
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
    if (t + 1 < total) keep(t + 1);       // the other buffer, which every thread left before the last meeting
    __syncthreads();
  }
  const Epilogue& e = p.e;
  const Activation f = activation_of(e.activation);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t row = m0 + (i / H) * (TILE / 2) + ty * H + i % H;
    if (row >= p.m) continue;
    float v[R];
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const float2 pair = both(acc[i][j]);
      v[2 * j] = pair.x;
      v[2 * j + 1] = pair.y;
    }
    if (gated) {                            // v[0, H) are g and v[H, R) u of the same columns
#pragma unroll
      for (int j = 0; j < H; ++j) {
        const int64_t col = n0 + tx * H + j;
        if (col >= p.n) continue;
        float a, slope;
        activate<false>(f, v[j], &a, &slope);
        put(e.c, e.type, row * e.ldc + col, a * v[H + j]);
        if (e.gate) {
          put(e.gate, e.gate_up_type, row * e.ld_gate + col, v[j]);
          put(e.up, e.gate_up_type, row * e.ld_up + col, v[H + j]);
        }
      }
      continue;
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int64_t col = n0 + (j / H) * (TILE / 2) + tx * H + j % H;
      if (col >= p.n) continue;
      if (e.kind == kPlain) {
        put(e.c, e.type, row * e.ldc + col, v[j]);
        continue;
      }
      const float g = element_of(e.in_gate, row, col), u = element_of(e.in_up, row, col);
      float a, slope;
      activate<false>(f, g, &a, &slope);
      put(e.gate, e.type, row * e.ld_gate + col, v[j] * u * slope);
      put(e.up, e.type, row * e.ld_up + col, v[j] * a);
      put(e.c, e.type, row * e.ldc + col, a * u);
    }
  }
}

}  // namespace

int launch_product_simt(const Product& p, int sms, cudaStream_t st) {
  if (p.m == 0 || p.n == 0) return 0;
  auto tiles = [&](int64_t tile) { return (p.m + tile - 1) / tile * ((p.n + (p.e.kind == kGated ? tile / 2 : tile) - 1) / (p.e.kind == kGated ? tile / 2 : tile)); };
  // A tile of 128 reads each operand half as often; with fewer of them than multiprocessors most of the device would stand still.
  const bool large = tiles(128) >= sms;
  const int64_t blocks = tiles(large ? 128 : 64);
  if (blocks > INT32_MAX) return MUON_ERR_UNSUPPORTED;
  if (large) product_kernel<128><<<unsigned(blocks), kThreads, 0, st>>>(p);
  else product_kernel<64><<<unsigned(blocks), kThreads, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

}  // namespace muon
