// Activations and weights in 8 bits: e4m3 codes with a power of two for each block of 1 x 128 or 128 x 128 elements, and back.
//
// The scale is the least 2^e with amax <= 448 * 2^e, so multiplying by 2^-e is exact and the only loss is the rounding to e4m3 (2^-4 relative for
// values down to 2^-14 of the block's largest); an amax exactly on the border keeps its block.  A general scale would use the last
// binade a little better, but cost a rounding here and one in every product, and the tensor cores could not apply it.
#include <cuda_fp8.h>

#include "product_ops.h"

namespace muon {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t codes2(float lo, float hi) { return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float2 values2(uint32_t pair) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(pair & 0xffffu), __NV_E4M3);
  return __half22float2(__half2(h));
}

// Eight consecutive elements of a row; those from `left` on count as zeros.
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T* p, int left, float (&v)[8]) {
  if constexpr (WIDE) {
    if (left >= 8) {
      if constexpr (sizeof(T) == 2) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[2 * i] = __uint_as_float(w[i] << 16);
          v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
      } else {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < left ? float(p[i]) : 0.f;
}

template <bool WIDE>
__device__ __forceinline__ void store8(uint8_t* p, int left, const float (&v)[8], float inverse) {
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = codes2(infinite_to_nan(v[2 * i]) * inverse, infinite_to_nan(v[2 * i + 1]) * inverse);
  if (WIDE && left >= 8) {
    *reinterpret_cast<uint2*>(p) = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) p[i] = uint8_t(c[i >> 1] >> (8 * (i & 1)));
}

// Blocks of 1 x 128: sixteen lanes hold a block, eight elements each, and find its largest magnitude by shuffles.  Blocks are counted along the rows,
// one row after the other; a group of lanes takes UNROLL consecutive ones, so that its loads are in flight together and the division that
// finds the row is made once.
template <typename T, bool WIDE, int UNROLL>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const T* x, int64_t ldx, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                                                                 int64_t rows, int32_t cols) {
  const int64_t per_row = (cols + kBlock - 1) / kBlock, total = rows * per_row;
  const int sub = threadIdx.x & 15;
  const int64_t first = (int64_t(blockIdx.x) * (kThreads / 16) + (threadIdx.x >> 4)) * UNROLL;
  int64_t row = first < total ? first / per_row : rows;
  int32_t blk = first < total ? int32_t(first - row * per_row) : 0;
  float v[UNROLL][8];
  int64_t at_row[UNROLL];
  int32_t at_blk[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    at_row[u] = row;
    at_blk[u] = blk;
    const int col = blk * kBlock + sub * 8;
    const int left = row < rows ? cols - col : 0;
    load8<T, WIDE>(x + row * ldx + col, left, v[u]);
    if (++blk == per_row) {
      blk = 0;
      ++row;
    }
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, finite_bits(v[u][i]));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
    if (at_row[u] >= rows) continue;
    const uint32_t e = scale_byte(top);
    const int col = at_blk[u] * kBlock + sub * 8;
    store8<WIDE>(codes + at_row[u] * ldc + col, cols - col, v[u], inverse_scale_of(e));
    if (sub == 0) scales[at_row[u] * lds + at_blk[u]] = uint8_t(e);
  }
}

// Blocks of 128 x 128: a thread block each, 64 elements a thread kept in registers between the maximum and the rounding.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) quantize_squares_kernel(const T* x, int64_t ldx, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                                                                    int64_t rows, int32_t cols) {
  __shared__ uint32_t tops[kThreads / 32];
  const int64_t per_row = (cols + kBlock - 1) / kBlock;
  const int64_t brow = int64_t(blockIdx.x) / per_row;
  const int bcol = int(int64_t(blockIdx.x) - brow * per_row);
  const int64_t row0 = brow * kBlock + (threadIdx.x >> 4);
  const int col = bcol * kBlock + (threadIdx.x & 15) * 8;
  float v[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) load8<T, WIDE>(x + (row0 + 16 * i) * ldx + col, row0 + 16 * i < rows ? cols - col : 0, v[i]);
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, finite_bits(v[i][j]));
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) top = max(top, tops[i]);
  const uint32_t e = scale_byte(top);
  const float inverse = inverse_scale_of(e);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (row0 + 16 * i < rows) store8<WIDE>(codes + (row0 + 16 * i) * ldc + col, cols - col, v[i], inverse);
  if (threadIdx.x == 0) scales[brow * lds + bcol] = uint8_t(e);
}

// Sixteen codes a thread: they lie in one block.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int32_t row_shift, T* y,
                                                              int64_t ldy, int64_t rows, int32_t cols) {
  const int64_t per_row = (cols + 15) / 16;
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t row = i / per_row;
  if (row >= rows) return;
  const int col = int(i - row * per_row) * 16;
  const int left = cols - col;
  const uint8_t* p = codes + row * ldc + col;
  T* out = y + row * ldy + col;
  const float scale = scale_of(__ldg(scales + (row >> row_shift) * lds + (col >> 7)));
  uint32_t w[4] = {0, 0, 0, 0};
  if (WIDE && left >= 16) {
    const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
    w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (k < left) w[k >> 2] |= uint32_t(p[k]) << (8 * (k & 3));
  }
  float v[16];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float2 f = values2(w[k >> 1] >> (16 * (k & 1)));
    v[2 * k] = f.x * scale;
    v[2 * k + 1] = f.y * scale;
  }
  if (WIDE && left >= 16) {
    if constexpr (sizeof(T) == 2) {
      uint32_t o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
        o[k] = *reinterpret_cast<const uint32_t*>(&b);
      }
      reinterpret_cast<uint4*>(out)[0] = make_uint4(o[0], o[1], o[2], o[3]);
      reinterpret_cast<uint4*>(out)[1] = make_uint4(o[4], o[5], o[6], o[7]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) reinterpret_cast<float4*>(out)[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 16; ++k)
    if (k < left) out[k] = T(v[k]);
}

bool wide(const void* p, int64_t ld_bytes, int align) { return reinterpret_cast<uintptr_t>(p) % align == 0 && ld_bytes % align == 0; }
int done(int n) { return cudaGetLastError() == cudaSuccess ? n : MUON_ERR_CUDA; }

template <typename T>
int quantize(int64_t rows, int64_t cols, const T* x, int64_t ldx, const Operand& out, cudaStream_t st) {
  uint8_t* codes = const_cast<uint8_t*>(static_cast<const uint8_t*>(out.data));
  uint8_t* scales = const_cast<uint8_t*>(out.scales);
  const bool w = wide(x, ldx * int64_t(sizeof(T)), 16) && wide(codes, out.ld, 8);
  const int64_t per_row = (cols + kBlock - 1) / kBlock;
  if (out.block_rows == 1) {
    constexpr int kUnroll = 4;
    const int64_t per_block = int64_t(kThreads / 16) * kUnroll, blocks = (rows * per_row + per_block - 1) / per_block;
    if (blocks > INT32_MAX) return MUON_ERR_UNSUPPORTED;
    auto* k = w ? quantize_rows_kernel<T, true, kUnroll> : quantize_rows_kernel<T, false, kUnroll>;
    k<<<unsigned(blocks), kThreads, 0, st>>>(x, ldx, codes, out.ld, scales, out.lds, rows, int32_t(cols));
  } else {
    const int64_t blocks = (rows + kBlock - 1) / kBlock * per_row;
    if (blocks > INT32_MAX) return MUON_ERR_UNSUPPORTED;
    auto* k = w ? quantize_squares_kernel<T, true> : quantize_squares_kernel<T, false>;
    k<<<unsigned(blocks), kThreads, 0, st>>>(x, ldx, codes, out.ld, scales, out.lds, rows, int32_t(cols));
  }
  return done(1);
}

template <typename T>
int dequantize(int64_t rows, int64_t cols, const Operand& in, T* y, int64_t ldy, cudaStream_t st) {
  const uint8_t* codes = static_cast<const uint8_t*>(in.data);
  const int64_t blocks = (rows * ((cols + 15) / 16) + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return MUON_ERR_UNSUPPORTED;
  const bool w = wide(codes, in.ld, 16) && wide(y, ldy * int64_t(sizeof(T)), 16);
  auto* k = w ? dequantize_kernel<T, true> : dequantize_kernel<T, false>;
  k<<<unsigned(blocks), kThreads, 0, st>>>(codes, in.ld, in.scales, in.lds, in.block_rows == 1 ? 0 : 7, y, ldy, rows, int32_t(cols));
  return done(1);
}

}  // namespace

int launch_quantize(int dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, const Operand& out, int, cudaStream_t st) {
  if (rows == 0) return 0;
  return dtype == kTypeBf16 ? quantize(rows, cols, static_cast<const __nv_bfloat16*>(x), ldx, out, st)
                            : quantize(rows, cols, static_cast<const float*>(x), ldx, out, st);
}

int launch_dequantize(int dtype, int64_t rows, int64_t cols, const Operand& in, void* y, int64_t ldy, int, cudaStream_t st) {
  if (rows == 0) return 0;
  return dtype == kTypeBf16 ? dequantize(rows, cols, in, static_cast<__nv_bfloat16*>(y), ldy, st) : dequantize(rows, cols, in, static_cast<float*>(y), ldy, st);
}

}  // namespace muon
