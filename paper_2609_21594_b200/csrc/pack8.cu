// Activations and weights in 8 bits: e4m3 codes with a power of two for each block of 1 x 128 or 128 x 128 elements, and back.
//
// The scale is the least 2^e with amax <= 448 * 2^e, so multiplying by 2^-e is exact and the only loss is the rounding to e4m3 (2^-4 relative for
// values down to 2^-14 of the block's largest); an amax exactly on the border keeps its block.  A general scale would use the last
// binade a little better, but cost a rounding here and one in every product, and the tensor cores could not apply it.
#include <cuda_fp8.h>

#include "product_ops.h"
#include "words.h"

namespace muon {
namespace {

constexpr int kThreads = 256, kSquareThreads = 512;

__device__ __forceinline__ uint32_t codes2(float lo, float hi) { return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float2 values2(uint32_t pair) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(pair & 0xffffu), __NV_E4M3);
  return __half22float2(__half2(h));
}

// Reads what no launch writes while this one runs.
struct ReadOnly {
  template <typename T> __device__ __forceinline__ T operator()(const T* p) const { return __ldg(p); }
};

// Up to N consecutive elements of a row, by 16 bytes; those from `left` on count as zeros.  WORDS: bf16 that begins anywhere in the row that begins at `first`,
// moved out of aligned words.
template <bool WORDS, typename T, int N>
__device__ __forceinline__ void load_run(const T* p, int left, const T* first, float (&v)[N]) {
  if constexpr (WORDS) {
    if (left >= N) {
      uint32_t w[N / 2 + 1];
      const uint32_t off = words_of_run<uint16_t, N>(reinterpret_cast<const char*>(p), reinterpret_cast<const char*>(first), reinterpret_cast<const char*>(p + left),
                                                     w, ReadOnly());
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const uint32_t x = __funnelshift_r(w[i], w[i + 1], 8 * off);
        v[2 * i] = __uint_as_float(x << 16);
        v[2 * i + 1] = __uint_as_float(x & 0xffff0000u);
      }
      return;
    }
  } else if (left >= N) {
#pragma unroll
    for (int q = 0; q < N * int(sizeof(T)) / 16; ++q) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + q);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
          v[q * 8 + 2 * i] = __uint_as_float(w[i] << 16);
          v[q * 8 + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
          v[q * 4 + i] = __uint_as_float(w[i]);
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i < left ? float(p[i]) : 0.f;
}
// Their codes; `odd`: infinities among them become NaN (the conversion would make them the largest code).
template <int N>
__device__ __forceinline__ void store_run(uint8_t* p, int left, const float (&v)[N], float inverse, bool odd) {
  uint32_t c[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = (odd ? infinite_to_nan(v[4 * i + k]) : v[4 * i + k]) * inverse;
    c[i] = codes2(x[0], x[1]) | codes2(x[2], x[3]) << 16;
  }
  if (left >= N) {
    if constexpr (N == 16) *reinterpret_cast<uint4*>(p) = make_uint4(c[0], c[1], c[2], c[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(c[0], c[1]);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < left) p[i] = uint8_t(c[i >> 2] >> (8 * (i & 3)));
}
// Eight values to an address on a 16-byte border.
__device__ __forceinline__ void store_values(__nv_bfloat16* out, const float* v) {
  uint32_t o[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
    o[k] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(out) = make_uint4(o[0], o[1], o[2], o[3]);
}
__device__ __forceinline__ void store_values(float* out, const float* v) {
  reinterpret_cast<float4*>(out)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(out)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
// The bits of the largest finite magnitude.  The plain maximum passes over NaN; only an infinity makes it look at every value again.
template <int N>
__device__ __forceinline__ uint32_t finite_top(const float (&v)[N], bool* odd) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(v[i]));
  uint32_t bits = __float_as_uint(top);
  *odd = bits == 0x7f800000u;
  if (*odd) {
    bits = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) bits = max(bits, finite_bits(v[i]));
  }
  return bits;
}

// Blocks of 1 x 128: eight lanes hold a block, sixteen elements each, and find its largest magnitude by shuffles.  Blocks are counted along the rows,
// one row after the other.  One block a group: with two or four, whose loads would be in flight together, the registers cost more threads
// than that gains (8192 x 14336 of bf16: 57 us, 5.6 TB/s moved is 1 block; 65 us 2; 110 us 4).  Bound by memory.
template <typename T, bool WORDS>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const T* x, int64_t ldx, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                                                                 int64_t rows, int32_t cols, uint32_t per_row) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // a product that follows may request its weights
  const int sub = threadIdx.x & 7;
  const int64_t block = int64_t(blockIdx.x) * (kThreads / 8) + (threadIdx.x >> 3);
  const int64_t row = block <= UINT32_MAX ? int64_t(uint32_t(block) / per_row) : block / per_row;
  const uint32_t blk = uint32_t(block - row * per_row);
  const int col = int(blk) * kBlock + sub * 16;
  float v[16];
  load_run<WORDS>(x + row * ldx + col, row < rows ? cols - col : 0, x + row * ldx, v);
  bool odd;
  uint32_t top = finite_top(v, &odd);
#pragma unroll
  for (int d = 1; d < 8; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (row >= rows) return;
  const uint32_t e = scale_byte(top);
  store_run(codes + row * ldc + col, cols - col, v, inverse_scale_of(e), odd);
  if (sub == 0) scales[row * lds + blk] = uint8_t(e);
}

// The same for rows that no wide load fits: a warp per block, a lane takes elements l, l + 32, l + 64, l + 96.
template <typename T, int UNROLL>
__global__ void __launch_bounds__(kThreads) quantize_rows_any_kernel(const T* x, int64_t ldx, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                                                                     int64_t rows, int32_t cols, uint32_t per_row) {
  const int lane = threadIdx.x & 31;
  const int64_t first = (int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5)) * UNROLL;
  int64_t row = first / per_row;
  uint32_t blk = uint32_t(first - row * per_row);
  float v[UNROLL][4];
  int64_t at_row[UNROLL];
  uint32_t at_blk[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    at_row[u] = row;
    at_blk[u] = blk;
    const T* p = x + row * ldx + int64_t(blk) * kBlock + lane;
    const int left = row < rows ? cols - int(blk) * kBlock - lane : 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[u][j] = 32 * j < left ? float(p[32 * j]) : 0.f;
    if (++blk == per_row) {
      blk = 0;
      ++row;
    }
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    bool odd;
    const uint32_t top = __reduce_max_sync(0xffffffffu, finite_top(v[u], &odd));
    if (at_row[u] >= rows) continue;
    const uint32_t e = scale_byte(top);
    const float inverse = inverse_scale_of(e);
    uint8_t* p = codes + at_row[u] * ldc + int64_t(at_blk[u]) * kBlock + lane;
    const int left = cols - int(at_blk[u]) * kBlock - lane;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (32 * j < left) p[32 * j] = uint8_t(codes2(infinite_to_nan(v[u][j]) * inverse, 0.f));
    if (lane == 0) scales[at_row[u] * lds + at_blk[u]] = uint8_t(e);
  }
}

// Blocks of 128 x 128: a thread block each, 32 elements a thread kept in registers between the maximum and the rounding.  WIDE: sixteen lanes to a
// row, eight elements each; else a warp to a row, elements 32 apart.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kSquareThreads, 3) quantize_squares_kernel(const T* x, int64_t ldx, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                                                                    int64_t rows, int32_t cols) {
  __shared__ uint32_t tops[kSquareThreads / 32];
  constexpr int kPer = WIDE ? 8 : 4, kTimes = kBlock * kBlock / kSquareThreads / kPer, kStride = kBlock / kTimes;      // elements of a row, rows of a thread and between them
  const int64_t per_row = (cols + kBlock - 1) / kBlock;
  const int64_t brow = int64_t(blockIdx.x) / per_row;
  const int bcol = int(int64_t(blockIdx.x) - brow * per_row);
  const int64_t row0 = brow * kBlock + (WIDE ? threadIdx.x >> 4 : threadIdx.x >> 5);
  const int col = bcol * kBlock + (WIDE ? int(threadIdx.x & 15) * 8 : int(threadIdx.x & 31));
  float v[kTimes][kPer];
  uint32_t top = 0;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < kTimes; ++i) {
    const int64_t row = row0 + kStride * i;
    const int left = row < rows ? cols - col : 0;
    if constexpr (WIDE) {
      load_run<false>(x + row * ldx + col, left, x + row * ldx, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j) v[i][j] = 32 * j < left ? float(x[row * ldx + col + 32 * j]) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < kTimes; ++i) {
    bool some;
    top = max(top, finite_top(v[i], &some));
    odd |= some;
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSquareThreads / 32; ++i) top = max(top, tops[i]);
  const uint32_t e = scale_byte(top);
  const float inverse = inverse_scale_of(e);
#pragma unroll
  for (int i = 0; i < kTimes; ++i) {
    const int64_t row = row0 + kStride * i;
    if (row >= rows) break;
    uint8_t* p = codes + row * ldc + col;
    if constexpr (WIDE) {
      store_run(p, cols - col, v[i], inverse, odd);
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (32 * j < cols - col) p[32 * j] = uint8_t(codes2(infinite_to_nan(v[i][j]) * inverse, 0.f));
    }
  }
  if (threadIdx.x == 0) scales[brow * lds + bcol] = uint8_t(e);
}

// Sixteen codes a thread, which lie in one block (8192 x 14336 to bf16: 57 to 61 us, 5.8 to 6.2 TB/s; two at a time 62 us).
template <typename T>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int32_t row_shift, T* y,
                                                              int64_t ldy, int64_t rows, int32_t cols, uint32_t per_row) {
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t row = i <= UINT32_MAX ? int64_t(uint32_t(i) / per_row) : i / per_row;
  if (row >= rows) return;
  const int col = int(i - row * per_row) * 16, left = cols - col;
  const uint8_t* p = codes + row * ldc + col;
  const float scale = scale_of(__ldg(scales + (row >> row_shift) * lds + (col >> 7)));
  uint32_t w[4] = {0, 0, 0, 0};
  if (left >= 16) {
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
  T* out = y + row * ldy + col;
  if (left < 16) {
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (k < left) out[k] = T(v[k]);
  } else {
    store_values(out, v);
    store_values(out + 8, v + 8);
  }
}

// Rows of y that begin anywhere: a thread takes the eight elements between two 16-byte borders of y (the first of a row those before the first
// border) and moves their codes, which begin anywhere, out of three aligned words.  They may lie in two blocks.
template <typename T>
__global__ void __launch_bounds__(kThreads) dequantize_any_kernel(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int32_t row_shift,
                                                                  T* y, int64_t ldy, int64_t rows, int32_t cols, uint32_t per_row) {
  constexpr int kBorder = 16 / int(sizeof(T));
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t row = i <= UINT32_MAX ? int64_t(uint32_t(i) / per_row) : i / per_row;
  if (row >= rows) return;
  const int g = int(i - row * per_row);
  const int head = (kBorder - (int(reinterpret_cast<uintptr_t>(y + row * ldy) / sizeof(T)) & (kBorder - 1))) & (kBorder - 1);
  const int col = g == 0 ? 0 : head + (g - 1) * 8, count = g == 0 ? min(head, cols) : min(8, cols - col);
  if (count <= 0) return;
  const bool whole = g > 0 && count == 8;
  const uint8_t* s = scales + (row >> row_shift) * lds;
  const uint32_t first = __ldg(s + (col >> 7)), second = __ldg(s + ((col + count - 1) >> 7));
  const char* begin = reinterpret_cast<const char*>(codes + row * ldc);
  const uint8_t* p = codes + row * ldc + col;
  uint32_t w[2] = {0, 0};
  if (whole) {
    uint32_t x[3];
    const uint32_t off = words_of_run<uint8_t, 8>(reinterpret_cast<const char*>(p), begin, begin + cols, x, ReadOnly());
    w[0] = __funnelshift_r(x[0], x[1], 8 * off);
    w[1] = __funnelshift_r(x[1], x[2], 8 * off);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < count) w[k >> 2] |= uint32_t(p[k]) << (8 * (k & 3));
  }
  const float lo = scale_of(first), hi = scale_of(second);
  const int border = ((col >> 7) + 1) * kBlock - col;       // elements from here on lie in the second block
  float v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 f = values2(w[k >> 1] >> (16 * (k & 1)));
    v[2 * k] = f.x * (2 * k < border ? lo : hi);
    v[2 * k + 1] = f.y * (2 * k + 1 < border ? lo : hi);
  }
  T* out = y + row * ldy + col;
  if (whole) return store_values(out, v);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < count) out[k] = T(v[k]);
}

struct CopyList {
  CopyTask task[kMaxCopies];
  int64_t begin[kMaxCopies];                 // first of a task's warps
  int32_t count;
};
// A warp moves a run of kRun bytes of a row: whole words of the destination, each out of the two words of the source that hold it, and what is left at the
// ends by elements.  [first, last): the row that the run is of.
constexpr int kRun = 1024;
template <typename E>
__device__ __forceinline__ void copy_run(const char* from, char* to, int bytes, const char* first, const char* last, int lane) {
  const int head = min(int((4 - (reinterpret_cast<uintptr_t>(to) & 3)) & 3), bytes), words = (bytes - head) / 4, tail = head + words * 4;
  for (int i = lane; i < words; i += 32) {
    uint32_t w[2];
    const uint32_t off = words_of_run<E, 4 / int(sizeof(E))>(from + head + 4 * i, first, last, w, ReadOnly());
    *reinterpret_cast<uint32_t*>(to + head + 4 * i) = __funnelshift_r(w[0], w[1], 8 * off);
  }
  const int at = lane * int(sizeof(E));
  if (at < head) *reinterpret_cast<E*>(to + at) = *reinterpret_cast<const E*>(from + at);
  if (tail + at < bytes) *reinterpret_cast<E*>(to + tail + at) = *reinterpret_cast<const E*>(from + tail + at);
}
__global__ void __launch_bounds__(kThreads) copy_rows_kernel(const __grid_constant__ CopyList L) {
  const int64_t warp = int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  int which = 0;
  for (int i = 1; i < L.count; ++i)
    if (warp >= L.begin[i]) which = i;
  const CopyTask& t = L.task[which];
  const int64_t per_row = (t.bytes + kRun - 1) / kRun, i = warp - L.begin[which], row = i / per_row, at = (i - row * per_row) * kRun;
  if (row >= t.rows) return;
  const char* first = static_cast<const char*>(t.from) + row * t.ld_from;
  const char* from = first + at;
  char* to = static_cast<char*>(t.to) + row * t.ld_to + at;
  const char* last = first + t.bytes;
  const int bytes = int(min(int64_t(kRun), t.bytes - at));
  if (t.unit == 1) copy_run<uint8_t>(from, to, bytes, first, last, threadIdx.x & 31);
  else copy_run<uint16_t>(from, to, bytes, first, last, threadIdx.x & 31);
}

bool wide(const void* p, int64_t ld_bytes, int align) { return reinterpret_cast<uintptr_t>(p) % align == 0 && ld_bytes % align == 0; }
int done(int n) { return cudaGetLastError() == cudaSuccess ? n : MUON_ERR_CUDA; }

template <typename T>
int quantize(int64_t rows, int64_t cols, const T* x, int64_t ldx, const Operand& out, cudaStream_t st) {
  uint8_t* codes = const_cast<uint8_t*>(static_cast<const uint8_t*>(out.data));
  uint8_t* scales = const_cast<uint8_t*>(out.scales);
  const bool w = wide(x, ldx * int64_t(sizeof(T)), 16) && wide(codes, out.ld, 16);
  const int64_t per_row = (cols + kBlock - 1) / kBlock;
  if (out.block_rows == 1) {
    constexpr int kAnyUnroll = 4;
    // bf16 that begins anywhere, into codes that begin at 16 bytes, as the torch front end's do
    const bool words = sizeof(T) == 2 && !w && wide(codes, out.ld, 16);
    const int64_t per_block = w || words ? kThreads / 8 : kThreads / 32 * kAnyUnroll, blocks = (rows * per_row + per_block - 1) / per_block;
    if (blocks > INT32_MAX) return MUON_ERR_UNSUPPORTED;
    auto* k = w ? quantize_rows_kernel<T, false> : quantize_rows_any_kernel<T, kAnyUnroll>;
    if constexpr (sizeof(T) == 2)
      if (words) k = quantize_rows_kernel<T, true>;
    k<<<unsigned(blocks), kThreads, 0, st>>>(x, ldx, codes, out.ld, scales, out.lds, rows, int32_t(cols), uint32_t(per_row));
  } else {
    const int64_t blocks = (rows + kBlock - 1) / kBlock * per_row;
    if (blocks > INT32_MAX) return MUON_ERR_UNSUPPORTED;
    auto* k = w ? quantize_squares_kernel<T, true> : quantize_squares_kernel<T, false>;
    k<<<unsigned(blocks), kSquareThreads, 0, st>>>(x, ldx, codes, out.ld, scales, out.lds, rows, int32_t(cols));
  }
  return done(1);
}

template <typename T>
int dequantize(int64_t rows, int64_t cols, const Operand& in, T* y, int64_t ldy, cudaStream_t st) {
  const uint8_t* codes = static_cast<const uint8_t*>(in.data);
  const bool w = wide(codes, in.ld, 16) && wide(y, ldy * int64_t(sizeof(T)), 16);
  const int64_t per_row = w ? (cols + 15) / 16 : (cols + 7) / 8 + 1;
  const int64_t blocks = (rows * per_row + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return MUON_ERR_UNSUPPORTED;
  auto* k = w ? dequantize_kernel<T> : dequantize_any_kernel<T>;
  k<<<unsigned(blocks), kThreads, 0, st>>>(codes, in.ld, in.scales, in.lds, in.block_rows == 1 ? 0 : 7, y, ldy, rows, int32_t(cols), uint32_t(per_row));
  return done(1);
}

}  // namespace

int launch_copies(const CopyTask* list, int count, int, cudaStream_t st) {
  CopyList L = {};
  int64_t warps = 0;
  for (int i = 0; i < count; ++i) {
    L.task[i] = list[i];
    L.begin[i] = warps;
    warps += list[i].rows * ((list[i].bytes + kRun - 1) / kRun);
  }
  L.count = count;
  const int64_t blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
  if (blocks == 0) return 0;
  if (blocks > INT32_MAX) return MUON_ERR_UNSUPPORTED;
  copy_rows_kernel<<<unsigned(blocks), kThreads, 0, st>>>(L);
  return done(1);
}

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
