// Layer norm, forward and backward, with the reduction of the weight's and the bias's gradient.
//
// Memory bound: forward reads x and writes y, backward reads dy and x and writes dx, once each.  A row is held in the registers of TPR
// threads (EPT elements each), so the centred sum of squares is taken from the row itself, not from a difference of sums.  Blocks are
// persistent: a thread keeps the weight and bias of its columns for all its rows (re-reading 8 bytes of them per 4 bytes of row
// traffic would make L2 the bound), asks for its next row before it reduces the present one, and in the backward pass adds its columns of
// dy xh and dy in registers.  The blocks' sums, [blocks][2][cols] fp32, are then added in block order by a second kernel.
//
// TPR by columns: one warp per row up to 512 (eight rows per block), then 128, 256, 512, 1024 threads at 16 elements each.  At 1024
// threads a thread has 64 registers: there the backward pass keeps its sums in shared memory, each thread its own columns.
#include <cuda_bf16.h>

#include "layer_ops.h"

namespace muon {
namespace {

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void down(float* p, float v) { *p = v; }
__device__ __forceinline__ void down(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Columns of thread t: piece i of N elements starts at (i * TPR + t) * N.
template <typename T, int N, int TPR, int EPT>
struct Row {
  Pack<T, N> p[EPT / N];
  __device__ __forceinline__ void load(const T* row, int t, int cols) {
#pragma unroll
    for (int i = 0; i < EPT / N; ++i) {
      const int c = (i * TPR + t) * N;
      if (c < cols) p[i] = *reinterpret_cast<const Pack<T, N>*>(row + c);
      else
#pragma unroll
        for (int e = 0; e < N; ++e) down(&p[i].v[e], 0.f);
    }
  }
  __device__ __forceinline__ float at(int i) const { return up(p[i / N].v[i % N]); }
};

template <typename T, int N, int TPR, int EPT>
__device__ __forceinline__ void store_row(T* row, const float (&y)[EPT], int t, int cols) {
#pragma unroll
  for (int i = 0; i < EPT / N; ++i) {
    const int c = (i * TPR + t) * N;
    if (c >= cols) continue;
    Pack<T, N> o;
#pragma unroll
    for (int e = 0; e < N; ++e) down(&o.v[e], y[i * N + e]);
    *reinterpret_cast<Pack<T, N>*>(row + c) = o;
  }
}

template <int N, int TPR, int EPT>
__device__ __forceinline__ void load_param(float (&w)[EPT], const void* p, int dtype, float missing, int t, int cols) {
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const int c = ((i / N) * TPR + t) * N + i % N;
    if (c >= cols) w[i] = 0.f;
    else if (!p) w[i] = missing;
    else w[i] = dtype == MUON_DTYPE_BF16 ? up(static_cast<const __nv_bfloat16*>(p)[c]) : static_cast<const float*>(p)[c];
  }
}

// Sums of K values over the TPR threads of a row, the same in every one of them.  `buf` alternates between two halves, so one
// barrier per call is enough: a half is written again only after everybody has passed the barrier of the call between.
template <int K, int TPR>
__device__ __forceinline__ void row_sum(float (&v)[K], float* buf, int& half) {
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int d = 16; d; d >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], d);
  if (TPR == 32) return;
  constexpr int W = TPR / 32;
  float* b = buf + half * (2 * 32);
  half ^= 1;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) b[k * 32 + threadIdx.x / 32] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float s = (threadIdx.x & 31) < W ? b[k * 32 + (threadIdx.x & 31)] : 0.f;
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    v[k] = s;
  }
}

template <int TPR> struct Geometry {
  static constexpr int kRows = TPR == 32 ? 8 : 1;     // rows of a block at a time
  static constexpr int kThreads = TPR * kRows;
};

template <typename T, int N, int TPR, int EPT>
__global__ void __launch_bounds__(Geometry<TPR>::kThreads) norm_forward_kernel(const NormArgs a) {
  constexpr int R = Geometry<TPR>::kRows;
  __shared__ float buf[128];
  const int t = threadIdx.x % TPR;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.out);
  float w[EPT], b[EPT];
  load_param<N, TPR, EPT>(w, a.weight, a.param_dtype, 1.f, t, a.cols);
  load_param<N, TPR, EPT>(b, a.bias, a.param_dtype, 0.f, t, a.cols);
  const float inv = 1.f / float(a.cols);
  const int64_t step = int64_t(gridDim.x) * R;
  int64_t r = int64_t(blockIdx.x) * R + threadIdx.x / TPR;
  int half = 0;
  Row<T, N, TPR, EPT> next;
  if (r < a.rows) next.load(x + r * a.ldx, t, a.cols);
  for (; r < a.rows; r += step) {
    const Row<T, N, TPR, EPT> cur = next;
    if (r + step < a.rows) next.load(x + (r + step) * a.ldx, t, a.cols);
    float v[EPT], mean = 0.f;
#pragma unroll
    for (int i = 0; i < EPT; ++i) v[i] = cur.at(i);
    if (a.center) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < EPT; ++i) s[0] += v[i];
      row_sum<1, TPR>(s, buf, half);
      mean = s[0] * inv;
#pragma unroll
      for (int i = 0; i < EPT; ++i) v[i] -= mean;
    }
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const int c = ((i / N) * TPR + t) * N + i % N;
      if (c < a.cols) s[0] = fmaf(v[i], v[i], s[0]);
    }
    row_sum<1, TPR>(s, buf, half);
    const float rstd = 1.f / sqrtf(s[0] * inv + a.eps);
#pragma unroll
    for (int i = 0; i < EPT; ++i) v[i] = fmaf(v[i] * rstd, w[i], b[i]);
    store_row<T, N, TPR, EPT>(y + r * a.ldo, v, t, a.cols);
    if (t == 0) {
      if (a.mean) a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

template <typename T, int N, int TPR, int EPT, bool SHARED_SUMS>
__global__ void __launch_bounds__(Geometry<TPR>::kThreads) norm_backward_kernel(const NormArgs a) {
  constexpr int R = Geometry<TPR>::kRows;
  extern __shared__ float sums[];                     // SHARED_SUMS: [2][EPT][TPR]; one warp per row: [8][2][32 * EPT] at the end
  __shared__ float buf[128];
  const int t = threadIdx.x % TPR;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.out);
  float w[SHARED_SUMS ? 1 : EPT], dw[SHARED_SUMS ? 1 : EPT], db[SHARED_SUMS ? 1 : EPT];
  if constexpr (SHARED_SUMS) {
    for (int i = 0; i < 2 * EPT; ++i) sums[i * TPR + t] = 0.f;
  } else {
    load_param<N, TPR, EPT>(w, a.weight, a.param_dtype, 1.f, t, a.cols);
#pragma unroll
    for (int i = 0; i < EPT; ++i) dw[i] = db[i] = 0.f;
  }
  const float inv = 1.f / float(a.cols);
  const int64_t step = int64_t(gridDim.x) * R;
  int64_t r = int64_t(blockIdx.x) * R + threadIdx.x / TPR;
  int half = 0;
  Row<T, N, TPR, EPT> nx, ny;
  if (r < a.rows) {
    nx.load(x + r * a.ldx, t, a.cols);
    ny.load(dy + r * a.lddy, t, a.cols);
  }
  for (; r < a.rows; r += step) {
    const Row<T, N, TPR, EPT> cx = nx, cy = ny;
    if (!SHARED_SUMS && r + step < a.rows) {          // with 64 registers there is no room for a second row
      nx.load(x + (r + step) * a.ldx, t, a.cols);
      ny.load(dy + (r + step) * a.lddy, t, a.cols);
    }
    const float mean = a.mean ? a.mean[r] : 0.f, rstd = a.rstd[r];
    auto weight = [&](int i) -> float {
      if constexpr (!SHARED_SUMS) return w[i];
      const int c = ((i / N) * TPR + t) * N + i % N;
      if (c >= a.cols) return 0.f;
      if (!a.weight) return 1.f;
      return a.param_dtype == MUON_DTYPE_BF16 ? up(static_cast<const __nv_bfloat16*>(a.weight)[c]) : static_cast<const float*>(a.weight)[c];
    };
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < EPT; ++i) {                   // columns past the end have dy = 0 and weight 0
      const float xh = (cx.at(i) - mean) * rstd, d = cy.at(i), g = d * weight(i);
      s[0] += g;
      s[1] = fmaf(g, xh, s[1]);
      if constexpr (SHARED_SUMS) {
        sums[i * TPR + t] = fmaf(d, xh, sums[i * TPR + t]);
        sums[(EPT + i) * TPR + t] += d;
      } else {
        dw[i] = fmaf(d, xh, dw[i]);
        db[i] += d;
      }
    }
    row_sum<2, TPR>(s, buf, half);
    const float m1 = a.mean ? s[0] * inv : 0.f, m2 = s[1] * inv;
    float v[EPT];
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const float xh = (cx.at(i) - mean) * rstd;
      v[i] = rstd * (cy.at(i) * weight(i) - m1 - xh * m2);
    }
    store_row<T, N, TPR, EPT>(dx + r * a.ldo, v, t, a.cols);
    if (SHARED_SUMS && r + step < a.rows) {
      nx.load(x + (r + step) * a.ldx, t, a.cols);
      ny.load(dy + (r + step) * a.lddy, t, a.cols);
    }
  }
  if (!a.parts) return;
  float* out = a.parts + int64_t(blockIdx.x) * 2 * a.cols;
  if constexpr (TPR == 32) {                          // the block's eight rows at a time: add its warps in order
    const int wp = threadIdx.x / 32;
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const int c = ((i / N) * TPR + t) * N + i % N;
      sums[(wp * 2) * (32 * EPT) + c] = dw[i];
      sums[(wp * 2 + 1) * (32 * EPT) + c] = db[i];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * a.cols; j += blockDim.x) {
      const int which = j >= a.cols, c = j - which * a.cols;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < R; ++k) s += sums[(k * 2 + which) * (32 * EPT) + c];
      out[j] = s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const int c = ((i / N) * TPR + t) * N + i % N;
      if (c >= a.cols) continue;
      if constexpr (SHARED_SUMS) {
        out[c] = sums[i * TPR + t];
        out[a.cols + c] = sums[(EPT + i) * TPR + t];
      } else {
        out[c] = dw[i];
        out[a.cols + c] = db[i];
      }
    }
  }
}

// Adds the blocks' sums: 32 columns per block, 32 threads share a column's parts, in a fixed order.
__global__ void __launch_bounds__(1024) norm_parts_kernel(const float* parts, int n, int cols, void* dweight, void* dbias, int param_dtype) {
  __shared__ float sm[32][33];
  const int which = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
  void* out = which ? dbias : dweight;
  float s = 0.f;
  if (c < cols && out)
    for (int k = threadIdx.y; k < n; k += 32) s += parts[(int64_t(k) * 2 + which) * cols + c];
  sm[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  float v = sm[threadIdx.x][threadIdx.y];
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  const int col = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && col < cols && out) {
    if (param_dtype == MUON_DTYPE_BF16) static_cast<__nv_bfloat16*>(out)[col] = __float2bfloat16_rn(v);
    else static_cast<float*>(out)[col] = v;
  }
}

int blocks_for(int64_t rows, int rows_per_block, int most) {
  const int64_t need = (rows + rows_per_block - 1) / rows_per_block;
  return int(need < most ? need : most);
}

template <typename T, int N, int TPR, int EPT>
int forward(const NormArgs& a, int sms, cudaStream_t st) {
  using G = Geometry<TPR>;
  const int blocks = blocks_for(a.rows, G::kRows, sms * (2048 / G::kThreads > 8 ? 8 : 2048 / G::kThreads));
  norm_forward_kernel<T, N, TPR, EPT><<<blocks, G::kThreads, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

template <typename T, int N, int TPR, int EPT, bool SHARED_SUMS = false>
int backward(const NormArgs& a, int sms, cudaStream_t st) {
  using G = Geometry<TPR>;
  constexpr int bytes = SHARED_SUMS ? 2 * EPT * TPR * 4 : TPR == 32 ? 8 * 2 * 32 * EPT * 4 : 0;
  auto kernel = norm_backward_kernel<T, N, TPR, EPT, SHARED_SUMS>;
  if (bytes > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess)
    return MUON_ERR_CUDA;
  const int most = sms * 4 < kNormMaxParts ? sms * 4 : kNormMaxParts;
  const int blocks = blocks_for(a.rows, G::kRows, TPR >= 512 ? (sms < most ? sms : most) : TPR == 256 ? (sms * 2 < most ? sms * 2 : most) : most);
  if (blocks) kernel<<<blocks, G::kThreads, bytes, st>>>(a);
  if (cudaGetLastError() != cudaSuccess) return MUON_ERR_CUDA;
  if (!a.dweight && !a.dbias) return blocks ? 1 : 0;      // no rows: the sums are zero
  norm_parts_kernel<<<dim3(unsigned((a.cols + 31) / 32), 2), dim3(32, 32), 0, st>>>(a.parts, blocks, a.cols, a.dweight, a.dbias, a.param_dtype);
  return cudaGetLastError() == cudaSuccess ? (blocks ? 2 : 1) : MUON_ERR_CUDA;
}

template <typename T, int N>
int forward_by_cols(const NormArgs& a, int sms, cudaStream_t st) {
  constexpr int E = N > 8 ? N : 8;
  if (a.cols <= 32 * E) return forward<T, N, 32, E>(a, sms, st);
  if (a.cols <= 512) return forward<T, N, 32, 16>(a, sms, st);
  if (a.cols <= 2048) return forward<T, N, 128, 16>(a, sms, st);
  if (a.cols <= 4096) return forward<T, N, 256, 16>(a, sms, st);
  if (a.cols <= 8192) return forward<T, N, 512, 16>(a, sms, st);
  return forward<T, N, 1024, 16>(a, sms, st);
}

template <typename T, int N>
int backward_by_cols(const NormArgs& a, int sms, cudaStream_t st) {
  constexpr int E = N > 8 ? N : 8;
  if (a.cols <= 32 * E) return backward<T, N, 32, E>(a, sms, st);
  if (a.cols <= 512) return backward<T, N, 32, 16>(a, sms, st);
  if (a.cols <= 2048) return backward<T, N, 128, 16>(a, sms, st);
  if (a.cols <= 4096) return backward<T, N, 256, 16>(a, sms, st);
  if (a.cols <= 8192) return backward<T, N, 512, 16>(a, sms, st);
  return backward<T, N, 1024, 16, true>(a, sms, st);
}

bool pieces(const void* p, int64_t ld, int bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * bytes) % 16 == 0; }

// 16-byte accesses need 16-byte aligned rows that are a whole number of them; other rows go element by element.
bool vector_rows(const NormArgs& a) {
  const int e = a.dtype == MUON_DTYPE_BF16 ? 2 : 4;
  return (a.cols * e) % 16 == 0 && pieces(a.x, a.ldx, e) && pieces(a.out, a.ldo, e) && (!a.dy || pieces(a.dy, a.lddy, e));
}

}  // namespace

int norm_parts(int64_t rows, int cols) { return blocks_for(rows, cols <= 512 ? 8 : 1, kNormMaxParts); }

int launch_norm_forward(const NormArgs& a, int sms, cudaStream_t st) {
  if (a.dtype == MUON_DTYPE_BF16)
    return vector_rows(a) ? forward_by_cols<__nv_bfloat16, 8>(a, sms, st) : forward_by_cols<__nv_bfloat16, 1>(a, sms, st);
  return vector_rows(a) ? forward_by_cols<float, 4>(a, sms, st) : forward_by_cols<float, 1>(a, sms, st);
}

int launch_norm_backward(const NormArgs& a, int sms, cudaStream_t st) {
  if (a.dtype == MUON_DTYPE_BF16)
    return vector_rows(a) ? backward_by_cols<__nv_bfloat16, 8>(a, sms, st) : backward_by_cols<__nv_bfloat16, 1>(a, sms, st);
  return vector_rows(a) ? backward_by_cols<float, 4>(a, sms, st) : backward_by_cols<float, 1>(a, sms, st);
}

}  // namespace muon
