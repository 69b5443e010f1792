// Layer norm, forward and backward, with the reduction of the weight's and the bias's gradient.
//
// Memory bound: forward reads x and writes y, backward reads dy and x and writes dx, once each.  A row is held in the registers of the
// threads that own it, so the centred sum of squares is taken from the row itself, not from a difference of sums.  Rows in 16-byte
// pieces travel by cp.async through a ring in shared memory: a thread copies and reads only its own columns, so the ring needs no
// barrier, rows ahead cost no registers, and pieces past the last column arrive as zeros.
//
// Forward: a row belongs to 32 to 512 threads with at most four pieces each (32 values of bf16: more would leave too few warps to hide
// the chain of two sums).  The row groups of a block do not wait for one another; weight and bias lie in shared memory as fp32.
//
// Backward: a thread keeps its 16 columns for all its rows, so it adds dy xh and dy in registers.  Rows wider than 8192 columns are
// cut between the two blocks of a cluster, which exchange their sums through distributed shared memory.  The blocks' sums,
// [blocks][2][cols] fp32, are added in block order by a second kernel.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "layer_ops.h"

namespace cg = cooperative_groups;

namespace muon {
namespace {

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void down(float* p, float v) { *p = v; }
__device__ __forceinline__ void down(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float param_at(const void* p, int dtype, float missing, int c) {
  if (!p) return missing;
  return dtype == MUON_DTYPE_BF16 ? up(static_cast<const __nv_bfloat16*>(p)[c]) : static_cast<const float*>(p)[c];
}

__device__ __forceinline__ void copy_piece(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Columns of thread t of a row: piece i of N elements starts at (i * TPR + t) * N.  In pieces of 16 bytes the thread asks for a row ahead
// of time (fetch) and takes it from its places of the ring; element by element (rows without the alignment) it reads the row directly.
template <typename T, int N, int TPR, int EPT, int THREADS>
struct Rows {
  static constexpr bool kRing = N * sizeof(T) == 16;
  static constexpr int kPieces = EPT / N;
  static constexpr int kStageBytes = kRing ? THREADS * kPieces * 16 : 0;
  __device__ static __forceinline__ void fetch(uint32_t stage, const T* row, int t, int cols) {
    if constexpr (kRing) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int c = (i * TPR + t) * N;
        copy_piece(stage + uint32_t(i * THREADS + threadIdx.x) * 16u, c < cols ? row + c : row, c < cols);
      }
    }
  }
  __device__ static __forceinline__ void raw(Pack<T, N> (&p)[kPieces], uint32_t stage, const T* row, int t, int cols) {
    if constexpr (kRing) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        uint32_t* u = reinterpret_cast<uint32_t*>(&p[i]);
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                     : "r"(stage + uint32_t(i * THREADS + threadIdx.x) * 16u));
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        const int c = i * TPR + t;
        if (c < cols) p[i].v[0] = row[c];
        else down(&p[i].v[0], 0.f);
      }
    }
  }
  __device__ static __forceinline__ void take(float (&v)[EPT], uint32_t stage, const T* row, int t, int cols) {
    Pack<T, N> p[kPieces];
    raw(p, stage, row, t, cols);
#pragma unroll
    for (int i = 0; i < EPT; ++i) v[i] = up(p[i / N].v[i % N]);
  }
};

// ------------------------------------------------------------------ forward
constexpr int FWD_THREADS = 512, FWD_STAGES = 2;

// Sum over the TPR threads of a row, the same in all of them.  The warps of a row meet at a named barrier of their own; `buf` has two
// halves that alternate, so one meeting per sum is enough.
template <int TPR>
__device__ __forceinline__ float group_sum(float v, float* buf, int& half) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  if (TPR == 32) return v;
  constexpr int W = TPR / 32;
  const int g = threadIdx.x / TPR;
  float* b = buf + (half * (FWD_THREADS / TPR) + g) * W;
  half ^= 1;
  if ((threadIdx.x & 31) == 0) b[(threadIdx.x % TPR) / 32] = v;
  asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "n"(TPR) : "memory");
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) s += b[i];
  return s;
}

template <typename T, int N, int TPR, int EPT, int BLOCKS, bool SHARED_PARAMS>
__global__ void __launch_bounds__(FWD_THREADS, BLOCKS) norm_forward_kernel(const NormArgs a) {
  using RW = Rows<T, N, TPR, EPT, FWD_THREADS>;
  extern __shared__ __align__(16) float param[];      // weight, then bias (unless they stay in global memory); then the ring
  __shared__ float buf[2 * FWD_THREADS / 32];
  constexpr int G = FWD_THREADS / TPR;
  const int t = threadIdx.x % TPR, pitch = SHARED_PARAMS ? (a.cols + 3) & ~3 : 0;
  const uint32_t ring = uint32_t(__cvta_generic_to_shared(param + 2 * pitch));
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.out);
  const int64_t step = int64_t(gridDim.x) * G;
  int64_t r = int64_t(blockIdx.x) * G + threadIdx.x / TPR;
  if (r < a.rows) RW::fetch(ring, x + r * a.ldx, t, a.cols);
  copy_commit();
  for (int c = threadIdx.x; SHARED_PARAMS && c < a.cols; c += FWD_THREADS) {
    param[c] = param_at(a.weight, a.param_dtype, 1.f, c);
    param[pitch + c] = param_at(a.bias, a.param_dtype, 0.f, c);
  }
  __syncthreads();
  const float inv = 1.f / float(a.cols);
  int half = 0;
  uint32_t stage = 0;
  for (; r < a.rows; r += step, stage ^= 1) {
    if (r + step < a.rows) RW::fetch(ring + (stage ^ 1) * RW::kStageBytes, x + (r + step) * a.ldx, t, a.cols);
    copy_commit();
    copy_wait<1>();
    float v[EPT], mean = 0.f;
    RW::take(v, ring + stage * RW::kStageBytes, x + r * a.ldx, t, a.cols);
    if (a.center) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < EPT; ++i) s[i & 1] += v[i];
      mean = group_sum<TPR>(s[0] + s[1], buf, half) * inv;
#pragma unroll
      for (int i = 0; i < EPT; ++i) v[i] -= mean;
    }
    float q[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < EPT / N; ++i)
      if ((i * TPR + t) * N < a.cols) {
#pragma unroll
        for (int e = 0; e < N; ++e) q[(i * N + e) & 1] = fmaf(v[i * N + e], v[i * N + e], q[(i * N + e) & 1]);
      }
    const float rstd = 1.f / sqrtf(group_sum<TPR>(q[0] + q[1], buf, half) * inv + a.eps);
#pragma unroll
    for (int i = 0; i < EPT / N; ++i) {
      const int c = (i * TPR + t) * N;
      if (c >= a.cols) continue;
      Pack<T, N> o;
      if constexpr (!SHARED_PARAMS) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          down(&o.v[e], fmaf(v[i * N + e] * rstd, param_at(a.weight, a.param_dtype, 1.f, c + e), param_at(a.bias, a.param_dtype, 0.f, c + e)));
      } else if constexpr (N >= 4) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
          const float4 w = *reinterpret_cast<const float4*>(param + c + e), b = *reinterpret_cast<const float4*>(param + pitch + c + e);
          down(&o.v[e], fmaf(v[i * N + e] * rstd, w.x, b.x));
          down(&o.v[e + 1], fmaf(v[i * N + e + 1] * rstd, w.y, b.y));
          down(&o.v[e + 2], fmaf(v[i * N + e + 2] * rstd, w.z, b.z));
          down(&o.v[e + 3], fmaf(v[i * N + e + 3] * rstd, w.w, b.w));
        }
      } else {
        down(&o.v[0], fmaf(v[i] * rstd, param[c], param[pitch + c]));
      }
      *reinterpret_cast<Pack<T, N>*>(y + r * a.ldo + c) = o;
    }
    if (t == 0) {
      if (a.mean) a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

// ------------------------------------------------------------------ backward
constexpr int BWD_EPT = 16, BWD_STAGES = 3;

// Two fp32 values in one instruction: half the issue slots of the arithmetic, which would otherwise bound the kernel.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 both(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// K = 2 or 4 sums over the threads of a row group (a warp, a block, or the two blocks of a cluster), the same in every thread.  Lanes trade
// values as they halve the distance, so K sums over a warp take K + 3 shuffles at most, and afterwards lane 32 / K * k holds sum k.  Two halves of
// `buf` alternate, so that a half is written again only after everybody has passed the meeting between.
template <int K, int TPR, int CLUSTER>
__device__ __forceinline__ void row_sums(float (&v)[K], float* buf, int& half) {
  static_assert(K == 2 || K == 4, "one or two rows");
  const int lane = threadIdx.x & 31;
  float z;
  if constexpr (K == 4) {
    const bool hi = lane & 16;
    const float a = (hi ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[2], 16);
    const float b = (hi ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, hi ? v[1] : v[3], 16);
    const bool mid = lane & 8;
    z = (mid ? b : a) + __shfl_xor_sync(0xffffffffu, mid ? a : b, 8);
  } else {
    const bool hi = lane & 16;
    z = (hi ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[1], 16);
    z += __shfl_xor_sync(0xffffffffu, z, 8);
  }
#pragma unroll
  for (int d = 4; d; d >>= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
  constexpr int S = 32 / K;                            // lanes of one sum
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32 * CLUSTER;
    float* b = buf + half * (K * W);
    half ^= 1;
    if constexpr (CLUSTER > 1) {
      cg::cluster_group cl = cg::this_cluster();
      if (lane % S < CLUSTER) cl.map_shared_rank(b, lane % S)[(lane / S) * W + int(cl.block_rank()) * (TPR / 32) + threadIdx.x / 32] = z;
      cl.sync();
    } else {
      if (lane % S == 0) b[(lane / S) * W + threadIdx.x / 32] = z;
      __syncthreads();
    }
    z = 0.f;
#pragma unroll
    for (int i = 0; i < (W + S - 1) / S; ++i)
      if (i * S + lane % S < W) z += b[(lane / S) * W + i * S + lane % S];
#pragma unroll
    for (int d = S / 2; d; d >>= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = __shfl_sync(0xffffffffu, z, k * S);
}

template <int TPR> struct Geometry {
  static constexpr int kGroups = TPR == 32 ? 8 : 1;   // row groups of a block
  static constexpr int kThreads = TPR * kGroups;
};
// Rows that a group takes at a time: what 32 registers of x and dy hold.
template <typename T, int N> constexpr int kRowsAtATime = sizeof(T) == 2 && N > 1 ? 2 : 1;

template <typename T, int N, int TPR, int CLUSTER, int BLOCKS>
__global__ void __launch_bounds__(Geometry<TPR>::kThreads, BLOCKS) norm_backward_kernel(const NormArgs a) {
  constexpr int G = Geometry<TPR>::kGroups, THREADS = Geometry<TPR>::kThreads, EPT = BWD_EPT, R = kRowsAtATime<T, N>, H = EPT / 2;
  using RW = Rows<T, N, TPR, EPT, THREADS>;
  extern __shared__ __align__(16) float dynamic[];    // the ring; one warp per row: at the end [8][2][32 * EPT] sums
  __shared__ float buf[2 * 2 * R * (TPR / 32) * CLUSTER];
  const int t = threadIdx.x % TPR;
  // the columns of this block: all of them, or a share that is a whole number of pieces
  const int width = CLUSTER == 1 ? a.cols : ((a.cols + CLUSTER - 1) / CLUSTER + 7) & ~7;
  const int c0 = CLUSTER == 1 ? 0 : int(blockIdx.x % CLUSTER) * width, cols = CLUSTER == 1 ? a.cols : max(0, min(width, a.cols - c0));
  const T* x = static_cast<const T*>(a.x) + c0;
  const T* dy = static_cast<const T*>(a.dy) + c0;
  T* dx = static_cast<T*>(a.out) + c0;
  const uint32_t ring = uint32_t(__cvta_generic_to_shared(dynamic));
  auto place = [&](uint32_t stage, int k, int which) { return ring + ((stage * R + k) * 2 + which) * uint32_t(RW::kStageBytes); };
  const int64_t step = int64_t(gridDim.x / CLUSTER) * G * R, r0 = (int64_t(blockIdx.x / CLUSTER) * G + threadIdx.x / TPR) * R;
  auto fetch = [&](uint32_t stage, int64_t r) {
#pragma unroll
    for (int k = 0; k < R; ++k) {                      // a row past the end is one of zeros
      const int has = r + k < a.rows ? cols : 0;
      RW::fetch(place(stage, k, 0), has ? x + (r + k) * a.ldx : x, t, has);
      RW::fetch(place(stage, k, 1), has ? dy + (r + k) * a.lddy : dy, t, has);
    }
    copy_commit();
  };
#pragma unroll
  for (int k = 0; k < BWD_STAGES - 1; ++k) fetch(k, r0 + k * step);
  uint64_t w[H], dw[H], db[H];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    float u[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int c = (((2 * i + e) / N) * TPR + t) * N + (2 * i + e) % N;
      u[e] = c < cols ? param_at(a.weight, a.param_dtype, 1.f, c0 + c) : 0.f;
    }
    w[i] = two(u[0], u[1]);
    dw[i] = db[i] = 0;
  }
  const float inv = 1.f / float(a.cols);
  float next_mean[R], next_rstd[R];
  auto statistics = [&](int64_t r) {                  // a row past the end has rstd = 0: it adds nothing
#pragma unroll
    for (int k = 0; k < R; ++k) {
      next_mean[k] = a.mean && r + k < a.rows ? a.mean[r + k] : 0.f;
      next_rstd[k] = r + k < a.rows ? a.rstd[r + k] : 0.f;
    }
  };
  statistics(r0);
  int half = 0;
  uint32_t stage = 0;
  for (int64_t r = r0; r < a.rows; r += step) {
    fetch((stage + BWD_STAGES - 1) % BWD_STAGES, r + (BWD_STAGES - 1) * step);
    float mean[R], rstd[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      mean[k] = next_mean[k];
      rstd[k] = next_rstd[k];
    }
    statistics(r + step);
    copy_wait<BWD_STAGES - 1>();
    float s[2 * R];
    Pack<T, N> px[R][EPT / N], py[R][EPT / N];
    // (x - mean, dy) of values 2 i and 2 i + 1; columns past the end have dy = 0 and weight 0
    auto pair = [&](int k, int i, uint64_t& xc, uint64_t& d) {
      xc = add2(two(up(px[k][2 * i / N].v[2 * i % N]), up(px[k][(2 * i + 1) / N].v[(2 * i + 1) % N])), two(-mean[k], -mean[k]));
      d = two(up(py[k][2 * i / N].v[2 * i % N]), up(py[k][(2 * i + 1) / N].v[(2 * i + 1) % N]));
    };
#pragma unroll
    for (int k = 0; k < R; ++k) {
      RW::raw(px[k], place(stage, k, 0), x + (r + k) * a.ldx, t, cols);
      RW::raw(py[k], place(stage, k, 1), dy + (r + k) * a.lddy, t, cols);
      uint64_t s0 = 0, s1 = 0;
#pragma unroll
      for (int i = 0; i < H; ++i) {
        uint64_t xc, d;
        pair(k, i, xc, d);
        dw[i] = fma2(mul2(xc, two(rstd[k], rstd[k])), d, dw[i]);
        db[i] = add2(db[i], d);
        const uint64_t g = mul2(d, w[i]);
        s0 = add2(s0, g);
        s1 = fma2(g, xc, s1);
      }
      const float2 f0 = both(s0), f1 = both(s1);
      s[2 * k] = f0.x + f0.y;
      s[2 * k + 1] = (f1.x + f1.y) * rstd[k];
    }
    stage = (stage + 1) % BWD_STAGES;
    row_sums<2 * R, TPR, CLUSTER>(s, buf, half);
#pragma unroll
    for (int k = 0; k < R; ++k) {                     // dx = rstd g - rstd mean(g) - (x - mean) rstd^2 mean(g xh)
      const float m1 = a.mean ? -rstd[k] * (s[2 * k] * inv) : 0.f, m2 = -rstd[k] * rstd[k] * (s[2 * k + 1] * inv);
      const int end = r + k < a.rows ? cols : 0;
      float v[EPT];
#pragma unroll
      for (int i = 0; i < H; ++i) {
        uint64_t xc, d;
        pair(k, i, xc, d);
        const float2 o = both(fma2(mul2(d, w[i]), two(rstd[k], rstd[k]), fma2(xc, two(m2, m2), two(m1, m1))));
        v[2 * i] = o.x;
        v[2 * i + 1] = o.y;
      }
#pragma unroll
      for (int i = 0; i < EPT / N; ++i) {
        const int c = (i * TPR + t) * N;
        if (c >= end) continue;
        Pack<T, N> o;
#pragma unroll
        for (int e = 0; e < N; ++e) down(&o.v[e], v[i * N + e]);
        *reinterpret_cast<Pack<T, N>*>(dx + (r + k) * a.ldo + c) = o;
      }
    }
  }
  cudaTriggerProgrammaticLaunchCompletion();           // the sums' kernel may take its place; it waits for this one's end
  if constexpr (CLUSTER > 1) cg::this_cluster().sync();    // nobody leaves while another may still write into its shared memory
  if (!a.parts) return;
  float* out = a.parts + int64_t(blockIdx.x / CLUSTER) * 2 * a.cols + c0;
  if constexpr (TPR == 32) {                          // add the block's warps in order
    const int wp = threadIdx.x / 32;
    copy_wait<0>();
    __syncthreads();                                  // the ring's memory is free
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const int c = ((i / N) * TPR + t) * N + i % N;
      const float2 fw = both(dw[i / 2]), fb = both(db[i / 2]);
      dynamic[(wp * 2) * (32 * EPT) + c] = i & 1 ? fw.y : fw.x;
      dynamic[(wp * 2 + 1) * (32 * EPT) + c] = i & 1 ? fb.y : fb.x;
    }
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * a.cols; j += blockDim.x) {
      const int which = j >= a.cols, c = j - which * a.cols;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < G; ++k) s += dynamic[(k * 2 + which) * (32 * EPT) + c];
      out[j] = s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const int c = ((i / N) * TPR + t) * N + i % N;
      if (c >= cols) continue;
      const float2 fw = both(dw[i / 2]), fb = both(db[i / 2]);
      out[c] = i & 1 ? fw.y : fw.x;
      out[a.cols + c] = i & 1 ? fb.y : fb.x;
    }
  }
}

// Adds the blocks' sums: 32 columns per block, 32 threads share a column's parts, in a fixed order.
__global__ void __launch_bounds__(1024) norm_parts_kernel(const float* parts, int n, int cols, void* dweight, void* dbias, int param_dtype) {
  __shared__ float sm[32][33];
  const int which = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
  void* out = which ? dbias : dweight;
  cudaGridDependencySynchronize();
  float s = 0.f;
  if (c < cols && out) {
    const float* at = parts + int64_t(which) * cols + c;
    const int64_t pitch = 2 * int64_t(cols);
#pragma unroll 10
    for (int k = threadIdx.y; k < n; k += 32) s += at[k * pitch];
  }
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
  // fp32 rows of more than 8192 columns: 128 KiB of ring, and as much again of weight and bias would not fit
  constexpr bool SHARED_PARAMS = !(N == 4 && EPT == 32);
  constexpr int BLOCKS = !SHARED_PARAMS ? 1 : EPT > 8 ? 2 : 3;
  const int bytes = (SHARED_PARAMS ? 2 * ((a.cols + 3) & ~3) * int(sizeof(float)) : 0) + FWD_STAGES * Rows<T, N, TPR, EPT, FWD_THREADS>::kStageBytes;
  // weight and bias of wide rows leave room for one block per SM only
  const int blocks = blocks_for(a.rows, FWD_THREADS / TPR, sms * (bytes * BLOCKS <= 216 * 1024 ? BLOCKS : bytes * 2 <= 216 * 1024 ? 2 : 1));
  auto kernel = norm_forward_kernel<T, N, TPR, EPT, BLOCKS, SHARED_PARAMS>;
  static SharedMemoryLimit limit;
  if (bytes > 40 * 1024 && !limit.raise(a.device, 220 * 1024, kernel)) return MUON_ERR_CUDA;
  kernel<<<blocks, FWD_THREADS, bytes, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

template <typename T, int N, int TPR, int BLOCKS, int CLUSTER = 1>
int backward(const NormArgs& a, int sms, cudaStream_t st) {
  using G = Geometry<TPR>;
  constexpr int R = kRowsAtATime<T, N>, ring = BWD_STAGES * R * 2 * Rows<T, N, TPR, BWD_EPT, G::kThreads>::kStageBytes, ends = TPR == 32 ? 8 * 2 * 32 * BWD_EPT * 4 : 0;
  constexpr int bytes = ring > ends ? ring : ends;
  const int most = sms * BLOCKS / CLUSTER < kNormMaxParts ? sms * BLOCKS / CLUSTER : kNormMaxParts;
  const int blocks = blocks_for(a.rows, G::kGroups * R, most);
  auto kernel = norm_backward_kernel<T, N, TPR, CLUSTER, BLOCKS>;
  static SharedMemoryLimit limit;
  if (bytes > 40 * 1024 && !limit.raise(a.device, bytes, kernel)) return MUON_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  cfg.stream = st;
  cfg.attrs = &at;
  if (blocks) {
    cfg.gridDim = dim3(unsigned(blocks * CLUSTER));
    cfg.blockDim = dim3(G::kThreads);
    cfg.dynamicSmemBytes = bytes;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = CLUSTER;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.numAttrs = CLUSTER > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) return MUON_ERR_CUDA;
  }
  if (!a.dweight && !a.dbias) return blocks ? 1 : 0;
  // launched while the blocks above still run (no rows: the sums are zero)
  cfg.gridDim = dim3(unsigned((a.cols + 31) / 32), 2);
  cfg.blockDim = dim3(32, 32);
  cfg.dynamicSmemBytes = 0;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = blocks ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, norm_parts_kernel, static_cast<const float*>(a.parts), blocks, a.cols, a.dweight, a.dbias, a.param_dtype) != cudaSuccess)
    return MUON_ERR_CUDA;
  return blocks ? 2 : 1;
}

// Values per thread: up to four pieces of 16 bytes, or 32 single elements; the widest fp32 rows take eight pieces.
template <typename T, int N>
int forward_by_cols(const NormArgs& a, int sms, cudaStream_t st) {
  constexpr int most = N == 1 ? 32 : 4 * N, least = N == 1 ? 8 : N;
  if (a.cols <= 32 * least) return forward<T, N, 32, least>(a, sms, st);
  if (a.cols <= 32 * most / 2) return forward<T, N, 32, most / 2>(a, sms, st);
  if (a.cols <= 32 * most) return forward<T, N, 32, most>(a, sms, st);
  if (a.cols <= 64 * most) return forward<T, N, 64, most>(a, sms, st);
  if (a.cols <= 128 * most) return forward<T, N, 128, most>(a, sms, st);
  if (a.cols <= 256 * most) return forward<T, N, 256, most>(a, sms, st);
  return forward<T, N, 512, most == 16 ? 32 : most>(a, sms, st);
}

template <typename T, int N>
int backward_by_cols(const NormArgs& a, int sms, cudaStream_t st) {
  if (a.cols <= 32 * BWD_EPT) return backward<T, N, 32, 2>(a, sms, st);
  if (a.cols <= 64 * BWD_EPT) return backward<T, N, 64, 4>(a, sms, st);
  if (a.cols <= 128 * BWD_EPT) return backward<T, N, 128, 4>(a, sms, st);
  if (a.cols <= 256 * BWD_EPT) return backward<T, N, 256, 2>(a, sms, st);
  if (a.cols <= 512 * BWD_EPT) return backward<T, N, 512, 1>(a, sms, st);
  return backward<T, N, 512, 1, 2>(a, sms, st);
}

bool pieces(const void* p, int64_t ld, int bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * bytes) % 16 == 0; }

// 16-byte accesses need 16-byte aligned rows that are a whole number of them; other rows go element by element.
bool vector_rows(const NormArgs& a) {
  const int e = a.dtype == MUON_DTYPE_BF16 ? 2 : 4;
  return (a.cols * e) % 16 == 0 && pieces(a.x, a.ldx, e) && pieces(a.out, a.ldo, e) && (!a.dy || pieces(a.dy, a.lddy, e));
}

}  // namespace

int norm_parts(int64_t rows, int cols) { return blocks_for(rows, cols <= 32 * BWD_EPT ? Geometry<32>::kGroups : 1, kNormMaxParts); }

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
