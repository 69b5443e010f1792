// Layer norm, forward and backward, with the reduction of the weight's and the bias's gradient.
//
//   forward:   xh = (x - mean) rstd,  y = xh w + b;  mean = sum x / n,  rstd = (sum (x - mean)^2 / n + eps)^-1/2   (no mean: RMS norm)
//   backward:  g = dy w,  dx = rstd (g - xh sum(g xh) / n - sum(g) / n),  dw = sum over rows dy xh,  db = sum over rows dy
//
// Memory bound: forward reads x and writes y, backward reads dy and x and writes dx, once each.  A row is held in the registers of the
// threads that own it, so the centred sum of squares is taken from the row itself, not from a difference of sums.  Rows in 16-byte
// pieces travel by bulk copies through a ring in shared memory: rows ahead cost no registers and one thread asks for them.
//
// Forward: a row belongs to 32 to 512 threads with at most four pieces each (32 values of bf16: more would leave too few warps to hide
// the chain of two sums).  The row groups of a block do not wait for one another; weight and bias lie in shared memory as fp32.
// 8192 x 4096 bf16, fp32 weight and bias: 26.7 to 28.7 us over several runs, 4.7 to 5.0 TB/s (a copy of the same size takes 24.8); 3001 x 5633 fp32
// (element by element): 34.3 us, 3.9 TB/s; 3000 x 12288 fp32: 64 us, 4.6 TB/s.
//
// Backward: a thread keeps its 16 columns for all its rows, so it adds dy xh and dy in registers.  Rows wider than 8192 columns are
// cut between the two blocks of a cluster, which exchange their sums through distributed shared memory.  The blocks' sums,
// [blocks][2][cols] fp32, are added in block order by a second kernel: no atomics, the same bits every time.
// 8192 x 4096 bf16: 48.6 to 49.5 us, 4.1 TB/s (an addition of two tensors of that size takes 32.9), about 4 us of it for the blocks' sums; the rest is
// the stream of two inputs, which neither fewer sums, more stages (3 to 6), one row at a time nor other block counts (46.4 us at best, in
// no launch shape that also holds for other sizes) changed by more than 5 %.  2048 x 14336 bf16: 61 us; 30000 x 300 fp32: 25 us.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "f32x2.cuh"
#include "layer_ops.h"
#include "tc_common.cuh"

namespace cg = cooperative_groups;

namespace muon {
namespace {

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void down(float* p, float v) { *p = v; }
__device__ __forceinline__ void down(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Values 2 i and 2 i + 1 of a thread's pieces.  Two bf16 share a word: the upper one is its fp32 value with the lower bits cleared.
template <typename T, int N>
__device__ __forceinline__ uint64_t pair_up(const Pack<T, N>* p, int i) {
  if constexpr (sizeof(T) == 2 && N > 1) {
    const uint32_t w = reinterpret_cast<const uint32_t*>(&p[2 * i / N])[2 * i % N / 2];
    return two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  } else {
    return two(up(p[2 * i / N].v[2 * i % N]), up(p[(2 * i + 1) / N].v[(2 * i + 1) % N]));
  }
}
template <typename T, int N>
__device__ __forceinline__ void pair_down(Pack<T, N>* p, int i, uint64_t v) {
  const float2 f = both(v);
  if constexpr (sizeof(T) == 2 && N > 1) {
    *reinterpret_cast<__nv_bfloat162*>(&p[2 * i / N].v[2 * i % N]) = __floats2bfloat162_rn(f.x, f.y);
  } else {
    down(&p[2 * i / N].v[2 * i % N], f.x);
    down(&p[(2 * i + 1) / N].v[(2 * i + 1) % N], f.y);
  }
}

__device__ __forceinline__ float param_at(const void* p, int dtype, float missing, int c) {
  if (!p) return missing;
  return dtype == MUON_DTYPE_BF16 ? up(static_cast<const __nv_bfloat16*>(p)[c]) : static_cast<const float*>(p)[c];
}

// Columns of thread t of a row: piece i of N elements starts at (i * TPR + t) * N.  Rows in 16-byte pieces come through a ring in shared
// memory: one thread of the row's group asks for whole rows ahead of time with bulk copies that arrive on an mbarrier.  Other rows
// (without the alignment) are read directly, element by element.
template <typename T, int N, int TPR, int EPT>
struct Rows {
  static constexpr bool kRing = N * sizeof(T) == 16;
  static constexpr int kPieces = EPT / N;
  static constexpr int kRowBytes = kRing ? TPR * kPieces * 16 : 0;      // room for a row of the widest kind
  __device__ static __forceinline__ void raw(Pack<T, N> (&p)[kPieces], uint32_t place, const T* row, int t, int cols) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int c = (i * TPR + t) * N;
      if constexpr (kRing) {
        uint32_t* u = reinterpret_cast<uint32_t*>(&p[i]);
        u[0] = u[1] = u[2] = u[3] = 0;
        if (c < cols)
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                       : "r"(place + uint32_t(i * TPR + t) * 16u));
      } else {
        if (c < cols) p[i].v[0] = row[c];
        else down(&p[i].v[0], 0.f);
      }
    }
  }
};

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// Bounded like every wait of the library; a copy that never arrives is recorded and the row computed from what is there.
__device__ __forceinline__ void await_copy(uint32_t bar, uint32_t phase, int32_t* status) {
  if (tc::mbar_try(bar, phase)) return;
  const long long t0 = clock64();
  while (!tc::mbar_try(bar, phase))
    if (clock64() - t0 > tc::WAIT_CYCLES) {
      atomicExch(status, 41);
      return;
    }
}

// ------------------------------------------------------------------ forward
// 512 threads and two or three blocks per SM.
constexpr int FWD_THREADS = 512;
// Rows asked for ahead, per row group.  fp32 rows of more than 8192 columns are 64 KiB, beside 128 KiB of weight and bias: one.
template <int N, int EPT> constexpr int kFwdStages = N == 4 && EPT == 32 ? 1 : 2;

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

template <typename T, int N, int TPR, int EPT, int BLOCKS>
__global__ void __launch_bounds__(FWD_THREADS, BLOCKS) norm_forward_kernel(const NormArgs a) {
  using RW = Rows<T, N, TPR, EPT>;
  extern __shared__ __align__(16) float param[];      // weight, then bias; then the ring
  __shared__ float buf[2 * FWD_THREADS / 32];
  constexpr int G = FWD_THREADS / TPR, STAGES = kFwdStages<N, EPT>;
  __shared__ __align__(8) uint64_t bars[G * STAGES];
  const int t = threadIdx.x % TPR, pitch = (a.cols + 3) & ~3;
  const int group = threadIdx.x / TPR;
  const uint32_t ring = uint32_t(__cvta_generic_to_shared(param + 2 * pitch)) + uint32_t(group * STAGES * RW::kRowBytes);
  const uint32_t bar = uint32_t(__cvta_generic_to_shared(bars + group * STAGES));
  if (threadIdx.x == 0) {
    for (int i = 0; i < G * STAGES; ++i) tc::mbar_init(uint32_t(__cvta_generic_to_shared(bars + i)), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int c = threadIdx.x; c < a.cols; c += FWD_THREADS) {
    // groups of four columns, the first groups of all pieces before the second ones: neighbouring threads read neighbouring 16 bytes
    const int at = N > 4 ? (c % N / 4 * (a.cols / N) + c / N) * 4 + c % 4 : c;
    param[at] = param_at(a.weight, a.param_dtype, 1.f, c);
    param[pitch + at] = param_at(a.bias, a.param_dtype, 0.f, c);
  }
  __syncthreads();
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.out);
  const int64_t step = int64_t(gridDim.x) * G;
  const int64_t r0 = int64_t(blockIdx.x) * G + group;
  auto fetch = [&](uint32_t stage, int64_t r) {
    if constexpr (RW::kRing)
      if (t == 0 && r < a.rows) {
        const uint32_t bytes = uint32_t(a.cols) * uint32_t(sizeof(T));
        tc::mbar_expect_tx(bar + stage * 8u, bytes);
        bulk_copy(ring + stage * uint32_t(RW::kRowBytes), x + r * a.ldx, bytes, bar + stage * 8u);
      }
  };
#pragma unroll
  for (int k = 0; k < STAGES; ++k) fetch(k, r0 + k * step);
  const float inv = 1.f / float(a.cols);
  int half = 0;
  uint32_t stage = 0, phase = 0;
  for (int64_t r = r0; r < a.rows; r += step) {
    if constexpr (RW::kRing) await_copy(bar + stage * 8u, phase, a.status);
    Pack<T, N> p[EPT / N];
    RW::raw(p, ring + stage * uint32_t(RW::kRowBytes), x + r * a.ldx, t, a.cols);
    uint64_t v[EPT / 2];
    float mean = 0.f;
#pragma unroll
    for (int i = 0; i < EPT / 2; ++i) v[i] = pair_up<T, N>(p, i);
    if (a.center) {
      uint64_t s[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < EPT / 2; ++i) s[i & 1] = add2(s[i & 1], v[i]);
      const float2 f = both(add2(s[0], s[1]));
      mean = group_sum<TPR>(f.x + f.y, buf, half) * inv;
#pragma unroll
      for (int i = 0; i < EPT / 2; ++i) v[i] = add2(v[i], twice(-mean));
    }
    // columns past the end are zeros that the mean has been taken from: they must not count
    if constexpr (N > 1) {
#pragma unroll
      for (int i = 0; i < EPT / N; ++i)
        if ((i * TPR + t) * N >= a.cols) {
#pragma unroll
          for (int e = 0; e < N / 2; ++e) v[i * N / 2 + e] = 0;
        }
    } else {
#pragma unroll
      for (int i = 0; i < EPT / 2; ++i) {
        const float2 f = both(v[i]);
        v[i] = two(2 * i * TPR + t < a.cols ? f.x : 0.f, (2 * i + 1) * TPR + t < a.cols ? f.y : 0.f);
      }
    }
    uint64_t q[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < EPT / 2; ++i) q[i & 1] = fma2(v[i], v[i], q[i & 1]);
    const float2 qq = both(add2(q[0], q[1]));
    const float rstd = 1.f / sqrtf(group_sum<TPR>(qq.x + qq.y, buf, half) * inv + a.eps);
    if constexpr (TPR == 32) __syncwarp();
    fetch(stage, r + STAGES * step);              // everybody has read the row: the sum above was a meeting
    if (++stage == STAGES) {
      stage = 0;
      phase ^= 1;
    }
    auto scaled = [&](int i, float w0, float w1, float b0, float b1) {
      pair_down<T, N>(p, i, fma2(mul2(v[i], twice(rstd)), two(w0, w1), two(b0, b1)));
    };
    T* out = y + r * a.ldo;
    if constexpr (N == 1) {
#pragma unroll
      for (int i = 0; i < EPT / 2; ++i) {
        const int c = (2 * i / N * TPR + t) * N + 2 * i % N, d = ((2 * i + 1) / N * TPR + t) * N + (2 * i + 1) % N;
        const bool ci = c < a.cols, di = d < a.cols;
        scaled(i, ci ? param[c] : 0.f, di ? param[d] : 0.f, ci ? param[pitch + c] : 0.f, di ? param[pitch + d] : 0.f);
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPT / 4; ++i) {
        const int piece = min(4 * i / N * TPR + t, a.cols / N - 1), c = (4 * i % N) * (a.cols / N) + piece * 4;
        const float4 w = *reinterpret_cast<const float4*>(param + c), b = *reinterpret_cast<const float4*>(param + pitch + c);
        scaled(2 * i, w.x, w.y, b.x, b.y);
        scaled(2 * i + 1, w.z, w.w, b.z, b.w);
      }
    }
#pragma unroll
    for (int i = 0; i < EPT / N; ++i) {
      const int c = (i * TPR + t) * N;
      if (c < a.cols) *reinterpret_cast<Pack<T, N>*>(out + c) = p[i];
    }
    if (t == 0) {
      if (a.mean) a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

// ------------------------------------------------------------------ backward
constexpr int BWD_EPT = 16, BWD_STAGES = 3;

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

// JOIN > 1: the launch is one cluster of that many blocks, which add their sums through distributed shared memory and write the gradients.
template <typename T, int N, int TPR, int CLUSTER, int BLOCKS, int JOIN>
__global__ void __launch_bounds__(Geometry<TPR>::kThreads, BLOCKS) norm_backward_kernel(const NormArgs a) {
  constexpr int G = Geometry<TPR>::kGroups, EPT = BWD_EPT, R = kRowsAtATime<T, N>, H = EPT / 2;
  using RW = Rows<T, N, TPR, EPT>;
  extern __shared__ __align__(16) float dynamic[];    // the ring; one warp per row: at the end [8][2][32 * EPT] sums
  __shared__ float buf[2 * 2 * R * (TPR / 32) * CLUSTER];
  const int t = threadIdx.x % TPR;
  // the columns of this block: all of them, or a share that is a whole number of pieces
  const int width = CLUSTER == 1 ? a.cols : ((a.cols + CLUSTER - 1) / CLUSTER + 7) & ~7;
  const int c0 = CLUSTER == 1 ? 0 : int(blockIdx.x % CLUSTER) * width, cols = CLUSTER == 1 ? a.cols : max(0, min(width, a.cols - c0));
  const T* x = static_cast<const T*>(a.x) + c0;
  const T* dy = static_cast<const T*>(a.dy) + c0;
  T* dx = static_cast<T*>(a.out) + c0;
  __shared__ __align__(8) uint64_t bars[G * BWD_STAGES];
  const int group = threadIdx.x / TPR;
  const uint32_t ring = uint32_t(__cvta_generic_to_shared(dynamic)) + uint32_t(group * BWD_STAGES * R * 2 * RW::kRowBytes);
  const uint32_t bar = uint32_t(__cvta_generic_to_shared(bars + group * BWD_STAGES));
  if (threadIdx.x == 0) {
    for (int i = 0; i < G * BWD_STAGES; ++i) tc::mbar_init(uint32_t(__cvta_generic_to_shared(bars + i)), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // The sums of a row are stored into the other block's shared memory, which may be touched only once that block runs: the cluster meets here.
  if constexpr (CLUSTER > 1) cg::this_cluster().sync();
  else __syncthreads();
  auto place = [&](uint32_t stage, int k, int which) { return ring + ((stage * R + k) * 2 + which) * uint32_t(RW::kRowBytes); };
  const int64_t step = int64_t(gridDim.x / CLUSTER) * G * R, r0 = (int64_t(blockIdx.x / CLUSTER) * G + group) * R;
  auto fetch = [&](uint32_t stage, int64_t r) {
    if constexpr (RW::kRing)
      if (t == 0 && r < a.rows && cols > 0) {
        const uint32_t bytes = uint32_t(cols) * uint32_t(sizeof(T)), rows = R == 2 && r + 1 < a.rows ? 2 : 1;
        tc::mbar_expect_tx(bar + stage * 8u, 2 * rows * bytes);
        for (uint32_t k = 0; k < rows; ++k) {
          bulk_copy(place(stage, k, 0), x + (r + k) * a.ldx, bytes, bar + stage * 8u);
          bulk_copy(place(stage, k, 1), dy + (r + k) * a.lddy, bytes, bar + stage * 8u);
        }
      }
  };
#pragma unroll
  for (int k = 0; k < BWD_STAGES; ++k) fetch(k, r0 + k * step);
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
  // Lane 2 k + 1 of every warp holds rstd of row k, lane 2 k its mean, two steps ahead; a row past the end has rstd = 0 and adds nothing.
  auto statistic = [&](int64_t r) {
    const int lane = threadIdx.x & 31;
    const float* from = lane & 1 ? a.rstd : a.mean;
    return lane < 2 * R && from && r + lane / 2 < a.rows ? from[r + lane / 2] : 0.f;
  };
  float stat = statistic(r0), stat_next = statistic(r0 + step);
  int half = 0;
  uint32_t stage = 0, phase = 0;
  for (int64_t r = r0; r < a.rows; r += step) {
    float mean[R], rstd[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      mean[k] = __shfl_sync(0xffffffffu, stat, 2 * k);
      rstd[k] = __shfl_sync(0xffffffffu, stat, 2 * k + 1);
    }
    stat = stat_next;
    stat_next = statistic(r + 2 * step);
    if constexpr (RW::kRing)
      if (cols > 0) await_copy(bar + stage * 8u, phase, a.status);
    float s[2 * R];
    Pack<T, N> px[R][EPT / N], py[R][EPT / N];        // columns past the end have dy = 0 and weight 0
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int has = r + k < a.rows ? cols : 0;      // a row past the end is one of zeros
      RW::raw(px[k], place(stage, k, 0), x + (r + k) * a.ldx, t, has);
      RW::raw(py[k], place(stage, k, 1), dy + (r + k) * a.lddy, t, has);
      uint64_t s0 = 0, s1 = 0;
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const uint64_t xc = add2(pair_up<T, N>(px[k], i), twice(-mean[k])), d = pair_up<T, N>(py[k], i);
        dw[i] = fma2(mul2(xc, twice(rstd[k])), d, dw[i]);
        db[i] = add2(db[i], d);
        const uint64_t g = mul2(d, w[i]);
        s0 = add2(s0, g);
        s1 = fma2(g, xc, s1);
      }
      const float2 f0 = both(s0), f1 = both(s1);
      s[2 * k] = f0.x + f0.y;
      s[2 * k + 1] = (f1.x + f1.y) * rstd[k];
    }
    row_sums<2 * R, TPR, CLUSTER>(s, buf, half);
    fetch(stage, r + BWD_STAGES * step);              // everybody has read the rows: the sums above were a meeting
    if (++stage == BWD_STAGES) {
      stage = 0;
      phase ^= 1;
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {                     // dx = rstd g - rstd mean(g) - (x - mean) rstd^2 mean(g xh)
      const float m1 = a.mean ? -rstd[k] * (s[2 * k] * inv) : 0.f, m2 = -rstd[k] * rstd[k] * (s[2 * k + 1] * inv);
      const int end = r + k < a.rows ? cols : 0;
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const uint64_t xc = add2(pair_up<T, N>(px[k], i), twice(-mean[k])), g = mul2(pair_up<T, N>(py[k], i), w[i]);
        pair_down<T, N>(px[k], i, fma2(g, twice(rstd[k]), fma2(xc, twice(m2), twice(m1))));
      }
#pragma unroll
      for (int i = 0; i < EPT / N; ++i) {
        const int c = (i * TPR + t) * N;
        if (c < end) *reinterpret_cast<Pack<T, N>*>(dx + (r + k) * a.ldo + c) = px[k][i];
      }
    }
  }
  if constexpr (JOIN == 1) cudaTriggerProgrammaticLaunchCompletion();   // the sums' kernel may take its place; it waits for this one's end
  if constexpr (CLUSTER > 1) cg::this_cluster().sync();    // nobody leaves while another may still write into its shared memory
  if (JOIN > 1 ? !a.dweight && !a.dbias : !a.parts) return;
  float* out = JOIN > 1 ? nullptr : a.parts + int64_t(blockIdx.x / CLUSTER) * 2 * a.cols + c0;
  if constexpr (TPR == 32) {                          // add the block's warps in order
    const int wp = threadIdx.x / 32;
    __syncthreads();                                  // the ring's memory is free
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const int c = ((i / N) * TPR + t) * N + i % N;
      const float2 fw = both(dw[i / 2]), fb = both(db[i / 2]);
      dynamic[(wp * 2) * (32 * EPT) + c] = i & 1 ? fw.y : fw.x;
      dynamic[(wp * 2 + 1) * (32 * EPT) + c] = i & 1 ? fb.y : fb.x;
    }
    __syncthreads();
    auto block_sum = [&](int j) {
      const int which = j >= a.cols, c = j - which * a.cols;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < G; ++k) s += dynamic[(k * 2 + which) * (32 * EPT) + c];
      return s;
    };
    if constexpr (JOIN > 1) {
      float* joined = dynamic + G * 2 * 32 * EPT;     // [2][cols]
      for (int j = threadIdx.x; j < 2 * a.cols; j += blockDim.x) joined[j] = block_sum(j);
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();
      for (int j = int(cl.block_rank()) * blockDim.x + threadIdx.x; j < 2 * a.cols; j += JOIN * blockDim.x) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < JOIN; ++k) s += cl.map_shared_rank(joined, k)[j];
        void* to = j >= a.cols ? a.dbias : a.dweight;
        const int c = j >= a.cols ? j - a.cols : j;
        if (!to) continue;
        if (a.param_dtype == MUON_DTYPE_BF16) down(static_cast<__nv_bfloat16*>(to) + c, s);
        else static_cast<float*>(to)[c] = s;
      }
      cl.sync();                                      // nobody leaves while another still reads its sums
    } else {
      for (int j = threadIdx.x; j < 2 * a.cols; j += blockDim.x) out[j] = block_sum(j);
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

// Adds the blocks' sums: 32 columns per block, 32 threads share a column's parts, in a fixed order.  Bound by latency: 296 parts of 4096 columns
// (9.7 MB) in about 4 us from the second-level cache (9.4 us when they have to come from memory); its start hides behind the kernel before it.
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
  constexpr int BLOCKS = kFwdStages<N, EPT> == 1 ? 1 : EPT > 8 ? 2 : 3;
  const int bytes = 2 * ((a.cols + 3) & ~3) * int(sizeof(float)) + kFwdStages<N, EPT> * (FWD_THREADS / TPR) * Rows<T, N, TPR, EPT>::kRowBytes;
  // weight and bias of wide rows leave room for one block per SM only
  const int blocks = blocks_for(a.rows, FWD_THREADS / TPR, sms * (bytes * BLOCKS <= 216 * 1024 ? BLOCKS : bytes * 2 <= 216 * 1024 ? 2 : 1));
  auto kernel = norm_forward_kernel<T, N, TPR, EPT, BLOCKS>;
  static SharedMemoryLimit limit;
  if (bytes > 40 * 1024 && !limit.raise(a.device, 220 * 1024, kernel)) return MUON_ERR_CUDA;
  kernel<<<blocks, FWD_THREADS, bytes, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

template <typename T, int N, int TPR, int BLOCKS, int CLUSTER = 1, int JOIN = 1>
int backward(const NormArgs& a, int sms, cudaStream_t st) {
  using G = Geometry<TPR>;
  constexpr int R = kRowsAtATime<T, N>;
  constexpr int ring = BWD_STAGES * R * 2 * G::kGroups * Rows<T, N, TPR, BWD_EPT>::kRowBytes, ends = TPR == 32 ? (8 + (JOIN > 1)) * 2 * 32 * BWD_EPT * 4 : 0;
  constexpr int bytes = ring > ends ? ring : ends;
  const int most = sms * BLOCKS / CLUSTER < kNormMaxParts ? sms * BLOCKS / CLUSTER : kNormMaxParts;
  const int blocks = JOIN > 1 ? JOIN : blocks_for(a.rows, G::kGroups * R, most);
  auto kernel = norm_backward_kernel<T, N, TPR, CLUSTER, BLOCKS, JOIN>;
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
    at.val.clusterDim.x = CLUSTER * JOIN;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.numAttrs = CLUSTER * JOIN > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) return MUON_ERR_CUDA;
  }
  if (JOIN > 1 || (!a.dweight && !a.dbias)) return blocks ? 1 : 0;
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
  if (a.cols <= 512 * most) return forward<T, N, 512, most>(a, sms, st);
  return forward<T, N, 512, 32>(a, sms, st);
}

// Few narrow rows: one cluster of eight blocks and one launch, no scratch.  Up to 128 rows that is faster on the device and in a call, from 192 on the device
// takes longer and from 256 to 512 the call does too.  Joined against two launches, device (replayed in a graph) and call, us:
//   fp32, 256 columns:  8 rows 4.1 - 4.6, 6.7 - 9.6;  128: 4.6 - 4.9, 6.7 - 9.3;  192: 5.2 - 4.9, 8.2 - 9.5;  512: 8.4 - 5.4, 10.3 - 9.3
//   fp32, 512 columns:  8 rows 4.5 - 4.9, 6.7 - 9.6;  128: 5.2 - 5.2, 8.2 - 9.7;  192: 6.2 - 5.2, 8.2 - 10.1; 512: 9.0 - 5.5, 11.4 - 9.6
//   bf16, 512 columns:  8 rows 5.2 - 5.4, 7.1 - 9.7;  128: 5.9 - 6.4, 8.2 - 9.4;  192: 7.4 - 6.4, 10.2 - 9.4; 512: 10.6 - 6.5, 12.9 - 9.6
constexpr int64_t kJoinRows = 128;
bool joins(int64_t rows, int cols) { return cols <= 32 * BWD_EPT && rows > 0 && rows <= kJoinRows; }

template <typename T, int N>
int backward_by_cols(const NormArgs& a, int sms, cudaStream_t st) {
  if (joins(a.rows, a.cols)) return backward<T, N, 32, 2, 1, 8>(a, sms, st);
  if (a.cols <= 32 * BWD_EPT) return backward<T, N, 32, 2>(a, sms, st);
  if (a.cols <= 64 * BWD_EPT) return backward<T, N, 64, 4>(a, sms, st);
  if (a.cols <= 128 * BWD_EPT) return backward<T, N, 128, 4>(a, sms, st);
  if (a.cols <= 256 * BWD_EPT) return backward<T, N, 256, 2>(a, sms, st);
  if (a.cols <= 512 * BWD_EPT) return backward<T, N, 512, 1>(a, sms, st);
  return backward<T, N, 512, 1, 2>(a, sms, st);
}

bool pieces(const void* p, int64_t ld, int bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * bytes) % 16 == 0; }

// 16-byte accesses need 16-byte aligned rows that are a whole number of them; other rows go element by element.  8192 rows of bf16:
// 4096 columns 26.7 to 28.7 us by pieces, 4095 columns 47.5 to 51.5 by elements; 3001 rows of fp32: 5632 columns 30.2 to 31.2, 5633 columns 36.4.
bool vector_rows(const NormArgs& a) {
  const int e = a.dtype == MUON_DTYPE_BF16 ? 2 : 4;
  return (a.cols * e) % 16 == 0 && pieces(a.x, a.ldx, e) && pieces(a.out, a.ldo, e) && (!a.dy || pieces(a.dy, a.lddy, e));
}

}  // namespace

int norm_parts(int64_t rows, int cols) { return joins(rows, cols) ? 0 : blocks_for(rows, cols <= 32 * BWD_EPT ? Geometry<32>::kGroups : 1, kNormMaxParts); }

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
