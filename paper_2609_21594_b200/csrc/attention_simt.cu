// Attention on CUDA cores, forward and backward: fp32 tensors (the accuracy anchor of the tensor-core kernels) and bf16 tensors whose
// strides, alignment or head size the tensor-core kernels do not take.  Products, softmax and sums in fp32.
//
// One pass over the keys with the running maximum m and sum l of the softmax: when a block of keys raises m to m', what is
// accumulated so far is multiplied by exp(m - m').  The backward pass forms P = exp(S - lse) anew; one kernel owns blocks of
// queries (dq), the other blocks of keys (dk, dv), so every result is summed by one thread in a fixed order, at the price of forming
// S and do v^T twice.
//
// 16 rows per block of 128 threads: thread (r, c) of 16 x 8 holds scores c, c + 8, ... of row r and elements c, c + 8, ... of its
// accumulators; the 32 streamed rows lie in shared memory at an odd pitch.  Bound by shared-memory reads (two per multiply-add pair) and, for few
// rows, by the latency of one block's walk: causal, fp32 arithmetic, 4 x 512 tokens of 32/8 heads of 128: forward 1.68 ms (10 TFLOP/s), backward
// 6.4 ms; one row of 128 tokens of 4 heads of 64: 51 and 135 us.
#include <cuda_bf16.h>

#include "layer_ops.h"

namespace muon {
namespace {

constexpr int ROWS = 16, COLS = 32, THREADS = 128, LANES = 8, PER = COLS / LANES;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T>
__device__ __forceinline__ T* row_of(const AttnTensor& t, int b, int token, int head) {
  return static_cast<T*>(t.data) + int64_t(b) * t.sb + int64_t(token) * t.st + int64_t(head) * t.sh;
}

// Rows [r0, r0 + n) of a head into shared memory; rows from `valid` on are zero, whatever memory holds there.
template <typename T>
__device__ __forceinline__ void load_rows(float* dst, const AttnTensor& t, int tb, int first, int head, int r0, int n, int valid, int dim) {
  for (int i = threadIdx.x; i < n * dim; i += THREADS) {
    const int r = i / dim, d = i - r * dim;
    dst[r * (dim + 1) + d] = r0 + r < valid ? to_f(row_of<T>(t, tb, first + r0 + r, head)[d]) : 0.f;
  }
}

__device__ __forceinline__ float dot(const float* x, const float* y, int dim) {
  float s = 0.f;
#pragma unroll 8
  for (int d = 0; d < dim; ++d) s = fmaf(x[d], y[d], s);
  return s;
}

template <typename T, int NACC>
__global__ void __launch_bounds__(THREADS) attention_forward_simt_kernel(const AttnArgs a) {
  extern __shared__ float sm[];
  const int pitch = a.dim + 1;
  float* sq = sm;
  float* sk = sq + ROWS * pitch;
  float* sv = sk + COLS * pitch;
  float* sp = sv + COLS * pitch;                     // [ROWS][COLS + 1]
  int si, blk;
  if (!attn_find_block(a, blockIdx.x, ROWS, false, &si, &blk)) return;
  const AttnSeq s = attn_seq(a, si);
  const int head = blockIdx.y, kvh = head / (a.hq / a.hkv);
  const int r0 = blk * ROWS, r = threadIdx.x / LANES, c = threadIdx.x % LANES, row = r0 + r;
  load_rows<T>(sq, a.q, s.tb, s.q0, head, r0, ROWS, s.qn, a.dim);
  const int lo = attn_key_lo(a, s, row), hi = attn_key_hi(a, s, row);
  const int last = min(r0 + ROWS, s.qn) - 1;
  const int klo = attn_key_lo(a, s, r0), khi = last >= r0 ? attn_key_hi(a, s, last) : 0;
  float m = -INFINITY, l = 0.f, acc[NACC];
#pragma unroll
  for (int i = 0; i < NACC; ++i) acc[i] = 0.f;
  for (int c0 = klo / COLS * COLS; c0 < khi; c0 += COLS) {
    __syncthreads();
    load_rows<T>(sk, a.k, s.tb, s.k0, kvh, c0, COLS, s.kn, a.dim);
    load_rows<T>(sv, a.v, s.tb, s.k0, kvh, c0, COLS, s.kn, a.dim);
    __syncthreads();
    float sc[PER], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int key = c0 + c + j * LANES;
      sc[j] = key >= lo && key < hi ? dot(sq + r * pitch, sk + (c + j * LANES) * pitch, a.dim) * a.scale : -INFINITY;
      top = fmaxf(top, sc[j]);
    }
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float mn = fmaxf(m, top), base = mn == -INFINITY ? 0.f : mn;
    const float shrink = m == -INFINITY ? 0.f : exp2f((m - base) * kLog2e);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const float p = exp2f((sc[j] - base) * kLog2e);
      sp[r * (COLS + 1) + c + j * LANES] = p;
      sum += p;
    }
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    l = l * shrink + sum;
    m = mn;
    __syncwarp();                                    // the eight threads of a row are in one warp
#pragma unroll
    for (int i = 0; i < NACC; ++i) acc[i] *= shrink;
    for (int k = 0; k < COLS; ++k) {
      const float p = sp[r * (COLS + 1) + k];
#pragma unroll
      for (int i = 0; i < NACC; ++i)
        if (c + i * LANES < a.dim) acc[i] = fmaf(p, sv[k * pitch + c + i * LANES], acc[i]);
    }
    __syncwarp();
  }
  if (row >= s.qext) return;
  T* out = row_of<T>(a.o, s.tb, s.q0 + row, head);
#pragma unroll
  for (int i = 0; i < NACC; ++i)
    if (c + i * LANES < a.dim) out[c + i * LANES] = from_f<T>(l == 0.f ? 0.f : acc[i] / l);
  if (c == 0) a.lse[(int64_t(s.tb) * a.hq + head) * a.nq + s.q0 + row] = l == 0.f ? -INFINITY : m + logf(l);
}

// -lse in units of log 2 and -delta, delta = sum_d do o, into the padded row blocks: P = exp2(scale' S + (-lse)) and dS = P (dP + (-delta)) are
// then a multiply-add and an add.  Memory bound: do and o are read once.  LANES threads share a row, one 16-byte piece each (N elements); a block
// of 256 takes the 128 rows in PASSES, the loads of four of them in flight together.  Heads vary fastest over the blocks: a token's heads lie
// together in memory, and a block alone touches 256 bytes of every 8 KiB.  Rows that 16-byte pieces do not fit take one warp each (N = 1).
// 4096 tokens of 32 heads of 128 in bf16 (67 MB): 16 us, 4.2 TB/s; with one pass in flight instead of four 65 us.
template <typename T, int N, int LANES>
__global__ void __launch_bounds__(256, 4) attention_rows_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int AT_ONCE = 256 / LANES, PASSES = kAttnRowBlock / AT_ONCE;
  __shared__ float sums[kAttnRowBlock];
  cudaTriggerProgrammaticLaunchCompletion();            // the kernel after this one may set itself up; it waits for this one's end
  int si, blk;
  if (!attn_find_block(a, int(blockIdx.x / unsigned(a.hq)), kAttnRowBlock, false, &si, &blk)) return;
  const AttnSeq s = attn_seq(a, si);
  const int head = int(blockIdx.x % unsigned(a.hq)), lane = threadIdx.x % LANES, first = threadIdx.x / LANES;
  const int rows = s.qn - blk * kAttnRowBlock;          // that count
  const T* px = row_of<T>(a.dout, s.tb, s.q0 + blk * kAttnRowBlock + first, head) + lane * N;
  const T* py = row_of<T>(a.o, s.tb, s.q0 + blk * kAttnRowBlock + first, head) + lane * N;
  float lse = -INFINITY;
  if (int(threadIdx.x) < min(rows, kAttnRowBlock)) lse = a.lse[(int64_t(s.tb) * a.hq + head) * a.nq + s.q0 + blk * kAttnRowBlock + threadIdx.x];
  if constexpr (N > 1) {
    struct alignas(sizeof(T) * N) Piece { T v[N]; };
    const bool in = lane * N < a.dim;
    const int64_t sx = AT_ONCE * a.dout.st, sy = AT_ONCE * a.o.st;
#pragma unroll 1
    for (int p0 = 0; p0 < PASSES; p0 += 4) {
      Piece x[4], y[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        if (in && first + (p0 + p) * AT_ONCE < rows) {
          x[p] = *reinterpret_cast<const Piece*>(px + p * sx);
          y[p] = *reinterpret_cast<const Piece*>(py + p * sy);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) x[p].v[e] = y[p].v[e] = from_f<T>(0.f);
        }
      }
      px += 4 * sx;
      py += 4 * sy;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float d = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) d = fmaf(-to_f(x[p].v[e]), to_f(y[p].v[e]), d);
#pragma unroll
        for (int k = LANES / 2; k; k >>= 1) d += __shfl_xor_sync(0xffffffffu, d, k);
        if (lane == 0) sums[first + (p0 + p) * AT_ONCE] = d;
      }
    }
  } else {
    for (int p = 0; p < PASSES; ++p) {
      float d = 0.f;
      if (first + p * AT_ONCE < rows)
        for (int i = 0; i + lane < a.dim; i += LANES) d = fmaf(-to_f(px[p * AT_ONCE * a.dout.st + i]), to_f(py[p * AT_ONCE * a.o.st + i]), d);
#pragma unroll
      for (int k = LANES / 2; k; k >>= 1) d += __shfl_xor_sync(0xffffffffu, d, k);
      if (lane == 0) sums[first + p * AT_ONCE] = d;
    }
  }
  __syncthreads();
  if (threadIdx.x >= kAttnRowBlock) return;
  float* out = a.rows + ((int64_t(s.tb) * a.hq + head) * attn_row_blocks(a) + (a.nseq ? s.q0 / kAttnRowBlock + si : 0) + blk) * (2 * kAttnRowBlock);
  const bool seen = lse != -INFINITY;
  out[threadIdx.x] = seen ? -lse * kLog2e : -INFINITY;
  out[kAttnRowBlock + threadIdx.x] = seen ? sums[threadIdx.x] : 0.f;          // whatever a row that counts for nothing holds
}

template <typename T, int NACC>
__global__ void __launch_bounds__(THREADS) attention_dq_simt_kernel(const AttnArgs a) {
  extern __shared__ float sm[];
  const int pitch = a.dim + 1;
  float* sq = sm;
  float* sdo = sq + ROWS * pitch;
  float* sk = sdo + ROWS * pitch;
  float* sv = sk + COLS * pitch;
  float* sp = sv + COLS * pitch;
  int si, blk;
  if (!attn_find_block(a, blockIdx.x, ROWS, false, &si, &blk)) return;
  const AttnSeq s = attn_seq(a, si);
  const int head = blockIdx.y, kvh = head / (a.hq / a.hkv);
  const int r0 = blk * ROWS, r = threadIdx.x / LANES, c = threadIdx.x % LANES, row = r0 + r;
  load_rows<T>(sq, a.q, s.tb, s.q0, head, r0, ROWS, s.qn, a.dim);
  load_rows<T>(sdo, a.dout, s.tb, s.q0, head, r0, ROWS, s.qn, a.dim);
  const float* info = a.rows + ((int64_t(s.tb) * a.hq + head) * attn_row_blocks(a) + (a.nseq ? s.q0 / kAttnRowBlock + si : 0) + row / kAttnRowBlock) *
                                   (2 * kAttnRowBlock) + row % kAttnRowBlock;
  const float l2 = info[0], delta = info[kAttnRowBlock], c2 = a.scale * kLog2e;
  const int lo = attn_key_lo(a, s, row), hi = attn_key_hi(a, s, row);
  const int last = min(r0 + ROWS, s.qn) - 1;
  const int klo = attn_key_lo(a, s, r0), khi = last >= r0 ? attn_key_hi(a, s, last) : 0;
  float acc[NACC];
#pragma unroll
  for (int i = 0; i < NACC; ++i) acc[i] = 0.f;
  for (int c0 = klo / COLS * COLS; c0 < khi; c0 += COLS) {
    __syncthreads();
    load_rows<T>(sk, a.k, s.tb, s.k0, kvh, c0, COLS, s.kn, a.dim);
    load_rows<T>(sv, a.v, s.tb, s.k0, kvh, c0, COLS, s.kn, a.dim);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int k = c + j * LANES, key = c0 + k;
      float ds = 0.f;
      if (key >= lo && key < hi)
        ds = exp2f(fmaf(dot(sq + r * pitch, sk + k * pitch, a.dim), c2, l2)) * (dot(sdo + r * pitch, sv + k * pitch, a.dim) + delta);
      sp[r * (COLS + 1) + k] = ds;
    }
    __syncwarp();
    for (int k = 0; k < COLS; ++k) {
      const float ds = sp[r * (COLS + 1) + k];
#pragma unroll
      for (int i = 0; i < NACC; ++i)
        if (c + i * LANES < a.dim) acc[i] = fmaf(ds, sk[k * pitch + c + i * LANES], acc[i]);
    }
    __syncwarp();
  }
  if (row >= s.qext) return;
  T* out = row_of<T>(a.dq, s.tb, s.q0 + row, head);
#pragma unroll
  for (int i = 0; i < NACC; ++i)
    if (c + i * LANES < a.dim) out[c + i * LANES] = from_f<T>(acc[i] * a.scale);
}

template <typename T, int NACC>
__global__ void __launch_bounds__(THREADS) attention_dkv_simt_kernel(const AttnArgs a) {
  extern __shared__ float sm[];
  const int pitch = a.dim + 1;
  float* sk = sm;
  float* sv = sk + ROWS * pitch;
  float* sq = sv + ROWS * pitch;
  float* sdo = sq + COLS * pitch;
  float* sp = sdo + COLS * pitch;
  float* sds = sp + ROWS * (COLS + 1);
  int si, blk;
  if (!attn_find_block(a, blockIdx.x, ROWS, true, &si, &blk)) return;
  const AttnSeq s = attn_seq(a, si);
  const int kvh = blockIdx.y, group = a.hq / a.hkv;
  const int r0 = blk * ROWS, r = threadIdx.x / LANES, c = threadIdx.x % LANES, key = r0 + r;
  load_rows<T>(sk, a.k, s.tb, s.k0, kvh, r0, ROWS, s.kn, a.dim);
  load_rows<T>(sv, a.v, s.tb, s.k0, kvh, r0, ROWS, s.kn, a.dim);
  const float c2 = a.scale * kLog2e;
  const int c1 = min(r0 + ROWS, s.kn);
  const int qlo = r0 < s.kn ? attn_query_lo(a, s, r0) : 0, qhi = r0 < s.kn ? attn_query_hi(a, s, c1) : 0;
  float dk[NACC], dv[NACC];
#pragma unroll
  for (int i = 0; i < NACC; ++i) dk[i] = dv[i] = 0.f;
  for (int h = kvh * group; h < (kvh + 1) * group; ++h) {
    const float* info = a.rows + ((int64_t(s.tb) * a.hq + h) * attn_row_blocks(a) + (a.nseq ? s.q0 / kAttnRowBlock + si : 0)) * (2 * kAttnRowBlock);
    for (int i0 = qlo / COLS * COLS; i0 < qhi; i0 += COLS) {
      __syncthreads();
      load_rows<T>(sq, a.q, s.tb, s.q0, h, i0, COLS, s.qn, a.dim);
      load_rows<T>(sdo, a.dout, s.tb, s.q0, h, i0, COLS, s.qn, a.dim);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int q = c + j * LANES, i = i0 + q;
        float p = 0.f, ds = 0.f;
        if (i < s.qn && key >= attn_key_lo(a, s, i) && key < attn_key_hi(a, s, i)) {
          const float* at = info + i / kAttnRowBlock * (2 * kAttnRowBlock) + i % kAttnRowBlock;
          p = exp2f(fmaf(dot(sk + r * pitch, sq + q * pitch, a.dim), c2, at[0]));
          ds = p * (dot(sv + r * pitch, sdo + q * pitch, a.dim) + at[kAttnRowBlock]);
        }
        sp[r * (COLS + 1) + q] = p;
        sds[r * (COLS + 1) + q] = ds;
      }
      __syncwarp();
      for (int q = 0; q < COLS; ++q) {
        const float p = sp[r * (COLS + 1) + q], ds = sds[r * (COLS + 1) + q];
#pragma unroll
        for (int i = 0; i < NACC; ++i)
          if (c + i * LANES < a.dim) {
            dv[i] = fmaf(p, sdo[q * pitch + c + i * LANES], dv[i]);
            dk[i] = fmaf(ds, sq[q * pitch + c + i * LANES], dk[i]);
          }
      }
      __syncwarp();
    }
  }
  if (key >= s.kext) return;
  T* ok = row_of<T>(a.dk, s.tb, s.k0 + key, kvh);
  T* ov = row_of<T>(a.dv, s.tb, s.k0 + key, kvh);
#pragma unroll
  for (int i = 0; i < NACC; ++i)
    if (c + i * LANES < a.dim) {
      ok[c + i * LANES] = from_f<T>(dk[i] * a.scale);
      ov[c + i * LANES] = from_f<T>(dv[i]);
    }
}

template <typename K>
int run(K kernel, const AttnArgs& a, bool keys, int row_tiles, int score_tiles, cudaStream_t st) {
  const int64_t blocks = attn_max_blocks(a, ROWS, keys);
  if (blocks == 0) return 0;
  const int heads = keys ? a.hkv : a.hq;
  if (blocks > 0x7fffffff || heads > 65535) return MUON_ERR_UNSUPPORTED;
  const int bytes = int(sizeof(float)) * ((row_tiles * ROWS + 2 * COLS) * (a.dim + 1) + score_tiles * ROWS * (COLS + 1));
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return MUON_ERR_CUDA;
  kernel<<<dim3(unsigned(blocks), unsigned(heads)), THREADS, bytes, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

// Registers are sized for the head: 8, 16 or 32 accumulators for up to 64, 128 or 256 elements.
template <typename T>
int forward(const AttnArgs& a, cudaStream_t st) {
  if (a.dim <= 64) return run(attention_forward_simt_kernel<T, 8>, a, false, 1, 1, st);
  if (a.dim <= 128) return run(attention_forward_simt_kernel<T, 16>, a, false, 1, 1, st);
  return run(attention_forward_simt_kernel<T, 32>, a, false, 1, 1, st);
}

template <typename T>
int backward(const AttnArgs& a, cudaStream_t st) {
  const int dq = a.dim <= 64    ? run(attention_dq_simt_kernel<T, 8>, a, false, 2, 1, st)
                 : a.dim <= 128 ? run(attention_dq_simt_kernel<T, 16>, a, false, 2, 1, st)
                                : run(attention_dq_simt_kernel<T, 32>, a, false, 2, 1, st);
  if (dq < 0) return dq;
  const int dkv = a.dim <= 64    ? run(attention_dkv_simt_kernel<T, 8>, a, true, 2, 2, st)
                  : a.dim <= 128 ? run(attention_dkv_simt_kernel<T, 16>, a, true, 2, 2, st)
                                 : run(attention_dkv_simt_kernel<T, 32>, a, true, 2, 2, st);
  return dkv < 0 ? dkv : dq + dkv;
}

}  // namespace

int launch_attention_rows(const AttnArgs& a, int dtype, cudaStream_t st) {
  const int64_t blocks = attn_max_blocks(a, kAttnRowBlock, false) * a.hq;
  if (blocks == 0) return 0;
  if (blocks > 0x7fffffff) return MUON_ERR_UNSUPPORTED;
  const unsigned grid = unsigned(blocks);
  auto pieces = [&](const AttnTensor& t, int64_t e) {
    return reinterpret_cast<uintptr_t>(t.data) % 16 == 0 && t.sb * e % 16 == 0 && t.st * e % 16 == 0 && t.sh * e % 16 == 0;
  };
  if (dtype == MUON_DTYPE_FP32) attention_rows_kernel<float, 1, 32><<<grid, 256, 0, st>>>(a);
  else if (a.dim % 8 || a.dim > 128 || !pieces(a.dout, 2) || !pieces(a.o, 2)) attention_rows_kernel<__nv_bfloat16, 1, 32><<<grid, 256, 0, st>>>(a);
  else if (a.dim <= 64) attention_rows_kernel<__nv_bfloat16, 8, 8><<<grid, 256, 0, st>>>(a);
  else attention_rows_kernel<__nv_bfloat16, 8, 16><<<grid, 256, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

int launch_attention_forward_simt(const AttnArgs& a, int dtype, cudaStream_t st) {
  return dtype == MUON_DTYPE_BF16 ? forward<__nv_bfloat16>(a, st) : forward<float>(a, st);
}

int launch_attention_backward_simt(const AttnArgs& a, int dtype, cudaStream_t st) {
  return dtype == MUON_DTYPE_BF16 ? backward<__nv_bfloat16>(a, st) : backward<float>(a, st);
}

}  // namespace muon
