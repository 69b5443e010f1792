// Attention on CUDA cores, forward and backward: fp32 tensors (the accuracy anchor of the tensor-core kernels) and bf16 tensors whose
// strides, alignment or head size the tensor-core kernels do not take.  Products, softmax and sums in fp32.
//
// One pass over the keys with the running maximum m and sum l of the softmax: when a block of keys raises m to m', what is
// accumulated so far is multiplied by exp(m - m').  The backward pass forms P = exp(S - lse) anew; one kernel owns blocks of
// queries (dq), the other blocks of keys (dk, dv), so every result is summed by one thread in a fixed order, at the price of forming
// S and do v^T twice.
//
// A block owns 64 rows and streams 64 (32 in the backward pass of heads of more than 128) of the other side through shared memory.  256 threads
// as 16 x 16: thread (ty, tx) forms the scores of rows 4 ty .. 4 ty + 3 with the streamed rows tx, tx + 16, ..., four elements of the head at a
// time from either side (16 bytes per access, 64 multiply-adds for eight of them), and owns columns 4 tx .. 4 tx + 3 of every 64 of the
// results of its rows.  Probabilities pass between the two through shared memory, transposed; those of a row stay within its half warp.
// Tiles lie at a pitch of 4 past a multiple of 64, so that neither kind of access meets a bank twice.  Bound by the multiply-adds and their
// operands from shared memory.
// Measured, causal, fp32, 4096 tokens of 8 heads of 128: forward 990 us (34.7 TFLOP/s of the pairs that count), backward 4.2 ms (20.4 of five
// products, 28.6 of the seven issued); 4 x 512 tokens of 32/8 heads of 128: 291 us and 1.3 ms; 128 tokens of 4 heads of 64: 21 and 64 us, one
// block's walk.  Few key heads leave SMs without a block of keys: 2048 tokens of 8/2 heads of 256 670 us and 6.3 ms.
#include <cuda_bf16.h>

#include "layer_ops.h"

namespace muon {
namespace {

constexpr int ROWS = 64, THREADS = 256, PP = ROWS + 4;   // PP: pitch of transposed probabilities
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

__device__ __forceinline__ void madd(float4& acc, float x, const float4& y) {
  acc.x = fmaf(x, y.x, acc.x);
  acc.y = fmaf(x, y.y, acc.y);
  acc.z = fmaf(x, y.z, acc.z);
  acc.w = fmaf(x, y.w, acc.w);
}
__device__ __forceinline__ float dot(const float4& x, const float4& y, float s) {
  return fmaf(x.w, y.w, fmaf(x.z, y.z, fmaf(x.y, y.y, fmaf(x.x, y.x, s))));
}
__device__ __forceinline__ float at(const float4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Heads of up to 64 DT elements, tiles of `n` rows.
template <int DT> struct Tile {
  static constexpr int kPitch = 64 * DT + 4;
  __host__ __device__ static constexpr int floats(int n) { return n * kPitch; }
};

template <typename T> struct alignas(4 * sizeof(T)) Four { T v[4]; };

// Rows [r0, r0 + n) of a head into shared memory; rows before `from`, rows from `valid` on and elements past the head are zero, whatever memory
// holds there.
template <typename T, int DT>
__device__ __forceinline__ void load_rows(float* dst, const AttnTensor& t, int tb, int first, int head, int r0, int n, int valid, int dim,
                                          int from = 0) {
  const T* src = row_of<T>(t, tb, first + r0, head);
  const bool whole = dim % 4 == 0 && reinterpret_cast<uintptr_t>(src) % sizeof(Four<T>) == 0 && t.st % 4 == 0;
#pragma unroll 8
  for (int i = threadIdx.x; i < n * 16 * DT; i += THREADS) {
    const int r = i / (16 * DT), d = i % (16 * DT) * 4;
    float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r0 + r >= from && r0 + r < valid && d < dim) {
      const T* p = src + int64_t(r) * t.st + d;
      if (whole) {
        const Four<T> v = *reinterpret_cast<const Four<T>*>(p);
        w = make_float4(to_f(v.v[0]), to_f(v.v[1]), to_f(v.v[2]), to_f(v.v[3]));
      } else {
        w.x = to_f(p[0]);
        if (d + 1 < dim) w.y = to_f(p[1]);
        if (d + 2 < dim) w.z = to_f(p[2]);
        if (d + 3 < dim) w.w = to_f(p[3]);
      }
    }
    *reinterpret_cast<float4*>(dst + r * Tile<DT>::kPitch + d) = w;
  }
}

// s[i][j] = <x_(4 ty + i), y_(tx + 16 j)>
template <int DT, int J>
__device__ __forceinline__ void products(float (&s)[4][J], const float* x, const float* y, int dim) {
  constexpr int P = Tile<DT>::kPitch;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < J; ++j) s[i][j] = 0.f;
#pragma unroll 2
  for (int d = 0; d < dim; d += 4) {
    float4 u[4], v[J];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const float4*>(x + (4 * ty + i) * P + d);
#pragma unroll
    for (int j = 0; j < J; ++j) v[j] = *reinterpret_cast<const float4*>(y + (tx + 16 * j) * P + d);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) s[i][j] = dot(u[i], v[j], s[i][j]);
  }
}

// The transposed probabilities of this thread: element (row, streamed row) at p[streamed row * PP + row].
template <int J>
__device__ __forceinline__ void put(float* p, const float (&s)[4][J]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int j = 0; j < J; ++j) *reinterpret_cast<float4*>(p + (tx + 16 * j) * PP + 4 * ty) = make_float4(s[0][j], s[1][j], s[2][j], s[3][j]);
}

// acc += P Y over `n` streamed rows
template <int DT>
__device__ __forceinline__ void accumulate(float4 (&acc)[4][DT], const float* p, const float* y, int n) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll 4
  for (int k = 0; k < n; ++k) {
    const float4 w = *reinterpret_cast<const float4*>(p + k * PP + 4 * ty);
#pragma unroll
    for (int c = 0; c < DT; ++c) {
      const float4 v = *reinterpret_cast<const float4*>(y + k * Tile<DT>::kPitch + 4 * tx + 64 * c);
#pragma unroll
      for (int i = 0; i < 4; ++i) madd(acc[i][c], at(w, i), v);
    }
  }
}

template <int DT> __device__ __forceinline__ void clear(float4 (&acc)[4][DT]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DT; ++c) acc[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
}

// A row times `scale`; a `dead` one saw nothing and has met zeros times whatever the others hold.
template <typename T, int DT>
__device__ __forceinline__ void store_row(T* out, const float4 (&acc)[DT], float scale, bool dead, int dim) {
#pragma unroll
  for (int c = 0; c < DT; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 4 * int(threadIdx.x % 16) + 64 * c + e;
      if (d < dim) out[d] = from_f<T>(dead ? 0.f : at(acc[c], e) * scale);
    }
}

__device__ __forceinline__ const float* row_info(const AttnArgs& a, const AttnSeq& s, int si, int head, int row) {
  return a.rows + ((int64_t(s.tb) * a.hq + head) * attn_row_blocks(a) + (a.nseq ? s.q0 / kAttnRowBlock + si : 0) + row / kAttnRowBlock) * (2 * kAttnRowBlock) +
         row % kAttnRowBlock;
}

// This block's head, sequence and 64 rows; false past the end.  Heads vary fastest; within a batched call the blocks with most to do go first (the
// last queries, the first keys).
__device__ __forceinline__ bool find_work(const AttnArgs& a, bool keys, int* head, int* si, int* blk) {
  const int heads = keys ? a.hkv : a.hq, t = int(blockIdx.x / unsigned(heads));
  *head = int(blockIdx.x % unsigned(heads));
  if (!attn_find_block(a, t, ROWS, keys, si, blk)) return false;
  if (!a.nseq) {
    *si = t % a.batch;
    *blk = keys ? t / a.batch : (a.nq + ROWS - 1) / ROWS - 1 - t / a.batch;
  }
  return true;
}

template <typename T, int DT>
__global__ void __launch_bounds__(THREADS, DT <= 2 ? 2 : 1) attention_forward_simt_kernel(const __grid_constant__ AttnArgs a) {
  extern __shared__ __align__(16) float sm[];
  float* sq = sm;
  float* sk = sq + Tile<DT>::floats(ROWS);
  float* sv = sk + Tile<DT>::floats(ROWS);
  float* sp = sk;                                    // the keys are not needed any more when there are probabilities
  int head, si, blk;
  if (!find_work(a, false, &head, &si, &blk)) return;
  const AttnSeq s = attn_seq(a, si);
  const int kvh = head / (a.hq / a.hkv), tx = threadIdx.x % 16;
  const int r0 = blk * ROWS, row = r0 + int(threadIdx.x) / 16 * 4;
  load_rows<T, DT>(sq, a.q, s.tb, s.q0, head, r0, ROWS, s.qn, a.dim);
  int lo[4], hi[4];
  float m[4], l[4];
  float4 acc[4][DT];
  clear(acc);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = attn_key_lo(a, s, row + i);
    hi[i] = attn_key_hi(a, s, row + i);
    m[i] = -INFINITY;
    l[i] = 0.f;
  }
  const int last = min(r0 + ROWS, s.qn) - 1;
  const int klo = attn_key_lo(a, s, r0), khi = last >= r0 ? attn_key_hi(a, s, last) : 0;
  for (int c0 = klo / ROWS * ROWS; c0 < khi; c0 += ROWS) {
    __syncthreads();
    load_rows<T, DT>(sk, a.k, s.tb, s.k0, kvh, c0, ROWS, s.kn, a.dim);
    load_rows<T, DT>(sv, a.v, s.tb, s.k0, kvh, c0, ROWS, s.kn, a.dim);
    __syncthreads();
    float p[4][4];
    products<DT, 4>(p, sq, sk, a.dim);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = c0 + tx + 16 * j;
        p[i][j] = key >= lo[i] && key < hi[i] ? p[i][j] * a.scale : -INFINITY;
        top = fmaxf(top, p[i][j]);
      }
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float mn = fmaxf(m[i], top), base = mn == -INFINITY ? 0.f : mn;
      const float shrink = m[i] == -INFINITY ? 0.f : exp2f((m[i] - base) * kLog2e);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += p[i][j] = exp2f((p[i][j] - base) * kLog2e);
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      l[i] = l[i] * shrink + sum;
      m[i] = mn;
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        acc[i][c].x *= shrink;
        acc[i][c].y *= shrink;
        acc[i][c].z *= shrink;
        acc[i][c].w *= shrink;
      }
    }
    __syncthreads();                                 // everybody has read the keys
    put(sp, p);
    __syncwarp();
    accumulate(acc, sp, sv, min(ROWS, khi - c0));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (row + i >= s.qext) break;
    store_row<T, DT>(row_of<T>(a.o, s.tb, s.q0 + row + i, head), acc[i], 1.f / l[i], l[i] == 0.f, a.dim);
    if (tx == 0) a.lse[(int64_t(s.tb) * a.hq + head) * a.nq + s.q0 + row + i] = l[i] == 0.f ? -INFINITY : m[i] + logf(l[i]);
  }
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

template <int DT> constexpr int kStreamed = DT == 4 ? 32 : 64;   // rows streamed at a time in the backward pass

template <typename T, int DT>
__global__ void __launch_bounds__(THREADS, DT == 1 ? 2 : 1) attention_dq_simt_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int COLS = kStreamed<DT>, J = COLS / 16;
  extern __shared__ __align__(16) float sm[];
  float* sq = sm;
  float* sdo = sq + Tile<DT>::floats(ROWS);
  float* sk = sdo + Tile<DT>::floats(ROWS);
  float* sv = sk + Tile<DT>::floats(COLS);
  float* sds = sv;                                   // the values are not needed any more when there is dS
  int head, si, blk;
  if (!find_work(a, false, &head, &si, &blk)) return;
  const AttnSeq s = attn_seq(a, si);
  const int kvh = head / (a.hq / a.hkv), tx = threadIdx.x % 16;
  const int r0 = blk * ROWS, row = r0 + int(threadIdx.x) / 16 * 4;
  load_rows<T, DT>(sq, a.q, s.tb, s.q0, head, r0, ROWS, s.qn, a.dim);
  load_rows<T, DT>(sdo, a.dout, s.tb, s.q0, head, r0, ROWS, s.qn, a.dim);
  const float* info = row_info(a, s, si, head, row);  // four rows of one block of 128: row is a multiple of four
  const float c2 = a.scale * kLog2e;
  int lo[4], hi[4];
  float l2[4], delta[4];
  float4 acc[4][DT];
  clear(acc);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = attn_key_lo(a, s, row + i);
    hi[i] = attn_key_hi(a, s, row + i);
    l2[i] = info[i];
    delta[i] = info[kAttnRowBlock + i];
  }
  const int last = min(r0 + ROWS, s.qn) - 1;
  const int klo = attn_key_lo(a, s, r0), khi = last >= r0 ? attn_key_hi(a, s, last) : 0;
  for (int c0 = klo / COLS * COLS; c0 < khi; c0 += COLS) {
    __syncthreads();
    load_rows<T, DT>(sk, a.k, s.tb, s.k0, kvh, c0, COLS, s.kn, a.dim);
    load_rows<T, DT>(sv, a.v, s.tb, s.k0, kvh, c0, COLS, s.kn, a.dim);
    __syncthreads();
    float p[4][J], dp[4][J];
    products<DT, J>(p, sq, sk, a.dim);
    products<DT, J>(dp, sdo, sv, a.dim);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int key = c0 + tx + 16 * j;
        p[i][j] = key >= lo[i] && key < hi[i] ? exp2f(fmaf(p[i][j], c2, l2[i])) * (dp[i][j] + delta[i]) : 0.f;
      }
    __syncthreads();                                 // everybody has read the values
    put(sds, p);
    __syncwarp();
    accumulate(acc, sds, sk, min(COLS, khi - c0));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (row + i < s.qext) store_row<T, DT>(row_of<T>(a.dq, s.tb, s.q0 + row + i, head), acc[i], a.scale, hi[i] <= lo[i], a.dim);
}

template <typename T, int DT>
__global__ void __launch_bounds__(THREADS, DT == 1 ? 2 : 1) attention_dkv_simt_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int COLS = kStreamed<DT>, J = COLS / 16;
  extern __shared__ __align__(16) float sm[];
  float* sk = sm;
  float* sv = sk + Tile<DT>::floats(ROWS);
  float* sq = sv + Tile<DT>::floats(ROWS);
  float* sdo = sq + Tile<DT>::floats(COLS);
  float* sp = sdo + Tile<DT>::floats(COLS);
  float* sds = sp + COLS * PP;
  int kvh, si, blk;
  if (!find_work(a, true, &kvh, &si, &blk)) return;
  const AttnSeq s = attn_seq(a, si);
  const int group = a.hq / a.hkv, tx = threadIdx.x % 16;
  const int r0 = blk * ROWS, key = r0 + int(threadIdx.x) / 16 * 4;
  load_rows<T, DT>(sk, a.k, s.tb, s.k0, kvh, r0, ROWS, s.kn, a.dim);
  load_rows<T, DT>(sv, a.v, s.tb, s.k0, kvh, r0, ROWS, s.kn, a.dim);
  const float c2 = a.scale * kLog2e;
  const int c1 = min(r0 + ROWS, s.kn), blind = attn_blind(a, s);
  const int qlo = r0 < s.kn ? attn_query_lo(a, s, r0) : 0, qhi = r0 < s.kn ? attn_query_hi(a, s, c1) : 0;
  float4 dk[4][DT], dv[4][DT];
  clear(dk);
  clear(dv);
  for (int h = kvh * group; h < (kvh + 1) * group; ++h)
    for (int i0 = qlo / COLS * COLS; i0 < qhi; i0 += COLS) {
      __syncthreads();
      load_rows<T, DT>(sq, a.q, s.tb, s.q0, h, i0, COLS, s.qn, a.dim, blind);
      load_rows<T, DT>(sdo, a.dout, s.tb, s.q0, h, i0, COLS, s.qn, a.dim, blind);
      __syncthreads();
      float p[4][J], ds[4][J];
      products<DT, J>(p, sk, sq, a.dim);
      products<DT, J>(ds, sv, sdo, a.dim);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int i = i0 + tx + 16 * j;
        const bool in = i < s.qn;
        const float* info = row_info(a, s, si, h, in ? i : 0);
        const int lo = in ? attn_key_lo(a, s, i) : 0, hi = in ? attn_key_hi(a, s, i) : 0;
        const float l2 = info[0], delta = info[kAttnRowBlock];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool seen = key + e >= lo && key + e < hi;
          p[e][j] = seen ? exp2f(fmaf(p[e][j], c2, l2)) : 0.f;
          ds[e][j] = seen ? p[e][j] * (ds[e][j] + delta) : 0.f;
        }
      }
      put(sp, p);                                    // read by this half warp alone, before the next meeting
      put(sds, ds);
      __syncwarp();
      const int n = min(COLS, qhi - i0);
      accumulate(dv, sp, sdo, n);
      accumulate(dk, sds, sq, n);
    }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (key + i < s.kext) {
      const bool unseen = key + i >= s.kn || attn_query_hi(a, s, key + i + 1) <= attn_query_lo(a, s, key + i);
      store_row<T, DT>(row_of<T>(a.dk, s.tb, s.k0 + key + i, kvh), dk[i], a.scale, unseen, a.dim);
      store_row<T, DT>(row_of<T>(a.dv, s.tb, s.k0 + key + i, kvh), dv[i], 1.f, unseen, a.dim);
    }
}

template <typename K>
int run(K kernel, const AttnArgs& a, bool keys, int floats, SharedMemoryLimit& limit, cudaStream_t st) {
  const int64_t blocks = attn_max_blocks(a, ROWS, keys) * (keys ? a.hkv : a.hq);
  if (blocks == 0) return 0;
  if (blocks > 0x7fffffff) return MUON_ERR_UNSUPPORTED;
  const int bytes = int(sizeof(float)) * floats;
  if (!limit.raise(a.device, bytes, kernel)) return MUON_ERR_CUDA;
  kernel<<<unsigned(blocks), THREADS, bytes, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

template <typename T, int DT>
int forward(const AttnArgs& a, cudaStream_t st) {
  static SharedMemoryLimit limit;
  return run(attention_forward_simt_kernel<T, DT>, a, false, 3 * Tile<DT>::floats(ROWS), limit, st);
}

template <typename T, int DT>
int backward(const AttnArgs& a, cudaStream_t st) {
  constexpr int C = kStreamed<DT>, tiles = 2 * Tile<DT>::floats(ROWS) + 2 * Tile<DT>::floats(C);
  static SharedMemoryLimit limit_dq, limit_dkv;
  const int dq = run(attention_dq_simt_kernel<T, DT>, a, false, tiles, limit_dq, st);
  if (dq < 0) return dq;
  const int dkv = run(attention_dkv_simt_kernel<T, DT>, a, true, tiles + 2 * C * PP, limit_dkv, st);
  return dkv < 0 ? dkv : dq + dkv;
}

// Registers and shared memory are sized for heads of up to 64, 128 or 256 elements.
template <typename T>
int forward_by_dim(const AttnArgs& a, cudaStream_t st) {
  return a.dim <= 64 ? forward<T, 1>(a, st) : a.dim <= 128 ? forward<T, 2>(a, st) : forward<T, 4>(a, st);
}
template <typename T>
int backward_by_dim(const AttnArgs& a, cudaStream_t st) {
  return a.dim <= 64 ? backward<T, 1>(a, st) : a.dim <= 128 ? backward<T, 2>(a, st) : backward<T, 4>(a, st);
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
  return dtype == MUON_DTYPE_BF16 ? forward_by_dim<__nv_bfloat16>(a, st) : forward_by_dim<float>(a, st);
}

int launch_attention_backward_simt(const AttnArgs& a, int dtype, cudaStream_t st) {
  return dtype == MUON_DTYPE_BF16 ? backward_by_dim<__nv_bfloat16>(a, st) : backward_by_dim<float>(a, st);
}

}  // namespace muon
