// Rotary positions of up to four tensors that share them, one launch.
//
// Memory bound: every element is read and written once.  A block takes a few tokens; it first forms the cosines and sines of its
// tokens in shared memory (one per token and pair, for all heads of all tensors), then turns the pairs.  The angle position * inv_freq
// is formed in whole turns and in double, its fraction taken there, and only the fraction goes to sincospif in fp32: a product in fp32
// would be off by position * 2^-24 radians, 0.06 at a million.
#include <cuda_bf16.h>

#include "layer_ops.h"

namespace muon {
namespace {

constexpr int THREADS = 256;

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void down(float* p, float v) { *p = v; }
__device__ __forceinline__ void down(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// A work item is N pairs of one head (2 N elements in two pieces), or, past the rotary part, N elements to copy.
template <typename T, int N, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS) rotary_kernel(const __grid_constant__ RotaryArgs a, int tokens_per_block) {
  extern __shared__ float2 turn[];                     // [tokens_per_block][pairs]
  const int64_t total = int64_t(a.batch) * a.tokens, t0 = int64_t(blockIdx.x) * tokens_per_block;
  const int n = int(total - t0 < tokens_per_block ? total - t0 : tokens_per_block);
  for (int i = threadIdx.x; i < n * a.pairs; i += THREADS) {
    const int64_t tok = t0 + i / a.pairs;
    const int64_t pos = a.position_offset + (a.positions ? int64_t(a.positions[tok]) : tok % a.tokens);
    const double x = double(pos) * a.turns[i % a.pairs];
    float s, c;
    sincospif(2.f * float(x - rint(x)), &s, &c);
    turn[i] = make_float2(c * a.amplitude, (a.inverse ? -s : s) * a.amplitude);
  }
  __syncthreads();
  const int heads = a.head_begin[a.count];
  const int turned = a.pairs / N, rest = (a.head_dim - 2 * a.pairs + N - 1) / N, per = turned + rest;
  for (int i = threadIdx.x; i < n * heads * per; i += THREADS) {
    const int w = i % per, h = i / per % heads, l = i / (per * heads);
    int k = 0;
    while (h >= a.head_begin[k + 1]) ++k;
    const muon_rotary_item_t& it = a.item[k];
    const int64_t tok = t0 + l, b = tok / a.tokens, at = tok - b * a.tokens, hh = h - a.head_begin[k];
    const T* in = static_cast<const T*>(it.in.data) + b * it.in.batch_stride + at * it.in.token_stride + hh * it.in.head_stride;
    T* out = static_cast<T*>(it.out.data) + b * it.out.batch_stride + at * it.out.token_stride + hh * it.out.head_stride;
    if (w >= turned) {
      const int d = 2 * a.pairs + (w - turned) * N;
      if (in != out) *reinterpret_cast<Pack<T, N>*>(out + d) = *reinterpret_cast<const Pack<T, N>*>(in + d);
      continue;
    }
    const float2* cs = turn + l * a.pairs + w * N;
    const int da = INTERLEAVED ? 2 * w * N : w * N, db = INTERLEAVED ? da + N : da + a.pairs;
    Pack<T, N> x = *reinterpret_cast<const Pack<T, N>*>(in + da), y = *reinterpret_cast<const Pack<T, N>*>(in + db), u, v;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      // interleaved: the 2 N elements are x then y, element 2 e and 2 e + 1 of them form pair e
      const T p = INTERLEAVED ? (2 * e < N ? x.v[(2 * e) % N] : y.v[(2 * e) % N]) : x.v[e];
      const T q = INTERLEAVED ? (2 * e + 1 < N ? x.v[(2 * e + 1) % N] : y.v[(2 * e + 1) % N]) : y.v[e];
      const float f = up(p), g = up(q);
      const float r = f * cs[e].x - g * cs[e].y, s = f * cs[e].y + g * cs[e].x;
      if constexpr (INTERLEAVED) {
        down(2 * e < N ? &u.v[(2 * e) % N] : &v.v[(2 * e) % N], r);
        down(2 * e + 1 < N ? &u.v[(2 * e + 1) % N] : &v.v[(2 * e + 1) % N], s);
      } else {
        down(&u.v[e], r);
        down(&v.v[e], s);
      }
    }
    *reinterpret_cast<Pack<T, N>*>(out + da) = u;
    *reinterpret_cast<Pack<T, N>*>(out + db) = v;
  }
}

bool vector_heads(const RotaryArgs& a, int n, int bytes) {
  if (a.pairs % n || a.head_dim % n) return false;
  for (int k = 0; k < a.count; ++k)
    for (const muon_heads_t* t : {&a.item[k].in, &a.item[k].out})
      if (reinterpret_cast<uintptr_t>(t->data) % 16 || t->batch_stride * bytes % 16 || t->token_stride * bytes % 16 || t->head_stride * bytes % 16)
        return false;
  return true;
}

template <typename T, int N>
int run(const RotaryArgs& a, int sms, cudaStream_t st) {
  const int64_t total = int64_t(a.batch) * a.tokens;
  const int per_token = a.head_begin[a.count] * (a.pairs / N + (a.head_dim - 2 * a.pairs + N - 1) / N);
  // four items per thread and block, but no fewer blocks than SMs, and at most 16 KiB of cosines and sines
  int64_t tpb = (4 * THREADS + per_token - 1) / per_token;
  const int64_t spread = (total + sms - 1) / sms;
  if (tpb > spread) tpb = spread;
  if (tpb > 2048 / a.pairs) tpb = 2048 / a.pairs;
  if (tpb < 1) tpb = 1;
  const int64_t blocks = (total + tpb - 1) / tpb;
  if (blocks > 0x7fffffff) return MUON_ERR_UNSUPPORTED;
  const size_t smem = size_t(tpb) * a.pairs * sizeof(float2);
  if (a.interleaved) rotary_kernel<T, N, true><<<unsigned(blocks), THREADS, smem, st>>>(a, int(tpb));
  else rotary_kernel<T, N, false><<<unsigned(blocks), THREADS, smem, st>>>(a, int(tpb));
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

}  // namespace

int launch_rotary(const RotaryArgs& a, int sms, cudaStream_t st) {
  if (a.dtype == MUON_DTYPE_BF16) return vector_heads(a, 8, 2) ? run<__nv_bfloat16, 8>(a, sms, st) : run<__nv_bfloat16, 1>(a, sms, st);
  return vector_heads(a, 4, 4) ? run<float, 4>(a, sms, st) : run<float, 1>(a, sms, st);
}

}  // namespace muon
