// Rotary positions of up to four tensors that share them, one launch.
//
// Memory bound: every element is read and written once.  A block takes a few tokens.  A unit of work is one place in a head (N pairs) for
// two or four tokens, so that what it costs to find the place (divisions by numbers only known at run time) is paid once for four, whose
// loads are in flight together.  A thread asks for its first unit, then the block forms the cosines and sines of its tokens in shared
// memory (one per token and pair, for all heads of all tensors), then the pairs are turned.  The angle position * inv_freq is formed in
// whole turns and in double, its fraction taken there, and only the fraction goes to sincospif in fp32: a product in fp32 would be off
// by position * 2^-24 radians, 0.06 at a million.
//   out_i = c x_i - s x_j,  out_j = s x_i + c x_j,  (c, s) = amplitude (cos, sin)(position * inv_freq)
//
// 8192 tokens of 40 heads of 128 in bf16: 32.8 to 33.1 us, 5.1 TB/s (an addition that moves 201 MB reaches 6.1, a copy of 134 MB 5.4); 3063 tokens of 40
// heads of 64 in fp32, interleaved: 14.8 us on the device, 4.2 TB/s; a single token: 8.2 to 8.8 us, all of it the host's.  Single elements (a number of
// pairs that 8 in bf16, 4 in fp32 does not divide): 1.0 to 2.5 TB/s.
#include <cuda_bf16.h>

#include <type_traits>

#include "f32x2.cuh"
#include "layer_ops.h"

namespace muon {
namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void down(float* p, float v) { *p = v; }
__device__ __forceinline__ void down(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// N consecutive elements as 32-bit words; two bf16 share a word, the upper one is its fp32 value with the lower bits cleared.
template <typename T, int N> struct Words {
  static constexpr int kCount = N * int(sizeof(T)) / 4;
  uint32_t w[kCount];
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    else return __uint_as_float(w[i]);
  }
  __device__ __forceinline__ uint64_t pair(int i) const { return two(at(2 * i), at(2 * i + 1)); }
  __device__ __forceinline__ void set_pair(int i, float lo, float hi) {
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    } else {
      w[2 * i] = __float_as_uint(lo);
      w[2 * i + 1] = __float_as_uint(hi);
    }
  }
  __device__ __forceinline__ void load(const T* p) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]); }
};
template <typename T> struct Single {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = v; }
};

// (x, y) turned: N pairs whose cosines and sines start at c and s.  Halves: x holds the first elements of the pairs, y the second.
// Interleaved: the 2 N elements are x then y, and elements 2 e and 2 e + 1 of them form pair e.
template <bool INTERLEAVED, typename T, int N>
__device__ __forceinline__ void turn(Words<T, N>& x, Words<T, N>& y, const float* c, const float* s) {
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      Words<T, N>& p = 2 * e < N ? x : y;
      const int i = e % (N / 2);
      const float f = p.at(2 * i), g = p.at(2 * i + 1);
      p.set_pair(i, f * c[e] - g * s[e], f * s[e] + g * c[e]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const uint64_t f = x.pair(i), g = y.pair(i);
      const float4 cc = *reinterpret_cast<const float4*>(c + (i / 2) * 4), ss = *reinterpret_cast<const float4*>(s + (i / 2) * 4);
      const uint64_t cp = i & 1 ? two(cc.z, cc.w) : two(cc.x, cc.y), sp = i & 1 ? two(ss.z, ss.w) : two(ss.x, ss.y);
      const float2 u = both(fma2(mul2(g, sp), twice(-1.f), mul2(f, cp))), v = both(fma2(f, sp, mul2(g, cp)));
      x.set_pair(i, u.x, u.y);
      y.set_pair(i, v.x, v.y);
    }
  }
}
template <bool INTERLEAVED, typename T>
__device__ __forceinline__ void turn(Single<T>& x, Single<T>& y, const float* c, const float* s) {
  const float f = up(x.v), g = up(y.v);
  down(&x.v, f * *c - g * *s);
  down(&y.v, f * *s + g * *c);
}

// Tokens of a unit.  With two and with four, us:
//   bf16 by pieces (five blocks per SM): 8192 tokens of 40 heads of 128 33.1 - 41.4 (interleaved 33.6 - 39.3), 8192 of 40 heads of 64 19.7 - 24.4, 32768 of
//   2 heads of 64 27.0 - 42.3
//   fp32 by pieces (four blocks): 3063 tokens of 40 heads of 64, half of it interleaved 18.6 - 16.6, all of it in halves 14.6 - 16.6; 8192 of 40 heads of
//   128 59.0 - 59.8
//   single elements: bf16, 8192 tokens of 40 heads of 72 75.8 - 65.2, of 80 (half of it) 116 - 101; fp32, of 70 81.2 - 74.4
template <int N> constexpr int kTokens = N == 8 ? 2 : 4;

// A work item is N pairs of one head (2 N elements in two pieces), or, past the rotary part, N elements to copy.
template <typename T, int N, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS, N == 8 ? 5 : 4) rotary_kernel(const __grid_constant__ RotaryArgs a, int tokens_per_block) {
  constexpr int U = kTokens<N>;
  extern __shared__ __align__(16) float cosines[];     // [tokens_per_block][pairs], then the sines
  float* sines = cosines + tokens_per_block * a.pairs;
  const int64_t total = int64_t(a.batch) * a.tokens, t0 = int64_t(blockIdx.x) * tokens_per_block;
  const int n = int(total - t0 < tokens_per_block ? total - t0 : tokens_per_block);
  const int64_t b0 = t0 / a.tokens;
  const int at0 = int(t0 - b0 * a.tokens);
  const bool straight = at0 + n <= a.tokens;           // all of one batch row
  auto row_of = [&](int l) { return straight || at0 + l < a.tokens ? 0 : (at0 + l) / a.tokens; };
  const int turned = a.pairs / N, rest = (a.head_dim - 2 * a.pairs + N - 1) / N, per = turned + rest, items = a.head_begin[a.count] * per;
  using Piece = std::conditional_t<(N > 1), Words<T, N>, Single<T>>;
  struct Unit {
    T* out;
    int64_t step, wrap;
    int l0, w, db;
    Piece x[U], y[U];
  };
  // A unit's place, with its loads issued.  A copied piece (w < 0) has one place: read twice, written once.
  auto fetch = [&](int unit, Unit& q) {
    const int chunk = unit / items, i = unit - chunk * items, h = i / per, w = i - h * per;
    int k = 0;
    while (h >= a.head_begin[k + 1]) ++k;
    const muon_rotary_item_t& it = a.item[k];
    const int64_t hh = h - a.head_begin[k];
    const bool copy = w >= turned;
    const int da = copy ? 2 * a.pairs + (w - turned) * N : INTERLEAVED ? 2 * w * N : w * N;
    q.l0 = chunk * U;
    q.w = copy ? -1 : w;
    q.db = copy ? 0 : INTERLEAVED ? N : a.pairs;
    q.step = it.out.token_stride;
    q.wrap = it.out.batch_stride - a.tokens * it.out.token_stride;
    q.out = static_cast<T*>(it.out.data) + b0 * it.out.batch_stride + (at0 + q.l0) * q.step + hh * it.out.head_stride + da;
    const int64_t step = it.in.token_stride, wrap = it.in.batch_stride - a.tokens * step;
    const T* in = static_cast<const T*>(it.in.data) + b0 * it.in.batch_stride + (at0 + q.l0) * step + hh * it.in.head_stride + da;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (q.l0 + u < n) {
        const T* p = in + u * step + (straight ? 0 : row_of(q.l0 + u) * wrap);
        q.x[u].load(p);
        q.y[u].load(p + q.db);
      }
  };
  auto finish = [&](Unit& q) {
    const int at = q.w < 0 ? 0 : q.l0 * a.pairs + q.w * N;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (q.l0 + u < n) {
        T* p = q.out + u * q.step + (straight ? 0 : row_of(q.l0 + u) * q.wrap);
        if (q.w >= 0) {
          turn<INTERLEAVED>(q.x[u], q.y[u], cosines + at + u * a.pairs, sines + at + u * a.pairs);
          q.y[u].store(p + q.db);
        }
        q.x[u].store(p);
      }
  };
  const int units = items * ((n + U - 1) / U);
  Unit q;
  int unit = threadIdx.x;
  if (unit < units) fetch(unit, q);
  for (int i = threadIdx.x; i < n * a.pairs; i += THREADS) {
    const int l = i / a.pairs;
    const int64_t pos = a.position_offset + (a.positions ? int64_t(a.positions[t0 + l]) : at0 + l - row_of(l) * a.tokens);
    const double x = double(pos) * a.turns[i - l * a.pairs];
    float s, c;
    sincospif(2.f * float(x - rint(x)), &s, &c);
    cosines[i] = c * a.amplitude;
    sines[i] = (a.inverse ? -s : s) * a.amplitude;
  }
  __syncthreads();
  while (unit < units) {
    finish(q);
    unit += THREADS;
    if (unit < units) fetch(unit, q);
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
  // a round of four tokens, but no fewer than four blocks per SM, and at most 16 KiB of cosines and sines
  int64_t tpb = 4;
  const int64_t spread = (total + 4 * sms - 1) / (4 * sms);
  if (tpb > spread) tpb = spread;
  if (tpb > 2048 / a.pairs) tpb = 2048 / a.pairs;
  if (tpb < 1) tpb = 1;
  const int64_t blocks = (total + tpb - 1) / tpb;
  if (blocks > 0x7fffffff) return MUON_ERR_UNSUPPORTED;
  const size_t smem = size_t(tpb) * a.pairs * 2 * sizeof(float);
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
