// Shared pieces of the tensor-core attention kernels: operand tiles, matrix instructions with A in tensor memory, tile ranges.
//
// An operand tile is 128 tokens of one head, kept as one or two 128B-swizzled boxes of 64 elements (16 KiB each): head sizes up to 64
// take one box, up to 128 two, and TMA fills what lies beyond head_dim with zeros.  The same tile serves as a K-major operand (rows
// times rows: q k^T) and as an MN-major one (the tokens are summed over: P v).
#pragma once

#include "f32x2.cuh"
#include "layer_ops.h"
#include "tc_common.cuh"

namespace muon {
namespace attn {

using namespace tc;

constexpr int BLK = 128;                         // tokens of a tile
constexpr uint32_t BOX_BYTES = BLK * 64 * 2;     // 16 KiB
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnMaps {
  CUtensorMap q, k, v, dout;
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int d, int head, int token, int batch) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(d), "r"(head), "r"(token), "r"(batch)
      : "memory");
}
// 128 tokens of a head; arrives with BOXES * BOX_BYTES on `bar`, which the caller has told to expect them.
template <int BOXES>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int token, int batch) {
#pragma unroll
  for (int i = 0; i < BOXES; ++i) tma_load_4d(dst + uint32_t(i) * BOX_BYTES, map, bar, i * 64, head, token, batch);
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// D (+)= A B with A read from tensor memory: lane = row, one 32-bit column = two consecutive bf16 of k.
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tc_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
      "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
      "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// Registers per thread of a warpgroup.  The sum over a block's warpgroups must not exceed what the block was launched with.
template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

__device__ __forceinline__ void tc_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ uint64_t words(uint32_t a, uint32_t b) { return two(__uint_as_float(a), __uint_as_float(b)); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t pack_bf16(uint64_t v) {
  const float2 f = both(v);
  return pack_bf16(f.x, f.y);
}
__device__ __forceinline__ uint64_t exp2_approx(uint64_t v) {
  const float2 f = both(v);
  return two(exp2_approx(f.x), exp2_approx(f.y));
}
// 2^x on the multiply-add pipe, for a share of the exponentials where two warps of a scheduler form them at the same time and the
// exponential unit (one warp's instruction in 8 clocks) is what both wait for.  x = n + r with n the nearest integer, which adding
// 1.5 * 2^23 puts in the low bits; 2^r on [-1/2, 1/2] by the polynomial of degree 4 whose largest relative error is least (2.7e-6 in
// fp32; fitted by reweighted least squares); 2^n is made from its exponent and multiplied on.  x is at most 127; below -126 the result is
// 2^-126.  A NaN stays one: the clamp hands it on, and the product keeps it (n added to the exponent's bits would make it a number).
__device__ __forceinline__ float clamp_below(float x) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(-126.f));
  return y;
}
__device__ __forceinline__ uint64_t exp2_poly(uint64_t v) {
  const float2 in = both(v);
  const uint64_t x = two(clamp_below(in.x), clamp_below(in.y));
  const uint64_t t = add2(x, twice(12582912.f));
  const uint64_t r = fma2(add2(t, twice(-12582912.f)), twice(-1.f), x);
  uint64_t p = fma2(twice(0.009570102207362652f), r, twice(0.05591786280274391f));
  p = fma2(p, r, twice(0.240247443318367f));
  p = fma2(p, r, twice(0.6931217908859253f));
  p = fma2(p, r, twice(0.9999992847442627f));
  const float2 n = both(t);
  return mul2(p, two(__int_as_float(0x3f800000 + (__float_as_int(n.x) << 23)), __int_as_float(0x3f800000 + (__float_as_int(n.y) << 23))));
}

// The issuing warp runs converged, its warp index taken from lane 0 and every wait followed by a vote, and one elected lane issues: then
// descriptors and addresses are values of the whole warp and stay in uniform registers.  A step has to take less than the 64 clocks that
// its instruction keeps the tensor cores busy; issued from a branch on the lane it took 85, with descriptors formed anew each time 107.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(one));
  return one != 0;
}
// Runs f on the elected lane.  Without the meeting behind it the other lanes go on to the next wait and share the issue slots with it.
template <typename F>
__device__ __forceinline__ void elected(bool go, F f) {
  if (go && elect_one()) f();
  __syncwarp();
}
__device__ __forceinline__ int uniform_warp() { return __shfl_sync(0xffffffffu, int(threadIdx.x >> 5), 0); }

// Descriptors are formed once per tile: a step adds to the address field, which no address in shared memory carries out of.
//
// S[128 x 128] = X Y^T over the head: both tiles K-major.  `ksteps` steps of 16 elements cover head_dim.
template <int BOXES>
__device__ __forceinline__ void mma_rows_rows(uint32_t d_tmem, uint32_t x, uint32_t y, int ksteps) {
  constexpr uint32_t idesc = make_idesc(false, BLK, BLK);
  const uint64_t dx = make_desc(x, 16, 1024), dy = make_desc(y, 16, 1024);
#pragma unroll
  for (int k = 0; k < BOXES * 4; ++k) {
    constexpr uint32_t box = BOX_BYTES >> 4;
    const uint32_t off = uint32_t(k >> 2) * box + uint32_t(k & 3) * 2u;
    if (k < ksteps) tc_mma(d_tmem, dx + off, dy + off, idesc, k > 0);
  }
}
// Steps [k0, k1) of D[128 x n] (+)= P[128 x 128] Y[128 tokens x n]: P from tensor memory, 64 columns of bf16 pairs from `p_lo` on for the first
// 64 tokens and from `p_hi` on for the others; Y MN-major.  `idesc` holds n (a multiple of 16 that covers head_dim).
template <int K0 = 0, int K1 = 8>
__device__ __forceinline__ void mma_probs_rows(uint32_t d_tmem, uint32_t p_lo, uint32_t p_hi, uint32_t y, uint32_t idesc, bool accumulate) {
  const uint64_t dy = make_desc(y, BOX_BYTES, 1024);
#pragma unroll
  for (int k = K0; k < K1; ++k)
    tc_mma_ts(d_tmem, (k < 4 ? p_lo : p_hi) + uint32_t(k & 3) * 8u, dy + uint32_t(k) * 128u, idesc, accumulate || k > K0);
}

// Clears the rows of a tile before `from` and those from `to` on (a whole warp) and arrives on `bar`.  Rows past a sequence's end hold another sequence's
// tokens or padding, and the first queries may see no key; such rows meet probabilities that are zero, but zero times a NaN or an infinity is
// not zero.
template <int BOXES>
__device__ __forceinline__ void clear_rows(uint32_t tile, int from, int to, int lane, uint32_t bar) {
  auto clear = [&](int first, int last) {
#pragma unroll
    for (int b = 0; b < BOXES; ++b)
      for (int i = first * 8 + lane; i < last * 8; i += 32)
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + uint32_t(b) * BOX_BYTES + uint32_t(i) * 16u), "r"(0) : "memory");
  };
  clear(0, from);
  clear(max(to, 0), BLK);
  fence_async_smem();
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// Blocks [n0, n1) of 128 keys that some query of rows [r0, r0 + 128) sees.
struct BlockRange {
  int n0, n1;
};
__device__ __forceinline__ BlockRange key_blocks(const AttnArgs& a, const AttnSeq& s, int r0) {
  const int last = min(r0 + BLK, s.qn) - 1;
  if (last < r0) return {0, 0};
  const int lo = attn_key_lo(a, s, r0), hi = attn_key_hi(a, s, last);
  if (hi <= lo) return {0, 0};
  return {lo / BLK, (hi + BLK - 1) / BLK};
}
// Whether some query that counts, of rows [r0, r0 + 128), does not see some key of [c0, c0 + 128).
__device__ __forceinline__ bool block_masked(const AttnArgs& a, const AttnSeq& s, int r0, int c0) {
  const int last = min(r0 + BLK, s.qn) - 1;
  return attn_key_hi(a, s, r0) < c0 + BLK || attn_key_lo(a, s, last) > c0;
}

// ------------------------------------------------------------------ host side
// Tensor-map rules: 16-byte aligned base, strides that are multiples of 16 bytes.
inline bool map_takes(const AttnTensor& t, int64_t batch, int64_t tokens, int64_t heads) {
  auto fits = [](int64_t n, int64_t s) { return n <= 1 || (s > 0 && s % 8 == 0 && s < (int64_t(1) << 38)); };
  return reinterpret_cast<uintptr_t>(t.data) % 16 == 0 && fits(batch, t.sb) && fits(tokens, t.st) && fits(heads, t.sh);
}

inline bool encode_tile_map(void* fn, CUtensorMap* map, const AttnTensor& t, int dim, int64_t batch, int64_t tokens, int64_t heads) {
  // the stride of a dimension of one element is never used, but has to be a legal one
  const cuuint64_t dims[4] = {cuuint64_t(dim), cuuint64_t(heads), cuuint64_t(tokens), cuuint64_t(batch)};
  const cuuint64_t strides[3] = {cuuint64_t(heads > 1 ? t.sh * 2 : 256), cuuint64_t(tokens > 1 ? t.st * 2 : 256),
                                 cuuint64_t(batch > 1 ? t.sb * 2 : 256)};
  const cuuint32_t box[4] = {64u, 1u, BLK, 1u};
  const cuuint32_t estr[4] = {1u, 1u, 1u, 1u};
  return reinterpret_cast<EncodeFn>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, t.data, dims, strides, box, estr,
                                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace attn
}  // namespace muon
