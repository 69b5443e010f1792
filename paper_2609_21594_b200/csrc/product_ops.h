// Shared declarations of the matrix products around the gated feed-forward block and the 8-bit linear layer.  Internal to the library.
//
//   C[m][n] = sum over segments s and k of A_s(m, k) B_s(n, k)
//
// with a choice of epilogues.  One description serves two engines: tensor cores (product_tc.cu) where TMA can address every tensor,
// CUDA cores (product_simt.cu) for fp32 and for everything else.
#pragma once

#include "layer_ops.h"

namespace muon {

// 8-bit blocks: e4m3 codes and a byte e for every block of 128 columns of `block_rows` (1 or 128) rows, which stands for 2^(e - 127).
constexpr int kBlock = 128;
constexpr int kTypeBf16 = MUON_DTYPE_BF16, kTypeFp32 = MUON_DTYPE_FP32, kTypeE4m3 = 2;

// A matrix as it lies in memory: rows of `ld` elements.
struct Operand {
  const void* data;
  int64_t ld;
  int32_t type;
  int32_t mn_major;            // 0: memory row = row of the operand, column = k;  1: memory row = k, column = row of the operand
  const uint8_t* scales;       // e4m3: [memory rows / block_rows][columns / 128]
  int64_t lds;
  int32_t block_rows;
};

enum EpilogueKind : int32_t {
  kPlain,                      // C
  kGated,                      // B_0 and B_1 are two matrices of n rows: g = A B_0', u = A B_1', h = act(g) u; writes h, and g and u where asked
  kGrad,                       // C = dh stays in the kernel; reads g and u; writes dg = dh u act'(g), du = dh act(g), h = act(g) u
};

struct Epilogue {
  EpilogueKind kind;
  int32_t type;                // of what is written: bf16 or fp32
  int32_t activation;
  int32_t gate_up_type;        // kGated: of g and u as written (bf16, fp32, e4m3); kGrad: as read
  void* c;                     // kPlain: C; kGated, kGrad: h
  int64_t ldc;
  void* gate;                  // kGated: g or null; kGrad: dg
  void* up;                    // kGated: u or null; kGrad: du
  int64_t ld_gate, ld_up;
  Operand in_gate, in_up;      // kGrad: g and u.  kGated with e4m3: where codes and scales of g and u go
  float* sums;                 // kPlain with a sum longer than kLongestSum: fp32 [m][ld_sums], where its parts meet; else null
  int64_t ld_sums;             // a multiple of 64
  int32_t add, hold;           // of a part: earlier ones are in `sums`; later ones follow, so that it stays there and C is not written
};

struct Product {
  Operand a[2], b[2];
  int32_t segments;
  int32_t m, n, k;             // k: of each segment
  Epilogue e;
};

constexpr int kMaxProducts = 3;   // of a launch

// The tensor cores cut a sum to fp32 where others round it, so a sum of many terms ends up too small: against 64 bits, of random terms, by 0.0012 of the
// result (norm) after 2^20 of them, 0.0049 after 2^22, 0.074 after 2^26, where the rounding to bf16 is 0.0016.  Sums over tokens, which may be that many,
// are therefore formed in parts of kLongestSum (0.0003), which are added in fp32, rounded.  Sums over dim, hidden and out have no such parts and go to
// the CUDA cores from kMostSum on.  No tile takes longer than 2^15 k-blocks of 560 to 800 clocks, a hundredth of what its waits are given.
constexpr int32_t kLongestSum = 1 << 18, kMostSum = 1 << 20;

// What TMA asks of rows of `ld` elements: the first, and the distance between two, on 16 bytes.
inline int size_of_type(int type) { return type == kTypeFp32 ? 4 : type == kTypeBf16 ? 2 : 1; }
inline bool addressable(const void* p, int64_t ld, int type) {
  const int64_t bytes = ld * size_of_type(type);
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && bytes % 16 == 0 && bytes < (int64_t(1) << 40);
}

// Rows of bytes to another place, for tensors that TMA cannot address: into rows that it can, or out of them.  `unit`: bytes of an element, which
// source and destination are aligned to.
struct CopyTask {
  const void* from;
  void* to;
  int64_t ld_from, ld_to, rows, bytes;     // in bytes
  int32_t unit;
};
constexpr int kMaxCopies = 8;
int launch_copies(const CopyTask* list, int count, int sms, cudaStream_t st);

// The tensor-core engine takes a list of products with operands of one type and one order in memory, if TMA can address all tensors.
bool products_tc_take(const Product* p, int count);
// What the launch right before this one in the stream is: anything; one of the same call, so this one may be brought up while that one ends; or one of
// the same call that does not write B, which may be read before that one has ended.
enum Before { kBeforeAny, kBeforeSameCall, kBeforeLeavesB };
int launch_products_tc(muon_ctx* ctx, const Product* p, int count, Before before, cudaStream_t st);
// About how many clocks they take there, from the rounds of tiles.
double products_tc_clocks(const Product* p, int count, int sms);
// Products of few rows, whose time is that of reading B, have a kernel of their own, which takes them where its blocks are expected to be done sooner.
constexpr int kFewRows = 1024;
bool product_few_takes(const Product& p, int sms);
// It begins early after kBeforeLeavesB alone: it asks for B at once.
int launch_product_few(muon_ctx* ctx, const Product& p, int sms, Before before, cudaStream_t st);
// Operands of one type.  siblings: products of about this size that a call may launch together, of which `count` are wanted now.
int launch_products_simt(const Product* p, int count, int siblings, int sms, cudaStream_t st);

int launch_quantize(int dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, const Operand& out, int sms, cudaStream_t st);
int launch_dequantize(int dtype, int64_t rows, int64_t cols, const Operand& in, void* y, int64_t ldy, int sms, cudaStream_t st);

#ifdef __CUDACC__
// 2^(e - 127) for a scale's byte; 255 is a NaN.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7fffffffu : e << 23); }
// 2^(127 - e): what a block is multiplied with before it is rounded.  e <= 247 as `scale_byte` gives it, so that this is a normal number.
__device__ __forceinline__ float inverse_scale_of(uint32_t e) { return __uint_as_float((254u - e) << 23); }
// The byte of the least power of two (from 2^-127 on) that brings `top`, the bits of a block's largest finite magnitude, to at most 448 =
// 1.75 * 2^8: a mantissa above 1.75 carries into the exponent.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  const int e = int((top + 0x1fffffu) >> 23) - 8;
  return uint32_t(e < 0 ? 0 : e);
}
// The magnitude's bits of a finite value, 0 of a NaN or an infinity: neither has a share in the scale, and both are kept as NaN.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
__device__ __forceinline__ float infinite_to_nan(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u ? x : __uint_as_float(0x7fffffffu); }

// act(g) = g s(w(g)) with the logistic function s and w = k g (1 + c g^2):  silu: k = 1, c = 0;  gelu (tanh form, (1 + tanh z) / 2 = s(2z)):
// k = 2 sqrt(2 / pi), c = 0.044715.  act'(g) = s + g s (1 - s) w'(g).  Both forms cost the same instructions: a branch between them, taken for
// every element, keeps the exponentials of neighbouring elements from overlapping.
struct Activation {
  float k, c;
};
__device__ __forceinline__ Activation activation_of(int kind) { return kind == MUON_ACTIVATION_GELU ? Activation{1.5957691216057308f, 0.044715f} : Activation{1.f, 0.f}; }
// FAST: the exponential and the reciprocal of the special-function unit, for results that are rounded to bf16.  The exponential's error grows with its
// argument (2 + 1.2 |w| units of 2^-23), and so does that of w's own roundings in it: s is off by at most (6 + 4 |w|) 2^-23 of its value, 2^-14 at w = -87, in
// both forms; the slope by as much of each of its two parts.  Below -87, where s is less than the least normal number, it may count as 0: act(g) is then
// off by less than 89 * 2^-126.
template <bool FAST>
__device__ __forceinline__ void activate(const Activation& f, float g, float* a, float* slope) {
  const float g2 = fminf(g * g, 1e12f);       // beyond, s is 0 or 1, and 0 times w' has to stay 0
  const float w = f.k * g * fmaf(f.c, g2, 1.f), dw = f.k * fmaf(3.f * f.c, g2, 1.f);
  float s;
  if constexpr (FAST) {
    const float t = 1.f + __expf(-w);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(t));
  } else {
    s = 1.f / (1.f + expf(-w));
  }
  *a = g * s;
  *slope = fmaf(*a * (1.f - s), dw, s);
}
#endif

}  // namespace muon
