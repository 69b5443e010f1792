// Shared pieces of the tensor-core kernels of the feed-forward block and the 8-bit linear layer: operands, scales, memory accesses.
#pragma once

#include <cuda_fp8.h>

#include <algorithm>

#include "product_ops.h"
#include "tc_common.cuh"

namespace muon {
namespace prod {

using namespace tc;

struct Scales {                                // of an operand in 8 bits: the byte of (row, k-block) is at (row >> row_shift) * row_step + block * block_step
  const uint8_t* p;
  int64_t row_step, block_step;
  int32_t row_shift, rows;
  int32_t wide;                                // blocks whose bytes lie together and aligned in every row: 16, 4 or 1
};
constexpr int kScaleBlocks = 16;               // k-blocks whose scales are gathered at a time: a round of gathering takes as long as the products of six

// Tensor memory is handed out to blocks as they ask for it, and a block that waits for some while its cluster waits for it could wait for good: its peers may
// hold what a block of another cluster, which holds what this one wants, is waiting for.  So every kernel of clusters that takes tensor memory also
// takes the same share of shared memory, of which a block is given all before it starts: then there is always enough of the former.
constexpr uint32_t kSmShared = 228 * 1024, kBlockReserved = 1024, kSmColumns = 512, kMostShared = 227 * 1024;
__host__ __device__ constexpr uint32_t shared_for_columns(uint32_t columns) {
  return columns * (kSmShared / kSmColumns) > kMostShared ? kMostShared : columns * (kSmShared / kSmColumns) - kBlockReserved;
}

// ------------------------------------------------------------------ PTX
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t map_to_cta(uint32_t local_addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local_addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// mbar_wait on what threads of the peer CTA wrote before they arrived.
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  const long long t0 = clock64();
  for (uint32_t spins = 1;; ++spins) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    if (ok) return true;
    if ((spins & 255u) == 0 && (*abort_flag || clock64() - t0 > WAIT_CYCLES)) return false;
  }
}
__device__ __forceinline__ void st_cluster_u32(uint32_t cluster_addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}
__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
               "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void load32(const void* p, uint32_t* w) {
  asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p));
}
// Descriptors are a constant high part and the address in 16-byte units.  K-major: 8 rows of 128 bytes each kilobyte.  MN-major: 8 values of k
// each kilobyte, and the next 64 columns (bf16) 8 KiB further.  Scales: no swizzle, 8 rows of 16 bytes each 128 bytes.
constexpr uint64_t kDescK = (uint64_t(1) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
constexpr uint64_t kDescMN = (uint64_t(8192 >> 4) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
constexpr uint64_t kDescScales = (uint64_t(128 >> 4) << 32) | (uint64_t(1) << 46);

// Instruction descriptor of the scaled kind: e4m3 operands, scales that are powers of two; which of a cell's four bytes holds them is added per k-block.
__device__ __forceinline__ constexpr uint32_t make_idesc_scaled(bool a_mn_major, bool b_mn_major, int m, int n) {
  return (uint32_t(a_mn_major ? 1 : 0) << 15) | (uint32_t(b_mn_major ? 1 : 0) << 16) | (uint32_t(n >> 3) << 17) | (1u << 23) | (uint32_t(m >> 4) << 24);
}
__device__ __forceinline__ uint32_t scale_byte_ids(uint32_t id) { return (id << 4) | (id << 29); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ float low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

// The bytes of k-blocks kb to kb + 15 (0 past the last), as four words, for rows `row0` + lane + 0, 32, 64 and 96 of an operand.  All loads are
// issued before the first is waited for.
__device__ __forceinline__ void gather_scales(const Scales& s, int row0, int kb, int kblocks, int lane, uint32_t (&w)[4][4]) {
  const uint8_t* base = s.p + int64_t(kb) * s.block_step;
  const int left = kblocks - kb, wide = kb % 16 == 0 ? s.wide : kb % 4 == 0 ? min(s.wide, 4) : 1;
  if (s.row_shift) {                           // blocks of 128 rows: one lane takes one byte, and all the words are the same for every row
    uint32_t v = 0;
    if (lane < kScaleBlocks && lane < left && row0 < s.rows) v = uint32_t(__ldg(base + int64_t(row0 >> s.row_shift) * s.row_step + lane * s.block_step));
    v <<= 8 * (lane & 3);
    v |= __shfl_xor_sync(0xffffffffu, v, 1);
    v |= __shfl_xor_sync(0xffffffffu, v, 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[0][i] = __shfl_sync(0xffffffffu, v, 4 * i);
#pragma unroll
    for (int r = 1; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) w[r][i] = w[0][i];
    return;
  }
  if (wide >= 16 && left >= 16) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(base + int64_t(min(row0 + lane + 32 * r, s.rows - 1)) * s.row_step));
      w[r][0] = x.x; w[r][1] = x.y; w[r][2] = x.z; w[r][3] = x.w;
    }
    return;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const uint8_t* q = base + int64_t(min(row0 + lane + 32 * r, s.rows - 1)) * s.row_step;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t x = 0;
      if (wide >= 4 && left >= 4 * i + 4) {
        x = __ldg(reinterpret_cast<const uint32_t*>(q) + i);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (4 * i + j < left) x |= uint32_t(__ldg(q + 4 * i + j)) << (8 * j);
      }
      w[r][i] = x;
    }
  }
}

// 16 columns (two to a word) of a row of bf16 that begins on 16 bytes, of which `left` are inside.
__device__ __forceinline__ void put16(__nv_bfloat16* p, const uint32_t* w, int left, bool sectors) {
  if (left >= 16 && sectors) return store32(p, w);
  if (left >= 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  if (left >= 16) {
    *reinterpret_cast<uint4*>(p + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < left && (left < 8) == (i < 8)) reinterpret_cast<uint16_t*>(p)[i] = uint16_t(w[i >> 1] >> (16 * (i & 1)));
}
__device__ __forceinline__ void get16(const __nv_bfloat16* p, uint32_t* w, int left, bool sectors) {
  if (left >= 16 && sectors) return load32(p, w);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (left >= 8 * (h + 1)) x = __ldg(reinterpret_cast<const uint4*>(p) + h);
    w[4 * h] = x.x; w[4 * h + 1] = x.y; w[4 * h + 2] = x.z; w[4 * h + 3] = x.w;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < left && left < 16 && (left < 8) == (i < 8)) w[i >> 1] |= uint32_t(__ldg(reinterpret_cast<const uint16_t*>(p) + i)) << (16 * (i & 1));
}

__device__ __forceinline__ float2 values_of(uint32_t pair) {
  return __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(pair & 0xffffu), __NV_E4M3)));
}

// ------------------------------------------------------------------ host
struct Encoder {
  muon_ctx* ctx;
  bool ok = true;
  void map(CUtensorMap* to, const void* data, int type, int64_t ld, int64_t cols, int64_t rows, uint32_t box_cols, uint32_t box_rows) {
    const cuuint64_t dims[2] = {cuuint64_t(cols), cuuint64_t(rows)};
    const cuuint64_t strides[1] = {cuuint64_t(ld * size_of_type(type))};
    const cuuint32_t box[2] = {box_cols, box_rows}, estr[2] = {1u, 1u};
    ok = ok && reinterpret_cast<EncodeFn>(ctx->tmap_encode)(
                   to, type == kTypeBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(data), dims, strides, box, estr,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    ++ctx->tmap_encodes;
  }
  // `rows`: of the operand in a tile of a CTA
  void operand(CUtensorMap* to, const Operand& o, int64_t n, int64_t k, uint32_t rows) {
    const uint32_t line = 128 / uint32_t(size_of_type(o.type));
    if (o.mn_major) map(to, o.data, o.type, o.ld, n, k, line, line);
    else map(to, o.data, o.type, o.ld, k, n, line, rows);
  }
};

inline Scales scales_of(const Operand& o, int rows) {
  const int shift = o.block_rows == 1 ? 0 : 7;
  if (o.mn_major) return {o.scales, 1, o.lds, 7, rows, 1};    // the block of a column; blocks of rows are those of k
  const uintptr_t place = reinterpret_cast<uintptr_t>(o.scales) | uintptr_t(o.lds);
  return {o.scales, o.lds, 1, shift, rows, place % 16 == 0 ? 16 : place % 4 == 0 ? 4 : 1};
}

}  // namespace prod
}  // namespace muon
