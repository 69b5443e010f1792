// Matrix products on the tensor cores: pairs of CTAs, persistent over a list of 256 x 256 tiles.
//
//   C[m][n] = sum_s sum_k A_s(m, k) B_s(n, k)          operands bf16, or e4m3 with a power of two for every 128 values of k
//
// CTA r of a pair owns 128 rows of the tile and stages, for each k-block of 128 bytes, its rows of A and half of the columns of B; the
// leader (r = 0) issues tcgen05.mma.cta_group::2 of 256 x N.  Operands come by TMA as they lie in memory, K-major or MN-major (summed
// over the rows: the backward products need no transposed copy).  Accumulators alternate between two places in tensor memory, so that a
// tile's epilogue runs under the next tile's products.  Eight epilogue warps, two per quarter of the rows; a thread holds 64 columns of one
// row at a time and reads and writes memory itself, 32 bytes (a sector) at a time.
//
// Gated product: the leader's half of B is 128 rows of w_gate and its peer's the same rows of w_up, so columns [0, 128) of the accumulator are g
// and [128, 256) are u of the same elements: one thread holds both, and 128 columns of g are one block of the 8-bit form.
// Gradient of the gate: the accumulator is dh, which never leaves the chip; g and u come in, dg, du and h go out.
//
// 8 bits: tcgen05.mma.kind::mxf8f6f4 multiplies each group of 32 values of k with the scales of its row of A and of B, taken from tensor memory.  A
// block of 128 is four such groups with one scale.  A warp of its own gathers the bytes of sixteen blocks into the order that tcgen05.cp spreads
// over the lanes; the issuer copies four blocks' bytes (12 columns) every fourth k-block.  Two accumulators of 256 columns would leave no room for them, so the
// second one begins 16 columns inside the first: the next tile begins when those 16 columns have been read, which the epilogue does first.
//
// What bounds it.  A k-block keeps the tensor cores busy for 512 clocks and brings 32 KiB to each multiprocessor, about what the second-level cache hands
// out in that time, and the matrix instructions read as much from shared memory as it has: so the epilogue stays away from shared memory (staged there
// and stored by TMA, the gated product with g and u kept ran at 88 % of the tensor pipe, the gradient at 68 %; now 98 and 84 to 86 %).  4096 tokens of
// 4096 x 14336 (under ncu, clocks 1.4 to 1.5 GHz under the power limit): gated 616 us, 1561 TFLOP/s; down 328, 1466; gradient 363, 1326;
// dx 659, 1461; the weights' gradients 949, 1521.  8 bits 180 us, 2667 TFLOP/s, 81 % of the pipe: between tiles the 16 shared columns and 3 copies
// of scales per four k-blocks.  The gradient's epilogue moves 320 KiB a tile and ends after the next tile's products do when k
// is short (3001 x 2048 x 5632: 79 us, 55 % of the pipe); sixteen epilogue warps instead of eight did not change that (80 us).
//
// Synchronisation as in the Newton-Schulz kernel, all waits bounded: full / empty per stage, tfull / tempty per accumulator, an abort flag in both CTAs.
#include "product_tc.cuh"

namespace muon {
namespace {

using namespace prod;

constexpr int kRows = 128;                     // of A per CTA
constexpr uint32_t kHalfBytes = kRows * 128;   // 16 KiB: 128 rows of 128 bytes
constexpr uint32_t kStageBytes = 2 * kHalfBytes;
constexpr int kEpiWarps = 8;
constexpr int kGroupTiles = 8;                 // tiles of rows that a stretch of the tile list stays in: what they and as many columns read fits L2
constexpr int kScaleRing = 2;
constexpr uint32_t kScaleWord = 3 * 512;       // scales of four k-blocks: 128 rows of A, 256 of B, four bytes each
constexpr uint32_t kScaleBytes = kScaleBlocks / 4 * kScaleWord;
constexpr uint32_t kScaleCol = 496;            // tensor memory columns of the scales
constexpr uint32_t kSecondAccumulator8 = 240;

template <bool EIGHT>
struct Shape {
  static constexpr int stages = EIGHT ? 6 : 7;
  static constexpr uint32_t scale_off = stages * kStageBytes;
  static constexpr uint32_t bar_off = scale_off + (EIGHT ? kScaleRing * kScaleBytes : 0);
  static constexpr uint32_t bytes = shared_for_columns(512);      // all there is: see there
  static_assert(bar_off + 512 + 1024 <= bytes, "227 KiB of shared memory");
  static constexpr int threads = 32 * (2 + kEpiWarps + (EIGHT ? 1 : 0));
};

struct TcProduct {
  CUtensorMap a[2], b[2];
  __nv_bfloat16* out[3];                       // C; or h, g, u; or h, dg, du
  int64_t ld[3];
  const __nv_bfloat16* in[2];                  // g, u
  int64_t ld_in[2];
  float* sums;                                 // where the parts of a long sum meet, or null
  int64_t ld_sums;
  Scales sa, sb;
  int32_t m, n, kblocks, segments;             // kblocks: of a segment
  int32_t tiles_m, tiles_n, tile_begin;
  int32_t tile_cols;                           // columns of C that a tile forms
};
struct TcProducts {
  TcProduct p[kMaxProducts];
  int32_t count, total_tiles;
  int32_t half;                                // columns of B per CTA: 128 or 64
  int32_t activation, keep;                    // keep: g and u are written
  int32_t add, hold;                           // of a part of a long sum, see Epilogue
  Operand gate, up;                            // 8-bit g and u
  int32_t codes_wide;                          // their rows take 16-byte accesses
  int32_t sectors;                             // all bf16 rows begin on a 32-byte sector
  int32_t* status;
};

// ------------------------------------------------------------------ PTX
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar_cluster_addr, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar_cluster_addr), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void tc_mma_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_mma_pair_scaled(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                                   uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
// 32 rows of 16 bytes into four columns, repeated in every quarter of the lanes, in both CTAs.
__device__ __forceinline__ void tc_copy_scales_pair(uint32_t d_tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(d_tmem), "l"(desc) : "memory");
}
// Arrives on the barrier at this shared-memory offset in both CTAs of the pair once everything issued so far is done.
__device__ __forceinline__ void tc_commit_pair(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .b16 m;\n\t"
      "mov.b16 m, 3;\n\t"
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}"
      ::"r"(bar)
      : "memory");
}

// ------------------------------------------------------------------ tiles
struct Tile {
  int prob, m0, n0;                            // first row of the pair, first column of C
};
// Within kGroupTiles tiles of rows the rows run fastest: the pairs at work at a time share the operands of about as many tiles of rows as of columns.
__device__ __forceinline__ Tile decode(const TcProducts& L, int t) {
  Tile r;
  r.prob = 0;
  for (int i = 1; i < L.count; ++i)
    if (t >= L.p[i].tile_begin) r.prob = i;
  const TcProduct& p = L.p[r.prob];
  t -= p.tile_begin;
  const int per_group = kGroupTiles * p.tiles_n;
  const int g = t / per_group, in = t - g * per_group;
  const int rows = min(kGroupTiles, p.tiles_m - g * kGroupTiles);
  const int c = in / rows;
  r.m0 = (g * kGroupTiles + in - c * rows) * (2 * kRows);
  r.n0 = c * p.tile_cols;
  return r;
}

template <int STAGES>
struct Ring {
  uint32_t it, s, ph;                          // k-blocks so far, place in the ring and its phase
  __device__ __forceinline__ void advance() {
    ++it;
    if (++s == uint32_t(STAGES)) {
      s = 0;
      ph ^= 1u;
    }
  }
};

// ------------------------------------------------------------------ epilogue
__device__ __forceinline__ void load64(uint32_t taddr, uint32_t (&v)[64]) {
  __syncwarp();
  tc_ld32(taddr, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
  tc_ld32(taddr + 32, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
}

// The bits of the largest finite magnitude in 128 columns of the accumulator; *odd: there is an infinity.
__device__ __forceinline__ uint32_t top_of_block(uint32_t taddr, bool* odd) {
  float top = 0.f;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t v[64];
    load64(taddr + uint32_t(i * 64), v);
    tc_wait_ld();
#pragma unroll
    for (int k = 0; k < 64; ++k) top = fmaxf(top, fabsf(__uint_as_float(v[k])));      // a NaN loses
  }
  *odd = top == __uint_as_float(0x7f800000u);
  if (__any_sync(0xffffffffu, *odd)) {
    uint32_t finite = 0;
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
      uint32_t v[32];
      tc_ld32(taddr + uint32_t(i * 32), v);
      tc_wait_ld();
#pragma unroll
      for (int k = 0; k < 32; ++k) finite = max(finite, finite_bits(__uint_as_float(v[k])));
    }
    return finite;
  }
  return __float_as_uint(top);
}
// 32 values as codes; the columns from `left` on are left alone.
__device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t* v, float inverse, bool odd, int left, bool wide) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t pair[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float lo = __uint_as_float(v[q * 16 + i * 4 + h * 2]), hi = __uint_as_float(v[q * 16 + i * 4 + h * 2 + 1]);
        if (odd) {
          lo = infinite_to_nan(lo);
          hi = infinite_to_nan(hi);
        }
        pair[h] = __nv_cvt_float2_to_fp8x2(make_float2(lo * inverse, hi * inverse), __NV_SATFINITE, __NV_E4M3);
      }
      w[i] = pair[0] | pair[1] << 16;
    }
    if (wide && left >= (q + 1) * 16) {
      *reinterpret_cast<uint4*>(p + q * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (q * 16 + i < left) p[q * 16 + i] = uint8_t(w[i >> 2] >> (8 * (i & 3)));
    }
  }
}
__device__ __forceinline__ void load_codes(const uint8_t* p, uint32_t (&w)[16], int left, bool wide) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (wide && left >= (q + 1) * 16) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + q);
      w[4 * q] = x.x; w[4 * q + 1] = x.y; w[4 * q + 2] = x.z; w[4 * q + 3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * q + i] = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (q * 16 + i < left) w[4 * q + (i >> 2)] |= uint32_t(__ldg(p + q * 16 + i)) << (8 * (i & 3));
    }
  }
}
// CODES: g and u, as they are written (kGated) or read (kGrad), are 8-bit blocks.
template <bool A_MN, bool B_MN, bool EIGHT, int EPI, bool CODES>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Shape<EIGHT>::threads, 1) product_pair_kernel(const __grid_constant__ TcProducts L) {
  using S = Shape<EIGHT>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - raw);
  const uint32_t bars = base + S::bar_off;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen_base + S::bar_off + 480);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_base + S::bar_off + 488);
  auto bar = [&](int i) { return bars + uint32_t(i) * 8u; };
  auto full_bar = [&](uint32_t s) { return bar(int(s)); };
  constexpr int kStages = S::stages, kT = 2 * kStages;
  auto empty_bar = [&](uint32_t s) { return bar(kStages + int(s)); };
  auto tfull_bar = [&](uint32_t i) { return bar(kT + int(i)); };
  auto tempty_bar = [&](uint32_t i) { return bar(kT + 2 + int(i)); };
  const uint32_t drain_bar = bar(kT + 4), shared_bar = bar(kT + 5);     // shared_bar: the columns that both accumulators use have been read
  auto sfull_bar = [&](uint32_t i) { return bar(kT + 6 + int(i)); };
  auto sempty_bar = [&](uint32_t i) { return bar(kT + 6 + kScaleRing + int(i)); };

  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const bool leader_cta = rank == 0;
  const int pair_id = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const uint32_t peer_abort = map_to_cta(base + S::bar_off + 488, rank ^ 1u);
  auto give_up = [&](int code) {
    *abort_flag = 1;
    st_cluster_u32(peer_abort, 1u);
    atomicExch(L.status, code);
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull_bar(i), 1);
      mbar_init(tempty_bar(i), 2 * kEpiWarps);
    }
    mbar_init(drain_bar, 1);
    mbar_init(shared_bar, kEpiWarps);                 // the four warps of each CTA that read those columns
    if constexpr (EIGHT)
      for (int i = 0; i < kScaleRing; ++i) {
        mbar_init(sfull_bar(i), 2);                   // both CTAs' scales
        mbar_init(sempty_bar(i), 1);
      }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // Where the launch before this one in the stream is of the same call, the barriers and columns above are set up while that one ends.  Nothing in
  // memory is read or written before the wait.  The next launch is let go after it alone: what it may read early, from the launches before this one,
  // is then there.  In turn with the same launches one after the other: 8-bit linear layer's backward 125 us against 130 (4001 tokens of 2048 x 5632),
  // a step of 700 tokens 183.5 against 187, the backward of 4096 tokens of 4096 x 14336 2010 against 2049.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  auto accumulator = [&](uint32_t acc) { return tmem_base + acc * (EIGHT ? kSecondAccumulator8 : 256u); };

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer (one per CTA)
    if (lane == 0) {
      Ring<kStages> c{0u, 0u, 0u};
      const uint32_t full0 = map_to_cta(full_bar(0), 0);
      const uint32_t stage_tx = 2 * (kHalfBytes + kHalfBytes / 128 * uint32_t(L.half));
      bool ok = true;
      for (int t = pair_id; t < L.total_tiles && ok; t += num_pairs) {
        const Tile tl = decode(L, t);
        const TcProduct& p = L.p[tl.prob];
        const int arow = tl.m0 + int(rank) * kRows;
        const int brow = EPI == kGated ? tl.n0 : tl.n0 + int(rank) * L.half;
        for (int seg = 0; seg < p.segments && ok; ++seg) {
          const CUtensorMap* ma = &p.a[seg];
          const CUtensorMap* mbm = EPI == kGated ? &p.b[rank] : &p.b[seg];
          for (int kb = 0; kb < p.kblocks; ++kb, c.advance()) {
            if (!mbar_wait(empty_bar(c.s), c.ph ^ 1u, abort_flag)) { ok = false; break; }
            const uint32_t sa = base + c.s * kStageBytes, sb = sa + kHalfBytes;
            if (leader_cta) mbar_expect_tx(full_bar(c.s), stage_tx);
            const uint32_t fb = full0 + c.s * 8u;
            const int k0 = kb * (EIGHT ? 128 : 64);
            if constexpr (A_MN) {
              tma_load_pair(sa, ma, fb, arow, k0);
              tma_load_pair(sa + kHalfBytes / 2, ma, fb, arow + 64, k0);
            } else {
              tma_load_pair(sa, ma, fb, k0, arow);
            }
            if constexpr (B_MN && !EIGHT) {
              tma_load_pair(sb, mbm, fb, brow, k0);
              if (L.half == 128) tma_load_pair(sb + kHalfBytes / 2, mbm, fb, brow + 64, k0);
            } else if constexpr (B_MN) {
              tma_load_pair(sb, mbm, fb, brow, k0);
            } else {
              tma_load_pair(sb, mbm, fb, k0, brow);
            }
          }
        }
      }
      if (!ok) give_up(31);
      if (leader_cta) {   // every armed stage (both CTAs' bytes) has landed before shared memory is released
        const uint32_t issued = c.it;
        for (uint32_t j = (issued > kStages ? issued - kStages : 0); j < issued; ++j)
          if (!mbar_wait(full_bar(j % kStages), (j / kStages) & 1u, abort_flag, false, WAIT_CYCLES / 8)) atomicExch(L.status, 32);
      }
      if (*abort_flag)    // loads this CTA issued for a stage the leader never armed: give them time to land
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (leader CTA only), converged: see elect_one
    if (leader_cta) {
      Ring<kStages> c{0u, 0u, 0u};
      uint32_t tile_it = 0, group = 0;
      bool ok = true;
      constexpr uint64_t a_hi = A_MN ? kDescMN : kDescK, b_hi = B_MN ? kDescMN : kDescK;
      // a step is 32 bytes of k: along a 128-byte row, or that many rows (16 of bf16, 32 of 8 bits) of 128 bytes
      constexpr uint32_t a_step = A_MN ? 16 * 128 / 16 : 2, b_step = B_MN ? (EIGHT ? 32 : 16) * 128 / 16 : 2;
      const uint32_t idesc = EIGHT ? make_idesc_scaled(false, B_MN, 2 * kRows, 2 * L.half) : make_idesc(B_MN, 2 * kRows, 2 * L.half, A_MN);
      auto all = [](bool v) { return __all_sync(0xffffffffu, v) != 0; };
      for (int t = pair_id; t < L.total_tiles && ok; t += num_pairs, ++tile_it) {
        const TcProduct& p = L.p[decode(L, t).prob];
        const uint32_t acc = tile_it & 1u, aph = (tile_it >> 1) & 1u;
        const int num_kb = p.kblocks * p.segments;
        ok = all(mbar_wait(tempty_bar(acc), aph ^ 1u, abort_flag));
        if (EIGHT && ok && tile_it > 0) ok = all(mbar_wait(shared_bar, (tile_it - 1) & 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const uint32_t d_tmem = accumulator(acc);
        for (int kb = 0; kb < num_kb; ++kb, c.advance()) {
          if constexpr (EIGHT) {
            if ((kb & 3) == 0) {
              const uint32_t place = group % kScaleRing;
              if (kb % kScaleBlocks == 0) {
                ok = all(mbar_wait_cluster(sfull_bar(place), (group / kScaleRing) & 1u, abort_flag));
                if (!ok) break;
                tc_fence_after();
              }
              const bool last = kb % kScaleBlocks == kScaleBlocks - 4 || kb + 4 >= num_kb;
              elected(true, [&] {
                const uint32_t from = (base + S::scale_off + place * kScaleBytes + uint32_t(kb % kScaleBlocks / 4) * kScaleWord) >> 4;
#pragma unroll
                for (int i = 0; i < 3; ++i) tc_copy_scales_pair(tmem_base + kScaleCol + uint32_t(4 * i), kDescScales | uint64_t(from + uint32_t(i) * 32u));
                if (last) tc_commit_pair(sempty_bar(place));
              });
              if (last) ++group;
            }
          }
          ok = all(mbar_wait(full_bar(c.s), c.ph, abort_flag));
          if (!ok) break;
          tc_fence_after();
          elected(true, [&] {
            const uint32_t a0 = (base + c.s * kStageBytes) >> 4, b0 = a0 + (kHalfBytes >> 4);
            const uint64_t da = a_hi | uint64_t(a0), db = b_hi | uint64_t(b0);
            const uint32_t id = EIGHT ? idesc | scale_byte_ids(uint32_t(kb & 3)) : idesc;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t more = (kb > 0 || k > 0) ? 1u : 0u;
              if constexpr (EIGHT)
                tc_mma_pair_scaled(d_tmem, da + uint64_t(k * a_step), db + uint64_t(k * b_step), id, tmem_base + kScaleCol, tmem_base + kScaleCol + 4, more);
              else
                tc_mma_pair(d_tmem, da + uint64_t(k * a_step), db + uint64_t(k * b_step), id, more);
            }
            tc_commit_pair(empty_bar(c.s));
          });
        }
        if (ok) elected(true, [&] { tc_commit_pair(tfull_bar(acc)); });
      }
      if (!ok && lane == 0) give_up(33);
      __syncwarp();
      elected(true, [&] { tc_commit_pair(drain_bar); });       // arrives in both CTAs once everything issued above has finished
    }
  } else if (EIGHT && warp == 2 + kEpiWarps) {
    // ------------------------------------------------------------------ scales
    if constexpr (EIGHT) {
      uint32_t group = 0;
      bool ok = true;
      const uint32_t sfull0 = map_to_cta(sfull_bar(0), 0);
      for (int t = pair_id; t < L.total_tiles && ok; t += num_pairs) {
        const Tile tl = decode(L, t);
        const TcProduct& p = L.p[tl.prob];
        for (int kb = 0; kb < p.kblocks; kb += kScaleBlocks, ++group) {
          const uint32_t place = group % kScaleRing;
          if (!mbar_wait(sempty_bar(place), ((group / kScaleRing) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          uint32_t w[3][4][4];
          gather_scales(p.sa, tl.m0 + int(rank) * kRows, kb, p.kblocks, lane, w[0]);
          gather_scales(p.sb, tl.n0, kb, p.kblocks, lane, w[1]);
          gather_scales(p.sb, tl.n0 + 128, kb, p.kblocks, lane, w[2]);
          const uint32_t to = base + S::scale_off + place * kScaleBytes + uint32_t(lane) * 16u;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int part = 0; part < 3; ++part)
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + uint32_t(i) * kScaleWord + uint32_t(part) * 512u), "r"(w[part][0][i]),
                           "r"(w[part][1][i]), "r"(w[part][2][i]), "r"(w[part][3][i])
                           : "memory");
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(sfull0 + place * 8u);
        }
      }
      if (!ok && lane == 0) give_up(36);
    }
  } else {
    // ------------------------------------------------------------------ epilogue warps (per CTA: its 128 rows)
    const int ew = warp - 2, quad = warp & 3, part = ew >> 2;
    const bool sectors = L.sectors != 0;
    const int chunks = (EPI == kGated ? L.half : 2 * L.half) / 64;
    const Activation act = activation_of(L.activation);
    uint32_t tile_it = 0;
    bool ok = true;
    for (int t = pair_id; t < L.total_tiles && ok; t += num_pairs, ++tile_it) {
      const Tile tl = decode(L, t);
      const TcProduct& p = L.p[tl.prob];
      const uint32_t acc = tile_it & 1u, aph = (tile_it >> 1) & 1u;
      const uint32_t taddr = accumulator(acc) + (uint32_t(quad * 32) << 16);
      const int row0 = tl.m0 + int(rank) * kRows + quad * 32, row = row0 + lane;
      bool ready = false;
      auto wait_tile = [&]() {
        if (!ready) {
          ready = mbar_wait(tfull_bar(acc), aph, abort_flag);
          tc_fence_after();
        }
        return ready;
      };
      // two halves of the chunks, one for each warp of a quarter; 8 bits: the half that holds the shared columns (the end of the first accumulator, the
      // beginning of the second) has them in its first chunk
      const int per_part = chunks >= 2 ? chunks / 2 : 1;
      const bool backwards = EIGHT && acc == 0;
      for (int i = 0; i < per_part && part * per_part < chunks && ok; ++i) {
        const int chunk = part * per_part + (backwards ? per_part - 1 - i : i);
        const int col = tl.n0 + chunk * 64;
        if constexpr (EPI == kPlain) {
          if (!wait_tile()) { ok = false; break; }
          uint32_t v[64], w[32];
          load64(taddr + uint32_t(chunk * 64), v);
          tc_wait_ld();
          if (EIGHT && i == 0 && part == (acc == 0 ? 1 : 0)) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(shared_bar, 0));
          }
          if constexpr (A_MN) {
            if (p.sums && row < p.m && col < p.n) {
              float4* s = reinterpret_cast<float4*>(p.sums + row * p.ld_sums + col);
              if (L.add) {
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                  const float4 x = s[q];
                  v[4 * q] = __float_as_uint(__uint_as_float(v[4 * q]) + x.x);
                  v[4 * q + 1] = __float_as_uint(__uint_as_float(v[4 * q + 1]) + x.y);
                  v[4 * q + 2] = __float_as_uint(__uint_as_float(v[4 * q + 2]) + x.z);
                  v[4 * q + 3] = __float_as_uint(__uint_as_float(v[4 * q + 3]) + x.w);
                }
              }
              if (L.hold) {
#pragma unroll
                for (int q = 0; q < 16; ++q)
                  s[q] = make_float4(__uint_as_float(v[4 * q]), __uint_as_float(v[4 * q + 1]), __uint_as_float(v[4 * q + 2]), __uint_as_float(v[4 * q + 3]));
              }
            }
            if (L.hold) continue;
          }
#pragma unroll
          for (int k = 0; k < 32; ++k) w[k] = pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1]));
          if (row < p.m) {
            __nv_bfloat16* o = p.out[0] + row * p.ld[0] + col;
#pragma unroll
            for (int q = 0; q < 4; ++q) put16(o + 16 * q, w + 8 * q, p.n - col - 16 * q, sectors);
          }
        } else if constexpr (EPI == kGated) {
          if (!wait_tile()) { ok = false; break; }
          const bool inside = col < p.n && row0 < p.m, full = !CODES && L.keep;
          if (!inside) continue;
          const uint32_t at = taddr + uint32_t(chunk * 64), up = uint32_t(L.half);
          uint32_t eg = 0, eu = 0;
          bool odd_g = false, odd_u = false;
          uint8_t *cg = nullptr, *cu = nullptr;
          if constexpr (CODES) {
            eg = scale_byte(top_of_block(taddr, &odd_g));
            eu = scale_byte(top_of_block(taddr + up, &odd_u));
            if (row < p.m) {
              cg = static_cast<uint8_t*>(const_cast<void*>(L.gate.data)) + row * L.gate.ld + col;
              cu = static_cast<uint8_t*>(const_cast<void*>(L.up.data)) + row * L.up.ld + col;
              if (part == 0) {
                const_cast<uint8_t*>(L.gate.scales)[row * L.gate.lds + (col >> 7)] = uint8_t(eg);
                const_cast<uint8_t*>(L.up.scales)[row * L.up.lds + (col >> 7)] = uint8_t(eu);
              }
            }
          }
          const float ig = inverse_scale_of(eg), iu = inverse_scale_of(eu);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t g[32], u[32];
            __syncwarp();
            tc_ld32(at + uint32_t(h * 32), g);
            tc_ld32(at + up + uint32_t(h * 32), u);
            tc_wait_ld();
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              const int c = col + h * 32 + q * 16, left = row < p.m ? p.n - c : 0;
              uint32_t w[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const int at = q * 16 + 2 * k;
                float a[2], s;
#pragma unroll
                for (int e = 0; e < 2; ++e) activate<true>(act, __uint_as_float(g[at + e]), &a[e], &s);
                w[k] = pack2(a[0] * __uint_as_float(u[at]), a[1] * __uint_as_float(u[at + 1]));
              }
              put16(p.out[0] + row * p.ld[0] + c, w, left, sectors);
              if (full) {
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = pack2(__uint_as_float(g[q * 16 + 2 * k]), __uint_as_float(g[q * 16 + 2 * k + 1]));
                put16(p.out[1] + row * p.ld[1] + c, w, left, sectors);
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = pack2(__uint_as_float(u[q * 16 + 2 * k]), __uint_as_float(u[q * 16 + 2 * k + 1]));
                put16(p.out[2] + row * p.ld[2] + c, w, left, sectors);
              }
            }
            if (CODES && cg) {
              store_codes(cg + h * 32, g, ig, odd_g, p.n - col - h * 32, L.codes_wide != 0);
              store_codes(cu + h * 32, u, iu, odd_u, p.n - col - h * 32, L.codes_wide != 0);
            }
          }
        } else {
          // g and u come while the products still run
          const bool inside = col < p.n && row0 < p.m;
          uint32_t cg[CODES ? 16 : 32], cu[CODES ? 16 : 32];
          float sg = 0.f, su = 0.f;
          if (inside) {
            const bool mine = row < p.m;
            if constexpr (CODES) {
              const int left = mine ? p.n - col : 0;
              load_codes(static_cast<const uint8_t*>(L.gate.data) + row * L.gate.ld + col, cg, left, L.codes_wide != 0);
              load_codes(static_cast<const uint8_t*>(L.up.data) + row * L.up.ld + col, cu, left, L.codes_wide != 0);
              if (mine) {
                sg = scale_of(__ldg(L.gate.scales + row * L.gate.lds + (col >> 7)));
                su = scale_of(__ldg(L.up.scales + row * L.up.lds + (col >> 7)));
              }
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const int left = mine ? p.n - col - 16 * q : 0;
                get16(p.in[0] + row * p.ld_in[0] + col + 16 * q, cg + 8 * q, left, sectors);
                get16(p.in[1] + row * p.ld_in[1] + col + 16 * q, cu + 8 * q, left, sectors);
              }
            }
          }
          if (!wait_tile()) { ok = false; break; }
          if (!inside) continue;
          uint32_t v[32];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (q % 2 == 0) {
              __syncwarp();
              tc_ld32(taddr + uint32_t(chunk * 64 + q * 16), v);
              tc_wait_ld();
            }
            uint32_t w[8], wg[8], wu[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int pair = q * 8 + k;
              float2 g, u;
              if constexpr (CODES) {
                g = values_of(cg[pair >> 1] >> (16 * (pair & 1)));
                u = values_of(cu[pair >> 1] >> (16 * (pair & 1)));
                g.x *= sg; g.y *= sg;
                u.x *= su; u.y *= su;
              } else {
                g = make_float2(low(cg[pair]), high(cg[pair]));
                u = make_float2(low(cu[pair]), high(cu[pair]));
              }
              const float d0 = __uint_as_float(v[(2 * pair) & 31]), d1 = __uint_as_float(v[(2 * pair + 1) & 31]);
              float a0, a1, s0, s1;
              activate<true>(act, g.x, &a0, &s0);
              activate<true>(act, g.y, &a1, &s1);
              wg[k] = pack2(d0 * u.x * s0, d1 * u.y * s1);
              wu[k] = pack2(d0 * a0, d1 * a1);
              w[k] = pack2(a0 * u.x, a1 * u.y);
            }
            const int c = col + 16 * q, left = row < p.m ? p.n - c : 0;
            put16(p.out[1] + row * p.ld[1] + c, wg, left, sectors);
            put16(p.out[2] + row * p.ld[2] + c, wu, left, sectors);
            put16(p.out[0] + row * p.ld[0] + c, w, left, sectors);
          }
        }
      }
      if (ok && !wait_tile()) ok = false;           // a warp without a chunk hands the accumulator back, too
      if (!ok) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_cta(tempty_bar(acc), 0));
    }
    if (!ok && lane == 0) give_up(34);
  }
  tc_fence_before();
  __syncthreads();
  // The CTA's last tile is done or given up, so what the leader issued is about to have finished, too.  Waited for from the launch's beginning on, as warp 1
  // of the leader's peer could, this would be a wait for the whole launch, which may take longer than any limit meant for a part of it.
  if (warp == 1) {
    if (lane == 0 && !mbar_wait(drain_bar, 0, abort_flag, false, WAIT_CYCLES / 8)) atomicExch(L.status, 35);
    __syncwarp();
  }
  cluster_sync_all();            // neither CTA retires while its peer may still signal its barriers or read its tiles
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
}

// ------------------------------------------------------------------ host
template <bool A_MN, bool B_MN, bool EIGHT, int EPI, bool CODES = false>
int launch(const TcProducts& L, int device, int pairs, bool follows, cudaStream_t st) {
  static SharedMemoryLimit limit;
  using S = Shape<EIGHT>;
  if (!limit.raise(device, S::bytes, product_pair_kernel<A_MN, B_MN, EIGHT, EPI, CODES>)) return MUON_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(2 * std::min(L.total_tiles, pairs)), 1, 1);
  cfg.blockDim = dim3(S::threads, 1, 1);
  cfg.dynamicSmemBytes = S::bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = follows ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, product_pair_kernel<A_MN, B_MN, EIGHT, EPI, CODES>, L) == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

// Columns of B per CTA, and about how many clocks the launch takes: rounds of tiles times k-blocks, which take 560 clocks with 256 columns and 450 with
// 128 (whose operands are three quarters of the bytes for half of the work), and 12000 for what does not grow.  Narrow tiles pay where wide ones
// leave pairs without work.  8 bits: the scales of blocks of kept g and u need 128 columns of both, and MN-major operands come 128 columns at a time.
struct PairPlan {
  int half;
  double clocks;
};
PairPlan plan_pairs(const Product* list, int count, int sms) {
  const Product& first = list[0];
  const bool eight = first.a[0].type == kTypeE4m3, gated = first.e.kind == kGated;
  const bool may_narrow = !(eight && first.b[0].mn_major) && !(gated && first.e.gate_up_type == kTypeE4m3);
  PairPlan best = {};
  for (int half = 128; half >= (may_narrow ? 64 : 128); half /= 2) {
    const int64_t cols = gated ? half : 2 * half, pairs = sms / 2;
    int64_t tiles = 0, kblocks = 0;
    for (int i = 0; i < count; ++i) {
      tiles += (int64_t(list[i].m) + 2 * kRows - 1) / (2 * kRows) * ((list[i].n + cols - 1) / cols);
      kblocks = std::max<int64_t>(kblocks, int64_t((list[i].k + (eight ? 127 : 63)) / (eight ? 128 : 64)) * list[i].segments);
    }
    const double clocks = double((tiles + pairs - 1) / pairs) * double(kblocks) * (half == 128 ? 560 : 450) + 12000;
    if (half == 128 || clocks < best.clocks) best = {half, clocks};
  }
  return best;
}

}  // namespace

double products_tc_clocks(const Product* list, int count, int sms) { return plan_pairs(list, count, sms).clocks; }

bool products_tc_take(const Product* list, int count) {
  if (count < 1 || count > kMaxProducts) return false;
  for (int i = 0; i < count; ++i) {
    const Product& p = list[i];
    const Epilogue& e = p.e;
    const int type = p.a[0].type, ns = e.kind == kGated ? 2 : p.segments;
    if (!e.sums && int64_t(p.k) * p.segments > kMostSum) return false;
    if (p.m < 1 || p.n < 1 || p.k < 1 || e.type != kTypeBf16 || e.kind != list[0].e.kind || type != list[0].a[0].type) return false;
    if (type != kTypeBf16 && type != kTypeE4m3) return false;
    for (int s = 0; s < ns; ++s) {
      const Operand& b = p.b[s];
      if (b.type != type || !addressable(b.data, b.ld, type) || b.mn_major != list[0].b[0].mn_major) return false;
      if (b.type == kTypeE4m3 && b.mn_major && b.block_rows != kBlock) return false;
    }
    for (int s = 0; s < p.segments; ++s) {
      const Operand& a = p.a[s];
      if (a.type != type || !addressable(a.data, a.ld, type) || a.mn_major != list[0].a[0].mn_major) return false;
    }
    const bool amn = p.a[0].mn_major, bmn = p.b[0].mn_major;
    if (type == kTypeE4m3 ? amn || e.kind != kPlain || p.segments != 1 : (e.kind == kGated && (amn || bmn)) || (e.kind == kGrad && (amn || !bmn)) || (amn && !bmn))
      return false;
    if (!addressable(e.c, e.ldc, kTypeBf16)) return false;
    if (e.kind == kGated && e.gate && (!addressable(e.gate, e.ld_gate, kTypeBf16) || !addressable(e.up, e.ld_up, kTypeBf16))) return false;
    if (e.kind == kGrad) {
      if (!addressable(e.gate, e.ld_gate, kTypeBf16) || !addressable(e.up, e.ld_up, kTypeBf16)) return false;
      if (e.gate_up_type == kTypeBf16 && (!addressable(e.in_gate.data, e.in_gate.ld, kTypeBf16) || !addressable(e.in_up.data, e.in_up.ld, kTypeBf16))) return false;
    }
  }
  return true;
}

int launch_products_tc(muon_ctx* ctx, const Product* list, int count, Before before, cudaStream_t st) {
  const int sms = tc_pair_grid_setup(ctx->device);
  if (sms < 0) return sms;
  if (!ctx->tmap_encode) return MUON_ERR_CUDA;
  const bool follows = before != kBeforeAny;
  TcProducts L = {};
  const Epilogue& e0 = list[0].e;
  const bool eight = list[0].a[0].type == kTypeE4m3, amn = list[0].a[0].mn_major, bmn = list[0].b[0].mn_major;
  const bool codes = e0.gate_up_type == kTypeE4m3 && e0.kind != kPlain;
  const int pairs = sms / 2, dev = ctx->device;
  L.count = count;
  L.half = plan_pairs(list, count, sms).half;
  L.activation = e0.activation;
  L.keep = e0.kind == kGated && e0.gate;
  L.add = e0.add;
  L.hold = e0.hold;
  L.gate = e0.in_gate;
  L.up = e0.in_up;
  L.codes_wide = codes && addressable(L.gate.data, L.gate.ld, kTypeE4m3) && addressable(L.up.data, L.up.ld, kTypeE4m3);
  L.sectors = 1;
  L.status = ctx->d_status;
  Encoder enc = {ctx};
  int64_t tiles = 0;
  for (int i = 0; i < count; ++i) {
    const Product& q = list[i];
    TcProduct& p = L.p[i];
    p.m = q.m;
    p.n = q.n;
    p.kblocks = (q.k + (eight ? 127 : 63)) / (eight ? 128 : 64);
    p.segments = q.segments;
    p.tile_cols = q.e.kind == kGated ? L.half : 2 * L.half;
    p.tiles_m = (q.m + 2 * kRows - 1) / (2 * kRows);
    p.tiles_n = (q.n + p.tile_cols - 1) / p.tile_cols;
    p.tile_begin = int32_t(tiles);
    tiles += int64_t(p.tiles_m) * p.tiles_n;
    if (tiles > INT32_MAX - 4096) return MUON_ERR_UNSUPPORTED;
    for (int s = 0; s < q.segments; ++s) enc.operand(&p.a[s], q.a[s], q.m, q.k, kRows);
    for (int s = 0; s < (q.e.kind == kGated ? 2 : q.segments); ++s) enc.operand(&p.b[s], q.b[s], q.n, q.k, uint32_t(L.half));
    auto rows = [&](__nv_bfloat16** to, int64_t* ld, const void* data, int64_t stride) {
      *to = static_cast<__nv_bfloat16*>(const_cast<void*>(data));
      *ld = stride;
      L.sectors = L.sectors && reinterpret_cast<uintptr_t>(data) % 32 == 0 && stride % 16 == 0;
    };
    rows(&p.out[0], &p.ld[0], q.e.c, q.e.ldc);
    if (q.e.kind == kGrad || (q.e.kind == kGated && q.e.gate)) {
      rows(&p.out[1], &p.ld[1], q.e.gate, q.e.ld_gate);
      rows(&p.out[2], &p.ld[2], q.e.up, q.e.ld_up);
    }
    if (q.e.kind == kGrad && !codes) {
      rows(const_cast<__nv_bfloat16**>(&p.in[0]), &p.ld_in[0], q.e.in_gate.data, q.e.in_gate.ld);
      rows(const_cast<__nv_bfloat16**>(&p.in[1]), &p.ld_in[1], q.e.in_up.data, q.e.in_up.ld);
    }
    p.sums = q.e.sums;
    p.ld_sums = q.e.ld_sums;
    if (eight) {
      p.sa = scales_of(q.a[0], q.m);
      p.sb = scales_of(q.b[0], q.n);
    }
  }
  if (!enc.ok) return MUON_ERR_CUDA;
  L.total_tiles = int32_t(tiles);
  if (eight) return bmn ? launch<false, true, true, kPlain>(L, dev, pairs, follows, st) : launch<false, false, true, kPlain>(L, dev, pairs, follows, st);
  if (e0.kind == kGated) return codes ? launch<false, false, false, kGated, true>(L, dev, pairs, follows, st) : launch<false, false, false, kGated>(L, dev, pairs, follows, st);
  if (e0.kind == kGrad) return codes ? launch<false, true, false, kGrad, true>(L, dev, pairs, follows, st) : launch<false, true, false, kGrad>(L, dev, pairs, follows, st);
  if (amn) return launch<true, true, false, kPlain>(L, dev, pairs, follows, st);
  return bmn ? launch<false, true, false, kPlain>(L, dev, pairs, follows, st) : launch<false, false, false, kPlain>(L, dev, pairs, follows, st);
}

}  // namespace muon
