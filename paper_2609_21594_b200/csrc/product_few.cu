// Matrix products of few rows (tokens) on the tensor cores: what counts is how fast the weights come in.
//
// The operands change places: 128 rows of the weights are the 128 rows of tcgen05.mma, the tokens (up to 128, a multiple of 16) its columns, so that a
// token costs no more than its own work.  A block takes one tile of weight rows (gated: the same 128 rows of w_gate and of w_up, two accumulators)
// and a part of k; the blocks of a cluster take the other parts.  Each leaves its sums in its shared memory, over the ring that
// the operands came through, the cluster meets, and every block adds the parts of some of the tokens in the order of the ranks, so the sum is
// the same in every run.  A warp then holds 128 columns of one token: a coalesced row, and one block of the 8-bit form.
//
// Two blocks run on a multiprocessor, so one loads while the other adds up.  Where the call before this one in the stream is a part of the same call,
// the launch may begin before that one has ended: weights, which it does not write, are requested at once, tokens after griddepcontrol.wait.
//
// What bounds it.  One token: the bytes of the weights (4096 x 14336, both products 58 us, 6.1 TB/s; the kernel of CTA pairs takes 137).  More tokens: 64
// bytes a clock that a multiprocessor takes in, and the sums on their way through shared memory (128 tokens 78 us against 109); from a few
// hundred on the pairs win, by the estimate of plan_few (2048 x 5632, two products: 256 tokens 33 us against 41, 512 tokens 51 with the pairs' first product
// and 85 without).
//
// All waits are bounded, as in the Newton-Schulz kernel; a block that gives up still meets its cluster.
#include "product_tc.cuh"

namespace muon {
namespace {

using namespace prod;

constexpr int kRowsW = 128;                     // weight rows of a tile
constexpr int kThreads = 256;                   // warp 0: TMA; 1: matrix instructions; 2: scales; 4 to 7 read the accumulators; all add up
constexpr uint32_t kTileBytes = kRowsW * 128;   // 16 KiB
constexpr int kMaxStages = 8;
constexpr uint32_t kHalfSm = 112 * 1024;        // of shared memory for each of two blocks
constexpr uint32_t kWholeSm = 224 * 1024;
constexpr uint32_t kWord = 2 * 512;             // scales of four k-blocks: 128 weight rows and 128 tokens
constexpr uint32_t kScales = kScaleBlocks / 4 * kWord;
constexpr int kScaleRing = 2;
constexpr int kMaxSplit = 8;
constexpr int kMaxTokens = 128;                 // of a block

struct FewArgs {
  CUtensorMap w[2], x[2];                       // of each segment; gated: w_gate and w_up
  __nv_bfloat16* out[3];                        // C; or h, g, u; or h, dg, du
  int64_t ld[3];
  const __nv_bfloat16* in[2];                   // g, u
  int64_t ld_in[2];
  Operand gate, up;                             // 8-bit g and u
  Scales sw, sx;
  int32_t m, n, kblocks, segments;
  int32_t tokens;                               // columns of the instruction, a multiple of 16; blockIdx.y: which of them
  int32_t stages, split, columns;               // columns: of tensor memory
  int32_t activation, keep, codes_wide;
  uint32_t stage_bytes, scale_off, bar_off;
  int32_t* status;
};

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void tc_mma_scaled(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_copy_scales(uint32_t d_tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(d_tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ float4 load_peer(uint32_t addr, uint32_t rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(map_to_cta(addr, rank)) : "memory");
  return v;
}
// The address field of a descriptor.  In a block that is not the first of its cluster the high bits of an address hold the rank, and would run
// into the field beside it.
__device__ __forceinline__ uint32_t descriptor_address(uint32_t saddr) { return (saddr & 0x3FFFFu) >> 4; }
__device__ __forceinline__ void wait_for_call_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// W_MN: the weights are summed over their rows.  CODES: as in the kernel of CTA pairs.
template <bool W_MN, bool EIGHT, int EPI, bool CODES>
__global__ void __launch_bounds__(kThreads, 2) product_few_kernel(const __grid_constant__ FewArgs L) {
  constexpr int kTiles = EPI == kGated ? 2 : 1;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (base - raw);
  const uint32_t bars = base + L.bar_off;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen_base + L.bar_off + 240);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_base + L.bar_off + 248);
  auto full_bar = [&](int s) { return bars + uint32_t(s) * 8u; };
  auto empty_bar = [&](int s) { return bars + uint32_t(kMaxStages + s) * 8u; };
  auto sfull_bar = [&](uint32_t s) { return bars + uint32_t(2 * kMaxStages + s) * 8u; };
  auto sempty_bar = [&](uint32_t s) { return bars + uint32_t(2 * kMaxStages + kScaleRing + s) * 8u; };
  const uint32_t done_bar = bars + uint32_t(2 * kMaxStages + 2 * kScaleRing) * 8u;

  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int n0 = int(blockIdx.x / unsigned(L.split)) * kRowsW, t0 = int(blockIdx.y) * L.tokens;
  const int all_kb = L.kblocks * L.segments;
  const int kb0 = int(int64_t(all_kb) * rank / L.split), kb1 = int(int64_t(all_kb) * (rank + 1) / L.split);
  auto give_up = [&](int code) {
    *abort_flag = 1;
    atomicExch(L.status, code);
  };
  if (threadIdx.x == 0) {
    for (int s = 0; s < L.stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (uint32_t s = 0; s < kScaleRing; ++s) {
      mbar_init(sfull_bar(s), 1);
      mbar_init(sempty_bar(s), 1);
    }
    mbar_init(done_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(L.columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // the next part of the call may begin
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t scale_col = tmem_base + uint32_t(kTiles * L.tokens);

  if (warp == 0) {
    if (lane == 0) {
      bool ok = true;
      auto weights = [&](int kb, int s) {
        const int seg = kb >= L.kblocks ? 1 : 0, k0 = (kb - seg * L.kblocks) * (EIGHT ? 128 : 64);
        const uint32_t to = base + uint32_t(s) * L.stage_bytes;
        mbar_expect_tx(full_bar(s), L.stage_bytes);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          const CUtensorMap* map = &L.w[kTiles == 2 ? i : seg];
          if constexpr (W_MN && !EIGHT) {
            tma_load(to, map, full_bar(s), n0, k0);
            tma_load(to + kTileBytes / 2, map, full_bar(s), n0 + 64, k0);
          } else if constexpr (W_MN) {
            tma_load(to, map, full_bar(s), n0, k0);
          } else {
            tma_load(to + uint32_t(i) * kTileBytes, map, full_bar(s), k0, n0);
          }
        }
      };
      auto rows = [&](int kb, int s) {
        const int seg = kb >= L.kblocks ? 1 : 0, k0 = (kb - seg * L.kblocks) * (EIGHT ? 128 : 64);
        tma_load(base + uint32_t(s) * L.stage_bytes + kTiles * kTileBytes, &L.x[seg], full_bar(s), k0, t0);
      };
      const int first = min(L.stages, kb1 - kb0);
      for (int i = 0; i < first; ++i) weights(kb0 + i, i);
      wait_for_call_before();
      for (int i = 0; i < first; ++i) rows(kb0 + i, i);
      int s = first == L.stages ? 0 : first;
      uint32_t ph = 0;
      for (int kb = kb0 + first; kb < kb1; ++kb) {
        if (!mbar_wait(empty_bar(s), ph, abort_flag)) { ok = false; break; }
        weights(kb, s);
        rows(kb, s);
        if (++s == L.stages) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (!ok) {
        give_up(41);
        for (int i = 0; i < 64; ++i) __nanosleep(1000);      // what was requested may still be landing
      }
    }
  } else if (warp == 1) {
    bool ok = true;
    auto all = [](bool v) { return __all_sync(0xffffffffu, v) != 0; };
    constexpr uint64_t w_hi = W_MN ? kDescMN : kDescK;
    constexpr uint32_t w_step = W_MN ? (EIGHT ? 32 : 16) * 128 / 16 : 2;
    const uint32_t idesc = EIGHT ? make_idesc_scaled(W_MN, false, kRowsW, L.tokens) : make_idesc(false, kRowsW, L.tokens, W_MN);
    int s = 0;
    uint32_t ph = 0, group = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      const int j = kb - kb0;
      if constexpr (EIGHT) {
        if (j % 4 == 0) {
          const uint32_t place = group % kScaleRing;
          if (j % kScaleBlocks == 0) {
            ok = all(mbar_wait(sfull_bar(place), (group / kScaleRing) & 1u, abort_flag));
            if (!ok) break;
            tc_fence_after();
          }
          const bool last = j % kScaleBlocks == kScaleBlocks - 4 || kb + 4 >= kb1;
          elected(true, [&] {
            const uint32_t from = descriptor_address(base + L.scale_off + place * kScales + uint32_t(j % kScaleBlocks / 4) * kWord);
#pragma unroll
            for (int i = 0; i < 2; ++i) tc_copy_scales(scale_col + uint32_t(4 * i), kDescScales | uint64_t(from + uint32_t(i) * 32u));
            if (last) tc_commit(sempty_bar(place));
          });
          if (last) ++group;
        }
      }
      ok = all(mbar_wait(full_bar(s), ph, abort_flag));
      if (!ok) break;
      tc_fence_after();
      elected(true, [&] {
        const uint32_t at = descriptor_address(base + uint32_t(s) * L.stage_bytes);
        const uint64_t dx = kDescK | uint64_t(at + uint32_t(kTiles) * (kTileBytes >> 4));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t more = (j > 0 || k > 0) ? 1u : 0u;
#pragma unroll
          for (int i = 0; i < kTiles; ++i) {
            const uint64_t dw = (w_hi | uint64_t(at + uint32_t(i) * (kTileBytes >> 4))) + uint64_t(k * w_step);
            if constexpr (EIGHT)
              tc_mma_scaled(tmem_base, dw, dx + uint64_t(k * 2), idesc | scale_byte_ids(uint32_t(j & 3)), scale_col, scale_col + 4, more);
            else
              tc_mma(tmem_base + uint32_t(i * L.tokens), dw, dx + uint64_t(k * 2), idesc, more);
          }
        }
        tc_commit(empty_bar(s));
      });
      if (++s == L.stages) {
        s = 0;
        ph ^= 1u;
      }
    }
    if (!ok && lane == 0) give_up(43);
    __syncwarp();
    elected(true, [&] { tc_commit(done_bar); });
  } else if (EIGHT && warp == 2) {
    if constexpr (EIGHT) {
      bool ok = true;
      wait_for_call_before();
      uint32_t group = 0;
      for (int kb = kb0; kb < kb1; kb += kScaleBlocks, ++group) {
        const uint32_t place = group % kScaleRing;
        ok = mbar_wait(sempty_bar(place), ((group / kScaleRing) & 1u) ^ 1u, abort_flag);
        if (!ok) break;
        uint32_t w[2][4][4];
        gather_scales(L.sw, n0, kb, kb1, lane, w[0]);
        gather_scales(L.sx, t0, kb, kb1, lane, w[1]);
        const uint32_t to = base + L.scale_off + place * kScales + uint32_t(lane) * 16u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int part = 0; part < 2; ++part)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + uint32_t(i) * kWord + uint32_t(part) * 512u), "r"(w[part][0][i]),
                         "r"(w[part][1][i]), "r"(w[part][2][i]), "r"(w[part][3][i])
                         : "memory");
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(sfull_bar(place));
      }
      if (!ok && lane == 0) give_up(46);
    }
  }
  // ------------------------------------------------------------------ sums of this part of k to shared memory: [accumulator][token][weight row]
  if (warp >= 4) {
    if (!mbar_wait(done_bar, 0, abort_flag, false) && lane == 0) atomicExch(L.status, 44);
    tc_fence_after();
    __syncwarp();
    const int quad = warp & 3;
    const uint32_t from = tmem_base + (uint32_t(quad * 32) << 16);
    float* to = reinterpret_cast<float*>(gen_base) + quad * 32 + lane;
    for (int c = 0; c < kTiles * L.tokens; c += 16) {
      uint32_t v[16];
      tc_ld16(from + uint32_t(c), v);
      tc_wait_ld();
#pragma unroll
      for (int i = 0; i < 16; ++i) to[(c + i) * kRowsW] = __uint_as_float(v[i]);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(L.columns) : "memory");
  }
  cluster_sync_all();                           // every block of the cluster has left its sums
  const Activation act = activation_of(L.activation);
  const int col = n0 + lane * 4;
  for (int i = int(rank) * (kThreads / 32) + warp; i < min(L.tokens, L.m - t0); i += L.split * (kThreads / 32)) {
    const int t = t0 + i;
    float sum[kTiles][4];
#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
      const uint32_t at = base + uint32_t((k * L.tokens + i) * kRowsW + lane * 4) * 4u;
      float4 part[kMaxSplit];
#pragma unroll
      for (int r = 0; r < kMaxSplit; ++r)
        if (r < L.split) part[r] = load_peer(at, uint32_t(r));
      float4 v = part[0];
#pragma unroll
      for (int r = 1; r < kMaxSplit; ++r)
        if (r < L.split) {
          v.x += part[r].x;
          v.y += part[r].y;
          v.z += part[r].z;
          v.w += part[r].w;
        }
      sum[k][0] = v.x; sum[k][1] = v.y; sum[k][2] = v.z; sum[k][3] = v.w;
    }
    const int left = L.n - col;
    const bool inside = left > 0, whole = left >= 4;
    auto put = [&](int which, float a, float b, float c, float d) {
      const uint32_t w[2] = {pack2(a, b), pack2(c, d)};
      __nv_bfloat16* to = L.out[which] + t * L.ld[which] + col;
      if (whole) {
        *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
      } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (i < left) reinterpret_cast<uint16_t*>(to)[i] = uint16_t(w[i >> 1] >> (16 * (i & 1)));
      }
    };
    if constexpr (EPI == kPlain) {
      put(0, sum[0][0], sum[0][1], sum[0][2], sum[0][3]);
    } else if constexpr (EPI == kGated) {
      const float(&g)[4] = sum[0];
      const float(&u)[4] = sum[kTiles - 1];
      float h[4], slope;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        activate<true>(act, g[i], &h[i], &slope);
        h[i] *= u[i];
      }
      put(0, h[0], h[1], h[2], h[3]);
      if constexpr (CODES) {                    // the warp's 128 columns are a block
        auto keep = [&](const Operand& o, const float (&v)[4]) {
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) top = max(top, finite_bits(v[i]));
          const uint32_t e = scale_byte(__reduce_max_sync(0xffffffffu, top));
          const float inverse = inverse_scale_of(e);
          uint32_t c[2];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            c[i] = __nv_cvt_float2_to_fp8x2(make_float2(infinite_to_nan(v[2 * i]) * inverse, infinite_to_nan(v[2 * i + 1]) * inverse), __NV_SATFINITE, __NV_E4M3);
          uint8_t* p = static_cast<uint8_t*>(const_cast<void*>(o.data)) + t * o.ld + col;
          if (whole && L.codes_wide) {
            *reinterpret_cast<uint32_t*>(p) = c[0] | c[1] << 16;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (i < left) p[i] = uint8_t(c[i >> 1] >> (8 * (i & 1)));
          }
          if (lane == 0) const_cast<uint8_t*>(o.scales)[t * o.lds + (col >> 7)] = uint8_t(e);
        };
        keep(L.gate, g);
        keep(L.up, u);
      } else if (L.keep) {
        put(1, g[0], g[1], g[2], g[3]);
        put(2, u[0], u[1], u[2], u[3]);
      }
    } else {
      float g[4] = {0, 0, 0, 0}, u[4] = {0, 0, 0, 0};
      if (inside) {
        if constexpr (CODES) {
          auto take = [&](const Operand& o, float (&v)[4]) {
            const uint8_t* p = static_cast<const uint8_t*>(o.data) + t * o.ld + col;
            const float scale = scale_of(__ldg(o.scales + t * o.lds + (col >> 7)));
            uint32_t c = 0;
            if (whole && L.codes_wide) {
              c = __ldg(reinterpret_cast<const uint32_t*>(p));
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (i < left) c |= uint32_t(__ldg(p + i)) << (8 * i);
            }
            const float2 lo = values_of(c), hi = values_of(c >> 16);
            v[0] = lo.x * scale; v[1] = lo.y * scale; v[2] = hi.x * scale; v[3] = hi.y * scale;
          };
          take(L.gate, g);
          take(L.up, u);
        } else {
          auto take = [&](int which, float (&v)[4]) {
            const __nv_bfloat16* from = L.in[which] + t * L.ld_in[which] + col;
            uint2 x = make_uint2(0, 0);
            if (whole) {
              x = __ldg(reinterpret_cast<const uint2*>(from));
            } else {
              const uint16_t* q = reinterpret_cast<const uint16_t*>(from);
              x.x = uint32_t(__ldg(q)) | (left > 1 ? uint32_t(__ldg(q + 1)) << 16 : 0u);
              x.y = left > 2 ? uint32_t(__ldg(q + 2)) : 0u;
            }
            v[0] = low(x.x); v[1] = high(x.x); v[2] = low(x.y); v[3] = high(x.y);
          };
          take(0, g);
          take(1, u);
        }
      }
      float a[4], s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) activate<true>(act, g[i], &a[i], &s[i]);
      const float(&d)[4] = sum[0];
      put(1, d[0] * u[0] * s[0], d[1] * u[1] * s[1], d[2] * u[2] * s[2], d[3] * u[3] * s[3]);
      put(2, d[0] * a[0], d[1] * a[1], d[2] * a[2], d[3] * a[3]);
      put(0, a[0] * u[0], a[1] * u[1], a[2] * u[2], a[3] * u[3]);
    }
  }
  cluster_sync_all();                           // a block's shared memory stays until its peers have read it
}

template <bool W_MN, bool EIGHT, int EPI, bool CODES = false>
int launch(const FewArgs& L, int device, uint32_t bytes, bool follows, cudaStream_t st) {
  static SharedMemoryLimit limit;
  if (!limit.raise(device, kWholeSm, product_few_kernel<W_MN, EIGHT, EPI, CODES>)) return MUON_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned((L.n + kRowsW - 1) / kRowsW * L.split), unsigned((L.m + L.tokens - 1) / L.tokens), 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(L.split);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = follows ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, product_few_kernel<W_MN, EIGHT, EPI, CODES>, L) == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

// How the work is cut, and about how many clocks that takes.
struct FewPlan {
  int tokens, split, stages;
  uint32_t stage_bytes, sums, extra;
  double clocks;
};
FewPlan plan_few(const Product& q, int sms) {
  FewPlan r = {};
  const bool eight = q.a[0].type == kTypeE4m3;
  const int tiles = q.e.kind == kGated ? 2 : 1;
  const int64_t wide = (int64_t(q.n) + kRowsW - 1) / kRowsW, total = int64_t((q.k + (eight ? 127 : 63)) / (eight ? 128 : 64)) * q.segments;
  r.extra = (eight ? kScaleRing * kScales : 0) + 256 + 1024;
  int64_t blocks = 0, on_sm = 0;
  uint32_t room = 0;
  // As many blocks as fit at once: first by parts of k, then, where tiles and k are few, by parts of the tokens, each of which reads the weights again
  // (from L2) but adds up less.
  for (int parts = (q.m + kMaxTokens - 1) / kMaxTokens;; parts *= 2) {
    r.tokens = ((q.m + parts - 1) / parts + 15) / 16 * 16;
    r.sums = uint32_t(tiles * r.tokens) * kRowsW * 4u;  // take the ring's place in the end
    room = r.sums + r.extra <= kHalfSm ? kHalfSm : kWholeSm;
    on_sm = room == kHalfSm ? 2 : 1;
    r.split = int(std::max<int64_t>(1, std::min<int64_t>({kMaxSplit, sms * on_sm / wide, total})));
    blocks = wide * r.split * ((q.m + r.tokens - 1) / r.tokens);
    if (r.tokens == 16 || blocks * 2 > sms * on_sm) break;
  }
  const int64_t each = (total + r.split - 1) / r.split;
  r.stage_bytes = uint32_t(tiles) * kTileBytes + uint32_t(r.tokens) * 128u;
  r.stages = int(std::min<int64_t>({kMaxStages, (room - r.extra) / r.stage_bytes, each}));
  // A multiprocessor takes in 64 bytes a clock; sums are written, read by a peer and added at 16 bytes a clock.
  const double busy = double(std::min<int64_t>(on_sm, (blocks + sms - 1) / sms)) * (double(each) * r.stage_bytes / 64 + r.sums / 16.0);
  r.clocks = double((blocks + sms * on_sm - 1) / (sms * on_sm)) * busy + 8000;
  return r;
}

}  // namespace

bool product_few_takes(const Product& p, int sms) {
  // what grows has to be clearly less, what does not is about 4000 clocks less in any case
  return p.m <= kFewRows && !p.a[0].mn_major && plan_few(p, sms).clocks < 0.85 * products_tc_clocks(&p, 1, sms) + 1800;
}

int launch_product_few(muon_ctx* ctx, const Product& q, int sms, Before before, cudaStream_t st) {
  if (!ctx->tmap_encode) return MUON_ERR_CUDA;
  const bool follows = before == kBeforeLeavesB;
  FewArgs L = {};
  const Epilogue& e = q.e;
  const bool eight = q.a[0].type == kTypeE4m3, wmn = q.b[0].mn_major, codes = e.kind != kPlain && e.gate_up_type == kTypeE4m3;
  const int tiles = e.kind == kGated ? 2 : 1;
  L.m = q.m;
  L.n = q.n;
  L.kblocks = (q.k + (eight ? 127 : 63)) / (eight ? 128 : 64);
  L.segments = q.segments;
  const FewPlan plan = plan_few(q, sms);
  L.tokens = plan.tokens;
  L.split = plan.split;
  L.stages = plan.stages;
  L.stage_bytes = plan.stage_bytes;
  const uint32_t ring = std::max(uint32_t(L.stages) * L.stage_bytes, plan.sums);
  L.scale_off = (ring + 1023u) & ~1023u;
  L.bar_off = L.scale_off + (eight ? kScaleRing * kScales : 0);
  const int columns = tiles * L.tokens + (eight ? 8 : 0);
  for (L.columns = 32; L.columns < columns;) L.columns *= 2;
  L.activation = e.activation;
  L.keep = e.kind == kGated && e.gate;
  L.gate = e.in_gate;
  L.up = e.in_up;
  L.codes_wide = codes && addressable(L.gate.data, L.gate.ld, kTypeE4m3) && addressable(L.up.data, L.up.ld, kTypeE4m3);
  L.status = ctx->d_status;
  Encoder enc = {ctx};
  for (int s = 0; s < (tiles == 2 ? 2 : q.segments); ++s) enc.operand(&L.w[s], q.b[s], q.n, q.k, kRowsW);
  for (int s = 0; s < q.segments; ++s) enc.operand(&L.x[s], q.a[s], q.m, q.k, uint32_t(L.tokens));
  if (!enc.ok) return MUON_ERR_CUDA;
  auto rows = [](auto* to, int64_t* ld, const void* data, int64_t stride) {
    *to = static_cast<__nv_bfloat16*>(const_cast<void*>(data));
    *ld = stride;
  };
  rows(&L.out[0], &L.ld[0], e.c, e.ldc);
  rows(&L.out[1], &L.ld[1], e.gate, e.ld_gate);
  rows(&L.out[2], &L.ld[2], e.up, e.ld_up);
  if (e.kind == kGrad && !codes) {
    rows(&L.in[0], &L.ld_in[0], e.in_gate.data, e.in_gate.ld);
    rows(&L.in[1], &L.ld_in[1], e.in_up.data, e.in_up.ld);
  }
  if (eight) {
    L.sw = scales_of(q.b[0], q.n);
    L.sx = scales_of(q.a[0], q.m);
  }
  const int dev = ctx->device;
  const uint32_t bytes = std::max(L.bar_off + 256 + 1024, shared_for_columns(uint32_t(L.columns)));
  if (eight) return wmn ? launch<true, true, kPlain>(L, dev, bytes, follows, st) : launch<false, true, kPlain>(L, dev, bytes, follows, st);
  if (e.kind == kGated) return codes ? launch<false, false, kGated, true>(L, dev, bytes, follows, st) : launch<false, false, kGated>(L, dev, bytes, follows, st);
  if (e.kind == kGrad) return codes ? launch<true, false, kGrad, true>(L, dev, bytes, follows, st) : launch<true, false, kGrad>(L, dev, bytes, follows, st);
  return wmn ? launch<true, false, kPlain>(L, dev, bytes, follows, st) : launch<false, false, kPlain>(L, dev, bytes, follows, st);
}

}  // namespace muon
