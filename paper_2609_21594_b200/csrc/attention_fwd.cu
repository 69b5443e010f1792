// Attention forward on the tensor cores (bf16): one pass over the keys with a running maximum and sum.
//
// A block owns two tiles of 128 queries of one head and walks the blocks of 128 keys that they see.  384 threads:
//   warps 0-3, 4-7  softmax of tile 0 and of tile 1: a thread owns one row (one TMEM lane) and keeps its 128 scores in registers, so maxima
//                   and sums need no exchange.  These two warpgroups take 216 registers per thread and leave 72 to the third: one spilled
//                   register costs dearly where shared memory leaves no first-level cache
//   warp 8          TMA producer: the two q tiles once, then rounds of a v tile and the k tile after it
//   warp 9          MMA issuer:  O_t += P_t v with P_t read from tensor memory, then S_t = q_t k^T of the next keys (128 x 128 x head_dim), for
//                   the tiles in turn.  (An issuer per tile lets the tiles' products mix, and each softmax waits for both: 519 against 507 us, below.)
//   warp 10         clears the rows of the last v tile that lie past the sequence's end
// Tensor memory: S_0, S_1 (128 columns each), O_0, O_1.  P_t takes the place of S_t, rounded once to bf16, the type of the product's
// operands: up to 2^-9 of each term, independently, so that o is off by about sqrt 2 of its own rounding.  The sum l takes P unrounded.  While one tile's softmax runs,
// the issuer works for the other.  A tcgen05.commit covers everything issued before it, so "S_t of block j is ready" also says that the
// product that read P_t of block j - 1 is done and O_t may be touched.
//
// The running maximum is raised only when a row's scores exceed it by more than 2^8 in the exponential: until then P is at most 256 and
// the sum is exact enough in fp32 (P's rounding is relative), and O, which sits in tensor memory, is not read and rewritten.
//
// Measured, causal, 32/8 heads of 128: 8192 tokens 507 to 522 us over several runs, 1053 to 1084 TFLOP/s of the pairs that count (63 to 65 % of the
// library's matrix product alone); 4 x 2048 tokens of heads of 64: 136 us, 502 TFLOP/s; a window of 1024 keys, 8192 tokens: 173 us, 747 TFLOP/s;
// 9 and 32 documents in 6000 tokens, heads of 64: 86 us, 260 and 126 TFLOP/s.  A round of one tile is a chain: softmax, about 1800 clocks, then O += P v and the next S,
// about 1150; two tiles share the tensor pipe, which is busy for 2200 of every 2980 clocks.  So the softmax bounds it, by issue slots: a share
// of the exponentials on the multiply-add pipe made it slower (570 to 600 us), as did two threads per row (539 to 580).  Heads of 64
// do half the products per exponential and come to half the rate.
#include <cuda_bf16.h>

#include "attention_tc.cuh"

namespace muon {
namespace {

using namespace attn;

constexpr int THREADS = 384, TMEM_COLS = 512, LOADER = 8, ISSUER = 9, SWEEPER = 10;
constexpr int SOFTMAX_REGS = 216, OTHER_REGS = 72;   // 2 x 216 + 72 = 3 x 168, what a block of 384 is launched with
constexpr float kRaise = 8.f;                    // log2 of the largest P

template <int BOXES> struct Smem {
  static constexpr uint32_t kTile = BOXES * BOX_BYTES;
  static constexpr int kStages = BOXES == 1 ? 4 : 2;
  static constexpr uint32_t q = 0, k = 2 * kTile, v = k + kStages * kTile, bars = v + kStages * kTile;
  static constexpr uint32_t bytes = bars + 256 + 1024;   // barriers, slack for the 1024-byte alignment of swizzled tiles
};

template <int BOXES>
__global__ void __launch_bounds__(THREADS, 1)
attention_forward_tc_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnArgs a) {
  using L = Smem<BOXES>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t bars = base + L::bars;
  auto q_full = [&](int t) { return bars + uint32_t(t) * 8u; };
  auto s_full = [&](int t) { return bars + uint32_t(2 + t) * 8u; };
  auto o_full = [&](int t) { return bars + uint32_t(4 + t) * 8u; };
  auto p_ready = [&](int t, int h) { return bars + uint32_t(6 + 2 * t + h) * 8u; };      // P of the first 64 keys, of the others
  constexpr int STAGES = L::kStages;
  auto full = [&](int s) { return bars + uint32_t(10 + s) * 8u; };
  auto empty = [&](int s) { return bars + uint32_t(10 + STAGES + s) * 8u; };
  const uint32_t done_bar = bars + uint32_t(10 + 2 * STAGES) * 8u, raw_bar = done_bar + 8u;
  static_assert((12 + 2 * STAGES) * 8 <= 192, "barriers");
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + L::bars + 192);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + L::bars + 200);

  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  // Heads vary fastest, so that blocks that share keys run together; within a batched call the last queries, which see most keys, go first.
  const int head = int(blockIdx.x % unsigned(a.hq)), kvh = head / (a.hq / a.hkv);
  int si, blk;
  if (!attn_find_block(a, int(blockIdx.x / unsigned(a.hq)), 2 * BLK, false, &si, &blk)) return;
  if (!a.nseq) {
    const int rest = int(blockIdx.x / unsigned(a.hq)), per = (a.nq + 2 * BLK - 1) / (2 * BLK);
    si = rest % a.batch;
    blk = per - 1 - rest / a.batch;
  }
  const AttnSeq s = attn_seq(a, si);
  const int r0 = blk * 2 * BLK;
  const BlockRange rg[2] = {key_blocks(a, s, r0), key_blocks(a, s, r0 + BLK)};
  int u0 = rg[0].n0, u1 = rg[0].n1;
  if (rg[1].n1 > rg[1].n0) {
    u0 = u1 > u0 ? min(u0, rg[1].n0) : rg[1].n0;
    u1 = max(u1, rg[1].n1);
  }

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full(t), 1);
      mbar_init(s_full(t), 1);
      mbar_init(p_ready(t, 0), 4);
      mbar_init(p_ready(t, 1), 4);
      mbar_init(o_full(t), 1);
    }
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 1);
    }
    mbar_init(done_bar, 1);
    mbar_init(raw_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == ISSUER) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t t_s[2] = {tmem, tmem + 128}, t_o[2] = {tmem + 256, tmem + 256 + BOXES * 64};
  const float c2 = a.scale * kLog2e;

  if (warp >= LOADER) {
    fewer_registers<OTHER_REGS>();
    if (warp == LOADER) {
      // ------------------------------------------------------------------ TMA producer
      if (lane == 0 && u1 > u0) {
        bool ok = true;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (rg[t].n1 <= rg[t].n0) continue;
          mbar_expect_tx(q_full(t), L::kTile);
          load_tile<BOXES>(base + L::q + t * L::kTile, &maps.q, q_full(t), head, s.q0 + r0 + t * BLK, s.tb);
        }
        // Round p brings v of block u0 + p - 1 and k of block u0 + p; the first has no v, the last no k.
        int p = 0;
        for (; p <= u1 - u0; ++p) {
          const int st = p % STAGES, j = u0 + p;
          if (!(ok = mbar_wait(empty(st), (uint32_t(p / STAGES) & 1u) ^ 1u, abort_flag))) break;
          // a v tile with rows past the end goes through the sweeper
          const uint32_t bar = j == u1 && u1 * BLK > s.kn ? raw_bar : full(st);
          mbar_expect_tx(bar, (p > 0) + (j < u1) == 2 ? 2 * L::kTile : L::kTile);
          if (p > 0) load_tile<BOXES>(base + L::v + st * L::kTile, &maps.v, bar, kvh, s.k0 + (j - 1) * BLK, s.tb);
          if (j < u1) load_tile<BOXES>(base + L::k + st * L::kTile, &maps.k, bar, kvh, s.k0 + j * BLK, s.tb);
        }
        if (!ok) {
          *abort_flag = 1;
          atomicExch(a.status, 21);
        }
        // Everything asked for must have landed before this block's shared memory is released.
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (rg[t].n1 > rg[t].n0) mbar_wait(q_full(t), 0, abort_flag, false, WAIT_CYCLES / 8);
        if (u1 * BLK > s.kn) mbar_wait(raw_bar, 0, abort_flag, false, WAIT_CYCLES / 8);
        for (int i = max(0, p - STAGES); i < p; ++i)
          if (!mbar_wait(full(i % STAGES), uint32_t(i / STAGES) & 1u, abort_flag, false, WAIT_CYCLES / 8)) atomicExch(a.status, 22);
      }
    } else if (warp == ISSUER) {
      // ------------------------------------------------------------------ MMA issuer
      if (u1 > u0) {
        const int ksteps = (a.dim + 15) / 16;
        const uint32_t idesc_o = make_idesc(true, BLK, ksteps * 16);
        bool ok = true;
        auto await = [&](uint32_t bar, uint32_t ph) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, ph, abort_flag)); };
        for (int p = 0; p <= u1 - u0 && ok; ++p) {
          const int st = p % STAGES, j = u0 + p - 1;
          const uint32_t v = base + L::v + uint32_t(st) * L::kTile, k = base + L::k + uint32_t(st) * L::kTile;
          await(full(st), uint32_t(p / STAGES) & 1u);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const bool pv = j >= rg[t].n0 && j < rg[t].n1, next = j + 1 >= rg[t].n0 && j + 1 < rg[t].n1;
            if (pv) {
              await(p_ready(t, 0), uint32_t(j - rg[t].n0) & 1u);
              tc_fence_after();                            // tensor memory written by other threads; tiles need no such fence
              elected(ok, [&] { mma_probs_rows<0, 4>(t_o[t], t_s[t], t_s[t] + 32, v, idesc_o, j > rg[t].n0); });
              await(p_ready(t, 1), uint32_t(j - rg[t].n0) & 1u);
              tc_fence_after();
            } else if (next) {
              await(q_full(t), 0);
            }
            elected(ok, [&] {
              if (pv) mma_probs_rows<4, 8>(t_o[t], t_s[t], t_s[t] + 32, v, idesc_o, true);
              if (pv && !next) tc_commit(o_full(t));
              if (next) {
                mma_rows_rows<BOXES>(t_s[t], base + L::q + uint32_t(t) * L::kTile, k, ksteps);    // over P_t, which the product before has read
                tc_commit(s_full(t));
              }
              if (t == 1) tc_commit(empty(st));
            });
          }
        }
        // Nothing may be in flight when tensor memory is freed.
        if (elect_one()) {
          if (!ok) {
            *abort_flag = 1;
            atomicExch(a.status, 23);
          }
          tc_commit(done_bar);
          if (!mbar_wait(done_bar, 0, abort_flag, false, WAIT_CYCLES / 8)) atomicExch(a.status, 24);
        }
      }
      __syncwarp();
    } else if (warp == SWEEPER) {
      // ------------------------------------------------------------------ rows past the end
      if (u1 > u0 && u1 * BLK > s.kn) {
        const int st = (u1 - u0) % STAGES;
        if (__all_sync(0xffffffffu, mbar_wait(raw_bar, 0, abort_flag)))
          clear_rows<BOXES>(base + L::v + uint32_t(st) * L::kTile, 0, s.kn - (u1 - 1) * BLK, lane, full(st));
        else if (lane == 0) *abort_flag = 1;
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax and results
    more_registers<SOFTMAX_REGS>();
    const int t = warp >> 2, quad = warp & 3;
    const int row = r0 + t * BLK + quad * 32 + lane;
    const uint32_t lanes = uint32_t(quad * 32) << 16;
    const BlockRange keys = t ? rg[1] : rg[0];
    const uint32_t ts = (t ? t_s[1] : t_s[0]) + lanes, to = (t ? t_o[1] : t_o[0]) + lanes;
    const int lo = attn_key_lo(a, s, row), hi = attn_key_hi(a, s, row);
    float m = -INFINITY;
    uint64_t l = 0;                                        // sums of the even and of the odd keys
    bool ok = true;
    for (int j = keys.n0; j < keys.n1; ++j) {
      ok = __all_sync(0xffffffffu, mbar_wait(s_full(t), uint32_t(j - keys.n0) & 1u, abort_flag));
      if (!ok) break;
      tc_fence_after();
      const int c0 = j * BLK;
      auto step = [&](auto with_mask) {
        constexpr bool MASK = decltype(with_mask)::value;
        uint32_t x[128];
#pragma unroll
        for (int i = 0; i < 4; ++i) tc_ld32(ts + i * 32, *reinterpret_cast<uint32_t(*)[32]>(&x[i * 32]));
        tc_wait_ld();
        if constexpr (MASK) {
          const int first = lo - c0, last = hi - c0;
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i < first || i >= last) x[i] = 0xff800000u;                // -inf
        }
        auto f = [&](int i) { return __uint_as_float(x[i]); };
        float top[4] = {f(0), f(1), f(2), f(3)};
#pragma unroll
        for (int i = 4; i < 124; i += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e) top[e] = max3(top[e], f(i + 2 * e), f(i + 2 * e + 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) top[e] = fmaxf(top[e], f(124 + e));
        const float mx = fmaxf(max3(top[0], top[1], top[2]), top[3]);
        const bool raise = mx > m && (m == -INFINITY || (mx - m) * c2 > kRaise);
        if (__any_sync(0xffffffffu, raise)) {
          const float shrink = raise ? exp2_approx((m - mx) * c2) : 1.f;
          if (raise) m = mx;
          l = mul2(l, twice(shrink));
          if (j > keys.n0) {
#pragma unroll 1
            for (int i = 0; i < BOXES * 8; ++i) {          // rare: few registers matter more than speed
              uint32_t o[8];
              tc_ld8(to + i * 8, o);
              tc_wait_ld();
#pragma unroll
              for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * shrink);
              tc_st8(to + i * 8, o);
            }
          }
        }
        const uint64_t scale = twice(c2), shift = twice(m == -INFINITY ? 0.f : -m * c2);
        uint64_t sum[2] = {0, 0};
        auto hand_over = [&](int h) {
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_ready(t, h));
        };
        uint32_t p[32];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint64_t v = exp2_approx(fma2(words(x[c * 32 + 2 * i], x[c * 32 + 2 * i + 1]), scale, shift));
            sum[i & 1] = add2(sum[i & 1], v);
            p[(c & 1) * 16 + i] = pack_bf16(v);
          }
          if (c == 2) hand_over(0);                        // the first half has long been stored: nothing waits
          if (c & 1) tc_st32(ts + (c >> 1) * 32, p);
        }
        hand_over(1);
        l = add2(l, add2(sum[0], sum[1]));
      };
      if (block_masked(a, s, r0 + t * BLK, c0)) step(Yes());
      else step(No());
    }
    const bool any = keys.n1 > keys.n0;
    if (ok && any) {
      ok = __all_sync(0xffffffffu, mbar_wait(o_full(t), 0, abort_flag));
      tc_fence_after();
    }
    if (!ok) {
      if (lane == 0) {
        *abort_flag = 1;
        atomicExch(a.status, 25);
      }
    } else {
      const float total = both(l).x + both(l).y;
      const bool dead = total == 0.f || hi <= lo;          // a row that sees nothing
      const float inv = dead ? 0.f : 1.f / total;
      const bool store = row < s.qext;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.o.data) + int64_t(s.tb) * a.o.sb + int64_t(s.q0 + row) * a.o.st + int64_t(head) * a.o.sh;
#pragma unroll
      for (int i = 0; i < BOXES * 2; ++i) {
        uint32_t o[32];
        if (any) {
          tc_ld32(to + i * 32, o);
          tc_wait_ld();
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = i * 32 + e * 8;
          uint4 w = make_uint4(0, 0, 0, 0);
          if (!dead) {
            w.x = pack_bf16(__uint_as_float(o[e * 8]) * inv, __uint_as_float(o[e * 8 + 1]) * inv);
            w.y = pack_bf16(__uint_as_float(o[e * 8 + 2]) * inv, __uint_as_float(o[e * 8 + 3]) * inv);
            w.z = pack_bf16(__uint_as_float(o[e * 8 + 4]) * inv, __uint_as_float(o[e * 8 + 5]) * inv);
            w.w = pack_bf16(__uint_as_float(o[e * 8 + 6]) * inv, __uint_as_float(o[e * 8 + 7]) * inv);
          }
          if (store && d < a.dim) *reinterpret_cast<uint4*>(out + d) = w;
        }
      }
      if (store) a.lse[(int64_t(s.tb) * a.hq + head) * a.nq + s.q0 + row] = dead ? -INFINITY : fmaf(m, a.scale, logf(total));
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == ISSUER) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
  }
}

template <int BOXES>
int run(const AttnMaps& maps, const AttnArgs& a, cudaStream_t st) {
  const int64_t blocks = attn_max_blocks(a, 2 * BLK, false) * a.hq;
  if (blocks > 0x7fffffff) return MUON_ERR_UNSUPPORTED;
  auto kernel = attention_forward_tc_kernel<BOXES>;
  static SharedMemoryLimit limit;
  if (!limit.raise(a.device, Smem<BOXES>::bytes, kernel)) return MUON_ERR_CUDA;
  kernel<<<unsigned(blocks), THREADS, Smem<BOXES>::bytes, st>>>(maps, a);
  return cudaGetLastError() == cudaSuccess ? 1 : MUON_ERR_CUDA;
}

}  // namespace

bool attention_forward_tc_takes(const AttnArgs& a) {
  return a.dim % 8 == 0 && a.dim <= 128 && a.nk > 0 && map_takes(a.q, a.batch, a.nq, a.hq) && map_takes(a.k, a.batch, a.nk, a.hkv) &&
         map_takes(a.v, a.batch, a.nk, a.hkv) && map_takes(a.o, a.batch, a.nq, a.hq);
}

int launch_attention_forward_tc(muon_ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  if (!ctx->tmap_encode) return MUON_ERR_CUDA;
  AttnMaps m;
  if (!encode_tile_map(ctx->tmap_encode, &m.q, a.q, a.dim, a.batch, a.nq, a.hq) ||
      !encode_tile_map(ctx->tmap_encode, &m.k, a.k, a.dim, a.batch, a.nk, a.hkv) ||
      !encode_tile_map(ctx->tmap_encode, &m.v, a.v, a.dim, a.batch, a.nk, a.hkv))
    return MUON_ERR_CUDA;
  m.dout = m.q;
  ctx->tmap_encodes += 3;
  return a.dim <= 64 ? run<1>(m, a, st) : run<2>(m, a, st);
}

}  // namespace muon
