// Attention backward on the tensor cores (bf16): two kernels that form S and P anew, one per result that is summed.
//
//   dk, dv:  a block owns 128 keys of a key head and walks the blocks of 128 queries that see them, for every query head of the group.
//            The scores are formed transposed, S^T = k q^T and dP^T = v do^T (keys in the lanes), so that P^T and dS^T are already the
//            A operands, read from tensor memory, of dv += P^T do and dk += dS^T q.  Nothing but q, do and 1 KiB of row statistics
//            per block of queries enters shared memory.
//   dq:      a block owns 128 queries and walks the blocks of keys they see: S = q k^T, dP = do v^T, dq += dS k.
//
// Seven products of 128 x 128 x head_dim per pair of blocks instead of the five that a single kernel needs: a single kernel would add every
// block's share of dq (or of dk and dv) with float atomics, whose order changes from run to run, or keep fp32 partial sums as large as
// the number of blocks; here every sum has one owner and a fixed order.
//
// 352 threads: eight warps compute (two per lane quadrant, half of the 128 columns each), one loads, one issues, one clears the rows of a
// streamed tile that lie past the sequence's end.  The issuer alternates: while the warps turn S into P it multiplies with the dS before,
// while they turn dP into dS it forms the next S.
#include <cuda_bf16.h>

#include "attention_tc.cuh"

namespace muon {
namespace {

using namespace attn;

constexpr int THREADS = 352, STAGES = 2, TMEM_COLS = 512, LOADER = 8, ISSUER = 9, SWEEPER = 10;
constexpr uint32_t ROWS_BYTES = 2 * kAttnRowBlock * sizeof(float);     // lse and delta of 128 queries

template <int BOXES> struct Smem {
  static constexpr uint32_t kTile = BOXES * BOX_BYTES;
  // two tiles that stay, two stages of the two that stream, row statistics
  static constexpr uint32_t own0 = 0, own1 = kTile, s0 = 2 * kTile, s1 = s0 + STAGES * kTile, rows = s1 + STAGES * kTile;
  static constexpr uint32_t bars = rows + STAGES * ROWS_BYTES;
  static constexpr uint32_t bytes = bars + 256 + 1024;
};

struct Bars {
  uint32_t base;
  __device__ __forceinline__ uint32_t own(int i) const { return base + uint32_t(i) * 8u; }
  __device__ __forceinline__ uint32_t s_full(int place = 0) const { return base + (place ? 120u : 16u); }
  __device__ __forceinline__ uint32_t dp_full() const { return base + 24u; }
  __device__ __forceinline__ uint32_t p_ready() const { return base + 32u; }
  __device__ __forceinline__ uint32_t ds_ready() const { return base + 40u; }
  __device__ __forceinline__ uint32_t all_done() const { return base + 48u; }
  __device__ __forceinline__ uint32_t full(int which, int st) const { return base + 56u + uint32_t(which * STAGES + st) * 8u; }
  __device__ __forceinline__ uint32_t empty(int which, int st) const { return base + 56u + uint32_t((2 + which) * STAGES + st) * 8u; }
  // where a tile with rows past the end arrives; the sweeper passes it on to `full`
  __device__ __forceinline__ uint32_t raw(int which, int st) const { return base + 128u + uint32_t(which * STAGES + st) * 8u; }
};

template <int BOXES>
__device__ __forceinline__ void set_up(const Bars& b, int warp, uint32_t* tmem_slot, volatile int* abort_flag) {
  if (threadIdx.x == 0) {
    mbar_init(b.own(0), 1);
    mbar_init(b.own(1), 1);
    mbar_init(b.s_full(0), 1);
    mbar_init(b.s_full(1), 1);
    mbar_init(b.dp_full(), 1);
    mbar_init(b.p_ready(), 8);
    mbar_init(b.ds_ready(), 8);
    mbar_init(b.all_done(), 1);
    for (int w = 0; w < 2; ++w)
      for (int i = 0; i < STAGES; ++i) {
        mbar_init(b.full(w, i), 1);
        mbar_init(b.empty(w, i), 1);
        mbar_init(b.raw(w, i), 1);
      }
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
}

__device__ __forceinline__ void tear_down(int warp, uint32_t tmem) {
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == ISSUER) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
  }
}

// Waits until everything issued is done, so that tensor memory may be freed (and, without an error, tells the computing warps).
__device__ __forceinline__ void finish_issue(const Bars& b, bool ok, volatile int* abort_flag, int32_t* status) {
  if (!ok) {
    *abort_flag = 1;
    atomicExch(status, 33);
  }
  tc_commit(b.all_done());
  if (!mbar_wait(b.all_done(), 0, abort_flag, false, WAIT_CYCLES / 8)) atomicExch(status, 34);
}

// Waits for what was asked for last of both streams, so that shared memory may be released.  After an error the sweeper may have left
// tiles on their raw barriers: those get time to land.
__device__ __forceinline__ void drain(const Bars& b, int issued, bool ok, volatile int* abort_flag, int32_t* status) {
  for (int w = 0; w < 2; ++w) {
    mbar_wait(b.own(w), 0, abort_flag, false, WAIT_CYCLES / 8);
    for (int i = max(0, issued - STAGES); i < issued; ++i)
      if (!mbar_wait(b.full(w, i % STAGES), uint32_t(i / STAGES) & 1u, abort_flag, false, WAIT_CYCLES / 8)) atomicExch(status, 32);
  }
  if (!ok) {
    *abort_flag = 1;
    atomicExch(status, 31);
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
}

// 64 columns of a row times `scale`, rounded, to global memory; the accumulator is ignored where `zero`.
__device__ __forceinline__ void store_half(const AttnTensor& t, int tb, int token, int head, int d0, int dim, uint32_t taddr, int cols, float scale,
                                           bool zero, bool store) {
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(t.data) + int64_t(tb) * t.sb + int64_t(token) * t.st + int64_t(head) * t.sh;
  for (int i = 0; i < cols / 32; ++i) {
    uint32_t o[32];
    if (!zero) {
      tc_ld32(taddr + uint32_t(i) * 32u, o);
      tc_wait_ld();
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = d0 + i * 32 + e * 8;
      uint4 w = make_uint4(0, 0, 0, 0);
      if (!zero) {
        w.x = pack_bf16(__uint_as_float(o[e * 8]) * scale, __uint_as_float(o[e * 8 + 1]) * scale);
        w.y = pack_bf16(__uint_as_float(o[e * 8 + 2]) * scale, __uint_as_float(o[e * 8 + 3]) * scale);
        w.z = pack_bf16(__uint_as_float(o[e * 8 + 4]) * scale, __uint_as_float(o[e * 8 + 5]) * scale);
        w.w = pack_bf16(__uint_as_float(o[e * 8 + 6]) * scale, __uint_as_float(o[e * 8 + 7]) * scale);
      }
      if (store && d < dim) *reinterpret_cast<uint4*>(out + d) = w;
    }
  }
}

struct Pairs { uint64_t a, b; };
__device__ __forceinline__ Pairs lds_pairs(uint32_t addr) {
  Pairs v;
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v.a), "=l"(v.b) : "r"(addr));
  return v;
}

// dS = P (dP + (-delta)), rounded.  Where a mask made P zero dP may be a NaN: selected, not multiplied.
template <bool MASK>
__device__ __forceinline__ uint32_t ds_pair(uint64_t p, uint64_t dp, uint64_t minus_delta) {
  const uint64_t v = mul2(p, add2(dp, minus_delta));
  if constexpr (!MASK) return pack_bf16(v);
  const float2 f = both(v), q = both(p);
  return pack_bf16(q.x == 0.f ? 0.f : f.x, q.y == 0.f ? 0.f : f.y);
}

// ------------------------------------------------------------------ dk, dv
template <int BOXES>
__global__ void __launch_bounds__(THREADS, 1)
attention_dkv_tc_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnArgs a) {
  using L = Smem<BOXES>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const Bars b{base + L::bars};
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + L::bars + 192);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + L::bars + 200);
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int kvh = int(blockIdx.x % unsigned(a.hkv)), group = a.hq / a.hkv;
  int si, blk;
  if (!attn_find_block(a, int(blockIdx.x / unsigned(a.hkv)), BLK, true, &si, &blk)) return;
  if (!a.nseq) {                                 // the first keys are seen by most queries: they go first
    const int rest = int(blockIdx.x / unsigned(a.hkv));
    si = rest % a.batch;
    blk = rest / a.batch;
  }
  const AttnSeq s = attn_seq(a, si);
  const int c0 = blk * BLK;
  int i0 = 0, i1 = 0;                            // blocks of queries
  if (c0 < s.kn) {
    const int lo = attn_query_lo(a, s, c0), hi = attn_query_hi(a, s, min(c0 + BLK, s.kn));
    if (hi > lo) {
      i0 = lo / BLK;
      i1 = (hi + BLK - 1) / BLK;
    }
  }
  const int per = i1 - i0, total = per * group;
  set_up<BOXES>(b, warp, tmem_slot, abort_flag);
  const uint32_t tmem = *tmem_slot, t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 256 + BOXES * 64;
  auto phase = [](int n) { return uint32_t(n / STAGES) & 1u; };

  if (warp == LOADER) {
    // ------------------------------------------------------------------ loads: stream 0 is q with its row statistics, stream 1 is do
    if (lane == 0 && total > 0) {
      const int64_t row_blocks = attn_row_blocks(a);
      for (int w = 0; w < 2; ++w) {
        mbar_expect_tx(b.own(w), L::kTile);
        load_tile<BOXES>(base + (w ? L::own1 : L::own0), w ? &maps.v : &maps.k, b.own(w), kvh, s.k0 + c0, s.tb);
      }
      bool ok = true;
      int n = 0;
      for (; n < total && ok; ++n) {
        const int h = kvh * group + n / per, i = i0 + n % per, st = n % STAGES;
        if (!(ok = mbar_wait(b.empty(0, st), phase(n) ^ 1u, abort_flag))) break;
        const bool ragged = (i + 1) * BLK > s.qn;
        const uint32_t bar0 = ragged ? b.raw(0, st) : b.full(0, st), bar1 = ragged ? b.raw(1, st) : b.full(1, st);
        mbar_expect_tx(bar0, L::kTile + ROWS_BYTES);
        load_tile<BOXES>(base + L::s0 + uint32_t(st) * L::kTile, &maps.q, bar0, h, s.q0 + i * BLK, s.tb);
        bulk_load(base + L::rows + uint32_t(st) * ROWS_BYTES,
                  a.rows + ((int64_t(s.tb) * a.hq + h) * row_blocks + (a.nseq ? s.q0 / kAttnRowBlock + si : 0) + i) * (2 * kAttnRowBlock), ROWS_BYTES, bar0);
        ok = mbar_wait(b.empty(1, st), phase(n) ^ 1u, abort_flag);
        mbar_expect_tx(bar1, L::kTile);                    // armed even when giving up, so that the drain is one rule
        load_tile<BOXES>(base + L::s1 + uint32_t(st) * L::kTile, &maps.dout, bar1, h, s.q0 + i * BLK, s.tb);
      }
      drain(b, n, ok, abort_flag, a.status);
    }
  } else if (warp == SWEEPER) {
    // ------------------------------------------------------------------ rows past the end: the last block of every head
    if (total > 0 && i1 * BLK > s.qn) {
      int uses[STAGES] = {};
      for (int h = 0; h < group; ++h) {
        const int st = (h * per + per - 1) % STAGES;
        const uint32_t ph = uint32_t(st ? uses[1]++ : uses[0]++) & 1u;
        bool ok = true;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          ok = ok && __all_sync(0xffffffffu, mbar_wait(b.raw(w, st), ph, abort_flag));
          if (ok) clear_rows<BOXES>(base + (w ? L::s1 : L::s0) + uint32_t(st) * L::kTile, s.qn - (i1 - 1) * BLK, lane, b.full(w, st));
        }
        if (!ok) {
          if (lane == 0) *abort_flag = 1;
          break;
        }
      }
    }
  } else if (warp == ISSUER) {
    // ------------------------------------------------------------------ MMA issuer
    if (total > 0) {
      const int ksteps = (a.dim + 15) / 16;
      const uint32_t idesc = make_idesc(true, BLK, ksteps * 16);
      bool ok = true;
      auto await = [&](uint32_t bar, uint32_t ph) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, ph, abort_flag)); };
      auto q_at = [&](int n) { return base + L::s0 + uint32_t(n % STAGES) * L::kTile; };
      auto do_at = [&](int n) { return base + L::s1 + uint32_t(n % STAGES) * L::kTile; };
      auto scores = [&](int n) {
        mma_rows_rows<BOXES>(t_s, base + L::own0, q_at(n), ksteps);
        tc_commit(b.s_full());
      };
      auto dprobs = [&](int n) {
        mma_rows_rows<BOXES>(t_dp, base + L::own1, do_at(n), ksteps);
        tc_commit(b.dp_full());
      };
      await(b.own(0), 0);
      await(b.full(0, 0), 0);
      if (ok && elect_one()) scores(0);
      await(b.own(1), 0);
      await(b.full(1, 0), 0);
      if (ok && elect_one()) dprobs(0);
      for (int n = 0; n < total && ok; ++n) {
        const bool next = n + 1 < total;
        if (next) await(b.full(0, (n + 1) % STAGES), phase(n + 1));
        await(b.p_ready(), uint32_t(n) & 1u);
        tc_fence_after();                                  // tensor memory written by other threads; tiles need no such fence
        if (ok && elect_one()) {
          mma_probs_rows(t_dv, t_s, t_s + 64, do_at(n), idesc, n > 0);       // dv += P^T do
          if (next) scores(n + 1);                         // takes the place of P^T, which dv has read by then
          tc_commit(b.empty(1, n % STAGES));               // dP^T of this block was issued earlier
        }
        if (next) await(b.full(1, (n + 1) % STAGES), phase(n + 1));
        await(b.ds_ready(), uint32_t(n) & 1u);
        tc_fence_after();
        if (ok && elect_one()) {
          mma_probs_rows(t_dk, t_dp, t_dp + 64, q_at(n), idesc, n > 0);      // dk += dS^T q
          if (next) dprobs(n + 1);
          tc_commit(b.empty(0, n % STAGES));
        }
      }
      if (elect_one()) finish_issue(b, ok, abort_flag, a.status);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ P^T and dS^T: lane = key, this warp's 64 of the 128 queries
    const int quad = warp & 3, half = warp >> 2;
    const int key = c0 + quad * 32 + lane;
    const uint32_t lanes = uint32_t(quad * 32) << 16;
    const uint32_t ts = t_s + lanes + uint32_t(half) * 64u, tp = t_dp + lanes + uint32_t(half) * 64u;
    const float c2 = a.scale * kLog2e;
    const int off = s.kn - s.qn;                           // key j is seen by queries j - off .. (causal), up to j - off + window - 1
    const int qlo = key < s.kn ? (a.causal ? key - off : 0) : 0x7fffffff;
    const int qhi = key < s.kn ? attn_query_hi(a, s, key + 1) : 0;
    bool ok = true;
    for (int n = 0; n < total; ++n) {
      const int r0 = (i0 + n % per) * BLK;
      ok = __all_sync(0xffffffffu, mbar_wait(b.full(0, n % STAGES), phase(n), abort_flag)) &&     // the row statistics
           __all_sync(0xffffffffu, mbar_wait(b.s_full(), uint32_t(n) & 1u, abort_flag));
      if (!ok) break;
      tc_fence_after();
      const uint32_t rows = base + L::rows + uint32_t(n % STAGES) * ROWS_BYTES + uint32_t(half) * 256u;
      const int first = qlo - r0 - half * 64, last = qhi - r0 - half * 64;
      auto step = [&](auto with_mask) {
        constexpr bool MASK = decltype(with_mask)::value;
        uint64_t p[32];
        {
          uint32_t x[64], w[32];
#pragma unroll
          for (int i = 0; i < 2; ++i) tc_ld32(ts + i * 32, *reinterpret_cast<uint32_t(*)[32]>(&x[i * 32]));
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const Pairs l2 = lds_pairs(rows + uint32_t(i) * 16u);
            p[2 * i] = exp2_approx(fma2(words(x[4 * i], x[4 * i + 1]), twice(c2), l2.a));
            p[2 * i + 1] = exp2_approx(fma2(words(x[4 * i + 2], x[4 * i + 3]), twice(c2), l2.b));
            if constexpr (MASK) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float2 f = both(p[2 * i + e]);
                const int q = 4 * i + 2 * e;
                p[2 * i + e] = two(q < first || q >= last ? 0.f : f.x, q + 1 < first || q + 1 >= last ? 0.f : f.y);
              }
            }
            w[2 * i] = pack_bf16(p[2 * i]);
            w[2 * i + 1] = pack_bf16(p[2 * i + 1]);
          }
          tc_st32(ts, w);                                  // into this warp's own columns: the other half may still be read
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b.p_ready());

        ok = __all_sync(0xffffffffu, mbar_wait(b.dp_full(), uint32_t(n) & 1u, abort_flag));
        if (!ok) return;
        tc_fence_after();
        uint32_t x[64], w[32];
#pragma unroll
        for (int i = 0; i < 2; ++i) tc_ld32(tp + i * 32, *reinterpret_cast<uint32_t(*)[32]>(&x[i * 32]));
        tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const Pairs d = lds_pairs(rows + kAttnRowBlock * 4u + uint32_t(i) * 16u);
          w[2 * i] = ds_pair<MASK>(p[2 * i], words(x[4 * i], x[4 * i + 1]), d.a);
          w[2 * i + 1] = ds_pair<MASK>(p[2 * i + 1], words(x[4 * i + 2], x[4 * i + 3]), d.b);
        }
        tc_st32(tp, w);
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b.ds_ready());
      };
      if (block_masked(a, s, r0, c0) || r0 + BLK > s.qn || c0 + BLK > s.kn) step(Yes());
      else step(No());
      if (!ok) break;
    }
    if (ok && total > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait(b.all_done(), 0, abort_flag));
      tc_fence_after();
    }
    if (!ok) {
      if (lane == 0) {
        *abort_flag = 1;
        atomicExch(a.status, 35);
      }
    } else {
      const bool zero = total == 0, store = key < s.kext;
      constexpr int cols = BOXES * 32;                     // the two warps of a quadrant share the head
      store_half(a.dv, s.tb, s.k0 + key, kvh, half * cols, a.dim, t_dv + lanes + uint32_t(half * cols), cols, 1.f, zero, store);
      store_half(a.dk, s.tb, s.k0 + key, kvh, half * cols, a.dim, t_dk + lanes + uint32_t(half * cols), cols, a.scale, zero, store);
    }
  }
  tear_down(warp, tmem);
}

// ------------------------------------------------------------------ dq
template <int BOXES>
__global__ void __launch_bounds__(THREADS, 1)
attention_dq_tc_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnArgs a) {
  using L = Smem<BOXES>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const Bars b{base + L::bars};
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + L::bars + 192);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + L::bars + 200);
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int head = int(blockIdx.x % unsigned(a.hq)), kvh = head / (a.hq / a.hkv);
  int si, blk;
  if (!attn_find_block(a, int(blockIdx.x / unsigned(a.hq)), BLK, false, &si, &blk)) return;
  if (!a.nseq) {
    const int rest = int(blockIdx.x / unsigned(a.hq)), per = (a.nq + BLK - 1) / BLK;
    si = rest % a.batch;
    blk = per - 1 - rest / a.batch;
  }
  const AttnSeq s = attn_seq(a, si);
  const int r0 = blk * BLK;
  const BlockRange rg = key_blocks(a, s, r0);
  const int total = rg.n1 - rg.n0;
  set_up<BOXES>(b, warp, tmem_slot, abort_flag);
  const uint32_t tmem = *tmem_slot, t_dp = tmem + 256, t_dq = tmem + 384;
  // Two places for S, each with its barrier: the next S is formed while this one is read, and a barrier that both shared could complete
  // twice before a slow warp looks at it.
  auto t_s = [&](int n) { return tmem + uint32_t(n & 1) * 128u; };
  auto phase = [](int n) { return uint32_t(n / STAGES) & 1u; };

  if (warp == LOADER) {
    // ------------------------------------------------------------------ loads: stream 0 is k, stream 1 is v
    if (lane == 0 && total > 0) {
      for (int w = 0; w < 2; ++w) {
        mbar_expect_tx(b.own(w), L::kTile);
        load_tile<BOXES>(base + (w ? L::own1 : L::own0), w ? &maps.dout : &maps.q, b.own(w), head, s.q0 + r0, s.tb);
      }
      bool ok = true;
      int n = 0;
      for (; n < total && ok; ++n) {
        const int st = n % STAGES, token = s.k0 + (rg.n0 + n) * BLK;
        if (!(ok = mbar_wait(b.empty(0, st), phase(n) ^ 1u, abort_flag))) break;
        const uint32_t bar0 = (rg.n0 + n + 1) * BLK > s.kn ? b.raw(0, st) : b.full(0, st);
        mbar_expect_tx(bar0, L::kTile);
        load_tile<BOXES>(base + L::s0 + uint32_t(st) * L::kTile, &maps.k, bar0, kvh, token, s.tb);
        ok = mbar_wait(b.empty(1, st), phase(n) ^ 1u, abort_flag);
        mbar_expect_tx(b.full(1, st), L::kTile);
        load_tile<BOXES>(base + L::s1 + uint32_t(st) * L::kTile, &maps.v, b.full(1, st), kvh, token, s.tb);
      }
      drain(b, n, ok, abort_flag, a.status);
    }
  } else if (warp == SWEEPER) {
    // ------------------------------------------------------------------ rows of the last k tile past the end: their dS is zero, and so must be dS k
    if (total > 0 && rg.n1 * BLK > s.kn) {
      const int st = (total - 1) % STAGES;
      if (__all_sync(0xffffffffu, mbar_wait(b.raw(0, st), 0, abort_flag)))
        clear_rows<BOXES>(base + L::s0 + uint32_t(st) * L::kTile, s.kn - (rg.n1 - 1) * BLK, lane, b.full(0, st));
      else if (lane == 0) *abort_flag = 1;
    }
  } else if (warp == ISSUER) {
    // ------------------------------------------------------------------ MMA issuer
    if (total > 0) {
      const int ksteps = (a.dim + 15) / 16;
      const uint32_t idesc = make_idesc(true, BLK, ksteps * 16);
      bool ok = true;
      auto await = [&](uint32_t bar, uint32_t ph) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, ph, abort_flag)); };
      auto k_at = [&](int n) { return base + L::s0 + uint32_t(n % STAGES) * L::kTile; };
      auto v_at = [&](int n) { return base + L::s1 + uint32_t(n % STAGES) * L::kTile; };
      auto scores = [&](int n) {
        mma_rows_rows<BOXES>(t_s(n), base + L::own0, k_at(n), ksteps);
        tc_commit(b.s_full(n & 1));
      };
      auto dprobs = [&](int n) {
        mma_rows_rows<BOXES>(t_dp, base + L::own1, v_at(n), ksteps);
        tc_commit(b.dp_full());
        tc_commit(b.empty(1, n % STAGES));
      };
      await(b.own(0), 0);
      await(b.full(0, 0), 0);
      if (ok && elect_one()) scores(0);
      await(b.own(1), 0);
      await(b.full(1, 0), 0);
      if (ok && elect_one()) dprobs(0);
      for (int n = 0; n < total && ok; ++n) {
        const bool next = n + 1 < total;
        if (next) {
          await(b.full(0, (n + 1) % STAGES), phase(n + 1));
          if (ok && elect_one()) scores(n + 1);            // its place was read before dS of block n - 1 was ready
          await(b.full(1, (n + 1) % STAGES), phase(n + 1));
        }
        await(b.ds_ready(), uint32_t(n) & 1u);
        tc_fence_after();                                  // tensor memory written by other threads; tiles need no such fence
        if (ok && elect_one()) {
          mma_probs_rows(t_dq, t_dp, t_dp + 64, k_at(n), idesc, n > 0);      // dq += dS k
          if (next) dprobs(n + 1);
          tc_commit(b.empty(0, n % STAGES));
        }
      }
      if (elect_one()) finish_issue(b, ok, abort_flag, a.status);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ dS: lane = query, this warp's 64 of the 128 keys
    const int quad = warp & 3, half = warp >> 2;
    const int row = r0 + quad * 32 + lane;
    const uint32_t lanes = uint32_t(quad * 32) << 16;
    const uint32_t tp = t_dp + lanes + uint32_t(half) * 64u;
    const float c2 = a.scale * kLog2e;
    const int lo = attn_key_lo(a, s, row), hi = attn_key_hi(a, s, row);
    const float* info = a.rows + ((int64_t(s.tb) * a.hq + head) * attn_row_blocks(a) + (a.nseq ? s.q0 / kAttnRowBlock + si : 0) + blk) * (2 * kAttnRowBlock) +
                        quad * 32 + lane;
    const float l2 = info[0], delta = info[kAttnRowBlock];
    bool ok = true;
    for (int n = 0; n < total; ++n) {
      const int c0 = (rg.n0 + n) * BLK;
      ok = __all_sync(0xffffffffu, mbar_wait(b.s_full(n & 1), uint32_t(n >> 1) & 1u, abort_flag));
      if (!ok) break;
      tc_fence_after();
      const int first = lo - c0 - half * 64, last = hi - c0 - half * 64;
      auto step = [&](auto with_mask) {
        constexpr bool MASK = decltype(with_mask)::value;
        uint64_t p[32];
        {
          uint32_t x[64];
#pragma unroll
          for (int i = 0; i < 2; ++i) tc_ld32(t_s(n) + lanes + uint32_t(half) * 64u + i * 32, *reinterpret_cast<uint32_t(*)[32]>(&x[i * 32]));
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            p[i] = exp2_approx(fma2(words(x[2 * i], x[2 * i + 1]), twice(c2), twice(l2)));
            if constexpr (MASK) {
              const float2 f = both(p[i]);
              p[i] = two(2 * i < first || 2 * i >= last ? 0.f : f.x, 2 * i + 1 < first || 2 * i + 1 >= last ? 0.f : f.y);
            }
          }
        }
        ok = __all_sync(0xffffffffu, mbar_wait(b.dp_full(), uint32_t(n) & 1u, abort_flag));
        if (!ok) return;
        tc_fence_after();
        uint32_t x[64], w[32];
#pragma unroll
        for (int i = 0; i < 2; ++i) tc_ld32(tp + i * 32, *reinterpret_cast<uint32_t(*)[32]>(&x[i * 32]));
        tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = ds_pair<MASK>(p[i], words(x[2 * i], x[2 * i + 1]), twice(delta));
        tc_st32(tp, w);
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b.ds_ready());
      };
      if (block_masked(a, s, r0, c0) || r0 + BLK > s.qn) step(Yes());
      else step(No());
      if (!ok) break;
    }
    if (ok && total > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait(b.all_done(), 0, abort_flag));
      tc_fence_after();
    }
    if (!ok) {
      if (lane == 0) {
        *abort_flag = 1;
        atomicExch(a.status, 35);
      }
    } else {
      constexpr int cols = BOXES * 32;
      store_half(a.dq, s.tb, s.q0 + row, head, half * cols, a.dim, t_dq + lanes + uint32_t(half * cols), cols, a.scale, total == 0,
                 row < s.qext);
    }
  }
  tear_down(warp, tmem);
}

template <int BOXES>
int run(const AttnMaps& m, const AttnArgs& a, cudaStream_t st) {
  const int64_t kb = attn_max_blocks(a, BLK, true) * a.hkv, qb = attn_max_blocks(a, BLK, false) * a.hq;
  if (kb > 0x7fffffff || qb > 0x7fffffff) return MUON_ERR_UNSUPPORTED;
  constexpr uint32_t bytes = Smem<BOXES>::bytes;
  static SharedMemoryLimit limit;
  if (!limit.raise(a.device, bytes, attention_dkv_tc_kernel<BOXES>, attention_dq_tc_kernel<BOXES>)) return MUON_ERR_CUDA;
  attention_dkv_tc_kernel<BOXES><<<unsigned(kb), THREADS, bytes, st>>>(m, a);
  attention_dq_tc_kernel<BOXES><<<unsigned(qb), THREADS, bytes, st>>>(m, a);
  return cudaGetLastError() == cudaSuccess ? 2 : MUON_ERR_CUDA;
}

}  // namespace

bool attention_backward_tc_takes(const AttnArgs& a) {
  return a.dim % 8 == 0 && a.dim <= 128 && a.nk > 0 && a.nq > 0 && map_takes(a.q, a.batch, a.nq, a.hq) && map_takes(a.dout, a.batch, a.nq, a.hq) &&
         map_takes(a.k, a.batch, a.nk, a.hkv) && map_takes(a.v, a.batch, a.nk, a.hkv) && map_takes(a.dq, a.batch, a.nq, a.hq) &&
         map_takes(a.dk, a.batch, a.nk, a.hkv) && map_takes(a.dv, a.batch, a.nk, a.hkv);
}

int launch_attention_backward_tc(muon_ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  if (!ctx->tmap_encode) return MUON_ERR_CUDA;
  AttnMaps m;
  if (!encode_tile_map(ctx->tmap_encode, &m.q, a.q, a.dim, a.batch, a.nq, a.hq) ||
      !encode_tile_map(ctx->tmap_encode, &m.k, a.k, a.dim, a.batch, a.nk, a.hkv) ||
      !encode_tile_map(ctx->tmap_encode, &m.v, a.v, a.dim, a.batch, a.nk, a.hkv) ||
      !encode_tile_map(ctx->tmap_encode, &m.dout, a.dout, a.dim, a.batch, a.nq, a.hq))
    return MUON_ERR_CUDA;
  ctx->tmap_encodes += 4;
  return a.dim <= 64 ? run<1>(m, a, st) : run<2>(m, a, st);
}

}  // namespace muon
