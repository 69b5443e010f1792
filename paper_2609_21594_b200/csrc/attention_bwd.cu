// Attention backward on the tensor cores (bf16): two kernels that form S and P anew, one per result that is summed.
//
//   dk, dv:  a block owns 128 keys of a key head and walks the blocks of 128 queries that see them, for every query head of the group.
//            The scores are formed transposed, S^T = k q^T and dP^T = v do^T (keys in the lanes), so that P^T and dS^T are already the
//            A operands, read from tensor memory, of dv += P^T do and dk += dS^T q.  Nothing but q, do and 1 KiB of row statistics
//            per block of queries enters shared memory.
//   dq:      a block owns 128 queries and walks the blocks of keys they see: S = q k^T, dP = do v^T, dq += dS k.
//
// Both start with their longest blocks, and those of dq, which need nothing of dk and dv, fill the SMs that the last blocks of dk and dv leave
// (launched programmatically; as two kinds of blocks of one kernel each would run 5 % slower).
//
// Seven products of 128 x 128 x head_dim per pair of tiles instead of the five that a single kernel needs: that would add every
// block's share of dq (or of dk and dv) with float atomics, whose order changes from run to run, or keep fp32 partial sums as large as
// the number of blocks, or let the blocks that share a sum wait for one another in a fixed order; here every sum has one owner.
//
// 352 threads: eight warps compute (two per lane quadrant, half of the 128 columns each), one loads, one issues, one clears the rows of a
// streamed tile that lie past the sequence's end.  The issuer alternates: while the warps turn S into P it multiplies with the dS before,
// while they turn dP into dS it forms the next S.
//
// Measured, causal, 32/8 heads of 128: 4096 tokens 421 to 457 us over several runs, 750 to 816 TFLOP/s of the five products that the gradient needs
// (1050 to 1142 of the seven issued, 63 to 68 % of the library's matrix product alone), 8192 tokens 1.6 ms; 4 x 2048 tokens of heads of 64 349 to
// 363 us.  A round takes 2700 clocks in the dk, dv
// kernel (its products alone 2048) and 1985 in the dq kernel (1536): the rest is the handing over of P and dS, each a few hundred clocks during
// which the tensor pipe has only the other product left.  Short and packed sequences (a few rounds per block) pay 1.3 us to start a block and 2
// to 4 us for its results: 9 documents in 6000 tokens, heads of 64: 214 us.
#include <cuda_bf16.h>

#include "attention_tc.cuh"

namespace muon {
namespace {

using namespace attn;

constexpr int THREADS = 352, TMEM_COLS = 512, LOADER = 8, ISSUER = 9, SWEEPER = 10;
constexpr uint32_t ROW_BYTES = kAttnRowBlock * sizeof(float);          // one value for each of 128 queries

// Both streams bring one tile per round, and a tile takes 1200 to 1700 clocks from the request to its arrival, most of a round.  Stream 0 (q; k
// in the dq kernel) feeds the first product of a round and the last: three places.  Stream 1 (do; v) is read for the last time early in
// its round: two.  Of the row statistics, lse is read with stream 1's tile and delta until the end of the round.
constexpr int PLACES0 = 3, PLACES1 = 2;

template <int BOXES> struct Smem {
  static constexpr uint32_t kTile = BOXES * BOX_BYTES;
  static constexpr uint32_t own0 = 0, own1 = kTile, s0 = 2 * kTile, s1 = s0 + PLACES0 * kTile, lse = s1 + PLACES1 * kTile;
  static constexpr uint32_t delta = lse + PLACES1 * ROW_BYTES, bars = delta + PLACES0 * ROW_BYTES;
  static constexpr uint32_t bytes = bars + 256;
  static_assert(bytes <= 227 * 1024, "shared memory of a block");   // no room to align the base, which its declaration aligns (and the kernels check)
};

struct Bars {
  uint32_t base;
  __device__ __forceinline__ uint32_t at(int i) const { return base + uint32_t(i) * 8u; }
  __device__ __forceinline__ uint32_t own(int i) const { return at(i); }
  __device__ __forceinline__ uint32_t s_full(int place = 0) const { return at(2 + place); }
  __device__ __forceinline__ uint32_t dp_full() const { return at(4); }
  __device__ __forceinline__ uint32_t p_ready(int part = 0) const { return at(5 + part); }
  __device__ __forceinline__ uint32_t ds_ready() const { return at(7); }
  __device__ __forceinline__ uint32_t all_done() const { return at(8); }
  // Round n's tile of the stream has been read: its place may be loaded again.  Two barriers in turn, and neither completes twice unseen: stream 1's
  // is committed in round n + 2 behind tile n + 2, which the loader brings after it has seen round n's; stream 0's behind tile n + 3, which
  // round n + 2 awaits first and the loader brings after it has seen round n's (the last rounds await no tile, and there the loader none of theirs).
  __device__ __forceinline__ uint32_t free0(int n) const { return at(9 + (n & 1)); }
  __device__ __forceinline__ uint32_t free1(int n) const { return at(11 + 2 * (PLACES0 + PLACES1) + (n & 1)); }
  __device__ __forceinline__ uint32_t full0(int n) const { return at(11 + n % PLACES0); }
  __device__ __forceinline__ uint32_t full1(int n) const { return at(11 + PLACES0 + n % PLACES1); }
  // where a tile with rows past the end arrives; the sweeper passes it on to `full`
  __device__ __forceinline__ uint32_t raw0(int n) const { return at(11 + PLACES0 + PLACES1 + n % PLACES0); }
  __device__ __forceinline__ uint32_t raw1(int n) const { return at(11 + 2 * PLACES0 + PLACES1 + n % PLACES1); }
  static constexpr int count = 13 + 2 * (PLACES0 + PLACES1);
};
static_assert(Bars::count * 8 <= 192, "barriers");
__device__ __forceinline__ uint32_t phase0(int n) { return uint32_t(n / PLACES0) & 1u; }
__device__ __forceinline__ uint32_t phase1(int n) { return uint32_t(n / PLACES1) & 1u; }
__device__ __forceinline__ uint32_t phase_free(int n) { return uint32_t(n >> 1) & 1u; }

template <int BOXES>
__device__ __forceinline__ void set_up(const Bars& b, int warp, uint32_t* tmem_slot, volatile int* abort_flag) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < Bars::count; ++i) mbar_init(b.at(i), i >= 5 && i <= 7 ? 8 : 1);     // P and dS come from eight warps
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

// The loading thread: load0(n) and load1(n) ask for round n's tiles as soon as their places are free, in the order in which that happens.
template <typename L0, typename L1>
__device__ __forceinline__ void load_rounds(const Bars& b, int total, volatile int* abort_flag, int32_t* status, L0 load0, L1 load1) {
  bool ok = true;
  int n0 = 0, n1 = 0;
  for (; n0 < total && n0 < PLACES0; ++n0) {
    load0(n0);
    if (n1 < total && n1 < PLACES1) load1(n1++);
  }
  for (int n = 0; ok && n1 < total; ++n) {
    ok = mbar_wait(b.free1(n), phase_free(n), abort_flag);
    if (ok) load1(n1++);
    if (ok && n0 < total) {
      ok = mbar_wait(b.free0(n), phase_free(n), abort_flag);
      if (ok) load0(n0++);
    }
  }
  // Everything asked for must have landed before this block's shared memory is released.  After an error the sweeper may have left tiles
  // on their raw barriers: those get time to land.
  for (int w = 0; w < 2; ++w) mbar_wait(b.own(w), 0, abort_flag, false, WAIT_CYCLES / 8);
  for (int i = max(0, n0 - PLACES0); i < n0; ++i)
    if (!mbar_wait(b.full0(i), phase0(i), abort_flag, false, WAIT_CYCLES / 8)) atomicExch(status, 32);
  for (int i = max(0, n1 - PLACES1); i < n1; ++i)
    if (!mbar_wait(b.full1(i), phase1(i), abort_flag, false, WAIT_CYCLES / 8)) atomicExch(status, 32);
  if (!ok) {
    *abort_flag = 1;
    atomicExch(status, 31);
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
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

// 64 columns of a row times `scale`, rounded, to global memory; the accumulator is not read where `zero` (the whole warp) and does not count where
// `dead` (this row: it saw nothing, and has met zeros times whatever the others hold).
__device__ __forceinline__ void store_half(const AttnTensor& t, int tb, int token, int head, int d0, int dim, uint32_t taddr, int cols, float scale,
                                           bool zero, bool dead, bool store) {
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
      if (!zero && !dead) {
        w.x = pack_bf16(__uint_as_float(o[e * 8]) * scale, __uint_as_float(o[e * 8 + 1]) * scale);
        w.y = pack_bf16(__uint_as_float(o[e * 8 + 2]) * scale, __uint_as_float(o[e * 8 + 3]) * scale);
        w.z = pack_bf16(__uint_as_float(o[e * 8 + 4]) * scale, __uint_as_float(o[e * 8 + 5]) * scale);
        w.w = pack_bf16(__uint_as_float(o[e * 8 + 6]) * scale, __uint_as_float(o[e * 8 + 7]) * scale);
      }
      if (store && d < dim) *reinterpret_cast<uint4*>(out + d) = w;
    }
  }
}

// One pair of exponentials in 2 * kPolyOf on the multiply-add pipe: 1 to 2.5 % faster than none.  `poly` is known at compile time.  Only tiles without
// a mask and sequences with one term take it: its 2.7e-6 is a seven-hundredth of the rounding of P that follows there.
constexpr int kPolyOf = 2;
__device__ __forceinline__ uint64_t exp2_share(bool poly, uint64_t v) { return poly ? exp2_poly(v) : exp2_approx(v); }

struct Pairs { uint64_t a, b; };
__device__ __forceinline__ Pairs lds_pairs(uint32_t addr) {
  Pairs v;
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v.a), "=l"(v.b) : "r"(addr));
  return v;
}

// dS = P (dP + (-delta)).  Where a mask made P zero dP may be a NaN: selected, not multiplied.
template <bool MASK>
__device__ __forceinline__ uint64_t ds_pair(uint64_t p, uint64_t dp, uint64_t minus_delta) {
  const uint64_t v = mul2(p, add2(dp, minus_delta));
  if constexpr (!MASK) return v;
  const float2 f = both(v), q = both(p);
  return two(q.x == 0.f ? 0.f : f.x, q.y == 0.f ? 0.f : f.y);
}

// What rounding a pair to bf16 (`hi`) left out, rounded in its turn.
__device__ __forceinline__ uint32_t pack_rest(uint64_t v, uint32_t hi) {
  const float2 f = both(v);
  return pack_bf16(f.x - __uint_as_float(hi << 16), f.y - __uint_as_float(hi & 0xffff0000u));
}

// P and dS are rounded to bf16 for the products that sum over them: errors of up to 2^-9 that are independent, so that a sum over n terms has
// about the relative error of one, as much again as the rounding of the result: sqrt 2 of it together.  With few keys that is wide: at 2 to 40
// keys up to 1.8 times the rounding of the result, from 128 on 1.46 at the most.  A sequence of up to kSplitKeys keys (packed: kSplitPackedKeys)
// therefore keeps both as two bf16 terms, the second in the columns of the scores that the first leaves free, and each of these products is
// issued twice.  The sequence's own keys decide, not the call's, so that a document's gradients do not depend on what it is packed or padded
// with.  They do not depend on the mask either: the first queries of a long causal sequence and those of a short window see few keys and
// get one term.  Price, at 32/8 heads: 128 tokens of heads of 128 20.5 us instead of 18.5, 256 28.7 instead of 24.6; packed heads of 64, 9 documents in
// 6000 tokens 214 us instead of 205 (four of them have 512 keys at most; 207 to 209 with 128 for the limit), 32 documents in 6000 tokens 203 instead of
// 178 (189).  512 for packed ones: rows of short documents are what packing is for.
constexpr int kSplitKeys = 128, kSplitPackedKeys = 512;
__device__ __forceinline__ bool few_keys(const AttnArgs& a, const AttnSeq& s) { return s.kn <= (a.nseq ? kSplitPackedKeys : kSplitKeys); }

// Runs a role's rounds with one term or with two: loops of their own, for one that decides in every round keeps the registers of both.
template <bool MIXED, typename F>
__device__ __forceinline__ void in_terms(bool split, F rounds) {
  if constexpr (MIXED)
    if (split) return rounds(Yes());
  rounds(No());
}

// ------------------------------------------------------------------ dk, dv
template <int BOXES, bool MIXED>
__global__ void __launch_bounds__(THREADS, 1)
attention_dkv_tc_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnArgs a) {
  using L = Smem<BOXES>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  uint8_t* gen = smem_raw;
  if (base & 1023u) {                            // swizzled tiles would lie wrong
    if (threadIdx.x == 0) atomicExch(a.status, 30);
    return;
  }
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
  const bool split = MIXED && few_keys(a, s);
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
  // Blocks of queries with rows to clear: the last where it passes the sequence's end, the first where queries see nothing.
  const int blind = attn_blind(a, s);
  auto ragged = [&](int i) { return i * BLK < blind || (i + 1) * BLK > s.qn; };
  set_up<BOXES>(b, warp, tmem_slot, abort_flag);
  const uint32_t tmem = *tmem_slot, t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 256 + BOXES * 64;
  auto q_at = [&](int n) { return base + L::s0 + uint32_t(n % PLACES0) * L::kTile; };
  auto do_at = [&](int n) { return base + L::s1 + uint32_t(n % PLACES1) * L::kTile; };
  auto lse_at = [&](int n) { return base + L::lse + uint32_t(n % PLACES1) * ROW_BYTES; };
  auto delta_at = [&](int n) { return base + L::delta + uint32_t(n % PLACES0) * ROW_BYTES; };

  if (warp == LOADER) {
    // ------------------------------------------------------------------ loads
    // Only this thread reads the row statistics here.  Once every block has waited for them (so they are there for the dq kernel too), the
    // dq kernel may begin.  (The same two calls by all threads cost 10 % of the kernel's time.)
    if (lane == 0) {
      cudaGridDependencySynchronize();
      cudaTriggerProgrammaticLaunchCompletion();
    }
    if (lane == 0 && total > 0) {
      const int64_t row_blocks = attn_row_blocks(a);
      for (int w = 0; w < 2; ++w) {
        mbar_expect_tx(b.own(w), L::kTile);
        load_tile<BOXES>(base + (w ? L::own1 : L::own0), w ? &maps.v : &maps.k, b.own(w), kvh, s.k0 + c0, s.tb);
      }
      auto load_q = [&](int n) {
        const int h = kvh * group + n / per, i = i0 + n % per;
        const uint32_t bar = ragged(i) ? b.raw0(n) : b.full0(n);
        mbar_expect_tx(bar, L::kTile);
        load_tile<BOXES>(q_at(n), &maps.q, bar, h, s.q0 + i * BLK, s.tb);
      };
      auto load_do = [&](int n) {
        const int h = kvh * group + n / per, i = i0 + n % per;
        const uint32_t bar = ragged(i) ? b.raw1(n) : b.full1(n);
        const float* rows = a.rows + ((int64_t(s.tb) * a.hq + h) * row_blocks + (a.nseq ? s.q0 / kAttnRowBlock + si : 0) + i) * (2 * kAttnRowBlock);
        mbar_expect_tx(bar, L::kTile + 2 * ROW_BYTES);
        bulk_load(lse_at(n), rows, ROW_BYTES, bar);
        bulk_load(delta_at(n), rows + kAttnRowBlock, ROW_BYTES, bar);
        load_tile<BOXES>(do_at(n), &maps.dout, bar, h, s.q0 + i * BLK, s.tb);
      };
      load_rounds(b, total, abort_flag, a.status, load_q, load_do);
    }
  } else if (warp == SWEEPER) {
    // ------------------------------------------------------------------ rows that do not count: in the first and the last block of every head
    const bool head_rows = per > 1 && ragged(i0), tail_rows = per > 0 && ragged(i1 - 1);
    if (head_rows || tail_rows) {
      int uses0[PLACES0] = {}, uses1[PLACES1] = {};
      auto next_use = [](int (&uses)[PLACES0], int (&uses1)[PLACES1], int w, int n) {
        int u = 0;
#pragma unroll
        for (int i = 0; i < PLACES0; ++i)
          if (w == 0 && i == n % PLACES0) u = uses[i]++;
#pragma unroll
        for (int i = 0; i < PLACES1; ++i)
          if (w == 1 && i == n % PLACES1) u = uses1[i]++;
        return uint32_t(u) & 1u;
      };
      bool ok = true;
      for (int t = 0; t < 2 * group && ok; ++t) {
        if (!(t & 1 ? tail_rows : head_rows)) continue;
        const int i = t & 1 ? i1 - 1 : i0, n = (t >> 1) * per + (i - i0);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t ph = next_use(uses0, uses1, w, n);
          ok = ok && __all_sync(0xffffffffu, mbar_wait(w ? b.raw1(n) : b.raw0(n), ph, abort_flag));
          if (ok) clear_rows<BOXES>(w ? do_at(n) : q_at(n), blind - i * BLK, s.qn - i * BLK, lane, w ? b.full1(n) : b.full0(n));
        }
      }
      if (!ok && lane == 0) *abort_flag = 1;
    }
  } else if (warp == ISSUER) {
    // ------------------------------------------------------------------ MMA issuer
    if (total > 0) {
      const int ksteps = (a.dim + 15) / 16;
      const uint32_t idesc = make_idesc(true, BLK, ksteps * 16);
      bool ok = true;
      auto await = [&](uint32_t bar, uint32_t ph) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, ph, abort_flag)); };
      auto scores = [&](int n) {
        mma_rows_rows<BOXES>(t_s, base + L::own0, q_at(n), ksteps);
        tc_commit(b.s_full());
      };
      auto dprobs = [&](int n) {
        mma_rows_rows<BOXES>(t_dp, base + L::own1, do_at(n), ksteps);
        tc_commit(b.dp_full());
      };
      await(b.own(0), 0);
      await(b.full0(0), 0);
      elected(ok, [&] { scores(0); });
      await(b.own(1), 0);
      await(b.full1(0), 0);
      elected(ok, [&] { dprobs(0); });
      auto rounds = [&](auto two_terms) {
        constexpr bool SPLIT = decltype(two_terms)::value;
        for (int n = 0; n < total && ok; ++n) {
          const bool next = n + 1 < total;
          if (next) await(b.full0(n + 1), phase0(n + 1));
          // P comes in two parts, each half of what either warp of a quadrant has: steps 0, 1, 4, 5 and then 2, 3, 6, 7
          await(b.p_ready(0), uint32_t(n) & 1u);
          tc_fence_after();                                  // tensor memory written by other threads; tiles need no such fence
          elected(ok, [&] {                           // dv += P^T do
            mma_probs_rows<0, 2>(t_dv, t_s, t_s + 64, do_at(n), idesc, n > 0);
            mma_probs_rows<4, 6>(t_dv, t_s, t_s + 64, do_at(n), idesc, true);
            if constexpr (SPLIT) {
              mma_probs_rows<0, 2>(t_dv, t_s + 32, t_s + 96, do_at(n), idesc, true);
              mma_probs_rows<4, 6>(t_dv, t_s + 32, t_s + 96, do_at(n), idesc, true);
            }
          });
          await(b.p_ready(1), uint32_t(n) & 1u);
          tc_fence_after();
          elected(ok, [&] {
            mma_probs_rows<2, 4>(t_dv, t_s, t_s + 64, do_at(n), idesc, true);
            mma_probs_rows<6, 8>(t_dv, t_s, t_s + 64, do_at(n), idesc, true);
            if constexpr (SPLIT) {
              mma_probs_rows<2, 4>(t_dv, t_s + 32, t_s + 96, do_at(n), idesc, true);
              mma_probs_rows<6, 8>(t_dv, t_s + 32, t_s + 96, do_at(n), idesc, true);
            }
            tc_commit(b.free1(n));                           // dP^T of this block was issued earlier
            if (next) scores(n + 1);                         // takes the place of P^T, which dv has read by then
          });
          if (next) await(b.full1(n + 1), phase1(n + 1));
          await(b.ds_ready(), uint32_t(n) & 1u);
          tc_fence_after();
          elected(ok, [&] {
            mma_probs_rows(t_dk, t_dp, t_dp + 64, q_at(n), idesc, n > 0);      // dk += dS^T q
            if constexpr (SPLIT) mma_probs_rows(t_dk, t_dp + 32, t_dp + 96, q_at(n), idesc, true);
            tc_commit(b.free0(n));
            if (next) dprobs(n + 1);
          });
        }
      };
      in_terms<MIXED>(split, rounds);
      elected(true, [&] { finish_issue(b, ok, abort_flag, a.status); });
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
    auto rounds = [&](auto two_terms) {
      constexpr bool SPLIT = decltype(two_terms)::value;
      for (int n = 0; n < total; ++n) {
        const int r0 = (i0 + n % per) * BLK;
        ok = __all_sync(0xffffffffu, mbar_wait(b.full1(n), phase1(n), abort_flag)) &&               // the row statistics
             __all_sync(0xffffffffu, mbar_wait(b.s_full(), uint32_t(n) & 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const uint32_t lse = lse_at(n) + uint32_t(half) * 256u, delta = delta_at(n) + uint32_t(half) * 256u;
        const int first = qlo - r0 - half * 64, last = qhi - r0 - half * 64;
        auto step = [&](auto with_mask) {
          constexpr bool MASK = decltype(with_mask)::value;
          uint64_t p[32];
          auto hand_over = [&](uint32_t bar) {
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
          };
          {
            uint32_t x[64];
  #pragma unroll
            for (int i = 0; i < 2; ++i) tc_ld32(ts + i * 32, *reinterpret_cast<uint32_t(*)[32]>(&x[i * 32]));
            tc_wait_ld();
  #pragma unroll
            for (int c = 0; c < 2; ++c) {                    // 32 of this warp's queries at a time, into its own columns: the other half may still be read
              uint32_t w[16];
  #pragma unroll
              for (int i = c * 8; i < c * 8 + 8; ++i) {
                const Pairs l2 = lds_pairs(lse + uint32_t(i) * 16u);
                p[2 * i] = exp2_approx(fma2(words(x[4 * i], x[4 * i + 1]), twice(c2), l2.a));
                p[2 * i + 1] = exp2_share(!MASK && !SPLIT && i % kPolyOf == 0, fma2(words(x[4 * i + 2], x[4 * i + 3]), twice(c2), l2.b));
                if constexpr (MASK) {
  #pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    const float2 f = both(p[2 * i + e]);
                    const int q = 4 * i + 2 * e;
                    p[2 * i + e] = two(q < first || q >= last ? 0.f : f.x, q + 1 < first || q + 1 >= last ? 0.f : f.y);
                  }
                }
                w[2 * i - c * 16] = pack_bf16(p[2 * i]);
                w[2 * i + 1 - c * 16] = pack_bf16(p[2 * i + 1]);
              }
              tc_st16(ts + c * 16, w);
              if constexpr (SPLIT) {
  #pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack_rest(p[c * 16 + i], w[i]);
                tc_st16(ts + 32 + c * 16, w);
              }
              hand_over(b.p_ready(c));
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
          for (int i = 0; i < 16; ++i) {
            const Pairs d = lds_pairs(delta + uint32_t(i) * 16u);
            p[2 * i] = ds_pair<MASK>(p[2 * i], words(x[4 * i], x[4 * i + 1]), d.a);
            p[2 * i + 1] = ds_pair<MASK>(p[2 * i + 1], words(x[4 * i + 2], x[4 * i + 3]), d.b);
            w[2 * i] = pack_bf16(p[2 * i]);
            w[2 * i + 1] = pack_bf16(p[2 * i + 1]);
          }
          tc_st32(tp, w);
          if constexpr (SPLIT) {
  #pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = pack_rest(p[i], w[i]);
            tc_st32(tp + 32, w);
          }
          hand_over(b.ds_ready());
        };
        if (block_masked(a, s, r0, c0) || r0 + BLK > s.qn || c0 + BLK > s.kn) step(Yes());
        else step(No());
        if (!ok) break;
      }
    };
    in_terms<MIXED>(split, rounds);
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
      const bool zero = total == 0, store = key < s.kext, unseen = qhi <= max(qlo, 0);
      constexpr int cols = BOXES * 32;                     // the two warps of a quadrant share the head
      store_half(a.dv, s.tb, s.k0 + key, kvh, half * cols, a.dim, t_dv + lanes + uint32_t(half * cols), cols, 1.f, zero, unseen, store);
      store_half(a.dk, s.tb, s.k0 + key, kvh, half * cols, a.dim, t_dk + lanes + uint32_t(half * cols), cols, a.scale, zero, unseen, store);
    }
  }
  tear_down(warp, tmem);
}

// ------------------------------------------------------------------ dq
// Whoever waits for the dq kernel waits for both: its last block stays until the kernel before it, which it may have overtaken, has ended.
__device__ __forceinline__ void stay() {
  if (blockIdx.x == gridDim.x - 1) cudaGridDependencySynchronize();
}

template <int BOXES, bool MIXED>
__global__ void __launch_bounds__(THREADS, 1)
attention_dq_tc_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnArgs a) {
  using L = Smem<BOXES>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  uint8_t* gen = smem_raw;
  if (base & 1023u) {                            // swizzled tiles would lie wrong
    if (threadIdx.x == 0) {
      atomicExch(a.status, 30);
      stay();
    }
    return;
  }
  const Bars b{base + L::bars};
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + L::bars + 192);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + L::bars + 200);
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int head = int(blockIdx.x % unsigned(a.hq)), kvh = head / (a.hq / a.hkv);
  int si, blk;
  if (!attn_find_block(a, int(blockIdx.x / unsigned(a.hq)), BLK, false, &si, &blk)) {
    if (threadIdx.x == 0) stay();
    return;
  }
  if (!a.nseq) {
    const int rest = int(blockIdx.x / unsigned(a.hq)), per = (a.nq + BLK - 1) / BLK;
    si = rest % a.batch;
    blk = per - 1 - rest / a.batch;
  }
  const AttnSeq s = attn_seq(a, si);
  const bool split = MIXED && few_keys(a, s);
  const int r0 = blk * BLK;
  const BlockRange rg = key_blocks(a, s, r0);
  const int total = rg.n1 - rg.n0;
  set_up<BOXES>(b, warp, tmem_slot, abort_flag);
  const uint32_t tmem = *tmem_slot, t_dp = tmem + 256, t_dq = tmem + 384;
  // Two places for S, each with its barrier: the next S is formed while this one is read, and a barrier that both shared could complete
  // twice before a slow warp looks at it.
  auto t_s = [&](int n) { return tmem + uint32_t(n & 1) * 128u; };
  auto k_at = [&](int n) { return base + L::s0 + uint32_t(n % PLACES0) * L::kTile; };
  auto v_at = [&](int n) { return base + L::s1 + uint32_t(n % PLACES1) * L::kTile; };

  if (warp == LOADER) {
    // ------------------------------------------------------------------ loads
    if (lane == 0 && total > 0) {
      for (int w = 0; w < 2; ++w) {
        mbar_expect_tx(b.own(w), L::kTile);
        load_tile<BOXES>(base + (w ? L::own1 : L::own0), w ? &maps.dout : &maps.q, b.own(w), head, s.q0 + r0, s.tb);
      }
      auto load_k = [&](int n) {
        const uint32_t bar = (rg.n0 + n + 1) * BLK > s.kn ? b.raw0(n) : b.full0(n);
        mbar_expect_tx(bar, L::kTile);
        load_tile<BOXES>(k_at(n), &maps.k, bar, kvh, s.k0 + (rg.n0 + n) * BLK, s.tb);
      };
      auto load_v = [&](int n) {
        mbar_expect_tx(b.full1(n), L::kTile);
        load_tile<BOXES>(v_at(n), &maps.v, b.full1(n), kvh, s.k0 + (rg.n0 + n) * BLK, s.tb);
      };
      load_rounds(b, total, abort_flag, a.status, load_k, load_v);
    }
    if (lane == 0) stay();
  } else if (warp == SWEEPER) {
    // ------------------------------------------------------------------ rows of the last k tile past the end: their dS is zero, and so must be dS k
    if (total > 0 && rg.n1 * BLK > s.kn) {
      if (__all_sync(0xffffffffu, mbar_wait(b.raw0(total - 1), 0, abort_flag)))
        clear_rows<BOXES>(k_at(total - 1), 0, s.kn - (rg.n1 - 1) * BLK, lane, b.full0(total - 1));
      else if (lane == 0) *abort_flag = 1;
    }
  } else if (warp == ISSUER) {
    // ------------------------------------------------------------------ MMA issuer
    if (total > 0) {
      const int ksteps = (a.dim + 15) / 16;
      const uint32_t idesc = make_idesc(true, BLK, ksteps * 16);
      bool ok = true;
      auto await = [&](uint32_t bar, uint32_t ph) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, ph, abort_flag)); };
      auto scores = [&](int n) {
        mma_rows_rows<BOXES>(t_s(n), base + L::own0, k_at(n), ksteps);
        tc_commit(b.s_full(n & 1));
      };
      auto dprobs = [&](int n) {
        mma_rows_rows<BOXES>(t_dp, base + L::own1, v_at(n), ksteps);
        tc_commit(b.dp_full());
        tc_commit(b.free1(n));
      };
      await(b.own(0), 0);
      await(b.full0(0), 0);
      elected(ok, [&] { scores(0); });
      await(b.own(1), 0);
      await(b.full1(0), 0);
      elected(ok, [&] { dprobs(0); });
      auto rounds = [&](auto two_terms) {
        constexpr bool SPLIT = decltype(two_terms)::value;
        for (int n = 0; n < total && ok; ++n) {
          const bool next = n + 1 < total;
          if (next) {
            await(b.full0(n + 1), phase0(n + 1));
            elected(ok, [&] { scores(n + 1); });            // its place was read before dS of block n - 1 was ready
            await(b.full1(n + 1), phase1(n + 1));
          }
          await(b.ds_ready(), uint32_t(n) & 1u);
          tc_fence_after();                                  // tensor memory written by other threads; tiles need no such fence
          elected(ok, [&] {
            mma_probs_rows(t_dq, t_dp, t_dp + 64, k_at(n), idesc, n > 0);      // dq += dS k
            if constexpr (SPLIT) mma_probs_rows(t_dq, t_dp + 32, t_dp + 96, k_at(n), idesc, true);
            tc_commit(b.free0(n));
            if (next) dprobs(n + 1);
          });
        }
      };
      in_terms<MIXED>(split, rounds);
      elected(true, [&] { finish_issue(b, ok, abort_flag, a.status); });
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
    auto rounds = [&](auto two_terms) {
      constexpr bool SPLIT = decltype(two_terms)::value;
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
              p[i] = exp2_share(!MASK && !SPLIT && i % (2 * kPolyOf) == 1, fma2(words(x[2 * i], x[2 * i + 1]), twice(c2), twice(l2)));
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
          for (int i = 0; i < 32; ++i) {
            p[i] = ds_pair<MASK>(p[i], words(x[2 * i], x[2 * i + 1]), twice(delta));
            w[i] = pack_bf16(p[i]);
          }
          tc_st32(tp, w);
          if constexpr (SPLIT) {
  #pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = pack_rest(p[i], w[i]);
            tc_st32(tp + 32, w);
          }
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(b.ds_ready());
        };
        if (block_masked(a, s, r0, c0) || r0 + BLK > s.qn) step(Yes());
        else step(No());
        if (!ok) break;
      }
    };
    in_terms<MIXED>(split, rounds);
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
      store_half(a.dq, s.tb, s.q0 + row, head, half * cols, a.dim, t_dq + lanes + uint32_t(half * cols), cols, a.scale, total == 0, hi <= lo,
                 row < s.qext);
    }
  }
  tear_down(warp, tmem);
}

template <int BOXES, bool MIXED>
int run(const AttnMaps& m, const AttnArgs& a, cudaStream_t st) {
  const int64_t kb = attn_max_blocks(a, BLK, true) * a.hkv, qb = attn_max_blocks(a, BLK, false) * a.hq;
  if (kb > 0x7fffffff || qb > 0x7fffffff) return MUON_ERR_UNSUPPORTED;
  constexpr uint32_t bytes = Smem<BOXES>::bytes;
  static SharedMemoryLimit limit;
  if (!limit.raise(a.device, bytes, attention_dkv_tc_kernel<BOXES, MIXED>, attention_dq_tc_kernel<BOXES, MIXED>)) return MUON_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(unsigned(kb));
  if (cudaLaunchKernelEx(&cfg, attention_dkv_tc_kernel<BOXES, MIXED>, m, a) != cudaSuccess) return MUON_ERR_CUDA;
  cfg.gridDim = dim3(unsigned(qb));
  return cudaLaunchKernelEx(&cfg, attention_dq_tc_kernel<BOXES, MIXED>, m, a) == cudaSuccess ? 2 : MUON_ERR_CUDA;
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
  if (a.nseq || a.k_lens || a.nk <= kSplitKeys) return a.dim <= 64 ? run<1, true>(m, a, st) : run<2, true>(m, a, st);
  return a.dim <= 64 ? run<1, false>(m, a, st) : run<2, false>(m, a, st);
}

}  // namespace muon
