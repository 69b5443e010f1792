// Shared declarations of the layer operators (layer norm, rotary positions, attention).  Internal to the library.
#pragma once

#include <atomic>

#include "internal.h"

namespace muon {

// Raises the dynamic shared memory that kernels may use, once per device (the call costs about as much as a launch).  One object serves one
// set of kernels and one size; host threads may race to it, setting the same value twice.
class SharedMemoryLimit {
  std::atomic<uint64_t> done_{0};             // a bit per device; devices past 63 set it every time

 public:
  template <typename... K>
  bool raise(int device, uint32_t bytes, K... kernels) {
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (done_.load(std::memory_order_relaxed) & bit) return true;
    const bool ok = ((cudaFuncSetAttribute(kernels, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes)) == cudaSuccess) && ...);
    if (ok) done_.fetch_or(bit, std::memory_order_relaxed);
    return ok;
  }
};

// ------------------------------------------------------------------ layer norm
constexpr int kNormMaxCols = 16384;
constexpr int kNormMaxParts = 592;       // rows of partial sums at most: four blocks on each of 148 SMs

struct NormArgs {
  const void* x;
  const void* dy;       // backward
  void* out;            // y or dx
  int64_t ldx, lddy, ldo;
  const void* weight;   // may be null
  const void* bias;     // forward, may be null
  float* mean;          // null without centring
  float* rstd;
  void* dweight;        // backward, may be null
  void* dbias;
  float* parts;         // backward: [blocks][2][cols]
  int64_t rows;
  int32_t cols, dtype, param_dtype, center;
  float eps;
  int32_t* status;
  int32_t device;
};
int launch_norm_forward(const NormArgs& a, int sms, cudaStream_t st);
int launch_norm_backward(const NormArgs& a, int sms, cudaStream_t st);
int norm_parts(int64_t rows, int cols);     // upper bound of the rows of partial sums that a backward pass writes

// ------------------------------------------------------------------ rotary positions
constexpr int kRotaryMaxPairs = 256, kRotaryMaxItems = 4;

struct RotaryArgs {
  muon_rotary_item_t item[kRotaryMaxItems];
  int32_t head_begin[kRotaryMaxItems + 1];   // heads of all items in a row
  int32_t count, dtype, interleaved, inverse, head_dim, pairs;
  int32_t batch, tokens;
  const int32_t* positions;
  int64_t position_offset;
  float amplitude;
  double turns[kRotaryMaxPairs];             // rotations per position
};
int launch_rotary(const RotaryArgs& a, int sms, cudaStream_t st);

// ------------------------------------------------------------------ attention
struct AttnTensor {
  void* data;
  int64_t sb, st, sh;                        // elements between batch rows, tokens, heads
};

struct AttnArgs {
  AttnTensor q, k, v, o, dout, dq, dk, dv;
  float* lse;
  float* rows;            // backward scratch: see attn_row_block
  int32_t batch, nq, nk;  // tokens of a batch row (packed: of all sequences)
  int32_t hq, hkv, dim;
  int32_t causal, window;
  float scale;
  int32_t nseq;           // packed: sequences; else 0
  const int32_t* q_lens;
  const int32_t* k_lens;
  const int32_t* q_off;
  const int32_t* k_off;
  int32_t* status;
  int32_t device;
};

// One sequence as the kernels see it.  Rows [q0, q0 + qext) of batch row `tb` are its queries; the first qn count, the others
// only have their results cleared.  The same for keys.
struct AttnSeq {
  int32_t tb, q0, qn, qext, k0, kn, kext;
};

#ifdef __CUDACC__
__device__ __forceinline__ int attn_clamp(int v, int hi) { return v < 0 ? 0 : v > hi ? hi : v; }

// Sequence `s` of the call.  Packed: s = nseq stands for the tokens after the last offset, which belong to no sequence.
// Offsets are clamped to the tensor, so a bad table gives wrong results but no access outside it.
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs& a, int s) {
  AttnSeq r;
  if (a.nseq) {
    const bool rest = s >= a.nseq;
    r.tb = 0;
    r.q0 = attn_clamp(a.q_off[s], a.nq);
    r.k0 = attn_clamp(a.k_off[s], a.nk);
    const int qe = rest ? a.nq : attn_clamp(a.q_off[s + 1], a.nq), ke = rest ? a.nk : attn_clamp(a.k_off[s + 1], a.nk);
    r.qext = qe > r.q0 ? qe - r.q0 : 0;
    r.kext = ke > r.k0 ? ke - r.k0 : 0;
    r.qn = rest ? 0 : r.qext;
    r.kn = rest ? 0 : r.kext;
  } else {
    r.tb = s;
    r.q0 = r.k0 = 0;
    r.qext = a.nq;
    r.kext = a.nk;
    r.qn = a.q_lens ? attn_clamp(a.q_lens[s], a.nq) : a.nq;
    r.kn = a.k_lens ? attn_clamp(a.k_lens[s], a.nk) : a.nk;
  }
  return r;
}

// Keys [lo, hi) that query i of the sequence sees (empty when lo >= hi).
__device__ __forceinline__ int attn_key_hi(const AttnArgs& a, const AttnSeq& s, int i) {
  if (i >= s.qn) return 0;
  const int h = a.causal ? i + s.kn - s.qn + 1 : s.kn;
  return h < s.kn ? h : s.kn;
}
__device__ __forceinline__ int attn_key_lo(const AttnArgs& a, const AttnSeq& s, int i) {
  if (!a.window) return 0;
  const int64_t l = int64_t(i) + s.kn - s.qn - a.window + 1;
  return l > 0 ? int(l) : 0;
}
// Queries [lo, hi) that see some key of [c0, c1).
__device__ __forceinline__ int attn_query_lo(const AttnArgs& a, const AttnSeq& s, int c0) {
  const int l = a.causal ? c0 - (s.kn - s.qn) : 0;
  return l > 0 ? l : 0;
}
__device__ __forceinline__ int attn_query_hi(const AttnArgs& a, const AttnSeq& s, int c1) {
  if (!a.window) return s.qn;
  const int64_t h = int64_t(c1) - 1 - (s.kn - s.qn) + a.window;
  return h < 0 ? 0 : h < s.qn ? int(h) : s.qn;
}

// The first queries of a sequence, which see nothing because it has fewer keys than queries (or none).  They count, so their rows lie inside the
// tiles that others are read from; whatever they hold has to be cleared there, for a probability of zero times a NaN is a NaN.
__device__ __forceinline__ int attn_blind(const AttnArgs& a, const AttnSeq& s) {
  if (s.kn == 0) return s.qn;
  return a.causal && s.qn > s.kn ? s.qn - s.kn : 0;
}

// Finds block `t` of the list "ceil(ext / rows) blocks of each sequence" (ext: its queries, or its keys); the whole warp calls it.
// Returns false past the end of the list.  Batched: the sequences have equal extents and no search is needed.
__device__ __forceinline__ bool attn_find_block(const AttnArgs& a, int t, int rows, bool keys, int* seq, int* block) {
  if (!a.nseq) {
    const int per = ((keys ? a.nk : a.nq) + rows - 1) / rows;
    *seq = t / per;
    *block = t - *seq * per;
    return *seq < a.batch;
  }
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int s0 = 0; s0 <= a.nseq; s0 += 32) {
    int n = 0;
    if (s0 + lane <= a.nseq) {
      const AttnSeq q = attn_seq(a, s0 + lane);
      n = ((keys ? q.kext : q.qext) + rows - 1) / rows;
    }
    int sum = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += up;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, t < before + sum);
    if (hit) {
      const int l = __ffs(hit) - 1;
      *seq = s0 + l;
      *block = t - before - (__shfl_sync(0xffffffffu, sum, l) - __shfl_sync(0xffffffffu, n, l));
      return true;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  return false;
}
#endif

// Blocks of `rows` queries (or keys) over all sequences; an upper bound for packed ones, whose lengths only the device knows.
inline int64_t attn_max_blocks(const AttnArgs& a, int rows, bool keys) {
  const int64_t n = keys ? a.nk : a.nq;
  return a.nseq ? n / rows + a.nseq + 1 : int64_t(a.batch) * ((n + rows - 1) / rows);
}

// Backward scratch: for every head and every block of 128 queries of a sequence, 128 values of -lse (in units of log 2; -inf for a row
// that sees nothing) and then 128 of -delta, so that a block's 1 KiB is one aligned copy.  Packed sequence s starts at block
// q0 / 128 + s, which leaves room for the blocks before it: floor(q0 / 128) + floor(n / 128) + 1 >= floor(q0 / 128) + ceil(n / 128).
constexpr int kAttnRowBlock = 128;
__host__ __device__ inline int64_t attn_row_blocks(const AttnArgs& a) {      // per head (batched: per batch row and head)
  return a.nseq ? int64_t(a.nq) / kAttnRowBlock + a.nseq + 2 : (int64_t(a.nq) + kAttnRowBlock - 1) / kAttnRowBlock;
}

int launch_attention_forward_simt(const AttnArgs& a, int dtype, cudaStream_t st);
int launch_attention_backward_simt(const AttnArgs& a, int dtype, cudaStream_t st);
// The tensor-core kernels take bf16 heads of a multiple of 8 up to 128 elements whose tensors TMA can address.
bool attention_forward_tc_takes(const AttnArgs& a);
int launch_attention_forward_tc(muon_ctx* ctx, const AttnArgs& a, cudaStream_t st);
bool attention_backward_tc_takes(const AttnArgs& a);
int launch_attention_backward_tc(muon_ctx* ctx, const AttnArgs& a, cudaStream_t st);
int launch_attention_rows(const AttnArgs& a, int dtype, cudaStream_t st);           // fills AttnArgs::rows

}  // namespace muon
