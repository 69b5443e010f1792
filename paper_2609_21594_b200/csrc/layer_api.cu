// extern "C" entry points of the layer operators: argument validation and the choice of kernels.
#include <cmath>
#include <initializer_list>

#include "boxes.h"
#include "layer_ops.h"

using namespace muon;

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;

bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool known_dtype(int32_t d) { return d == MUON_DTYPE_BF16 || d == MUON_DTYPE_FP32; }

size_t bytes_of(int32_t d) { return d == MUON_DTYPE_BF16 ? 2 : 4; }

// The context's device must be current; its SM count comes with the answer.
int device_of(const muon_ctx* ctx, int* sms) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev != ctx->device) return MUON_ERR_CUDA;
  return cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess ? MUON_OK : MUON_ERR_CUDA;
}

int launched(muon_ctx* ctx, int n) {
  if (n < 0) {
    (void)cudaGetLastError();      // a refused launch is this call's error, not the next one's
    return n;
  }
  ctx->launches += n;
  return MUON_OK;
}

int check_norm(const muon_norm_desc_t* d) {
  if (!d || !known_dtype(d->dtype) || !known_dtype(d->param_dtype) || (d->center != 0 && d->center != 1) || d->reserved != 0) return MUON_ERR_INVALID_ARG;
  if (d->rows < 0 || d->cols < 1 || !(d->eps >= 0.f) || !std::isfinite(d->eps)) return MUON_ERR_INVALID_ARG;
  return d->cols > kNormMaxCols ? MUON_ERR_UNSUPPORTED : MUON_OK;
}

NormArgs norm_args(const muon_norm_desc_t* d) {
  NormArgs a = {};
  a.rows = d->rows;
  a.cols = d->cols;
  a.dtype = d->dtype;
  a.param_dtype = d->param_dtype;
  a.center = d->center;
  a.eps = d->eps;
  return a;
}

// A tensor that has elements needs a pointer aligned to its type and strides that are not negative.
bool good_heads(const muon_heads_t* t, size_t elem) {
  return t && t->data && aligned_to(t->data, elem) && t->batch_stride >= 0 && t->token_stride >= 0 && t->head_stride >= 0;
}

// A result has a stride in every dimension longer than one; box_meets_itself looks at whether its elements share a place.
bool good_output(const muon_heads_t* t, size_t elem, int64_t batch, int64_t tokens, int64_t heads) {
  return good_heads(t, elem) && (batch <= 1 || t->batch_stride > 0) && (tokens <= 1 || t->token_stride > 0) && (heads <= 1 || t->head_stride > 0);
}

Box box_of(const muon_heads_t* t, size_t elem, int64_t batch, int64_t tokens, int64_t heads, int64_t dim) {
  const int64_t e = int64_t(elem);
  return Box(t->data, batch, tokens, heads, dim * e, t->batch_stride * e, t->token_stride * e, t->head_stride * e);
}
Box rows_of(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t elem) {
  const int64_t e = int64_t(elem);
  return Box(p, 1, 1, rows, cols * e, 0, 0, ld * e);
}

// Whether a result lies over an input or over another result.  The first result may be one of `in_place` exactly.
bool results_clash(std::initializer_list<Box> results, std::initializer_list<Box> inputs, std::initializer_list<Box> in_place = {}) {
  for (const Box* r = results.begin(); r != results.end(); ++r) {
    for (const Box& in : inputs)
      if (boxes_meet(*r, in)) return true;
    for (const Box& in : in_place)
      if (!(r == results.begin() && same_box(*r, in)) && boxes_meet(*r, in)) return true;
    for (const Box* other = results.begin(); other != r; ++other)
      if (boxes_meet(*r, *other)) return true;
  }
  return false;
}

int check_attention(const muon_attention_desc_t* d) {
  if (!d || !known_dtype(d->dtype) || d->reserved != 0) return MUON_ERR_INVALID_ARG;
  if (d->batch < 0 || d->q_tokens < 0 || d->k_tokens < 0 || d->q_heads < 1 || d->kv_heads < 1 || d->head_dim < 1) return MUON_ERR_INVALID_ARG;
  if (d->q_heads % d->kv_heads != 0 || (d->causal != 0 && d->causal != 1) || d->window < 0 || (d->window > 0 && !d->causal)) return MUON_ERR_INVALID_ARG;
  if (!(d->scale > 0.f) || !std::isfinite(d->scale) || d->num_seqs < 0) return MUON_ERR_INVALID_ARG;
  if ((d->q_offsets != nullptr) != (d->num_seqs > 0) || (d->k_offsets != nullptr) != (d->num_seqs > 0)) return MUON_ERR_INVALID_ARG;
  if (d->num_seqs > 0 && (d->batch != 1 || d->q_lens || d->k_lens)) return MUON_ERR_INVALID_ARG;
  for (const int32_t* p : {d->q_lens, d->k_lens, d->q_offsets, d->k_offsets})
    if (!aligned_to(p, 4)) return MUON_ERR_INVALID_ARG;
  if (d->head_dim > 256 || d->q_heads > 65535) return MUON_ERR_UNSUPPORTED;
  if (int64_t(d->batch) * (int64_t(d->q_tokens) + d->k_tokens) > (int64_t(1) << 30)) return MUON_ERR_UNSUPPORTED;
  return MUON_OK;
}

AttnTensor attn_tensor(const muon_heads_t* t) { return {t->data, t->batch_stride, t->token_stride, t->head_stride}; }

AttnArgs attention_args(const muon_ctx* ctx, const muon_attention_desc_t* d) {
  AttnArgs a = {};
  a.batch = d->batch;
  a.nq = d->q_tokens;
  a.nk = d->k_tokens;
  a.hq = d->q_heads;
  a.hkv = d->kv_heads;
  a.dim = d->head_dim;
  a.causal = d->causal;
  a.window = d->window;
  a.scale = d->scale;
  a.nseq = d->num_seqs;
  a.q_lens = d->q_lens;
  a.k_lens = d->k_lens;
  a.q_off = d->q_offsets;
  a.k_off = d->k_offsets;
  a.status = ctx ? ctx->d_status : nullptr;
  a.device = ctx ? ctx->device : -1;
  return a;
}

size_t attention_scratch(const AttnArgs& a) {
  return size_t(a.batch) * size_t(a.hq) * size_t(attn_row_blocks(a)) * (2 * kAttnRowBlock) * sizeof(float);
}

}  // namespace

extern "C" {

int muon_layer_norm_forward(muon_ctx_t* ctx, const muon_norm_desc_t* desc, const void* x, int64_t ldx, const void* weight,
                            const void* bias, void* y, int64_t ldy, float* mean, float* rstd, void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_norm(desc);
  if (rc != MUON_OK) return rc;
  if (desc->rows == 0) return MUON_OK;
  const size_t e = bytes_of(desc->dtype), pe = bytes_of(desc->param_dtype);
  if (!x || !y || !rstd || (mean != nullptr) != (desc->center == 1) || ldx < desc->cols || ldy < desc->cols) return MUON_ERR_INVALID_ARG;
  if (!aligned_to(x, e) || !aligned_to(y, e) || !aligned_to(weight, pe) || !aligned_to(bias, pe) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
    return MUON_ERR_INVALID_ARG;
  if (y == x && ldy != ldx) return MUON_ERR_INVALID_ARG;
  const int64_t rows = desc->rows, cols = desc->cols, params = cols * int64_t(pe);
  if (results_clash({rows_of(y, rows, cols, ldy, e), run_of(mean, rows * 4), run_of(rstd, rows * 4)}, {run_of(weight, params), run_of(bias, params)},
                    {rows_of(x, rows, cols, ldx, e)}))
    return MUON_ERR_INVALID_ARG;
  int sms = 0;
  if ((rc = device_of(ctx, &sms)) != MUON_OK) return rc;
  NormArgs a = norm_args(desc);
  a.device = ctx->device;
  a.status = ctx->d_status;
  a.x = x;
  a.ldx = ldx;
  a.weight = weight;
  a.bias = bias;
  a.out = y;
  a.ldo = ldy;
  a.mean = mean;
  a.rstd = rstd;
  return launched(ctx, launch_norm_forward(a, sms, static_cast<cudaStream_t>(stream)));
}

int muon_layer_norm_workspace_bytes(const muon_norm_desc_t* desc, size_t* bytes) {
  if (!bytes) return MUON_ERR_INVALID_ARG;
  const int rc = check_norm(desc);
  if (rc != MUON_OK) return rc;
  *bytes = size_t(norm_parts(desc->rows, desc->cols)) * 2 * size_t(desc->cols) * sizeof(float);
  return MUON_OK;
}

int muon_layer_norm_backward(muon_ctx_t* ctx, const muon_norm_desc_t* desc, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                             const void* weight, const float* mean, const float* rstd, void* dx, int64_t lddx, void* dweight,
                             void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_norm(desc);
  if (rc != MUON_OK) return rc;
  const size_t e = bytes_of(desc->dtype), pe = bytes_of(desc->param_dtype);
  if (!aligned_to(weight, pe) || !aligned_to(dweight, pe) || !aligned_to(dbias, pe) || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return MUON_ERR_INVALID_ARG;
  if (desc->rows > 0) {
    if (!x || !dy || !dx || !rstd || (mean != nullptr) != (desc->center == 1)) return MUON_ERR_INVALID_ARG;
    if (ldx < desc->cols || lddy < desc->cols || lddx < desc->cols || !aligned_to(x, e) || !aligned_to(dy, e) || !aligned_to(dx, e)) return MUON_ERR_INVALID_ARG;
    if ((dx == x && lddx != ldx) || (dx == dy && lddx != lddy)) return MUON_ERR_INVALID_ARG;
  }
  const bool sums = dweight || dbias;
  if (desc->rows == 0 && !sums) return MUON_OK;
  size_t need = 0;
  muon_layer_norm_workspace_bytes(desc, &need);
  if (sums && need > 0) {
    if (!workspace || workspace_bytes < need) return MUON_ERR_WORKSPACE_TOO_SMALL;
    if (!aligned_to(workspace, 256)) return MUON_ERR_INVALID_ARG;
  }
  const int64_t rows = desc->rows, cols = desc->cols, params = cols * int64_t(pe);
  if (results_clash({rows_of(dx, rows, cols, lddx, e), run_of(dweight, params), run_of(dbias, params), run_of(sums ? workspace : nullptr, int64_t(need))},
                    {run_of(weight, params), run_of(mean, rows * 4), run_of(rstd, rows * 4)},
                    {rows_of(dy, rows, cols, lddy, e), rows_of(x, rows, cols, ldx, e)}))
    return MUON_ERR_INVALID_ARG;
  int sms = 0;
  if ((rc = device_of(ctx, &sms)) != MUON_OK) return rc;
  NormArgs a = norm_args(desc);
  a.device = ctx->device;
  a.status = ctx->d_status;
  a.x = x;
  a.ldx = ldx;
  a.dy = dy;
  a.lddy = lddy;
  a.weight = weight;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.out = dx;
  a.ldo = lddx;
  a.dweight = dweight;
  a.dbias = dbias;
  a.parts = sums && need > 0 ? static_cast<float*>(workspace) : nullptr;
  return launched(ctx, launch_norm_backward(a, sms, static_cast<cudaStream_t>(stream)));
}

int muon_heads_overlap(const muon_heads_t* a, const int32_t* a_shape, const muon_heads_t* b, const int32_t* b_shape, int32_t elem_size, int32_t* overlap) {
  if (!a || !a_shape || (b && !b_shape) || elem_size < 1 || !overlap) return MUON_ERR_INVALID_ARG;
  for (const muon_heads_t* t : {a, b})
    if (t && (t->batch_stride < 0 || t->token_stride < 0 || t->head_stride < 0)) return MUON_ERR_INVALID_ARG;
  const Box box = box_of(a, size_t(elem_size), a_shape[0], a_shape[1], a_shape[2], a_shape[3]);
  *overlap = b ? boxes_meet(box, box_of(b, size_t(elem_size), b_shape[0], b_shape[1], b_shape[2], b_shape[3])) : box_meets_itself(box);
  return MUON_OK;
}

int muon_rotary(muon_ctx_t* ctx, const muon_rotary_desc_t* desc, const muon_rotary_item_t* items, int32_t count, void* stream) {
  if (!ctx || !desc || count < 0 || count > kRotaryMaxItems || (count > 0 && !items)) return MUON_ERR_INVALID_ARG;
  if (!known_dtype(desc->dtype) || (desc->interleaved != 0 && desc->interleaved != 1) || (desc->inverse != 0 && desc->inverse != 1)) return MUON_ERR_INVALID_ARG;
  if (desc->rotary_dim < 2 || desc->rotary_dim % 2 || desc->rotary_dim > desc->head_dim || desc->batch < 0 || desc->tokens < 0) return MUON_ERR_INVALID_ARG;
  if (!std::isfinite(desc->amplitude) || !desc->inv_freq || !aligned_to(desc->positions, 4)) return MUON_ERR_INVALID_ARG;
  if (desc->rotary_dim > 2 * kRotaryMaxPairs || desc->head_dim > 65536) return MUON_ERR_UNSUPPORTED;
  RotaryArgs a = {};
  const size_t e = bytes_of(desc->dtype);
  for (int k = 0; k < count; ++k) {
    const muon_rotary_item_t& it = items[k];
    if (it.heads < 0 || it.heads > 65536 || it.reserved != 0) return MUON_ERR_INVALID_ARG;
    if (it.heads > 0 && int64_t(desc->batch) * desc->tokens > 0) {
      if (!good_heads(&it.in, e) || !good_output(&it.out, e, desc->batch, desc->tokens, it.heads)) return MUON_ERR_INVALID_ARG;
      if (it.in.data == it.out.data && ((desc->batch > 1 && it.in.batch_stride != it.out.batch_stride) ||
                                        (desc->tokens > 1 && it.in.token_stride != it.out.token_stride) ||
                                        (it.heads > 1 && it.in.head_stride != it.out.head_stride)))
        return MUON_ERR_INVALID_ARG;
    }
    a.item[k] = it;
    a.head_begin[k + 1] = a.head_begin[k] + it.heads;
  }
  if (int64_t(a.head_begin[count]) * desc->head_dim > (int64_t(1) << 24)) return MUON_ERR_UNSUPPORTED;   // items of a block fit 32 bits
  if (int64_t(desc->batch) * desc->tokens == 0 || a.head_begin[count] == 0) return MUON_OK;
  auto box = [&](const muon_heads_t& t, int k) { return box_of(&t, e, desc->batch, desc->tokens, items[k].heads, desc->head_dim); };
  for (int k = 0; k < count; ++k) {                  // a tensor may be turned in place, but not over another one
    const Box out = box(items[k].out, k);
    if (box_meets_itself(out)) return MUON_ERR_INVALID_ARG;
    for (int j = 0; j < count; ++j) {
      const Box in = box(items[j].in, j);
      if (!(j == k && same_box(out, in)) && boxes_meet(out, in)) return MUON_ERR_INVALID_ARG;
      if (j < k && boxes_meet(out, box(items[j].out, j))) return MUON_ERR_INVALID_ARG;
    }
  }
  a.count = count;
  a.dtype = desc->dtype;
  a.interleaved = desc->interleaved;
  a.inverse = desc->inverse;
  a.head_dim = desc->head_dim;
  a.pairs = desc->rotary_dim / 2;
  a.batch = desc->batch;
  a.tokens = desc->tokens;
  a.positions = desc->positions;
  a.position_offset = desc->position_offset;
  a.amplitude = desc->amplitude;
  for (int i = 0; i < a.pairs; ++i) a.turns[i] = desc->inv_freq[i] / kTwoPi;
  int sms = 0;
  const int rc = device_of(ctx, &sms);
  if (rc != MUON_OK) return rc;
  return launched(ctx, launch_rotary(a, sms, static_cast<cudaStream_t>(stream)));
}

int muon_rotary_frequencies(double base, int32_t rotary_dim, int32_t scaling, double factor, double original_length, double low,
                            double high, double* inv_freq) {
  if (!inv_freq || !(base > 0.0) || !std::isfinite(base) || rotary_dim < 2 || rotary_dim % 2) return MUON_ERR_INVALID_ARG;
  if (scaling != MUON_ROTARY_PLAIN && scaling != MUON_ROTARY_LINEAR && scaling != MUON_ROTARY_BY_PARTS) return MUON_ERR_INVALID_ARG;
  if (scaling != MUON_ROTARY_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return MUON_ERR_INVALID_ARG;
  if (scaling == MUON_ROTARY_BY_PARTS && (!(original_length > 0.0) || !(high > low) || !std::isfinite(high) || !std::isfinite(low))) return MUON_ERR_INVALID_ARG;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rotary_dim);
    if (scaling == MUON_ROTARY_LINEAR) f /= factor;
    if (scaling == MUON_ROTARY_BY_PARTS) {
      double k = (original_length * f / kTwoPi - low) / (high - low);
      k = k < 0.0 ? 0.0 : k > 1.0 ? 1.0 : k;
      f = k * f + (1.0 - k) * f / factor;
    }
    inv_freq[i] = f;
  }
  return MUON_OK;
}

int muon_attention_forward(muon_ctx_t* ctx, const muon_attention_desc_t* desc, const muon_heads_t* q, const muon_heads_t* k,
                           const muon_heads_t* v, const muon_heads_t* o, float* lse, void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_attention(desc);
  if (rc != MUON_OK) return rc;
  const int64_t nq = int64_t(desc->batch) * desc->q_tokens, nk = int64_t(desc->batch) * desc->k_tokens;
  if (nq == 0) return MUON_OK;
  const size_t e = bytes_of(desc->dtype);
  if (!good_heads(q, e) || !good_output(o, e, desc->batch, desc->q_tokens, desc->q_heads) || !lse || !aligned_to(lse, 4)) return MUON_ERR_INVALID_ARG;
  if (!k || !v || (nk > 0 && (!good_heads(k, e) || !good_heads(v, e)))) return MUON_ERR_INVALID_ARG;
  if (o->data == q->data || o->data == k->data || o->data == v->data) return MUON_ERR_INVALID_ARG;
  const Box bq = box_of(q, e, desc->batch, desc->q_tokens, desc->q_heads, desc->head_dim), bo = box_of(o, e, desc->batch, desc->q_tokens, desc->q_heads, desc->head_dim);
  const Box bk = box_of(k, e, desc->batch, desc->k_tokens, desc->kv_heads, desc->head_dim), bv = box_of(v, e, desc->batch, desc->k_tokens, desc->kv_heads, desc->head_dim);
  if (box_meets_itself(bo) || results_clash({bo, run_of(lse, nq * desc->q_heads * 4)}, {bq, bk, bv})) return MUON_ERR_INVALID_ARG;
  int sms = 0;
  if ((rc = device_of(ctx, &sms)) != MUON_OK) return rc;
  AttnArgs a = attention_args(ctx, desc);
  a.q = attn_tensor(q);
  a.k = attn_tensor(k);
  a.v = attn_tensor(v);
  a.o = attn_tensor(o);
  a.lse = lse;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (desc->dtype == MUON_DTYPE_BF16 && attention_forward_tc_takes(a)) return launched(ctx, launch_attention_forward_tc(ctx, a, st));
  return launched(ctx, launch_attention_forward_simt(a, desc->dtype, st));
}

int muon_attention_workspace_bytes(const muon_attention_desc_t* desc, size_t* bytes) {
  if (!bytes) return MUON_ERR_INVALID_ARG;
  const int rc = check_attention(desc);
  if (rc != MUON_OK) return rc;
  *bytes = attention_scratch(attention_args(nullptr, desc));
  return MUON_OK;
}

int muon_attention_backward(muon_ctx_t* ctx, const muon_attention_desc_t* desc, const muon_heads_t* dout, const muon_heads_t* q,
                            const muon_heads_t* k, const muon_heads_t* v, const muon_heads_t* o, const float* lse,
                            const muon_heads_t* dq, const muon_heads_t* dk, const muon_heads_t* dv, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_attention(desc);
  if (rc != MUON_OK) return rc;
  const int64_t nq = int64_t(desc->batch) * desc->q_tokens, nk = int64_t(desc->batch) * desc->k_tokens;
  if (nq == 0 && nk == 0) return MUON_OK;
  const size_t e = bytes_of(desc->dtype);
  if (!dout || !q || !k || !v || !o || !dq || !dk || !dv) return MUON_ERR_INVALID_ARG;
  if (nq > 0) {
    if (!good_heads(q, e) || !good_heads(o, e) || !good_heads(dout, e) || !lse || !aligned_to(lse, 4)) return MUON_ERR_INVALID_ARG;
    if (!good_output(dq, e, desc->batch, desc->q_tokens, desc->q_heads)) return MUON_ERR_INVALID_ARG;
  }
  if (nk > 0) {
    if (!good_heads(k, e) || !good_heads(v, e)) return MUON_ERR_INVALID_ARG;
    if (!good_output(dk, e, desc->batch, desc->k_tokens, desc->kv_heads) || !good_output(dv, e, desc->batch, desc->k_tokens, desc->kv_heads))
      return MUON_ERR_INVALID_ARG;
  }
  const muon_heads_t* in[5] = {dout, q, k, v, o};
  const muon_heads_t* out[3] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i) {
    for (const muon_heads_t* t : in)
      if (out[i]->data && out[i]->data == t->data) return MUON_ERR_INVALID_ARG;
    if (out[i]->data && out[i]->data == out[(i + 1) % 3]->data) return MUON_ERR_INVALID_ARG;
  }
  AttnArgs a = attention_args(ctx, desc);
  const size_t need = attention_scratch(a);
  if (need > 0) {
    if (!workspace || workspace_bytes < need) return MUON_ERR_WORKSPACE_TOO_SMALL;
    if (!aligned_to(workspace, 256)) return MUON_ERR_INVALID_ARG;
  }
  auto queries = [&](const muon_heads_t* t) { return box_of(t, e, desc->batch, desc->q_tokens, desc->q_heads, desc->head_dim); };
  auto keys = [&](const muon_heads_t* t) { return box_of(t, e, desc->batch, desc->k_tokens, desc->kv_heads, desc->head_dim); };
  if (box_meets_itself(queries(dq)) || box_meets_itself(keys(dk)) || box_meets_itself(keys(dv)) ||
      results_clash({queries(dq), keys(dk), keys(dv), run_of(workspace, int64_t(need))},
                    {queries(dout), queries(q), keys(k), keys(v), queries(o), run_of(lse, nq * desc->q_heads * 4)}))
    return MUON_ERR_INVALID_ARG;
  int sms = 0;
  if ((rc = device_of(ctx, &sms)) != MUON_OK) return rc;
  a.q = attn_tensor(q);
  a.k = attn_tensor(k);
  a.v = attn_tensor(v);
  a.o = attn_tensor(o);
  a.dout = attn_tensor(dout);
  a.dq = attn_tensor(dq);
  a.dk = attn_tensor(dk);
  a.dv = attn_tensor(dv);
  a.lse = const_cast<float*>(lse);
  a.rows = static_cast<float*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int rows = launch_attention_rows(a, desc->dtype, st);
  if (rows < 0) return launched(ctx, rows);
  ctx->launches += rows;
  if (desc->dtype == MUON_DTYPE_BF16 && attention_backward_tc_takes(a)) return launched(ctx, launch_attention_backward_tc(ctx, a, st));
  return launched(ctx, launch_attention_backward_simt(a, desc->dtype, st));
}

}  // extern "C"
