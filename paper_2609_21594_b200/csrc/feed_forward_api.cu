// extern "C" entry points of the gated feed-forward block, of activations in 8 bits and of the 8-bit linear layer: argument validation, layout
// of the scratch, and the list of products that each call is.
#include "layer_checks.h"
#include "product_ops.h"

using namespace muon;

namespace {

constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 1 - 512;      // tile coordinates past the last row stay in 32 bits
constexpr int64_t kUnalignedRows = 512;                           // rows at a time whose fp32 g and u wait for their 8 bits (CUDA cores only)

int64_t up_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

// ------------------------------------------------------------------ checks
bool good_rows(const muon_rows_t* t, int64_t rows, int64_t cols, size_t elem) {
  return rows == 0 || cols == 0 || (t && t->data && aligned_to(t->data, elem) && t->ld >= cols && t->ld <= (int64_t(1) << 40));
}
bool good_blocks(const muon_blocks_t* t, int64_t rows, int64_t cols, int32_t block_rows) {
  if (rows == 0 || cols == 0) return true;
  if (!t || !t->codes || !t->scales || t->reserved != 0 || (block_rows ? t->block_rows != block_rows : t->block_rows != 1 && t->block_rows != kBlock)) return false;
  return t->ld >= cols && t->lds >= blocks_of(cols) && t->ld <= (int64_t(1) << 40) && t->lds <= (int64_t(1) << 40);
}
Box rows_box(const muon_rows_t* t, int64_t rows, int64_t cols, size_t elem) {
  return t ? rows_of(t->data, rows, cols, t->ld, elem) : run_of(nullptr, 0);
}
Box codes_box(const muon_blocks_t& t, int64_t rows, int64_t cols) { return rows_of(t.codes, rows, cols, t.ld, 1); }
Box scales_box(const muon_blocks_t& t, int64_t rows, int64_t cols) {
  return rows_of(t.scales, t.block_rows == 1 ? rows : blocks_of(rows), blocks_of(cols), t.lds, 1);
}

// ------------------------------------------------------------------ operands and launches
Operand operand(const void* data, int64_t ld, int dtype, bool mn_major = false) {
  Operand o = {};
  o.data = data;
  o.ld = ld;
  o.type = dtype;
  o.mn_major = mn_major;
  return o;
}
Operand operand(const muon_rows_t* t, int dtype, bool mn_major = false) { return operand(t->data, t->ld, dtype, mn_major); }
Operand operand(const muon_blocks_t* t, bool mn_major = false) {
  Operand o = operand(t->codes, t->ld, kTypeE4m3, mn_major);
  o.scales = t->scales;
  o.lds = t->lds;
  o.block_rows = t->block_rows;
  return o;
}
Product plain(int64_t m, int64_t n, int64_t k, const Operand& a, const Operand& b, void* c, int64_t ldc, int type) {
  Product p = {};
  p.m = int32_t(m);
  p.n = int32_t(n);
  p.k = int32_t(k);
  p.segments = 1;
  p.a[0] = a;
  p.b[0] = b;
  p.e.kind = kPlain;
  p.e.type = type;
  p.e.c = c;
  p.e.ldc = ldc;
  return p;
}

// A call's launches in order; the first error ends it.
struct Launches {
  muon_ctx* ctx;
  int sms;
  cudaStream_t st;
  int rc = MUON_OK;
  void count(int n) {
    const int r = launched(ctx, n);
    if (rc == MUON_OK) rc = r;
  }
  // follows: the call's last launch is right before this one in the stream, and writes nothing but what it takes as A
  void products(const Product* p, int n, int siblings, bool follows = false) {
    if (rc != MUON_OK || n == 0) return;
    if (products_tc_take(p, n)) return count(n == 1 && product_few_takes(*p, sms) ? launch_product_few(ctx, *p, sms, follows, st) : launch_products_tc(ctx, p, n, st));
    count(launch_products_simt(p, n, siblings, sms, st));
  }
  void product(const Product& p, bool follows = false) { products(&p, 1, 1, follows); }
  void quantize(int dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, const Operand& out) {
    if (rc == MUON_OK) count(launch_quantize(dtype, rows, cols, x, ldx, out, sms, st));
  }
  void dequantize(int dtype, int64_t rows, int64_t cols, const Operand& in, void* y, int64_t ldy) {
    if (rc == MUON_OK) count(launch_dequantize(dtype, rows, cols, in, y, ldy, sms, st));
  }
};

// Pieces of a workspace, each aligned to 256 bytes.  Without a base it only adds them up.
struct Scratch {
  char* base;
  size_t used = 0;
  void* take(int64_t bytes) {
    void* p = base ? base + used : nullptr;
    used += size_t(up_to(bytes, 256));
    return p;
  }
};
int check_scratch(const void* workspace, size_t have, size_t need) {
  if (need == 0) return MUON_OK;
  if (!workspace || have < need) return MUON_ERR_WORKSPACE_TOO_SMALL;
  return aligned_to(workspace, 256) ? MUON_OK : MUON_ERR_INVALID_ARG;
}

// ------------------------------------------------------------------ feed-forward block
int check_feed_forward(const muon_feed_forward_desc_t* d) {
  if (!d || !known_dtype(d->dtype) || (d->activation != MUON_ACTIVATION_SILU && d->activation != MUON_ACTIVATION_GELU)) return MUON_ERR_INVALID_ARG;
  if (d->keep != MUON_KEEP_NONE && d->keep != MUON_KEEP_FULL && d->keep != MUON_KEEP_8BIT) return MUON_ERR_INVALID_ARG;
  if (d->tokens < 0 || d->dim < 1 || d->hidden < 1) return MUON_ERR_INVALID_ARG;
  return d->tokens > kMaxTokens || d->dim > kMaxTokens || d->hidden > kMaxTokens ? MUON_ERR_UNSUPPORTED : MUON_OK;
}

bool good_kept(const muon_feed_forward_desc_t* d, const muon_feed_forward_kept_t* k) {
  if (d->keep == MUON_KEEP_NONE || d->tokens == 0) return true;
  if (!k) return false;
  if (d->keep == MUON_KEEP_FULL) return good_rows(&k->gate, d->tokens, d->hidden, bytes_of(d->dtype)) && good_rows(&k->up, d->tokens, d->hidden, bytes_of(d->dtype));
  return good_blocks(&k->x8, d->tokens, d->dim, 1) && good_blocks(&k->gate8, d->tokens, d->hidden, 1) && good_blocks(&k->up8, d->tokens, d->hidden, 1);
}

// Memory of what is kept, as up to six boxes.
struct KeptBoxes {
  Box box[6];
  KeptBoxes(const muon_feed_forward_desc_t* d, const muon_feed_forward_kept_t* k)
      : box{run_of(nullptr, 0), run_of(nullptr, 0), run_of(nullptr, 0), run_of(nullptr, 0), run_of(nullptr, 0), run_of(nullptr, 0)} {
    if (d->tokens == 0) return;
    if (d->keep == MUON_KEEP_FULL) {
      box[0] = rows_box(&k->gate, d->tokens, d->hidden, bytes_of(d->dtype));
      box[1] = rows_box(&k->up, d->tokens, d->hidden, bytes_of(d->dtype));
    } else if (d->keep == MUON_KEEP_8BIT) {
      const muon_blocks_t* b[3] = {&k->x8, &k->gate8, &k->up8};
      for (int i = 0; i < 3; ++i) {
        const int64_t cols = i ? d->hidden : d->dim;
        box[2 * i] = codes_box(*b[i], d->tokens, cols);
        box[2 * i + 1] = scales_box(*b[i], d->tokens, cols);
      }
    }
  }
};

struct ForwardScratch {
  int64_t ldh;
  void *h, *gate, *up;           // gate, up: fp32, for kUnalignedRows rows
};
ForwardScratch forward_scratch(const muon_feed_forward_desc_t* d, Scratch* s) {
  ForwardScratch r = {};
  r.ldh = up_to(d->hidden, 8);
  r.h = s->take(d->tokens * r.ldh * int64_t(bytes_of(d->dtype)));
  if (d->keep == MUON_KEEP_8BIT) {
    const int64_t rows = d->tokens < kUnalignedRows ? d->tokens : kUnalignedRows;
    r.gate = s->take(rows * d->hidden * 4);
    r.up = s->take(rows * d->hidden * 4);
  }
  return r;
}
struct BackwardScratch {
  int64_t ldh, ldx;
  void *dgate, *dup, *h, *x;
};
BackwardScratch backward_scratch(const muon_feed_forward_desc_t* d, Scratch* s) {
  BackwardScratch r = {};
  const int64_t e = int64_t(bytes_of(d->dtype));
  r.ldh = up_to(d->hidden, 8);
  r.ldx = up_to(d->dim, 8);
  r.dgate = s->take(d->tokens * r.ldh * e);
  r.dup = s->take(d->tokens * r.ldh * e);
  r.h = s->take(d->tokens * r.ldh * e);
  if (d->keep == MUON_KEEP_8BIT) r.x = s->take(d->tokens * r.ldx * e);
  return r;
}

// ------------------------------------------------------------------ 8-bit linear layer
int check_linear(const muon_linear_blocks_desc_t* d) {
  if (!d || d->reserved != 0 || d->tokens < 0 || d->dim < 1 || d->out < 1) return MUON_ERR_INVALID_ARG;
  return d->tokens > kMaxTokens || d->dim > kMaxTokens || d->out > kMaxTokens ? MUON_ERR_UNSUPPORTED : MUON_OK;
}
struct LinearScratch {
  muon_blocks_t dy8;
  void* x;
  int64_t ldx;
};
LinearScratch linear_scratch(const muon_linear_blocks_desc_t* d, Scratch* s) {
  LinearScratch r = {};
  r.dy8.ld = up_to(d->out, 16);
  r.dy8.lds = up_to(blocks_of(d->out), 16);       // the tensor cores' scales are read 16 bytes at a time
  r.dy8.block_rows = 1;
  r.dy8.codes = s->take(d->tokens * r.dy8.ld);
  r.dy8.scales = static_cast<uint8_t*>(s->take(d->tokens * r.dy8.lds));
  r.ldx = up_to(d->dim, 8);
  r.x = s->take(d->tokens * r.ldx * 2);
  return r;
}

}  // namespace

extern "C" {

int muon_quantize(muon_ctx_t* ctx, int32_t dtype, int64_t rows, int64_t cols, const muon_rows_t* x, const muon_blocks_t* out, void* stream) {
  if (!ctx || !known_dtype(dtype) || rows < 0 || cols < 0) return MUON_ERR_INVALID_ARG;
  if (rows > (int64_t(1) << 40) || cols > kMaxTokens) return MUON_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return MUON_OK;
  const size_t e = bytes_of(dtype);
  if (!good_rows(x, rows, cols, e) || !good_blocks(out, rows, cols, 0)) return MUON_ERR_INVALID_ARG;
  if (results_clash({codes_box(*out, rows, cols), scales_box(*out, rows, cols)}, {rows_box(x, rows, cols, e)})) return MUON_ERR_INVALID_ARG;
  Launches l = {ctx, 0, static_cast<cudaStream_t>(stream)};
  const int rc = device_of(ctx, &l.sms);
  if (rc != MUON_OK) return rc;
  l.quantize(dtype, rows, cols, x->data, x->ld, operand(out));
  return l.rc;
}

int muon_dequantize(muon_ctx_t* ctx, int32_t dtype, int64_t rows, int64_t cols, const muon_blocks_t* in, const muon_rows_t* y, void* stream) {
  if (!ctx || !known_dtype(dtype) || rows < 0 || cols < 0) return MUON_ERR_INVALID_ARG;
  if (rows > (int64_t(1) << 40) || cols > kMaxTokens) return MUON_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return MUON_OK;
  const size_t e = bytes_of(dtype);
  if (!good_rows(y, rows, cols, e) || !good_blocks(in, rows, cols, 0)) return MUON_ERR_INVALID_ARG;
  if (results_clash({rows_box(y, rows, cols, e)}, {codes_box(*in, rows, cols), scales_box(*in, rows, cols)})) return MUON_ERR_INVALID_ARG;
  Launches l = {ctx, 0, static_cast<cudaStream_t>(stream)};
  const int rc = device_of(ctx, &l.sms);
  if (rc != MUON_OK) return rc;
  l.dequantize(dtype, rows, cols, operand(in), y->data, y->ld);
  return l.rc;
}

int muon_feed_forward_workspace_bytes(const muon_feed_forward_desc_t* desc, int32_t backward, size_t* bytes) {
  if (!bytes || (backward != 0 && backward != 1)) return MUON_ERR_INVALID_ARG;
  const int rc = check_feed_forward(desc);
  if (rc != MUON_OK) return rc;
  Scratch s = {nullptr};
  if (backward) backward_scratch(desc, &s);
  else forward_scratch(desc, &s);
  *bytes = s.used;
  return MUON_OK;
}

int muon_feed_forward_forward(muon_ctx_t* ctx, const muon_feed_forward_desc_t* d, const muon_rows_t* x, const muon_rows_t* w_gate, const muon_rows_t* w_up,
                              const muon_rows_t* w_down, const muon_rows_t* y, const muon_feed_forward_kept_t* kept, void* workspace,
                              size_t workspace_bytes, void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_feed_forward(d);
  if (rc != MUON_OK) return rc;
  if (d->tokens == 0) return MUON_OK;
  const int64_t t = d->tokens, dim = d->dim, hidden = d->hidden;
  const size_t e = bytes_of(d->dtype);
  if (!good_rows(x, t, dim, e) || !good_rows(y, t, dim, e) || !good_rows(w_gate, hidden, dim, e) || !good_rows(w_up, hidden, dim, e) ||
      !good_rows(w_down, dim, hidden, e) || !good_kept(d, kept))
    return MUON_ERR_INVALID_ARG;
  Scratch s = {static_cast<char*>(workspace)};
  const ForwardScratch w = forward_scratch(d, &s);
  if ((rc = check_scratch(workspace, workspace_bytes, s.used)) != MUON_OK) return rc;
  const KeptBoxes k(d, kept);
  if (results_clash({rows_box(y, t, dim, e), run_of(workspace, int64_t(s.used)), k.box[0], k.box[1], k.box[2], k.box[3], k.box[4], k.box[5]},
                    {rows_box(x, t, dim, e), rows_box(w_gate, hidden, dim, e), rows_box(w_up, hidden, dim, e), rows_box(w_down, dim, hidden, e)}))
    return MUON_ERR_INVALID_ARG;
  Launches l = {ctx, 0, static_cast<cudaStream_t>(stream)};
  if ((rc = device_of(ctx, &l.sms)) != MUON_OK) return rc;

  Product p = plain(t, hidden, dim, operand(x, d->dtype), operand(w_gate, d->dtype), w.h, w.ldh, d->dtype);
  p.b[1] = operand(w_up, d->dtype);
  p.e.kind = kGated;
  p.e.activation = d->activation;
  p.e.gate_up_type = d->dtype;
  if (d->keep == MUON_KEEP_FULL) {
    p.e.gate = kept->gate.data;
    p.e.ld_gate = kept->gate.ld;
    p.e.up = kept->up.data;
    p.e.ld_up = kept->up.ld;
  } else if (d->keep == MUON_KEEP_8BIT) {
    p.e.gate_up_type = kTypeE4m3;
    p.e.in_gate = operand(&kept->gate8);
    p.e.in_up = operand(&kept->up8);
    l.quantize(d->dtype, t, dim, x->data, x->ld, operand(&kept->x8));
  }
  if (d->keep != MUON_KEEP_8BIT || products_tc_take(&p, 1)) {
    l.product(p);
  } else {                       // on CUDA cores a tile does not hold a block's columns: g and u wait in fp32, some rows at a time
    for (int64_t r = 0; r < t && l.rc == MUON_OK; r += kUnalignedRows) {
      const int64_t n = t - r < kUnalignedRows ? t - r : kUnalignedRows;
      Product q = p;
      q.m = int32_t(n);
      q.a[0].data = static_cast<const char*>(x->data) + r * x->ld * int64_t(e);
      q.e.c = static_cast<char*>(w.h) + r * w.ldh * int64_t(e);
      q.e.gate_up_type = kTypeFp32;
      q.e.gate = w.gate;
      q.e.up = w.up;
      q.e.ld_gate = q.e.ld_up = hidden;
      l.count(launch_products_simt(&q, 1, 1, l.sms, l.st));
      for (const Operand* o : {&p.e.in_gate, &p.e.in_up}) {
        Operand part = *o;
        part.data = static_cast<const uint8_t*>(o->data) + r * o->ld;
        part.scales = o->scales + r * o->lds;
        l.quantize(kTypeFp32, n, hidden, o == &p.e.in_gate ? w.gate : w.up, hidden, part);
      }
    }
  }
  l.product(plain(t, dim, hidden, operand(w.h, w.ldh, d->dtype), operand(w_down, d->dtype), y->data, y->ld, d->dtype), true);
  return l.rc;
}

int muon_feed_forward_backward(muon_ctx_t* ctx, const muon_feed_forward_desc_t* d, const muon_rows_t* dy, const muon_rows_t* x, const muon_rows_t* w_gate,
                               const muon_rows_t* w_up, const muon_rows_t* w_down, const muon_feed_forward_kept_t* kept, const muon_rows_t* dx,
                               const muon_rows_t* dw_gate, const muon_rows_t* dw_up, const muon_rows_t* dw_down, void* workspace, size_t workspace_bytes,
                               void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_feed_forward(d);
  if (rc != MUON_OK) return rc;
  if (d->keep == MUON_KEEP_NONE) return MUON_ERR_INVALID_ARG;
  const int64_t t = d->tokens, dim = d->dim, hidden = d->hidden;
  const size_t e = bytes_of(d->dtype);
  const bool given_x = d->keep == MUON_KEEP_FULL;
  if (!dx && !dw_gate && !dw_up && !dw_down) return MUON_OK;
  if (!good_rows(dy, t, dim, e) || (given_x ? !good_rows(x, t, dim, e) : x != nullptr) || !good_rows(w_gate, hidden, dim, e) || !good_rows(w_up, hidden, dim, e) ||
      !good_rows(w_down, dim, hidden, e) || !good_kept(d, kept))
    return MUON_ERR_INVALID_ARG;
  if ((dx && !good_rows(dx, t, dim, e)) || (dw_gate && !good_rows(dw_gate, hidden, dim, e)) || (dw_up && !good_rows(dw_up, hidden, dim, e)) ||
      (dw_down && !good_rows(dw_down, dim, hidden, e)))
    return MUON_ERR_INVALID_ARG;
  Scratch s = {static_cast<char*>(workspace)};
  const BackwardScratch w = backward_scratch(d, &s);
  if ((rc = check_scratch(workspace, workspace_bytes, s.used)) != MUON_OK) return rc;
  const KeptBoxes k(d, kept);
  if (results_clash({rows_box(dx, t, dim, e), rows_box(dw_gate, hidden, dim, e), rows_box(dw_up, hidden, dim, e), rows_box(dw_down, dim, hidden, e),
                     run_of(workspace, int64_t(s.used))},
                    {rows_box(dy, t, dim, e), rows_box(x, t, dim, e), rows_box(w_gate, hidden, dim, e), rows_box(w_up, hidden, dim, e),
                     rows_box(w_down, dim, hidden, e), k.box[0], k.box[1], k.box[2], k.box[3], k.box[4], k.box[5]}))
    return MUON_ERR_INVALID_ARG;
  Launches l = {ctx, 0, static_cast<cudaStream_t>(stream)};
  if ((rc = device_of(ctx, &l.sms)) != MUON_OK) return rc;

  const int dt = d->dtype;
  const muon_rows_t none = {nullptr, dim};
  if (!dy) dy = &none;           // no tokens: the products below have no k
  if (!x) x = &none;
  if (t > 0) {
    Product p = plain(t, hidden, dim, operand(dy, dt), operand(w_down, dt, true), w.h, w.ldh, dt);
    p.e.kind = kGrad;
    p.e.activation = d->activation;
    p.e.gate = w.dgate;
    p.e.up = w.dup;
    p.e.ld_gate = p.e.ld_up = w.ldh;
    p.e.in_gate = given_x ? operand(&kept->gate, dt) : operand(&kept->gate8);
    p.e.in_up = given_x ? operand(&kept->up, dt) : operand(&kept->up8);
    p.e.gate_up_type = p.e.in_gate.type;
    l.product(p);
  }
  if (dx && t > 0) {
    Product p = plain(t, dim, hidden, operand(w.dgate, w.ldh, dt), operand(w_gate, dt, true), dx->data, dx->ld, dt);
    p.segments = 2;
    p.a[1] = operand(w.dup, w.ldh, dt);
    p.b[1] = operand(w_up, dt, true);
    l.product(p, true);
  }
  Operand ox = operand(x, dt, true);
  if (!given_x && (dw_gate || dw_up)) {
    if (t > 0) l.dequantize(dt, t, dim, operand(&kept->x8), w.x, w.ldx);
    ox = operand(w.x, w.ldx, dt, true);
  }
  Product list[kMaxProducts];
  int n = 0;
  if (dw_gate) list[n++] = plain(hidden, dim, t, operand(w.dgate, w.ldh, dt, true), ox, dw_gate->data, dw_gate->ld, dt);
  if (dw_up) list[n++] = plain(hidden, dim, t, operand(w.dup, w.ldh, dt, true), ox, dw_up->data, dw_up->ld, dt);
  if (dw_down) list[n++] = plain(dim, hidden, t, operand(dy, dt, true), operand(w.h, w.ldh, dt, true), dw_down->data, dw_down->ld, dt);
  l.products(list, n, kMaxProducts);
  return l.rc;
}

int muon_linear_blocks_forward(muon_ctx_t* ctx, const muon_linear_blocks_desc_t* d, const muon_rows_t* x, const muon_blocks_t* w8, const muon_rows_t* y,
                             const muon_blocks_t* x8, void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_linear(d);
  if (rc != MUON_OK) return rc;
  if (d->tokens == 0) return MUON_OK;
  const int64_t t = d->tokens, dim = d->dim, out = d->out;
  if (!good_rows(x, t, dim, 2) || !good_rows(y, t, out, 2) || !good_blocks(w8, out, dim, kBlock) || !good_blocks(x8, t, dim, 1)) return MUON_ERR_INVALID_ARG;
  if (results_clash({rows_box(y, t, out, 2), codes_box(*x8, t, dim), scales_box(*x8, t, dim)},
                    {rows_box(x, t, dim, 2), codes_box(*w8, out, dim), scales_box(*w8, out, dim)}))
    return MUON_ERR_INVALID_ARG;
  Launches l = {ctx, 0, static_cast<cudaStream_t>(stream)};
  if ((rc = device_of(ctx, &l.sms)) != MUON_OK) return rc;
  l.quantize(kTypeBf16, t, dim, x->data, x->ld, operand(x8));
  l.product(plain(t, out, dim, operand(x8), operand(w8), y->data, y->ld, kTypeBf16), true);
  return l.rc;
}

int muon_linear_blocks_workspace_bytes(const muon_linear_blocks_desc_t* desc, size_t* bytes) {
  if (!bytes) return MUON_ERR_INVALID_ARG;
  const int rc = check_linear(desc);
  if (rc != MUON_OK) return rc;
  Scratch s = {nullptr};
  linear_scratch(desc, &s);
  *bytes = s.used;
  return MUON_OK;
}

int muon_linear_blocks_backward(muon_ctx_t* ctx, const muon_linear_blocks_desc_t* d, const muon_rows_t* dy, const muon_blocks_t* x8, const muon_blocks_t* w8,
                              const muon_rows_t* dx, const muon_rows_t* dw, void* workspace, size_t workspace_bytes, void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_linear(d);
  if (rc != MUON_OK) return rc;
  if (!dx && !dw) return MUON_OK;
  const int64_t t = d->tokens, dim = d->dim, out = d->out;
  if (!good_rows(dy, t, out, 2) || (dw && !good_blocks(x8, t, dim, 1)) || (dx && t > 0 && !good_blocks(w8, out, dim, kBlock)) ||
      (dx && !good_rows(dx, t, dim, 2)) || (dw && !good_rows(dw, out, dim, 2)))
    return MUON_ERR_INVALID_ARG;
  Scratch s = {static_cast<char*>(workspace)};
  const LinearScratch w = linear_scratch(d, &s);
  if ((rc = check_scratch(workspace, workspace_bytes, s.used)) != MUON_OK) return rc;
  const Box nothing = run_of(nullptr, 0);
  const bool rx = dw && t > 0, rw = dx && t > 0;
  if (results_clash({rows_box(dx, t, dim, 2), rows_box(dw, out, dim, 2), run_of(workspace, int64_t(s.used))},
                    {rows_box(dy, t, out, 2), rx ? codes_box(*x8, t, dim) : nothing, rx ? scales_box(*x8, t, dim) : nothing,
                     rw ? codes_box(*w8, out, dim) : nothing, rw ? scales_box(*w8, out, dim) : nothing}))
    return MUON_ERR_INVALID_ARG;
  Launches l = {ctx, 0, static_cast<cudaStream_t>(stream)};
  if ((rc = device_of(ctx, &l.sms)) != MUON_OK) return rc;
  if (rw) {
    l.quantize(kTypeBf16, t, out, dy->data, dy->ld, operand(&w.dy8));
    l.product(plain(t, dim, out, operand(&w.dy8), operand(w8, true), dx->data, dx->ld, kTypeBf16), true);
  }
  if (dw) {
    const muon_rows_t none = {nullptr, out};
    if (rx) l.dequantize(kTypeBf16, t, dim, operand(x8), w.x, w.ldx);
    l.product(plain(out, dim, t, operand(rx ? dy : &none, kTypeBf16, true), operand(w.x, w.ldx, kTypeBf16, true), dw->data, dw->ld, kTypeBf16));
  }
  return l.rc;
}

}  // extern "C"
