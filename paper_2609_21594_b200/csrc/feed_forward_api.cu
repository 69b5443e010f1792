// extern "C" entry points of the gated feed-forward block, of activations in 8 bits and of the 8-bit linear layer: argument validation, layout
// of the scratch, and the list of products that each call is.
#include <algorithm>

#include "layer_checks.h"
#include "product_ops.h"

using namespace muon;

namespace {

constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 1 - 512;      // tile coordinates past the last row stay in 32 bits
constexpr int64_t kUnalignedRows = 512;                           // rows at a time whose fp32 g and u wait for their 8 bits (CUDA cores only)
// Multiply-adds of a product from which on it is worth copying what TMA cannot address (rows of an odd number of elements) into rows that it can:
// two launches more against CUDA cores.  20 x 301 x 700 (2^22), 8-bit linear layer: 27 us there, 21 by copies, backward 51 and 33; 8 x 4096 x 1003 85 and 18.
constexpr int64_t kWorthCopies = int64_t(1) << 21;

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
  // Each product's engine is its own affair: a gradient has the same bits whichever others are wanted.
  void products(const Product* p, int n, int siblings, Before before = kBeforeAny) {
    Product part[2][kMaxProducts];
    int count[2] = {0, 0};
    for (int i = 0; i < n; ++i) {
      const int tc = products_tc_take(p + i, 1) ? 1 : 0;
      part[tc][count[tc]++] = p[i];
    }
    if (rc == MUON_OK && count[1] == 1 && product_few_takes(part[1][0], sms)) this->count(launch_product_few(ctx, part[1][0], sms, before, st));
    else if (count[1] > 0) products_tc(part[1], count[1], before);
    if (rc == MUON_OK && count[0] > 0) this->count(launch_products_simt(part[0], count[0], siblings, sms, st));
  }
  // Sums over more tokens than kLongestSum one part after the other, a launch each.
  void products_tc(Product* p, int n, Before before) {
    const int64_t k = p[0].k, step = p[0].e.sums ? kLongestSum : k;
    for (int64_t k0 = 0; k0 < k && rc == MUON_OK; k0 += step) {
      for (int i = 0; i < n; ++i) {
        p[i].k = int32_t(std::min(step, k - k0));
        p[i].e.add = k0 > 0;
        p[i].e.hold = k0 + step < k;
      }
      this->count(launch_products_tc(ctx, p, n, k0 > 0 ? kBeforeSameCall : before, st));
      if (k0 + step < k)
        for (int i = 0; i < n; ++i)
          for (Operand* o : {&p[i].a[0], &p[i].b[0]}) o->data = static_cast<const char*>(o->data) + step * o->ld * size_of_type(o->type);
    }
  }
  void product(const Product& p, Before before = kBeforeAny) { products(&p, 1, 1, before); }
  void copies(const CopyTask* list, int n) {
    if (rc == MUON_OK && n > 0) count(launch_copies(list, n, sms, st));
  }
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

// Where the parts of the sum over `tokens` meet that a gradient of rows x cols is.
struct Sums {
  float* data;
  int64_t ld;
};
Sums sums_of(Scratch* s, int64_t tokens, int64_t rows, int64_t cols, int type) {
  if (tokens <= kLongestSum || type != kTypeBf16) return {nullptr, 0};
  const int64_t ld = up_to(cols, 64);
  return {static_cast<float*>(s->take(rows * ld * 4)), ld};
}
Product with(Product p, const Sums& s) {
  p.e.sums = s.data;
  p.e.ld_sums = s.ld;
  return p;
}

// Operands and results that TMA cannot address and that have room in the scratch are copied there and back.
struct Copies {
  CopyTask in[kMaxCopies], out[kMaxCopies];
  int ins = 0, outs = 0;
  static int64_t pitch(int64_t cols, int type) { return up_to(cols, 16 / size_of_type(type)); }
  Operand take(Operand o, int64_t rows, int64_t cols, void* room) {
    if (!room || addressable(o.data, o.ld, o.type)) return o;
    const int e = size_of_type(o.type);
    const int64_t ld = pitch(cols, o.type);
    in[ins++] = {o.data, room, o.ld * e, ld * e, rows, cols * e, e};
    o.data = room;
    o.ld = ld;
    return o;
  }
  muon_rows_t give(const muon_rows_t* to, int64_t rows, int64_t cols, void* room, int type) {
    if (!room || addressable(to->data, to->ld, type)) return *to;
    const int e = size_of_type(type);
    const int64_t ld = pitch(cols, type);
    out[outs++] = {room, to->data, ld * e, to->ld * e, rows, cols * e, e};
    return {room, ld};
  }
};
void* room(Scratch* s, bool odd, int64_t rows, int64_t cols, int type) {
  return odd ? s->take(rows * Copies::pitch(cols, type) * size_of_type(type)) : nullptr;
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

// Whether rows of dim and of hidden elements get room for copies.
struct Odd {
  bool dim, hidden;
  explicit Odd(const muon_feed_forward_desc_t* d) {
    const bool worth = d->dtype == kTypeBf16 && int64_t(d->tokens) * d->dim >= (kWorthCopies + d->hidden - 1) / d->hidden;
    dim = worth && d->dim % 8 != 0;
    hidden = worth && d->hidden % 8 != 0;
  }
};
struct ForwardScratch {
  int64_t ldh;
  void *h, *gate, *up;           // gate, up: fp32, for kUnalignedRows rows
  void *x, *w_gate, *w_up, *w_down, *y, *kept_gate, *kept_up;      // copies
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
  const Odd odd(d);
  const int64_t t = d->tokens;
  r.x = room(s, odd.dim, t, d->dim, d->dtype);
  r.w_gate = room(s, odd.dim, d->hidden, d->dim, d->dtype);
  r.w_up = room(s, odd.dim, d->hidden, d->dim, d->dtype);
  r.y = room(s, odd.dim, t, d->dim, d->dtype);
  r.w_down = room(s, odd.hidden, d->dim, d->hidden, d->dtype);
  r.kept_gate = room(s, odd.hidden && d->keep == MUON_KEEP_FULL, t, d->hidden, d->dtype);
  r.kept_up = room(s, odd.hidden && d->keep == MUON_KEEP_FULL, t, d->hidden, d->dtype);
  return r;
}
struct BackwardScratch {
  int64_t ldh, ldx;
  void *dgate, *dup, *h, *x;
  void *dy, *given_x, *w_gate, *w_up, *w_down, *gate, *up, *dx, *dw_gate, *dw_up, *dw_down;      // copies
  Sums sum_gate, sum_up, sum_down;
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
  const Odd odd(d);
  const bool full = d->keep == MUON_KEEP_FULL;
  const int64_t t = d->tokens;
  r.dy = room(s, odd.dim, t, d->dim, d->dtype);
  r.given_x = room(s, odd.dim && full, t, d->dim, d->dtype);
  r.w_gate = room(s, odd.dim, d->hidden, d->dim, d->dtype);
  r.w_up = room(s, odd.dim, d->hidden, d->dim, d->dtype);
  r.dx = room(s, odd.dim, t, d->dim, d->dtype);
  r.dw_gate = room(s, odd.dim, d->hidden, d->dim, d->dtype);
  r.dw_up = room(s, odd.dim, d->hidden, d->dim, d->dtype);
  r.w_down = room(s, odd.hidden, d->dim, d->hidden, d->dtype);
  r.dw_down = room(s, odd.hidden, d->dim, d->hidden, d->dtype);
  r.gate = room(s, odd.hidden && full, t, d->hidden, d->dtype);
  r.up = room(s, odd.hidden && full, t, d->hidden, d->dtype);
  r.sum_gate = sums_of(s, t, d->hidden, d->dim, d->dtype);
  r.sum_up = sums_of(s, t, d->hidden, d->dim, d->dtype);
  r.sum_down = sums_of(s, t, d->dim, d->hidden, d->dtype);
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
  void *w8, *y, *dy, *dx, *dw;   // copies
  Sums sum;                      // of dw
};
LinearScratch linear_scratch(const muon_linear_blocks_desc_t* d, bool backward, Scratch* s) {
  LinearScratch r = {};
  const bool worth = int64_t(d->tokens) * d->dim >= (kWorthCopies + d->out - 1) / d->out;
  r.w8 = room(s, worth && d->dim % 16 != 0, d->out, d->dim, kTypeE4m3);
  if (!backward) {
    r.y = room(s, worth && d->out % 8 != 0, d->tokens, d->out, kTypeBf16);
    return r;
  }
  r.dy = room(s, worth && d->out % 8 != 0, d->tokens, d->out, kTypeBf16);
  r.dx = room(s, worth && d->dim % 8 != 0, d->tokens, d->dim, kTypeBf16);
  r.dw = room(s, worth && d->dim % 8 != 0, d->out, d->dim, kTypeBf16);
  r.dy8.ld = up_to(d->out, 16);
  r.dy8.lds = up_to(blocks_of(d->out), 16);       // the tensor cores' scales are read 16 bytes at a time
  r.dy8.block_rows = 1;
  r.dy8.codes = s->take(d->tokens * r.dy8.ld);
  r.dy8.scales = static_cast<uint8_t*>(s->take(d->tokens * r.dy8.lds));
  r.ldx = up_to(d->dim, 8);
  r.x = s->take(d->tokens * r.ldx * 2);
  r.sum = sums_of(s, d->tokens, d->out, d->dim, kTypeBf16);
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

  const int dt = d->dtype;
  Copies c;
  const Operand ox = c.take(operand(x, dt), t, dim, w.x);
  Product p = plain(t, hidden, dim, ox, c.take(operand(w_gate, dt), hidden, dim, w.w_gate), w.h, w.ldh, dt);
  p.b[1] = c.take(operand(w_up, dt), hidden, dim, w.w_up);
  const Operand down = c.take(operand(w_down, dt), dim, hidden, w.w_down);
  const muon_rows_t oy = c.give(y, t, dim, w.y, dt);
  p.e.kind = kGated;
  p.e.activation = d->activation;
  p.e.gate_up_type = dt;
  if (d->keep == MUON_KEEP_FULL) {
    const muon_rows_t gate = c.give(&kept->gate, t, hidden, w.kept_gate, dt), up = c.give(&kept->up, t, hidden, w.kept_up, dt);
    p.e.gate = gate.data;
    p.e.ld_gate = gate.ld;
    p.e.up = up.data;
    p.e.ld_up = up.ld;
  } else if (d->keep == MUON_KEEP_8BIT) {
    p.e.gate_up_type = kTypeE4m3;
    p.e.in_gate = operand(&kept->gate8);
    p.e.in_up = operand(&kept->up8);
    l.quantize(dt, t, dim, x->data, x->ld, operand(&kept->x8));
  }
  l.copies(c.in, c.ins);
  if (d->keep != MUON_KEEP_8BIT || products_tc_take(&p, 1)) {
    l.product(p);
  } else {                       // on CUDA cores a tile does not hold a block's columns: g and u wait in fp32, some rows at a time
    for (int64_t r = 0; r < t && l.rc == MUON_OK; r += kUnalignedRows) {
      const int64_t n = t - r < kUnalignedRows ? t - r : kUnalignedRows;
      Product q = p;
      q.m = int32_t(n);
      q.a[0].data = static_cast<const char*>(ox.data) + r * ox.ld * int64_t(e);
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
  l.product(plain(t, dim, hidden, operand(w.h, w.ldh, dt), down, oy.data, oy.ld, dt), kBeforeLeavesB);
  l.copies(c.out, c.outs);
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
  const muon_feed_forward_kept_t nothing = {};
  if (t == 0) kept = &nothing;   // no tokens: the products below have no k, and what has rows of tokens may be NULL
  if (!dy) dy = &none;
  if (!x) x = &none;
  const bool weights = dw_gate || dw_up || dw_down, by_x = dw_gate || dw_up;
  Copies c;
  auto turned = [](Operand o) {
    o.mn_major = 1;
    return o;
  };
  const Operand ody = c.take(operand(dy, dt), t, dim, w.dy), down = c.take(operand(w_down, dt, true), dim, hidden, w.w_down);
  Operand gate = operand(&kept->gate8), up = operand(&kept->up8), ox = operand(w.x, w.ldx, dt);
  if (given_x) {
    gate = c.take(operand(&kept->gate, dt), t, hidden, w.gate);
    up = c.take(operand(&kept->up, dt), t, hidden, w.up);
    ox = by_x ? c.take(operand(x, dt), t, dim, w.given_x) : operand(x, dt);
  }
  muon_rows_t odx = none, odg = none, odu = none, odd = none;
  Operand by_gate = {}, by_up = {};
  if (dx) {
    by_gate = c.take(operand(w_gate, dt, true), hidden, dim, w.w_gate);
    by_up = c.take(operand(w_up, dt, true), hidden, dim, w.w_up);
    odx = c.give(dx, t, dim, w.dx, dt);
  }
  if (dw_gate) odg = c.give(dw_gate, hidden, dim, w.dw_gate, dt);
  if (dw_up) odu = c.give(dw_up, hidden, dim, w.dw_up, dt);
  if (dw_down) odd = c.give(dw_down, dim, hidden, w.dw_down, dt);
  if (t > 0) {
    l.copies(c.in, c.ins);
    Product p = plain(t, hidden, dim, ody, down, w.h, w.ldh, dt);
    p.e.kind = kGrad;
    p.e.activation = d->activation;
    p.e.gate = w.dgate;
    p.e.up = w.dup;
    p.e.ld_gate = p.e.ld_up = w.ldh;
    p.e.in_gate = gate;
    p.e.in_up = up;
    p.e.gate_up_type = gate.type;
    l.product(p);
  }
  if (dx && t > 0) {
    Product p = plain(t, dim, hidden, operand(w.dgate, w.ldh, dt), by_gate, odx.data, odx.ld, dt);
    p.segments = 2;
    p.a[1] = operand(w.dup, w.ldh, dt);
    p.b[1] = by_up;
    l.product(p, kBeforeLeavesB);
  }
  if (weights) {
    if (!given_x && by_x && t > 0) l.dequantize(dt, t, dim, operand(&kept->x8), w.x, w.ldx);
    Product list[kMaxProducts];
    int n = 0;
    if (dw_gate) list[n++] = with(plain(hidden, dim, t, operand(w.dgate, w.ldh, dt, true), turned(ox), odg.data, odg.ld, dt), w.sum_gate);
    if (dw_up) list[n++] = with(plain(hidden, dim, t, operand(w.dup, w.ldh, dt, true), turned(ox), odu.data, odu.ld, dt), w.sum_up);
    if (dw_down) list[n++] = with(plain(dim, hidden, t, turned(ody), operand(w.h, w.ldh, dt, true), odd.data, odd.ld, dt), w.sum_down);
    l.products(list, n, kMaxProducts, t > 0 ? kBeforeSameCall : kBeforeAny);
  }
  l.copies(c.out, c.outs);
  return l.rc;
}

int muon_linear_blocks_forward(muon_ctx_t* ctx, const muon_linear_blocks_desc_t* d, const muon_rows_t* x, const muon_blocks_t* w8, const muon_rows_t* y,
                             const muon_blocks_t* x8, void* workspace, size_t workspace_bytes, void* stream) {
  if (!ctx) return MUON_ERR_INVALID_ARG;
  int rc = check_linear(d);
  if (rc != MUON_OK) return rc;
  if (d->tokens == 0) return MUON_OK;
  const int64_t t = d->tokens, dim = d->dim, out = d->out;
  if (!good_rows(x, t, dim, 2) || !good_rows(y, t, out, 2) || !good_blocks(w8, out, dim, kBlock) || !good_blocks(x8, t, dim, 1)) return MUON_ERR_INVALID_ARG;
  Scratch s = {static_cast<char*>(workspace)};
  const LinearScratch w = linear_scratch(d, false, &s);
  if ((rc = check_scratch(workspace, workspace_bytes, s.used)) != MUON_OK) return rc;
  if (results_clash({rows_box(y, t, out, 2), codes_box(*x8, t, dim), scales_box(*x8, t, dim), run_of(workspace, int64_t(s.used))},
                    {rows_box(x, t, dim, 2), codes_box(*w8, out, dim), scales_box(*w8, out, dim)}))
    return MUON_ERR_INVALID_ARG;
  Launches l = {ctx, 0, static_cast<cudaStream_t>(stream)};
  if ((rc = device_of(ctx, &l.sms)) != MUON_OK) return rc;
  Copies c;
  const Operand ow = c.take(operand(w8), out, dim, w.w8);
  const muon_rows_t oy = c.give(y, t, out, w.y, kTypeBf16);
  l.copies(c.in, c.ins);
  l.quantize(kTypeBf16, t, dim, x->data, x->ld, operand(x8));
  l.product(plain(t, out, dim, operand(x8), ow, oy.data, oy.ld, kTypeBf16), kBeforeLeavesB);
  l.copies(c.out, c.outs);
  return l.rc;
}

int muon_linear_blocks_workspace_bytes(const muon_linear_blocks_desc_t* desc, int32_t backward, size_t* bytes) {
  if (!bytes || (backward != 0 && backward != 1)) return MUON_ERR_INVALID_ARG;
  const int rc = check_linear(desc);
  if (rc != MUON_OK) return rc;
  Scratch s = {nullptr};
  linear_scratch(desc, backward == 1, &s);
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
  const LinearScratch w = linear_scratch(d, true, &s);
  if ((rc = check_scratch(workspace, workspace_bytes, s.used)) != MUON_OK) return rc;
  const Box nothing = run_of(nullptr, 0);
  const bool rx = dw && t > 0, rw = dx && t > 0;
  if (results_clash({rows_box(dx, t, dim, 2), rows_box(dw, out, dim, 2), run_of(workspace, int64_t(s.used))},
                    {rows_box(dy, t, out, 2), rx ? codes_box(*x8, t, dim) : nothing, rx ? scales_box(*x8, t, dim) : nothing,
                     rw ? codes_box(*w8, out, dim) : nothing, rw ? scales_box(*w8, out, dim) : nothing}))
    return MUON_ERR_INVALID_ARG;
  Launches l = {ctx, 0, static_cast<cudaStream_t>(stream)};
  if ((rc = device_of(ctx, &l.sms)) != MUON_OK) return rc;
  const muon_rows_t none = {nullptr, out};
  if (t == 0) dy = &none;
  Copies c;
  const Operand ody = dw ? c.take(operand(dy, kTypeBf16, true), t, out, w.dy) : operand(dy, kTypeBf16, true);
  Operand ow = {};
  muon_rows_t odx = none, odw = none;
  if (rw) {
    ow = c.take(operand(w8, true), out, dim, w.w8);
    odx = c.give(dx, t, dim, w.dx, kTypeBf16);
  }
  if (dw) odw = c.give(dw, out, dim, w.dw, kTypeBf16);
  if (t > 0) l.copies(c.in, c.ins);
  if (rw) {
    l.quantize(kTypeBf16, t, out, dy->data, dy->ld, operand(&w.dy8));
    l.product(plain(t, dim, out, operand(&w.dy8), ow, odx.data, odx.ld, kTypeBf16), kBeforeLeavesB);
  }
  if (dw) {
    if (rx) l.dequantize(kTypeBf16, t, dim, operand(x8), w.x, w.ldx);
    l.product(with(plain(out, dim, t, ody, operand(w.x, w.ldx, kTypeBf16, true), odw.data, odw.ld, kTypeBf16), w.sum),
              rx ? kBeforeSameCall : kBeforeAny);
  }
  l.copies(c.out, c.outs);
  return l.rc;
}

}  // extern "C"
