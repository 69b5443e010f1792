// Python module `_front`: the torch front end of the layer operators.  Checks of tensors, allocation of results and marshalling into the C ABI;
// no arithmetic.  It stands in C++ because a small call's time is the host's: the same checks in Python cost 14 to 18 us per call, of which
// the device needed 5.
//
// Every host thread has a context of its own per device (autograd calls backward passes from another thread); they share one status word.
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <pybind11/numpy.h>
#include <torch/extension.h>

#include <algorithm>
#include <cmath>
#include <mutex>
#include <optional>
#include <string>
#include <tuple>
#include <utility>
#include <vector>

#include "../../include/muon_b200.h"

namespace py = pybind11;
using at::Tensor;
using MaybeTensor = std::optional<Tensor>;

namespace {

// A thread that ends leaves its contexts to the next one.  Nothing here is ever destroyed: threads (autograd's among them) end while the
// process exits too, when CUDA may be gone already and a call into it would crash.
struct Contexts {
  struct Pool {
    std::mutex lock;
    std::vector<std::pair<int, muon_ctx_t*>> free;
    std::vector<int32_t*> word;                // per device: the status word that all its contexts share
  };
  static Pool& pool() {
    static Pool* p = new Pool;
    return *p;
  }
  std::vector<muon_ctx_t*> of;
  muon_ctx_t* take(int index) {
    std::lock_guard<std::mutex> hold(pool().lock);
    for (auto& f : pool().free)
      if (f.first == index) {
        muon_ctx_t* c = f.second;
        f = pool().free.back();
        pool().free.pop_back();
        return c;
      }
    return nullptr;
  }
  // A bounded wait that expires is seen from every thread: autograd's backward passes run in threads that nobody can ask.
  static int share(int index, muon_ctx_t* c) {
    std::lock_guard<std::mutex> hold(pool().lock);
    std::vector<int32_t*>& word = pool().word;
    if (index >= int(word.size())) word.resize(size_t(index) + 1, nullptr);
    return word[size_t(index)] ? muon_share_device_status(c, word[size_t(index)]) : muon_device_status_word(c, &word[size_t(index)]);
  }
  ~Contexts() {
    std::lock_guard<std::mutex> hold(pool().lock);
    for (size_t i = 0; i < of.size(); ++i)
      if (of[i]) pool().free.push_back({int(i), of[i]});
  }
};

py::object* g_refused = nullptr;  // refused(code, function): raises the package's error

void check(int code, const char* where) {
  if (code == MUON_OK) return;
  py::gil_scoped_acquire gil;
  (*g_refused)(code, where);
}

// The calling thread's context of a device, which is the current one.
muon_ctx_t* context(int index) {
  thread_local Contexts mine;
  if (index >= int(mine.of.size())) mine.of.resize(size_t(index) + 1, nullptr);
  muon_ctx_t*& c = mine.of[size_t(index)];
  if (!c) c = mine.take(index);
  if (!c) {
    muon_options_t opt;
    muon_default_options(&opt);
    check(muon_create(&c, &opt), "muon_create");
    check(Contexts::share(index, c), "muon_share_device_status");
  }
  return c;
}

[[noreturn]] void bad(const std::string& what) { throw py::value_error(what); }

std::string shape_text(const Tensor& t) {
  std::string s = "(";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + ")";
}

int dtype_of(const Tensor& t, const char* what) {
  if (t.scalar_type() == at::kBFloat16) return MUON_DTYPE_BF16;
  if (t.scalar_type() == at::kFloat) return MUON_DTYPE_FP32;
  bad(std::string(what) + " must be bf16 or fp32, not " + c10::toString(t.scalar_type()));
}

// The device that all the tensors are on.
int index_of(const Tensor& t) {
  if (!t.is_cuda()) bad("the layer operators take CUDA tensors (there is no CPU fallback)");
  return t.get_device();
}
void same_device(const Tensor& t, int index) {
  if (!t.is_cuda() || t.get_device() != index) bad("tensors on " + t.device().str() + " and cuda:" + std::to_string(index) + " in one call");
}
void same_device(const MaybeTensor& t, int index) {
  if (t) same_device(*t, index);
}

void* address(const MaybeTensor& t) { return t ? t->data_ptr() : nullptr; }
void* stream_of(int index) { return c10::cuda::getCurrentCUDAStream(c10::DeviceIndex(index)).stream(); }

int32_t narrow(int64_t v) {
  if (v > INT32_MAX) bad("a size of " + std::to_string(v) + " is too large");
  return int32_t(v);
}

Tensor new_like(const Tensor& t) { return at::empty(t.sizes(), t.options()); }
Tensor new_floats(const Tensor& t, at::IntArrayRef sizes) { return at::empty(sizes, t.options().dtype(at::kFloat)); }

// ------------------------------------------------------------------ layer norm
// [..., cols] as [rows, cols] with contiguous rows: a view where the strides allow one, else a copy.
Tensor rows_of(const Tensor& t, const char* what) {
  if (t.dim() < 1 || t.size(-1) < 1) bad(std::string(what) + " needs a last dimension of at least one element");
  Tensor r = t.dim() == 2 ? t : t.reshape({-1, t.size(-1)});
  const bool fits = (r.size(1) == 1 || r.stride(1) == 1) && (r.size(0) <= 1 || r.stride(0) >= r.size(1));
  return fits ? r : r.contiguous();
}
int64_t row_stride(const Tensor& r) { return r.size(0) > 1 ? std::max(r.stride(0), r.size(1)) : r.size(1); }

MaybeTensor param(const MaybeTensor& p, int64_t cols, const char* what) {
  if (!p) return p;
  if (p->dim() != 1 || p->size(0) != cols) bad(std::string(what) + " must have shape (" + std::to_string(cols) + ",), not " + shape_text(*p));
  return p->is_contiguous() ? p : MaybeTensor(p->contiguous());
}

std::tuple<Tensor, MaybeTensor, Tensor> layer_norm_forward(const Tensor& x, const MaybeTensor& weight_, const MaybeTensor& bias_, double eps, bool center) {
  const int index = index_of(x);
  same_device(weight_, index);
  same_device(bias_, index);
  c10::cuda::OptionalCUDAGuard guard(x.device());
  const Tensor r = rows_of(x, "x");
  const int64_t cols = r.size(1);
  const MaybeTensor weight = param(weight_, cols, "weight"), bias = param(bias_, cols, "bias");
  if (weight && bias && weight->scalar_type() != bias->scalar_type()) bad("weight and bias must have one dtype");
  muon_norm_desc_t d = {};
  d.dtype = dtype_of(x, "x");
  d.param_dtype = weight || bias ? dtype_of(weight ? *weight : *bias, "weight and bias") : MUON_DTYPE_FP32;
  d.center = center;
  d.cols = narrow(cols);
  d.rows = r.size(0);
  d.eps = float(eps);
  const at::IntArrayRef stat = x.sizes().slice(0, size_t(x.dim() - 1));
  Tensor y = new_like(x), rstd = new_floats(x, stat);
  MaybeTensor mean;
  if (center) mean = new_floats(x, stat);
  check(muon_layer_norm_forward(context(index), &d, r.data_ptr(), row_stride(r), address(weight), address(bias), y.data_ptr(), cols,
                                static_cast<float*>(address(mean)), static_cast<float*>(rstd.data_ptr()), stream_of(index)),
        "muon_layer_norm_forward");
  return {y, mean, rstd};
}

std::tuple<Tensor, MaybeTensor, MaybeTensor> layer_norm_backward(const Tensor& dy, const Tensor& x, const MaybeTensor& weight_, const MaybeTensor& mean_,
                                                                 const Tensor& rstd_, bool bias, std::optional<at::ScalarType> bias_dtype) {
  const int index = index_of(x);
  for (const Tensor* t : {&dy, &rstd_}) same_device(*t, index);
  same_device(weight_, index);
  same_device(mean_, index);
  c10::cuda::OptionalCUDAGuard guard(x.device());
  if (!dy.sizes().equals(x.sizes()) || dy.scalar_type() != x.scalar_type()) bad("dy must have the shape and dtype of x");
  const Tensor r = rows_of(x, "x"), g = rows_of(dy, "dy");
  const int64_t cols = r.size(1);
  const at::IntArrayRef stat = x.sizes().slice(0, size_t(x.dim() - 1));
  if (!rstd_.sizes().equals(stat) || (mean_ && !mean_->sizes().equals(stat))) bad("mean and rstd must have the shape of x without its last dimension");
  if (rstd_.scalar_type() != at::kFloat || (mean_ && mean_->scalar_type() != at::kFloat)) bad("mean and rstd must be fp32");
  const MaybeTensor weight = param(weight_, cols, "weight");
  const Tensor rstd = rstd_.contiguous();
  MaybeTensor mean;
  if (mean_) mean = mean_->contiguous();
  muon_norm_desc_t d = {};
  d.dtype = dtype_of(x, "x");
  const at::ScalarType pt = weight ? weight->scalar_type() : bias_dtype.value_or(at::kFloat);
  if (pt != at::kFloat && pt != at::kBFloat16) bad(std::string("gradients must be bf16 or fp32, not ") + c10::toString(pt));
  d.param_dtype = pt == at::kFloat ? MUON_DTYPE_FP32 : MUON_DTYPE_BF16;
  d.center = mean.has_value();
  d.cols = narrow(cols);
  d.rows = r.size(0);
  Tensor dx = new_like(x);
  MaybeTensor dw, db, ws;
  if (weight) dw = new_like(*weight);
  if (bias) db = at::empty({cols}, x.options().dtype(pt));
  size_t n = 0;
  if (dw || db) check(muon_layer_norm_workspace_bytes(&d, &n), "muon_layer_norm_workspace_bytes");
  if (n) ws = at::empty({int64_t(n)}, x.options().dtype(at::kByte));
  check(muon_layer_norm_backward(context(index), &d, g.data_ptr(), row_stride(g), r.data_ptr(), row_stride(r), address(weight),
                                 static_cast<const float*>(address(mean)), static_cast<const float*>(rstd.data_ptr()), dx.data_ptr(), cols, address(dw),
                                 address(db), address(ws), n, stream_of(index)),
        "muon_layer_norm_backward");
  return {dx, dw, db};
}

// ------------------------------------------------------------------ strided [batch, tokens, heads, dim] tensors
// With a contiguous last dimension (a copy only where it is not); [tokens, heads, dim] has a batch of one.
Tensor heads_of(const Tensor& t, const char* what) {
  if (t.dim() != 3 && t.dim() != 4) bad(std::string(what) + " must be [batch, tokens, heads, dim] or [tokens, heads, dim]");
  return t.stride(-1) == 1 || t.size(-1) == 1 ? t : t.contiguous();
}
muon_heads_t describe(const Tensor& t) { return {t.data_ptr(), t.dim() == 4 ? t.stride(0) : 0, t.stride(-3), t.stride(-2)}; }
int64_t batch_of(const Tensor& t) { return t.dim() == 4 ? t.size(0) : 1; }

// ------------------------------------------------------------------ rotary positions
using Frequencies = py::array_t<double, py::array::c_style | py::array::forcecast>;

std::vector<Tensor> rotary(const std::vector<Tensor>& tensors, const Frequencies& inv_freq,
                           const std::string& layout, double amplitude, const MaybeTensor& positions_, int64_t offset, bool inverse,
                           const std::optional<std::vector<Tensor>>& out) {
  if (tensors.empty() || tensors.size() > 4) bad("one to four tensors");
  const bool interleaved = layout == "interleaved";
  if (!interleaved && layout != "half") bad("layout is 'half' or 'interleaved'");
  const Tensor& first = tensors[0];
  const int index = index_of(first);
  for (const Tensor& t : tensors) same_device(t, index);
  same_device(positions_, index);
  c10::cuda::OptionalCUDAGuard guard(first.device());
  muon_rotary_desc_t d = {};
  muon_rotary_item_t items[4] = {};
  std::vector<Tensor> keep, result;
  if (out && out->size() != tensors.size()) bad("out must match the tensors");
  for (size_t i = 0; i < tensors.size(); ++i) {
    const Tensor& t = tensors[i];
    keep.push_back(heads_of(t, "a tensor"));
    const Tensor& x = keep.back();
    if (batch_of(x) != batch_of(keep[0]) || x.size(-3) != keep[0].size(-3) || x.size(-1) != keep[0].size(-1) || t.scalar_type() != first.scalar_type())
      bad("the tensors must agree in batch, tokens, head size and dtype");
    if (out) {
      const Tensor& o = (*out)[i];
      if (!o.sizes().equals(t.sizes()) || o.scalar_type() != t.scalar_type() || o.device() != t.device()) bad("out must match the tensors");
      if (o.stride(-1) != 1 && o.size(-1) > 1) bad("out must have a contiguous last dimension");
      if (o.requires_grad() && at::GradMode::is_enabled()) bad("out requires grad, and what is written there is not recorded: use rotary, or no_grad");
      result.push_back(o);
    } else {
      result.push_back(new_like(t));
    }
    items[i].in = describe(x);
    items[i].out = describe(result.back());
    items[i].heads = narrow(x.size(-2));
  }
  const int64_t b = batch_of(keep[0]), n = keep[0].size(-3), dim = keep[0].size(-1), pairs = inv_freq.size();
  if (inv_freq.ndim() != 1 || pairs < 1 || pairs > dim / 2)
    bad("inv_freq must hold one to " + std::to_string(dim / 2) + " frequencies for heads of " + std::to_string(dim));
  MaybeTensor positions;
  if (positions_) {
    if (positions_->scalar_type() != at::kInt || positions_->numel() != b * n) bad("positions must be int32, one for each token");
    positions = positions_->contiguous();
  }
  d.dtype = dtype_of(first, "the tensors");
  d.interleaved = interleaved;
  d.inverse = inverse;
  d.head_dim = narrow(dim);
  d.rotary_dim = narrow(2 * pairs);
  d.batch = narrow(b);
  d.tokens = narrow(n);
  d.amplitude = float(amplitude);
  d.inv_freq = inv_freq.data();
  d.positions = static_cast<const int32_t*>(address(positions));
  d.position_offset = offset;
  check(muon_rotary(context(index), &d, items, int32_t(tensors.size()), stream_of(index)), "muon_rotary");
  if (out)                                             // what another operation saved of them is not there any more: autograd must know
    for (const Tensor& o : result)
      if (!o.is_inference()) o.unsafeGetTensorImpl()->bump_version();
  return result;
}

// ------------------------------------------------------------------ attention
struct AttentionCall {
  int index;
  muon_attention_desc_t d = {};
  Tensor q, k, v;                                     // with contiguous heads
  MaybeTensor q_lens, k_lens, q_offsets, k_offsets;   // what the descriptor points into
  std::vector<int64_t> stat;                          // shape of lse
};

MaybeTensor table(const MaybeTensor& t, int64_t n, const char* what) {
  if (!t) return t;
  if (t->scalar_type() != at::kInt || t->dim() != 1 || t->numel() != n) bad(std::string(what) + " must be a 1-D int32 tensor of " + std::to_string(n));
  return t->contiguous();
}

AttentionCall attention_call(const Tensor& q, const Tensor& k, const Tensor& v, bool causal, int64_t window, std::optional<double> scale,
                             const MaybeTensor& q_lens, const MaybeTensor& k_lens, const MaybeTensor& q_offsets, const MaybeTensor& k_offsets) {
  AttentionCall c;
  c.index = index_of(q);
  same_device(k, c.index);
  same_device(v, c.index);
  for (const MaybeTensor* t : {&q_lens, &k_lens, &q_offsets, &k_offsets}) same_device(*t, c.index);
  const bool packed = q_offsets || k_offsets;
  const int64_t dims = packed ? 3 : 4;
  if (q.dim() != dims || k.dim() != dims || v.dim() != dims) bad("q, k, v are [batch, tokens, heads, dim], or [tokens, heads, dim] with offsets");
  if (q.scalar_type() != k.scalar_type() || q.scalar_type() != v.scalar_type()) bad("q, k and v must have one dtype");
  const int64_t b = batch_of(q), nq = q.size(-3), hq = q.size(-2), dim = q.size(-1), nk = k.size(-3), hkv = k.size(-2);
  if (!k.sizes().equals(v.sizes()) || k.size(-1) != dim || batch_of(k) != b)
    bad("shapes do not fit: q " + shape_text(q) + ", k " + shape_text(k) + ", v " + shape_text(v));
  if (hkv < 1 || hq < 1 || hq % hkv) bad(std::to_string(hq) + " query heads cannot share " + std::to_string(hkv) + " key heads evenly");
  int64_t nseq = 0;
  if (packed) {
    if (!q_offsets || !k_offsets || q_lens || k_lens) bad("packed sequences take q_offsets and k_offsets, and no lengths");
    nseq = q_offsets->numel() - 1;
    if (nseq < 1) bad("offsets need at least two entries");
    c.q_offsets = table(q_offsets, nseq + 1, "q_offsets");
    c.k_offsets = table(k_offsets, nseq + 1, "k_offsets");
  }
  c.q_lens = table(q_lens, b, "q_lens");
  c.k_lens = table(k_lens, b, "k_lens");
  c.q = heads_of(q, "q");
  c.k = heads_of(k, "k");
  c.v = heads_of(v, "v");
  muon_attention_desc_t& d = c.d;
  d.dtype = dtype_of(q, "q, k and v");
  d.batch = narrow(b);
  d.q_tokens = narrow(nq);
  d.k_tokens = narrow(nk);
  d.q_heads = narrow(hq);
  d.kv_heads = narrow(hkv);
  d.head_dim = narrow(dim);
  d.causal = causal;
  d.window = window < INT32_MIN ? INT32_MIN : window > INT32_MAX ? INT32_MAX : int32_t(window);
  d.scale = float(scale ? *scale : dim > 0 ? 1.0 / std::sqrt(double(dim)) : 1.0);
  d.num_seqs = narrow(nseq);
  d.q_lens = static_cast<const int32_t*>(address(c.q_lens));
  d.k_lens = static_cast<const int32_t*>(address(c.k_lens));
  d.q_offsets = static_cast<const int32_t*>(address(c.q_offsets));
  d.k_offsets = static_cast<const int32_t*>(address(c.k_offsets));
  if (packed) c.stat = {hq, nq};
  else c.stat = {b, hq, nq};
  return c;
}

std::tuple<Tensor, Tensor> attention_forward(const Tensor& q, const Tensor& k, const Tensor& v, bool causal, int64_t window, std::optional<double> scale,
                                             const MaybeTensor& q_lens, const MaybeTensor& k_lens, const MaybeTensor& q_offsets,
                                             const MaybeTensor& k_offsets) {
  const AttentionCall c = attention_call(q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets);
  c10::cuda::OptionalCUDAGuard guard(q.device());
  Tensor o = new_like(q), lse = new_floats(q, c.stat);
  const muon_heads_t hq = describe(c.q), hk = describe(c.k), hv = describe(c.v), ho = describe(o);
  check(muon_attention_forward(context(c.index), &c.d, &hq, &hk, &hv, &ho, static_cast<float*>(lse.data_ptr()), stream_of(c.index)),
        "muon_attention_forward");
  return {o, lse};
}

std::tuple<Tensor, Tensor, Tensor> attention_backward(const Tensor& dout, const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& o,
                                                      const Tensor& lse_, bool causal, int64_t window, std::optional<double> scale,
                                                      const MaybeTensor& q_lens, const MaybeTensor& k_lens, const MaybeTensor& q_offsets,
                                                      const MaybeTensor& k_offsets) {
  const AttentionCall c = attention_call(q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets);
  for (const Tensor* t : {&dout, &o, &lse_}) same_device(*t, c.index);
  if (!dout.sizes().equals(q.sizes()) || !o.sizes().equals(q.sizes()) || dout.scalar_type() != q.scalar_type() || o.scalar_type() != q.scalar_type())
    bad("do and o must have the shape and dtype of q");
  if (!lse_.sizes().equals(c.stat) || lse_.scalar_type() != at::kFloat) bad("lse must be fp32 of shape [(batch,) heads, tokens]");
  c10::cuda::OptionalCUDAGuard guard(q.device());
  const Tensor g = heads_of(dout, "do"), out = heads_of(o, "o"), lse = lse_.contiguous();
  Tensor dq = new_like(q), dk = new_like(k), dv = new_like(v);
  size_t n = 0;
  check(muon_attention_workspace_bytes(&c.d, &n), "muon_attention_workspace_bytes");
  MaybeTensor ws;
  if (n) ws = at::empty({int64_t(n)}, q.options().dtype(at::kByte));
  const muon_heads_t hg = describe(g), hq = describe(c.q), hk = describe(c.k), hv = describe(c.v), ho = describe(out), hdq = describe(dq),
                     hdk = describe(dk), hdv = describe(dv);
  check(muon_attention_backward(context(c.index), &c.d, &hg, &hq, &hk, &hv, &ho, static_cast<const float*>(lse.data_ptr()), &hdq, &hdk, &hdv, address(ws),
                                n, stream_of(c.index)),
        "muon_attention_backward");
  return {dq, dk, dv};
}

// ------------------------------------------------------------------ 8-bit blocks
// Codes [..., cols] with rows 16 bytes apart or a multiple of that, so that the tensor cores can take them, and their scales, whose rows are
// 4 bytes apart or a multiple of 16 where there are more than 8: so they are read fastest.
struct Packed {
  Tensor codes, scales;
};
Tensor new_pitched(at::IntArrayRef sizes, int64_t ld, const at::TensorOptions& options) {
  if (ld == sizes.back()) return at::empty(sizes, options);
  c10::SmallVector<int64_t, 6> strides(sizes.size(), 1);
  int64_t next = ld;
  for (size_t i = sizes.size() - 1; i-- > 0; next *= std::max<int64_t>(sizes[i], 1)) strides[i] = next;
  return at::empty_strided(sizes, strides, options);
}
Packed new_packed(at::IntArrayRef sizes, const at::TensorOptions& options, int64_t block_rows) {
  c10::SmallVector<int64_t, 6> scales(sizes.begin(), sizes.end());
  const int64_t cols = sizes.back(), blocks = (cols + 127) / 128;
  scales.back() = blocks;
  if (block_rows > 1) scales[0] = (scales[0] + block_rows - 1) / block_rows;
  return {new_pitched(sizes, (cols + 15) / 16 * 16, options.dtype(at::kFloat8_e4m3fn)),
          new_pitched(scales, blocks > 8 ? (blocks + 15) / 16 * 16 : (blocks + 3) / 4 * 4, options.dtype(at::kByte))};
}

// A packed matrix as the C ABI takes it, and the tensors that keep its memory.
struct PackedView {
  Tensor codes, scales;
  int64_t rows, cols;
  muon_blocks_t b = {};
};
PackedView packed(const Tensor& codes, const Tensor& scales, int64_t block_rows, const char* what) {
  PackedView v;
  if (codes.scalar_type() != at::kFloat8_e4m3fn) bad(std::string(what) + " must have codes of float8_e4m3fn, not " + c10::toString(codes.scalar_type()));
  if (scales.scalar_type() != at::kByte) bad(std::string(what) + " must have scales of uint8, not " + c10::toString(scales.scalar_type()));
  v.codes = rows_of(codes, what);
  v.rows = v.codes.size(0);
  v.cols = v.codes.size(1);
  c10::SmallVector<int64_t, 6> each(codes.sizes().begin(), codes.sizes().end());
  each.back() = (v.cols + 127) / 128;
  const bool rows = scales.sizes().equals(at::IntArrayRef(each));
  const bool squares = codes.dim() == 2 && scales.dim() == 2 && scales.size(0) == (v.rows + 127) / 128 && scales.size(1) == each.back();
  if (block_rows == 0) block_rows = rows ? 1 : 128;     // one row alone: both are the same
  if (!(block_rows == 1 ? rows : squares))
    bad(std::string(what) + " has codes " + shape_text(codes) + " and scales " + shape_text(scales) + ", which do not fit blocks of " +
        std::to_string(block_rows) + " x 128");
  v.scales = rows_of(scales, what);
  v.b.codes = v.codes.data_ptr();
  v.b.ld = v.rows > 1 ? row_stride(v.codes) : (v.cols + 15) / 16 * 16;
  v.b.scales = static_cast<uint8_t*>(v.scales.data_ptr());
  v.b.lds = row_stride(v.scales);
  v.b.block_rows = int32_t(block_rows);
  return v;
}

// One row alone has no distance to a next one, and gets one that the tensor cores take.
muon_rows_t rows_view(const Tensor& r) { return {r.data_ptr(), r.size(0) > 1 ? row_stride(r) : (r.size(1) + 7) / 8 * 8}; }
const muon_rows_t* maybe(const MaybeTensor& t, muon_rows_t* v) {
  if (!t) return nullptr;
  *v = rows_view(*t);
  return v;
}
MaybeTensor new_scratch(size_t bytes, const Tensor& like) {
  return bytes ? MaybeTensor(at::empty({int64_t(bytes)}, like.options().dtype(at::kByte))) : MaybeTensor();
}

std::tuple<Tensor, Tensor> quantize(const Tensor& x, int64_t block_rows) {
  const int index = index_of(x);
  if (block_rows != 1 && block_rows != 128) bad("block_rows is 1 or 128");
  if (block_rows == 128 && x.dim() != 2) bad("blocks of 128 x 128 take a matrix");
  c10::cuda::OptionalCUDAGuard guard(x.device());
  const int dtype = dtype_of(x, "x");
  const Tensor r = rows_of(x, "x");
  const Packed out = new_packed(x.sizes(), x.options(), block_rows);
  const PackedView v = packed(out.codes, out.scales, block_rows, "the result");
  const muon_rows_t in = rows_view(r);
  check(muon_quantize(context(index), dtype, r.size(0), r.size(1), &in, &v.b, stream_of(index)), "muon_quantize");
  return {out.codes, out.scales};
}

Tensor dequantize(const Tensor& codes, const Tensor& scales, at::ScalarType dtype) {
  const int index = index_of(codes);
  same_device(scales, index);
  if (dtype != at::kBFloat16 && dtype != at::kFloat) bad(std::string("dtype must be bf16 or fp32, not ") + c10::toString(dtype));
  c10::cuda::OptionalCUDAGuard guard(codes.device());
  const PackedView v = packed(codes, scales, 0, "the input");
  Tensor y = at::empty(codes.sizes(), codes.options().dtype(dtype));
  const muon_rows_t out = {y.data_ptr(), v.cols};
  check(muon_dequantize(context(index), dtype_of(y, "y"), v.rows, v.cols, &v.b, &out, stream_of(index)), "muon_dequantize");
  return y;
}

// ------------------------------------------------------------------ gated feed-forward block
struct FeedForwardCall {
  int index;
  muon_feed_forward_desc_t d = {};
  Tensor gate, up, down;                               // the weights, with contiguous rows
  std::vector<int64_t> hidden_shape;                   // of g and u
  muon_rows_t w[3];
};
// `x`: x, or dy of the same shape.
FeedForwardCall feed_forward_call(const Tensor& x, const char* name, const Tensor& w_gate, const Tensor& w_up, const Tensor& w_down,
                                  const std::string& activation) {
  FeedForwardCall c;
  c.index = index_of(x);
  for (const Tensor* w : {&w_gate, &w_up, &w_down}) same_device(*w, c.index);
  if (activation != "silu" && activation != "gelu") bad("activation is 'silu' or 'gelu'");
  if (x.dim() < 1 || w_gate.dim() != 2 || !w_up.sizes().equals(w_gate.sizes()) || w_down.dim() != 2 || w_down.size(0) != w_gate.size(1) ||
      w_down.size(1) != w_gate.size(0) || x.size(-1) != w_gate.size(1) || w_gate.numel() == 0)
    bad("shapes do not fit: " + std::string(name) + " " + shape_text(x) + ", w_gate " + shape_text(w_gate) + ", w_up " + shape_text(w_up) + ", w_down " +
        shape_text(w_down));
  for (const Tensor* w : {&w_gate, &w_up, &w_down})
    if (w->scalar_type() != x.scalar_type()) bad(std::string(name) + " and the weights must have one dtype");
  c.d.dtype = dtype_of(x, name);
  c.d.activation = activation == "silu" ? MUON_ACTIVATION_SILU : MUON_ACTIVATION_GELU;
  c.d.dim = narrow(w_gate.size(1));
  c.d.hidden = narrow(w_gate.size(0));
  c.d.tokens = narrow(x.numel() / c.d.dim);
  c.hidden_shape.assign(x.sizes().begin(), x.sizes().end());
  c.hidden_shape.back() = c.d.hidden;
  return c;
}
// After the device is set: copies of weights whose rows are not contiguous.
void lay_out(FeedForwardCall& c, const Tensor& w_gate, const Tensor& w_up, const Tensor& w_down) {
  c.gate = rows_of(w_gate, "w_gate");
  c.up = rows_of(w_up, "w_up");
  c.down = rows_of(w_down, "w_down");
  c.w[0] = rows_view(c.gate);
  c.w[1] = rows_view(c.up);
  c.w[2] = rows_view(c.down);
}

std::tuple<Tensor, std::vector<Tensor>> feed_forward_forward(const Tensor& x, const Tensor& w_gate, const Tensor& w_up, const Tensor& w_down,
                                                             const std::string& activation, const std::string& checkpoint) {
  FeedForwardCall c = feed_forward_call(x, "x", w_gate, w_up, w_down, activation);
  if (checkpoint != "full" && checkpoint != "8bit" && checkpoint != "none") bad("checkpoint is 'full', '8bit' or 'none'");
  c10::cuda::OptionalCUDAGuard guard(x.device());
  lay_out(c, w_gate, w_up, w_down);
  c.d.keep = checkpoint == "full" ? MUON_KEEP_FULL : checkpoint == "8bit" ? MUON_KEEP_8BIT : MUON_KEEP_NONE;
  const Tensor r = rows_of(x, "x");
  Tensor y = new_like(x);
  std::vector<Tensor> kept;
  std::vector<PackedView> views;
  muon_feed_forward_kept_t k = {};
  if (c.d.keep == MUON_KEEP_FULL) {
    for (muon_rows_t* t : {&k.gate, &k.up}) {
      const int64_t ld = (int64_t(c.d.hidden) + 7) / 8 * 8;
      kept.push_back(new_pitched(c.hidden_shape, ld, x.options()));
      *t = {kept.back().data_ptr(), ld};
    }
  } else if (c.d.keep == MUON_KEEP_8BIT) {
    for (muon_blocks_t* t : {&k.x8, &k.gate8, &k.up8}) {
      const Packed p = new_packed(t == &k.x8 ? x.sizes() : at::IntArrayRef(c.hidden_shape), x.options(), 1);
      kept.push_back(p.codes);
      kept.push_back(p.scales);
      views.push_back(packed(p.codes, p.scales, 1, "the result"));
      *t = views.back().b;
    }
  }
  size_t n = 0;
  check(muon_feed_forward_workspace_bytes(&c.d, 0, &n), "muon_feed_forward_workspace_bytes");
  const MaybeTensor ws = new_scratch(n, x);
  const muon_rows_t in = rows_view(r), out = {y.data_ptr(), c.d.dim};
  check(muon_feed_forward_forward(context(c.index), &c.d, &in, &c.w[0], &c.w[1], &c.w[2], &out, &k, address(ws), n, stream_of(c.index)),
        "muon_feed_forward_forward");
  return {y, kept};
}

std::tuple<MaybeTensor, MaybeTensor, MaybeTensor, MaybeTensor> feed_forward_backward(const Tensor& dy, const MaybeTensor& x, const Tensor& w_gate,
                                                                                     const Tensor& w_up, const Tensor& w_down,
                                                                                     const std::vector<Tensor>& kept, const std::string& activation,
                                                                                     const std::vector<bool>& need) {
  FeedForwardCall c = feed_forward_call(dy, "dy", w_gate, w_up, w_down, activation);
  same_device(x, c.index);
  for (const Tensor& t : kept) same_device(t, c.index);
  if (need.size() != 4) bad("need says of x, w_gate, w_up and w_down whether their gradients are wanted");
  if (kept.size() != 2 && kept.size() != 6) bad("kept is what feed_forward_forward gave: two tensors (checkpoint 'full') or six ('8bit')");
  c10::cuda::OptionalCUDAGuard guard(dy.device());
  lay_out(c, w_gate, w_up, w_down);
  muon_feed_forward_kept_t k = {};
  std::vector<Tensor> hold;
  std::vector<PackedView> views;
  muon_rows_t in_x = {};
  if (kept.size() == 2) {
    c.d.keep = MUON_KEEP_FULL;
    if (!x) bad("x is needed with checkpoint 'full'");
    if (!x->sizes().equals(dy.sizes()) || x->scalar_type() != dy.scalar_type()) bad("x must have the shape and dtype of dy");
    for (const Tensor& t : kept) {
      if (!t.sizes().equals(c.hidden_shape) || t.scalar_type() != dy.scalar_type()) bad("what was kept does not fit dy and the weights");
      hold.push_back(rows_of(t, "kept"));
    }
    k.gate = rows_view(hold[0]);
    k.up = rows_view(hold[1]);
    hold.push_back(rows_of(*x, "x"));
    in_x = rows_view(hold[2]);
  } else {
    c.d.keep = MUON_KEEP_8BIT;
    if (x) bad("x is part of what was kept in 8 bits: give None");
    muon_blocks_t* to[3] = {&k.x8, &k.gate8, &k.up8};
    for (int i = 0; i < 3; ++i) {
      if (!kept[size_t(2 * i)].sizes().equals(i ? at::IntArrayRef(c.hidden_shape) : dy.sizes())) bad("what was kept does not fit dy and the weights");
      views.push_back(packed(kept[size_t(2 * i)], kept[size_t(2 * i + 1)], 1, "kept"));
      *to[i] = views.back().b;
    }
  }
  const Tensor r = rows_of(dy, "dy");
  MaybeTensor dx, dw[3];
  muon_rows_t out[4];
  if (need[0]) dx = new_like(dy);
  for (int i = 0; i < 3; ++i)
    if (need[size_t(i + 1)]) dw[i] = at::empty({i < 2 ? c.d.hidden : c.d.dim, i < 2 ? c.d.dim : c.d.hidden}, dy.options());
  size_t n = 0;
  check(muon_feed_forward_workspace_bytes(&c.d, 1, &n), "muon_feed_forward_workspace_bytes");
  const MaybeTensor ws = new_scratch(n, dy);
  const muon_rows_t in = rows_view(r);
  if (dx) out[0] = {dx->data_ptr(), c.d.dim};
  check(muon_feed_forward_backward(context(c.index), &c.d, &in, kept.size() == 2 ? &in_x : nullptr, &c.w[0], &c.w[1], &c.w[2], &k, dx ? &out[0] : nullptr,
                                   maybe(dw[0], &out[1]), maybe(dw[1], &out[2]), maybe(dw[2], &out[3]), address(ws), n, stream_of(c.index)),
        "muon_feed_forward_backward");
  return {dx, dw[0], dw[1], dw[2]};
}

// ------------------------------------------------------------------ 8-bit linear layer
std::tuple<Tensor, Tensor, Tensor> linear_8bit_forward(const Tensor& x, const Tensor& w_codes, const Tensor& w_scales) {
  const int index = index_of(x);
  same_device(w_codes, index);
  same_device(w_scales, index);
  if (x.scalar_type() != at::kBFloat16) bad(std::string("x must be bf16, not ") + c10::toString(x.scalar_type()));
  if (w_codes.dim() != 2 || x.dim() < 1 || x.size(-1) != w_codes.size(1) || w_codes.numel() == 0)
    bad("shapes do not fit: x " + shape_text(x) + ", weight " + shape_text(w_codes));
  c10::cuda::OptionalCUDAGuard guard(x.device());
  const PackedView w = packed(w_codes, w_scales, 128, "the weight");
  const Tensor r = rows_of(x, "x");
  muon_linear_blocks_desc_t d = {};
  d.tokens = narrow(r.size(0));
  d.dim = narrow(r.size(1));
  d.out = narrow(w.rows);
  std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
  shape.back() = w.rows;
  Tensor y = at::empty(shape, x.options());
  const Packed p = new_packed(x.sizes(), x.options(), 1);
  const PackedView x8 = packed(p.codes, p.scales, 1, "the result");
  const muon_rows_t in = rows_view(r), out = {y.data_ptr(), w.rows};
  size_t n = 0;
  check(muon_linear_blocks_workspace_bytes(&d, 0, &n), "muon_linear_blocks_workspace_bytes");
  const MaybeTensor ws = new_scratch(n, x);
  check(muon_linear_blocks_forward(context(index), &d, &in, &w.b, &out, &x8.b, address(ws), n, stream_of(index)), "muon_linear_blocks_forward");
  return {y, p.codes, p.scales};
}

std::tuple<MaybeTensor, MaybeTensor> linear_8bit_backward(const Tensor& dy, const Tensor& x_codes, const Tensor& x_scales, const Tensor& w_codes,
                                                          const Tensor& w_scales, const std::vector<bool>& need) {
  const int index = index_of(dy);
  for (const Tensor* t : {&x_codes, &x_scales, &w_codes, &w_scales}) same_device(*t, index);
  if (need.size() != 2) bad("need says of x and the weight whether their gradients are wanted");
  if (dy.scalar_type() != at::kBFloat16) bad(std::string("dy must be bf16, not ") + c10::toString(dy.scalar_type()));
  if (w_codes.dim() != 2 || dy.dim() < 1 || dy.dim() != x_codes.dim() || dy.size(-1) != w_codes.size(0) || x_codes.size(-1) != w_codes.size(1) ||
      w_codes.numel() == 0 || !dy.sizes().slice(0, size_t(dy.dim() - 1)).equals(x_codes.sizes().slice(0, size_t(dy.dim() - 1))))
    bad("shapes do not fit: dy " + shape_text(dy) + ", x " + shape_text(x_codes) + ", weight " + shape_text(w_codes));
  c10::cuda::OptionalCUDAGuard guard(dy.device());
  const PackedView w = packed(w_codes, w_scales, 128, "the weight"), x = packed(x_codes, x_scales, 1, "x");
  const Tensor r = rows_of(dy, "dy");
  muon_linear_blocks_desc_t d = {};
  d.tokens = narrow(r.size(0));
  d.dim = narrow(w.cols);
  d.out = narrow(w.rows);
  MaybeTensor dx, dw;
  muon_rows_t out[2] = {};
  if (need[0]) {
    dx = at::empty(x_codes.sizes(), dy.options());
    out[0] = {dx->data_ptr(), w.cols};
  }
  if (need[1]) dw = at::empty({w.rows, w.cols}, dy.options());
  size_t n = 0;
  check(muon_linear_blocks_workspace_bytes(&d, 1, &n), "muon_linear_blocks_workspace_bytes");
  const MaybeTensor ws = new_scratch(n, dy);
  const muon_rows_t in = rows_view(r);
  check(muon_linear_blocks_backward(context(index), &d, &in, &x.b, &w.b, dx ? &out[0] : nullptr, maybe(dw, &out[1]), address(ws), n, stream_of(index)),
        "muon_linear_blocks_backward");
  return {dx, dw};
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
  m.doc() = "Checks and marshalling of paper_2609_21594_b200.functional";
  m.def("set_refused", [](py::object refused) {
    delete g_refused;
    g_refused = new py::object(std::move(refused));
  });
  m.def("context", [](int index) {
    c10::cuda::OptionalCUDAGuard guard(c10::Device(c10::DeviceType::CUDA, c10::DeviceIndex(index)));
    return reinterpret_cast<uintptr_t>(context(index));
  });
  using release = py::call_guard<py::gil_scoped_release>;
  const auto none = py::none();
  m.def("layer_norm_forward", &layer_norm_forward, release(), py::arg("x"), py::arg("weight") = none, py::arg("bias") = none, py::arg("eps") = 1e-5,
        py::arg("center") = true,
        "(y, mean, rstd) over the last dimension; center=False is RMS norm and gives mean = None.  mean, rstd: fp32, x.shape[:-1].");
  m.def("layer_norm_backward", &layer_norm_backward, release(), py::arg("dy"), py::arg("x"), py::arg("weight"), py::arg("mean"), py::arg("rstd"),
        py::arg("bias") = true, py::arg("bias_dtype") = none,
        "(dx, dweight, dbias); dweight is None without a weight, dbias unless `bias`.  The gradients have the weight's dtype (without a weight:\n"
        "bias_dtype, fp32 by default).");
  m.def(
      "rotary_forward",
      [](const std::vector<Tensor>& tensors, const Frequencies& inv_freq, const std::string& layout, double amplitude, const MaybeTensor& positions,
         int64_t offset, bool inverse, const std::optional<std::vector<Tensor>>& out) {
        std::vector<Tensor> r;
        {
          py::gil_scoped_release no_gil;
          r = rotary(tensors, inv_freq, layout, amplitude, positions, offset, inverse, out);
        }
        return py::tuple(py::cast(r));
      },
      py::arg("tensors"), py::arg("inv_freq"), py::arg("layout") = "half", py::arg("amplitude") = 1.0, py::arg("positions") = none, py::arg("offset") = 0,
      py::arg("inverse") = false, py::arg("out") = none,
      "Turns up to four [batch, tokens, heads, dim] (or [tokens, heads, dim]) tensors that share positions, in one launch.\n\n"
      "inv_freq: host, fp64 radians per position of each pair (see `rotary_frequencies`); twice its length is the part of the head that is\n"
      "turned, the rest is copied.  layout: \"half\" (i with i + n/2) or \"interleaved\" (2i with 2i + 1).  positions: int32 [batch, tokens] on\n"
      "the device, else offset + 0, 1, 2...; offset is added to given positions too.  inverse turns back, which is the backward pass.\n"
      "out: tensors to write, which may be the inputs themselves; written in place for autograd too, so none may require grad while it records.");
  m.def("attention_forward", &attention_forward, release(), py::arg("q"), py::arg("k"), py::arg("v"), py::arg("causal") = true, py::arg("window") = 0,
        py::arg("scale") = none, py::arg("q_lens") = none, py::arg("k_lens") = none, py::arg("q_offsets") = none, py::arg("k_offsets") = none,
        "(o, lse).  q: [batch, tokens, heads, dim]; k, v: [batch, tokens, kv heads, dim], heads a multiple of kv heads; any strides with a\n"
        "contiguous last dimension.  q_lens, k_lens (int32 [batch]): how many tokens of each row count.  With q_offsets and k_offsets (int32\n"
        "[sequences + 1]) the tensors are [tokens, heads, dim] and hold packed sequences.  causal aligns the last query with the last key;\n"
        "window > 0 limits it to that many keys.  scale: dim ** -0.5 by default.  lse: fp32 [batch, heads, tokens] ([heads, tokens] packed).");
  m.def("attention_backward", &attention_backward, release(), py::arg("do"), py::arg("q"), py::arg("k"), py::arg("v"), py::arg("o"), py::arg("lse"),
        py::arg("causal") = true, py::arg("window") = 0, py::arg("scale") = none, py::arg("q_lens") = none, py::arg("k_lens") = none,
        py::arg("q_offsets") = none, py::arg("k_offsets") = none, "(dq, dk, dv) from what `attention_forward` took and gave.");
  m.def("quantize", &quantize, release(), py::arg("x"), py::arg("block_rows") = 1,
        "(codes, scales) of bf16 or fp32 x [..., cols]: float8_e4m3fn codes of x's shape and uint8 scales e that stand for 2 ** (e - 127), one for each\n"
        "1 x 128 elements ([..., ceil(cols / 128)]; activations) or, with block_rows=128, 128 x 128 of a matrix (weights).  The scale is the least\n"
        "that brings the block's largest finite magnitude to at most 448; codes are the nearest, ties to even.  NaN and infinities are kept as NaN.");
  m.def(
      "dequantize",
      [](const Tensor& codes, const Tensor& scales, const py::object& dtype) {
        const at::ScalarType t = torch::python::detail::py_object_to_dtype(dtype);
        py::gil_scoped_release no_gil;
        return dequantize(codes, scales, t);
      },
      py::arg("codes"), py::arg("scales"), py::arg("dtype"), "What `quantize` gave, as bf16 or fp32 (rounded once).");
  m.def(
      "feed_forward_forward",
      [](const Tensor& x, const Tensor& w_gate, const Tensor& w_up, const Tensor& w_down, const std::string& activation, const std::string& checkpoint) {
        std::tuple<Tensor, std::vector<Tensor>> r;
        {
          py::gil_scoped_release no_gil;
          r = feed_forward_forward(x, w_gate, w_up, w_down, activation, checkpoint);
        }
        return py::make_tuple(std::get<0>(r), py::tuple(py::cast(std::get<1>(r))));
      },
      py::arg("x"), py::arg("w_gate"), py::arg("w_up"), py::arg("w_down"), py::arg("activation") = "silu", py::arg("checkpoint") = "full",
        "(y, kept): y = (act(x w_gate') * (x w_up')) w_down' for x [..., dim], w_gate, w_up [hidden, dim], w_down [dim, hidden], all bf16 or fp32.\n"
        "activation: 'silu' or 'gelu' (tanh form).  checkpoint, what is kept for the backward pass: 'full' (gate, up) in x's dtype; '8bit' codes and\n"
        "scales of x, gate and up as `quantize` gives them; 'none' ().  Sums are fp32; the hidden activation is rounded once to x's dtype.");
  m.def("feed_forward_backward", &feed_forward_backward, release(), py::arg("dy"), py::arg("x"), py::arg("w_gate"), py::arg("w_up"), py::arg("w_down"),
        py::arg("kept"), py::arg("activation") = "silu", py::arg("need") = std::vector<bool>(4, true),
        "(dx, dw_gate, dw_up, dw_down) from what `feed_forward_forward` took and kept; x is None where '8bit' kept it.  need: which of them are formed\n"
        "(the others are None).  The gradients are those of the block at the kept gate and up.");
  m.def("linear_8bit_forward", &linear_8bit_forward, release(), py::arg("x"), py::arg("w_codes"), py::arg("w_scales"),
        "(y, x_codes, x_scales): y = Q(x) w' for bf16 x [..., dim] and w [out, dim] in 8 bits (`quantize` with block_rows=128); Q(x) in blocks of 1 x 128\n"
        "is what the backward pass takes.");
  m.def("linear_8bit_backward", &linear_8bit_backward, release(), py::arg("dy"), py::arg("x_codes"), py::arg("x_scales"), py::arg("w_codes"),
        py::arg("w_scales"), py::arg("need") = std::vector<bool>(2, true),
        "(dx, dw), bf16: dx = Q(dy) w, dw = dy' Q(x) with dy itself.  need: which of the two are formed (the other is None).");
}
