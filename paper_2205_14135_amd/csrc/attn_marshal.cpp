// Argument marshalling of the binding's forward and backward calls (paper_2205_14135_amd/binding.py)
// as a CPython extension: tensor checks, output allocation, parameter block and the library call in
// one native call.  The same steps in Python and ctypes took 9 us of a forward call with its
// buffers given, and 30 + 46 us of a training step through autograd, whose backward runs on the engine's own
// thread with cold caches; a small problem's kernels take 5 to 10 us each.  A pass with the one binding and with the other, over
// the same library, in turn: one forward call of one head of 128 tokens 9.5 -> 4.6 us, a training step of 96 heads of 197 tokens
// 149 -> 85 us (4 % between runs), of a padded batch of 128 heads of up to 700 tokens 147 -> 86 us (6 %).
// The autograd node of flash_attention (paper_2205_14135_amd/autograd.py) is here too: the engine runs backwards on a thread
// of its own, and a node in Python waits there for the interpreter lock, twice, with cold caches.  Host time of a training step of 96
// heads of 197 tokens, node in Python | here: 82 | 64 us, or 39 | 34 where the machine happens to run both threads close together (33 us
// and more of either are the engine's own change of threads: so much takes the backward of a single product).
// The functions take positional arguments only (binding.py holds the public signatures and
// defaults) and raise what the Python marshalling of the measurement entry points raises: ValueError, TypeError, AttnError.
#include "attn_marshal.h"

#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/saved_variable.h>

#include <algorithm>
#include <mutex>
#include <vector>

PyObject* marshal::attn_error = nullptr;

namespace {

using namespace marshal;

// Entry points of the library that binding.load() opened.
struct Library {
  decltype(&attn_fwd) fwd = nullptr;
  decltype(&attn_bwd) bwd = nullptr;
  decltype(&attn_bwd_workspace_bytes) workspace_bytes = nullptr;
  decltype(&attn_blocksparse_fwd) sparse_fwd = nullptr;
  decltype(&attn_blocksparse_bwd) sparse_bwd = nullptr;
  decltype(&attn_blocksparse_bwd_workspace_bytes) sparse_workspace_bytes = nullptr;
};
Library lib;
struct WindowLibrary {
  decltype(&attn_window_fwd) fwd = nullptr;
  decltype(&attn_window_bwd) bwd = nullptr;
  decltype(&attn_window_bwd_workspace_bytes) workspace_bytes = nullptr;
};
WindowLibrary window_lib;
// Of the three kinds of attention.
enum Kind { kDense, kSparse, kWindow };
const char* const kForwardNames[] = {"attn_fwd", "attn_blocksparse_fwd", "attn_window_fwd"};
const char* const kBackwardNames[] = {"attn_bwd", "attn_blocksparse_bwd", "attn_window_bwd"};
struct Window { int32_t window, sinks; };   // window 0: none
bool alike(const at::Tensor& ref, const at::Tensor& t) {
  return t.sizes() == ref.sizes() && t.strides() == ref.strides() && t.device() == ref.device();
}
void same_layout(const at::Tensor& ref, const at::Tensor& t) {
  if (!alike(ref, t)) raise(PyExc_ValueError, "all [B,H,N,d] tensors must share shape, strides and device");
}

// The arguments that every call has, in the order of the Python wrappers.
struct Options {
  PyObject *softmax_scale, *causal, *dropout_p, *seed, *offset, *o_fp32, *stream, *key_lengths;
};
Options options(PyObject* const* a) { return {a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]}; }
constexpr Py_ssize_t kOptions = 8;

attn_params make_params(PyObject* q_object, const Options& o) {
  const at::Tensor& q = tensor(q_object);
  if (q.dim() != 4 || q.stride(3) != 1) raise(PyExc_ValueError, "expected a [B,H,N,d] tensor with contiguous last axis");
  attn_params p = {};
  p.B = (int32_t)q.size(0); p.H = (int32_t)q.size(1); p.N = (int32_t)q.size(2); p.d = (int32_t)q.size(3);
  if (q.scalar_type() == at::kHalf) p.dtype = ATTN_FP16;
  else if (q.scalar_type() == at::kBFloat16) p.dtype = ATTN_BF16;
  else {
    PyObject* dtype = PyObject_GetAttrString(q_object, "dtype");
    if (dtype == nullptr) throw Raised();
    PyErr_Format(PyExc_TypeError, "Q/K/V must be float16 or bfloat16, got %S", dtype);
    Py_DECREF(dtype);
    throw Raised();
  }
  p.stride_b = q.stride(0); p.stride_h = q.stride(1); p.stride_n = q.stride(2);
  p.softmax_scale = (float)number(o.softmax_scale);
  p.causal = truth(o.causal);
  p.dropout_p = (float)number(o.dropout_p);
  p.seed = low64(o.seed);
  p.offset = low64(o.offset);
  p.o_fp32 = truth(o.o_fp32);
  if (o.stream != Py_None) p.stream = (void*)(uintptr_t)low64(o.stream);
  else if (q.is_cuda()) p.stream = (void*)c10::hip::getCurrentHIPStream(q.device().index()).stream();
  if (o.key_lengths != Py_None) {
    const at::Tensor& k = tensor(o.key_lengths);
    if (k.scalar_type() != at::kInt || k.dim() != 1 || k.size(0) != q.size(0) || !k.is_contiguous())
      raise(PyExc_TypeError, "key_lengths must be a contiguous int32 tensor of shape [B]");
    p.key_lengths = (const int32_t*)k.data_ptr();
  }
  return p;
}

// Block mask arguments of the block-sparse calls: mask tensor, mask_block.
struct Mask { const uint8_t* ptr; int32_t block; int64_t stride_h; };
Mask mask_args(PyObject* mask, PyObject* mask_block, int64_t H) {
  const at::Tensor& m = tensor(mask);
  if (m.scalar_type() != at::kByte || !m.is_contiguous())
    raise(PyExc_TypeError, "block_mask must be a contiguous uint8 tensor [T,T] or [H,T,T]");
  Mask r = {nullptr, (int32_t)low64(mask_block), 0};
  if (m.dim() == 3 && m.size(0) == H) r.stride_h = m.stride(0);
  else if (m.dim() != 2) raise(PyExc_ValueError, "block_mask must be [T,T] or [H,T,T]");
  r.ptr = (const uint8_t*)m.data_ptr();
  return r;
}

// window, sinks
Window window_args(PyObject* const* a) {
  const Window w = {clamped32(a[0]), clamped32(a[1])};
  if (w.window < 1 || w.sinks < 0) raise(PyExc_ValueError, "window must be at least 1, and sinks must not be negative");
  return w;
}

at::Tensor like(const at::Tensor& q, at::ScalarType type) {
  return at::empty_strided(q.sizes(), q.strides(), q.options().dtype(type));
}

// What the calls with a window ask of their tensors beside what all calls do: one type, one GPU, and outputs that hold what is written.
void expect_type(const at::Tensor& q, std::initializer_list<const at::Tensor*> others) {
  if (!q.is_cuda()) raise(PyExc_RuntimeError, "runs on the GPU only: there is no CPU path");
  for (const at::Tensor* t : others)
    if (t->scalar_type() != q.scalar_type()) raise(PyExc_TypeError, "all [B,H,N,d] tensors must have the same type");
}
void expect_rows_like(const at::Tensor& q, const at::Tensor& t, bool fp32) {
  if (!alike(q, t) || t.scalar_type() != (fp32 ? at::kFloat : q.scalar_type())) raise(PyExc_ValueError, "a tensor of rows has another shape, other strides, another type or device than Q");
}
void expect_statistic(const at::Tensor& q, const at::Tensor& t) {
  if (t.scalar_type() != at::kFloat || t.sizes() != q.sizes().slice(0, 3) || !t.is_contiguous() || t.device() != q.device())
    raise(PyExc_ValueError, "lse must be a contiguous float32 tensor [B,H,N] on the device of Q");
}
void expect_lengths(const at::Tensor& q, PyObject* lengths) {   // (their type and shape: make_params)
  if (lengths != Py_None && tensor(lengths).device() != q.device()) raise(PyExc_ValueError, "all tensors must be on the same device");
}

void expect_args(Py_ssize_t n, Py_ssize_t want) {
  if (n != want || lib.fwd == nullptr) raise(PyExc_TypeError, "internal call with the wrong arguments, or before attach()");
}

// ---- autograd: the forward call keeps what the backward one needs (the O(N) state: O, the row statistic and the generator state)

// What a backward call takes from its forward call beside the saved tensors.
struct Attention {
  attn_params p;            // pointers (stream, key lengths) are set again for each call
  at::Tensor key_lengths, block_mask;
};

attn_params on_current_stream(const Attention& a, const at::Tensor& q) {
  attn_params p = a.p;
  p.stride_b = q.stride(0); p.stride_h = q.stride(1); p.stride_n = q.stride(2);
  p.stream = (void*)c10::hip::getCurrentHIPStream(q.device().index()).stream();
  p.key_lengths = a.key_lengths.defined() ? (const int32_t*)a.key_lengths.data_ptr() : nullptr;
  return p;
}
int64_t mask_stride(const at::Tensor& mask) { return mask.dim() == 3 ? mask.stride(0) : 0; }

// What the marshalling of a backward call asks of its tensors (backward() below, make_params), of the saved ones as they come back: hooks
// of the program may have moved, converted or laid out anew some of them, or have given them another batch than the lengths and the masks are for.
void check_saved(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& d_out, const Attention& a) {
  if (q.dim() != 4 || q.stride(3) != 1)
    refused_in_backward([] { raise(PyExc_ValueError, "expected a [B,H,N,d] tensor with contiguous last axis"); });
  if (q.scalar_type() != at::kHalf && q.scalar_type() != at::kBFloat16)
    refused_in_backward([] { raise(PyExc_TypeError, "Q/K/V must be float16 or bfloat16"); });
  if (!q.is_cuda()) refused_in_backward([] { raise(PyExc_ValueError, "the saved tensors are not on the GPU"); });
  if (!alike(q, k) || !alike(q, v) || !alike(q, d_out))
    refused_in_backward([] { raise(PyExc_ValueError, "all [B,H,N,d] tensors must share shape, strides and device"); });
  if (a.key_lengths.defined() && a.key_lengths.size(0) != q.size(0))
    refused_in_backward([] { raise(PyExc_TypeError, "key_lengths must be a contiguous int32 tensor of shape [B]"); });
  if (a.block_mask.defined() && a.block_mask.dim() == 3 && a.block_mask.size(0) != q.size(1))
    refused_in_backward([] { raise(PyExc_ValueError, "block_mask must be [T,T] or [H,T,T]"); });
}

using torch::autograd::AutogradContext;
using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

struct FlashAttention : torch::autograd::Function<FlashAttention> {
  static at::Tensor forward(AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const Attention& a) {
    const bool sparse = a.block_mask.defined();
    const attn_params p = on_current_stream(a, q);
    const at::Tensor out = like(q, q.scalar_type()), lse = at::empty(q.sizes().slice(0, 3), q.options().dtype(at::kFloat));
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr();
    void* op = out.data_ptr();
    float* lp = (float*)lse.data_ptr();
    check_status(without_gil([&] {
      return sparse ? lib.sparse_fwd(&p, (const uint8_t*)a.block_mask.data_ptr(), 128, mask_stride(a.block_mask), qp, kp, vp, op, lp)
                    : lib.fwd(&p, qp, kp, vp, op, lp);
    }), sparse ? "attn_blocksparse_fwd" : "attn_fwd");
    ctx->save_for_backward({q, k, v, out, lse});
    auto& data = ctx->saved_data;
    data["softmax_scale"] = (double)a.p.softmax_scale;
    data["causal"] = a.p.causal != 0;
    data["dropout_p"] = (double)a.p.dropout_p;
    data["seed"] = (int64_t)a.p.seed;
    data["offset"] = (int64_t)a.p.offset;
    if (a.key_lengths.defined()) data["key_lengths"] = a.key_lengths;
    if (sparse) data["block_mask"] = a.block_mask;
    return out;
  }

  static variable_list backward(AutogradContext* ctx, const variable_list& d_outs) {
    const variable_list saved = ctx->get_saved_variables();
    const at::Tensor &q = saved[0], &k = saved[1], &v = saved[2], &out = saved[3], &lse = saved[4];
    at::Tensor d_out = d_outs[0];
    if (d_out.sizes() != q.sizes() || d_out.strides() != q.strides())   // the library addresses dO with the strides of q
      d_out = like(q, q.scalar_type()).copy_(d_out);
    auto& data = ctx->saved_data;
    Attention a = {};
    if (data.count("key_lengths")) a.key_lengths = data["key_lengths"].toTensor();
    if (data.count("block_mask")) a.block_mask = data["block_mask"].toTensor();
    check_saved(q, k, v, d_out, a);
    a.p.B = (int32_t)q.size(0); a.p.H = (int32_t)q.size(1); a.p.N = (int32_t)q.size(2); a.p.d = (int32_t)q.size(3);
    a.p.dtype = q.scalar_type() == at::kHalf ? ATTN_FP16 : ATTN_BF16;
    a.p.softmax_scale = (float)data["softmax_scale"].toDouble();
    a.p.causal = data["causal"].toBool();
    a.p.dropout_p = (float)data["dropout_p"].toDouble();
    a.p.seed = (uint64_t)data["seed"].toInt();
    a.p.offset = (uint64_t)data["offset"].toInt();
    const bool sparse = a.block_mask.defined();
    const attn_params p = on_current_stream(a, q);
    at::Tensor g[3];
    for (at::Tensor& t : g) t = like(q, q.scalar_type());
    const size_t need = sparse ? lib.sparse_workspace_bytes(&p) : lib.workspace_bytes(&p);
    const at::Tensor ws = at::empty({(int64_t)std::max<size_t>(need, 256)}, q.options().dtype(at::kByte));
    const float* lp = (const float*)lse.data_ptr();
    const int status =
        sparse ? lib.sparse_bwd(&p, (const uint8_t*)a.block_mask.data_ptr(), 128, mask_stride(a.block_mask), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                out.data_ptr(), d_out.data_ptr(), lp, g[0].data_ptr(), g[1].data_ptr(), g[2].data_ptr(), ws.data_ptr(), ws.numel())
               : lib.bwd(&p, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), d_out.data_ptr(), lp, g[0].data_ptr(), g[1].data_ptr(),
                         g[2].data_ptr(), ws.data_ptr(), ws.numel());
    if (status != ATTN_OK) refused_in_backward([&] { check_status(status, sparse ? "attn_blocksparse_bwd" : "attn_bwd"); });
    return {g[0], g[1], g[2], at::Tensor()};
  }
};

// Attention with a sliding window: a node of its own class, whose fields are members (a torch::autograd::Function keeps them in a dictionary by name).
struct WindowAttentionBackward : torch::autograd::Node {
  SavedVariable q, k, v, out, lse, key_lengths;
  attn_params p = {};   // strides and pointers are set again for each call
  Window w = {};

  variable_list apply(variable_list&& grads) override {
    at::Tensor t[5];
    Attention a = {};
    {
      // (another thread may run the same graph, and its engine let go of the saved tensors)
      const std::lock_guard<std::mutex> lock(mutex_);
      t[0] = q.unpack();
      t[1] = k.unpack();
      t[2] = v.unpack();
      t[3] = out.unpack(shared_from_this());
      t[4] = lse.unpack();
      a.key_lengths = key_lengths.unpack();
    }
    variable_list g(3);
    if (!grads[0].defined()) return g;
    // (hooks of the program may have handed back something else than what was saved)
    const at::Tensor& x = t[0];
    at::Tensor d_out = grads[0];
    // The library addresses dO with the strides of q, and reads 16 bytes at a time: what a concatenation hands back, a view somewhere in a longer gradient, may start anywhere.
    if (x.sizes() == d_out.sizes() && (x.strides() != d_out.strides() || ((uintptr_t)d_out.data_ptr() & 15u) != 0)) d_out = like(x, x.scalar_type()).copy_(d_out);
    check_saved(x, t[1], t[2], d_out, a);
    if (x.size(0) != p.B || x.size(1) != p.H || x.size(2) != p.N || x.size(3) != p.d || (x.scalar_type() == at::kHalf ? ATTN_FP16 : ATTN_BF16) != p.dtype || !alike(x, t[3]) ||
        t[3].scalar_type() != x.scalar_type() || t[1].scalar_type() != x.scalar_type() || t[2].scalar_type() != x.scalar_type() || d_out.scalar_type() != x.scalar_type() ||
        t[4].scalar_type() != at::kFloat || t[4].numel() != x.size(0) * x.size(1) * x.size(2) || !t[4].is_contiguous() || t[4].device() != x.device() ||
        (a.key_lengths.defined() && (a.key_lengths.scalar_type() != at::kInt || a.key_lengths.dim() != 1 || !a.key_lengths.is_contiguous() || a.key_lengths.device() != x.device())))
      refused_in_backward([] { raise(PyExc_ValueError, "the saved tensors are not those of the forward call"); });
    const c10::DeviceGuard guard(x.device());
    a.p = p;
    const attn_params now = on_current_stream(a, x);
    for (at::Tensor& y : g) y = like(x, x.scalar_type());
    const at::Tensor ws = at::empty({(int64_t)std::max<size_t>(window_lib.workspace_bytes(&now, w.window, w.sinks), 256)}, x.options().dtype(at::kByte));
    const int status = window_lib.bwd(&now, w.window, w.sinks, x.data_ptr(), t[1].data_ptr(), t[2].data_ptr(), t[3].data_ptr(), d_out.data_ptr(), (const float*)t[4].data_ptr(),
                                      g[0].data_ptr(), g[1].data_ptr(), g[2].data_ptr(), ws.data_ptr(), ws.numel());
    if (status != ATTN_OK) refused_in_backward([&] { check_status(status, "attn_window_bwd"); });
    mark_once_differentiable(*this, g, "the gradients of attention with a window cannot be differentiated again");
    return g;
  }
  void release_variables() override {
    const std::lock_guard<std::mutex> lock(mutex_);
    for (SavedVariable* s : {&q, &k, &v, &out, &lse, &key_lengths}) s->reset_data();
  }
  std::string name() const override { return "WindowAttentionBackward"; }
};

// window_attention(Q, K, V, softmax_scale, dropout_p, seed, offset, key_lengths, window, sinks) -> O, differentiable
PyObject* py_window_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 10);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
    same_layout(q, k);
    same_layout(q, v);
    Attention at = {};
    at.p = make_params(a[0], {a[3], Py_True, a[4], a[5], a[6], Py_False, Py_None, a[7]});
    if (a[7] != Py_None) at.key_lengths = tensor(a[7]);
    const Window w = window_args(a + 8);
    expect_type(q, {&k, &v});
    expect_lengths(q, a[7]);
    if (at::GradMode::is_enabled()) refuse_eager_graphs({&q, &k, &v});
    const c10::DeviceGuard guard(q.device());
    const at::Tensor lse = at::empty(q.sizes().slice(0, 3), q.options().dtype(at::kFloat));
    at::Tensor out = like(q, q.scalar_type());
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr();
    void* op = out.data_ptr();
    float* lp = (float*)lse.data_ptr();
    const attn_params p = on_current_stream(at, q);
    check_status(without_gil([&] { return window_lib.fwd(&p, w.window, w.sinks, qp, kp, vp, op, lp); }), "attn_window_fwd");
    if (torch::autograd::compute_requires_grad(q, k, v)) {
      const std::shared_ptr<WindowAttentionBackward> node(new WindowAttentionBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(q, k, v));
      node->q = SavedVariable(q, false);
      node->k = SavedVariable(k, false);
      node->v = SavedVariable(v, false);
      node->lse = SavedVariable(lse, false);
      node->key_lengths = SavedVariable(at.key_lengths, false);
      node->p = at.p;
      node->w = w;
      torch::autograd::set_history(out, node);
      node->out = SavedVariable(out, true);
    }
    return wrap(out);
  });
}

// attention(Q, K, V, softmax_scale, causal, dropout_p, seed, offset, key_lengths, block_mask) -> O, differentiable
PyObject* py_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 10);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
    same_layout(q, k);
    same_layout(q, v);
    Attention at = {};
    at.p = make_params(a[0], {a[3], a[4], a[5], a[6], a[7], Py_False, Py_None, a[8]});
    if (a[8] != Py_None) at.key_lengths = tensor(a[8]);
    if (a[9] != Py_None) {
      PyObject* block = PyLong_FromLong(128);
      if (block == nullptr) throw Raised();
      try {
        mask_args(a[9], block, q.size(1));
      } catch (...) {
        Py_DECREF(block);
        throw;
      }
      Py_DECREF(block);
      at.block_mask = tensor(a[9]);
    }
    return wrap(FlashAttention::apply(q, k, v, at));
  });
}

// fwd(Q, K, V, <options>, out, lse[, block_mask, mask_block | window, sinks]) -> (O, LSE)
PyObject* forward(PyObject* const* a, Py_ssize_t n, Kind kind) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 3 + kOptions + 2 + (kind != kDense ? 2 : 0));
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
    same_layout(q, k);
    same_layout(q, v);
    const attn_params p = make_params(a[0], options(a + 3));
    PyObject* const* r = a + 3 + kOptions;
    Mask m = {};
    Window w = {};
    if (kind == kSparse) m = mask_args(r[2], r[3], q.size(1));
    if (kind == kWindow) w = window_args(r + 2);
    const at::Tensor out = r[0] != Py_None ? tensor(r[0]) : like(q, p.o_fp32 ? at::kFloat : q.scalar_type());
    const at::Tensor lse = r[1] != Py_None ? tensor(r[1]) : at::empty(q.sizes().slice(0, 3), q.options().dtype(at::kFloat));
    c10::OptionalDeviceGuard guard;
    if (kind == kWindow) {
      expect_type(q, {&k, &v});
      expect_rows_like(q, out, p.o_fp32);
      expect_statistic(q, lse);
      expect_lengths(q, a[3 + 7]);
      guard.reset_device(q.device());
    }
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr();
    void* op = out.data_ptr();
    float* lp = (float*)lse.data_ptr();
    check_status(without_gil([&] {
      if (kind == kWindow) return window_lib.fwd(&p, w.window, w.sinks, qp, kp, vp, op, lp);
      return kind == kSparse ? lib.sparse_fwd(&p, m.ptr, m.block, m.stride_h, qp, kp, vp, op, lp) : lib.fwd(&p, qp, kp, vp, op, lp);
    }), kForwardNames[kind]);
    return tuple({r[0] != Py_None ? Py_NewRef(r[0]) : wrap(out), r[1] != Py_None ? Py_NewRef(r[1]) : wrap(lse)});
  });
}

// bwd(Q, K, V, O, dO, LSE, <options>, workspace, allocate, dQ, dK, dV[, block_mask, mask_block | window, sinks]) -> (dQ, dK, dV);
// allocate: dQ, dK and dV are made here, else they are the caller's
PyObject* backward(PyObject* const* a, Py_ssize_t n, Kind kind) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 6 + kOptions + 5 + (kind != kDense ? 2 : 0));
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]), &go = tensor(a[4]);
    same_layout(q, k);
    same_layout(q, v);
    same_layout(q, go);
    const attn_params p = make_params(a[0], options(a + 6));
    PyObject* const* r = a + 6 + kOptions;
    Mask m = {};
    Window w = {};
    if (kind == kSparse) m = mask_args(r[5], r[6], q.size(1));
    if (kind == kWindow) w = window_args(r + 5);
    const bool allocate = truth(r[1]);
    at::Tensor g[3];
    void* gp[3];
    for (int i = 0; i < 3; ++i) {
      if (allocate) g[i] = like(q, q.scalar_type());
      gp[i] = allocate ? g[i].data_ptr() : data(r[2 + i]);
    }
    c10::OptionalDeviceGuard guard;
    if (kind == kWindow) {
      expect_type(q, {&k, &v, &go});
      expect_rows_like(q, tensor(a[3]), p.o_fp32);
      expect_statistic(q, tensor(a[5]));
      expect_lengths(q, a[6 + 7]);
      for (int i = 0; i < 3 && !allocate; ++i) expect_rows_like(q, tensor(r[2 + i]), false);
      if (r[0] != Py_None && (!tensor(r[0]).is_contiguous() || tensor(r[0]).device() != q.device())) raise(PyExc_ValueError, "the workspace must be contiguous, on the device of Q");
      guard.reset_device(q.device());
    }
    at::Tensor ws;
    if (r[0] != Py_None) {
      ws = tensor(r[0]);
    } else {
      const size_t need = kind == kWindow ? window_lib.workspace_bytes(&p, w.window, w.sinks) : (kind == kSparse ? lib.sparse_workspace_bytes(&p) : lib.workspace_bytes(&p));
      ws = at::empty({(int64_t)std::max<size_t>(need, 256)}, q.options().dtype(at::kByte));
    }
    const size_t ws_bytes = (size_t)ws.numel() * ws.element_size();
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr(), *op = data(a[3]), *gop = go.data_ptr();
    const float* lp = (const float*)data(a[5]);
    void* wp = ws.data_ptr();
    check_status(without_gil([&] {
      if (kind == kWindow) return window_lib.bwd(&p, w.window, w.sinks, qp, kp, vp, op, gop, lp, gp[0], gp[1], gp[2], wp, ws_bytes);
      return kind == kSparse ? lib.sparse_bwd(&p, m.ptr, m.block, m.stride_h, qp, kp, vp, op, gop, lp, gp[0], gp[1], gp[2], wp, ws_bytes)
                    : lib.bwd(&p, qp, kp, vp, op, gop, lp, gp[0], gp[1], gp[2], wp, ws_bytes);
    }), kBackwardNames[kind]);
    PyObject* t[3];
    for (int i = 0; i < 3; ++i) t[i] = allocate ? wrap(g[i]) : Py_NewRef(r[2 + i]);
    return tuple({t[0], t[1], t[2]});
  });
}

PyObject* py_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return forward(a, n, kDense); }
PyObject* py_sparse_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return forward(a, n, kSparse); }
PyObject* py_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return backward(a, n, kDense); }
PyObject* py_sparse_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return backward(a, n, kSparse); }
PyObject* py_window_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return forward(a, n, kWindow); }
PyObject* py_window_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return backward(a, n, kWindow); }

// attach(AttnError, address of attn_fwd, attn_bwd, attn_bwd_workspace_bytes, and the three block-sparse ones)
PyObject* py_attach(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 7) raise(PyExc_TypeError, "attach() takes the error class and six addresses");
    Library l;
    l.fwd = (decltype(l.fwd))low64(a[1]);
    l.bwd = (decltype(l.bwd))low64(a[2]);
    l.workspace_bytes = (decltype(l.workspace_bytes))low64(a[3]);
    l.sparse_fwd = (decltype(l.sparse_fwd))low64(a[4]);
    l.sparse_bwd = (decltype(l.sparse_bwd))low64(a[5]);
    l.sparse_workspace_bytes = (decltype(l.sparse_workspace_bytes))low64(a[6]);
    Py_INCREF(a[0]);
    Py_XDECREF(attn_error);
    attn_error = a[0];
    lib = l;
    Py_RETURN_NONE;
  });
}

// attach_window(address of attn_window_fwd, attn_window_bwd, attn_window_bwd_workspace_bytes)
PyObject* py_attach_window(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 3) raise(PyExc_TypeError, "attach_window() takes three addresses");
    WindowLibrary l;
    l.fwd = (decltype(l.fwd))low64(a[0]);
    l.bwd = (decltype(l.bwd))low64(a[1]);
    l.workspace_bytes = (decltype(l.workspace_bytes))low64(a[2]);
    window_lib = l;
    Py_RETURN_NONE;
  });
}

const PyMethodDef own_methods[] = {
    {"attach_window", (PyCFunction)(void*)py_attach_window, METH_FASTCALL, nullptr},
    {"window_attention", (PyCFunction)(void*)py_window_attention, METH_FASTCALL, nullptr},
    {"window_fwd", (PyCFunction)(void*)py_window_fwd, METH_FASTCALL, nullptr},
    {"window_bwd", (PyCFunction)(void*)py_window_bwd, METH_FASTCALL, nullptr},
    {"attach", (PyCFunction)(void*)py_attach, METH_FASTCALL, nullptr},
    {"attention", (PyCFunction)(void*)py_attention, METH_FASTCALL, nullptr},
    {"fwd", (PyCFunction)(void*)py_fwd, METH_FASTCALL, nullptr},
    {"bwd", (PyCFunction)(void*)py_bwd, METH_FASTCALL, nullptr},
    {"blocksparse_fwd", (PyCFunction)(void*)py_sparse_fwd, METH_FASTCALL, nullptr},
    {"blocksparse_bwd", (PyCFunction)(void*)py_sparse_bwd, METH_FASTCALL, nullptr}};
std::vector<PyMethodDef> methods;   // of both sources
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  methods.assign(std::begin(own_methods), std::end(own_methods));
  for (const PyMethodDef* m = paged_methods;; ++m) {
    methods.push_back(*m);
    if (m->ml_name == nullptr) break;
  }
  module.m_methods = methods.data();
  return PyModule_Create(&module);
}
