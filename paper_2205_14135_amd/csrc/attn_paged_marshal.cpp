// Argument marshalling of the rotary positions and of the paged cache's calls (paper_2205_14135_amd/binding.py), and the autograd node of the rotation
// (paper_2205_14135_amd/autograd.py), natively for the reason given in attn_marshal.cpp: a step of a running batch is a handful of kernels of 5 to 20 us each.
// Everything runs on torch's current stream of the tensors' device, which is made the current one for the call.
#include "attn_marshal.h"

#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/autograd/variable.h>

#include <mutex>
#include <unordered_set>
#include <vector>

namespace {

using namespace marshal;

struct Library {
  decltype(&attn_rotary) rotary = nullptr;
  decltype(&attn_paged_append) append = nullptr;
  decltype(&attn_paged_workspace_bytes) workspace_bytes = nullptr;
  decltype(&attn_paged_fwd) fwd = nullptr;
  decltype(&attn_paged_copy) copy = nullptr;
};
Library lib;
struct NormLibrary {
  decltype(&attn_norm_rotary) fwd = nullptr;
  decltype(&attn_norm_rotary_bwd_workspace_bytes) workspace_bytes = nullptr;
  decltype(&attn_norm_rotary_bwd) bwd = nullptr;
  decltype(&attn_paged_norm_append) append = nullptr;
};
NormLibrary norm_lib;
decltype(&attn_paged_window_fwd) window_fwd = nullptr;

void expect_args(Py_ssize_t n, Py_ssize_t want) {
  if (n != want || lib.rotary == nullptr) raise(PyExc_TypeError, "internal call with the wrong arguments, or before attach_paged()");
}

void* current_stream(const at::Tensor& t) { return (void*)c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

int dtype_of(const at::Tensor& t, const char* what) {
  if (t.scalar_type() == at::kHalf) return ATTN_FP16;
  if (t.scalar_type() == at::kBFloat16) return ATTN_BF16;
  PyErr_Format(PyExc_TypeError, "%s must be float16 or bfloat16", what);
  throw Raised();
}
// (the stride of an axis of one entry or none says nothing)
int64_t axis_stride(const at::Tensor& t, int64_t axis) { return t.size(axis) > 1 ? t.stride(axis) : 0; }
void expect_rows(const at::Tensor& t, int64_t dims, const char* text) {
  if (t.dim() != dims || (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1)) raise(PyExc_ValueError, text);
}
void expect_like(const at::Tensor& t, const at::Tensor& ref, const char* what) {
  if (t.sizes() != ref.sizes() || t.scalar_type() != ref.scalar_type()) {
    PyErr_Format(PyExc_ValueError, "%s has another shape or type than what it goes with", what);
    throw Raised();
  }
}
void expect_ints(const at::Tensor& t, bool shape_ok, const char* text) {
  if (t.scalar_type() != at::kInt || !shape_ok) raise(PyExc_TypeError, text);
}
// All tensors of a call on one GPU: there is no CPU path.
void expect_gpu(const at::Tensor& ref, std::initializer_list<const at::Tensor*> others) {
  if (!ref.is_cuda()) raise(PyExc_RuntimeError, "runs on the GPU only: there is no CPU path");
  for (const at::Tensor* t : others)
    if (t->defined() && t->device() != ref.device()) raise(PyExc_ValueError, "all tensors must be on the same device");
}
at::Tensor maybe(PyObject* o) { return o == Py_None ? at::Tensor() : tensor(o); }
const void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// An output with the strides of what it comes from, so that Q and K keep V's (the attention takes three tensors of the same strides); packed where the input repeats rows.
at::Tensor output_like(const at::Tensor& x) {
  for (int64_t i = 0; i + 1 < x.dim(); ++i)
    if (x.size(i) > 1 && x.stride(i) == 0) return at::empty(x.sizes(), x.options());
  return at::empty_strided(x.sizes(), x.strides(), x.options());
}

// An output that need not share strides with anything: in its input's order of axes, without the input's gaps (Q may be a part of a projection's rows, or one
// token's of a long tensor).
at::Tensor packed_like(const at::Tensor& x) {
  for (int64_t i = 0; i + 1 < x.dim(); ++i)
    if (x.size(i) > 1 && x.stride(i) == 0) return at::empty(x.sizes(), x.options());
  return at::empty_like(x, x.options(), at::MemoryFormat::Preserve);
}

int32_t narrow(int64_t v) { return v > INT32_MAX ? -1 : (int32_t)v; }   // (the library refuses what is negative)

// ---- rotary positions

struct Rotation {
  at::Tensor frequencies, positions;   // frequencies may be undefined where a norm goes without a rotation
  bool interleaved, inverse;
  double magnitude;
};
void check_frequencies(const at::Tensor& f) {
  if (f.scalar_type() != at::kDouble || f.dim() != 1 || !f.is_contiguous()) raise(PyExc_TypeError, "frequencies must be a contiguous float64 tensor [rotary_dim / 2]");
}
attn_rotary_spec spec_of(const at::Tensor& f, bool interleaved, double magnitude) {
  if (!f.defined()) return {};
  return {(const double*)f.data_ptr(), narrow(2 * f.size(0)), interleaved, (float)magnitude};
}
void check_rotation(const at::Tensor& q, const at::Tensor& k, const Rotation& r) {
  expect_rows(q, 4, "expected a [B,H,N,d] tensor with contiguous last axis");
  dtype_of(q, "Q and K");
  if (k.defined()) {
    expect_rows(k, 4, "expected a [B,H,N,d] tensor with contiguous last axis");
    if (k.scalar_type() != q.scalar_type() || k.size(0) != q.size(0) || k.size(2) != q.size(2) || k.size(3) != q.size(3))
      raise(PyExc_ValueError, "Q and K must share type, batch, length and head dimension");
  }
  if (r.frequencies.defined()) check_frequencies(r.frequencies);
  if (r.positions.defined()) {
    const at::Tensor& p = r.positions;
    const bool one = p.dim() == 1 && p.size(0) == q.size(2), each = p.dim() == 2 && p.size(0) == q.size(0) && p.size(1) == q.size(2);
    if (p.scalar_type() != at::kInt || !(one || each) || (q.size(2) > 1 && p.stride(p.dim() - 1) != 1))
      raise(PyExc_TypeError, "positions must be an int32 tensor [N] or [B,N] with contiguous last axis");
  }
  expect_gpu(q, {&k, &r.frequencies, &r.positions});
}
attn_rotary_params params_of(const at::Tensor& q, const Rotation& r) {
  attn_rotary_params p = {};
  p.B = narrow(q.size(0)); p.N = narrow(q.size(2)); p.d = narrow(q.size(3));
  p.dtype = q.scalar_type() == at::kHalf ? ATTN_FP16 : ATTN_BF16;
  p.rotary = spec_of(r.frequencies, r.interleaved, r.magnitude);
  p.inverse = r.inverse;
  if (r.positions.defined()) {
    p.positions = (const int32_t*)r.positions.data_ptr();
    p.position_stride_b = r.positions.dim() == 2 ? axis_stride(r.positions, 0) : 0;
  }
  p.stream = current_stream(q);
  return p;
}
// the tensors that there are; returns their number
int fill(attn_rotary_tensor (&t)[2], const at::Tensor& q, const at::Tensor& k, const at::Tensor& qo, const at::Tensor& ko) {
  int n = 0;
  for (const auto& [x, y] : {std::pair<const at::Tensor&, const at::Tensor&>(q, qo), std::pair<const at::Tensor&, const at::Tensor&>(k, ko)}) {
    if (!x.defined()) continue;
    t[n++] = {x.data_ptr(), y.data_ptr(), narrow(x.size(1)), axis_stride(x, 0), axis_stride(x, 1), axis_stride(x, 2), axis_stride(y, 0), axis_stride(y, 1), axis_stride(y, 2)};
  }
  return n;
}
int rotate(const at::Tensor& q, const at::Tensor& k, const at::Tensor& qo, const at::Tensor& ko, const Rotation& r) {
  const attn_rotary_params p = params_of(q, r);
  attn_rotary_tensor t[2];
  const int n = fill(t, q, k, qo, ko);
  return lib.rotary(&p, t, n);
}
// outputs that the caller gives for Q and K
void check_outputs(const at::Tensor& q, const at::Tensor& k, const at::Tensor& qo, const at::Tensor& ko) {
  for (const auto& [x, y] : {std::pair<const at::Tensor&, const at::Tensor&>(q, qo), std::pair<const at::Tensor&, const at::Tensor&>(k, ko)}) {
    if (!y.defined()) continue;
    if (!x.defined()) raise(PyExc_ValueError, "an output for K without K");
    expect_like(y, x, "an output");
    expect_rows(y, 4, "expected a [B,H,N,d] tensor with contiguous last axis");
  }
}

// rotary(Q, K, frequencies, interleaved, magnitude, positions, inverse, Qout, Kout) -> (Q', K')
PyObject* py_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 9);
    const at::Tensor &q = tensor(a[0]), k = maybe(a[1]);
    const Rotation r = {tensor(a[2]), maybe(a[5]), truth(a[3]), truth(a[6]), number(a[4])};
    at::Tensor qo = maybe(a[7]), ko = maybe(a[8]);
    check_outputs(q, k, qo, ko);
    check_rotation(q, k, r);
    expect_gpu(q, {&qo, &ko});
    const c10::DeviceGuard guard(q.device());
    if (!qo.defined()) qo = output_like(q);
    if (k.defined() && !ko.defined()) ko = output_like(k);
    check_status(without_gil([&] { return rotate(q, k, qo, ko, r); }), "attn_rotary");
    PyObject* const second = k.defined() ? (a[8] != Py_None ? Py_NewRef(a[8]) : wrap(ko)) : Py_NewRef(Py_None);
    return tuple({a[7] != Py_None ? Py_NewRef(a[7]) : wrap(qo), second});
  });
}

using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

// What the library can read: rows in one piece that start on 16 bytes.
at::Tensor readable(const at::Tensor& t) {
  bool ok = axis_stride(t, 3) == (t.size(3) > 1 ? 1 : 0) && ((uintptr_t)t.data_ptr() & 15u) == 0;
  for (int64_t i = 0; i < 3; ++i) ok = ok && axis_stride(t, i) >= 0 && axis_stride(t, i) % 8 == 0;
  return ok ? t : t.clone(at::MemoryFormat::Contiguous);
}

variable_list rotary_embedding(const at::Tensor& q, const at::Tensor& k, const Rotation& r, at::Tensor (*make)(const at::Tensor&));

// The gradient of a rotation is the rotation by the negative angle, with a node of the same kind where it is to be differentiated again.  A node of its own class, with
// its fields as members: with a torch::autograd::Function (its context keeps them in a dictionary by name) a forward and backward of 8 x 16 heads
// of 1024 tokens took 75 us of host time.
struct RotaryBackward : torch::autograd::Node {
  SavedVariable frequencies, positions;
  int64_t pairs = 0;   // that turn
  bool interleaved = false, inverse = false;
  double magnitude = 1.0;

  variable_list apply(variable_list&& grads) override {
    Rotation r = {at::Tensor(), at::Tensor(), interleaved, !inverse, magnitude};
    {
      // (another thread may run the same graph, and its engine let go of the saved tensors)
      const std::lock_guard<std::mutex> lock(mutex_);
      r.frequencies = frequencies.unpack();
      r.positions = positions.unpack();
    }
    const at::Tensor q = grads[0].defined() && should_compute_output(0) ? readable(grads[0]) : at::Tensor();
    const at::Tensor k = grads[1].defined() && should_compute_output(1) ? readable(grads[1]) : at::Tensor();
    const at::Tensor& x = q.defined() ? q : k;
    if (!x.defined()) return {at::Tensor(), at::Tensor()};
    // (hooks of the program may have handed back something else than what was saved)
    const at::Tensor &f = r.frequencies, &p = r.positions;
    if (f.scalar_type() != at::kDouble || f.dim() != 1 || f.size(0) != pairs || !f.is_contiguous() || f.device() != x.device() ||
        (p.defined() && (p.device() != x.device() || p.scalar_type() != at::kInt || (p.dim() == 1 ? p.size(0) != x.size(2) : p.dim() != 2 || p.size(0) != x.size(0) || p.size(1) != x.size(2)) ||
                         (x.size(2) > 1 && p.stride(p.dim() - 1) != 1))))
      refused_in_backward([] { raise(PyExc_ValueError, "the saved frequencies or positions are not those of the forward call"); });
    return rotary_embedding(q, k, r, packed_like);
  }
  void release_variables() override {
    const std::lock_guard<std::mutex> lock(mutex_);
    frequencies.reset_data();
    positions.reset_data();
  }
  std::string name() const override { return "RotaryBackward"; }
};

// q or k may be undefined; make: their outputs.  Called without the interpreter lock.
variable_list rotary_embedding(const at::Tensor& q, const at::Tensor& k, const Rotation& r, at::Tensor (*make)(const at::Tensor&)) {
  const at::Tensor& x = q.defined() ? q : k;
  const c10::DeviceGuard guard(x.device());
  at::Tensor qo, ko;
  if (q.defined()) qo = make(q);
  if (k.defined()) ko = make(k);
  const int status = q.defined() ? rotate(q, k, qo, ko, r) : rotate(k, q, ko, qo, r);
  if (status != ATTN_OK) refused_in_backward([&] { check_status(status, "attn_rotary"); });
  if (torch::autograd::compute_requires_grad(q, k)) {
    const std::shared_ptr<RotaryBackward> node(new RotaryBackward(), torch::autograd::deleteNode);
    node->set_next_edges(torch::autograd::collect_next_edges(q, k));
    node->frequencies = SavedVariable(r.frequencies, false);
    node->positions = SavedVariable(r.positions, false);
    node->pairs = r.frequencies.size(0);
    node->interleaved = r.interleaved;
    node->inverse = r.inverse;
    node->magnitude = r.magnitude;
    // (both are outputs of the node, also where only one of the inputs asks for a gradient)
    for (at::Tensor* y : {&qo, &ko}) {
      if (y->defined()) torch::autograd::set_history(*y, node);
      else node->add_input_metadata(torch::autograd::Node::undefined_input());
    }
  }
  return {qo, ko};
}

// rotary_embedding(Q, K, frequencies, interleaved, magnitude, positions, V) -> (Q', K'), differentiable.  V: of the same pass, or None.
PyObject* py_rotary_embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 7);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), v = maybe(a[6]);
    const Rotation r = {tensor(a[2]), maybe(a[5]), truth(a[3]), false, number(a[4])};
    check_rotation(q, k, r);
    if (at::GradMode::is_enabled()) {
      const c10::DeviceGuard guard(q.device());
      refuse_eager_graphs({&q, &k, &v});
    }
    variable_list out;
    {
      PyThreadState* const s = PyEval_SaveThread();
      try {
        out = rotary_embedding(q, k, r, output_like);
      } catch (...) {
        PyEval_RestoreThread(s);
        throw;
      }
      PyEval_RestoreThread(s);
    }
    return tuple({wrap(out[0]), wrap(out[1])});
  });
}

// ---- the norm of Q and K, with the rotation

struct Norm { at::Tensor wq, wk; double eps; };   // wk may be undefined where there is no K
void check_norm(const at::Tensor& q, const at::Tensor& k, const Norm& n) {
  for (const at::Tensor* w : {&n.wq, &n.wk}) {
    if (!w->defined()) continue;
    if (w->dim() != 1 || w->size(0) != q.size(q.dim() - 1) || !w->is_contiguous()) raise(PyExc_ValueError, "the norm's weights must be contiguous tensors [d]");
    if ((w->scalar_type() != at::kFloat && w->scalar_type() != q.scalar_type()) || (n.wq.defined() && w->scalar_type() != n.wq.scalar_type()))
      raise(PyExc_TypeError, "the norm's weights must be float32 or of the tensors' type, both the same");
  }
  if (!n.wq.defined() || (k.defined() && !n.wk.defined())) raise(PyExc_ValueError, "the norm has no weights for a tensor that is given");
  expect_gpu(q, {&n.wq, &n.wk});
}
attn_norm_spec norm_spec(const Norm& n) {
  const at::Tensor& w = n.wq.defined() ? n.wq : n.wk;
  return {ptr(n.wq), ptr(n.wk), w.scalar_type() == at::kFloat, (float)n.eps};
}
int norm_rotate(const at::Tensor& q, const at::Tensor& k, const at::Tensor& qo, const at::Tensor& ko, const Norm& n, const Rotation& r) {
  const attn_rotary_params p = params_of(q, r);
  const attn_norm_spec s = norm_spec(n);
  attn_rotary_tensor t[2];
  const int count = fill(t, q, k, qo, ko);
  return norm_lib.fwd(&p, &s, t, count);
}
// What a backward call reads and writes for one tensor; dw may be undefined.
struct Grad { at::Tensor x, dy, dx, w, dw; };
// (of one or two tensors; the first weights are the first tensor's)
int norm_gradients(const std::vector<Grad>& g, double eps, const Rotation& r, const at::Tensor& ws) {
  const attn_rotary_params p = params_of(g[0].x, r);
  attn_norm_grad t[2] = {};
  for (size_t i = 0; i < g.size(); ++i) {
    const at::Tensor &x = g[i].x, &y = g[i].dy, &d = g[i].dx;
    t[i] = {x.data_ptr(), y.data_ptr(), d.data_ptr(), const_cast<void*>(ptr(g[i].dw)), narrow(x.size(1)), axis_stride(x, 0), axis_stride(x, 1), axis_stride(x, 2),
            axis_stride(y, 0), axis_stride(y, 1), axis_stride(y, 2), axis_stride(d, 0), axis_stride(d, 1), axis_stride(d, 2)};
  }
  const attn_norm_spec s = {ptr(g[0].w), g.size() > 1 ? ptr(g[1].w) : nullptr, g[0].w.scalar_type() == at::kFloat, (float)eps};
  return norm_lib.bwd(&p, &s, t, (int)g.size(), const_cast<void*>(ptr(ws)), ws.defined() ? (size_t)ws.numel() * ws.element_size() : 0);
}
at::Tensor norm_workspace(const at::Tensor& x) {
  return at::empty({(int64_t)std::max<size_t>(norm_lib.workspace_bytes(narrow(x.size(3))), 256)}, x.options().dtype(at::kByte));
}
void check_no_lost_positions(const Rotation& r) {
  if (r.positions.defined() && !r.frequencies.defined()) raise(PyExc_ValueError, "positions are of no use without rotary");
}

// norm_rotary(Q, K, q_weight, k_weight, eps, frequencies, interleaved, magnitude, positions, Qout, Kout) -> (Q', K')
PyObject* py_norm_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 11);
    const at::Tensor &q = tensor(a[0]), k = maybe(a[1]);
    const Norm norm = {maybe(a[2]), maybe(a[3]), number(a[4])};
    const Rotation r = {maybe(a[5]), maybe(a[8]), truth(a[6]), false, number(a[7])};
    at::Tensor qo = maybe(a[9]), ko = maybe(a[10]);
    check_outputs(q, k, qo, ko);
    check_rotation(q, k, r);
    check_no_lost_positions(r);
    check_norm(q, k, norm);
    expect_gpu(q, {&qo, &ko});
    const c10::DeviceGuard guard(q.device());
    if (!qo.defined()) qo = output_like(q);
    if (k.defined() && !ko.defined()) ko = output_like(k);
    check_status(without_gil([&] { return norm_rotate(q, k, qo, ko, norm, r); }), "attn_norm_rotary");
    PyObject* const second = k.defined() ? (a[10] != Py_None ? Py_NewRef(a[10]) : wrap(ko)) : Py_NewRef(Py_None);
    return tuple({a[9] != Py_None ? Py_NewRef(a[9]) : wrap(qo), second});
  });
}

// norm_rotary_bwd(Q, K, dQ', dK', q_weight, k_weight, eps, frequencies, interleaved, magnitude, positions, workspace) -> (dQ, dK, dq_weight, dk_weight)
PyObject* py_norm_rotary_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 12);
    const at::Tensor &q = tensor(a[0]), k = maybe(a[1]), &gq = tensor(a[2]), gk = maybe(a[3]);
    const Norm norm = {maybe(a[4]), maybe(a[5]), number(a[6])};
    const Rotation r = {maybe(a[7]), maybe(a[10]), truth(a[8]), false, number(a[9])};
    at::Tensor ws = maybe(a[11]);
    if (k.defined() != gk.defined()) raise(PyExc_ValueError, "K and its gradient go together");
    check_outputs(q, k, gq, gk);
    check_rotation(q, k, r);
    check_no_lost_positions(r);
    check_norm(q, k, norm);
    if (ws.defined() && !ws.is_contiguous()) raise(PyExc_ValueError, "the workspace must be contiguous");
    expect_gpu(q, {&gq, &gk, &ws});
    const c10::DeviceGuard guard(q.device());
    if (!ws.defined()) ws = norm_workspace(q);
    std::vector<Grad> g = {{q, gq, packed_like(q), norm.wq, at::empty_like(norm.wq)}};
    if (k.defined()) g.push_back({k, gk, packed_like(k), norm.wk, at::empty_like(norm.wk)});
    check_status(without_gil([&] { return norm_gradients(g, norm.eps, r, ws); }), "attn_norm_rotary_bwd");
    if (!k.defined()) return tuple({wrap(g[0].dx), Py_NewRef(Py_None), wrap(g[0].dw), Py_NewRef(Py_None)});
    return tuple({wrap(g[0].dx), wrap(g[1].dx), wrap(g[0].dw), wrap(g[1].dw)});
  });
}

struct NormRotaryBackward : torch::autograd::Node {
  SavedVariable x[2], w[2], frequencies, positions;
  bool interleaved = false;
  double magnitude = 1.0, eps = 0.0;
  int64_t pairs = 0;

  // inputs: q, k, q_weight, k_weight
  variable_list apply(variable_list&& grads) override {
    Rotation r = {at::Tensor(), at::Tensor(), interleaved, false, magnitude};
    at::Tensor xs[2], ws[2];
    {
      const std::lock_guard<std::mutex> lock(mutex_);
      r.frequencies = frequencies.unpack();
      r.positions = positions.unpack();
      for (int i = 0; i < 2; ++i) {
        xs[i] = x[i].unpack();
        ws[i] = w[i].unpack();
      }
    }
    variable_list out(4);
    std::vector<Grad> g;
    int which[2];
    for (int i = 0; i < 2; ++i) {
      if (!grads[i].defined() || !(should_compute_output(i) || should_compute_output(2 + i))) continue;
      // (hooks of the program may have handed back something else than what was saved)
      const at::Tensor &f = r.frequencies, &p = r.positions;
      const bool ok = xs[i].defined() && xs[i].dim() == 4 && xs[i].sizes() == grads[i].sizes() && xs[i].scalar_type() == grads[i].scalar_type() && xs[i].device() == grads[i].device() &&
                      ws[i].defined() && ws[i].dim() == 1 && ws[i].size(0) == xs[i].size(3) && ws[i].is_contiguous() && ws[i].device() == xs[i].device() &&
                      (ws[i].scalar_type() == at::kFloat || ws[i].scalar_type() == xs[i].scalar_type()) && (g.empty() || ws[i].scalar_type() == g[0].w.scalar_type()) &&
                      (pairs == 0 ? !f.defined() : f.defined() && f.scalar_type() == at::kDouble && f.dim() == 1 && f.size(0) == pairs && f.is_contiguous() && f.device() == xs[i].device()) &&
                      (!p.defined() || (p.device() == xs[i].device() && p.scalar_type() == at::kInt &&
                                        (p.dim() == 1 ? p.size(0) == xs[i].size(2) : p.dim() == 2 && p.size(0) == xs[i].size(0) && p.size(1) == xs[i].size(2)) &&
                                        (xs[i].size(2) <= 1 || p.stride(p.dim() - 1) == 1)));
      if (!ok) refused_in_backward([] { raise(PyExc_ValueError, "the saved tensors are not those of the forward call"); });
      const c10::DeviceGuard guard(xs[i].device());
      const at::Tensor from = readable(xs[i]);
      which[g.size()] = i;
      g.push_back({from, readable(grads[i]), packed_like(xs[i]), ws[i], should_compute_output(2 + i) ? at::empty_like(ws[i]) : at::Tensor()});
    }
    if (g.empty()) return out;
    const c10::DeviceGuard guard(g[0].x.device());
    bool weights = false;
    for (const Grad& t : g) weights = weights || t.dw.defined();
    const int status = norm_gradients(g, eps, r, weights ? norm_workspace(g[0].x) : at::Tensor());
    if (status != ATTN_OK) refused_in_backward([&] { check_status(status, "attn_norm_rotary_bwd"); });
    for (size_t n = 0; n < g.size(); ++n) {
      if (should_compute_output(which[n])) out[which[n]] = g[n].dx;
      out[2 + which[n]] = g[n].dw;
    }
    mark_once_differentiable(*this, out, "the gradients of norm_rotary_embedding cannot be differentiated again");
    return out;
  }
  void release_variables() override {
    const std::lock_guard<std::mutex> lock(mutex_);
    for (SavedVariable* s : {&x[0], &x[1], &w[0], &w[1], &frequencies, &positions}) s->reset_data();
  }
  std::string name() const override { return "NormRotaryBackward"; }
};

// norm_rotary_embedding(Q, K, q_weight, k_weight, eps, frequencies, interleaved, magnitude, positions, V) -> (Q', K'), differentiable.  V: of the same pass, or None.
PyObject* py_norm_rotary_embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 10);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), v = maybe(a[9]);
    const Norm norm = {maybe(a[2]), maybe(a[3]), number(a[4])};
    const Rotation r = {maybe(a[5]), maybe(a[8]), truth(a[6]), false, number(a[7])};
    check_rotation(q, k, r);
    check_no_lost_positions(r);
    check_norm(q, k, norm);
    const c10::DeviceGuard guard(q.device());
    const bool track = torch::autograd::compute_requires_grad(q, k, norm.wq, norm.wk);
    if (at::GradMode::is_enabled()) refuse_eager_graphs({&q, &k, &v, &norm.wq, &norm.wk});
    at::Tensor qo = output_like(q), ko = output_like(k);
    check_status(without_gil([&] { return norm_rotate(q, k, qo, ko, norm, r); }), "attn_norm_rotary");
    if (track) {
      const std::shared_ptr<NormRotaryBackward> node(new NormRotaryBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(q, k, norm.wq, norm.wk));
      node->x[0] = SavedVariable(q, false);
      node->x[1] = SavedVariable(k, false);
      node->w[0] = SavedVariable(norm.wq, false);
      node->w[1] = SavedVariable(norm.wk, false);
      node->frequencies = SavedVariable(r.frequencies, false);
      node->positions = SavedVariable(r.positions, false);
      node->pairs = r.frequencies.defined() ? r.frequencies.size(0) : 0;
      node->interleaved = r.interleaved;
      node->magnitude = r.magnitude;
      node->eps = norm.eps;
      torch::autograd::set_history(qo, node);
      torch::autograd::set_history(ko, node);
    }
    return tuple({wrap(qo), wrap(ko)});
  });
}

// ---- the paged cache

// What the calls share: caches, table, lengths, starts.
struct Batch { at::Tensor kc, vc, table, lengths, starts; };
Batch batch_of(PyObject* const* a) { return {tensor(a[0]), tensor(a[1]), tensor(a[2]), tensor(a[3]), maybe(a[4])}; }

void check_caches(const at::Tensor& kc, const at::Tensor& vc, int64_t dims) {
  const char* text = dims == 4 ? "expected caches [pages,Hk,page_size,d] with contiguous last axis" : "expected caches [layers,pages,Hk,page_size,d] with contiguous last axis";
  expect_rows(kc, dims, text);
  if (vc.sizes() != kc.sizes() || vc.strides() != kc.strides() || vc.scalar_type() != kc.scalar_type())
    raise(PyExc_ValueError, "the caches of K and V must share shape, strides and type");
  dtype_of(kc, "the caches");
}
// rows: [T, heads, d], one of the call's token tensors
attn_paged_params params_of(const at::Tensor& rows, const Batch& b) {
  expect_rows(rows, 3, "expected a [T,heads,d] tensor with contiguous last axis");
  check_caches(b.kc, b.vc, 4);
  if (rows.scalar_type() != b.kc.scalar_type() || rows.size(2) != b.kc.size(3)) raise(PyExc_ValueError, "tokens and caches must share type and head dimension");
  const int64_t B = b.lengths.dim() == 1 ? b.lengths.size(0) : -1;
  expect_ints(b.lengths, B >= 0 && b.lengths.is_contiguous(), "lengths must be a contiguous int32 tensor [B]");
  expect_ints(b.table, b.table.dim() == 2 && b.table.size(0) == B && (b.table.size(1) <= 1 || b.table.stride(1) == 1),
              "block_table must be an int32 tensor [B,table_width] with contiguous last axis");
  if (b.starts.defined())
    expect_ints(b.starts, b.starts.dim() == 1 && b.starts.size(0) == B + 1 && b.starts.is_contiguous(), "query_starts must be a contiguous int32 tensor [B + 1]");
  attn_paged_params p = {};
  p.B = narrow(B); p.T = narrow(rows.size(0));
  p.Hk = narrow(b.kc.size(1)); p.d = narrow(rows.size(2));
  p.dtype = dtype_of(rows, "tokens");
  p.pages = narrow(b.kc.size(0)); p.page_size = narrow(b.kc.size(2)); p.table_width = narrow(b.table.size(1));
  p.page_stride = axis_stride(b.kc, 0); p.head_stride = axis_stride(b.kc, 1); p.row_stride = axis_stride(b.kc, 2);
  p.table_stride = axis_stride(b.table, 0);
  p.block_table = (const int32_t*)b.table.data_ptr();
  p.lengths = (const int32_t*)b.lengths.data_ptr();
  p.query_starts = (const int32_t*)ptr(b.starts);
  return p;
}
// the last check of a call
void expect_gpu(const at::Tensor& rows, const Batch& b, std::initializer_list<const at::Tensor*> others) {
  expect_gpu(rows, {&b.kc, &b.vc, &b.table, &b.lengths, &b.starts});
  expect_gpu(rows, others);
}

// paged_append(K, V, k_cache, v_cache, block_table, lengths, query_starts, Q, frequencies, interleaved, magnitude, out[, q_weight, k_weight, eps]) -> the turned Q, or None
PyObject* append(PyObject* const* a, Py_ssize_t n, bool normed) {
  return guarded([&]() -> PyObject* {
    expect_args(n, normed ? 15 : 12);
    const at::Tensor &k = tensor(a[0]), &v = tensor(a[1]);
    const Batch b = batch_of(a + 2);
    attn_paged_params p = params_of(k, b);
    expect_like(v, k, "V");
    expect_rows(v, 3, "expected a [T,heads,d] tensor with contiguous last axis");
    if (k.size(1) != b.kc.size(1)) raise(PyExc_ValueError, "K and the caches must have the same number of heads");
    p.k_stride_t = axis_stride(k, 0); p.k_stride_h = axis_stride(k, 1); p.v_stride_t = axis_stride(v, 0); p.v_stride_h = axis_stride(v, 1);
    p.Hq = p.Hk;
    const at::Tensor q = maybe(a[7]), f = maybe(a[8]);
    at::Tensor out = maybe(a[11]);
    attn_rotary_spec spec = {};
    if (f.defined()) {
      check_frequencies(f);
      spec = spec_of(f, truth(a[9]), number(a[10]));
    }
    if (q.defined()) {
      if (!f.defined() && !normed) raise(PyExc_ValueError, "Q is taken only with a rotation");
      expect_rows(q, 3, "expected a [T,heads,d] tensor with contiguous last axis");
      if (q.scalar_type() != k.scalar_type() || q.size(0) != k.size(0) || q.size(2) != k.size(2)) raise(PyExc_ValueError, "Q and K must share type, tokens and head dimension");
      if (out.defined()) {
        expect_like(out, q, "out");
        expect_rows(out, 3, "expected a [T,heads,d] tensor with contiguous last axis");
      }
    } else if (out.defined()) {
      raise(PyExc_ValueError, "an output for Q without Q");
    }
    expect_gpu(k, b, {&v, &q, &f, &out});
    attn_norm_spec norm = {};
    Norm weights = {};
    if (normed) {
      weights = {maybe(a[12]), maybe(a[13]), number(a[14])};
      if (!weights.wk.defined()) raise(PyExc_ValueError, "the norm has no weights for a tensor that is given");
      if (!q.defined()) weights.wq = weights.wk;   // (of no use then)
      check_norm(k, k, weights);
      norm = norm_spec(weights);
    }
    const c10::DeviceGuard guard(k.device());
    p.stream = current_stream(k);
    if (q.defined()) {
      if (!out.defined()) out = packed_like(q);
      p.Hq = narrow(q.size(1));
      p.q_stride_t = axis_stride(q, 0); p.q_stride_h = axis_stride(q, 1); p.o_stride_t = axis_stride(out, 0); p.o_stride_h = axis_stride(out, 1);
    }
    check_status(without_gil([&] {
      const attn_rotary_spec* const turn = f.defined() ? &spec : nullptr;
      void* const qo = const_cast<void*>(ptr(out));
      return normed ? norm_lib.append(&p, turn, &norm, k.data_ptr(), v.data_ptr(), b.kc.data_ptr(), b.vc.data_ptr(), ptr(q), qo)
                    : lib.append(&p, turn, k.data_ptr(), v.data_ptr(), b.kc.data_ptr(), b.vc.data_ptr(), ptr(q), qo);
    }), normed ? "attn_paged_norm_append" : "attn_paged_append");
    return !q.defined() ? Py_NewRef(Py_None) : (a[11] != Py_None ? Py_NewRef(a[11]) : wrap(out));
  });
}
PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return append(a, n, false); }
PyObject* py_norm_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return append(a, n, true); }

// paged_fwd(Q, k_cache, v_cache, block_table, lengths, query_starts, softmax_scale, causal, out, lse, workspace[, window, sinks]) -> (O, LSE)
PyObject* forward(PyObject* const* a, Py_ssize_t n, bool windowed) {
  return guarded([&]() -> PyObject* {
    expect_args(n, windowed ? 13 : 11);
    const int32_t window = windowed ? clamped32(a[11]) : 0, sinks = windowed ? clamped32(a[12]) : 0;
    if (windowed && (window < 1 || sinks < 0)) raise(PyExc_ValueError, "window must be at least 1, and sinks must not be negative");
    const at::Tensor& q = tensor(a[0]);
    const Batch b = batch_of(a + 1);
    attn_paged_params p = params_of(q, b);
    p.Hq = narrow(q.size(1));
    p.softmax_scale = (float)number(a[6]);
    p.causal = truth(a[7]);
    if (windowed && !p.causal) raise(PyExc_ValueError, "a window needs the causal mask");
    at::Tensor out = maybe(a[8]), lse = maybe(a[9]), ws = maybe(a[10]);
    if (out.defined()) {
      expect_like(out, q, "out");
      expect_rows(out, 3, "expected a [T,heads,d] tensor with contiguous last axis");
    }
    if (lse.defined() && (lse.scalar_type() != at::kFloat || lse.dim() != 2 || lse.size(0) != q.size(1) || lse.size(1) != q.size(0) || !lse.is_contiguous()))
      raise(PyExc_ValueError, "lse must be a contiguous float32 tensor [Hq,T]");
    if (ws.defined() && !ws.is_contiguous()) raise(PyExc_ValueError, "the workspace must be contiguous");
    expect_gpu(q, b, {&out, &lse, &ws});
    const c10::DeviceGuard guard(q.device());
    p.stream = current_stream(q);
    if (!out.defined()) out = packed_like(q);
    if (!lse.defined()) lse = at::empty({q.size(1), q.size(0)}, q.options().dtype(at::kFloat));
    p.q_stride_t = axis_stride(q, 0); p.q_stride_h = axis_stride(q, 1); p.o_stride_t = axis_stride(out, 0); p.o_stride_h = axis_stride(out, 1);
    if (!ws.defined()) ws = at::empty({(int64_t)std::max<size_t>(lib.workspace_bytes(&p), 256)}, q.options().dtype(at::kByte));
    check_status(without_gil([&] {
      const size_t bytes = (size_t)ws.numel() * ws.element_size();
      return windowed ? window_fwd(&p, window, sinks, q.data_ptr(), b.kc.data_ptr(), b.vc.data_ptr(), out.data_ptr(), (float*)lse.data_ptr(), ws.data_ptr(), bytes)
                      : lib.fwd(&p, q.data_ptr(), b.kc.data_ptr(), b.vc.data_ptr(), out.data_ptr(), (float*)lse.data_ptr(), ws.data_ptr(), bytes);
    }), windowed ? "attn_paged_window_fwd" : "attn_paged_fwd");
    return tuple({a[8] != Py_None ? Py_NewRef(a[8]) : wrap(out), a[9] != Py_None ? Py_NewRef(a[9]) : wrap(lse)});
  });
}
PyObject* py_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return forward(a, n, false); }
PyObject* py_window_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return forward(a, n, true); }

// paged_workspace_bytes(Q, k_cache, sequences) -> bytes; 0: the sizes are refused
PyObject* py_workspace_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 3);
    const at::Tensor &q = tensor(a[0]), &kc = tensor(a[1]);
    expect_rows(q, 3, "expected a [T,heads,d] tensor with contiguous last axis");
    check_caches(kc, kc, 4);
    attn_paged_params p = {};
    p.B = narrow((int64_t)low64(a[2])); p.T = narrow(q.size(0)); p.Hq = narrow(q.size(1)); p.Hk = narrow(kc.size(1)); p.d = narrow(q.size(2));
    p.dtype = dtype_of(q, "tokens");
    p.pages = narrow(kc.size(0)); p.page_size = narrow(kc.size(2)); p.table_width = 1;
    p.softmax_scale = 1.f;
    p.page_stride = axis_stride(kc, 0); p.head_stride = axis_stride(kc, 1); p.row_stride = axis_stride(kc, 2);
    p.q_stride_t = p.o_stride_t = q.size(1) * q.size(2);
    p.q_stride_h = p.o_stride_h = q.size(2);
    int32_t some_starts = 0;
    p.query_starts = &some_starts;   // (nothing is read: the size is the same with and without)
    return PyLong_FromSize_t(lib.workspace_bytes(&p));
  });
}

// paged_copy(k_cache, v_cache, pairs)
PyObject* py_copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 3);
    const at::Tensor &kc = tensor(a[0]), &vc = tensor(a[1]), &pairs = tensor(a[2]);
    const bool layered = kc.dim() == 5;
    check_caches(kc, vc, layered ? 5 : 4);
    if (pairs.scalar_type() != at::kInt || pairs.dim() != 2 || pairs.size(1) != 2 || !pairs.is_contiguous() || !pairs.is_cpu())
      raise(PyExc_TypeError, "pairs must be a contiguous int32 tensor [n,2] on the CPU");
    expect_gpu(kc, {&vc});
    const int64_t l = layered ? 1 : 0;
    attn_paged_copy_params p = {};
    p.layers = layered ? narrow(kc.size(0)) : 1;
    p.pages = narrow(kc.size(l)); p.Hk = narrow(kc.size(l + 1)); p.page_size = narrow(kc.size(l + 2)); p.d = narrow(kc.size(l + 3));
    p.dtype = dtype_of(kc, "the caches");
    p.layer_stride = layered ? axis_stride(kc, 0) : 0;
    p.page_stride = axis_stride(kc, l); p.head_stride = axis_stride(kc, l + 1); p.row_stride = axis_stride(kc, l + 2);
    p.stream = current_stream(kc);
    const c10::DeviceGuard guard(kc.device());
    check_status(without_gil([&] {
      return lib.copy(&p, kc.data_ptr(), vc.data_ptr(), (const int32_t*)pairs.data_ptr(), pairs.size(0));
    }), "attn_paged_copy");
    Py_RETURN_NONE;
  });
}

// attach_paged(addresses of attn_rotary, attn_paged_append, attn_paged_workspace_bytes, attn_paged_fwd, attn_paged_copy)
PyObject* py_attach(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 5) raise(PyExc_TypeError, "attach_paged() takes five addresses");
    Library l;
    l.rotary = (decltype(l.rotary))low64(a[0]);
    l.append = (decltype(l.append))low64(a[1]);
    l.workspace_bytes = (decltype(l.workspace_bytes))low64(a[2]);
    l.fwd = (decltype(l.fwd))low64(a[3]);
    l.copy = (decltype(l.copy))low64(a[4]);
    lib = l;
    Py_RETURN_NONE;
  });
}

// attach_paged_window(address of attn_paged_window_fwd)
PyObject* py_attach_window(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 1) raise(PyExc_TypeError, "attach_paged_window() takes one address");
    window_fwd = (decltype(window_fwd))low64(a[0]);
    Py_RETURN_NONE;
  });
}

// attach_norm(addresses of attn_norm_rotary, attn_norm_rotary_bwd_workspace_bytes, attn_norm_rotary_bwd, attn_paged_norm_append)
PyObject* py_attach_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 4) raise(PyExc_TypeError, "attach_norm() takes four addresses");
    NormLibrary l;
    l.fwd = (decltype(l.fwd))low64(a[0]);
    l.workspace_bytes = (decltype(l.workspace_bytes))low64(a[1]);
    l.bwd = (decltype(l.bwd))low64(a[2]);
    l.append = (decltype(l.append))low64(a[3]);
    norm_lib = l;
    Py_RETURN_NONE;
  });
}

}  // namespace

// The node that sums a leaf's gradient lives as long as any graph that leads to the leaf, and keeps the stream it was made on.  A captured backward pass that meets one of the
// default stream makes that stream wait for the capture, which ends the process; so the forward pass refuses.  In a model the leaves are weights, behind other operations: all
// nodes that a backward pass from these tensors reaches are looked at (under capture alone: once in the life of a graph).
void marshal::refuse_eager_graphs(std::initializer_list<const at::Tensor*> tensors) {
  using torch::autograd::Node;
  if (c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None) return;
  std::vector<std::shared_ptr<Node>> todo;
  std::unordered_set<const Node*> seen;
  for (const at::Tensor* t : tensors) {
    if (!t->defined() || !t->requires_grad()) continue;
    todo.push_back(t->is_leaf() ? torch::autograd::impl::try_get_grad_accumulator(*t) : t->grad_fn());
  }
  while (!todo.empty()) {
    const std::shared_ptr<Node> node = std::move(todo.back());
    todo.pop_back();
    if (node == nullptr || !seen.insert(node.get()).second) continue;
    if (node->stream().has_value() && node->stream()->id() == 0)
      raise(PyExc_RuntimeError, "captured while a graph made on the default stream still leads to the same leaf: drop that graph (its outputs) first, or make it on another stream");
    for (const torch::autograd::Edge& e : node->next_edges()) todo.push_back(e.function);
  }
}

void marshal::mark_once_differentiable(const torch::autograd::Node& node, variable_list& grads, const char* text) {
  if (!at::GradMode::is_enabled()) return;
  torch::autograd::edge_list edges = node.next_edges();
  const std::shared_ptr<torch::autograd::Node> error(new torch::autograd::Error(text, std::move(edges)), torch::autograd::deleteNode);
  for (at::Tensor& g : grads)
    if (g.defined()) torch::autograd::set_history(g, error);
}

PyMethodDef marshal::paged_methods[] = {
    {"attach_paged_window", (PyCFunction)(void*)py_attach_window, METH_FASTCALL, nullptr},
    {"paged_window_fwd", (PyCFunction)(void*)py_window_fwd, METH_FASTCALL, nullptr},
    {"attach_norm", (PyCFunction)(void*)py_attach_norm, METH_FASTCALL, nullptr},
    {"norm_rotary", (PyCFunction)(void*)py_norm_rotary, METH_FASTCALL, nullptr},
    {"norm_rotary_bwd", (PyCFunction)(void*)py_norm_rotary_bwd, METH_FASTCALL, nullptr},
    {"norm_rotary_embedding", (PyCFunction)(void*)py_norm_rotary_embedding, METH_FASTCALL, nullptr},
    {"paged_norm_append", (PyCFunction)(void*)py_norm_append, METH_FASTCALL, nullptr},
    {"attach_paged", (PyCFunction)(void*)py_attach, METH_FASTCALL, nullptr},
    {"rotary", (PyCFunction)(void*)py_rotary, METH_FASTCALL, nullptr},
    {"rotary_embedding", (PyCFunction)(void*)py_rotary_embedding, METH_FASTCALL, nullptr},
    {"paged_append", (PyCFunction)(void*)py_append, METH_FASTCALL, nullptr},
    {"paged_fwd", (PyCFunction)(void*)py_fwd, METH_FASTCALL, nullptr},
    {"paged_workspace_bytes", (PyCFunction)(void*)py_workspace_bytes, METH_FASTCALL, nullptr},
    {"paged_copy", (PyCFunction)(void*)py_copy, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
