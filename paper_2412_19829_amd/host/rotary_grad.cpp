// gformer_rotary_positions of autograd.py as a node of torch's graph in C++: the wrapper's own Python takes the host about as long for a
// step of 8192 rows, both ways, as the device.
//
// rotary_positions(entry, q, k, freqs, positions, cu, start, interleaved, factor) takes the library's entry point by address and
// returns the pair of outputs, the gf_status of a call that failed, or None for what is not the plain, well-formed call, which the
// wrapper's own code then does or refuses.  The backward pass is the same node, turning back, and so differentiable again.
#include "call.hpp"

#include <ATen/Functions.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/custom_function.h>

#include <algorithm>
#include <stdexcept>
#include <string>

namespace gformer_host {
namespace {

using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

decltype(&gformer_rotary) entry = nullptr;   // the process has one library

// (row, head) strides, those of single rows as if the tensor were dense; false where the library would not take them.
bool strides(const at::Tensor& t, int64_t (&out)[2]) {
  const auto n = t.sizes(), s = t.strides();
  if (s[2] != 1 && n[2] > 1) return false;
  out[1] = n[1] > 1 ? s[1] : n[2];
  out[0] = n[0] > 1 ? s[0] : n[2] * std::max<int64_t>(n[1], 1);
  return out[0] >= n[2] && out[1] >= n[2] && out[0] % 8 == 0 && out[1] % 8 == 0 && out[0] <= 1 << 20;
}
bool fits(const at::Tensor& t, int64_t (&out)[2]) { return strides(t, out) && ((uintptr_t)t.data_ptr() & 15) == 0; }
// Gradients come in any layout.
at::Tensor taken(const at::Tensor& t, int64_t (&out)[2]) {
  if (!t.defined() || fits(t, out)) return t;
  const at::Tensor x = t.clone(at::MemoryFormat::Contiguous);
  fits(x, out);
  return x;
}
template <typename P> P at_of(const at::Tensor& t) { return t.defined() ? static_cast<P>(t.data_ptr()) : nullptr; }

struct How {
  at::Tensor where[4];   // frequencies, positions, offsets, starts
  int64_t interleaved = 0, inverse = 0, stream = 0;
  double factor = 1.0;
  bool keep = false;
  gf_status status = GF_OK;
};

// The turned rows of q and, where it is defined, of k.
variable_list turned(AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k, How* how) {
  const at::Tensor &freqs = how->where[0], &cu = how->where[2];
  gformer_rotary_params p;
  std::memset(&p, 0, sizeof(p));
  p.struct_size = sizeof(p);
  p.rot = (int32_t)(2 * freqs.numel());
  p.interleaved = (int32_t)how->interleaved;
  p.inverse = (int32_t)how->inverse;
  p.zero_tail = 1;
  p.factor = (float)how->factor;
  const at::Tensor a = taken(q, p.q_stride), b = taken(k, p.k_stride);
  p.dtype = a.scalar_type() == at::kBFloat16 ? GF_BF16 : GF_F32;
  variable_list out{at::empty(a.sizes(), a.options())};
  if (b.defined()) out.push_back(at::empty(b.sizes(), b.options()));
  how->status = entry(a.data_ptr(), at_of<const void*>(b), out[0].data_ptr(), b.defined() ? out[1].data_ptr() : nullptr, at_of<const float*>(freqs),
                      at_of<const int32_t*>(how->where[1]), at_of<const int32_t*>(cu), at_of<const int32_t*>(how->where[3]),
                      cu.defined() ? (int)cu.numel() - 1 : 0, (int)a.size(0), (int)a.size(1), b.defined() ? (int)b.size(1) : 0, (int)a.size(2),
                      &p, reinterpret_cast<void*>(how->stream));
  ctx->set_materialize_grads(false);
  if (how->keep) {
    ctx->save_for_backward({how->where[0], how->where[1], how->where[2], how->where[3]});
    ctx->saved_data["interleaved"] = how->interleaved;
    ctx->saved_data["inverse"] = how->inverse;
    ctx->saved_data["factor"] = how->factor;
  }
  return out;
}

// How the gradients of such rows turn back.
How back(AutogradContext* ctx, const at::Tensor& like) {
  How how;
  const variable_list saved = ctx->get_saved_variables();
  for (int i = 0; i < 4; ++i) how.where[i] = saved[i];
  how.interleaved = ctx->saved_data["interleaved"].toInt();
  how.inverse = 1 - ctx->saved_data["inverse"].toInt();
  how.factor = ctx->saved_data["factor"].toDouble();
  how.keep = c10::GradMode::is_enabled();   // create_graph
  const PyGILState_STATE lock = PyGILState_Ensure();   // the engine's thread has its own current stream
  const bool known = current_stream(like.get_device(), how.stream);
  if (!known) PyErr_Clear();
  PyGILState_Release(lock);
  if (!known) throw std::runtime_error("the current stream is not known");
  return how;
}
void succeeded(const How& how) {
  if (how.status != GF_OK) throw std::runtime_error("gformer status " + std::to_string((int)how.status) + " in the backward pass of rotary positions");
}

// Nodes of one tensor and of two: a node's inputs are all defined.
struct RotaryOne : torch::autograd::Function<RotaryOne> {
  static variable_list forward(AutogradContext* ctx, const at::Tensor& x, How* how) { return turned(ctx, x, at::Tensor(), how); }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    variable_list out(2);   // one for each argument of forward
    if (!grads[0].defined()) return out;
    const c10::DeviceGuard guard(grads[0].device());
    How how = back(ctx, grads[0]);
    out[0] = RotaryOne::apply(grads[0], &how)[0];
    succeeded(how);
    return out;
  }
};
struct RotaryTwo : torch::autograd::Function<RotaryTwo> {
  static variable_list forward(AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k, How* how) { return turned(ctx, q, k, how); }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    variable_list out(3);
    const bool q = grads[0].defined() && ctx->needs_input_grad(0), k = grads[1].defined() && ctx->needs_input_grad(1);
    if (!q && !k) return out;
    const at::Tensor& like = q ? grads[0] : grads[1];
    const c10::DeviceGuard guard(like.device());
    How how = back(ctx, like);
    const variable_list got = q && k ? RotaryTwo::apply(grads[0], grads[1], &how) : RotaryOne::apply(like, &how);
    succeeded(how);
    if (q) out[0] = got.front();
    if (k) out[1] = got.back();
    return out;
  }
};

bool ints(const at::Tensor* t, int64_t n) {
  return t->scalar_type() == at::kInt && t->dim() == 1 && t->numel() <= INT_MAX && (n < 0 || t->numel() == n);
}

}  // namespace

PyObject* rotary_positions(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 9) {
    PyErr_SetString(PyExc_TypeError, "rotary_positions takes 9 arguments");
    return nullptr;
  }
  try {   // no C++ exception may leave a function that the interpreter called
    const at::Tensor *q = strided(a[1]), *k = a[2] == Py_None ? nullptr : strided(a[2]);
    How how;
    at::Tensor (&where)[4] = how.where;
    for (int i = 0; i < 4; ++i) {
      if (i > 0 && a[3 + i] == Py_None) continue;
      const at::Tensor* t = plain(a[3 + i]);
      if (!t) Py_RETURN_NONE;
      where[i] = *t;
    }
    if (!q || (a[2] != Py_None && !k) || !raw_stream_getter) Py_RETURN_NONE;
    const auto type = q->scalar_type();
    if ((type != at::kBFloat16 && type != at::kFloat) || q->dim() != 3 ||
        (k && (k->scalar_type() != type || k->dim() != 3 || k->size(0) != q->size(0) || k->size(2) != q->size(2))))
      Py_RETURN_NONE;
    const at::Tensor &freqs = where[0], &positions = where[1], &cu = where[2], &start = where[3];
    if (freqs.scalar_type() != at::kFloat || freqs.dim() != 1 || 2 * freqs.numel() > INT_MAX) Py_RETURN_NONE;
    if (positions.defined() ? cu.defined() || start.defined() || !ints(&positions, q->size(0))
                            : !cu.defined() || !ints(&cu, -1) || cu.numel() < 1 || (start.defined() && !ints(&start, cu.numel() - 1)))
      Py_RETURN_NONE;
    for (const at::Tensor* t : {q, k})
      for (int i = 0; t && i < 3; ++i)
        if (t->size(i) > INT_MAX) Py_RETURN_NONE;
    float factor;
    if (!to_long(a[7], 0, 1, how.interleaved) || !to_float(a[8], factor)) Py_RETURN_NONE;
    how.factor = factor;
    if (!q->is_cuda()) Py_RETURN_NONE;
    const auto index = q->get_device();
    for (const at::Tensor* t : {k, &freqs, &positions, &cu, &start})
      if (t && t->defined() && (!t->is_cuda() || t->get_device() != index)) Py_RETURN_NONE;
    if (c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index() != index) Py_RETURN_NONE;
    int64_t given[2];
    if (!strides(*q, given) || (k && !strides(*k, given))) Py_RETURN_NONE;
    entry = reinterpret_cast<decltype(entry)>(PyLong_AsVoidPtr(a[0]));
    if (!entry) Py_RETURN_NONE;
    if (!current_stream(index, how.stream)) return nullptr;
    how.keep = c10::GradMode::is_enabled() && (q->requires_grad() || (k && k->requires_grad()));
    const variable_list out = k ? RotaryTwo::apply(*q, *k, &how) : RotaryOne::apply(*q, &how);
    if (how.status != GF_OK) return PyLong_FromLong((long)how.status);
    PyObject* first = THPVariable_Wrap(out[0]);
    PyObject* second = k ? THPVariable_Wrap(out[1]) : (Py_INCREF(Py_None), Py_None);
    PyObject* pair = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return pair;
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

}  // namespace gformer_host
