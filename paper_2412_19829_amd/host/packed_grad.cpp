// gformer_packed_attention of autograd.py as a node of torch's graph in C++: the wrapper's own Python takes the host 109 us for a
// step of 64 tokens of 8 heads, forward and backward, and 14 us for the forward alone; this takes 80 and 8.
//
// attention(forward, backward, workspace's size, q, k, v, cu_q, cu_k, softmax_scale) takes the library's entry points by address
// and returns the output, the gf_status of a forward call that failed, or None for what is not the plain, well-formed
// call, which the wrapper's own code then does or refuses.
#include "call.hpp"

#include <ATen/Functions.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>

#include <algorithm>
#include <memory>
#include <stdexcept>
#include <string>

namespace gformer_host {
namespace {

using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

struct Entries {
  decltype(&gformer_packed_attn_fwd) fwd;
  decltype(&gformer_packed_attn_bwd) bwd;
  decltype(&gformer_packed_attn_bwd_workspace_bytes) workspace;
};
Entries entries = {};   // the process has one library

// (row, head) strides, those of single rows as if the tensor were dense; false where the library would not take them.
bool strides(const at::Tensor& t, int64_t (&out)[2]) {
  const auto n = t.sizes(), s = t.strides();
  if (s[2] != 1 && n[2] > 1) return false;
  out[1] = n[1] > 1 ? s[1] : n[2];
  out[0] = n[0] > 1 ? s[0] : n[2] * std::max<int64_t>(n[1], 1);
  return out[0] >= n[2] && out[1] >= n[2] && out[0] % 8 == 0 && out[1] % 8 == 0 && out[0] <= 1 << 20;
}
bool fits(const at::Tensor& t, int64_t (&out)[2]) { return strides(t, out) && ((uintptr_t)t.data_ptr() & 15) == 0; }

const int32_t* ints(const at::Tensor& t) { return t.defined() ? static_cast<const int32_t*>(t.data_ptr()) : nullptr; }

struct Attention : torch::autograd::Function<Attention> {
  static at::Tensor forward(AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor* starts_q,
                            const at::Tensor* starts_k, const gformer_packed_params& params, int64_t stream, bool keep,
                            gf_status* status) {
    const at::Tensor& cu_q = *starts_q;
    const at::Tensor cu_k = starts_k ? *starts_k : at::Tensor();
    gformer_packed_params p = params;
    const at::Tensor out = at::empty(q.sizes(), q.options());
    const at::Tensor lse = at::empty({q.size(1), q.size(0)}, q.options().dtype(at::kFloat));
    const at::Tensor rest = keep && p.dtype == GF_BF16 ? at::empty(q.sizes(), q.options()) : at::Tensor();
    *status = entries.fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), rest.defined() ? rest.data_ptr() : nullptr,
                    static_cast<float*>(lse.data_ptr()), ints(cu_q), ints(cu_k), (int)cu_q.numel() - 1, (int)q.size(0), (int)k.size(0),
                    (int)q.size(1), (int)k.size(1), (int)q.size(2), &p, reinterpret_cast<void*>(stream));
    if (keep) {
      ctx->save_for_backward({q, k, v, out, rest, lse, cu_q, cu_k});
      ctx->saved_data["softmax_scale"] = (double)p.softmax_scale;
    }
    return out;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    variable_list none(9);    // one for each argument of forward
    if (!grads[0].defined()) return none;
    const variable_list saved = ctx->get_saved_variables();
    const at::Tensor &q = saved[0], &k = saved[1], &v = saved[2], &out = saved[3], &rest = saved[4], &lse = saved[5], &cu_q = saved[6],
                     &cu_k = saved[7];
    variable_list result(3);
    {
      at::NoGradGuard no_grad;
      const c10::DeviceGuard guard(q.device());
      gformer_packed_params p;
      std::memset(&p, 0, sizeof(p));
      p.struct_size = sizeof(p);
      p.dtype = q.scalar_type() == at::kBFloat16 ? GF_BF16 : GF_F32;
      p.zero_tail = 1;
      p.softmax_scale = (float)ctx->saved_data["softmax_scale"].toDouble();
      // a gradient may come in any layout: broadcast, or strided as the library does not take it
      at::Tensor g = grads[0];
      if (!fits(g, p.do_stride)) {
        g = g.contiguous();
        if (!fits(g, p.do_stride)) g = g.clone(at::MemoryFormat::Contiguous);
        fits(g, p.do_stride);
      }
      strides(q, p.q_stride);
      strides(k, p.k_stride);
      strides(v, p.v_stride);   // out and the gradients are dense
      for (int i = 0; i < 3; ++i) result[i] = at::empty(saved[i].sizes(), saved[i].options());
      const int n = (int)cu_q.numel() - 1, tq = (int)q.size(0), tk = (int)k.size(0), H = (int)q.size(1), Hkv = (int)k.size(1), d = (int)q.size(2);
      const int64_t bytes = (int64_t)entries.workspace(tq, tk, n, H, Hkv, d, &p);
      const at::Tensor workspace = at::empty({std::max<int64_t>(bytes, 1)}, q.options().dtype(at::kByte));
      int64_t stream = 0;
      const PyGILState_STATE lock = PyGILState_Ensure();   // the engine's thread has its own current stream
      const bool known = current_stream(q.get_device(), stream);
      if (!known) PyErr_Clear();
      PyGILState_Release(lock);
      if (!known) throw std::runtime_error("the current stream is not known");
      const gf_status st = entries.bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), rest.defined() ? rest.data_ptr() : nullptr,
                               static_cast<const float*>(lse.data_ptr()), g.data_ptr(), result[0].data_ptr(), result[1].data_ptr(),
                               result[2].data_ptr(), ints(cu_q), ints(cu_k), n, tq, tk, H, Hkv, d, &p, workspace.data_ptr(), (size_t)bytes,
                               reinterpret_cast<void*>(stream));
      if (st != GF_OK) throw std::runtime_error("gformer status " + std::to_string((int)st) + " in the backward pass of packed attention");
    }
    if (c10::GradMode::is_enabled()) {   // create_graph: the gradients have none, and say so when they are asked for theirs
      for (auto& t : result) t.set_requires_grad(true);
      auto error = std::make_shared<torch::autograd::DelayedError>("packed attention is differentiable once", 3);
      result = (*error)(std::move(result));
    }
    for (int i = 0; i < 3; ++i) none[i] = result[i];
    return none;
  }
};

}  // namespace

PyObject* packed_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 9) {
    PyErr_SetString(PyExc_TypeError, "attention takes 9 arguments");
    return nullptr;
  }
  try {   // no C++ exception may leave a function that the interpreter called
    const at::Tensor *q = strided(a[3]), *k = strided(a[4]), *v = strided(a[5]), *cu_q = plain(a[6]);
    const at::Tensor* cu_k = a[7] == Py_None ? nullptr : plain(a[7]);
    if (!q || !k || !v || !cu_q || (a[7] != Py_None && !cu_k) || !raw_stream_getter) Py_RETURN_NONE;
    const auto type = q->scalar_type();
    if ((type != at::kBFloat16 && type != at::kFloat) || k->scalar_type() != type || v->scalar_type() != type || q->dim() != 3 ||
        k->dim() != 3 || k->sizes() != v->sizes() || q->size(2) != k->size(2))
      Py_RETURN_NONE;
    for (const at::Tensor* c : {cu_q, cu_k})
      if (c && (c->scalar_type() != at::kInt || c->dim() != 1 || c->numel() < 1 || c->numel() > INT_MAX || c->numel() != cu_q->numel()))
        Py_RETURN_NONE;
    if (!cu_k && q->size(0) != k->size(0)) Py_RETURN_NONE;
    for (int i = 0; i < 3; ++i)
      if (q->size(i) > INT_MAX || k->size(i) > INT_MAX) Py_RETURN_NONE;
    gformer_packed_params p;
    std::memset(&p, 0, sizeof(p));
    p.struct_size = sizeof(p);
    p.dtype = type == at::kBFloat16 ? GF_BF16 : GF_F32;
    p.zero_tail = 1;
    if (!to_float(a[8], p.softmax_scale) || !strides(*q, p.q_stride) || !strides(*k, p.k_stride) || !strides(*v, p.v_stride)) Py_RETURN_NONE;
    if (!q->is_cuda()) Py_RETURN_NONE;
    const auto index = q->get_device();
    for (const at::Tensor* t : {k, v, cu_q, cu_k})
      if (t && (!t->is_cuda() || t->get_device() != index)) Py_RETURN_NONE;
    if (c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index() != index) Py_RETURN_NONE;
    entries = {reinterpret_cast<decltype(Entries::fwd)>(PyLong_AsVoidPtr(a[0])),
                       reinterpret_cast<decltype(Entries::bwd)>(PyLong_AsVoidPtr(a[1])),
                       reinterpret_cast<decltype(Entries::workspace)>(PyLong_AsVoidPtr(a[2]))};
    if (!entries.fwd || !entries.bwd || !entries.workspace) Py_RETURN_NONE;
    int64_t stream = 0;
    if (!current_stream(index, stream)) return nullptr;
    const bool keep = c10::GradMode::is_enabled() && (q->requires_grad() || k->requires_grad() || v->requires_grad());
    gf_status st = GF_OK;
    const at::Tensor out = Attention::apply(*q, *k, *v, cu_q, cu_k, p, stream, keep, &st);
    return st == GF_OK ? THPVariable_Wrap(out) : PyLong_FromLong((long)st);
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

}  // namespace gformer_host
