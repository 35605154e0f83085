// The host sides of the packed and paged calls, for the functions of the same names in binding.py: checking and marshalling in
// Python takes 10 to 15 us a call, and the smallest ones 3 to 9 us on the device (a prompt of 128 tokens of 12 heads and its way
// into the cache: 31 us among others, 9 with this; a token of one user over 2047: 26 and 9).
//
// Every function takes the library's entry points by address, the binding's arguments and the stream (or None), and returns
// the gf_status of the call, or None for anything that is not the plain, well-formed call: wrapped tensors, shapes, types or
// devices that do not fit, numbers out of range.  The binding's own code then does or refuses the call, with its own messages.
#include "call.hpp"

#include <ATen/Functions.h>
#include <c10/core/impl/VirtualGuardImpl.h>

#include <initializer_list>

namespace gformer_host {
namespace {

// Strides of [rows, heads, d] or [pages, heads, tokens, d] without the last, those of single rows as if the tensor were
// dense; false where the binding would refuse them.
template <int N> bool row_strides(const at::Tensor& t, int64_t (&out)[N]) {
  const auto n = t.sizes(), s = t.strides();
  if (s[N] != 1 && n[N] > 1) return false;
  int64_t dense = n[N];
  for (int i = N - 1; i >= 0; --i) {
    if (n[i] > 1 && s[i] == 0) return false;
    out[i] = n[i] > 1 ? s[i] : dense;
    dense *= n[i] > 1 ? n[i] : 1;
  }
  return true;
}

bool fits_int(int64_t x) { return x >= 0 && x <= INT_MAX; }

struct Call {
  const at::Tensor* like = nullptr;
  int64_t stream = 0;
  bool named = false;    // the caller named the stream

  // tensors of one type and n dimensions
  bool tensors(std::initializer_list<const at::Tensor*> all, int dims) {
    for (const at::Tensor* t : all) {
      if (!t || t->dim() != dims) return false;
      if (!like) {
        if (t->scalar_type() != at::kBFloat16 && t->scalar_type() != at::kFloat) return false;
        like = t;
      } else if (t->scalar_type() != like->scalar_type()) {
        return false;
      }
      for (const int64_t n : t->sizes())
        if (!fits_int(n)) return false;
    }
    return true;
  }
  int32_t dtype() const { return like->scalar_type() == at::kBFloat16 ? GF_BF16 : GF_F32; }
  bool stream_of(PyObject* o) {
    named = o != Py_None;
    return !named || to_long(o, 0, LLONG_MAX, stream);
  }
  // Asked last, so that host tensors go through all of the above: all on the current device.
  bool device(std::initializer_list<const at::Tensor*> all) const {
    if (!like->is_cuda()) return false;
    const auto index = like->get_device();
    for (const at::Tensor* t : all)
      if (t && (!t->is_cuda() || t->get_device() != index)) return false;
    return c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index() == index;
  }
};

const at::Tensor* numbers(PyObject* o, int dims) {
  const at::Tensor* t = plain(o);
  return t && t->scalar_type() == at::kInt && t->dim() == dims ? t : nullptr;
}
// A tensor or None; `ok` turns false for anything else.
const at::Tensor* optional(PyObject* o, bool& ok) {
  if (o == Py_None) return nullptr;
  const at::Tensor* t = strided(o);
  ok = ok && t;
  return t;
}
void* at_of(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
const int32_t* ints(const at::Tensor* t) { return static_cast<const int32_t*>(at_of(t)); }

// Runs `gather`, which leaves the call in `go` (both may throw), with the stream and the interpreter's lock settled.
template <typename G, typename F> PyObject* run(Call& c, G gather, F go) {
  try {   // no C++ exception may leave a function that the interpreter called
    if (!gather()) Py_RETURN_NONE;
  } catch (...) {
    Py_RETURN_NONE;
  }
  if (!c.named) {
    if (!raw_stream_getter) Py_RETURN_NONE;
    if (!current_stream(c.like->get_device(), c.stream)) return nullptr;
  }
  gf_status st;
  Py_BEGIN_ALLOW_THREADS
  st = go(reinterpret_cast<void*>(c.stream));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

PyObject* wrong_count(const char* what) {
  PyErr_SetString(PyExc_TypeError, what);
  return nullptr;
}
template <typename F> F address(PyObject* o) { return reinterpret_cast<F>(PyLong_AsVoidPtr(o)); }

// The caller's workspace, or one of `need` bytes that `own` holds; false where that is the binding's business.
bool scratch(PyObject* o, size_t need, const Call& c, at::Tensor& own, void*& at, size_t& bytes) {
  at = nullptr;
  bytes = 0;
  if (o != Py_None) {
    const at::Tensor* t = plain(o);
    if (!t || !t->is_cuda() || t->get_device() != c.like->get_device()) return false;
    at = t->data_ptr();
    bytes = (size_t)t->numel() * t->element_size();
  } else if (need) {
    if (c.named) return false;   // it is that stream's memory
    own = at::empty({(int64_t)need}, c.like->options().dtype(at::kByte));
    at = own.data_ptr();
    bytes = need;
  }
  return true;
}

struct Packed {
  const at::Tensor *q, *k, *v, *out, *cu_q, *cu_k;
  int n, tq, tk, H, Hkv, d;
  bool of(Call& c, PyObject* const* a, gformer_packed_params& p) {
    q = strided(a[0]), k = strided(a[1]), v = strided(a[2]), out = strided(a[3]);
    if (!c.tensors({q, k, v, out}, 3) || out->sizes() != q->sizes() || v->sizes() != k->sizes() || k->size(2) != q->size(2)) return false;
    cu_q = numbers(a[4], 1);
    cu_k = a[5] == Py_None ? nullptr : numbers(a[5], 1);
    if (!cu_q || cu_q->numel() < 1 || !fits_int(cu_q->numel()) || (a[5] != Py_None && (!cu_k || cu_k->sizes() != cu_q->sizes()))) return false;
    if (a[5] == Py_None && k->size(0) != q->size(0)) return false;
    n = (int)cu_q->numel() - 1;
    tq = (int)q->size(0), H = (int)q->size(1), d = (int)q->size(2), tk = (int)k->size(0), Hkv = (int)k->size(1);
    std::memset(&p, 0, sizeof(p));
    p.struct_size = sizeof(p);
    p.dtype = c.dtype();
    return row_strides(*q, p.q_stride) && row_strides(*k, p.k_stride) && row_strides(*v, p.v_stride) && row_strides(*out, p.o_stride);
  }
  bool lse(const at::Tensor* t) const {
    return t && t->scalar_type() == at::kFloat && t->dim() == 2 && t->size(0) == H && t->size(1) == tq && t->is_contiguous();
  }
  bool rest(const at::Tensor* t) const {
    return t->scalar_type() == out->scalar_type() && t->sizes() == out->sizes() && t->strides() == out->strides();
  }
};

struct Pages {
  const at::Tensor *k, *v;
  bool of(Call& c, PyObject* ko, PyObject* vo, gformer_paged_params& p) {
    k = strided(ko), v = strided(vo);
    if (!c.tensors({k, v}, 4) || k->sizes() != v->sizes()) return false;
    std::memset(&p, 0, sizeof(p));
    p.struct_size = sizeof(p);
    p.dtype = c.dtype();
    p.page_size = (int32_t)k->size(2);
    p.softmax_scale = 1.f;
    return row_strides(*k, p.kpage_stride) && row_strides(*v, p.vpage_stride);
  }
  int count() const { return (int)k->size(0); }
  int heads() const { return (int)k->size(1); }
  int d() const { return (int)k->size(3); }
};

}  // namespace

// address, q, k, v, out, cu_q, cu_k, lse, out_rest, softmax_scale, zero_tail, stream
PyObject* packed_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 12) return wrong_count("packed_fwd takes 12 arguments");
  Call c;
  Packed x;
  gformer_packed_params p;
  void *lse = nullptr, *rest = nullptr;
  const auto call = address<decltype(&gformer_packed_attn_fwd)>(a[0]);
  return run(c, [&] {
    bool ok = call != nullptr;
    const at::Tensor *l = optional(a[7], ok), *r = optional(a[8], ok);
    int64_t zero;
    if (!ok || !x.of(c, a + 1, p) || (l && !x.lse(l)) || (r && !x.rest(r)) || !to_float(a[9], p.softmax_scale) ||
        !to_long(a[10], INT_MIN, INT_MAX, zero) || !c.stream_of(a[11]) || !c.device({x.q, x.k, x.v, x.out, x.cu_q, x.cu_k, l, r}))
      return false;
    p.zero_tail = (int32_t)zero;
    lse = at_of(l);
    rest = at_of(r);
    return true;
  }, [&](void* s) {
    return call(at_of(x.q), at_of(x.k), at_of(x.v), at_of(x.out), rest, static_cast<float*>(lse), ints(x.cu_q), ints(x.cu_k), x.n, x.tq,
                x.tk, x.H, x.Hkv, x.d, &p, s);
  });
}

// address, address of the workspace's size, q, k, v, out, cu_q, cu_k, lse, dout, dq, dk, dv, out_rest, softmax_scale, zero_tail, workspace, stream
PyObject* packed_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 18) return wrong_count("packed_bwd takes 18 arguments");
  Call c;
  Packed x;
  gformer_packed_params p;
  const at::Tensor *g = nullptr, *dq = nullptr, *dk = nullptr, *dv = nullptr;
  void *lse = nullptr, *rest = nullptr, *ws = nullptr;
  size_t bytes = 0;
  at::Tensor own;
  const auto call = address<decltype(&gformer_packed_attn_bwd)>(a[0]);
  const auto size = address<decltype(&gformer_packed_attn_bwd_workspace_bytes)>(a[1]);
  return run(c, [&] {
    bool ok = call && size;
    const at::Tensor *l = strided(a[8]), *r = optional(a[13], ok);
    g = strided(a[9]), dq = strided(a[10]), dk = strided(a[11]), dv = strided(a[12]);
    int64_t zero;
    if (!ok || !x.of(c, a + 2, p) || !c.tensors({g, dq, dk, dv}, 3) || g->sizes() != x.q->sizes() || dq->sizes() != x.q->sizes() ||
        dk->sizes() != x.k->sizes() || dv->sizes() != x.k->sizes() || !x.lse(l) || (r && !x.rest(r)) || !row_strides(*g, p.do_stride) ||
        !row_strides(*dq, p.dq_stride) || !row_strides(*dk, p.dk_stride) || !row_strides(*dv, p.dv_stride) ||
        !to_float(a[14], p.softmax_scale) || !to_long(a[15], INT_MIN, INT_MAX, zero) || !c.stream_of(a[17]) ||
        !c.device({x.q, x.k, x.v, x.out, x.cu_q, x.cu_k, l, r, g, dq, dk, dv}))
      return false;
    p.zero_tail = (int32_t)zero;
    lse = at_of(l);
    rest = at_of(r);
    return scratch(a[16], size(x.tq, x.tk, x.n, x.H, x.Hkv, x.d, &p), c, own, ws, bytes);
  }, [&](void* s) {
    return call(at_of(x.q), at_of(x.k), at_of(x.v), at_of(x.out), rest, static_cast<float*>(lse), at_of(g), at_of(dq), at_of(dk), at_of(dv),
                ints(x.cu_q), ints(x.cu_k), x.n, x.tq, x.tk, x.H, x.Hkv, x.d, &p, ws, bytes, s);
  });
}

// address, k, v, kpages, vpages, table, start, cu, stream
PyObject* paged_fill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 9) return wrong_count("paged_fill takes 9 arguments");
  Call c;
  Pages x;
  gformer_paged_params p;
  const at::Tensor *k = nullptr, *v = nullptr, *table = nullptr, *start = nullptr, *cu = nullptr;
  const auto call = address<decltype(&gformer_paged_fill)>(a[0]);
  return run(c, [&] {
    k = strided(a[1]), v = strided(a[2]);
    table = numbers(a[5], 2), start = numbers(a[6], 1), cu = numbers(a[7], 1);
    return call && c.tensors({k, v}, 3) && x.of(c, a[3], a[4], p) && k->sizes() == v->sizes() && k->size(1) == x.heads() &&
           k->size(2) == x.d() && row_strides(*k, p.k_stride) && row_strides(*v, p.v_stride) && table && start && cu &&
           cu->numel() >= 1 && fits_int(cu->numel()) && table->size(0) == cu->numel() - 1 && fits_int(table->size(1)) &&
           start->numel() == cu->numel() - 1 && c.stream_of(a[8]) && c.device({k, v, x.k, x.v, table, start, cu});
  }, [&](void* s) {
    return call(at_of(k), at_of(v), at_of(x.k), at_of(x.v), ints(table), ints(start), ints(cu), (int)cu->numel() - 1, (int)k->size(0),
                x.heads(), x.d(), x.count(), (int)table->size(1), &p, s);
  });
}

// address, address of the workspace's size, q, k, v, out, kpages, vpages, table, lens, max_len, softmax_scale, workspace, stream
PyObject* paged_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 14) return wrong_count("paged_decode takes 14 arguments");
  Call c;
  Pages x;
  gformer_paged_params p;
  const at::Tensor *q = nullptr, *k = nullptr, *v = nullptr, *out = nullptr, *table = nullptr, *lens = nullptr;
  int64_t max_len = 0;
  void* ws = nullptr;
  size_t bytes = 0;
  at::Tensor own;
  const auto call = address<decltype(&gformer_paged_decode)>(a[0]);
  const auto size = address<decltype(&gformer_paged_decode_workspace_bytes)>(a[1]);
  return run(c, [&] {
    bool ok = call && size && (a[3] == Py_None) == (a[4] == Py_None);
    q = strided(a[2]), k = optional(a[3], ok), v = optional(a[4], ok), out = strided(a[5]);
    table = numbers(a[8], 2), lens = numbers(a[9], 1);
    if (!ok || !c.tensors({q, out}, 3) || (k && !c.tensors({k, v}, 3)) || !x.of(c, a[6], a[7], p) || out->sizes() != q->sizes() ||
        q->size(2) != x.d() || !table || !lens || table->size(0) != q->size(0) || lens->numel() != q->size(0) || !fits_int(table->size(1)))
      return false;
    if (k) {
      const int64_t rows[3] = {q->size(0), x.heads(), x.d()};
      if (k->sizes() != at::IntArrayRef(rows, 3) || v->sizes() != at::IntArrayRef(rows, 3) || !row_strides(*k, p.k_stride) ||
          !row_strides(*v, p.v_stride))
        return false;
    }
    if (!row_strides(*q, p.q_stride) || !row_strides(*out, p.o_stride) || !to_long(a[10], INT_MIN, INT_MAX, max_len) ||
        !to_float(a[11], p.softmax_scale) || !c.stream_of(a[13]) || !c.device({q, k, v, out, x.k, x.v, table, lens}))
      return false;
    return scratch(a[12], size((int)q->size(0), (int)q->size(1), x.heads(), x.d(), (int)table->size(1), (int)max_len, &p), c, own, ws, bytes);
  }, [&](void* s) {
    return call(at_of(q), at_of(k), at_of(v), at_of(out), at_of(x.k), at_of(x.v), ints(table), ints(lens), (int)q->size(0), (int)q->size(1),
                x.heads(), x.d(), x.count(), (int)table->size(1), (int)max_len, &p, ws, bytes, s);
  });
}

// address, kpages, vpages, src, dst, stream
PyObject* pages_copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) return wrong_count("pages_copy takes 6 arguments");
  Call c;
  Pages x;
  gformer_paged_params p;
  const at::Tensor *src = nullptr, *dst = nullptr;
  const auto call = address<decltype(&gformer_pages_copy)>(a[0]);
  return run(c, [&] {
    src = numbers(a[3], 1), dst = numbers(a[4], 1);
    return call && x.of(c, a[1], a[2], p) && src && dst && fits_int(src->numel()) && src->sizes() == dst->sizes() && c.stream_of(a[5]) &&
           c.device({x.k, x.v, src, dst});
  }, [&](void* s) {
    return call(at_of(x.k), at_of(x.v), ints(src), ints(dst), (int)src->numel(), x.heads(), x.d(), x.count(), &p, s);
  });
}

}  // namespace gformer_host
