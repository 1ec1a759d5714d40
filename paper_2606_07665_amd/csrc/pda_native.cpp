// Native argument marshalling of the binding's hot calls (CPython extension).
//
// A small decode call is ~10 us of GPU time; checking its tensors one
// attribute at a time in Python and converting its arguments through ctypes
// took 5-10 us of host time on top of the launches (a prelude with the append
// 14-16 us a call, o_proj 13).  These functions make the same checks on the
// tensors themselves and call the C ABI.
//
// Each returns the library's status code, or kDeclined where anything is not
// the plain accepted case -- another type than a plain torch.Tensor, a wrong
// dtype, shape, device or layout, an argument that is not a number of its
// range.  The caller then takes the Python path, which makes every check
// again in its documented order and raises the specific error, so this file
// decides nothing on its own but the accepted case.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <vector>

#include "pda.h"

namespace {

constexpr int kDeclined = -1;

// Entry points of the loaded library, given by address (init).
struct Lib {
  decltype(&paged_decode_attention_ext) attention_ext = nullptr;
  decltype(&paged_decode_attention_noalloc) attention_noalloc = nullptr;
  decltype(&paged_decode_attention_append) attention_append = nullptr;
  decltype(&pda_kv_append_n) kv_append_n = nullptr;
  decltype(&pda_attention_prelude) prelude = nullptr;
  decltype(&pda_attention_prelude_append) prelude_append = nullptr;
  decltype(&pda_o_proj_residual_norm) o_proj = nullptr;
  decltype(&paged_decode_attention_sink) attention_sink = nullptr;
  decltype(&paged_decode_attention_kv4) attention_kv4 = nullptr;
  decltype(&pda_kv4_append) kv4_append = nullptr;
  decltype(&pda_kv4_read) kv4_read = nullptr;
  decltype(&pda_pages_update) pages_update = nullptr;
  decltype(&pda_pages_compact) pages_compact = nullptr;
  decltype(&pda_pages_copy) pages_copy = nullptr;
  decltype(&pda_linear) linear = nullptr;
  decltype(&pda_moe_route) moe_route = nullptr;
  decltype(&pda_moe_experts) moe_experts = nullptr;
  decltype(&pda_block_norm) block_norm = nullptr;
} g_lib;
PyObject* g_raw_stream = nullptr;  // torch._C._cuda_getCurrentRawStream
PyObject* g_device = nullptr;      // torch._C._cuda_getDevice

// One call's accepted tensors: all on one GPU, contiguous.
struct Checker {
  bool ok = true;
  int device = -1;

  // The tensor if it is a plain one of this dtype and rank, else null; with
  // `rows` its rows may lie apart.
  const at::Tensor* take(PyObject* o, at::ScalarType dt, int64_t ndim, bool rows = false) {
    if (!ok || !THPVariable_CheckExact(o)) return reject();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.dim() != ndim || t.scalar_type() != dt || !t.is_cuda()) return reject();
    if (!t.is_contiguous() && !(rows && t.stride(ndim - 1) == 1 && t.stride(0) >= t.size(1))) return reject();
    const int d = static_cast<int>(t.get_device());
    if (d < 0 || (device >= 0 && d != device)) return reject();
    device = d;
    return &t;
  }
  const at::Tensor* reject() {
    ok = false;
    return nullptr;
  }
  const at::Tensor* take_or_none(PyObject* o, at::ScalarType dt, int64_t ndim) {
    return o == Py_None ? nullptr : take(o, dt, ndim);
  }
  bool truth(PyObject* o) {
    if (o != Py_True && o != Py_False) ok = false;
    return o == Py_True;
  }
  void same(int64_t a, int64_t b) { ok = ok && a == b; }
  int32_t i32(int64_t v) {
    if (v < INT32_MIN || v > INT32_MAX) ok = false;
    return static_cast<int32_t>(v);
  }
  int32_t integer(PyObject* o) {
    if (!ok || !PyLong_CheckExact(o)) {
      ok = false;
      return 0;
    }
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) ok = false;
    return i32(v);
  }
  float number(PyObject* o) {
    if (!ok) return 0.f;
    if (PyFloat_CheckExact(o)) return static_cast<float>(PyFloat_AS_DOUBLE(o));
    if (!PyLong_CheckExact(o)) {
      ok = false;
      return 0.f;
    }
    const double v = PyLong_AsDouble(o);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return static_cast<float>(v);
  }
  // The raw handle of `stream`, or of torch's current stream on the tensors'
  // device.  of_current: the call takes the current device's stream instead,
  // so tensors on another device are left to the Python path.
  void* stream(PyObject* o, bool of_current) {
    if (!ok) return nullptr;
    PyObject* h;
    if (o == Py_None) {
      if (of_current) {
        PyObject* d = PyObject_CallNoArgs(g_device);
        if (!d || PyLong_AsLong(d) != device) ok = false;
        Py_XDECREF(d);
        if (PyErr_Occurred()) PyErr_Clear();
        if (!ok) return nullptr;
      }
      PyObject* d = PyLong_FromLong(device);
      h = d ? PyObject_CallOneArg(g_raw_stream, d) : nullptr;
      Py_XDECREF(d);
    } else {
      h = PyObject_GetAttrString(o, "cuda_stream");
    }
    void* p = h ? PyLong_AsVoidPtr(h) : nullptr;
    Py_XDECREF(h);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return p;
  }
};

const at::ScalarType kBf = at::ScalarType::BFloat16, kI32 = at::ScalarType::Int, kU8 = at::ScalarType::Byte;
const at::ScalarType kF32 = at::ScalarType::Float;

// k_cache, v_cache [N, P, Hkv, D], block_table [B, M], context_lens [B].
struct Cache {
  const at::Tensor *k, *v, *bt, *lens;
  int64_t n = 0, p = 0, hkv = 0, d = 0, m = 0;
  Cache(Checker& c, PyObject* const* a, int64_t batch) {
    k = c.take(a[0], kBf, 4);
    v = c.take(a[1], kBf, 4);
    bt = c.take(a[2], kI32, 2);
    lens = c.take(a[3], kI32, 1);
    if (!c.ok) return;
    n = k->size(0), p = k->size(1), hkv = k->size(2), d = k->size(3), m = bt->size(1);
    c.ok = v->sizes() == k->sizes();
    c.same(bt->size(0), batch);
    c.same(lens->size(0), batch);
  }
};

int32_t* ints(const at::Tensor* t) { return static_cast<int32_t*>(t->data_ptr()); }

// Runs one call's body, which returns the status (or kDeclined); nothing a
// tensor throws (one without storage, say) leaves this file.
template <class F>
PyObject* guarded(Py_ssize_t nargs, Py_ssize_t want, F body) {
  int rc = kDeclined;
  if (nargs == want) {
    try {
      rc = body();
    } catch (...) {
      PyErr_Clear();
      rc = kDeclined;
    }
  }
  return PyLong_FromLong(rc);
}

template <class F>
int released(F call) {  // the library call without the interpreter lock, as ctypes makes it
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc;
}

// (q, k, v, bt, lens, out, scale, window, stream, noalloc); q [B, Hq, D], or
// [B, T, Hq, D] with a window argument that is not None
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 10, [&]() -> int {
    Checker c;
    const bool ext = a[7] != Py_None;
    const at::Tensor* q = c.take(a[0], kBf, ext ? 4 : 3);
    if (!c.ok) return kDeclined;
    Cache kv(c, a + 1, q->size(0));
    const at::Tensor* out = c.take(a[5], kBf, ext ? 4 : 3);
    if (!c.ok) return kDeclined;
    c.ok = out->sizes() == q->sizes();
    const int32_t b = c.i32(q->size(0)), t = ext ? c.i32(q->size(1)) : 1, hq = c.i32(q->size(ext ? 2 : 1));
    const int32_t d = c.i32(q->size(ext ? 3 : 2));
    c.same(kv.d, d);
    const int32_t hkv = c.i32(kv.hkv), p = c.i32(kv.p), n = c.i32(kv.n), m = c.i32(kv.m);
    const int32_t window = ext ? c.integer(a[7]) : 0;
    const float scale = c.number(a[6]);
    void* st = c.stream(a[8], /*of_current=*/ext);
    if (!c.ok) return kDeclined;
    void *qp = q->data_ptr(), *kp = kv.k->data_ptr(), *vp = kv.v->data_ptr(), *op = out->data_ptr();
    int32_t *bp = ints(kv.bt), *lp = ints(kv.lens);
    if (a[9] == Py_True)
      return released([&] { return g_lib.attention_noalloc(qp, kp, vp, bp, lp, op, b, hq, hkv, d, p, n, m, scale, st); });
    return released([&] { return g_lib.attention_ext(qp, kp, vp, bp, lp, op, b, hq, hkv, d, p, n, m, t, window, scale, st); });
  });
}

// (k_new, v_new, k, v, bt, lens, several, stream); k_new [B, Hkv, D], or
// [B, T, Hkv, D] where `several` is True
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 8, [&]() -> int {
    Checker c;
    const bool several = a[6] == Py_True;
    const at::Tensor* kn = c.take(a[0], kBf, several ? 4 : 3);
    const at::Tensor* vn = c.take(a[1], kBf, several ? 4 : 3);
    if (!c.ok) return kDeclined;
    Cache kv(c, a + 2, kn->size(0));
    if (!c.ok) return kDeclined;
    c.ok = vn->sizes() == kn->sizes();
    const int32_t b = c.i32(kn->size(0)), t = several ? c.i32(kn->size(1)) : 1;
    c.same(kn->size(several ? 2 : 1), kv.hkv);
    c.same(kn->size(several ? 3 : 2), kv.d);
    const int32_t hkv = c.i32(kv.hkv), d = c.i32(kv.d), p = c.i32(kv.p), n = c.i32(kv.n), m = c.i32(kv.m);
    void* st = c.stream(a[7], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *knp = kn->data_ptr(), *vnp = vn->data_ptr(), *kp = kv.k->data_ptr(), *vp = kv.v->data_ptr();
    int32_t *bp = ints(kv.bt), *lp = ints(kv.lens);
    return released([&] { return g_lib.kv_append_n(knp, vnp, kp, vp, bp, lp, b, t, hkv, d, p, n, m, st); });
  });
}

// (q, k_new, v_new, k, v, bt, lens, out, scale, stream)
PyObject* attention_append(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 10, [&]() -> int {
    Checker c;
    const at::Tensor* q = c.take(a[0], kBf, 3);
    const at::Tensor* kn = c.take(a[1], kBf, 3);
    const at::Tensor* vn = c.take(a[2], kBf, 3);
    if (!c.ok) return kDeclined;
    Cache kv(c, a + 3, q->size(0));
    const at::Tensor* out = c.take(a[7], kBf, 3);
    if (!c.ok) return kDeclined;
    c.ok = out->sizes() == q->sizes() && vn->sizes() == kn->sizes();
    c.same(kn->size(0), q->size(0));
    c.same(kn->size(1), kv.hkv);
    c.same(kn->size(2), q->size(2));
    c.same(kv.d, q->size(2));
    const int32_t b = c.i32(q->size(0)), hq = c.i32(q->size(1)), d = c.i32(q->size(2));
    const int32_t hkv = c.i32(kv.hkv), p = c.i32(kv.p), n = c.i32(kv.n), m = c.i32(kv.m);
    const float scale = c.number(a[8]);
    void* st = c.stream(a[9], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *qp = q->data_ptr(), *knp = kn->data_ptr(), *vnp = vn->data_ptr();
    void *kp = kv.k->data_ptr(), *vp = kv.v->data_ptr(), *op = out->data_ptr();
    int32_t *bp = ints(kv.bt), *lp = ints(kv.lens);
    return released([&] { return g_lib.attention_append(qp, knp, vnp, kp, vp, bp, lp, op, b, hq, hkv, d, p, n, m, scale, st); });
  });
}

// (x, w_packed, lens, q_out, k, v, block_table or None, num_q_heads,
//  num_kv_heads, head_dim, rope_theta, rotary_dim, interleaved, bias, q_norm,
//  k_norm, eps, stream); k, v are the outputs, or with a block table the caches
PyObject* prelude(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 18, [&]() -> int {
    Checker c;
    const bool append = a[6] != Py_None;
    const at::Tensor* x = c.take(a[0], kBf, 2);
    const at::Tensor* w = c.take(a[1], kBf, 2);
    const at::Tensor* lens = c.take(a[2], kI32, 1);
    const at::Tensor* q = c.take(a[3], kBf, 3);
    const at::Tensor* k = c.take(a[4], kBf, append ? 4 : 3);
    const at::Tensor* v = c.take(a[5], kBf, append ? 4 : 3);
    const at::Tensor* bt = append ? c.take(a[6], kI32, 2) : nullptr;
    const at::Tensor* bias = a[13] != Py_None ? c.take(a[13], kBf, 1) : nullptr;
    const at::Tensor* qn = a[14] != Py_None ? c.take(a[14], kBf, 1) : nullptr;
    const at::Tensor* kn = a[15] != Py_None ? c.take(a[15], kBf, 1) : nullptr;
    pda_prelude_dims dm;
    dm.num_q_heads = c.integer(a[7]);
    dm.num_kv_heads = c.integer(a[8]);
    dm.head_dim = c.integer(a[9]);
    dm.rope_theta = c.number(a[10]);
    dm.rotary_dim = a[11] == Py_None ? dm.head_dim : c.integer(a[11]);
    if (a[12] != Py_True && a[12] != Py_False) c.ok = false;
    dm.interleaved = a[12] == Py_True;
    dm.eps = c.number(a[16]);
    if (!c.ok || (qn == nullptr) != (kn == nullptr)) return kDeclined;
    const int64_t hq = dm.num_q_heads, hkv = dm.num_kv_heads, d = dm.head_dim, rows = (hq + 2 * hkv) * d;
    dm.batch = c.i32(x->size(0));
    dm.hidden = c.i32(x->size(1));
    c.same(w->size(0), rows);
    c.same(w->size(1), x->size(1));
    c.same(lens->size(0), x->size(0));
    c.same(q->size(0), x->size(0));
    c.same(q->size(1), hq);
    c.same(q->size(2), d);
    c.ok = c.ok && k->sizes() == v->sizes();
    c.same(k->size(append ? 2 : 1), hkv);
    c.same(k->size(append ? 3 : 2), d);
    if (append)
      c.same(bt->size(0), x->size(0));
    else
      c.same(k->size(0), x->size(0));
    if (bias) c.same(bias->size(0), rows);
    if (qn) c.same(qn->size(0), d), c.same(kn->size(0), d);
    const int32_t pages = append ? c.i32(k->size(0)) : 0, page = append ? c.i32(k->size(1)) : 0;
    const int32_t m = append ? c.i32(bt->size(1)) : 0;
    void* st = c.stream(a[17], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    auto ptr = [](const at::Tensor* t) -> void* { return t ? t->data_ptr() : nullptr; };
    void *xp = ptr(x), *wp = ptr(w), *bp = ptr(bias), *qnp = ptr(qn), *knp = ptr(kn), *qp = ptr(q), *kp = ptr(k), *vp = ptr(v);
    int32_t *lp = ints(lens), *tp = append ? ints(bt) : nullptr;
    if (append)
      return released([&] { return g_lib.prelude_append(xp, wp, bp, qnp, knp, lp, qp, kp, vp, tp, page, pages, m, &dm, st); });
    return released([&] { return g_lib.prelude(xp, wp, bp, qnp, knp, lp, qp, kp, vp, &dm, st); });
  });
}

// (attn, w_packed, residual, norm_w, residual_out, normed_out, eps, stream)
PyObject* o_proj(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 8, [&]() -> int {
    Checker c;
    const at::Tensor* x = c.take(a[0], kBf, 2);
    const at::Tensor* w = c.take(a[1], kBf, 2);
    const at::Tensor* res = c.take(a[2], kBf, 2);
    const at::Tensor* nw = c.take(a[3], kBf, 1);
    const at::Tensor* z = c.take(a[4], kBf, 2);
    const at::Tensor* h = c.take(a[5], kBf, 2);
    const float eps = c.number(a[6]);
    if (!c.ok) return kDeclined;
    const int32_t b = c.i32(x->size(0)), k = c.i32(x->size(1)), n = c.i32(w->size(0));
    c.same(w->size(1), x->size(1));
    c.same(res->size(0), x->size(0));
    c.same(res->size(1), w->size(0));
    c.same(nw->size(0), w->size(0));
    c.ok = c.ok && z->sizes() == res->sizes() && h->sizes() == res->sizes();
    void* st = c.stream(a[7], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *xp = x->data_ptr(), *wp = w->data_ptr(), *rp = res->data_ptr(), *np = nw->data_ptr();
    void *zp = z->data_ptr(), *hp = h->data_ptr();
    return released([&] { return g_lib.o_proj(xp, wp, rp, np, zp, hp, b, k, n, eps, st); });
  });
}

// (q, k, v, bt, lens, out, scale, window, sinks, stream); q [B, T, Hq, D]
PyObject* attention_sink(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 10, [&]() -> int {
    Checker c;
    const at::Tensor* q = c.take(a[0], kBf, 4);
    if (!c.ok) return kDeclined;
    Cache kv(c, a + 1, q->size(0));
    const at::Tensor* out = c.take(a[5], kBf, 4);
    if (!c.ok) return kDeclined;
    c.ok = out->sizes() == q->sizes();
    const int32_t b = c.i32(q->size(0)), t = c.i32(q->size(1)), hq = c.i32(q->size(2)), d = c.i32(q->size(3));
    c.same(kv.d, d);
    const int32_t hkv = c.i32(kv.hkv), p = c.i32(kv.p), n = c.i32(kv.n), m = c.i32(kv.m);
    const float scale = c.number(a[6]);
    const int32_t window = c.integer(a[7]), sinks = c.integer(a[8]);
    void* st = c.stream(a[9], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *qp = q->data_ptr(), *kp = kv.k->data_ptr(), *vp = kv.v->data_ptr(), *op = out->data_ptr();
    int32_t *bp = ints(kv.bt), *lp = ints(kv.lens);
    return released([&] { return g_lib.attention_sink(qp, kp, vp, bp, lp, op, b, hq, hkv, d, p, n, m, t, window, sinks, scale, st); });
  });
}

// k codes, k scales, v codes, v scales, block_table [B, M], context_lens [B]
struct Cache4 {
  const at::Tensor* t[4];
  const at::Tensor *bt, *lens;
  int64_t n = 0, p = 0, hkv = 0, d = 0, m = 0;
  Cache4(Checker& c, PyObject* const* a, int64_t batch) {
    for (int i = 0; i < 4; ++i) t[i] = c.take(a[i], kU8, i % 2 ? 4 : 5);
    bt = c.take(a[4], kI32, 2);
    lens = c.take(a[5], kI32, 1);
    if (!c.ok) return;
    n = t[0]->size(0), hkv = t[0]->size(1), d = 32 * t[0]->size(2), p = t[0]->size(3), m = bt->size(1);
    c.ok = t[2]->sizes() == t[0]->sizes() && t[3]->sizes() == t[1]->sizes();
    c.same(t[0]->size(4), 16);
    for (int i = 0; i < 4; ++i) c.same(t[1]->size(i), t[0]->size(i));
    c.same(bt->size(0), batch);
    c.same(lens->size(0), batch);
  }
  void* at(int i) const { return t[i]->data_ptr(); }
};

// (q, k codes, k scales, v codes, v scales, bt, lens, out, scale, window, sinks, stream); q [B, T, Hq, D]
PyObject* attention_kv4(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 12, [&]() -> int {
    Checker c;
    const at::Tensor* q = c.take(a[0], kBf, 4);
    if (!c.ok) return kDeclined;
    Cache4 kv(c, a + 1, q->size(0));
    const at::Tensor* out = c.take(a[7], kBf, 4);
    if (!c.ok) return kDeclined;
    c.ok = out->sizes() == q->sizes();
    const int32_t b = c.i32(q->size(0)), t = c.i32(q->size(1)), hq = c.i32(q->size(2)), d = c.i32(q->size(3));
    c.same(kv.d, d);
    const int32_t hkv = c.i32(kv.hkv), p = c.i32(kv.p), n = c.i32(kv.n), m = c.i32(kv.m);
    const float scale = c.number(a[8]);
    const int32_t window = c.integer(a[9]), sinks = c.integer(a[10]);
    void* st = c.stream(a[11], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *qp = q->data_ptr(), *op = out->data_ptr(), *kp = kv.at(0), *ksp = kv.at(1), *vp = kv.at(2), *vsp = kv.at(3);
    int32_t *bp = ints(kv.bt), *lp = ints(kv.lens);
    return released([&] {
      return g_lib.attention_kv4(qp, kp, ksp, vp, vsp, bp, lp, op, b, hq, hkv, d, p, n, m, t, window, sinks, scale, st);
    });
  });
}

// (k, v, k codes, k scales, v codes, v scales, bt, lens, read, stream); k, v [B, T, Hkv, D]: the new
// tokens, or with `read` True what they are read to
PyObject* kv4_tokens(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 10, [&]() -> int {
    Checker c;
    const at::Tensor* k = c.take(a[0], kBf, 4);
    const at::Tensor* v = c.take(a[1], kBf, 4);
    if (!c.ok) return kDeclined;
    Cache4 kv(c, a + 2, k->size(0));
    if (!c.ok) return kDeclined;
    c.ok = v->sizes() == k->sizes();
    const int32_t b = c.i32(k->size(0)), t = c.i32(k->size(1)), hkv = c.i32(kv.hkv), d = c.i32(kv.d);
    c.same(k->size(2), kv.hkv);
    c.same(k->size(3), kv.d);
    const int32_t p = c.i32(kv.p), n = c.i32(kv.n), m = c.i32(kv.m);
    const bool read = a[8] == Py_True;
    void* st = c.stream(a[9], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *k_p = k->data_ptr(), *v_p = v->data_ptr(), *kp = kv.at(0), *ksp = kv.at(1), *vp = kv.at(2), *vsp = kv.at(3);
    int32_t *bp = ints(kv.bt), *lp = ints(kv.lens);
    return released([&] {
      return read ? g_lib.kv4_read(k_p, v_p, kp, ksp, vp, vsp, bp, lp, b, t, hkv, d, p, n, m, st)
                  : g_lib.kv4_append(k_p, v_p, kp, ksp, vp, vsp, bp, lp, b, t, hkv, d, p, n, m, st);
    });
  });
}

// (block_table, lens, parents or None, new_lens, refcount, table_out, refcount_out, src, dst, info,
//  page_size, window, sinks, num_queries, stream)
PyObject* pages_update(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 15, [&]() -> int {
    Checker c;
    const at::Tensor* t[10];
    for (int i = 0; i < 10; ++i) t[i] = i == 2 && a[2] == Py_None ? nullptr : c.take(a[i], kI32, i == 0 || i == 5 ? 2 : 1);
    if (!c.ok) return kDeclined;
    const int64_t b = t[0]->size(0), m = t[0]->size(1), r = t[3]->size(0), n = t[4]->size(0);
    c.same(t[1]->size(0), b);
    if (t[2]) c.same(t[2]->size(0), r);
    c.same(t[5]->size(0), r);
    c.same(t[5]->size(1), m);
    c.same(t[6]->size(0), n);
    c.same(t[7]->size(0), r);
    c.same(t[8]->size(0), r);
    c.same(t[9]->size(0), 2);
    const int32_t page = c.integer(a[10]), window = c.integer(a[11]), sinks = c.integer(a[12]), nq = c.integer(a[13]);
    const int32_t bi = c.i32(b), mi = c.i32(m), ri = c.i32(r), ni = c.i32(n);
    void* st = c.stream(a[14], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    int32_t* p[10];
    for (int i = 0; i < 10; ++i) p[i] = t[i] ? ints(t[i]) : nullptr;
    return released([&] {
      return g_lib.pages_update(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], bi, ri, page, ni, mi, nq, window,
                                sinks, st);
    });
  });
}

// (block_table, lens, refcount, table_out, refcount_out, page_map, src, dst, info, page_size, stream)
PyObject* pages_compact(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 11, [&]() -> int {
    Checker c;
    const at::Tensor* t[9];
    for (int i = 0; i < 9; ++i) t[i] = c.take(a[i], kI32, i == 0 || i == 3 ? 2 : 1);
    if (!c.ok) return kDeclined;
    const int64_t b = t[0]->size(0), m = t[0]->size(1), n = t[2]->size(0);
    c.same(t[1]->size(0), b);
    c.ok = c.ok && t[3]->sizes() == t[0]->sizes();
    for (int i = 4; i < 8; ++i) c.same(t[i]->size(0), n);
    c.same(t[8]->size(0), 2);
    const int32_t page = c.integer(a[9]), bi = c.i32(b), mi = c.i32(m), ni = c.i32(n);
    void* st = c.stream(a[10], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    int32_t* p[9];
    for (int i = 0; i < 9; ++i) p[i] = ints(t[i]);
    return released(
        [&] { return g_lib.pages_compact(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], bi, page, ni, mi, st); });
  });
}

// (pools, src, dst, count or None, stream); pools: a list or tuple of tensors of any type
PyObject* pages_copy(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 5, [&]() -> int {
    if (!PyList_CheckExact(a[0]) && !PyTuple_CheckExact(a[0])) return kDeclined;
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(a[0]);
    PyObject** items = PySequence_Fast_ITEMS(a[0]);
    Checker c;
    const at::Tensor* src = c.take(a[1], kI32, 1);
    const at::Tensor* dst = c.take(a[2], kI32, 1);
    const at::Tensor* count = a[3] != Py_None ? c.take(a[3], kI32, 1) : nullptr;
    if (!c.ok || k == 0) return kDeclined;
    c.same(dst->size(0), src->size(0));
    if (count) c.same(count->size(0), 1);
    std::vector<pda_pool> pools(static_cast<size_t>(k));
    int64_t n = 0;
    for (Py_ssize_t i = 0; i < k && c.ok; ++i) {
      if (!THPVariable_CheckExact(items[i])) return kDeclined;
      const at::Tensor& t = THPVariable_Unpack(items[i]);
      if (!t.defined() || t.dim() < 2 || !t.is_cuda() || !t.is_contiguous() || t.get_device() != c.device) return kDeclined;
      if (i == 0) n = t.size(0);
      c.same(t.size(0), n);
      if (!c.ok || n == 0) return kDeclined;
      pools[i].data = t.data_ptr();
      pools[i].page_bytes = t.numel() / n * t.element_size();
    }
    const int32_t ki = c.i32(k), ni = c.i32(n), most = c.i32(src->size(0));
    void* st = c.stream(a[4], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    int32_t *sp = ints(src), *dp = ints(dst), *cp = count ? ints(count) : nullptr;
    return released([&] { return g_lib.pages_copy(pools.data(), ki, sp, dp, cp, most, ni, st); });
  });
}

void* address(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// (x, w_packed, out, bias or None, residual or None, activation, gated, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 8, [&]() -> int {
    Checker c;
    const at::Tensor* x = c.take(a[0], kBf, 2);
    const at::Tensor* w = c.take(a[1], kBf, 2);
    if (!c.ok || !THPVariable_CheckExact(a[2])) return kDeclined;
    pda_linear_dims d;
    d.out_f32 = THPVariable_Unpack(a[2]).scalar_type() == kF32;
    const at::Tensor* out = c.take(a[2], d.out_f32 ? kF32 : kBf, 2);
    const at::Tensor* bias = c.take_or_none(a[3], kBf, 1);
    const at::Tensor* res = c.take_or_none(a[4], kBf, 2);
    d.activation = c.integer(a[5]);
    d.gated = c.truth(a[6]);
    if (!c.ok) return kDeclined;
    d.batch = c.i32(x->size(0)), d.in_features = c.i32(x->size(1)), d.out_features = c.i32(out->size(1));
    const int64_t rows = out->size(1) * (d.gated ? 2 : 1);
    c.same(out->size(0), x->size(0));
    c.same(w->size(0), rows);
    c.same(w->size(1), x->size(1));
    if (bias) c.same(bias->size(0), rows);
    if (res) c.ok = c.ok && res->sizes() == out->sizes();
    void* st = c.stream(a[7], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *xp = address(x), *wp = address(w), *bp = address(bias), *rp = address(res), *op = address(out);
    return released([&] { return g_lib.linear(xp, wp, bp, rp, op, &d, st); });
  });
}

// (logits, expert_ids, expert_weights, select_bias or None, sigmoid, renormalise, scale, stream)
PyObject* moe_route(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 8, [&]() -> int {
    Checker c;
    const at::Tensor* l = c.take(a[0], kF32, 2, /*rows=*/true);
    const at::Tensor* ids = c.take(a[1], kI32, 2);
    const at::Tensor* w = c.take(a[2], kF32, 2);
    const at::Tensor* bias = c.take_or_none(a[3], kF32, 1);
    pda_route_dims d;
    d.sigmoid = c.integer(a[4]);
    d.renormalise = c.truth(a[5]);
    d.scale = c.number(a[6]);
    if (!c.ok) return kDeclined;
    d.tokens = c.i32(l->size(0)), d.num_experts = c.i32(l->size(1)), d.top_k = c.i32(ids->size(1));
    d.logit_stride = d.tokens > 1 ? c.i32(l->stride(0)) : d.num_experts;
    c.same(ids->size(0), l->size(0));
    c.ok = c.ok && w->sizes() == ids->sizes();
    if (bias) c.same(bias->size(0), l->size(1));
    void* st = c.stream(a[7], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    float *lp = static_cast<float*>(address(l)), *bp = static_cast<float*>(address(bias)), *wp = static_cast<float*>(address(w));
    int32_t* ip = ints(ids);
    return released([&] { return g_lib.moe_route(lp, bp, ip, wp, &d, st); });
  });
}

// (x, expert_ids, expert_weights, w_gate_up, w_down, out, residual or None, activation, stream)
PyObject* moe_experts(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 9, [&]() -> int {
    Checker c;
    const at::Tensor* x = c.take(a[0], kBf, 2);
    const at::Tensor* ids = c.take(a[1], kI32, 2);
    const at::Tensor* w = c.take(a[2], kF32, 2);
    const at::Tensor* gu = c.take(a[3], kBf, 3);
    const at::Tensor* dn = c.take(a[4], kBf, 3);
    const at::Tensor* out = c.take(a[5], kBf, 2);
    const at::Tensor* res = c.take_or_none(a[6], kBf, 2);
    pda_moe_dims d;
    d.activation = c.integer(a[7]);
    if (!c.ok) return kDeclined;
    d.tokens = c.i32(x->size(0)), d.hidden = c.i32(x->size(1)), d.inter = c.i32(dn->size(2));
    d.num_experts = c.i32(dn->size(0)), d.top_k = c.i32(ids->size(1));
    c.same(ids->size(0), x->size(0));
    c.same(dn->size(1), x->size(1));
    c.same(gu->size(0), dn->size(0));
    c.same(gu->size(1), 2 * dn->size(2));
    c.same(gu->size(2), x->size(1));
    c.ok = c.ok && w->sizes() == ids->sizes() && out->sizes() == x->sizes() && (!res || res->sizes() == x->sizes());
    void* st = c.stream(a[8], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *xp = address(x), *gp = address(gu), *dp = address(dn), *rp = address(res), *op = address(out);
    float* wp = static_cast<float*>(address(w));
    int32_t* ip = ints(ids);
    return released([&] { return g_lib.moe_experts(xp, ip, wp, gp, dp, rp, op, &d, st); });
  });
}

// (y, residual or None, residual_out, normed_out or None, post_w, pre_w, gate or None, scale, weight_offset, eps, stream)
PyObject* block_norm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 11, [&]() -> int {
    Checker c;
    const at::Tensor* y = c.take(a[0], kBf, 2);
    const at::Tensor* res = c.take_or_none(a[1], kBf, 2);
    const at::Tensor* z = c.take(a[2], kBf, 2);
    const at::Tensor* h = c.take_or_none(a[3], kBf, 2);
    const at::Tensor* post = c.take_or_none(a[4], kBf, 1);
    const at::Tensor* pre = c.take_or_none(a[5], kBf, 1);
    if (!c.ok) return kDeclined;
    const bool rows = a[6] != Py_None && THPVariable_CheckExact(a[6]) && THPVariable_Unpack(a[6]).dim() == 2;
    const at::Tensor* gate = c.take_or_none(a[6], kBf, rows ? 2 : 1);
    pda_block_norm_dims d;
    d.gate_rows = rows;
    d.scale = c.number(a[7]), d.weight_offset = c.number(a[8]), d.eps = c.number(a[9]);
    if (!c.ok || (pre == nullptr) != (h == nullptr)) return kDeclined;
    d.rows = c.i32(y->size(0)), d.hidden = c.i32(y->size(1));
    c.ok = c.ok && z->sizes() == y->sizes() && (!res || res->sizes() == y->sizes()) && (!h || h->sizes() == y->sizes()) &&
           (!gate || !rows || gate->sizes() == y->sizes());
    for (const at::Tensor* t : {post, pre, rows ? nullptr : gate})
      if (t) c.same(t->size(0), y->size(1));
    void* st = c.stream(a[10], /*of_current=*/true);
    if (!c.ok) return kDeclined;
    void *yp = address(y), *rp = address(res), *pp = address(post), *np = address(pre), *gp = address(gate);
    void *zp = address(z), *hp = address(h);
    return released([&] { return g_lib.block_norm(yp, rp, pp, np, gp, zp, hp, &d, st); });
  });
}

// ({name: address}, raw_stream, device): the loaded library's entry points,
// torch's current raw stream of a device and its current device
PyObject* init(PyObject*, PyObject* args) {
  PyObject *table, *raw, *device;
  if (!PyArg_ParseTuple(args, "O!OO", &PyDict_Type, &table, &raw, &device)) return nullptr;
  auto set = [&](const char* name, auto& fn) {
    PyObject* v = PyDict_GetItemString(table, name);
    void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
    if (!p) {
      if (!PyErr_Occurred()) PyErr_Format(PyExc_KeyError, "no address for %s", name);
      return false;
    }
    fn = reinterpret_cast<typename std::remove_reference<decltype(fn)>::type>(p);
    return true;
  };
  if (!set("paged_decode_attention_ext", g_lib.attention_ext) ||
      !set("paged_decode_attention_noalloc", g_lib.attention_noalloc) ||
      !set("paged_decode_attention_append", g_lib.attention_append) || !set("pda_kv_append_n", g_lib.kv_append_n) ||
      !set("pda_attention_prelude", g_lib.prelude) ||
      !set("pda_attention_prelude_append", g_lib.prelude_append) ||
      !set("pda_o_proj_residual_norm", g_lib.o_proj) || !set("paged_decode_attention_sink", g_lib.attention_sink) ||
      !set("paged_decode_attention_kv4", g_lib.attention_kv4) || !set("pda_kv4_append", g_lib.kv4_append) ||
      !set("pda_kv4_read", g_lib.kv4_read) || !set("pda_pages_update", g_lib.pages_update) ||
      !set("pda_pages_compact", g_lib.pages_compact) || !set("pda_pages_copy", g_lib.pages_copy) ||
      !set("pda_linear", g_lib.linear) || !set("pda_moe_route", g_lib.moe_route) ||
      !set("pda_moe_experts", g_lib.moe_experts) || !set("pda_block_norm", g_lib.block_norm))
    return nullptr;
  Py_INCREF(raw);
  Py_XDECREF(g_raw_stream);
  g_raw_stream = raw;
  Py_INCREF(device);
  Py_XDECREF(g_device);
  g_device = device;
  Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {FAST(attention), FAST(kv_append), FAST(attention_append), FAST(prelude), FAST(o_proj),
                          FAST(attention_sink), FAST(attention_kv4), FAST(kv4_tokens), FAST(pages_update),
                          FAST(pages_compact), FAST(pages_copy), FAST(linear), FAST(moe_route), FAST(moe_experts),
                          FAST(block_norm),
                          {"init", init, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "pda_native", "Native marshalling of the binding's hot calls.", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_pda_native() {
  PyObject* m = PyModule_Create(&kModule);
  if (m && PyModule_AddStringConstant(m, "built_for", PDA_BUILT_FOR) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
