// Native call path of ops.py (CPython extension `_binding`).
//
// An operator call from Python spent 14 to 19 us on argument checks, string
// formatting and ctypes conversions (measured without the launches), more than
// the kernels of a small call take. Each function here does the same checks on
// the tensors directly, allocates the outputs and workspace that the caller
// left out and calls the C entry point: 1 to 2 us. It takes exactly the calls
// that ops.py's checks accept; for anything else (other argument types, a
// failed check, an exception from the tensor library) it returns None and
// ops.py's own path runs, which raises the error or handles the call. Nothing
// is kept between calls except the Python callables looked up at import.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/Functions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/rocs_layer.h"

namespace {

PyObject* g_get_device;   // torch._C._cuda_getDevice
PyObject* g_raw_stream;   // torch._C._cuda_getCurrentRawStream
PyObject* g_check;        // _lib.check(status, name): raises RocsError
PyObject* g_cuda_stream;  // "cuda_stream"

struct Refuse {};         // not a call for this path
struct PyError {};        // a Python exception is set

void need(bool ok) {
  if (!ok) throw Refuse();
}

// A tensor argument: plain strided device tensors with storage of their own
// only (not torch.func's wrappers); null for None.
struct Ten {
  const at::Tensor* t = nullptr;
  at::Tensor own;
  explicit operator bool() const { return t != nullptr; }
  const at::Tensor* operator->() const { return t; }
  void* ptr() const { return t == nullptr ? nullptr : t->data_ptr(); }
  const int32_t* i32() const { return static_cast<const int32_t*>(ptr()); }
  const float* f32() const { return static_cast<const float*>(ptr()); }
  size_t bytes() const { return t == nullptr ? 0 : (size_t)t->nbytes(); }
};

// The address in a Python integer (a new reference, or null after an error).
void* address(PyObject* v) {
  if (v == nullptr) throw PyError();
  void* p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  if (p == nullptr && PyErr_Occurred()) throw PyError();
  return p;
}

// The current stream of a device (its number, a new reference).
void* current_stream(PyObject* device) {
  if (device == nullptr) throw PyError();
  PyObject* v = PyObject_CallOneArg(g_raw_stream, device);
  Py_DECREF(device);
  return address(v);
}

// The given stream, or the current one of the current device.
void* stream_of(PyObject* o) {
  if (o == Py_None) return current_stream(PyObject_CallNoArgs(g_get_device));
  return address(PyObject_GetAttr(o, g_cuda_stream));
}

struct Call {
  c10::Device dev{c10::DeviceType::CPU};
  bool any = false;
  PyObject* stream;

  explicit Call(PyObject* s) : stream(s) {}

  Ten get(PyObject* o) {
    Ten r;
    if (o == Py_None) return r;
    need(THPVariable_CheckExact(o));
    r.t = &THPVariable_Unpack(o);
    need(r.t->is_cuda() && r.t->layout() == c10::kStrided && r.t->has_storage());
    if (!any) dev = r.t->device();
    any = true;
    need(r.t->device() == dev);
    return r;
  }
  Ten must(PyObject* o) {
    need(o != Py_None);
    return get(o);
  }
  // The caller's output or workspace, or a new one.
  Ten or_new(PyObject* o, c10::IntArrayRef shape, c10::ScalarType type) {
    Ten r = get(o);
    if (!r) {
      // Memory for a call on another stream is that stream's: ops.py takes it.
      need(stream == Py_None || stream_of(stream) == current_stream(PyLong_FromLong(dev.index())));
      r.own = at::empty(shape, c10::TensorOptions().dtype(type).device(dev));
      return r;
    }
    need(r->sizes() == shape && r->scalar_type() == type && r->is_contiguous());
    return r;
  }
};

const at::Tensor& tensor(const Ten& t) { return t.t != nullptr ? *t.t : t.own; }
void* data(const Ten& t) { return t.t != nullptr || t.own.defined() ? tensor(t).data_ptr() : nullptr; }
size_t nbytes(const Ten& t) { return t.t != nullptr || t.own.defined() ? tensor(t).nbytes() : 0; }

int32_t dtype_code(const Ten& t) {
  const c10::ScalarType s = t->scalar_type();
  need(s == c10::kBFloat16 || s == c10::kFloat);
  return s == c10::kBFloat16 ? ROCS_DTYPE_BF16 : ROCS_DTYPE_F32;
}

int32_t activation(PyObject* o) {
  if (o == Py_None) return ROCS_ACT_NONE;
  need(PyUnicode_CheckExact(o));
  if (PyUnicode_CompareWithASCIIString(o, "relu") == 0) return ROCS_ACT_RELU;
  need(PyUnicode_CompareWithASCIIString(o, "none") == 0);
  return ROCS_ACT_NONE;
}

int64_t integer(PyObject* o) {
  need(PyLong_CheckExact(o));
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refuse();
  }
  return v;
}

float scale_of(PyObject* o) {           // float(scale or 0.0)
  if (o == Py_None) return 0.f;
  need(PyFloat_CheckExact(o) || PyLong_CheckExact(o));
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refuse();
  }
  return (float)v;
}

void offsets(const Ten& t, int64_t n_req) {
  need(t->scalar_type() == c10::kInt && t->dim() == 1 && t->is_contiguous() &&
       t->numel() == n_req + 1);
}

void same(const Ten& t, const Ten& as) {          // optional input of the common dtype
  need(!t || (t->scalar_type() == as->scalar_type() && t->is_contiguous()));
}

void shape_is(const Ten& t, c10::IntArrayRef s) { need(t->sizes() == s); }

void bias_of(const Ten& t, int64_t n) {
  need(!t || (t->scalar_type() == c10::kFloat && t->dim() == 1 && t->size(0) == n &&
              t->is_contiguous()));
}

// Without the interpreter lock for its lifetime, however the scope is left.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// Calls the C entry point without the interpreter lock. Every pointer and size
// is an argument here, so it has been taken while the lock was held: data_ptr()
// throws for a tensor without storage (inside torch.vmap or torch.func.grad).
template <typename... P, typename... A>
void run(const char* name, int32_t (*call)(P...), A... args) {
  static_assert(sizeof...(P) == sizeof...(A), "argument count");
  int32_t status;
  {
    Unlocked unlocked;
    status = call(args...);
  }
  if (status == ROCS_OK) return;
  PyObject* r = PyObject_CallFunction(g_check, "is", (int)status, name);
  Py_XDECREF(r);
  if (r == nullptr) throw PyError();
}

// The caller's own object, or the new tensor.
PyObject* result(PyObject* given, const Ten& t) {
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  return THPVariable_Wrap(t.own);
}

PyObject* pair(PyObject* a, PyObject* b) {
  if (a == nullptr || b == nullptr) {
    Py_XDECREF(a);
    Py_XDECREF(b);
    return nullptr;
  }
  PyObject* r = PyTuple_Pack(2, a, b);
  Py_DECREF(a);
  Py_DECREF(b);
  return r;
}

template <int N, PyObject* (*F)(PyObject* const*)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return F(args);
  } catch (const PyError&) {
    return nullptr;
  } catch (const Refuse&) {
  } catch (const std::exception&) {
    PyErr_Clear();
  }
  Py_RETURN_NONE;
}

// x_cand, w_cand, x_req, w_req, index, mapped, bias, activation, x_cand_add,
// out, workspace, stream
PyObject* linear(PyObject* const* a) {
  Call c(a[11]);
  const Ten x = c.must(a[0]), w = c.must(a[1]), xr = c.get(a[2]), wr = c.get(a[3]),
            index = c.get(a[4]), bias = c.get(a[6]), add = c.get(a[8]);
  const bool mapped = a[5] == Py_True;
  const int32_t act = activation(a[7]);
  need(x->dim() == 2 && w->dim() == 2);
  const int64_t n = x->size(0), k = x->size(1), d = w->size(0);
  need(w->size(1) == k);
  const int32_t code = dtype_code(x);
  for (const Ten* t : {&x, &w, &xr, &wr, &add}) same(*t, x);
  int64_t r = 0, kr = 0;
  if (xr) {
    need(wr && index && xr->dim() == 2);
    r = xr->size(0);
    kr = xr->size(1);
    shape_is(wr, {d, kr});
  } else {
    need(!wr);
    if (!mapped && index) r = index->numel() - 1;
  }
  if (index) {
    if (mapped) need(index->scalar_type() == c10::kInt && index->dim() == 1 &&
                     index->is_contiguous() && index->numel() == n);
    else offsets(index, r);
  }
  if (add) shape_is(add, x->sizes());
  bias_of(bias, d);
  const Ten out = c.or_new(a[9], {n, d}, x->scalar_type());
  const size_t bytes = rocs_ikbo_linear_workspace_size(r, n, d, kr);
  Ten ws = c.get(a[10]);
  if (!ws && bytes > 0) ws = c.or_new(Py_None, {(int64_t)bytes}, c10::kByte);
  void* s = stream_of(c.stream);
  if (mapped)
    run("rocs_ikbo_linear_mapped", rocs_ikbo_linear_mapped, xr.ptr(), kr, x.ptr(), add.ptr(), k,
        wr.ptr(), w.ptr(), bias.f32(), index.i32(), r, n, d, code, act, data(out), data(ws),
        nbytes(ws), s);
  else
    run("rocs_ikbo_linear", rocs_ikbo_linear, xr.ptr(), kr, x.ptr(), add.ptr(), k, wr.ptr(),
        w.ptr(), bias.f32(), index.i32(), r, n, d, code, act, data(out), data(ws), nbytes(ws), s);
  return result(a[9], out);
}

// x_req, x_cand, w_rr, w_cr, w_cc, cand_offsets, b_req, b_cand, activation,
// x_cand_add, y_req, y_cand, workspace, stream
PyObject* glm_linear(PyObject* const* a) {
  Call c(a[13]);
  const Ten xr = c.must(a[0]), x = c.must(a[1]), wrr = c.must(a[2]), wr = c.must(a[3]),
            w = c.must(a[4]), off = c.must(a[5]), br = c.get(a[6]), bias = c.get(a[7]),
            add = c.get(a[9]);
  const int32_t act = activation(a[8]);
  need(xr->dim() == 2 && x->dim() == 2 && wrr->dim() == 2 && w->dim() == 2);
  const int64_t r = xr->size(0), kr = xr->size(1), n = x->size(0), k = x->size(1),
                dr = wrr->size(0), d = w->size(0);
  shape_is(wrr, {dr, kr});
  shape_is(wr, {d, kr});
  shape_is(w, {d, k});
  const int32_t code = dtype_code(x);
  for (const Ten* t : {&x, &xr, &wrr, &wr, &w, &add}) same(*t, x);
  offsets(off, r);
  if (add) shape_is(add, x->sizes());
  bias_of(br, dr);
  need(!br || br->is_contiguous());
  bias_of(bias, d);
  const Ten yr = c.or_new(a[10], {r, dr}, x->scalar_type());
  const Ten out = c.or_new(a[11], {n, d}, x->scalar_type());
  const size_t bytes = rocs_ikbo_linear_workspace_size(r, n, d, kr);
  Ten ws = c.get(a[12]);
  if (!ws && bytes > 0) ws = c.or_new(Py_None, {(int64_t)bytes}, c10::kByte);
  void* s = stream_of(c.stream);
  run("rocs_glm_linear", rocs_glm_linear, xr.ptr(), kr, x.ptr(), add.ptr(), k, wrr.ptr(), wr.ptr(),
      w.ptr(), br.f32(), bias.f32(), off.i32(), r, n, dr, d, code, act, data(yr), data(out),
      data(ws), nbytes(ws), s);
  return pair(result(a[10], yr), result(a[11], out));
}

// x_cand, w1_cand, w2, x_req, w1_req, cand_offsets, b1, b2, activation1,
// activation2, out, workspace, stream
PyObject* mlp2(PyObject* const* a) {
  Call c(a[12]);
  const Ten x = c.must(a[0]), w1 = c.must(a[1]), w2 = c.must(a[2]), xr = c.get(a[3]),
            wr = c.get(a[4]), off = c.get(a[5]), b1 = c.get(a[6]), b2 = c.get(a[7]);
  const int32_t act1 = activation(a[8]), act2 = activation(a[9]);
  need(x->dim() == 2 && w1->dim() == 2 && w2->dim() == 2);
  const int64_t n = x->size(0), k = x->size(1), dh = w1->size(0), d = w2->size(0);
  need(w1->size(1) == k && w2->size(1) == dh);
  const int32_t code = dtype_code(x);
  for (const Ten* t : {&x, &w1, &w2, &xr, &wr}) same(*t, x);
  int64_t r = 0, kr = 0;
  if (xr) {
    need(wr && off && xr->dim() == 2);
    r = xr->size(0);
    kr = xr->size(1);
    shape_is(wr, {dh, kr});
    offsets(off, r);
  } else {
    need(!wr && !off);
  }
  bias_of(b1, dh);
  bias_of(b2, d);
  const Ten out = c.or_new(a[10], {n, d}, x->scalar_type());
  const size_t bytes = rocs_ikbo_mlp2_workspace_size(r, n, kr, k, dh, d, code);
  Ten ws = c.get(a[11]);
  if (!ws && bytes > 0) ws = c.or_new(Py_None, {(int64_t)bytes}, c10::kByte);
  void* s = stream_of(c.stream);
  run("rocs_ikbo_mlp2", rocs_ikbo_mlp2, xr.ptr(), kr, x.ptr(), k, wr.ptr(), w1.ptr(), b1.f32(),
      w2.ptr(), b2.f32(), off.i32(), r, n, dh, d, code, act1, act2, data(out), data(ws), nbytes(ws),
      s);
  return result(a[10], out);
}

// x_req, x_cand, cand_offsets, w_req, w_cand, bias, activation, out,
// workspace, stream
PyObject* fm_linear(PyObject* const* a) {
  Call c(a[9]);
  const Ten xr = c.must(a[0]), x = c.must(a[1]), off = c.must(a[2]), wr = c.must(a[3]),
            w = c.must(a[4]), bias = c.get(a[5]);
  const int32_t act = activation(a[6]);
  need(xr->dim() == 3 && x->dim() == 3 && xr->size(2) == x->size(2) && w->dim() == 2);
  const int64_t r = xr->size(0), fr = xr->size(1), e = xr->size(2), n = x->size(0),
                fc = x->size(1), d = w->size(0);
  offsets(off, r);
  shape_is(wr, {d, fr * fr});
  shape_is(w, {d, fc * (fr + fc)});
  need(fr <= INT32_MAX && fc <= INT32_MAX && e <= INT32_MAX);
  const int32_t code = dtype_code(x);
  for (const Ten* t : {&x, &xr, &wr, &w}) same(*t, x);
  bias_of(bias, d);
  const Ten out = c.or_new(a[7], {n, d}, x->scalar_type());
  const size_t bytes = rocs_glm_fm_linear_workspace_size(r, n, (int32_t)fr, (int32_t)fc,
                                                         (int32_t)e, d, code);
  Ten ws = c.get(a[8]);
  if (!ws && bytes > 0) ws = c.or_new(Py_None, {(int64_t)bytes}, c10::kByte);
  void* s = stream_of(c.stream);
  run("rocs_glm_fm_linear", rocs_glm_fm_linear, xr.ptr(), x.ptr(), off.i32(), r, n, (int32_t)fr,
      (int32_t)fc, (int32_t)e, wr.ptr(), w.ptr(), bias.f32(), d, code, act, data(out), data(ws),
      nbytes(ws), s);
  return result(a[7], out);
}

// x_req, x_cand, w_rr, w_cr, w_cc, index, mapped, y_req, y_cand, workspace,
// stream
PyObject* lcb(PyObject* const* a) {
  Call c(a[10]);
  const Ten xr = c.must(a[0]), x = c.must(a[1]), wrr = c.get(a[2]), wcr = c.must(a[3]),
            wcc = c.must(a[4]), index = c.must(a[5]);
  const bool mapped = a[6] == Py_True;
  need(xr->dim() == 3 && x->dim() == 3 && xr->size(2) == x->size(2) && wcc->dim() == 2);
  const int64_t r = xr->size(0), fr = xr->size(1), e = xr->size(2), n = x->size(0),
                fc = x->size(1), oc = wcc->size(0);
  shape_is(wcc, {oc, fc});
  shape_is(wcr, {oc, fr});
  int64_t orq = 0;
  if (wrr) {
    need(wrr->dim() == 2);
    orq = wrr->size(0);
    shape_is(wrr, {orq, fr});
  }
  need(orq > 0 || a[7] == Py_None);
  need(fr <= INT32_MAX && fc <= INT32_MAX && e <= INT32_MAX && oc <= INT32_MAX && orq <= INT32_MAX);
  const int32_t code = dtype_code(xr);
  for (const Ten* t : {&xr, &x, &wrr, &wcr, &wcc}) same(*t, xr);
  if (mapped) need(index->scalar_type() == c10::kInt && index->dim() == 1 &&
                   index->is_contiguous() && index->numel() == n);
  else offsets(index, r);
  Ten yr;
  if (orq > 0) yr = c.or_new(a[7], {r, orq, e}, xr->scalar_type());
  const Ten yc = c.or_new(a[8], {n, oc, e}, xr->scalar_type());
  const size_t bytes = rocs_ikbo_lcb_workspace_size(r, oc, e);
  Ten ws = c.get(a[9]);
  if (!ws) ws = c.or_new(Py_None, {(int64_t)(bytes > 0 ? bytes : 1)}, c10::kByte);
  void* s = stream_of(c.stream);
  if (mapped)
    run("rocs_ikbo_lcb_mapped", rocs_ikbo_lcb_mapped, xr.ptr(), x.ptr(), wrr.ptr(), wcr.ptr(),
        wcc.ptr(), index.i32(), r, n, (int32_t)fr, (int32_t)fc, (int32_t)orq, (int32_t)oc,
        (int32_t)e, code, data(yr), data(yc), data(ws), nbytes(ws), s);
  else
    run("rocs_ikbo_lcb", rocs_ikbo_lcb, xr.ptr(), x.ptr(), wrr.ptr(), wcr.ptr(), wcc.ptr(),
        index.i32(), r, n, (int32_t)fr, (int32_t)fc, (int32_t)orq, (int32_t)oc, (int32_t)e, code,
        data(yr), data(yc), data(ws), nbytes(ws), s);
  PyObject* first = Py_None;
  if (orq > 0) first = result(a[7], yr);
  else Py_INCREF(first);
  return pair(first, result(a[8], yc));
}

// cand_offsets, kv_offsets, num_cand, heads, q_len, plan, stream
PyObject* plan(PyObject* const* a) {
  Call c(a[6]);
  const Ten co = c.must(a[0]), ko = c.must(a[1]);
  const int64_t n = integer(a[2]), h = integer(a[3]), q = integer(a[4]);
  need(h >= 0 && h <= INT32_MAX && q >= 0 && q <= INT32_MAX);
  const int64_t r = ko->numel() - 1;
  offsets(ko, r);
  offsets(co, r);
  const int64_t bytes = (int64_t)rocs_dca_attention_plan_size(r);
  Ten p = c.get(a[5]);
  if (p) need(p->scalar_type() == c10::kByte && p->is_contiguous() && p->numel() >= bytes);
  else p = c.or_new(Py_None, {bytes}, c10::kByte);
  void* s = stream_of(c.stream);
  run("rocs_dca_attention_plan", rocs_dca_attention_plan, co.i32(), ko.i32(), r, n, (int32_t)q,
      (int32_t)h, data(p), nbytes(p), s);
  return result(a[5], p);
}

// q (or x), w_q, heads, k, v, cand_offsets, ids, kv_offsets, plan, residual,
// scale, out, out_sum, workspace, stream, ex (the extended entry point)
PyObject* attention(PyObject* const* a) {
  Call c(a[14]);
  const Ten q = c.must(a[0]), wq = c.get(a[1]), k = c.must(a[3]), v = c.must(a[4]),
            co = c.get(a[5]), ids = c.get(a[6]), ko = c.must(a[7]), pl = c.get(a[8]),
            res = c.get(a[9]);
  const float scale = scale_of(a[10]);
  int64_t n, t, h, d, d_in = 0;
  need(q->is_contiguous());
  if (wq) {
    need(q->dim() == 3 && wq->dim() == 2 && wq->is_contiguous() && !ids);
    h = integer(a[2]);
    n = q->size(0);
    t = q->size(1);
    d_in = q->size(2);
    need(h > 0 && wq->size(1) == d_in && wq->size(0) % h == 0 &&
         wq->scalar_type() == q->scalar_type());
    d = wq->size(0) / h;
  } else {
    need(q->dim() == 4);
    n = q->size(0);
    t = q->size(1);
    h = q->size(2);
    d = q->size(3);
  }
  const int32_t code = dtype_code(q);
  need(t <= INT32_MAX && h <= INT32_MAX && d <= INT32_MAX);
  need(k->dim() == 3 && v->dim() == 3 && k->sizes() == v->sizes() && k->size(1) == h &&
       k->size(2) == d);
  need(k->stride(2) == 1 && k->stride(1) == d && v->stride(2) == 1 && v->stride(1) == d &&
       k->stride(0) == v->stride(0));
  need(k->scalar_type() == q->scalar_type() && v->scalar_type() == q->scalar_type());
  const int64_t r = ko->numel() - 1;
  offsets(ko, r);
  if (ids) {
    need(!co && !pl && !res && ids->scalar_type() == c10::kInt && ids->dim() == 1 &&
         ids->is_contiguous() && ids->numel() == n);
  } else {
    need((bool)co);
    offsets(co, r);
  }
  if (pl) need(pl->scalar_type() == c10::kByte && pl->is_contiguous());
  const c10::IntArrayRef shape_q = q->sizes();
  const int64_t full[4] = {n, t, h, d};
  const c10::IntArrayRef shape = wq ? c10::IntArrayRef(full, 4) : shape_q;
  const Ten out = c.or_new(a[11], shape, q->scalar_type());
  Ten sum;
  if (res) {
    need(res->sizes() == shape && res->scalar_type() == q->scalar_type() && res->is_contiguous());
    sum = c.or_new(a[12], shape, q->scalar_type());
  }
  const int64_t stride = k->size(0) > 1 ? k->stride(0) : h * d;
  if (ids) {
    const size_t bytes = rocs_dca_attention_mapped_workspace_size(r, n);
    Ten ws = c.get(a[13]);
    if (!ws && bytes > 0) ws = c.or_new(Py_None, {(int64_t)bytes}, c10::kByte);
    void* s = stream_of(c.stream);
    run("rocs_dca_attention_mapped", rocs_dca_attention_mapped, q.ptr(), k.ptr(), v.ptr(),
        ids.i32(), ko.i32(), r, n, (int32_t)t, (int32_t)h, (int32_t)d, stride, scale, code,
        data(out), data(ws), nbytes(ws), s);
    return result(a[11], out);
  }
  void* s = stream_of(c.stream);
  if (a[15] != Py_True) {
    need(!wq && !pl);
    if (res)
      run("rocs_dca_attention_residual", rocs_dca_attention_residual, q.ptr(), k.ptr(), v.ptr(),
          co.i32(), ko.i32(), r, n, (int32_t)t, (int32_t)h, (int32_t)d, stride, scale, code,
          res.ptr(), data(out), data(sum), s);
    else
      run("rocs_dca_attention", rocs_dca_attention, q.ptr(), k.ptr(), v.ptr(), co.i32(), ko.i32(),
          r, n, (int32_t)t, (int32_t)h, (int32_t)d, stride, scale, code, data(out), s);
    return res ? pair(result(a[11], out), result(a[12], sum)) : result(a[11], out);
  }
  run("rocs_dca_attention_ex", rocs_dca_attention_ex, q.ptr(), d_in, wq.ptr(), k.ptr(), v.ptr(),
      co.i32(), ko.i32(), pl.ptr(), pl.bytes(), r, n, (int32_t)t, (int32_t)h, (int32_t)d, stride,
      scale, code, res.ptr(), data(out), data(sum), s);
  return res ? pair(result(a[11], out), result(a[12], sum)) : result(a[11], out);
}

// --- attention over histories, the cache's pages -----------------------------

// Row stride of [.., rows, heads, d] with dense rows (0: a single row).
int64_t row_stride(const Ten& t) {
  const int64_t n = t->dim(), h = t->size(n - 2), d = t->size(n - 1);
  need((d == 1 || t->stride(n - 1) == 1) && (h == 1 || t->stride(n - 2) == d));
  if (t->size(n - 3) <= 1) return 0;
  need(t->stride(n - 3) >= h * d);
  return t->stride(n - 3);
}

void int_vector(const Ten& t, int64_t n) {
  need(!t || (t->scalar_type() == c10::kInt && t->dim() == 1 && t->is_contiguous() &&
              t->numel() == n));
}

int32_t truth(PyObject* o) {
  need(o == Py_True || o == Py_False);
  return o == Py_True;
}

// None (0) or a count of at least 0.
int64_t count_of(PyObject* o) {
  const int64_t v = o == Py_None ? 0 : integer(o);
  need(v >= 0);
  return v;
}

// The caller's workspace, or a new one of `bytes`.
Ten scratch(Call& c, PyObject* o, size_t bytes) {
  Ten ws = c.get(o);
  if (!ws && bytes > 0) return c.or_new(Py_None, {(int64_t)bytes}, c10::kByte);
  need(!ws || ws->is_contiguous());
  return ws;
}

// The kernels run on the current device; ops.py takes calls on another.
void on_current_device(const Call& c) {
  PyObject* v = PyObject_CallNoArgs(g_get_device);
  if (v == nullptr) throw PyError();
  const long dev = PyLong_AsLong(v);
  Py_DECREF(v);
  need(dev == c.dev.index());
}

struct Rules {
  int64_t n, r, most;
  int32_t h, hk, d, code, causal;
  float cap, scale;
};

// What both attentions check alike; k: packed rows or pages.
Rules rules(const Ten& q, const Ten& k, const Ten& v, const Ten& off, const Ten& prefix,
            const Ten& slopes, PyObject* cap, PyObject* causal, PyObject* most, PyObject* scale) {
  Rules x;
  need(q->dim() == 3 && k->sizes() == v->sizes());
  const int64_t h = q->size(1), d = q->size(2), hk = k->size(k->dim() - 2);
  need(k->size(k->dim() - 1) == d && hk >= 1 && h <= INT32_MAX && d <= INT32_MAX && h % hk == 0);
  x.code = dtype_code(q);
  need(k->scalar_type() == q->scalar_type() && v->scalar_type() == q->scalar_type());
  x.n = q->size(0);
  x.h = (int32_t)h;
  x.hk = (int32_t)hk;
  x.d = (int32_t)d;
  x.r = off->numel() - 1;
  need(x.r >= 0);
  offsets(off, x.r);
  int_vector(prefix, x.r);
  need(!slopes || (slopes->scalar_type() == c10::kFloat && slopes->dim() == 1 &&
                   slopes->size(0) == h && slopes->is_contiguous()));
  x.cap = scale_of(cap);
  need(x.cap == 0.f || (x.cap >= 1e-30f && x.cap < 3.4e38f));
  x.causal = truth(causal);
  x.most = count_of(most);
  x.scale = scale_of(scale);
  return x;
}

// q, k, v, q_offsets, kv_offsets, causal, prefix_lens, q_docs, kv_docs, slopes,
// cap, max_kv_len, scale, out, workspace, stream
PyObject* history(PyObject* const* a) {
  Call c(a[15]);
  const Ten q = c.must(a[0]), k = c.must(a[1]), v = c.must(a[2]), qo = c.must(a[3]),
            ko = c.must(a[4]), prefix = c.get(a[6]), qd = c.get(a[7]), kd = c.get(a[8]),
            slopes = c.get(a[9]);
  on_current_device(c);
  need(k->dim() == 3);
  const Rules x = rules(q, k, v, qo, prefix, slopes, a[10], a[5], a[11], a[12]);
  const int64_t rows = k->size(0);
  offsets(ko, x.r);
  need((bool)qd == (bool)kd);
  int_vector(qd, x.n);
  int_vector(kd, rows);
  const int64_t qs = row_stride(q), ks = row_stride(k);
  need(row_stride(v) == ks);
  const Ten out = c.or_new(a[13], q->sizes(), q->scalar_type());
  const Ten ws = scratch(c, a[14], rocs_history_workspace_size(x.r, x.n, x.h, x.hk, x.d,
                                                               x.most > 0 ? x.most : rows, x.code));
  void* s = stream_of(c.stream);
  run("rocs_history_attention", rocs_history_attention, q.ptr(), qs, k.ptr(), v.ptr(), ks,
      qo.i32(), ko.i32(), prefix.i32(), qd.i32(), kd.i32(), slopes.f32(), x.r, x.n, rows, x.h,
      x.hk, x.d, x.scale, x.cap, x.causal, x.most, x.code, data(out), data(ws), nbytes(ws), s);
  return result(a[13], out);
}

// q, k_pages, v_pages, page_table, kv_lens, q_offsets, slots, causal,
// prefix_lens, slopes, cap, max_kv_len, scale, out, workspace, stream
PyObject* paged(PyObject* const* a) {
  Call c(a[15]);
  const Ten q = c.must(a[0]), k = c.must(a[1]), v = c.must(a[2]), table = c.must(a[3]),
            lens = c.must(a[4]), qo = c.must(a[5]), slots = c.get(a[6]), prefix = c.get(a[8]),
            slopes = c.get(a[9]);
  on_current_device(c);
  need(k->dim() == 4);
  const Rules x = rules(q, k, v, qo, prefix, slopes, a[10], a[7], a[11], a[12]);
  const int64_t pages = k->size(0), page = k->size(1);
  need(pages >= 1 && page >= 1 && page <= INT32_MAX);
  need(table->scalar_type() == c10::kInt && table->dim() == 2 && table->is_contiguous() &&
       table->size(1) >= 1);
  const int64_t n_slots = table->size(0), width = table->size(1);
  need(width <= INT32_MAX / page);
  int_vector(lens, n_slots);
  int_vector(slots, x.r);
  need(slots || x.r <= n_slots);
  const int64_t qs = row_stride(q), ks = row_stride(k);
  need(row_stride(v) == ks);
  int64_t ps = 0;
  if (pages > 1) {
    ps = k->stride(0);
    need(v->stride(0) == ps && ps >= (page - 1) * ks + (int64_t)x.hk * x.d);
  }
  const int64_t all = width * page, bound = x.most > 0 && x.most < all ? x.most : all;
  const Ten out = c.or_new(a[13], q->sizes(), q->scalar_type());
  const Ten ws = scratch(c, a[14],
                         rocs_history_workspace_size(x.r, x.n, x.h, x.hk, x.d, bound, x.code));
  void* s = stream_of(c.stream);
  run("rocs_paged_attention", rocs_paged_attention, q.ptr(), qs, k.ptr(), v.ptr(), ps, ks,
      table.i32(), width, lens.i32(), slots.i32(), n_slots, qo.i32(), prefix.i32(), slopes.f32(),
      x.r, x.n, pages, (int32_t)page, x.h, x.hk, x.d, x.scale, x.cap, x.causal, x.most, x.code,
      data(out), data(ws), nbytes(ws), s);
  return result(a[13], out);
}

// A cache's bookkeeping, changed in place.
struct State {
  int32_t *table, *lens, *refs;
  int64_t slots, width, pages;
};
State state_of(Call& c, PyObject* table, PyObject* lens, PyObject* refs) {
  const Ten t = c.must(table), l = c.must(lens), r = c.must(refs);
  on_current_device(c);
  need(t->scalar_type() == c10::kInt && t->dim() == 2 && t->is_contiguous() && t->size(0) >= 1 &&
       t->size(1) >= 1);
  int_vector(l, t->size(0));
  int_vector(r, r->numel());
  need(r->numel() >= 1);
  return {static_cast<int32_t*>(t.ptr()), static_cast<int32_t*>(l.ptr()),
          static_cast<int32_t*>(r.ptr()), t->size(0), t->size(1), r->numel()};
}

// layers, page size and row bytes of a pool [layers, pages, page_size, ...].
struct Layers {
  int64_t layers, page, row_bytes;
};
Layers layers_of(const Ten& pool, int64_t pages) {
  need(pool->dim() >= 4 && pool->is_contiguous() && pool->size(1) == pages && pool->numel() > 0 &&
       pool->size(2) <= INT32_MAX);
  const int64_t l = pool->size(0), p = pool->size(2);
  return {l, p, pool->numel() / (l * pages * p) * (int64_t)pool->element_size()};
}

// slots, row_offsets, num_rows, page_table, lens, refs, page_size, rows,
// status, workspace, stream
PyObject* cache_reserve(PyObject* const* a) {
  Call c(a[10]);
  const Ten slots = c.must(a[0]), off = c.must(a[1]);
  const int64_t n = slots->numel(), m = integer(a[2]), page = integer(a[6]);
  int_vector(slots, n);
  offsets(off, n);
  need(m >= 0 && (n > 0 || m == 0) && page >= 1 && page <= INT32_MAX);
  const State st = state_of(c, a[3], a[4], a[5]);
  const Ten rows = c.or_new(a[7], {m}, c10::kInt), status = c.or_new(a[8], {2}, c10::kInt);
  const Ten ws = scratch(c, a[9], rocs_cache_workspace_size(n, st.pages));
  void* s = stream_of(c.stream);
  run("rocs_cache_reserve", rocs_cache_reserve, slots.i32(), off.i32(), n, m, st.table, st.width,
      st.lens, st.slots, st.refs, st.pages, (int32_t)page, static_cast<int32_t*>(data(rows)),
      static_cast<int32_t*>(data(status)), data(ws), nbytes(ws), s);
  return pair(result(a[7], rows), result(a[8], status));
}

// x, rows, pool, stream
PyObject* cache_write(PyObject* const* a) {
  Call c(a[3]);
  const Ten x = c.must(a[0]), rows = c.must(a[1]), pool = c.must(a[2]);
  on_current_device(c);
  need(pool->dim() >= 3 && pool->is_contiguous() && pool->numel() > 0 &&
       x->scalar_type() == pool->scalar_type() && x->dim() >= 2);
  const int64_t pool_rows = pool->size(0) * pool->size(1), width = pool->numel() / pool_rows;
  const int64_t m = x->size(0), size = x->element_size();
  need(x->numel() == m * width && m > 0);
  int_vector(rows, m);
  int64_t dense = 1;                       // every dimension after the first is dense
  for (int64_t i = x->dim() - 1; i > 0; --i) {
    need(x->size(i) == 1 || x->stride(i) == dense);
    dense *= x->size(i);
  }
  need(m == 1 || x->stride(0) >= width);
  void* s = stream_of(c.stream);
  run("rocs_cache_write", rocs_cache_write, x.ptr(), (m > 1 ? x->stride(0) : width) * size,
      rows.i32(), m, pool.ptr(), pool_rows, width * size, s);
  Py_INCREF(a[2]);
  return a[2];
}

// parents, children, page_table, lens, refs, pool, status, workspace, stream
PyObject* cache_fork(PyObject* const* a) {
  Call c(a[8]);
  const Ten par = c.must(a[0]), kid = c.must(a[1]);
  const int64_t n = par->numel();
  int_vector(par, n);
  int_vector(kid, n);
  const State st = state_of(c, a[2], a[3], a[4]);
  const Ten pool = c.must(a[5]);
  const Layers l = layers_of(pool, st.pages);
  const Ten status = c.or_new(a[6], {2}, c10::kInt);
  const Ten ws = scratch(c, a[7], rocs_cache_workspace_size(n, st.pages));
  void* s = stream_of(c.stream);
  run("rocs_cache_fork", rocs_cache_fork, par.i32(), kid.i32(), n, st.table, st.width, st.lens,
      st.slots, st.refs, st.pages, (int32_t)l.page, pool.ptr(), l.layers, l.row_bytes,
      static_cast<int32_t*>(data(status)), data(ws), nbytes(ws), s);
  return result(a[6], status);
}

// slots, page_table, lens, refs, page_size, stream
PyObject* cache_free(PyObject* const* a) {
  Call c(a[5]);
  const Ten slots = c.must(a[0]);
  const int64_t n = slots->numel(), page = integer(a[4]);
  int_vector(slots, n);
  need(page >= 1 && page <= INT32_MAX);
  const State st = state_of(c, a[1], a[2], a[3]);
  void* s = stream_of(c.stream);
  run("rocs_cache_free", rocs_cache_free, slots.i32(), n, st.table, st.width, st.lens, st.slots,
      st.refs, st.pages, (int32_t)page, s);
  Py_RETURN_TRUE;
}

// page_table, lens, refs, pool, status, workspace, stream
PyObject* cache_compact(PyObject* const* a) {
  Call c(a[6]);
  const State st = state_of(c, a[0], a[1], a[2]);
  const Ten pool = c.must(a[3]);
  const Layers l = layers_of(pool, st.pages);
  const Ten status = c.or_new(a[4], {2}, c10::kInt);
  const Ten ws = scratch(c, a[5], rocs_cache_workspace_size(0, st.pages));
  void* s = stream_of(c.stream);
  run("rocs_cache_compact", rocs_cache_compact, st.table, st.width, st.slots, st.refs, st.pages,
      (int32_t)l.page, pool.ptr(), l.layers, l.row_bytes, static_cast<int32_t*>(data(status)),
      data(ws), nbytes(ws), s);
  return result(a[4], status);
}

// --- adapters, rotated rows, a cache in 4 bits --------------------------------

// x, w, a, b, offsets, adapter_ids, scales, bias, activation, out, workspace, stream
PyObject* adapter(PyObject* const* a) {
  Call c(a[11]);
  const Ten x = c.must(a[0]), w = c.must(a[1]), la = c.must(a[2]), lb = c.must(a[3]),
            off = c.must(a[4]), ids = c.must(a[5]), scales = c.get(a[6]), bias = c.get(a[7]);
  on_current_device(c);
  need(x->dim() == 2 && w->dim() == 2 && la->dim() == 3 && lb->dim() == 3);
  const int64_t n = x->size(0), k = x->size(1), d = w->size(0), count = la->size(0), rank = la->size(1);
  need(w->size(1) == k && k >= 1 && d >= 1 && rank >= 1 && rank <= INT32_MAX && lb->size(0) == count &&
       la->size(2) == k && lb->size(1) == d && lb->size(2) == rank);
  const int32_t code = dtype_code(x), act = activation(a[8]);
  const c10::ScalarType type = x->scalar_type();
  need(w->scalar_type() == type && la->scalar_type() == type && lb->scalar_type() == type);
  need(w->is_contiguous() && la->is_contiguous() && lb->is_contiguous());
  need((k == 1 || x->stride(1) == 1) && (n <= 1 || x->stride(0) >= k));
  const int64_t r = off->numel() - 1;
  need(r >= 0);
  offsets(off, r);
  int_vector(ids, r);
  need(!scales || (scales->scalar_type() == c10::kFloat && scales->dim() == 1 &&
                   scales->size(0) == count && scales->is_contiguous()));
  need(!bias || (bias->scalar_type() == c10::kFloat && bias->dim() == 1 && bias->size(0) == d &&
                 bias->is_contiguous()));
  const Ten out = c.or_new(a[9], {n, d}, type);
  const Ten ws = scratch(c, a[10], rocs_adapter_workspace_size(r, n, k, d, (int32_t)rank, code));
  void* s = stream_of(c.stream);
  run("rocs_adapter_linear", rocs_adapter_linear, x.ptr(), n > 1 ? x->stride(0) : 0, w.ptr(),
      la.ptr(), lb.ptr(), scales.f32(), bias.f32(), off.i32(), ids.i32(), r, n, k, d, (int32_t)rank,
      count, code, act, data(out), data(ws), nbytes(ws), s);
  return result(a[9], out);
}

// A rotation's arguments.
struct Turn {
  int64_t rot = 0, r = 0, slots = 0;
};
Turn turn_of(const Ten& freqs, const Ten& pos, const Ten& off, const Ten& slots, const Ten& lens,
             int64_t m, int64_t d) {
  Turn x;
  int_vector(pos, m);
  if (freqs) {
    need(freqs->scalar_type() == c10::kFloat && freqs->dim() == 1 && freqs->is_contiguous() &&
         2 * freqs->numel() <= d);
    x.rot = 2 * freqs->numel();
  }
  if (off) {
    x.r = off->numel() - 1;
    need(x.r >= 0);
    offsets(off, x.r);
    int_vector(slots, x.r);
    if (lens) {
      x.slots = lens->numel();
      int_vector(lens, x.slots);
      need(slots || x.r <= x.slots);
    }
  } else {
    need(!slots && !lens);
  }
  need(x.rot == 0 || pos || (off && lens));
  return x;
}

// x, freqs, positions, offsets, slots, lens, interleaved, out, stream
PyObject* rotate(PyObject* const* a) {
  Call c(a[8]);
  const Ten x = c.must(a[0]), freqs = c.get(a[1]), pos = c.get(a[2]), off = c.get(a[3]),
            slots = c.get(a[4]), lens = c.get(a[5]);
  on_current_device(c);
  need(x->dim() == 3 && x->size(1) >= 1 && x->size(2) >= 1 && x->size(1) <= INT32_MAX &&
       x->size(2) <= INT32_MAX);
  const int64_t m = x->size(0), h = x->size(1), d = x->size(2);
  const int32_t code = dtype_code(x), inter = truth(a[6]);
  const Turn t = turn_of(freqs, pos, off, slots, lens, m, d);
  const int64_t stride = row_stride(x);
  const Ten out = c.or_new(a[7], x->sizes(), x->scalar_type());
  void* s = stream_of(c.stream);
  run("rocs_rotate", rocs_rotate, x.ptr(), stride, freqs.f32(), (int32_t)t.rot, inter, pos.i32(),
      off.i32(), slots.i32(), lens.i32(), t.r, t.slots, m, (int32_t)h, (int32_t)d, code, data(out), s);
  return result(a[7], out);
}

// rows, pool, kv_heads, head_dim, bf16, out, stream
PyObject* read_fp4(PyObject* const* a) {
  Call c(a[6]);
  const Ten rows = c.must(a[0]), pool = c.must(a[1]);
  on_current_device(c);
  const int64_t hk = integer(a[2]), d = integer(a[3]), m = rows->numel();
  need(hk >= 1 && hk <= INT32_MAX && d >= 1 && d <= INT32_MAX);
  const int64_t row = (int64_t)rocs_fp4_row_bytes((int32_t)hk, (int32_t)d);
  need(row > 0 && pool->scalar_type() == c10::kByte && pool->dim() == 3 && pool->is_contiguous() &&
       pool->size(2) == row && pool->size(0) >= 1 && pool->size(1) >= 1);
  int_vector(rows, m);
  const bool bf16 = truth(a[4]) != 0;
  const Ten out = c.or_new(a[5], {m, 2, hk, d}, bf16 ? c10::kBFloat16 : c10::kFloat);
  void* s = stream_of(c.stream);
  run("rocs_cache_read_fp4", rocs_cache_read_fp4, rows.i32(), m, pool.ptr(), pool->size(0) * pool->size(1),
      (int32_t)hk, (int32_t)d, bf16 ? ROCS_DTYPE_BF16 : ROCS_DTYPE_F32, data(out), s);
  return result(a[5], out);
}

// k, v, rows, pool, freqs, q, positions, offsets, slots, lens, interleaved,
// q_out, stream
PyObject* append(PyObject* const* a) {
  Call c(a[12]);
  const Ten k = c.must(a[0]), v = c.must(a[1]), rows = c.must(a[2]), pool = c.must(a[3]),
            freqs = c.get(a[4]), q = c.get(a[5]), pos = c.get(a[6]), off = c.get(a[7]),
            slots = c.get(a[8]), lens = c.get(a[9]);
  on_current_device(c);
  need(k->dim() == 3 && k->sizes() == v->sizes() && k->scalar_type() == v->scalar_type());
  const int64_t m = k->size(0), hk = k->size(1), d = k->size(2);
  need(hk >= 1 && d >= 1 && hk <= INT32_MAX && d <= INT32_MAX);
  const int32_t code = dtype_code(k), inter = truth(a[10]);
  const int64_t stride = row_stride(k);
  need(row_stride(v) == stride);
  int_vector(rows, m);
  const Turn t = turn_of(freqs, pos, off, slots, lens, m, d);
  int32_t form = ROCS_POOL_ROWS;
  need(pool->is_contiguous() && pool->dim() >= 3 && pool->size(0) >= 1 && pool->size(1) >= 1);
  const int64_t pool_rows = pool->size(0) * pool->size(1);
  if (pool->scalar_type() == c10::kByte) {
    form = ROCS_POOL_FP4;
    const int64_t row = (int64_t)rocs_fp4_row_bytes((int32_t)hk, (int32_t)d);
    need(pool->dim() == 3 && row > 0 && pool->size(2) == row);
  } else {
    need(pool->scalar_type() == k->scalar_type() && pool->dim() == 5 && pool->size(2) == 2 &&
         pool->size(3) == hk && pool->size(4) == d);
  }
  int64_t h = 0, q_stride = 0;
  Ten q_out;
  need(q || a[11] == Py_None);
  if (q) {
    need(q->dim() == 3 && q->size(0) == m && q->size(1) >= 1 && q->size(1) <= INT32_MAX &&
         q->size(2) == d && q->scalar_type() == k->scalar_type());
    h = q->size(1);
    q_stride = row_stride(q);
    q_out = c.or_new(a[11], q->sizes(), q->scalar_type());
  }
  void* s = stream_of(c.stream);
  run("rocs_cache_append", rocs_cache_append, q.ptr(), q_stride, k.ptr(), v.ptr(), stride,
      rows.i32(), freqs.f32(), (int32_t)t.rot, inter, pos.i32(), off.i32(), slots.i32(), lens.i32(), t.r,
      t.slots, m, (int32_t)h, (int32_t)hk, (int32_t)d, code, pool.ptr(), pool_rows, form,
      data(q_out), s);
  if (!q) Py_RETURN_TRUE;
  return result(a[11], q_out);
}

// q, pages, page_table, kv_lens, q_offsets, kv_heads, slots, causal,
// prefix_lens, slopes, cap, max_kv_len, scale, out, workspace, stream
PyObject* paged_fp4(PyObject* const* a) {
  Call c(a[15]);
  const Ten q = c.must(a[0]), pages = c.must(a[1]), table = c.must(a[2]), lens = c.must(a[3]),
            qo = c.must(a[4]), slots = c.get(a[6]), prefix = c.get(a[8]), slopes = c.get(a[9]);
  on_current_device(c);
  need(q->dim() == 3);
  const int64_t n = q->size(0), h = q->size(1), d = q->size(2), hk = integer(a[5]);
  need(hk >= 1 && hk <= h && h <= INT32_MAX && h % hk == 0 && d <= INT32_MAX);
  const int32_t code = dtype_code(q), causal = truth(a[7]);
  const int64_t row = (int64_t)rocs_fp4_row_bytes((int32_t)hk, (int32_t)d);
  need(row > 0 && pages->scalar_type() == c10::kByte && pages->dim() == 3 && pages->is_contiguous() &&
       pages->size(2) == row && pages->size(0) >= 1 && pages->size(1) >= 1 &&
       pages->size(1) <= INT32_MAX);
  const int64_t n_pages = pages->size(0), page = pages->size(1), r = qo->numel() - 1;
  need(r >= 0);
  offsets(qo, r);
  int_vector(prefix, r);
  int_vector(slots, r);
  need(!slopes || (slopes->scalar_type() == c10::kFloat && slopes->dim() == 1 &&
                   slopes->size(0) == h && slopes->is_contiguous()));
  const float cap = scale_of(a[10]), scale = scale_of(a[12]);
  need(cap == 0.f || (cap >= 1e-30f && cap < 3.4e38f));
  const int64_t most = count_of(a[11]);
  need(table->scalar_type() == c10::kInt && table->dim() == 2 && table->is_contiguous() &&
       table->size(1) >= 1);
  const int64_t n_slots = table->size(0), width = table->size(1);
  need(width <= INT32_MAX / page);
  int_vector(lens, n_slots);
  need(slots || r <= n_slots);
  const int64_t qs = row_stride(q), all = width * page, bound = most > 0 && most < all ? most : all;
  const Ten out = c.or_new(a[13], q->sizes(), q->scalar_type());
  const Ten ws = scratch(c, a[14], rocs_paged_fp4_workspace_size(r, n, (int32_t)h, (int32_t)hk,
                                                                 (int32_t)d, bound, code));
  void* s = stream_of(c.stream);
  run("rocs_paged_attention_fp4", rocs_paged_attention_fp4, q.ptr(), qs, pages.ptr(), table.i32(),
      width, lens.i32(), slots.i32(), n_slots, qo.i32(), prefix.i32(), slopes.f32(), r, n, n_pages,
      (int32_t)page, (int32_t)h, (int32_t)hk, (int32_t)d, scale, cap, causal, most, code, data(out),
      data(ws), nbytes(ws), s);
  return result(a[13], out);
}

#define ROCS_ENTRY(name, n) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<n, name>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    ROCS_ENTRY(linear, 12),   ROCS_ENTRY(glm_linear, 14), ROCS_ENTRY(mlp2, 13),
    ROCS_ENTRY(fm_linear, 10), ROCS_ENTRY(lcb, 11),        ROCS_ENTRY(plan, 7),
    ROCS_ENTRY(attention, 16), ROCS_ENTRY(history, 16),    ROCS_ENTRY(paged, 16),
    ROCS_ENTRY(cache_reserve, 11), ROCS_ENTRY(cache_write, 4), ROCS_ENTRY(cache_fork, 9),
    ROCS_ENTRY(cache_free, 6), ROCS_ENTRY(cache_compact, 7),
    ROCS_ENTRY(adapter, 12),  ROCS_ENTRY(append, 13),     ROCS_ENTRY(paged_fp4, 16),
    ROCS_ENTRY(rotate, 9),    ROCS_ENTRY(read_fp4, 7),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

PyObject* attribute(const char* module, const char* name) {
  PyObject* m = PyImport_ImportModule(module);
  if (m == nullptr) return nullptr;
  PyObject* v = PyObject_GetAttrString(m, name);
  Py_DECREF(m);
  return v;
}

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  g_get_device = attribute("torch._C", "_cuda_getDevice");
  g_raw_stream = attribute("torch._C", "_cuda_getCurrentRawStream");
  g_check = attribute("paper_2607_27744_amd._lib", "check");
  g_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  if (!g_get_device || !g_raw_stream || !g_check || !g_cuda_stream) return nullptr;
  return PyModule_Create(&g_module);
}
