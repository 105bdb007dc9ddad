// What the native calls share: tensor and argument checks, references, the library call and its error, the
// outputs and the split-key scratch.
#pragma once

#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/TensorSubclassLikeUtils.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstdint>
#include <exception>
#include <memory>

#include "unstep.h"

namespace {

constexpr int64_t kD = UNSTEP_HEAD_DIM;

// What the calls need of a Cache object (the handle stays owned by it).
struct CacheInfo {
  unstep_cache* handle;
  int64_t B, H, T;
  c10::Device device;
  PyObject* scratch_methods;    // the tuple (Cache.workspace, Cache.workspace_bytes, Cache._step_workspace)
  ~CacheInfo() { Py_XDECREF(scratch_methods); }
};

// A plain strided tensor on a GPU: exactly torch.Tensor or Parameter, no subclass, no functorch
// wrapper, no fake or tracing tensor.
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || at::isTensorSubclassLike(t) || t.is_neg())
    return nullptr;
  return &t;
}

bool usable(const at::Tensor& t) { return t.defined() && t.is_cuda() && !at::isTensorSubclassLike(t) && t.has_storage(); }

bool is(const at::Tensor* t, at::ScalarType type, at::IntArrayRef shape, c10::Device dev) {
  return t && t->scalar_type() == type && t->sizes() == shape && t->device() == dev && t->is_contiguous();
}

bool to_i32(PyObject* o, int32_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long x = PyLong_AsLongAndOverflow(o, &over);
  if (over || x < INT32_MIN || x > INT32_MAX) return false;
  *v = int32_t(x);
  return true;
}

bool to_f64(PyObject* o, double* v) {
  if (!PyFloat_CheckExact(o)) return false;
  *v = PyFloat_AS_DOUBLE(o);
  return true;
}

void* current_stream() { return c10::hip::getCurrentHIPStreamMasqueradingAsCUDA().stream(); }

PyObject* none() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// A Python reference owned here.
struct Ref {
  PyObject* o;
  explicit Ref(PyObject* x) : o(x) {}
  Ref(const Ref&) = delete;
  ~Ref() { Py_XDECREF(o); }
  PyObject* release() {
    PyObject* r = o;
    o = nullptr;
    return r;
  }
};

// Sets the package's UnstepError(rc, message) for the library's last error on this thread.
void raise(int rc) {
  const Ref pkg{PyImport_ImportModule("paper_2609_32518_amd")};
  const Ref type{pkg.o ? PyObject_GetAttrString(pkg.o, "UnstepError") : nullptr};
  const Ref err{type.o ? PyObject_CallFunction(type.o, "is", rc, unstep_last_error()) : nullptr};
  if (err.o) PyErr_SetObject(type.o, err.o);
}

// Runs the library call without the GIL; on an error of the library false, with that error raised.
// A tensor's data_ptr may throw (a storage without memory), so the pointers are read before this: an
// exception must not leave a region without the GIL.
template <class F>
bool call(F&& f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = f();
  Py_END_ALLOW_THREADS;
  if (rc != UNSTEP_OK) raise(rc);
  return rc == UNSTEP_OK;
}

// No C++ exception leaves a function of the module.
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception&) {
    return none();
  }
}

at::Tensor new_bf16(at::IntArrayRef shape, c10::Device dev) {
  return at::empty(shape, at::TensorOptions().dtype(at::kBFloat16).device(dev));
}

void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// q, k, v of a chunk: [B, N, H, 128] bf16, unit stride on the last axis, batch stride N * token
// stride, one (token, head) stride pair for all; cos, sin: fp32 [N, pairs] (pairs < 0: any).
struct Chunk {
  int32_t f0, C;
  int64_t N;
  const at::Tensor *q, *k, *v, *cos, *sin;
  int64_t ts, hs, pairs;
  const void *qp, *kp, *vp;
  const float *cp, *sp;
};

bool chunk_of(const CacheInfo& c, PyObject* const* a, bool q_optional, int64_t pairs, Chunk* o) {
  if (!to_i32(a[0], &o->f0) || !to_i32(a[1], &o->C) || o->C < 1) return false;
  o->N = int64_t(o->C) * c.T;
  const int64_t shape[4] = {c.B, o->N, c.H, kD};
  o->q = nullptr;
  if (a[2] != Py_None || !q_optional) {
    if (!(o->q = plain(a[2]))) return false;
  }
  if (!(o->k = plain(a[3])) || !(o->v = plain(a[4]))) return false;
  o->ts = o->hs = -1;
  for (const at::Tensor* t : {o->k, o->v, o->q}) {
    if (!t) continue;
    if (t->scalar_type() != at::kBFloat16 || t->sizes() != at::IntArrayRef(shape, 4) || t->device() != c.device) return false;
    if (t->stride(3) != 1 || (c.B > 1 && t->stride(0) != o->N * t->stride(1))) return false;
    if (t == o->k) {
      o->ts = t->stride(1);
      o->hs = t->stride(2);
    } else if (t->stride(1) != o->ts || t->stride(2) != o->hs) {
      return false;
    }
  }
  o->cos = plain(a[5]);
  o->sin = plain(a[6]);
  if (pairs < 0 && o->cos && o->cos->dim() == 2) pairs = o->cos->size(1);
  const int64_t tab[2] = {o->N, pairs};
  o->pairs = pairs;
  if (!is(o->cos, at::kFloat, at::IntArrayRef(tab, 2), c.device) || !is(o->sin, at::kFloat, at::IntArrayRef(tab, 2), c.device))
    return false;
  o->qp = ptr(o->q);
  o->kp = ptr(o->k);
  o->vp = ptr(o->v);
  o->cp = static_cast<const float*>(ptr(o->cos));
  o->sp = static_cast<const float*>(ptr(o->sin));
  return true;
}

// A given [B, N, H, 128] output checked, or a new one in *made.
const at::Tensor* chunk_out(const CacheInfo& c, int64_t N, PyObject* o, at::Tensor* made) {
  const int64_t shape[4] = {c.B, N, c.H, kD};
  if (o == Py_None) {
    *made = new_bf16(at::IntArrayRef(shape, 4), c.device);
    return usable(*made) ? made : nullptr;
  }
  const at::Tensor* t = plain(o);
  return is(t, at::kBFloat16, at::IntArrayRef(shape, 4), c.device) ? t : nullptr;
}

// The object that a call returns, made before the library's call (null, with a Python error, if that
// fails).
Ref result(PyObject* given, const at::Tensor& made) {
  if (given != Py_None) {
    Py_INCREF(given);
    return Ref{given};
  }
  return Ref{THPVariable_Wrap(made)};
}

// lse: None or fp32 [B, H, N]
bool lse_of(const CacheInfo& c, int64_t N, PyObject* o, float** p) {
  *p = nullptr;
  if (o == Py_None) return true;
  const int64_t shape[3] = {c.B, c.H, N};
  const at::Tensor* t = plain(o);
  if (!is(t, at::kFloat, at::IntArrayRef(shape, 3), c.device)) return false;
  *p = static_cast<float*>(ptr(t));
  return true;
}

// Whether the scratch methods that a call would ask (`step`: _step_workspace too) are the binding's own on
// `owner`: a subclass, or a program that replaced one, is asked through the Python path.
PyObject* scratch_names[3];    // interned, made with the module
bool own_scratch(const CacheInfo& c, PyObject* owner, bool step) {
  for (int i = 0; i < (step ? 3 : 2); ++i) {
    const Ref m{PyObject_GetAttr(owner, scratch_names[i])};
    if (!m.o || !PyMethod_Check(m.o) || PyMethod_GET_FUNCTION(m.o) != PyTuple_GET_ITEM(c.scratch_methods, i) ||
        PyMethod_GET_SELF(m.o) != owner)
      return false;
  }
  return true;
}

// The split-key scratch: the given tensor, or (use_split) the one the Cache object keeps as _ws,
// replaced by a larger one when it is too small, as Cache.workspace does.  The kept tensor is held in
// *hold until the call has been enqueued.
bool workspace_of(const CacheInfo& c, int32_t f0, int32_t C, int32_t W, PyObject* given, PyObject* use_split, PyObject* owner,
                  bool step, at::Tensor* hold, void** p, size_t* bytes) {
  *p = nullptr;
  *bytes = 0;
  if (given != Py_None) {
    const at::Tensor* t = plain(given);
    if (!t || t->device() != c.device || !t->is_contiguous()) return false;
    *p = t->data_ptr();
    *bytes = size_t(t->numel()) * t->element_size();
    return true;
  }
  if (use_split == Py_False) return true;
  if (use_split != Py_True || !own_scratch(c, owner, step)) return false;
  size_t need = 0;
  if (unstep_attn_workspace_size(c.handle, f0, C, W, &need) != UNSTEP_OK) return false;
  if (need == 0) return true;
  const Ref kept{PyObject_GetAttrString(owner, "_ws")};
  if (!kept.o) return false;
  const at::Tensor* t = kept.o == Py_None ? nullptr : plain(kept.o);
  if (kept.o != Py_None && !t) return false;
  if (t && size_t(t->numel()) >= need) {
    *hold = *t;
  } else {
    *hold = at::empty({int64_t(need)}, at::TensorOptions().dtype(at::kByte).device(c.device));
    if (!usable(*hold)) return false;
    const Ref made{THPVariable_Wrap(*hold)};
    if (!made.o || PyObject_SetAttrString(owner, "_ws", made.o) != 0) return false;
  }
  *p = hold->data_ptr();
  *bytes = size_t(hold->numel());
  return true;
}

}  // namespace
