// The native calls of the rotary options and the quantised cache, as calls.cpp has those of the bf16 path: the
// ordinary call (plain CUDA tensors on the current device, the current stream) is checked, its outputs
// allocated and its kernels enqueued without Python in between; anything else returns None before the
// library's call and takes the Python path.
#include "common.hpp"

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPGraphsC10Utils.h>

#include <cstring>

namespace {

constexpr int64_t kScales = 4;
constexpr const char* kBf16Capsule = "unstep.Cache";
constexpr const char* kMx8Capsule = "unstep.CacheMX8";

bool current(c10::Device d) { return d.index() == c10::hip::current_device(); }

const CacheInfo* cache_of(PyObject* o, const char* name) {
  const auto* c = static_cast<const CacheInfo*>(PyCapsule_GetPointer(o, name));
  return c && current(c->device) ? c : nullptr;
}

bool layout_of(PyObject* o, int32_t* layout) {
  const char* s = PyUnicode_CheckExact(o) ? PyUnicode_AsUTF8(o) : nullptr;
  if (!s) return false;
  if (std::strcmp(s, "half") == 0)
    *layout = UNSTEP_ROTARY_HALF;
  else if (std::strcmp(s, "interleaved") == 0)
    *layout = UNSTEP_ROTARY_INTERLEAVED;
  else
    return false;
  return true;
}

// The norm weights (both None, or wk and, with queries, wq) and epsilon.
bool norm_of(const CacheInfo& c, bool with_q, PyObject* owq, PyObject* owk, PyObject* oeps, const void** wq, const void** wk,
             double* eps) {
  *wq = *wk = nullptr;
  if (!to_f64(oeps, eps)) return false;
  if (owq == Py_None && owk == Py_None) return true;
  const int64_t shape[1] = {c.H * kD};
  const at::Tensor* k = plain(owk);
  if (!is(k, at::kBFloat16, at::IntArrayRef(shape, 1), c.device)) return false;
  *wk = ptr(k);
  if (!with_q) return owq == Py_None;
  const at::Tensor* q = plain(owq);
  if (!is(q, at::kBFloat16, at::IntArrayRef(shape, 1), c.device)) return false;
  *wq = ptr(q);
  return true;
}

// A given tensor of this type and shape checked, or a new one in *made.
const at::Tensor* out_of(at::ScalarType type, at::IntArrayRef shape, c10::Device dev, PyObject* o, at::Tensor* made) {
  if (o == Py_None) {
    *made = at::empty(shape, at::TensorOptions().dtype(type).device(dev));
    return usable(*made) ? made : nullptr;
  }
  const at::Tensor* t = plain(o);
  return is(t, type, shape, dev) ? t : nullptr;
}

// Two new tensors in one allocation, the second after the first (whose bytes are a multiple of 32): an
// allocation and its release cost the host 1.3 us, a third of a small call.
bool two(c10::Device dev, at::ScalarType type_a, at::IntArrayRef a, at::ScalarType type_b, at::IntArrayRef b, at::Tensor* ta,
         at::Tensor* tb) {
  const int64_t bytes_a = c10::multiply_integers(a) * int64_t(c10::elementSize(type_a));
  const int64_t bytes_b = c10::multiply_integers(b) * int64_t(c10::elementSize(type_b));
  const at::Tensor base = at::empty({bytes_a + bytes_b}, at::TensorOptions().dtype(at::kByte).device(dev));
  if (!usable(base)) return false;
  auto part = [&](at::ScalarType type, at::IntArrayRef shape, int64_t offset) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base.storage()), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                            c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
    t.unsafeGetTensorImpl()->set_storage_offset(offset / int64_t(c10::elementSize(type)));
    return t;
  };
  *ta = part(type_a, a, 0);
  *tb = part(type_b, b, bytes_a);
  return true;
}

// The quantised queries and their scales, given or made.
struct Queries {
  at::Tensor made8, made_scale;
  const at::Tensor *q8, *scale;
  bool get(const CacheInfo& c, int64_t N, PyObject* o8, PyObject* os) {
    const int64_t v[4] = {c.B, N, c.H, kD}, s[4] = {c.B, N, c.H, kScales};
    if (o8 == Py_None && os == Py_None) {
      q8 = &made8;
      scale = &made_scale;
      return two(c.device, at::kFloat8_e4m3fn, at::IntArrayRef(v, 4), at::kByte, at::IntArrayRef(s, 4), &made8, &made_scale);
    }
    q8 = out_of(at::kFloat8_e4m3fn, at::IntArrayRef(v, 4), c.device, o8, &made8);
    scale = q8 ? out_of(at::kByte, at::IntArrayRef(s, 4), c.device, os, &made_scale) : nullptr;
    return scale != nullptr;
  }
};

// Whether a call would take the kept scratch into a captured graph, which needs one of its own: the Python path.
bool captures_scratch(PyObject* given, PyObject* use_split) {
  if (given != Py_None || use_split == Py_False) return false;
  return current_stream() && c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None;
}

// (a, b) as a tuple, made before the library's call.
Ref pair(PyObject* given_a, const at::Tensor& a, PyObject* given_b, const at::Tensor& b) {
  Ref ra = result(given_a, a), rb = result(given_b, b);
  return Ref{ra.o && rb.o ? Py_BuildValue("(NN)", ra.release(), rb.release()) : nullptr};
}

// ---- functions ------------------------------------------------------------------------------------

// cache(handle, B, H, T, k8, scratch_methods) -> capsule
PyObject* f_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const at::Tensor* k = n == 6 ? plain(a[4]) : nullptr;
    if (!k || !PyTuple_CheckExact(a[5]) || PyTuple_GET_SIZE(a[5]) != 3) return none();
    auto info = std::unique_ptr<CacheInfo>(new CacheInfo{static_cast<unstep_cache*>(PyLong_AsVoidPtr(a[0])), PyLong_AsLongLong(a[1]),
                                                         PyLong_AsLongLong(a[2]), PyLong_AsLongLong(a[3]), k->device(),
                                                         (Py_INCREF(a[5]), a[5])});
    if (PyErr_Occurred()) return none();
    PyObject* cap = PyCapsule_New(info.get(), kMx8Capsule, [](PyObject* o) {
      delete static_cast<CacheInfo*>(PyCapsule_GetPointer(o, kMx8Capsule));
    });
    if (cap) info.release();
    return cap;
  });
}

// tables(f0, C, gh, gw, d_t, d_h, d_w, theta, scaling, factor, trained, fast, slow, amplitude) -> (cos, sin) on the
// current device
PyObject* f_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int32_t v[8];
    double d[6];
    if (n != 14) return none();
    for (int i = 0; i < 7; ++i)
      if (!to_i32(a[i], &v[i])) return none();
    if (!to_i32(a[8], &v[7]) || !to_f64(a[7], &d[0])) return none();
    for (int i = 0; i < 5; ++i)
      if (!to_f64(a[9 + i], &d[1 + i])) return none();
    for (int i = 1; i < 4; ++i)
      if (v[i] < 1 || v[i] > (1 << 23)) return none();
    for (int i = 4; i < 7; ++i)
      if (v[i] < 0 || v[i] > kD) return none();
    if (int64_t(v[1]) * v[2] > (1 << 23)) return none();
    const int64_t shape[2] = {int64_t(v[1]) * v[2] * v[3], (v[4] + v[5] + v[6]) / 2};
    if (shape[0] > (1 << 23)) return none();
    const unstep_rotary r{v[4], v[5], v[6], v[7], d[0], d[1], d[2], d[3], d[4], d[5]};
    const c10::Device dev(c10::kCUDA, c10::hip::current_device());
    at::Tensor c, s;
    if (!two(dev, at::kFloat, at::IntArrayRef(shape, 2), at::kFloat, at::IntArrayRef(shape, 2), &c, &s)) return none();
    Ref res = pair(Py_None, c, Py_None, s);
    if (!res.o) return none();
    void* st = current_stream();
    auto *cp = static_cast<float*>(c.data_ptr()), *sp = static_cast<float*>(s.data_ptr());
    if (!call([&] { return unstep_rotary_tables(v[0], v[1], v[2], v[3], &r, cp, sp, st); })) return nullptr;
    return res.release();
  });
}

// append_rotary(bf16 cache, f0, C, q, k, v, cos, sin, layout, wq, wk, eps, q_rot) -> (q_rot or None,)
PyObject* f_append_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const CacheInfo* c = n == 13 ? cache_of(a[0], kBf16Capsule) : nullptr;
    Chunk k;
    int32_t layout;
    const void *wq, *wk;
    double eps;
    if (!c || !chunk_of(*c, a + 1, true, -1, &k) || !layout_of(a[8], &layout) ||
        !norm_of(*c, k.q != nullptr, a[9], a[10], a[11], &wq, &wk, &eps))
      return none();
    at::Tensor made;
    const at::Tensor* qr = nullptr;
    if (k.q ? !(qr = chunk_out(*c, k.N, a[12], &made)) : a[12] != Py_None) return none();
    Ref q = k.q ? result(a[12], made) : Ref{(Py_INCREF(Py_None), Py_None)};
    Ref r{q.o ? Py_BuildValue("(O)", q.o) : nullptr};
    if (!r.o) return none();
    void *st = current_stream(), *qrp = ptr(qr);
    if (!call([&] {
          return unstep_kv_append_rotary(c->handle, k.f0, k.C, k.qp, k.kp, k.vp, k.ts, k.hs, k.cp, k.sp, layout,
                                         int32_t(2 * k.pairs), wq, wk, eps, qrp, st);
        }))
      return nullptr;
    return r.release();
  });
}

// append_mx8(cache, f0, C, q, k, v, cos, sin, layout, wq, wk, eps, scale, q8, q_scale) -> ((q8, q_scale) or None,)
PyObject* f_append_mx8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const CacheInfo* c = n == 15 ? cache_of(a[0], kMx8Capsule) : nullptr;
    Chunk k;
    int32_t layout;
    const void *wq, *wk;
    double eps, scale;
    if (!c || !chunk_of(*c, a + 1, true, -1, &k) || !layout_of(a[8], &layout) ||
        !norm_of(*c, k.q != nullptr, a[9], a[10], a[11], &wq, &wk, &eps) || !to_f64(a[12], &scale))
      return none();
    Queries q{};
    if (k.q ? !q.get(*c, k.N, a[13], a[14]) : (a[13] != Py_None || a[14] != Py_None)) return none();
    Ref p = k.q ? pair(a[13], q.made8, a[14], q.made_scale) : Ref{(Py_INCREF(Py_None), Py_None)};
    Ref r{p.o ? Py_BuildValue("(O)", p.o) : nullptr};
    if (!r.o) return none();
    void *st = current_stream(), *q8 = ptr(q.q8), *qs = ptr(q.scale);
    if (!call([&] {
          return unstep_kv_append_mx8(c->handle, k.f0, k.C, k.qp, k.kp, k.vp, k.ts, k.hs, k.cp, k.sp, layout,
                                      int32_t(2 * k.pairs), wq, wk, eps, float(scale), q8, qs, st);
        }))
      return nullptr;
    return r.release();
  });
}

// window_attn_mx8(cache, f0, C, W, q8, q_scale, out, lse, workspace, use_split, owner) -> out
PyObject* f_window_attn_mx8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const CacheInfo* c = n == 11 ? cache_of(a[0], kMx8Capsule) : nullptr;
    int32_t f0, C, W;
    if (!c || !to_i32(a[1], &f0) || !to_i32(a[2], &C) || C < 1 || !to_i32(a[3], &W)) return none();
    const int64_t N = int64_t(C) * c->T;
    float* lse;
    void* ws;
    size_t bytes;
    at::Tensor made, hold;
    Queries q{};
    if (captures_scratch(a[8], a[9]) || a[4] == Py_None || a[5] == Py_None || !q.get(*c, N, a[4], a[5]) || !lse_of(*c, N, a[7], &lse) ||
        !workspace_of(*c, f0, C, W, a[8], a[9], a[10], false, &hold, &ws, &bytes))
      return none();
    const at::Tensor* out = chunk_out(*c, N, a[6], &made);
    if (!out) return none();
    Ref r = result(a[6], made);
    if (!r.o) return none();
    void *st = current_stream(), *q8 = ptr(q.q8), *qs = ptr(q.scale), *op = ptr(out);
    if (!call([&] { return unstep_window_attn_mx8(c->handle, f0, C, W, q8, qs, op, lse, ws, bytes, st); })) return nullptr;
    return r.release();
  });
}

// step_mx8(cache, f0, C, q, k, v, cos, sin, W, layout, wq, wk, eps, scale, q8, q_scale, out, lse, workspace, use_split,
// owner) -> out
PyObject* f_step_mx8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const CacheInfo* c = n == 21 ? cache_of(a[0], kMx8Capsule) : nullptr;
    Chunk k;
    int32_t W, layout;
    const void *wq, *wk;
    double eps, scale;
    float* lse;
    void* ws;
    size_t bytes;
    at::Tensor made, hold;
    Queries q{};
    if (!c || captures_scratch(a[18], a[19]) || !chunk_of(*c, a + 1, false, -1, &k) || !to_i32(a[8], &W) || !layout_of(a[9], &layout) ||
        !norm_of(*c, true, a[10], a[11], a[12], &wq, &wk, &eps) || !to_f64(a[13], &scale) || !lse_of(*c, k.N, a[17], &lse) ||
        !workspace_of(*c, k.f0, k.C, W, a[18], a[19], a[20], false, &hold, &ws, &bytes) || !q.get(*c, k.N, a[14], a[15]))
      return none();
    const at::Tensor* out = chunk_out(*c, k.N, a[16], &made);
    if (!out) return none();
    Ref r = result(a[16], made);
    if (!r.o) return none();
    void *st = current_stream(), *q8 = ptr(q.q8), *qs = ptr(q.scale), *op = ptr(out);
    if (!call([&] {
          return unstep_step_mx8(c->handle, k.f0, k.C, W, k.qp, k.kp, k.vp, k.ts, k.hs, k.cp, k.sp, layout,
                                 int32_t(2 * k.pairs), wq, wk, eps, float(scale), q8, qs, op, lse, ws, bytes, st);
        }))
      return nullptr;
    return r.release();
  });
}

// read_mx8(cache, f0, C, k_out, v_out) -> (k, v)
PyObject* f_read_mx8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const CacheInfo* c = n == 5 ? cache_of(a[0], kMx8Capsule) : nullptr;
    int32_t f0, C;
    if (!c || !to_i32(a[1], &f0) || !to_i32(a[2], &C) || C < 1) return none();
    const int64_t N = int64_t(C) * c->T;
    if (int64_t(c->B) * c->H * N > (int64_t(1) << 27)) return none();
    at::Tensor made_k, made_v;
    const at::Tensor *k = &made_k, *v = &made_v;
    const int64_t shape[4] = {c->B, N, c->H, kD};
    if (a[3] == Py_None && a[4] == Py_None) {
      const at::IntArrayRef each(shape, 4);
      if (!two(c->device, at::kBFloat16, each, at::kBFloat16, each, &made_k, &made_v)) return none();
    } else if (!(k = chunk_out(*c, N, a[3], &made_k)) || !(v = chunk_out(*c, N, a[4], &made_v))) {
      return none();
    }
    Ref r = pair(a[3], made_k, a[4], made_v);
    if (!r.o) return none();
    void *st = current_stream(), *kp = ptr(k), *vp = ptr(v);
    if (!call([&] { return unstep_kv_read_mx8(c->handle, f0, C, kp, vp, st); })) return nullptr;
    return r.release();
  });
}

// dequantize(x8, scale, out) -> out
PyObject* f_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const at::Tensor *x = n == 3 ? plain(a[0]) : nullptr, *s = x ? plain(a[1]) : nullptr;
    if (!s || x->scalar_type() != at::kFloat8_e4m3fn || !x->is_contiguous() || x->dim() < 1 || x->size(-1) != kD ||
        x->numel() == 0 || !current(x->device()))
      return none();
    at::DimVector shape(x->sizes().begin(), x->sizes().end());
    shape.back() = kScales;
    if (!is(s, at::kByte, shape, x->device())) return none();
    at::Tensor made;
    const at::Tensor* out = out_of(at::kBFloat16, x->sizes(), x->device(), a[2], &made);
    if (!out) return none();
    Ref r = result(a[2], made);
    if (!r.o) return none();
    const int64_t rows = x->numel() / kD;
    void *st = current_stream(), *xp = ptr(x), *sp = ptr(s), *op = ptr(out);
    if (!call([&] { return unstep_mx8_dequantize(xp, sp, op, rows, st); })) return nullptr;
    return r.release();
  });
}

#define UNSTEP_FN(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {UNSTEP_FN(cache),           UNSTEP_FN(tables),   UNSTEP_FN(append_rotary), UNSTEP_FN(append_mx8),
                         UNSTEP_FN(window_attn_mx8), UNSTEP_FN(step_mx8), UNSTEP_FN(read_mx8),      UNSTEP_FN(dequantize),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls_mx8", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls_mx8() {
  const char* const names[3] = {"workspace", "workspace_bytes", "_step_workspace"};
  for (int i = 0; i < 3; ++i)
    if (!(scratch_names[i] = PyUnicode_InternFromString(names[i]))) return nullptr;
  return PyModule_Create(&module);
}
