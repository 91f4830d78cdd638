// layer_calls.cpp -- the calls of the decoder-layer operators from Python, for
// arguments that need no allocation and no error message.
//
// A small call's time is host time: the checks of a dozen tensors through their
// Python attributes and the marshalling of thirty arguments took 3.4 us of 7.4
// (sf_add_rms_norm, 5 rows) and 7.6 of 12.4 (sf_kv_append, 5 rows), the launch about
// 2.  Here the tensors are looked at directly.  Each function checks what the
// binding (specflash_verify.py) checks and calls the C entry point; where anything is
// missing or not as it should be it returns None, and the binding goes through the
// arguments itself, allocates what was not given, or raises.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "specflash_verify.h"

namespace {

decltype(&sf_add_rms_norm) g_add_rms_norm = nullptr;
decltype(&sf_kv_append) g_kv_append = nullptr;
decltype(&sf_shared_prefix_attention) g_shared_prefix = nullptr;

// Thrown for arguments that the binding has to look at.
struct Unusual {};

const at::Tensor &tensor(PyObject *o, at::ScalarType type, int dim) {
  if (!THPVariable_Check(o)) throw Unusual();
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != type || t.dim() != dim || t.layout() != at::kStrided) throw Unusual();
  return t;
}

const at::Tensor &contiguous(PyObject *o, at::ScalarType type, int dim) {
  const at::Tensor &t = tensor(o, type, dim);
  if (!t.is_contiguous()) throw Unusual();
  return t;
}

void need(bool ok) {
  if (!ok) throw Unusual();
}

template <typename T>
T *data(const at::Tensor &t) {
  return static_cast<T *>(t.data_ptr());
}

int size(const at::Tensor &t, int i) {
  const int64_t n = t.size(i);
  need(n <= 0x7fffffff);
  return static_cast<int>(n);
}

// Elements between the neighbours along dimension i; the last dimension's are
// next to each other.
long long stride(const at::Tensor &t, int i) {
  const int last = static_cast<int>(t.dim()) - 1;
  need(t.size(last) == 1 || t.stride(last) == 1);
  return t.stride(i);
}

// Elements between the rows of a tensor [T][d].  A contiguous one's are d apart, also
// where it has a single row whose stride says something else.
long long row_stride(const at::Tensor &t) { return t.is_contiguous() ? t.size(1) : stride(t, 0); }

at::ScalarType rows_type(PyObject *o) {
  if (!THPVariable_Check(o)) throw Unusual();
  const at::ScalarType t = THPVariable_Unpack(o).scalar_type();
  need(t == at::kBFloat16 || t == at::kFloat);
  return t;
}

float number(PyObject *o) {
  need(PyFloat_CheckExact(o));
  return static_cast<float>(PyFloat_AS_DOUBLE(o));
}

cudaStream_t stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// Runs `call` with `n` arguments; its status as an int, or None.
template <typename F>
PyObject *guarded(Py_ssize_t given, Py_ssize_t n, void *entry, F call) {
  if (given != n) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", given, n);
    return nullptr;
  }
  try {
    need(entry != nullptr);
    return PyLong_FromLong(call());
  } catch (...) {  // an Unusual one, or what torch throws over a tensor that it cannot look into
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (x, weight, residual, eps, group, out, residual_out, scales)
PyObject *add_rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 8, reinterpret_cast<void *>(g_add_rms_norm), [&] {
    const at::ScalarType type = rows_type(a[0]), wtype = rows_type(a[1]);
    const at::Tensor &x = tensor(a[0], type, 2), &w = contiguous(a[1], wtype, 1);
    const int T = size(x, 0), d = size(x, 1);
    need(w.size(0) == d && PyLong_CheckExact(a[4]));
    const long group = PyLong_AsLong(a[4]);
    need(group == 0 || group == 128);
    void *r = nullptr, *ro = nullptr;
    long long r_row = 0, ro_row = 0;
    if (a[2] != Py_None) {
      const at::Tensor &t = tensor(a[2], type, 2), &u = tensor(a[6], type, 2);
      need(t.sizes() == x.sizes() && u.sizes() == x.sizes());
      r = t.data_ptr();
      ro = u.data_ptr();
      r_row = row_stride(t);
      ro_row = row_stride(u);
    } else {
      need(a[6] == Py_None);
    }
    need(THPVariable_Check(a[5]));
    const bool e4m3 = THPVariable_Unpack(a[5]).scalar_type() == at::kFloat8_e4m3fn;
    const at::Tensor &out = tensor(a[5], e4m3 ? at::kFloat8_e4m3fn : at::kBFloat16, 2);
    need(out.sizes() == x.sizes());
    float *scales = nullptr;
    if (e4m3) {
      const at::Tensor &s = contiguous(a[7], at::kFloat, 2);
      need(s.size(0) == T && s.size(1) == (group ? (d + group - 1) / group : 1));
      scales = data<float>(s);
    } else {
      need(a[7] == Py_None && group == 0);
    }
    return g_add_rms_norm(x.data_ptr(), r, w.data_ptr(), type == at::kFloat ? SF_F32 : SF_BF16,
                          wtype == at::kFloat ? SF_F32 : SF_BF16, T, d, row_stride(x), r_row, number(a[3]), ro, ro_row,
                          out.data_ptr(), e4m3 ? SF_E4M3 : SF_BF16, row_stride(out), static_cast<int>(group), scales,
                          stream());
  });
}

// (q, k, v, positions, inv_freq, k_cache, v_cache, block_table, seq_lens, axis,
//  row_starts, interleaved, amplitude, q_out, workspace)
PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 15, reinterpret_cast<void *>(g_kv_append), [&] {
    const at::ScalarType type = rows_type(a[1]);
    const at::Tensor &k = tensor(a[1], type, 3), &v = tensor(a[2], type, 3);
    const int T = size(k, 0), H_kv = size(k, 1), d = size(k, 2);
    need(v.sizes() == k.sizes());
    const void *q = nullptr;
    void *q_out = nullptr;
    long long q_row = 0, q_head = 0;
    int H_q = 0;
    if (a[0] != Py_None) {
      const at::Tensor &t = tensor(a[0], type, 3), &o = contiguous(a[13], at::kBFloat16, 3);
      need(t.size(0) == T && t.size(2) == d && o.sizes() == t.sizes());
      H_q = size(t, 1);
      q = t.data_ptr();
      q_out = o.data_ptr();
      q_row = stride(t, 0);
      q_head = stride(t, 1);
    } else {
      need(a[13] == Py_None);
    }
    const at::Tensor &kc = contiguous(a[5], at::kBFloat16, 4), &vc = contiguous(a[6], at::kBFloat16, 4);
    need(vc.sizes() == kc.sizes() && kc.size(1) == H_kv && kc.size(3) == d);
    const at::Tensor &bt = contiguous(a[7], at::kInt, 2), &sl = contiguous(a[8], at::kInt, 1);
    const int B = size(bt, 0);
    need(sl.size(0) == B);
    int axes = 0, pairs = 0;
    const int32_t *pos = nullptr, *axis = nullptr, *starts = nullptr;
    const double *freq = nullptr;
    if (a[4] != Py_None) {
      const at::Tensor &f = contiguous(a[4], at::kDouble, 1), &p = contiguous(a[3], at::kInt, 2);
      need(p.size(1) == T);
      axes = size(p, 0);
      pairs = size(f, 0);
      need(pairs <= 0x3fffffff);
      pos = data<const int32_t>(p);
      freq = data<const double>(f);
      if (a[9] != Py_None) {
        const at::Tensor &x = contiguous(a[9], at::kInt, 1);
        need(x.size(0) == pairs);
        axis = data<const int32_t>(x);
      }
    } else {
      need(a[3] == Py_None && a[9] == Py_None);
    }
    if (a[10] != Py_None) {
      const at::Tensor &s = contiguous(a[10], at::kInt, 1);
      need(s.size(0) == B + 1);
      starts = data<const int32_t>(s);
    }
    need(PyBool_Check(a[11]));
    const at::Tensor &ws = contiguous(a[14], at::kByte, 1);
    return g_kv_append(q, k.data_ptr(), v.data_ptr(), type == at::kFloat ? SF_F32 : SF_BF16, q_row, q_head, stride(k, 0),
                       stride(k, 1), stride(v, 0), stride(v, 1), pos, axes, freq, axis, 2 * pairs, a[11] == Py_True,
                       number(a[12]), data<const int32_t>(bt), data<const int32_t>(sl), starts, T, B, H_q, H_kv, d,
                       size(kc, 2), size(kc, 0), size(bt, 1), q_out, kc.data_ptr(), vc.data_ptr(), ws.data_ptr(),
                       static_cast<size_t>(ws.numel()), stream());
  });
}

// (q, k_cache, v_cache, prefix_table, prefix_lens, group_starts, block_table,
//  seq_lens, softmax_scale, out, lse, workspace)
PyObject *shared_prefix_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 12, reinterpret_cast<void *>(g_shared_prefix), [&] {
    const at::Tensor &q = contiguous(a[0], at::kBFloat16, 4);
    const at::Tensor &kc = contiguous(a[1], at::kBFloat16, 4), &vc = contiguous(a[2], at::kBFloat16, 4);
    need(vc.sizes() == kc.sizes() && kc.size(3) == q.size(3));
    const at::Tensor &pt = contiguous(a[3], at::kInt, 2), &pl = contiguous(a[4], at::kInt, 1);
    const at::Tensor &gs = contiguous(a[5], at::kInt, 1), &bt = contiguous(a[6], at::kInt, 2);
    const at::Tensor &sl = contiguous(a[7], at::kInt, 1);
    const int B = size(q, 0), groups = size(pt, 0);
    need(bt.size(0) == B && sl.size(0) == B && pl.size(0) == groups && gs.size(0) == groups + 1);
    const at::Tensor &out = contiguous(a[9], at::kBFloat16, 4);
    need(out.sizes() == q.sizes());
    float *lse = nullptr;
    if (a[10] != Py_None) {
      const at::Tensor &l = contiguous(a[10], at::kFloat, 3);
      need(l.size(0) == B && l.size(1) == q.size(1) && l.size(2) == q.size(2));
      lse = data<float>(l);
    }
    const at::Tensor &ws = contiguous(a[11], at::kByte, 1);
    return g_shared_prefix(q.data_ptr(), kc.data_ptr(), vc.data_ptr(), data<const int32_t>(pt), data<const int32_t>(pl),
                           data<const int32_t>(gs), data<const int32_t>(bt), data<const int32_t>(sl), B, size(q, 1),
                           size(q, 2), size(kc, 1), size(q, 3), size(kc, 2), size(kc, 0), groups, size(pt, 1),
                           size(bt, 1), number(a[8]), out.data_ptr(), lse, ws.data_ptr(),
                           static_cast<size_t>(ws.numel()), stream());
  });
}

// Addresses of the three entry points in the loaded library.
PyObject *set_entries(PyObject *, PyObject *const *a, Py_ssize_t n) {
  void *p[3] = {};
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "three addresses expected");
    return nullptr;
  }
  for (int i = 0; i < 3; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_add_rms_norm = reinterpret_cast<decltype(g_add_rms_norm)>(p[0]);
  g_kv_append = reinterpret_cast<decltype(g_kv_append)>(p[1]);
  g_shared_prefix = reinterpret_cast<decltype(g_shared_prefix)>(p[2]);
  Py_RETURN_NONE;
}

#define SF_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SF_METHOD(add_rms_norm), SF_METHOD(kv_append), SF_METHOD(shared_prefix_attention),
                         SF_METHOD(set_entries), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layer_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layer_calls() { return PyModule_Create(&module); }
