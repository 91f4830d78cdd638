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
decltype(&sf_tree_mask) g_tree_mask = nullptr;
decltype(&sf_tree_attention) g_tree_attention = nullptr;
decltype(&sf_tree_commit) g_tree_commit = nullptr;
decltype(&sf_attention_mass) g_attention_mass = nullptr;
decltype(&sf_kv_evict) g_kv_evict = nullptr;

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

int whole(PyObject *o) {
  need(PyLong_CheckExact(o));
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  need(overflow == 0 && v >= -0x7fffffffL && v <= 0x7fffffffL);
  return static_cast<int>(v);
}

// A contiguous tensor of `like`'s shape.
const at::Tensor &same(PyObject *o, at::ScalarType type, const at::Tensor &like) {
  const at::Tensor &t = contiguous(o, type, static_cast<int>(like.dim()));
  need(t.sizes() == like.sizes());
  return t;
}

// The layers' pointers of one tensor [layers][...] (`dim` dimensions without the
// first), each layer contiguous, and the sizes of a layer.  A list of tensors is
// left to the binding.
struct Layers {
  void *at[SF_MAX_LAYERS];
  int count;
  at::IntArrayRef sizes;
};

void layers(PyObject *o, at::ScalarType type, int dim, Layers *out) {
  const at::Tensor &t = tensor(o, type, dim + 1);
  need(t.size(0) <= SF_MAX_LAYERS);
  int64_t inner = 1;
  for (int i = dim; i > 0; --i) {
    need(t.size(i) == 1 || t.stride(i) == inner);
    inner *= t.size(i);
  }
  out->count = static_cast<int>(t.size(0));
  out->sizes = t.sizes().slice(1);
  char *first = static_cast<char *>(t.data_ptr());
  for (int i = 0; i < out->count; ++i) out->at[i] = first + i * t.stride(0) * static_cast<int64_t>(t.element_size());
}

// The stack of free pages, or nothing.
struct Stack {
  int32_t *pages = nullptr, *count = nullptr;
  int capacity = 0;
  Stack(PyObject *p, PyObject *c) {
    need((p == Py_None) == (c == Py_None));
    if (p == Py_None) return;
    const at::Tensor &t = contiguous(p, at::kInt, 1), &n = contiguous(c, at::kInt, 1);
    need(n.size(0) == 1);
    pages = data<int32_t>(t);
    count = data<int32_t>(n);
    capacity = size(t, 0);
  }
};

// (parents, start, mask, positions, workspace)
PyObject *tree_mask(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 5, reinterpret_cast<void *>(g_tree_mask), [&] {
    const at::Tensor &p = contiguous(a[0], at::kInt, 2);
    const int32_t *start = nullptr;
    if (a[1] != Py_None) {
      const at::Tensor &t = contiguous(a[1], at::kInt, 1);
      need(t.size(0) == p.size(0));
      start = data<const int32_t>(t);
    }
    const at::Tensor &mask = same(a[2], at::kLong, p), &pos = same(a[3], at::kInt, p);
    const at::Tensor &ws = contiguous(a[4], at::kByte, 1);
    return g_tree_mask(data<const int32_t>(p), start, size(p, 0), size(p, 1), data<uint64_t>(mask), data<int32_t>(pos),
                       ws.data_ptr(), static_cast<size_t>(ws.numel()), stream());
  });
}

// (q, k_cache, v_cache, block_table, seq_lens, mask, softmax_scale, out, lse, workspace)
PyObject *tree_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 10, reinterpret_cast<void *>(g_tree_attention), [&] {
    const at::Tensor &q = contiguous(a[0], at::kBFloat16, 4);
    const at::Tensor &kc = contiguous(a[1], at::kBFloat16, 4), &vc = same(a[2], at::kBFloat16, kc);
    need(kc.size(3) == q.size(3));
    const at::Tensor &bt = contiguous(a[3], at::kInt, 2), &sl = contiguous(a[4], at::kInt, 1);
    const int B = size(q, 0);
    need(bt.size(0) == B && sl.size(0) == B && THPVariable_Check(a[5]));
    const int mask_dim = THPVariable_Unpack(a[5]).dim() == 1 ? 1 : 2;
    const at::Tensor &mask = tensor(a[5], at::kLong, mask_dim);
    need(mask.size(mask_dim - 1) == q.size(1));
    long long mask_stride = 0;
    if (mask_dim == 2) {
      need(mask.size(0) == B);
      mask_stride = row_stride(mask);
    } else {
      need(mask.is_contiguous());
    }
    const at::Tensor &out = same(a[7], at::kBFloat16, q);
    float *lse = nullptr;
    if (a[8] != Py_None) {
      const at::Tensor &l = contiguous(a[8], at::kFloat, 3);
      need(l.size(0) == B && l.size(1) == q.size(1) && l.size(2) == q.size(2));
      lse = data<float>(l);
    }
    const at::Tensor &ws = contiguous(a[9], at::kByte, 1);
    return g_tree_attention(q.data_ptr(), kc.data_ptr(), vc.data_ptr(), data<const int32_t>(bt), data<const int32_t>(sl),
                            data<const uint64_t>(mask), mask_stride, B, size(q, 1), size(q, 2), size(kc, 1), size(q, 3),
                            size(kc, 2), size(kc, 0), size(bt, 1), number(a[6]), out.data_ptr(), lse, ws.data_ptr(),
                            static_cast<size_t>(ws.numel()), stream());
  });
}

// (tokens, sampled, parents, k_caches, v_caches, block_table, seq_lens, num_accepted,
//  out_tokens, path, row_weights, n_q_next, free_pages, free_count, workspace)
PyObject *tree_commit(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 15, reinterpret_cast<void *>(g_tree_commit), [&] {
    const at::Tensor &tok = contiguous(a[0], at::kInt, 2), &smp = same(a[1], at::kInt, tok), &par = same(a[2], at::kInt, tok);
    Layers k, v;
    layers(a[3], at::kBFloat16, 4, &k);
    layers(a[4], at::kBFloat16, 4, &v);
    need(k.count > 0 && k.count == v.count && k.sizes == v.sizes);
    for (const int64_t x : k.sizes) need(x <= 0x7fffffff);
    const at::Tensor &bt = contiguous(a[5], at::kInt, 2), &sl = contiguous(a[6], at::kInt, 1);
    const at::Tensor &acc = contiguous(a[7], at::kInt, 1);
    const int B = size(tok, 0);
    need(bt.size(0) == B && sl.size(0) == B && acc.size(0) == B);
    const at::Tensor &out = same(a[8], at::kInt, tok), &path = same(a[9], at::kInt, tok), &w = same(a[10], at::kFloat, tok);
    const int next = a[11] == Py_None ? size(tok, 1) : whole(a[11]);
    const Stack stack(a[12], a[13]);
    const at::Tensor &ws = contiguous(a[14], at::kByte, 1);
    return g_tree_commit(data<const int32_t>(tok), data<const int32_t>(smp), data<const int32_t>(par), k.at, v.at, k.count,
                         data<int32_t>(bt), data<int32_t>(sl), B, size(tok, 1), static_cast<int>(k.sizes[1]),
                         static_cast<int>(k.sizes[3]), static_cast<int>(k.sizes[2]), static_cast<int>(k.sizes[0]),
                         size(bt, 1), data<int32_t>(acc), data<int32_t>(out), data<int32_t>(path), data<float>(w), next,
                         stack.pages, stack.count, stack.capacity, ws.data_ptr(), static_cast<size_t>(ws.numel()),
                         stream());
  });
}

// (q, lse, k_cache, block_table, seq_lens, mass, row_weights, softmax_scale, out, workspace)
PyObject *attention_mass(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 10, reinterpret_cast<void *>(g_attention_mass), [&] {
    const at::Tensor &q = contiguous(a[0], at::kBFloat16, 4), &lse = contiguous(a[1], at::kFloat, 3);
    const at::Tensor &kc = contiguous(a[2], at::kBFloat16, 4);
    const at::Tensor &bt = contiguous(a[3], at::kInt, 2), &sl = contiguous(a[4], at::kInt, 1);
    const at::Tensor &out = contiguous(a[8], at::kFloat, 3);
    const int B = size(q, 0);
    need(lse.size(0) == B && lse.size(1) == q.size(1) && lse.size(2) == q.size(2) && kc.size(3) == q.size(3));
    need(bt.size(0) == B && sl.size(0) == B && out.size(0) == B && out.size(1) == kc.size(1));
    const float *mass = a[5] == Py_None ? nullptr : data<const float>(same(a[5], at::kFloat, out));
    const float *weights = nullptr;
    if (a[6] != Py_None) {
      const at::Tensor &w = contiguous(a[6], at::kFloat, 2);
      need(w.size(0) == B && w.size(1) == q.size(1));
      weights = data<const float>(w);
    }
    const at::Tensor &ws = contiguous(a[9], at::kByte, 1);
    return g_attention_mass(q.data_ptr(), data<const float>(lse), kc.data_ptr(), data<const int32_t>(bt),
                            data<const int32_t>(sl), mass, weights, B, size(q, 1), size(q, 2), size(kc, 1), size(q, 3),
                            size(kc, 2), size(kc, 0), size(bt, 1), size(out, 2), number(a[7]), data<float>(out),
                            ws.data_ptr(), static_cast<size_t>(ws.numel()), stream());
  });
}

// (mass, k_caches, v_caches, block_table, seq_lens, budget, first, recent, n_q, mass_out,
//  seq_lens_out, kept, free_pages, free_count, workspace)
PyObject *kv_evict(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 15, reinterpret_cast<void *>(g_kv_evict), [&] {
    Layers mass, k, v, out, kept;
    layers(a[0], at::kFloat, 3, &mass);
    layers(a[1], at::kBFloat16, 4, &k);
    layers(a[2], at::kBFloat16, 4, &v);
    layers(a[9], at::kFloat, 3, &out);
    need(k.count > 0 && k.count == v.count && k.count == mass.count && k.count == out.count);
    need(k.sizes == v.sizes && mass.sizes == out.sizes);
    for (const int64_t x : k.sizes) need(x <= 0x7fffffff);
    const at::Tensor &bt = contiguous(a[3], at::kInt, 2), &sl = contiguous(a[4], at::kInt, 1);
    const at::Tensor &lo = contiguous(a[10], at::kInt, 1);
    const int B = size(bt, 0), budget = whole(a[5]);
    need(sl.size(0) == B && lo.size(0) == B && mass.sizes[0] == B && mass.sizes[1] == k.sizes[1]);
    need(mass.sizes[2] <= 0x7fffffff);
    int32_t *kept_at[SF_MAX_LAYERS];
    if (a[11] != Py_None) {
      layers(a[11], at::kInt, 3, &kept);
      need(kept.count == k.count && kept.sizes[0] == B && kept.sizes[1] == k.sizes[1] && kept.sizes[2] == budget);
      for (int i = 0; i < kept.count; ++i) kept_at[i] = static_cast<int32_t *>(kept.at[i]);
    }
    const float *mass_at[SF_MAX_LAYERS];
    float *out_at[SF_MAX_LAYERS];
    for (int i = 0; i < k.count; ++i) {
      mass_at[i] = static_cast<const float *>(mass.at[i]);
      out_at[i] = static_cast<float *>(out.at[i]);
    }
    const Stack stack(a[12], a[13]);
    const at::Tensor &ws = contiguous(a[14], at::kByte, 1);
    return g_kv_evict(mass_at, k.at, v.at, k.count, data<int32_t>(bt), data<const int32_t>(sl), B,
                      static_cast<int>(k.sizes[1]), static_cast<int>(k.sizes[3]), static_cast<int>(k.sizes[2]),
                      static_cast<int>(k.sizes[0]), size(bt, 1), static_cast<int>(mass.sizes[2]), budget, whole(a[6]),
                      whole(a[7]), whole(a[8]), out_at, data<int32_t>(lo), a[11] == Py_None ? nullptr : kept_at,
                      stack.pages, stack.count, stack.capacity, ws.data_ptr(), static_cast<size_t>(ws.numel()), stream());
  });
}

// Addresses of the entry points in the loaded library.
PyObject *set_entries(PyObject *, PyObject *const *a, Py_ssize_t n) {
  void *p[8] = {};
  if (n != 8) {
    PyErr_SetString(PyExc_TypeError, "eight addresses expected");
    return nullptr;
  }
  for (int i = 0; i < 8; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_add_rms_norm = reinterpret_cast<decltype(g_add_rms_norm)>(p[0]);
  g_kv_append = reinterpret_cast<decltype(g_kv_append)>(p[1]);
  g_shared_prefix = reinterpret_cast<decltype(g_shared_prefix)>(p[2]);
  g_tree_mask = reinterpret_cast<decltype(g_tree_mask)>(p[3]);
  g_tree_attention = reinterpret_cast<decltype(g_tree_attention)>(p[4]);
  g_tree_commit = reinterpret_cast<decltype(g_tree_commit)>(p[5]);
  g_attention_mass = reinterpret_cast<decltype(g_attention_mass)>(p[6]);
  g_kv_evict = reinterpret_cast<decltype(g_kv_evict)>(p[7]);
  Py_RETURN_NONE;
}

#define SF_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SF_METHOD(add_rms_norm), SF_METHOD(kv_append), SF_METHOD(shared_prefix_attention),
                         SF_METHOD(tree_mask), SF_METHOD(tree_attention), SF_METHOD(tree_commit),
                         SF_METHOD(attention_mass), SF_METHOD(kv_evict), SF_METHOD(set_entries), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layer_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layer_calls() { return PyModule_Create(&module); }
