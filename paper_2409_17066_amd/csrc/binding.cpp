// The convenience calls of the Python package over torch tensors, marshalled in C++: a decode-sized kernel takes a few
// microseconds, and checking the tensors, asking for the stream, allocating the result and converting the arguments through
// ctypes took longer than that (256 x 384, one row, calls back to back: 8.9 us against 4.4 us here).  Every function returns
// None when the arguments are not the plain ones it takes -- the Python code then does the call, with its own checks and
// errors --, the status code when the library refused, and the result otherwise.  The calls around a paged cache and the norms have
// no second way: what they do not take is a ValueError.
#include <Python.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <stdexcept>
#include <string>

#include "../../include/vq.h"
#include "vq_lend.h"

namespace {

decltype(&vq_gemv) p_gemv;
decltype(&vq_gemv_with_workspace) p_gemv_ws;
decltype(&vq_lend_gemv_bytes) p_lend_gemv_bytes;
decltype(&vq_gemv_multi) p_gemv_multi;
decltype(&vq_gemm) p_gemm, p_gemm_default;
decltype(&vq_gemm_workspace_bytes) p_gemm_workspace_bytes, p_gemm_default_workspace_bytes, p_lend_gemm_least_bytes;
decltype(&vq_dequant) p_dequant;
decltype(&vq_lend_assign) p_lend_assign;
decltype(&vq_kv_append) p_kv_append;
decltype(&vq_attention) p_attention;
decltype(&vq_attention_workspace_bytes) p_attention_workspace_bytes;
decltype(&vq_residual_norm) p_residual_norm;
decltype(&vq_attention_shared) p_attention_shared;
decltype(&vq_attention_shared_workspace_bytes) p_attention_shared_workspace_bytes;
decltype(&vq_embed) p_embed;
decltype(&vq_sample) p_sample;

PyObject *s_desc, *s_places;

// The layer's descriptor: the memory of the ctypes structure in its attribute `desc`.
struct Desc {
  Py_buffer view;
  bool held = false;
  const vq_layer_desc *get(PyObject *layer) {
    PyObject *d = PyObject_GetAttr(layer, s_desc);
    if (!d) { PyErr_Clear(); return nullptr; }
    held = PyObject_GetBuffer(d, &view, PyBUF_SIMPLE) == 0;
    Py_DECREF(d);
    if (!held) { PyErr_Clear(); return nullptr; }
    return view.len == (Py_ssize_t)sizeof(vq_layer_desc) ? static_cast<const vq_layer_desc *>(view.buf) : nullptr;
  }
  ~Desc() { if (held) PyBuffer_Release(&view); }
};

// A device tensor [rows][columns] of halfs with adjacent columns, else nullptr.
const at::Tensor *half_matrix(PyObject *o) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  return t.is_cuda() && t.scalar_type() == at::kHalf && t.dim() == 2 && t.stride(1) == 1 ? &t : nullptr;
}

at::TensorBase empty(at::IntArrayRef size, at::ScalarType type) {
  return at::detail::empty_cuda(size, type, c10::Device(c10::kCUDA, c10::hip::current_device()), std::nullopt);
}

void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

template <typename Call>
int released(Call call) {                       // the library call, without the interpreter's lock as ctypes makes it
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc;
}

PyObject *tensor_or_status(int rc, at::TensorBase &&fresh, PyObject *given) {
  if (rc != VQ_OK) return PyLong_FromLong(rc);
  if (given != Py_None) { Py_INCREF(given); return given; }
  return THPVariable_Wrap(std::move(fresh));
}

// Workspace for one call, from torch's allocator, or nullptr: there is a route without.  On a full card the allocator would first give
// all its unused memory back and wait for the GPU, in every call: beyond the size of small results it is asked only for what it has
// unused or the device has free.
void *borrow(at::TensorBase &scratch, size_t bytes) {
  try {
    if (bytes > (1u << 20)) {
      using c10::CachingAllocator::StatType;
      const auto stats = c10::hip::HIPCachingAllocator::getDeviceStats(c10::hip::current_device());
      const auto sum = static_cast<size_t>(StatType::AGGREGATE);
      const size_t unused = (size_t)(stats.reserved_bytes[sum].current - stats.allocated_bytes[sum].current);
      size_t free = 0, total = 0;
      if (unused < bytes && hipMemGetInfo(&free, &total) == hipSuccess && free + unused < bytes) return nullptr;
    }
    scratch = empty({(int64_t)bytes}, at::kByte);
    return scratch.data_ptr();
  } catch (const c10::Error &) {
    return nullptr;
  }
}

#define VQ_TRY try {
#define VQ_CATCH                                            \
  } catch (const std::invalid_argument &e) {                \
    PyErr_SetString(PyExc_ValueError, e.what());            \
    return nullptr;                                         \
  } catch (const std::exception &e) {                       \
    PyErr_SetString(PyExc_RuntimeError, e.what());          \
    return nullptr;                                         \
  }

// Whether gemv() without a workspace may borrow one (vq_lend.h says how much): the layers that never do are spared the question.
bool may_borrow(const vq_layer_desc &d) { return (!d.group_vectors && (d.v != 6 || d.k <= 2048 || d.col_perm)) || (d.v == 6 && (d.in_features & 1)); }

// gemv(layer, x, out or None, workspace or None)
PyObject *gemv(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  Desc desc;
  const vq_layer_desc *d;
  const at::Tensor *x;
  if (n != 4 || !(x = half_matrix(args[1])) || !(d = desc.get(args[0]))) Py_RETURN_NONE;
  const bool has_ws = args[3] != Py_None;
  if (has_ws && !THPVariable_Check(args[3])) Py_RETURN_NONE;
  at::TensorBase fresh;
  const at::TensorBase *y = &fresh;
  if (args[2] != Py_None) {
    if (!THPVariable_Check(args[2])) Py_RETURN_NONE;
    y = &THPVariable_Unpack(args[2]);
    if (y->dim() != 2) Py_RETURN_NONE;
  } else {
    fresh = empty({x->size(0), d->out_features}, at::kHalf);
  }
  const void *xp = x->data_ptr();
  void *yp = y->data_ptr(), *s = stream();
  const int64_t ldx = x->stride(0), ldy = y->stride(0);
  const int32_t batch = (int32_t)x->size(0);
  int rc;
  if (has_ws) {
    const at::Tensor &ws = THPVariable_Unpack(args[3]);
    void *wp = ws.data_ptr();
    const size_t bytes = (size_t)ws.numel();
    rc = released([&] { return p_gemv_ws(d, xp, ldx, batch, yp, ldy, wp, bytes, s); });
  } else if (const size_t bytes = may_borrow(*d) ? p_lend_gemv_bytes(d, batch) : 0) {
    at::TensorBase scratch;
    void *wp = borrow(scratch, bytes);
    rc = released([&] { return p_gemv_ws(d, xp, ldx, batch, yp, ldy, wp, wp ? bytes : 0, s); });
  } else {
    rc = released([&] { return p_gemv(d, xp, ldx, batch, yp, ldy, s); });
  }
  return tensor_or_status(rc, std::move(fresh), args[2]);
  VQ_CATCH
}

// gemv_multi(list of layers, x)
PyObject *gemv_multi(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  constexpr Py_ssize_t MOST = 8;
  const at::Tensor *x;
  if (n != 2 || !PyList_CheckExact(args[0]) || !(x = half_matrix(args[1]))) Py_RETURN_NONE;
  const Py_ssize_t layers = PyList_GET_SIZE(args[0]);
  if (layers < 1 || layers > MOST) Py_RETURN_NONE;
  Desc desc[MOST];
  const vq_layer_desc *d[MOST];
  at::TensorBase y[MOST];
  void *yp[MOST];
  int64_t ldy[MOST];
  for (Py_ssize_t i = 0; i < layers; ++i)
    if (!(d[i] = desc[i].get(PyList_GET_ITEM(args[0], i)))) Py_RETURN_NONE;
  for (Py_ssize_t i = 0; i < layers; ++i) {
    y[i] = empty({x->size(0), d[i]->out_features}, at::kHalf);
    yp[i] = y[i].data_ptr();
    ldy[i] = y[i].stride(0);
  }
  const void *xp = x->data_ptr();
  void *s = stream();
  const int rc = released([&] { return p_gemv_multi(d, (int32_t)layers, xp, x->stride(0), (int32_t)x->size(0), yp, ldy, s); });
  if (rc != VQ_OK) return PyLong_FromLong(rc);
  PyObject *out = PyList_New(layers);
  for (Py_ssize_t i = 0; out && i < layers; ++i) PyList_SET_ITEM(out, i, THPVariable_Wrap(std::move(y[i])));
  return out;
  VQ_CATCH
}

// gemm(layer, X, out or None, workspace or None)
PyObject *gemm(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  Desc desc;
  const vq_layer_desc *d;
  const at::Tensor *x;
  if (n != 4 || !(x = half_matrix(args[1])) || !(d = desc.get(args[0]))) Py_RETURN_NONE;
  void *wp = nullptr;
  size_t bytes = 0;
  at::TensorBase scratch;
  auto call = p_gemm;
  const int32_t tokens = (int32_t)x->size(0);
  if (args[3] != Py_None) {
    if (!THPVariable_Check(args[3])) Py_RETURN_NONE;
    const at::Tensor &ws = THPVariable_Unpack(args[3]);
    wp = ws.data_ptr();
    bytes = (size_t)ws.numel() * ws.element_size();
  } else if (tokens > 8) {
    call = p_gemm_default;
    if ((bytes = p_gemm_default_workspace_bytes(d, tokens)) != 0 && !(wp = borrow(scratch, bytes))) {
      const size_t least = p_lend_gemm_least_bytes(d, tokens);
      bytes = least < bytes && (wp = borrow(scratch, least)) ? least : 0;
    }
  }
  if (p_gemm_workspace_bytes(d, tokens) > bytes) Py_RETURN_NONE;
  at::TensorBase fresh;
  const at::TensorBase *y = &fresh;
  if (args[2] != Py_None) {
    if (!THPVariable_Check(args[2])) Py_RETURN_NONE;
    y = &THPVariable_Unpack(args[2]);
    if (y->dim() != 2) Py_RETURN_NONE;
  } else {
    fresh = empty({x->size(0), d->out_features}, at::kHalf);
  }
  const void *xp = x->data_ptr();
  void *yp = y->data_ptr(), *s = stream();
  const int64_t ldx = x->stride(0), ldy = y->stride(0);
  const int rc = released([&] { return call(d, xp, ldx, tokens, yp, ldy, wp, bytes, s); });
  return tensor_or_status(rc, std::move(fresh), args[2]);
  VQ_CATCH
}

// dequant(layer): all of W written, rows in_features apart
PyObject *dequant(PyObject *, PyObject *layer) {
  VQ_TRY
  Desc desc;
  const vq_layer_desc *d = desc.get(layer);
  if (!d) Py_RETURN_NONE;
  PyObject *places = PyObject_GetAttr(layer, s_places);
  if (!places) { PyErr_Clear(); Py_RETURN_NONE; }
  const bool all = places == Py_True;
  Py_DECREF(places);
  if (!all) Py_RETURN_NONE;
  at::TensorBase W = empty({d->out_features, d->in_features}, at::kHalf);
  void *wp = W.data_ptr(), *s = stream();
  const int rc = released([&] { return p_dequant(d, wp, d->in_features, s); });
  return tensor_or_status(rc, std::move(W), Py_None);
  VQ_CATCH
}

// assign(W, codebook, base or None, orientation): all columns of W
PyObject *assign(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  const at::Tensor *W, *C, *B = nullptr;
  if (n != 4 || !(W = half_matrix(args[0])) || !(C = half_matrix(args[1])) || !C->is_contiguous() || !PyLong_CheckExact(args[3])) Py_RETURN_NONE;
  if (args[2] != Py_None && (!(B = half_matrix(args[2])) || B->sizes() != W->sizes() || B->strides() != W->strides())) Py_RETURN_NONE;
  const bool down = PyLong_AsLong(args[3]) != 0;
  const int64_t rows = W->size(0), cols = W->size(1), k = C->size(0), v = C->size(1);
  if (rows < 1 || cols < 1 || v < 1 || k < 1) Py_RETURN_NONE;
  int bits = 1;
  while ((int64_t(1) << bits) < k) ++bits;
  const int64_t streams = down ? (rows + v - 1) / v : rows, per_stream = down ? cols : (cols + v - 1) / v;
  const int64_t stride = (per_stream * bits + 127) / 128 * 16;
  at::TensorBase idx = empty({streams, stride}, at::kByte);
  const void *wp = W->data_ptr(), *bp = B ? B->data_ptr() : nullptr, *cp = C->data_ptr();
  void *ip = idx.data_ptr(), *s = stream();
  const int64_t ld = W->stride(0);
  const int rc = released([&] { return p_lend_assign(wp, bp, ld, (int32_t)rows, (int32_t)cols, cp, (int32_t)v, (int32_t)k, ip, stride, down, s); });
  if (rc != VQ_OK) return PyLong_FromLong(rc);
  return THPVariable_Wrap(std::move(idx));
  VQ_CATCH
}

// ---- paged cache, attention, norms: what the tensors have to be is checked here, the sizes' limits by the library ----
[[noreturn]] void refuse(const char *name, const char *what) { throw std::invalid_argument(std::string(name) + ": " + what); }

const at::Tensor *tensor(PyObject *o, const char *name, at::ScalarType type, int64_t dim, bool optional = false) {
  if (optional && o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(name, "a tensor is expected");
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.get_device() != c10::hip::current_device()) refuse(name, "a tensor on the current GPU is expected");
  if (t.scalar_type() != type) refuse(name, "wrong type of elements");
  if (t.dim() != dim) refuse(name, "wrong number of dimensions");
  return &t;
}
// Dimension d's elements are `stride` apart (dimensions of one element may say anything).
bool apart(const at::Tensor &t, int64_t d, int64_t stride) { return t.size(d) <= 1 || t.stride(d) == stride; }
int32_t narrow(int64_t n, const char *name) {
  if (n < INT32_MIN || n > INT32_MAX) refuse(name, "out of range");
  return (int32_t)n;
}
int32_t whole(PyObject *o, const char *name) {
  const long long n = PyLong_AsLongLong(o);
  if (n == -1 && PyErr_Occurred()) { PyErr_Clear(); refuse(name, "an integer is expected"); }
  return narrow(n, name);
}
float number(PyObject *o, const char *name) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) { PyErr_Clear(); refuse(name, "a number is expected"); }
  return (float)x;
}
bool truth(PyObject *o, const char *name) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) { PyErr_Clear(); refuse(name, "a truth value is expected"); }
  return x != 0;
}
int64_t leading(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.numel(); }       // (one row: its stride may say anything)

// [tokens][heads][head_dim] with adjacent heads
const at::Tensor *tokens(PyObject *o, const char *name, bool optional = false) {
  const at::Tensor *t = tensor(o, name, at::kHalf, 3, optional);
  if (t && (!apart(*t, 2, 1) || !apart(*t, 1, t->size(2)))) refuse(name, "the heads of a token have to lie next to each other");
  return t;
}

// pages, table, lengths, scales and starts: args[0 .. 6], most new tokens and longest length: args[7], args[8] (None: no bound is known)
void cache_of(PyObject *const *args, int64_t n_tokens, vq_kv_desc &d) {
  if (!THPVariable_Check(args[0])) refuse("k_pages", "a tensor is expected");
  const at::ScalarType type = THPVariable_Unpack(args[0]).scalar_type();
  if (type != at::kHalf && type != at::kFloat8_e4m3fn) refuse("k_pages", "float16 or float8_e4m3fn is expected");
  const at::Tensor &k = *tensor(args[0], "k_pages", type, 4), &v = *tensor(args[1], "v_pages", type, 4);
  const int64_t heads = k.size(1), size = k.size(2), dim = k.size(3);
  if (v.size(0) != k.size(0) || v.size(1) != heads || v.size(2) != dim || v.size(3) != size) refuse("v_pages", "[pages][heads][head_dim][page_tokens] beside k_pages [pages][heads][page_tokens][head_dim] is expected");
  if (!apart(k, 3, 1) || !apart(k, 2, dim) || !apart(k, 1, size * dim)) refuse("k_pages", "a page has to be contiguous");
  if (!apart(v, 3, 1) || !apart(v, 2, size) || !apart(v, 1, size * dim)) refuse("v_pages", "a page has to be contiguous");
  const at::Tensor &table = *tensor(args[2], "page_table", at::kInt, 2), &lengths = *tensor(args[3], "lengths", at::kInt, 1);
  const int64_t seqs = lengths.size(0);
  if (table.size(0) != seqs || !apart(table, 1, 1)) refuse("page_table", "[sequences][pages] with adjacent entries is expected");
  if (!apart(lengths, 0, 1)) refuse("lengths", "adjacent entries are expected");
  const bool e4m3 = type == at::kFloat8_e4m3fn;
  const at::Tensor *scales[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i) {
    const char *name = i ? "v_scales" : "k_scales";
    if (!e4m3) {
      if (args[4 + i] != Py_None) refuse(name, "16-bit pages have none");
      continue;
    }
    scales[i] = tensor(args[4 + i], name, at::kFloat, 2);
    if (scales[i]->size(0) != k.size(0) || scales[i]->size(1) != heads || !scales[i]->is_contiguous()) refuse(name, "contiguous [pages][heads] is expected");
  }
  const at::Tensor *starts = tensor(args[6], "starts", at::kInt, 1, true);
  if (starts && (starts->size(0) != seqs + 1 || !apart(*starts, 0, 1))) refuse("starts", "one entry more than sequences is expected");
  d = vq_kv_desc{};
  d.struct_size = sizeof d;
  d.type = e4m3 ? VQ_KV_E4M3 : VQ_KV_FP16;
  d.kv_heads = narrow(heads, "heads"); d.head_dim = narrow(dim, "head_dim"); d.page_tokens = narrow(size, "page_tokens");
  d.n_pages = narrow(k.size(0), "pages"); d.n_seqs = narrow(seqs, "sequences"); d.n_tokens = narrow(n_tokens, "tokens");
  d.table_pages = narrow(table.size(1), "page_table");
  d.max_new = args[7] != Py_None ? whole(args[7], "max_new") : starts ? d.n_tokens : seqs ? d.n_tokens / d.n_seqs : 0;
  d.max_length = args[8] != Py_None ? whole(args[8], "max_length") : narrow(table.size(1) * size, "max_length");
  d.k_pages = k.data_ptr(); d.v_pages = v.data_ptr();
  d.k_page_stride = k.size(0) > 1 ? k.stride(0) : heads * size * dim;
  d.v_page_stride = v.size(0) > 1 ? v.stride(0) : heads * size * dim;
  if (e4m3) { d.k_scales = static_cast<float *>(scales[0]->data_ptr()); d.v_scales = static_cast<float *>(scales[1]->data_ptr()); }
  d.page_table = static_cast<const int32_t *>(table.data_ptr());
  d.table_stride = leading(table);
  d.lengths = static_cast<const int32_t *>(lengths.data_ptr());
  d.starts = starts ? static_cast<const int32_t *>(starts->data_ptr()) : nullptr;
}

// kv_append(k_pages, v_pages, page_table, lengths, k_scales, v_scales, starts, max_new, max_length, k, v, q, q_out, cos, sin, position, interleaved)
PyObject *kv_append(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  if (n != 17) refuse("kv_append", "17 arguments are expected");
  const at::Tensor &k = *tokens(args[9], "k"), &v = *tokens(args[10], "v"), *q = tokens(args[11], "q", true), *to = tokens(args[12], "q_out", true);
  vq_kv_desc d;
  cache_of(args, k.size(0), d);
  if (k.size(1) != d.kv_heads || k.size(2) != d.head_dim || v.sizes() != k.sizes()) refuse("k, v", "[tokens][heads][head_dim] of the pages is expected");
  if (q && (q->size(0) != k.size(0) || q->size(2) != d.head_dim)) refuse("q", "[tokens][query heads][head_dim] is expected");
  if (to && (!q || to->sizes() != q->sizes())) refuse("q_out", "the sizes of q are expected");
  vq_rotary r{};
  const at::Tensor *cos = tensor(args[13], "cos", at::kFloat, 2, true), *sin = tensor(args[14], "sin", at::kFloat, 2, true);
  if (!cos != !sin) refuse("cos, sin", "both or none is expected");
  if (!cos && args[15] != Py_None) refuse("position", "without cos and sin there is nothing to look up");
  if (cos) {
    if (cos->sizes() != sin->sizes() || !apart(*cos, 1, 1) || !apart(*sin, 1, 1) || leading(*cos) != leading(*sin)) refuse("cos, sin", "[positions][pairs] of the same layout is expected");
    const at::Tensor *position = tensor(args[15], "position", at::kInt, 1, true);
    if (position && (position->size(0) != k.size(0) || !apart(*position, 0, 1))) refuse("position", "one entry for each token is expected");
    const int turned = truth(args[16], "interleaved");
    r = vq_rotary{static_cast<const float *>(cos->data_ptr()), static_cast<const float *>(sin->data_ptr()), leading(*cos), narrow(cos->size(0), "cos"),
                  narrow(2 * cos->size(1), "cos"), turned, position ? static_cast<const int32_t *>(position->data_ptr()) : nullptr};
  }
  at::TensorBase fresh;
  void *qp = nullptr, *tp = nullptr;
  int64_t ldq = 0, ldt = 0;
  if (q) {
    if (!to) fresh = empty(q->sizes(), at::kHalf);
    qp = q->data_ptr();
    ldq = leading(*q);
    tp = to ? to->data_ptr() : fresh.data_ptr();
    ldt = to ? leading(*to) : q->size(1) * q->size(2);
  }
  const void *kp = k.data_ptr(), *vp = v.data_ptr();
  const int64_t ldk = leading(k), ldv = leading(v);
  const int32_t heads = q ? narrow(q->size(1), "q") : 0;
  void *s = stream();
  const int rc = released([&] { return p_kv_append(&d, kp, ldk, vp, ldv, qp, ldq, heads, tp, ldt, cos ? &r : nullptr, s); });
  if (rc != VQ_OK) return PyLong_FromLong(rc);
  if (!q) Py_RETURN_NONE;
  if (to) { Py_INCREF(args[12]); return args[12]; }
  return THPVariable_Wrap(std::move(fresh));
  VQ_CATCH
}

// What attention and attention_shared have in common: the call with its workspace (args: scale, out, return_lse, workspace).
template <typename Size, typename Call>
PyObject *attend(const vq_kv_desc &d, const at::Tensor &q, PyObject *scale_of, PyObject *out_of, PyObject *lse_of, PyObject *workspace_of, Size size, Call call) {
  const at::Tensor *out = tokens(out_of, "out", true);
  if (q.size(2) != d.head_dim) refuse("q", "[tokens][query heads][head_dim] is expected");
  if (out && out->sizes() != q.sizes()) refuse("out", "the sizes of q are expected");
  const float scale = scale_of != Py_None ? number(scale_of, "scale") : 1.f / std::sqrt((float)d.head_dim);
  const int32_t heads = narrow(q.size(1), "q");
  const bool with_lse = truth(lse_of, "return_lse");
  void *wp = nullptr;
  size_t bytes = 0;
  at::TensorBase scratch, fresh, lse;
  if (workspace_of == Py_None) {
    bytes = size(heads);
    wp = bytes ? borrow(scratch, bytes) : nullptr;
    if (!wp) bytes = 0;
  } else {
    const at::Tensor &ws = *tensor(workspace_of, "workspace", at::kByte, 1);
    if (!ws.is_contiguous()) refuse("workspace", "adjacent bytes are expected");
    bytes = (size_t)ws.numel();
    wp = bytes ? ws.data_ptr() : nullptr;
  }
  if (!out) fresh = empty(q.sizes(), at::kHalf);
  if (with_lse) lse = empty({q.size(0), q.size(1)}, at::kFloat);
  void *op = out ? out->data_ptr() : fresh.data_ptr(), *s = stream();
  const int64_t ldo = out ? leading(*out) : q.size(1) * q.size(2), ldq = leading(q);
  const void *qp = q.data_ptr();
  float *lp = with_lse ? static_cast<float *>(lse.data_ptr()) : nullptr;
  const int rc = released([&] { return call(qp, ldq, heads, scale, op, ldo, lp, wp, bytes, s); });
  if (rc != VQ_OK) return PyLong_FromLong(rc);
  PyObject *result = out ? (Py_INCREF(out_of), out_of) : THPVariable_Wrap(std::move(fresh));
  if (!with_lse || !result) return result;
  PyObject *second = THPVariable_Wrap(std::move(lse)), *both = second ? PyTuple_Pack(2, result, second) : nullptr;
  Py_DECREF(result);
  Py_XDECREF(second);
  return both;
}

// attention(k_pages, v_pages, page_table, lengths, k_scales, v_scales, starts, max_new, max_length, q, scale, window, sinks, out, return_lse, workspace)
PyObject *attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  if (n != 16) refuse("attention", "16 arguments are expected");
  const at::Tensor &q = *tokens(args[9], "q");
  vq_kv_desc d;
  cache_of(args, q.size(0), d);
  const int32_t window = whole(args[11], "window"), sinks = whole(args[12], "sinks");
  return attend(d, q, args[10], args[13], args[14], args[15], [&](int32_t heads) { return p_attention_workspace_bytes(&d, heads, window, sinks); },
                [&](const void *qp, int64_t ldq, int32_t heads, float scale, void *op, int64_t ldo, float *lp, void *wp, size_t bytes, void *s) {
                  return p_attention(&d, qp, ldq, heads, scale, window, sinks, op, ldo, lp, wp, bytes, s);
                });
  VQ_CATCH
}

// attention_shared(k_pages, v_pages, page_table, lengths, k_scales, v_scales, starts, max_new, max_length, prefix_table, prefix_lengths, members, max_prefix, max_members, max_own,
// q, scale, out, return_lse, workspace)
PyObject *attention_shared(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  if (n != 20) refuse("attention_shared", "20 arguments are expected");
  const at::Tensor &q = *tokens(args[15], "q");
  vq_kv_desc d;
  cache_of(args, q.size(0), d);
  const at::Tensor &table = *tensor(args[9], "prefix_table", at::kInt, 2), &lengths = *tensor(args[10], "prefix_lengths", at::kInt, 1), *members = tensor(args[11], "members", at::kInt, 1, true);
  const int64_t prefixes = lengths.size(0);
  if (table.size(0) != prefixes || !apart(table, 1, 1)) refuse("prefix_table", "[prefixes][pages] with adjacent entries is expected");
  if (!apart(lengths, 0, 1)) refuse("prefix_lengths", "adjacent entries are expected");
  if (members && (members->size(0) != prefixes + 1 || !apart(*members, 0, 1))) refuse("members", "one entry more than prefixes is expected");
  if (!members && prefixes != 1) refuse("members", "several prefixes need them");
  vq_prefix_desc x{};
  x.struct_size = sizeof x;
  x.n_prefixes = narrow(prefixes, "prefix_lengths");
  x.table_pages = narrow(table.size(1), "prefix_table");
  x.max_length = args[12] != Py_None ? whole(args[12], "max_prefix") : narrow(table.size(1) * d.page_tokens, "max_prefix");
  x.max_members = args[13] != Py_None ? whole(args[13], "max_members") : d.n_seqs;
  // (what the bounds of the lengths leave; where they say nothing of it, all: a prefix is not worth a launch of its own then)
  x.max_own = args[14] != Py_None ? whole(args[14], "max_own") : x.max_length >= 0 && x.max_length < d.max_length ? std::max(d.max_length - x.max_length, d.max_new) : d.max_length;
  x.page_table = static_cast<const int32_t *>(table.data_ptr());
  x.table_stride = leading(table);
  x.lengths = static_cast<const int32_t *>(lengths.data_ptr());
  x.members = members ? static_cast<const int32_t *>(members->data_ptr()) : nullptr;
  return attend(d, q, args[16], args[17], args[18], args[19], [&](int32_t heads) { return p_attention_shared_workspace_bytes(&d, &x, heads); },
                [&](const void *qp, int64_t ldq, int32_t heads, float scale, void *op, int64_t ldo, float *lp, void *wp, size_t bytes, void *s) {
                  return p_attention_shared(&d, &x, qp, ldq, heads, scale, op, ldo, lp, wp, bytes, s);
                });
  VQ_CATCH
}

// embed(ids, table, scale, dtype or None, out or None)
PyObject *embed(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  if (n != 5) refuse("embed", "five arguments are expected");
  const at::Tensor &ids = *tensor(args[0], "ids", at::kInt, 1), &table = *tensor(args[1], "table", at::kHalf, 2);
  if (!apart(ids, 0, 1)) refuse("ids", "adjacent entries are expected");
  if (!apart(table, 1, 1)) refuse("table", "adjacent elements are expected");
  const float scale = number(args[2], "scale");
  at::ScalarType type = at::kHalf;
  const bool given = args[4] != Py_None;
  if (given && THPVariable_Check(args[4])) type = THPVariable_Unpack(args[4]).scalar_type();
  if (args[3] != Py_None) {
    if (!THPDtype_Check(args[3])) refuse("dtype", "a torch.dtype is expected");
    const at::ScalarType asked = reinterpret_cast<THPDtype *>(args[3])->scalar_type;
    if (given && asked != type) refuse("out", "the type of dtype is expected");
    type = asked;
  }
  if (type != at::kHalf && type != at::kFloat) refuse(given ? "out" : "dtype", "float16 or float32 is expected");
  const at::Tensor *out = tensor(args[4], "out", type, 2, true);
  const int64_t rows = ids.size(0), width = table.size(1);
  if (out && (out->size(0) != rows || out->size(1) != width || !apart(*out, 1, 1))) refuse("out", "[tokens][width] with adjacent elements is expected");
  at::TensorBase fresh;
  if (!out) fresh = empty({rows, width}, type);
  void *yp = out ? out->data_ptr() : fresh.data_ptr(), *s = stream();
  const int32_t m = narrow(rows, "ids"), words = narrow(table.size(0), "table"), w = narrow(width, "table");
  const int32_t *ip = static_cast<const int32_t *>(ids.data_ptr());
  const void *tp = table.data_ptr();
  const int64_t ld = leading(table), ldy = out ? leading(*out) : width;
  const int rc = released([&] { return p_embed(ip, m, tp, ld, words, w, scale, type == at::kFloat, yp, ldy, s); });
  return tensor_or_status(rc, std::move(fresh), args[4]);
  VQ_CATCH
}

// sample(logits, uniform, temperature, top_k, top_p, min_p, out or None, return_prob)
PyObject *sample(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  if (n != 8) refuse("sample", "eight arguments are expected");
  const at::Tensor &logits = *tensor(args[0], "logits", at::kHalf, 2), &uniform = *tensor(args[1], "uniform", at::kFloat, 1);
  if (!apart(logits, 1, 1)) refuse("logits", "adjacent elements are expected");
  const int64_t rows = logits.size(0);
  auto of_rows = [&](const at::Tensor &t, const char *name) {
    if (t.size(0) != rows || !apart(t, 0, 1)) refuse(name, "one entry for each row is expected");
    return t.data_ptr();
  };
  const float *up = static_cast<const float *>(of_rows(uniform, "uniform"));
  vq_sampling how{};
  how.struct_size = sizeof how;
  auto setting = [&](PyObject *o, const char *name, float &one, const float *&each) {
    if (THPVariable_Check(o)) each = static_cast<const float *>(of_rows(*tensor(o, name, at::kFloat, 1), name));
    else one = number(o, name);
  };
  setting(args[2], "temperature", how.temperature, how.temperatures);
  if (THPVariable_Check(args[3])) how.top_ks = static_cast<const int32_t *>(of_rows(*tensor(args[3], "top_k", at::kInt, 1), "top_k"));
  else how.top_k = whole(args[3], "top_k");
  setting(args[4], "top_p", how.top_p, how.top_ps);
  setting(args[5], "min_p", how.min_p, how.min_ps);
  const at::Tensor *out = tensor(args[6], "out", at::kInt, 1, true);
  if (out) of_rows(*out, "out");
  const bool with_prob = truth(args[7], "return_prob");
  at::TensorBase fresh, prob;
  if (!out) fresh = empty({rows}, at::kInt);
  if (with_prob) prob = empty({rows}, at::kFloat);
  int32_t *tp = static_cast<int32_t *>(out ? out->data_ptr() : fresh.data_ptr());
  float *pp = with_prob ? static_cast<float *>(prob.data_ptr()) : nullptr;
  const void *lp = logits.data_ptr();
  void *s = stream();
  const int64_t ld = leading(logits);
  const int32_t m = narrow(rows, "logits"), words = narrow(logits.size(1), "logits");
  const int rc = released([&] { return p_sample(lp, ld, m, words, up, &how, tp, pp, s); });
  if (rc != VQ_OK) return PyLong_FromLong(rc);
  PyObject *result = out ? (Py_INCREF(args[6]), args[6]) : THPVariable_Wrap(std::move(fresh));
  if (!with_prob || !result) return result;
  PyObject *second = THPVariable_Wrap(std::move(prob)), *both = second ? PyTuple_Pack(2, result, second) : nullptr;
  Py_DECREF(result);
  Py_XDECREF(second);
  return both;
  VQ_CATCH
}

// residual_norm(h or None, x, pre or None, post or None, gate or None, scale, eps, y or None, z or None) -> (y, z or None)
PyObject *residual_norm(PyObject *, PyObject *const *args, Py_ssize_t n) {
  VQ_TRY
  if (n != 9) refuse("residual_norm", "nine arguments are expected");
  if (!THPVariable_Check(args[1])) refuse("x", "a tensor is expected");
  const at::ScalarType type = THPVariable_Unpack(args[1]).scalar_type();
  if (type != at::kHalf && type != at::kFloat) refuse("x", "float16 or float32 is expected");
  const at::Tensor &x = *tensor(args[1], "x", type, 2), *h = tensor(args[0], "h", at::kHalf, 2, true);
  const int64_t rows = x.size(0), width = x.size(1);
  auto matrix = [&](const at::Tensor *t, const char *name) {
    if (t && (t->size(0) != rows || t->size(1) != width || !apart(*t, 1, 1))) refuse(name, "[rows][width] of x with adjacent elements is expected");
    return t;
  };
  auto weight = [&](PyObject *o, const char *name) -> const void * {
    const at::Tensor *t = tensor(o, name, at::kHalf, 1, true);
    if (t && (t->size(0) != width || !apart(*t, 0, 1))) refuse(name, "one entry for each of a row's elements is expected");
    return t ? t->data_ptr() : nullptr;
  };
  matrix(&x, "x");
  matrix(h, "h");
  const void *pre = weight(args[2], "pre"), *post = weight(args[3], "post"), *gate = nullptr;
  int64_t ldgate = 0;
  if (args[4] != Py_None) {
    if (THPVariable_Check(args[4]) && THPVariable_Unpack(args[4]).dim() == 1) {
      gate = weight(args[4], "gate");
    } else {
      const at::Tensor &g = *matrix(tensor(args[4], "gate", at::kHalf, 2), "gate");
      gate = g.data_ptr();
      ldgate = rows > 1 ? g.stride(0) : 0;
    }
  }
  const float scale = number(args[5], "scale"), eps = number(args[6], "eps");
  const at::Tensor *y = matrix(tensor(args[7], "y", type, 2, true), "y"), *z = matrix(tensor(args[8], "z", at::kHalf, 2, true), "z");
  if (z && !pre) refuse("z", "without pre there is nothing to write");
  at::TensorBase fresh_y, fresh_z;
  if (!y) fresh_y = empty({rows, width}, type);
  if (!z && pre) fresh_z = empty({rows, width}, at::kHalf);
  void *yp = y ? y->data_ptr() : fresh_y.data_ptr(), *zp = z ? z->data_ptr() : pre ? fresh_z.data_ptr() : nullptr, *s = stream();
  const void *xp = x.data_ptr(), *hp = h ? h->data_ptr() : nullptr;
  const int64_t ldx = leading(x), ldh = h ? leading(*h) : 0, ldy = y ? leading(*y) : width, ldz = z ? leading(*z) : width;
  const int32_t m = narrow(rows, "rows"), w = narrow(width, "width");
  const int rc = released([&] { return p_residual_norm(hp, ldh, xp, ldx, post, gate, ldgate, scale, pre, eps, type == at::kFloat, m, w, yp, ldy, zp, ldz, s); });
  if (rc != VQ_OK) return PyLong_FromLong(rc);
  PyObject *first = y ? (Py_INCREF(args[7]), args[7]) : THPVariable_Wrap(std::move(fresh_y));
  PyObject *second = z ? (Py_INCREF(args[8]), args[8]) : pre ? THPVariable_Wrap(std::move(fresh_z)) : (Py_INCREF(Py_None), Py_None);
  PyObject *both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
  Py_XDECREF(first);
  Py_XDECREF(second);
  return both;
  VQ_CATCH
}

PyMethodDef methods[] = {{"gemv", (PyCFunction)(void *)gemv, METH_FASTCALL, nullptr},
                         {"gemv_multi", (PyCFunction)(void *)gemv_multi, METH_FASTCALL, nullptr},
                         {"gemm", (PyCFunction)(void *)gemm, METH_FASTCALL, nullptr},
                         {"dequant", dequant, METH_O, nullptr},
                         {"assign", (PyCFunction)(void *)assign, METH_FASTCALL, nullptr},
                         {"kv_append", (PyCFunction)(void *)kv_append, METH_FASTCALL, nullptr},
                         {"attention", (PyCFunction)(void *)attention, METH_FASTCALL, nullptr},
                         {"residual_norm", (PyCFunction)(void *)residual_norm, METH_FASTCALL, nullptr},
                         {"attention_shared", (PyCFunction)(void *)attention_shared, METH_FASTCALL, nullptr},
                         {"embed", (PyCFunction)(void *)embed, METH_FASTCALL, nullptr},
                         {"sample", (PyCFunction)(void *)sample, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

// bind(addresses): the library's entry points, which the package has loaded
PyObject *bind(PyObject *, PyObject *addresses) {
  auto at = [&](const char *name, auto &f) {
    PyObject *a = PyDict_GetItemString(addresses, name);
    if (!a) return false;
    f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(PyLong_AsVoidPtr(a));
    return f != nullptr;
  };
  if (!at("vq_gemv", p_gemv) || !at("vq_gemv_with_workspace", p_gemv_ws) || !at("vq_gemv_multi", p_gemv_multi) || !at("vq_gemm", p_gemm) || !at("vq_gemm_default", p_gemm_default) ||
      !at("vq_gemm_workspace_bytes", p_gemm_workspace_bytes) || !at("vq_lend_gemv_bytes", p_lend_gemv_bytes) || !at("vq_gemm_default_workspace_bytes", p_gemm_default_workspace_bytes) ||
      !at("vq_lend_gemm_least_bytes", p_lend_gemm_least_bytes) ||
       !at("vq_dequant", p_dequant) || !at("vq_lend_assign", p_lend_assign) || !at("vq_kv_append", p_kv_append) || !at("vq_attention", p_attention) ||
       !at("vq_attention_workspace_bytes", p_attention_workspace_bytes) || !at("vq_residual_norm", p_residual_norm) ||
       !at("vq_attention_shared", p_attention_shared) || !at("vq_attention_shared_workspace_bytes", p_attention_shared_workspace_bytes) || !at("vq_embed", p_embed) || !at("vq_sample", p_sample)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point is missing");
    return nullptr;
  }
  Py_RETURN_NONE;
}
PyMethodDef bind_method = {"bind", bind, METH_O, nullptr};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  PyObject *m = PyModule_Create(&module);
  if (!m) return nullptr;
  s_desc = PyUnicode_InternFromString("desc");
  s_places = PyUnicode_InternFromString("places_every_column");
  PyObject *f = PyCFunction_New(&bind_method, nullptr);
  if (!f || PyModule_AddObject(m, "bind", f) != 0) return nullptr;
  return m;
}
