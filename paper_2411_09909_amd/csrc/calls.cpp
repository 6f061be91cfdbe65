// The calls of a serving loop - casts and products into buffers that the caller keeps - without the interpreter and ctypes
// between torch and the C ABI: tensors are taken apart here, and the call made, in 0.3 us instead of 1.8 to 2.9 (a kernel
// launch through the runtime takes 2.3 to 2.9 us itself; a cast and a product of 64 x 1024 x 1024 among others: 11.3 -> 8.2 us, of
// which the kernels and the gaps between them are 6.5).
// Every function returns the status of the C call, or None for arguments that it does not take as they are (buffers to be
// allocated, anything that is not a plain tensor on the GPU, wrong dimensions); binding.py then goes its general way, which
// also says what is wrong with them.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPStream.h>

#include "../../include/amxfp4.h"
#include "../../include/amxfp4_paged.h"

namespace {

// Entry points by address, from the library that binding.py has loaded (bind()).
struct {
  decltype(&amxfp4_quantize) quantize;
  decltype(&amxfp4_quantize_scaled) quantize_scaled;
  decltype(&amxfp4_quantize_batched) quantize_batched;
  decltype(&amxfp4_tensor_scale) tensor_scale;
  decltype(&amxfp4_gemm) gemm;
  decltype(&amxfp4_gemm_scaled) gemm_scaled;
  decltype(&amxfp4_gemm_prepared) gemm_prepared;
  decltype(&amxfp4_attention) attention;
  decltype(&amxfp4_attention_merged) attention_merged;
  decltype(&amxfp4_attention_decode) attention_decode;
  decltype(&amxfp4_paged_plan) paged_plan;
  decltype(&amxfp4_paged_write) paged_write;
  decltype(&amxfp4_paged_read) paged_read;
  decltype(&amxfp4_paged_attention) paged_attention;
} entry;
constexpr const char* kEntries[] = {"amxfp4_quantize", "amxfp4_quantize_scaled", "amxfp4_quantize_batched", "amxfp4_tensor_scale",
                                    "amxfp4_gemm", "amxfp4_gemm_scaled", "amxfp4_gemm_prepared", "amxfp4_attention",
                                    "amxfp4_attention_merged", "amxfp4_attention_decode", "amxfp4_paged_plan", "amxfp4_paged_write",
                                    "amxfp4_paged_read", "amxfp4_paged_attention"};
constexpr size_t kNumEntries = sizeof(kEntries) / sizeof(kEntries[0]);
static_assert(sizeof(entry) == kNumEntries * sizeof(void*), "one name per entry point");

// A plain tensor (torch.Tensor or Parameter itself, no subclass with ways of its own) on the GPU, or null.
const at::Tensor* tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() ? &t : nullptr;
}

// The first n arguments from `from` on as such tensors; contiguous: all of them.
bool tensors(PyObject* const* args, int from, int n, const at::Tensor** out, bool contiguous) {
  for (int i = 0; i < n; ++i)
    if (!(out[i] = tensor(args[from + i])) || (contiguous && !out[i]->is_contiguous())) return false;
  return true;
}

uint8_t* bytes(const at::Tensor* t) { return static_cast<uint8_t*>(t->data_ptr()); }
size_t size_of(const at::Tensor* t) { return (size_t)t->numel() * t->element_size(); }

// a tensor-scale pair: a contiguous float32 tensor of two elements or more
const at::Tensor* pair(PyObject* o) {
  const at::Tensor* t = tensor(o);
  return t && t->scalar_type() == at::kFloat && t->numel() >= 2 && t->is_contiguous() ? t : nullptr;
}

// The format, out of its ctypes structure (the class given to bind(), or one derived from it: other structures and bytes of the
// same size are no formats).
PyTypeObject* format_type = nullptr;
bool format(PyObject* o, amx_format_t& f) {
  if (!format_type || !PyObject_TypeCheck(o, format_type)) return false;
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
    PyErr_Clear();
    return false;
  }
  const bool ok = view.len == (Py_ssize_t)sizeof(f);
  if (ok) memcpy(&f, view.buf, sizeof(f));
  PyBuffer_Release(&view);
  return ok;
}

// Runs the C call with the interpreter released, on the current stream of the current device.
template <class Call>
PyObject* run(Call call) {
  int status;
  void* stream = c10::hip::getCurrentHIPStream().stream();
  Py_BEGIN_ALLOW_THREADS;
  status = call(stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(status);
}

// quantize(fmt, x, along_rows, codes, scales, tensor_pair or None)
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  const at::Tensor *x, *out[2], *p = nullptr;
  if (n != 6 || !format(args[0], f) || !(x = tensor(args[1])) || x->dim() != 2 || x->element_size() != 2 ||
      !tensors(args, 3, 2, out, false) || (args[5] != Py_None && !(p = pair(args[5]))))
    Py_RETURN_NONE;
  const int r = args[2] == Py_True ? 0 : 1;  // the dimension of x that holds the rows
  const int64_t rows = x->size(r), K = x->size(1 - r), row_stride = x->stride(r), k_stride = x->stride(1 - r);
  const void* from = x->data_ptr();
  uint8_t *codes = bytes(out[0]), *scales = bytes(out[1]);
  const float* ratio = p ? static_cast<const float*>(p->data_ptr()) : nullptr;
  return run([&](void* s) {
    return ratio ? entry.quantize_scaled(&f, from, rows, K, row_stride, k_stride, ratio, codes, scales, s)
                 : entry.quantize(&f, from, rows, K, row_stride, k_stride, codes, scales, s);
  });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// quantize_batched(fmt, x, along_rows, codes, scales)
PyObject* quantize_batched(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  const at::Tensor *x, *out[2];
  if (n != 5 || !format(args[0], f) || !(x = tensor(args[1])) || x->dim() != 3 || x->element_size() != 2 ||
      !tensors(args, 3, 2, out, false))
    Py_RETURN_NONE;
  const int r = args[2] == Py_True ? 1 : 2;
  const int64_t batch = x->size(0), batch_stride = x->stride(0), rows = x->size(r), K = x->size(3 - r);
  const int64_t row_stride = x->stride(r), k_stride = x->stride(3 - r);
  const void* from = x->data_ptr();
  uint8_t *codes = bytes(out[0]), *scales = bytes(out[1]);
  return run([&](void* s) {
    return entry.quantize_batched(&f, from, batch, batch_stride, rows, K, row_stride, k_stride, codes, scales, s);
  });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// tensor_scale(x, out)
PyObject* tensor_scale(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  const at::Tensor *x, *out;
  if (n != 2 || !(x = tensor(args[0])) || !(out = tensor(args[1])) || x->dim() != 2 || x->element_size() != 2 || x->stride(1) != 1)
    Py_RETURN_NONE;
  const void* from = x->data_ptr();
  float* to = static_cast<float*>(out->data_ptr());
  return run([&](void* s) { return entry.tensor_scale(from, x->size(0), x->size(1), x->stride(0), to, s); });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// gemm(fmt, a_codes, a_scales, b_codes, b_scales, out, workspace, a_pair or None, b_pair or None)
PyObject* gemm(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  const at::Tensor *t[4], *to[2], *pa = nullptr, *pb = nullptr;
  if (n != 9 || !format(args[0], f) || !tensors(args, 1, 4, t, true) || !tensors(args, 5, 2, to, false)) Py_RETURN_NONE;
  const bool scaled = args[7] != Py_None || args[8] != Py_None;
  if (scaled && (!(pa = pair(args[7])) || !(pb = pair(args[8])))) Py_RETURN_NONE;
  if ((t[0]->dim() != 2 && t[0]->dim() != 3) || t[2]->dim() < 2 || to[0]->dim() < 2) Py_RETURN_NONE;
  const int64_t batch = t[0]->dim() == 3 ? t[0]->size(0) : 1, M = t[0]->size(-2), K = t[0]->size(-1) * 2, N = t[2]->size(-2);
  const int64_t ldc = to[0]->stride(-2);
  uint8_t *ac = bytes(t[0]), *as = bytes(t[1]), *bc = bytes(t[2]), *bs = bytes(t[3]), *ws = bytes(to[1]);
  float *c = static_cast<float*>(to[0]->data_ptr()), *ra = nullptr, *rb = nullptr;
  if (scaled) ra = static_cast<float*>(pa->data_ptr()), rb = static_cast<float*>(pb->data_ptr());
  const size_t ws_bytes = size_of(to[1]);
  return run([&](void* s) {
    return scaled ? entry.gemm_scaled(&f, M, N, K, ac, as, ra, bc, bs, rb, c, ldc, batch, ws, ws_bytes, s)
                  : entry.gemm(&f, M, N, K, ac, as, bc, bs, c, ldc, batch, ws, ws_bytes, s);
  });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// gemm_prepared(fmt, a_codes, a_scales, b_codes, b_scales, prepared, out, workspace)
PyObject* gemm_prepared(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  const at::Tensor* t[7];
  if (n != 8 || !format(args[0], f) || !tensors(args, 1, 7, t, false)) Py_RETURN_NONE;
  if (t[0]->dim() != 2 || t[2]->dim() < 1 || t[5]->dim() < 2) Py_RETURN_NONE;
  const int64_t M = t[0]->size(0), K = t[0]->size(1) * 2, N = t[2]->size(0), ldc = t[5]->stride(-2);
  uint8_t *ac = bytes(t[0]), *as = bytes(t[1]), *bc = bytes(t[2]), *bs = bytes(t[3]), *ws = bytes(t[6]);
  const size_t prepared_bytes = size_of(t[4]), ws_bytes = size_of(t[6]);
  void* prepared = prepared_bytes ? t[4]->data_ptr() : nullptr;
  float* c = static_cast<float*>(t[5]->data_ptr());
  return run([&](void* s) {
    return entry.gemm_prepared(&f, M, N, K, ac, as, bc, bs, prepared, prepared_bytes, c, ldc, ws, ws_bytes, s);
  });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// q_codes [Hq, Sq, D/2], .., k_codes [Hkv, Sk, D/2], .., v_codes [Hkv, D, Sk/2], ..: whether the shapes go together
bool heads(const at::Tensor* const* t) {
  return t[0]->dim() == 3 && t[2]->dim() == 3 && t[4]->dim() == 3 && t[2]->size(2) == t[0]->size(2) && t[4]->size(0) == t[2]->size(0) &&
         t[4]->size(1) == 2 * t[0]->size(2) && t[4]->size(2) == t[2]->size(1) / 2;
}

// attention(fmt, q_codes, q_scales, k_codes, k_scales, v_codes, v_scales, scale, causal, out, workspace, merged)
PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  const at::Tensor *t[6], *to[2];
  if (n != 12 || !format(args[0], f) || !tensors(args, 1, 6, t, true) || !heads(t) || !tensors(args, 9, 2, to, false) ||
      !PyFloat_CheckExact(args[7]))
    Py_RETURN_NONE;
  const bool merged = args[11] == Py_True, causal = args[8] == Py_True;
  if (!to[0]->is_contiguous() || to[0]->scalar_type() != (merged ? at::kBFloat16 : at::kFloat)) Py_RETURN_NONE;
  const int64_t Hq = t[0]->size(0), Sq = t[0]->size(1), D = t[0]->size(2) * 2, Hkv = t[2]->size(0), Sk = t[2]->size(1);
  uint8_t* p[6];
  for (int i = 0; i < 6; ++i) p[i] = bytes(t[i]);
  const float scale = (float)PyFloat_AS_DOUBLE(args[7]);
  float* out = static_cast<float*>(to[0]->data_ptr());
  uint8_t* ws = bytes(to[1]);
  const size_t ws_bytes = size_of(to[1]);
  return run([&](void* s) {
    return merged ? entry.attention_merged(&f, Hq, Hkv, Sq, Sk, D, p[0], p[1], p[2], p[3], p[4], p[5], scale, causal,
                                           reinterpret_cast<uint16_t*>(out), ws, ws_bytes, s)
                  : entry.attention(&f, Hq, Hkv, Sq, Sk, D, p[0], p[1], p[2], p[3], p[4], p[5], scale, causal, out, ws, ws_bytes, s);
  });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// attention_decode(fmt, q_codes, q_scales, k_codes, k_scales, v_codes, v_scales, scale, causal, key_splits, out, workspace)
PyObject* attention_decode(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  const at::Tensor *t[6], *to[2];
  if (n != 12 || !format(args[0], f) || !tensors(args, 1, 6, t, true) || !heads(t) || !tensors(args, 10, 2, to, false) ||
      !PyFloat_CheckExact(args[7]) || !PyLong_CheckExact(args[9]))
    Py_RETURN_NONE;
  const long long splits = PyLong_AsLongLong(args[9]);
  if (splits == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  const int64_t Hq = t[0]->size(0), Sq = t[0]->size(1), D = t[0]->size(2) * 2, Hkv = t[2]->size(0), Sk = t[2]->size(1);
  uint8_t* p[6];
  for (int i = 0; i < 6; ++i) p[i] = bytes(t[i]);
  const float scale = (float)PyFloat_AS_DOUBLE(args[7]);
  const bool causal = args[8] == Py_True;
  float* out = static_cast<float*>(to[0]->data_ptr());
  uint8_t* ws = bytes(to[1]);
  const size_t ws_bytes = size_of(to[1]);
  return run([&](void* s) {
    return entry.attention_decode(&f, Hq, Hkv, Sq, Sk, D, p[0], p[1], p[2], p[3], p[4], p[5], scale, causal, splits, out, ws, ws_bytes, s);
  });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// ---- the paged cache: contiguous tensors on the current device, as binding.py's general way wants them

const at::Tensor* here(PyObject* o) {
  const at::Tensor* t = tensor(o);
  return t && t->is_contiguous() && t->get_device() == c10::hip::current_device() ? t : nullptr;
}

// one-dimensional int32 of n elements (any number for n < 0)
int32_t* ints(PyObject* o, int64_t n, int64_t* count = nullptr) {
  const at::Tensor* t = here(o);
  if (!t || t->scalar_type() != at::kInt || t->dim() != 1 || (n >= 0 && t->numel() != n)) return nullptr;
  if (count) *count = t->numel();
  return static_cast<int32_t*>(t->data_ptr());
}

// int32 [seqs, max_pages]
int32_t* block_table(PyObject* o, int64_t seqs, int64_t& max_pages) {
  const at::Tensor* t = here(o);
  if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != seqs) return nullptr;
  max_pages = t->size(1);
  return static_cast<int32_t*>(t->data_ptr());
}

// four uint8 tensors as in binding.PagedPool
bool pool(PyObject* o, const amx_format_t& f, amx_paged_pool_t& p) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return false;
  const at::Tensor* t[4];
  for (int i = 0; i < 4; ++i)
    if (!(t[i] = here(PyTuple_GET_ITEM(o, i))) || t[i]->scalar_type() != at::kByte) return false;
  if (t[0]->dim() != 4 || t[2]->sizes() != t[0]->sizes() || t[3]->sizes() != t[1]->sizes() || t[1]->dim() != (f.asymmetric ? 5 : 4)) return false;
  const at::Tensor &c = *t[0], &s = *t[1];
  if (s.size(0) != c.size(0) || s.size(1) != c.size(1) || s.size(2) != c.size(3) / 16 || s.size(3) != c.size(2) ||
      (f.asymmetric && s.size(4) != 2) || c.size(1) > INT32_MAX || c.size(2) > INT32_MAX || c.size(3) > INT32_MAX / 2)
    return false;
  p = {c.size(0), (int32_t)c.size(2), (int32_t)c.size(1), (int32_t)c.size(3) * 2, 0, bytes(t[0]), bytes(t[1]), bytes(t[2]), bytes(t[3])};
  return true;
}

bool integer(PyObject* o, int64_t& v) {
  if (!PyLong_CheckExact(o)) return false;
  v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}

// paged_plan(lens, new_rows, table, queue, state, page_size, (lens, starts, slots, positions, state))
PyObject* paged_plan(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  if (n != 7 || !PyTuple_Check(args[6]) || PyTuple_GET_SIZE(args[6]) != 5) Py_RETURN_NONE;
  int64_t seqs, pages, max_pages, page_size, rows;
  int32_t *lens, *fresh, *table, *queue, *state, *out[5];
  if (!(lens = ints(args[0], -1, &seqs)) || !(fresh = ints(args[1], seqs)) || !(table = block_table(args[2], seqs, max_pages)) ||
      !(queue = ints(args[3], -1, &pages)) || !(state = ints(args[4], 4)) || !integer(args[5], page_size) ||
      !(out[2] = ints(PyTuple_GET_ITEM(args[6], 2), -1, &rows)))
    Py_RETURN_NONE;
  const int64_t want[5] = {seqs, seqs + 1, rows, rows, 4};
  for (int i = 0; i < 5; ++i)
    if (!(out[i] = ints(PyTuple_GET_ITEM(args[6], i), want[i]))) Py_RETURN_NONE;
  return run([&](void* s) {
    return entry.paged_plan(lens, fresh, seqs, rows, page_size, pages, max_pages, state, queue, table, out[0], out[1], out[2], out[3], out[4], s);
  });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// paged_write(fmt, proj, pool, slots, positions, q_heads, theta, q)
PyObject* paged_write(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  amx_paged_pool_t p;
  const at::Tensor *x, *q;
  int64_t heads;
  if (n != 8 || !format(args[0], f) || !(x = tensor(args[1])) || !pool(args[2], f, p) || !integer(args[5], heads) || !PyFloat_CheckExact(args[6]) ||
      !(q = here(args[7])))
    Py_RETURN_NONE;
  if (x->scalar_type() != at::kFloat || x->dim() != 2 || x->stride(1) != 1 || x->get_device() != c10::hip::current_device() ||
      q->scalar_type() != at::kBFloat16 || heads <= 0 || heads > 1024)
    Py_RETURN_NONE;
  const int64_t rows = x->size(0), width = (heads + 2 * (int64_t)p.kv_heads) * p.head_dim, ld = rows > 1 ? x->stride(0) : width;
  int32_t *slots = ints(args[3], rows), *positions = ints(args[4], rows);
  if (!slots || !positions || x->size(1) < width || q->numel() != rows * heads * p.head_dim) Py_RETURN_NONE;
  const float* in = static_cast<const float*>(x->data_ptr());
  const double theta = PyFloat_AS_DOUBLE(args[6]);
  void* to = q->data_ptr();
  return run([&](void* s) { return entry.paged_write(&f, &p, in, rows, ld, heads, slots, positions, theta, to, s); });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// paged_read(fmt, pool, slots, k, v)
PyObject* paged_read(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  amx_paged_pool_t p;
  const at::Tensor *k, *v;
  int64_t rows;
  if (n != 5 || !format(args[0], f) || !pool(args[1], f, p) || !(k = here(args[3])) || !(v = here(args[4]))) Py_RETURN_NONE;
  int32_t* slots = ints(args[2], -1, &rows);
  const bool bf16 = k->scalar_type() == at::kBFloat16;
  if (!slots || (!bf16 && k->scalar_type() != at::kFloat) || v->scalar_type() != k->scalar_type() || k->dim() != 3 || v->sizes() != k->sizes() ||
      k->size(0) != rows || k->size(1) != p.kv_heads || k->size(2) != p.head_dim)
    Py_RETURN_NONE;
  void *to_k = k->data_ptr(), *to_v = v->data_ptr();
  return run([&](void* s) { return entry.paged_read(&f, &p, slots, rows, bf16, to_k, to_v, s); });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// paged_attention(fmt, q, pool, table, lens, starts, positions, scale, max_keys, out, workspace)
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n) try {
  amx_format_t f;
  amx_paged_pool_t p;
  const at::Tensor *q, *out, *ws;
  int64_t seqs, max_pages, max_keys;
  if (n != 11 || !format(args[0], f) || !(q = here(args[1])) || !pool(args[2], f, p) || !PyFloat_CheckExact(args[7]) || !integer(args[8], max_keys) ||
      !(out = here(args[9])) || !(ws = here(args[10])))
    Py_RETURN_NONE;
  int32_t *lens = ints(args[4], -1, &seqs), *table, *starts, *positions;
  if (!lens || q->scalar_type() != at::kBFloat16 || q->dim() != 3 || q->size(2) != p.head_dim || out->scalar_type() != at::kBFloat16 ||
      out->numel() != q->numel() || !(table = block_table(args[3], seqs, max_pages)) || !(starts = ints(args[5], seqs + 1)) ||
      !(positions = ints(args[6], q->size(0))))
    Py_RETURN_NONE;
  const int64_t rows = q->size(0), heads = q->size(1);
  const float scale = (float)PyFloat_AS_DOUBLE(args[7]);
  const void* from = q->data_ptr();
  void *to = out->data_ptr(), *scratch = ws->data_ptr();
  const size_t ws_bytes = size_of(ws);
  return run([&](void* s) {
    return entry.paged_attention(&f, &p, from, rows, heads, table, seqs, max_pages, lens, starts, positions, scale, max_keys, to, scratch, ws_bytes, s);
  });
} catch (const std::exception&) {
  Py_RETURN_NONE;
}

// bind(class of the formats, address of each of `entries`)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void* address[kNumEntries];
  if (n != (Py_ssize_t)kNumEntries + 1 || !PyType_Check(args[0]))
    return PyErr_Format(PyExc_TypeError, "bind: a class and %zu addresses", kNumEntries);
  for (size_t i = 0; i < kNumEntries; ++i) {
    address[i] = PyLong_AsVoidPtr(args[i + 1]);
    if (!address[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "bind: %s is null", kEntries[i]);
  }
  memcpy(&entry, address, sizeof(address));
  Py_INCREF(args[0]);
  PyTypeObject* before = format_type;
  format_type = reinterpret_cast<PyTypeObject*>(args[0]);
  Py_XDECREF(before);
  Py_RETURN_NONE;
}

#define CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {CALL(quantize), CALL(quantize_batched), CALL(tensor_scale), CALL(gemm), CALL(gemm_prepared),
                          CALL(attention), CALL(attention_decode), CALL(paged_plan), CALL(paged_write), CALL(paged_read),
                          CALL(paged_attention), CALL(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  PyObject* m = PyModule_Create(&kModule);
  PyObject* names = m ? PyTuple_New(kNumEntries) : nullptr;
  for (size_t i = 0; names && i < kNumEntries; ++i) PyTuple_SET_ITEM(names, i, PyUnicode_FromString(kEntries[i]));
  if (!names || PyModule_AddObject(m, "entries", names) != 0) return nullptr;
  if (PyModule_AddStringConstant(m, "torch_version", AMX_TORCH_VERSION) != 0) return nullptr;  // binding.py asks before bind()
  return m;
}
