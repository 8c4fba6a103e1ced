// Native half of the Python binding of the operators between the linear layers
// (kvcache.py): torch tensors checked, outputs made, the C entry point called.  An
// eager decode step is bound by its host work, and this is a third of what the same
// checks take through ctypes.  Nothing here touches the GPU but the allocator and the
// entry points of libtq.so, whose addresses the Python side passes in once.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>

#include <cmath>
#include <cstdarg>
#include <string>

#include "tq.h"

namespace {

struct Failed {};    // a Python exception is set

[[noreturn]] void fail(PyObject *type, const char *format, ...) {
  va_list args;
  va_start(args, format);
  PyErr_FormatV(type, format, args);
  va_end(args);
  throw Failed();
}

std::string shape_of(const at::Tensor &t) {
  std::string s = "(";
  for (int64_t i = 0; i < t.dim(); i++) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + ")";
}

// ------------------------------------------------------------------ the library
struct Entries {
  decltype(&tq_qk_norm_rope) norm_rope;
  decltype(&tq_kv_append) append;
  decltype(&tq_qk_norm_rope_append) norm_rope_append;
  decltype(&tq_kv_read) read;
  decltype(&tq_paged_attention_scratch_bytes) scratch_bytes;
  decltype(&tq_prompt_attention_scratch_bytes) prompt_bytes;
  decltype(&tq_prompt_attention) prompt;
  decltype(&tq_paged_attention_scored) attend_scored;
  decltype(&tq_shared_prefix_attention_scratch_bytes) prefix_bytes;
  decltype(&tq_shared_prefix_attention) prefix;
  decltype(&tq_add_rms_norm) add_norm;
} L;
PyObject *tq_error;         // TQError(code, where)
PyObject *out_of_memory;    // torch's

void check(tq_status st, const char *where) {
  if (st == TQ_OK) return;
  PyObject *e = tq_error ? PyObject_CallFunction(tq_error, "is", (int)st, where) : nullptr;
  if (e != nullptr) {
    PyErr_SetObject(tq_error, e);
    Py_DECREF(e);
  }
  throw Failed();
}

// ------------------------------------------------------------------ arguments
const at::Tensor &tensor(PyObject *o, const char *name) {
  if (o == Py_None) fail(PyExc_ValueError, "%s: missing", name);
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s: expected a torch tensor, got %s", name, Py_TYPE(o)->tp_name);
  return THPVariable_Unpack(o);
}

void on_gpu(const at::Tensor &t, const char *name, int64_t device) {
  if (!t.is_cuda()) fail(PyExc_ValueError, "%s: must be a GPU tensor", name);
  if (t.get_device() != device)
    fail(PyExc_ValueError, "%s: on device %d, but the current device is %d", name, (int)t.get_device(), (int)device);
}

bool half(at::ScalarType t) { return t == at::kHalf || t == at::kBFloat16; }
tq_dtype dtype_of(at::ScalarType t) { return t == at::kHalf ? TQ_F16 : TQ_BF16; }

[[noreturn]] void bad_dtype(const at::Tensor &t, const char *name, const char *want) {
  fail(PyExc_TypeError, "%s: dtype %s, expected %s", name, c10::toString(t.scalar_type()), want);
}

// address of a contiguous tensor of one type and shape
void *plain(PyObject *o, const char *name, at::ScalarType type, at::IntArrayRef shape, int64_t device) {
  const at::Tensor &t = tensor(o, name);
  on_gpu(t, name, device);
  if (t.scalar_type() != type) bad_dtype(t, name, c10::toString(type));
  if (t.sizes() != shape) {
    std::string want = "(";
    for (size_t i = 0; i < shape.size(); i++) want += (i ? ", " : "") + std::to_string(shape[i]);
    fail(PyExc_ValueError, "%s: shape %s, expected %s)", name, shape_of(t).c_str(), want.c_str());
  }
  if (!t.is_contiguous()) fail(PyExc_ValueError, "%s: must be contiguous", name);
  return t.data_ptr();
}
void *plain_or_null(PyObject *o, const char *name, at::ScalarType type, at::IntArrayRef shape, int64_t device) {
  return o == Py_None ? nullptr : plain(o, name, type, shape, device);
}

// a new tensor's memory from torch's allocator, without the dispatcher's way there
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, int64_t device) {
  return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, (at::DeviceIndex)device), std::nullopt);
}

// rows [tokens, heads, head_dim] (tokens, heads: -1 for any number)
const at::Tensor &rows(PyObject *o, const char *name, int64_t device, int64_t tokens, int64_t heads, int64_t head_dim,
                       tq_head_rows &out) {
  const at::Tensor &t = tensor(o, name);
  on_gpu(t, name, device);
  if (!half(t.scalar_type())) bad_dtype(t, name, "Half or BFloat16");
  if (t.dim() != 3 || (tokens >= 0 && t.size(0) != tokens) || (heads >= 0 && t.size(1) != heads) || t.size(2) != head_dim) {
    const std::string n = tokens < 0 ? "tokens" : std::to_string(tokens), h = heads < 0 ? "heads" : std::to_string(heads);
    fail(PyExc_ValueError, "%s: shape %s, expected [%s, %s, %d]", name, shape_of(t).c_str(), n.c_str(), h.c_str(), (int)head_dim);
  }
  const int64_t ts = t.size(0) > 1 ? t.stride(0) : 0, hs = t.size(1) > 1 ? t.stride(1) : 0;
  out.data = t.data_ptr();
  if (t.stride(2) != 1 || ((ts | hs) & 7) != 0 || (reinterpret_cast<uintptr_t>(out.data) & 15) != 0)
    fail(PyExc_ValueError, "%s: rows must be contiguous and start on 16 bytes (strides %d, %d, %d); pass %s.contiguous()", name,
         (int)t.stride(0), (int)t.stride(1), (int)t.stride(2), name);
  out.token_stride = ts;
  out.head_stride = hs;
  return t;
}
void same_type(const at::Tensor &t, const char *name, at::ScalarType type) {
  if (t.scalar_type() != type) bad_dtype(t, name, c10::toString(type));
}

int64_t to_int(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Failed();
  return v;
}
int size32(int64_t v, const char *name) {
  if (v > INT32_MAX) fail(PyExc_ValueError, "%s: %lld is too large", name, (long long)v);
  return (int)v;
}
double to_double(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Failed();
  return v;
}
bool to_bool(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Failed();
  return v != 0;
}
void *to_stream(PyObject *o) {
  void *p = PyLong_AsVoidPtr(o);
  if (p == nullptr && PyErr_Occurred()) throw Failed();
  return p;
}

// ------------------------------------------------------------------ the cache
struct Cache {
  tq_kv_cache c;
  int64_t device;
  at::Tensor kept[4];    // k, v, k_scales, v_scales
};
const char *const kCapsule = "tq_kv_cache";

const Cache &cache_of(PyObject *o, int64_t device) {
  const Cache *c = static_cast<const Cache *>(PyCapsule_GetPointer(o, kCapsule));
  if (c == nullptr) throw Failed();
  if (c->device != device)
    fail(PyExc_ValueError, "cache: on device %d, but the current device is %d", (int)c->device, (int)device);
  // (a tensor's memory can be exchanged or resized under it)
  const void *const at[4] = {c->c.k, c->c.v, c->c.k_scales, c->c.v_scales};
  const int64_t places = (int64_t)c->c.pages * c->c.kv_heads * c->c.page_size;
  for (int i = 0; i < (c->c.bits == 16 ? 2 : 4); i++) {
    const at::Tensor &t = c->kept[i];
    const int64_t row = i >= 2 ? 1 : c->c.bits == 4 ? c->c.head_dim / 8 : c->c.head_dim;
    if (t.numel() != places * row || t.data_ptr() != at[i])
      fail(PyExc_ValueError, "cache: its tensors were moved or resized; make a new KVCache of them");
  }
  return *c;
}
// a row's type next to the cache's
void cache_type(const Cache &c, const at::Tensor &t, const char *name) {
  if (c.c.bits == 16) same_type(t, name, c.c.dtype == TQ_F16 ? at::kHalf : at::kBFloat16);
}

// make_cache(k, v, k_scales, v_scales): (handle, pages, page_size, kv_heads, head_dim, bits, device)
PyObject *make_cache(PyObject *const *a, Py_ssize_t) {
  const at::Tensor &k = tensor(a[0], "k");
  if (!k.is_cuda()) fail(PyExc_ValueError, "k: must be a GPU tensor");
  const at::ScalarType type = k.scalar_type();
  const int bits = half(type) ? 16 : type == at::kFloat8_e4m3fn ? 8 : type == at::kInt ? 4 : 0;
  if (bits == 0) bad_dtype(k, "k", "Half, BFloat16, Float8_e4m3fn or Int");
  if (k.dim() != 4) fail(PyExc_ValueError, "k: shape %s, expected [pages, kv_heads, page_size, row]", shape_of(k).c_str());
  Cache c = {};
  c.device = k.get_device();
  const at::IntArrayRef shape = k.sizes(), scales = shape.slice(0, 3);
  c.c.k = plain(a[0], "k", type, shape, c.device);
  c.c.v = plain(a[1], "v", type, shape, c.device);
  if (bits == 16) {
    if (a[2] != Py_None || a[3] != Py_None) fail(PyExc_ValueError, "k_scales, v_scales: a 16-bit cache has none");
  } else {
    if (a[2] == Py_None || a[3] == Py_None) fail(PyExc_ValueError, "k_scales, v_scales: a %d-bit cache needs both", bits);
    c.c.k_scales = plain(a[2], "k_scales", at::kHalf, scales, c.device);
    c.c.v_scales = plain(a[3], "v_scales", at::kHalf, scales, c.device);
  }
  const int64_t d = bits == 4 ? shape[3] * 8 : shape[3], size = shape[2];
  if (d != 64 && d != 128 && d != 256) fail(PyExc_ValueError, "k: rows of %lld values; 64, 128 or 256 are supported", (long long)d);
  if (size < 16 || size > 32768 || (size & (size - 1)) != 0)
    fail(PyExc_ValueError, "k: page size %lld; a power of two from 16 to 32768 is supported", (long long)size);
  if (shape[1] < 1 || shape[1] > 1024 || shape[0] < 1 || shape[0] > INT32_MAX || shape[0] * size > (int64_t)1 << 40)
    fail(PyExc_ValueError, "k: %lld pages of %lld heads", (long long)shape[0], (long long)shape[1]);
  c.c.pages = (int32_t)shape[0];
  c.c.page_size = (int32_t)size;
  c.c.kv_heads = (int32_t)shape[1];
  c.c.head_dim = (int32_t)d;
  c.c.bits = bits;
  c.c.dtype = type == at::kBFloat16 ? TQ_BF16 : TQ_F16;
  for (int i = 0; i < (bits == 16 ? 2 : 4); i++) c.kept[i] = THPVariable_Unpack(a[i]);
  Cache *kept = new Cache(c);
  PyObject *handle = PyCapsule_New(kept, kCapsule, [](PyObject *o) {
    delete static_cast<Cache *>(PyCapsule_GetPointer(o, kCapsule));
  });
  if (handle == nullptr) {
    delete kept;
    throw Failed();
  }
  return Py_BuildValue("Niiiiii", handle, c.c.pages, c.c.page_size, c.c.kv_heads, c.c.head_dim, bits, (int)c.device);
}

PyObject *wrap(const at::Tensor &t) { return THPVariable_Wrap(t); }
PyObject *wrap2(const at::Tensor &x, const at::Tensor &y) { return Py_BuildValue("NN", wrap(x), wrap(y)); }

const int64_t *slots_of(PyObject *o, int64_t tokens, int64_t device) {
  return static_cast<const int64_t *>(plain(o, "slots", at::kLong, {tokens}, device));
}

// append(cache, k, v, slots, device, stream)
PyObject *append(PyObject *const *a, Py_ssize_t) {
  const int64_t dev = to_int(a[4]);
  const Cache &c = cache_of(a[0], dev);
  tq_head_rows k, v;
  const at::Tensor &kt = rows(a[1], "k", dev, -1, c.c.kv_heads, c.c.head_dim, k);
  cache_type(c, kt, "k");
  const int tokens = size32(kt.size(0), "k");
  same_type(rows(a[2], "v", dev, tokens, c.c.kv_heads, c.c.head_dim, v), "v", kt.scalar_type());
  const int64_t *slots = slots_of(a[3], tokens, dev);
  if (tokens > 0) check(L.append(&c.c, &k, &v, slots, tokens, dtype_of(kt.scalar_type()), to_stream(a[5])), "tq_kv_append");
  Py_RETURN_NONE;
}

// read(cache, slots, bf16 or None, device, stream): (k, v)
PyObject *read(PyObject *const *a, Py_ssize_t) {
  const int64_t dev = to_int(a[3]);
  const Cache &c = cache_of(a[0], dev);
  const at::Tensor &st = tensor(a[1], "slots");
  if (st.dim() != 1) fail(PyExc_ValueError, "slots: shape %s, expected (tokens)", shape_of(st).c_str());
  const int tokens = size32(st.size(0), "slots");
  const int64_t *slots = slots_of(a[1], tokens, dev);
  bool bf16 = a[2] != Py_None && to_bool(a[2]);
  if (c.c.bits == 16) {
    if (a[2] != Py_None && bf16 != (c.c.dtype == TQ_BF16))
      fail(PyExc_TypeError, "bf16: the cache holds %s", c.c.dtype == TQ_BF16 ? "bfloat16" : "float16");
    bf16 = c.c.dtype == TQ_BF16;
  }
  const at::ScalarType type = bf16 ? at::kBFloat16 : at::kHalf;
  const at::Tensor k = fresh({tokens, c.c.kv_heads, c.c.head_dim}, type, dev);
  const at::Tensor v = fresh({tokens, c.c.kv_heads, c.c.head_dim}, type, dev);
  if (tokens > 0)
    check(L.read(&c.c, slots, tokens, k.data_ptr(), v.data_ptr(), bf16 ? TQ_BF16 : TQ_F16, to_stream(a[4])), "tq_kv_read");
  return wrap2(k, v);
}

// positions, table, q_weight, k_weight, eps, interleaved from a[0]
tq_norm_rope norm_rope_args(PyObject *const *a, int64_t tokens, int64_t head_dim, at::ScalarType type, int64_t dev) {
  tq_norm_rope p = {};
  p.q_weight = plain_or_null(a[2], "q_weight", type, {head_dim}, dev);
  p.k_weight = plain_or_null(a[3], "k_weight", type, {head_dim}, dev);
  p.eps = (float)to_double(a[4]);
  p.interleaved = to_bool(a[5]);
  if (a[1] == Py_None) return p;
  const at::Tensor &t = tensor(a[1], "table");
  if (t.dim() != 2) fail(PyExc_ValueError, "table: shape %s, expected [max_positions, rotary_dim]", shape_of(t).c_str());
  p.table = static_cast<const float *>(plain(a[1], "table", at::kFloat, t.sizes(), dev));
  const int64_t n = t.size(0), rot = t.size(1);
  if (rot < 1 || rot > head_dim || rot % 16 != 0 || n < 1 || n > INT32_MAX)
    fail(PyExc_ValueError, "table: %lld positions of %lld values; a multiple of 16 up to head_dim %d", (long long)n,
         (long long)rot, (int)head_dim);
  if (a[0] == Py_None) fail(PyExc_ValueError, "positions: a rotation needs them");
  p.positions = static_cast<const int32_t *>(plain(a[0], "positions", at::kInt, {tokens}, dev));
  p.rotary_dim = (int32_t)rot;
  p.max_positions = (int32_t)n;
  return p;
}

// norm_rope(q, k, positions, table, q_weight, k_weight, eps, interleaved, device, stream): (q, k)
PyObject *norm_rope(PyObject *const *a, Py_ssize_t) {
  const int64_t dev = to_int(a[8]);
  const at::Tensor &first = tensor(a[0], "q");
  const int64_t d = first.dim() == 3 ? first.size(2) : 0;
  on_gpu(first, "q", dev);
  if (d != 64 && d != 128 && d != 256)
    fail(PyExc_ValueError, "q: shape %s; [tokens, heads, head_dim] with head_dim 64, 128 or 256", shape_of(first).c_str());
  tq_head_rows q, k;
  const at::Tensor &qt = rows(a[0], "q", dev, -1, -1, d, q);
  const at::ScalarType type = qt.scalar_type();
  const int tokens = size32(qt.size(0), "q"), hq = size32(qt.size(1), "q");
  const at::Tensor &kt = rows(a[1], "k", dev, tokens, -1, d, k);
  same_type(kt, "k", type);
  const int hkv = size32(kt.size(1), "k");
  const tq_norm_rope p = norm_rope_args(a + 2, tokens, d, type, dev);
  const at::Tensor qo = fresh({tokens, hq, d}, qt.scalar_type(), dev), ko = fresh({tokens, hkv, d}, qt.scalar_type(), dev);
  if (tokens > 0)
    check(L.norm_rope(&p, &q, &k, tokens, hq, hkv, (int)d, dtype_of(type), qo.data_ptr(), ko.data_ptr(), to_stream(a[9])),
          "tq_qk_norm_rope");
  return wrap2(qo, ko);
}

// norm_rope_append(cache, q, k, v, slots, positions, table, q_weight, k_weight, eps, interleaved, return_k, device,
//                  stream): q or (q, k)
PyObject *norm_rope_append(PyObject *const *a, Py_ssize_t) {
  const int64_t dev = to_int(a[12]);
  const Cache &c = cache_of(a[0], dev);
  const int64_t d = c.c.head_dim, hkv = c.c.kv_heads;
  tq_head_rows q, k, v;
  const at::Tensor &qt = rows(a[1], "q", dev, -1, -1, d, q);
  cache_type(c, qt, "q");
  const at::ScalarType type = qt.scalar_type();
  const int tokens = size32(qt.size(0), "q"), hq = size32(qt.size(1), "q");
  same_type(rows(a[2], "k", dev, tokens, hkv, d, k), "k", type);
  same_type(rows(a[3], "v", dev, tokens, hkv, d, v), "v", type);
  const int64_t *slots = slots_of(a[4], tokens, dev);
  const tq_norm_rope p = norm_rope_args(a + 5, tokens, d, type, dev);
  const bool return_k = to_bool(a[11]);
  const at::Tensor qo = fresh({tokens, hq, d}, qt.scalar_type(), dev);
  at::Tensor ko;
  if (return_k) ko = fresh({tokens, hkv, d}, qt.scalar_type(), dev);
  if (tokens > 0)
    check(L.norm_rope_append(&p, &c.c, &q, &k, &v, slots, tokens, hq, dtype_of(type), qo.data_ptr(),
                             return_k ? ko.data_ptr() : nullptr, to_stream(a[13])),
          "tq_qk_norm_rope_append");
  return return_k ? wrap2(qo, ko) : wrap(qo);
}

// page_table [batch, max_pages] of strided rows: its address, and max_pages
const int32_t *page_table_of(PyObject *o, const char *name, int64_t batch, int64_t dev, int &pages, int64_t &stride) {
  const at::Tensor &t = tensor(o, name);
  on_gpu(t, name, dev);
  if (t.scalar_type() != at::kInt) bad_dtype(t, name, "Int");
  if (t.dim() != 2 || t.size(0) != batch || t.size(1) == 0)
    fail(PyExc_ValueError, "%s: shape %s, expected [%d, max_pages]", name, shape_of(t).c_str(), (int)batch);
  pages = size32(t.size(1), name);
  if ((t.stride(1) != 1 && pages > 1) || (t.stride(0) < pages && batch > 1)) fail(PyExc_ValueError, "%s: rows must be contiguous", name);
  stride = t.stride(0);
  return static_cast<const int32_t *>(t.data_ptr());
}

// scale or None, window, softcap, slopes or None: the scores of a call
tq_scores scores_of(PyObject *scale, PyObject *window, PyObject *softcap, PyObject *slopes, int64_t hq, int64_t d, int64_t dev) {
  tq_scores s = {};
  s.scale = scale == Py_None ? (float)(1.0 / std::sqrt((double)d)) : (float)to_double(scale);
  const int64_t win = window == nullptr ? 0 : to_int(window);
  if (win < 0) fail(PyExc_ValueError, "window %lld: must not be negative", (long long)win);
  s.window = win > INT32_MAX ? 0 : (int32_t)win;      // (past any length: none)
  s.softcap = (float)to_double(softcap);
  if (!(s.softcap >= 0.0f) || std::isinf(s.softcap)) fail(PyExc_ValueError, "softcap: must be finite and not negative (0: none)");
  s.slopes = static_cast<const float *>(plain_or_null(slopes, "slopes", at::kFloat, {hq}, dev));
  return s;
}

// query rows next to a cache: tokens (or -1), and their heads, a multiple of the cache's
const at::Tensor &queries(PyObject *o, const Cache &c, int64_t dev, tq_head_rows &q) {
  const at::Tensor &t = rows(o, "q", dev, -1, -1, c.c.head_dim, q);
  cache_type(c, t, "q");
  if (t.size(1) == 0 || t.size(1) % c.c.kv_heads != 0)
    fail(PyExc_ValueError, "q: %d heads are no multiple of the cache's %d", (int)t.size(1), c.c.kv_heads);
  return t;
}

// attend(cache, q, page_table, lengths, scale or None, window, return_lse, softcap, slopes or None, device, stream):
// out or (out, lse)
PyObject *attend(PyObject *const *a, Py_ssize_t) {
  const int64_t dev = to_int(a[9]);
  const Cache &c = cache_of(a[0], dev);
  tq_head_rows q;
  const at::Tensor &qt = queries(a[1], c, dev, q);
  const int batch = size32(qt.size(0), "q"), hq = size32(qt.size(1), "q");
  int pages;
  int64_t stride;
  const int32_t *table = page_table_of(a[2], "page_table", batch, dev, pages, stride);
  const int32_t *lengths = static_cast<const int32_t *>(plain(a[3], "lengths", at::kInt, {batch}, dev));
  const tq_scores s = scores_of(a[4], a[5], a[7], a[8], hq, c.c.head_dim, dev);
  const bool return_lse = to_bool(a[6]);
  const size_t bytes = L.scratch_bytes(&c.c, batch, hq, pages, s.window);
  const at::Tensor out = fresh({batch, hq, c.c.head_dim}, qt.scalar_type(), dev);
  at::Tensor lse, scratch;
  if (return_lse) lse = fresh({batch, hq}, at::kFloat, dev);
  if (bytes > 0) scratch = fresh({(int64_t)(bytes / 4)}, at::kFloat, dev);
  if (batch > 0)
    check(L.attend_scored(&c.c, &q, dtype_of(qt.scalar_type()), batch, hq, table, stride, pages, lengths, &s, out.data_ptr(),
                          return_lse ? static_cast<float *>(lse.data_ptr()) : nullptr, bytes > 0 ? scratch.data_ptr() : nullptr,
                          to_stream(a[10])),
          "tq_paged_attention");
  return return_lse ? wrap2(out, lse) : wrap(out);
}

// prefix(cache, q, members, prefix_table, prefix_lengths, page_table, lengths, scale or None, softcap, slopes or None,
//        exact, return_lse, device, stream): out or (out, lse)
PyObject *prefix(PyObject *const *a, Py_ssize_t) {
  const int64_t dev = to_int(a[12]);
  const Cache &c = cache_of(a[0], dev);
  tq_head_rows q;
  const at::Tensor &qt = queries(a[1], c, dev, q);
  const int batch = size32(qt.size(0), "q"), hq = size32(qt.size(1), "q");
  const at::Tensor &mt = tensor(a[2], "members");
  if (mt.dim() != 1 || mt.size(0) < 2) fail(PyExc_ValueError, "members: shape %s, expected (groups + 1) with at least 1 group", shape_of(mt).c_str());
  const int groups = size32(mt.size(0) - 1, "members");
  const int32_t *members = static_cast<const int32_t *>(plain(a[2], "members", at::kInt, {groups + 1}, dev));
  int prefix_pages, pages;
  int64_t prefix_stride, stride;
  const int32_t *prefix_table = page_table_of(a[3], "prefix_table", groups, dev, prefix_pages, prefix_stride);
  const int32_t *prefix_lengths = static_cast<const int32_t *>(plain(a[4], "prefix_lengths", at::kInt, {groups}, dev));
  const int32_t *table = page_table_of(a[5], "page_table", batch, dev, pages, stride);
  const int32_t *lengths = static_cast<const int32_t *>(plain(a[6], "lengths", at::kInt, {batch}, dev));
  tq_scores s = scores_of(a[7], nullptr, a[8], a[9], hq, c.c.head_dim, dev);
  s.exact = to_bool(a[10]);
  const bool return_lse = to_bool(a[11]);
  const size_t bytes = L.prefix_bytes(&c.c, batch, hq, groups, prefix_pages, pages);
  const at::Tensor out = fresh({batch, hq, c.c.head_dim}, qt.scalar_type(), dev);
  at::Tensor lse, scratch;
  if (return_lse) lse = fresh({batch, hq}, at::kFloat, dev);
  if (bytes > 0) scratch = fresh({(int64_t)((bytes + 3) / 4)}, at::kFloat, dev);
  if (batch > 0)
    check(L.prefix(&c.c, &q, dtype_of(qt.scalar_type()), batch, hq, groups, members, prefix_table, prefix_stride, prefix_pages,
                   prefix_lengths, table, stride, pages, lengths, &s, out.data_ptr(),
                   return_lse ? static_cast<float *>(lse.data_ptr()) : nullptr, bytes > 0 ? scratch.data_ptr() : nullptr,
                   to_stream(a[13])),
          "tq_shared_prefix_attention");
  return return_lse ? wrap2(out, lse) : wrap(out);
}

// prompt(cache, q, starts, page_table, lengths, scale or None, window, prefix or None, first or None, softcap,
//        slopes or None, exact, return_lse, device, stream): out or (out, lse)
PyObject *prompt(PyObject *const *a, Py_ssize_t) {
  const int64_t dev = to_int(a[13]);
  const Cache &c = cache_of(a[0], dev);
  tq_head_rows q;
  const at::Tensor &qt = queries(a[1], c, dev, q);
  const int tokens = size32(qt.size(0), "q"), hq = size32(qt.size(1), "q");
  const at::Tensor &st = tensor(a[2], "starts");
  if (st.dim() != 1 || st.size(0) < 2) fail(PyExc_ValueError, "starts: shape %s, expected (batch + 1) with a batch of at least 1", shape_of(st).c_str());
  const int batch = size32(st.size(0) - 1, "starts");
  const int32_t *starts = static_cast<const int32_t *>(plain(a[2], "starts", at::kInt, {batch + 1}, dev));
  int pages;
  int64_t stride;
  const int32_t *table = page_table_of(a[3], "page_table", batch, dev, pages, stride);
  const int32_t *lengths = static_cast<const int32_t *>(plain(a[4], "lengths", at::kInt, {batch}, dev));
  const int32_t *prefix = static_cast<const int32_t *>(plain_or_null(a[7], "prefix", at::kInt, {batch}, dev));
  const int32_t *first = static_cast<const int32_t *>(plain_or_null(a[8], "first", at::kInt, {tokens}, dev));
  tq_scores s = scores_of(a[5], a[6], a[9], a[10], hq, c.c.head_dim, dev);
  s.exact = to_bool(a[11]);
  const bool return_lse = to_bool(a[12]);
  const size_t bytes = L.prompt_bytes(&c.c, tokens, batch, hq, pages, s.window);
  const at::Tensor out = fresh({tokens, hq, c.c.head_dim}, qt.scalar_type(), dev);
  at::Tensor lse, scratch;
  if (return_lse) lse = fresh({tokens, hq}, at::kFloat, dev);
  if (bytes > 0) scratch = fresh({(int64_t)(bytes / 4)}, at::kFloat, dev);
  if (tokens > 0)
    check(L.prompt(&c.c, &q, dtype_of(qt.scalar_type()), tokens, batch, hq, starts, table, stride, pages, lengths, prefix, first,
                   &s, out.data_ptr(), return_lse ? static_cast<float *>(lse.data_ptr()) : nullptr,
                   bytes > 0 ? scratch.data_ptr() : nullptr, to_stream(a[14])),
          "tq_prompt_attention");
  return return_lse ? wrap2(out, lse) : wrap(out);
}

// rows [tokens, n] of one type, the last axis contiguous: address and stride
const void *wide_rows(PyObject *o, const char *name, at::ScalarType type, int64_t tokens, int64_t n, int64_t dev, int64_t &stride) {
  const at::Tensor &t = tensor(o, name);
  on_gpu(t, name, dev);
  if (t.scalar_type() != type) bad_dtype(t, name, c10::toString(type));
  if (t.dim() != 2 || t.size(0) != tokens || t.size(1) != n)
    fail(PyExc_ValueError, "%s: shape %s, expected [%lld, %lld]", name, shape_of(t).c_str(), (long long)tokens, (long long)n);
  stride = tokens > 1 ? t.stride(0) : 0;
  if (t.stride(1) != 1 || (stride & 7) != 0 || (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15) != 0)
    fail(PyExc_ValueError, "%s: rows must be contiguous and start on 16 bytes (strides %lld, %lld); pass %s.contiguous()", name,
         (long long)t.stride(0), (long long)t.stride(1), name);
  return t.data_ptr();
}

// add_norm(x, residual or None, weight or None, post_weight or None, gate or None, scale, eps, return_sum, device, stream):
// sum, normed or (sum, normed)
PyObject *add_norm(PyObject *const *a, Py_ssize_t) {
  const int64_t dev = to_int(a[8]);
  const at::Tensor &xt = tensor(a[0], "x");
  on_gpu(xt, "x", dev);
  const at::ScalarType type = xt.scalar_type();
  if (!half(type)) bad_dtype(xt, "x", "Half or BFloat16");
  if (xt.dim() != 2) fail(PyExc_ValueError, "x: shape %s, expected [tokens, n]", shape_of(xt).c_str());
  const int64_t n = xt.size(1);
  const int tokens = size32(xt.size(0), "x");
  if (n < 8 || n > 32768 || n % 8 != 0) fail(PyExc_ValueError, "x: rows of %lld values; a multiple of 8 up to 32768", (long long)n);
  tq_residual_norm p = {};
  p.x = wide_rows(a[0], "x", type, tokens, n, dev, p.x_stride);
  if (a[1] != Py_None) p.residual = wide_rows(a[1], "residual", type, tokens, n, dev, p.residual_stride);
  p.weight = plain_or_null(a[2], "weight", type, {n}, dev);
  p.post_weight = plain_or_null(a[3], "post_weight", type, {n}, dev);
  if (a[4] != Py_None) {
    if (tensor(a[4], "gate").dim() == 1) p.gate = plain(a[4], "gate", type, {n}, dev);
    else p.gate = wide_rows(a[4], "gate", type, tokens, n, dev, p.gate_stride);
  }
  p.scale = (float)to_double(a[5]);
  p.eps = (float)to_double(a[6]);
  const bool return_sum = to_bool(a[7]);
  if (!return_sum && p.weight == nullptr) fail(PyExc_ValueError, "weight: missing, and the sum is not asked for");
  at::Tensor sum, normed;
  if (return_sum) sum = fresh({tokens, n}, type, dev);
  if (p.weight != nullptr) normed = fresh({tokens, n}, type, dev);
  if (tokens > 0)
    check(L.add_norm(&p, tokens, (int)n, dtype_of(type), return_sum ? sum.data_ptr() : nullptr,
                     p.weight != nullptr ? normed.data_ptr() : nullptr, to_stream(a[9])),
          "tq_add_rms_norm");
  return p.weight == nullptr ? wrap(sum) : return_sum ? wrap2(sum, normed) : wrap(normed);
}

// bind(TQError, torch.OutOfMemoryError, addresses of the entry points, in the order of Entries)
PyObject *bind(PyObject *const *a, Py_ssize_t) {
  Py_INCREF(a[0]);
  Py_XSETREF(tq_error, a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(out_of_memory, a[1]);
  ++a;
  L.norm_rope = reinterpret_cast<decltype(L.norm_rope)>(to_stream(a[1]));
  L.append = reinterpret_cast<decltype(L.append)>(to_stream(a[2]));
  L.norm_rope_append = reinterpret_cast<decltype(L.norm_rope_append)>(to_stream(a[3]));
  L.read = reinterpret_cast<decltype(L.read)>(to_stream(a[4]));
  L.scratch_bytes = reinterpret_cast<decltype(L.scratch_bytes)>(to_stream(a[5]));
  L.prompt_bytes = reinterpret_cast<decltype(L.prompt_bytes)>(to_stream(a[6]));
  L.prompt = reinterpret_cast<decltype(L.prompt)>(to_stream(a[7]));
  L.attend_scored = reinterpret_cast<decltype(L.attend_scored)>(to_stream(a[8]));
  L.prefix_bytes = reinterpret_cast<decltype(L.prefix_bytes)>(to_stream(a[9]));
  L.prefix = reinterpret_cast<decltype(L.prefix)>(to_stream(a[10]));
  L.add_norm = reinterpret_cast<decltype(L.add_norm)>(to_stream(a[11]));
  Py_RETURN_NONE;
}

// no C++ exception leaves through the interpreter
template <PyObject *(*F)(PyObject *const *, Py_ssize_t), int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "expected %d arguments, got %d", N, (int)n);
    return nullptr;
  }
  try {
    return F(args, n);
  } catch (const Failed &) {
    return nullptr;
  } catch (const c10::OutOfMemoryError &e) {
    PyErr_SetString(out_of_memory != nullptr ? out_of_memory : PyExc_MemoryError, e.what_without_backtrace());
    return nullptr;
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    return nullptr;
  }
}

#define TQ_METHOD(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(entry<name, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TQ_METHOD(bind, 13), TQ_METHOD(make_cache, 4), TQ_METHOD(append, 6), TQ_METHOD(read, 5),
                         TQ_METHOD(norm_rope, 10), TQ_METHOD(norm_rope_append, 14), TQ_METHOD(attend, 11), TQ_METHOD(prompt, 15), TQ_METHOD(prefix, 14), TQ_METHOD(add_norm, 10),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tqtorch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tqtorch() { return PyModule_Create(&module); }
