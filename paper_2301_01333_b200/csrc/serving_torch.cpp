// The torch side of the served attention block's operators: checks of tensors, outputs and workspaces from torch's allocator,
// the current stream, and the call of the C entry point (include/gc.h).  A served step makes hundreds of these calls, each of
// which may be a few microseconds on the GPU; marshalling them in Python took three times as long as the launch itself (20
// against 6 us a call).  serving.py is the public face; nothing here computes.
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cstdarg>
#include <cstdio>
#include <stdexcept>
#include <string>

#include "../../include/gc.h"

namespace {

struct TypeFault : std::runtime_error {
  using std::runtime_error::runtime_error;
};
struct GcFault {
  gc_status_t status;
};

PyObject* g_gc_error = nullptr;                // binding.GcError, handed over by serving.py

[[noreturn]] void refuse(const char* fmt, ...) {
  char msg[384];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  throw std::invalid_argument(msg);
}

std::string shape_of(const at::Tensor& t) {
  std::string s = std::string(c10::toString(t.scalar_type())) + " [";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + "] on " + t.device().str();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw TypeFault(std::string(name) + " must be a torch.Tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && at::GradMode::is_enabled())
    refuse("%s requires a gradient, which this call does not give: detach it, or call under torch.no_grad()", name);
  return t;
}
bool given(PyObject* o) { return o != Py_None; }

int on_cuda(const at::Tensor& t, const char* name) {
  if (!t.is_cuda()) refuse("%s must be on a CUDA device, not %s", name, t.device().str().c_str());
  return t.get_device();
}

int32_t row_type(const at::Tensor& t, const char* name) {
  if (t.scalar_type() == at::kFloat) return GC_F32;
  if (t.scalar_type() == at::kBFloat16) return GC_BF16;
  throw TypeFault(std::string(name) + " must be float32 or bfloat16, not " + c10::toString(t.scalar_type()));
}

// rows of heads [n0, n1, n2], the last dimension contiguous; `output`: no two elements may share memory
gc_heads_t heads(const at::Tensor& t, const char* name, int64_t n0, int64_t n1, int64_t n2, at::ScalarType type, const at::Device& device,
                 bool output) {
  if (t.dim() != 3 || t.size(0) != n0 || t.size(1) != n1 || t.size(2) != n2 || t.scalar_type() != type || t.device() != device)
    refuse("%s must be %s [%lld, %lld, %lld] on %s, not %s", name, c10::toString(type), (long long)n0, (long long)n1, (long long)n2,
           device.str().c_str(), shape_of(t).c_str());
  if (n2 > 1 && t.stride(2) != 1 && t.numel()) refuse("%s: the last dimension must be contiguous", name);
  const int64_t s0 = n0 > 1 ? t.stride(0) : 0, s1 = n1 > 1 ? t.stride(1) : 0;
  if (output && ((n0 > 1 && s0 == 0) || (n1 > 1 && s1 == 0))) refuse("%s: an output cannot be an expanded tensor", name);
  return gc_heads_t{t.data_ptr(), s0, s1};
}

const void* vec(const at::Tensor& t, const char* name, int64_t n, at::ScalarType type, const at::Device& device) {
  if (t.scalar_type() != type || t.dim() != 1 || t.size(0) != n || t.device() != device || (n > 1 && t.stride(0) != 1))
    refuse("%s must be a contiguous %s vector of %lld on %s, not %s", name, c10::toString(type), (long long)n, device.str().c_str(),
           shape_of(t).c_str());
  return t.data_ptr();
}

at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const at::Device& device) {
  return at::detail::empty_cuda(sizes, type, device, std::nullopt);
}

void* stream_of(int device) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream(); }

// Tells autograd that a tensor the caller handed over has been written to (one it keeps for a backward pass is then missed there).
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void written(PyObject* tensors) {
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(tensors); ++i) written(THPVariable_Unpack(PyTuple_GET_ITEM(tensors, i)));
}

void check(gc_status_t st) {
  if (st != GC_OK) throw GcFault{st};
}

double number(PyObject* o) {
  const double d = PyFloat_AsDouble(o);
  if (d == -1.0 && PyErr_Occurred()) throw TypeFault("");
  return d;
}
int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw TypeFault("");
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw TypeFault("");
  return v != 0;
}
int32_t small(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) refuse("%s is out of range", name);
  return static_cast<int32_t>(v);
}
// The descriptor of a cache, whose pointers must still be those of its tensors (set_, resize_ or an assigned .data move them).
const gc_kv4_cache_t* cache_at(PyObject* at, PyObject* tensors) {
  const gc_kv4_cache_t* c = static_cast<const gc_kv4_cache_t*>(PyLong_AsVoidPtr(at));
  const void* held[4] = {c->k_codes, c->k_params, c->v_codes, c->v_params};
  for (int i = 0; i < 4; ++i)
    if (THPVariable_Unpack(PyTuple_GET_ITEM(tensors, i)).data_ptr() != held[i])
      refuse("a tensor of the cache has moved since the KV4Cache was made: make another one over the tensors as they are now");
  return c;
}
at::Device device_of(const gc_kv4_cache_t* c) { return at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(c->cuda_device)); }

// Runs `f`, turning what it throws into Python exceptions.
template <typename F>
PyObject* guarded(Py_ssize_t nargs, Py_ssize_t want, F f) {
  if (nargs != want) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, nargs);
    return nullptr;
  }
  try {
    return f();
  } catch (const GcFault& e) {
    THPObjectPtr x(PyObject_CallFunction(g_gc_error, "is", static_cast<int>(e.status), gc_last_error()));
    if (x) PyErr_SetObject(g_gc_error, x.get());
  } catch (const TypeFault& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const std::invalid_argument& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const c10::OutOfMemoryError& e) {
    THPObjectPtr torch(PyImport_ImportModule("torch")), type(torch ? PyObject_GetAttrString(torch.get(), "OutOfMemoryError") : nullptr);
    PyErr_SetString(type ? type.get() : PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// (q, k, positions, inv_freq, q_weight, k_weight, norm, eps, interleaved, attention_factor, q_out, k_out)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &pos = tensor(a[2], "positions"), &inv = tensor(a[3], "inv_freq");
    if (q.dim() != 3 || k.dim() != 3) refuse("q and k must be [tokens, heads, head_dim]");
    const at::Device device = q.device();
    const at::ScalarType type = q.scalar_type();
    gc_qk_norm_rope_t d = {};
    d.dtype = row_type(q, "q");
    d.cuda_device = on_cuda(q, "q");
    d.tokens = q.size(0);
    d.q_heads = small(q.size(1), "q");
    d.k_heads = small(k.size(1), "k");
    d.head_dim = small(q.size(2), "head_dim");
    if (inv.dim() != 1) refuse("inv_freq must be a vector");
    d.rot_dim = small(2 * inv.size(0), "inv_freq");
    d.norm = truth(a[6]);
    d.eps = static_cast<float>(number(a[7]));
    d.interleaved = truth(a[8]);
    d.attention_factor = static_cast<float>(number(a[9]));
    d.q = heads(q, "q", d.tokens, d.q_heads, d.head_dim, type, device, false);
    d.k = heads(k, "k", d.tokens, d.k_heads, d.head_dim, type, device, false);
    d.positions = static_cast<const int64_t*>(vec(pos, "positions", d.tokens, at::kLong, device));
    d.inv_freq = static_cast<const float*>(vec(inv, "inv_freq", d.rot_dim / 2, at::kFloat, device));
    if (given(a[4])) d.q_weight = vec(tensor(a[4], "q_weight"), "q_weight", d.head_dim, type, device);
    if (given(a[5])) d.k_weight = vec(tensor(a[5], "k_weight"), "k_weight", d.head_dim, type, device);
    const at::Tensor qo = given(a[10]) ? tensor(a[10], "q_out") : empty(q.sizes(), type, device);
    const at::Tensor ko = given(a[11]) ? tensor(a[11], "k_out") : empty(k.sizes(), type, device);
    d.q_out = heads(qo, "q_out", d.tokens, d.q_heads, d.head_dim, type, device, true);
    d.k_out = heads(ko, "k_out", d.tokens, d.k_heads, d.head_dim, type, device, true);
    check(gc_qk_norm_rope(stream_of(d.cuda_device), &d));
    if (given(a[10])) written(qo);
    if (given(a[11])) written(ko);
    THPObjectPtr x(THPVariable_Wrap(qo)), y(THPVariable_Wrap(ko));
    return x && y ? PyTuple_Pack(2, x.get(), y.get()) : nullptr;
  });
}

// (cache, k, v, slots, the cache's four tensors)
PyObject* kv4_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    const gc_kv4_cache_t* c = cache_at(a[0], a[4]);
    const at::Tensor &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &slots = tensor(a[3], "slots");
    const at::Device device = device_of(c);
    const int32_t type = row_type(k, "k");
    const int64_t tokens = slots.dim() == 1 ? slots.size(0) : -1;
    const int64_t* s = static_cast<const int64_t*>(vec(slots, "slots", tokens, at::kLong, device));
    const gc_heads_t kh = heads(k, "k", tokens, c->kv_heads, c->head_dim, k.scalar_type(), device, false);
    const gc_heads_t vh = heads(v, "v", tokens, c->kv_heads, c->head_dim, k.scalar_type(), device, false);
    check(gc_kv4_append(stream_of(c->cuda_device), c, type, tokens, &kh, &vh, s));
    written(a[4]);
    Py_RETURN_NONE;
  });
}

// (cache, slots, k_out, v_out, the cache's four tensors)
PyObject* kv4_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    const gc_kv4_cache_t* c = cache_at(a[0], a[4]);
    const at::Tensor &slots = tensor(a[1], "slots"), &k = tensor(a[2], "k_out"), &v = tensor(a[3], "v_out");
    const at::Device device = device_of(c);
    const int32_t type = row_type(k, "k_out");
    const int64_t tokens = slots.dim() == 1 ? slots.size(0) : -1;
    const int64_t* s = static_cast<const int64_t*>(vec(slots, "slots", tokens, at::kLong, device));
    const gc_heads_t kh = heads(k, "k_out", tokens, c->kv_heads, c->head_dim, k.scalar_type(), device, true);
    const gc_heads_t vh = heads(v, "v_out", tokens, c->kv_heads, c->head_dim, k.scalar_type(), device, true);
    check(gc_kv4_read(stream_of(c->cuda_device), c, type, tokens, &kh, &vh, s));
    written(k);
    written(v);
    Py_RETURN_NONE;
  });
}

// (cache, q, block_table, lengths, scale, max_length, out, the cache's four tensors)
PyObject* kv4_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const gc_kv4_cache_t* c = cache_at(a[0], a[7]);
    const at::Tensor &q = tensor(a[1], "q"), &table = tensor(a[2], "block_table"), &lengths = tensor(a[3], "lengths");
    const at::Device device = device_of(c);
    if (q.dim() != 4 || q.scalar_type() != at::kBFloat16 || q.device() != device || q.size(3) != c->head_dim || q.stride(3) != 1)
      refuse("q must be bfloat16 [batch, queries, q_heads, %d] on %s, its last dimension contiguous, not %s", c->head_dim,
             device.str().c_str(), shape_of(q).c_str());
    if (table.dim() != 2 || table.scalar_type() != at::kInt || table.size(0) != q.size(0) || table.device() != device ||
        (table.size(1) > 1 && table.stride(1) != 1))
      refuse("block_table must be int32 [%lld, width] on %s, its rows contiguous, not %s", (long long)q.size(0), device.str().c_str(),
             shape_of(table).c_str());
    const at::Tensor out = given(a[6]) ? tensor(a[6], "out") : empty(q.sizes(), at::kBFloat16, device);
    if (given(a[6])) {
      if (out.sizes() != q.sizes() || out.scalar_type() != at::kBFloat16 || out.device() != device || out.stride(3) != 1)
        refuse("out must be like q, its last dimension contiguous");
      for (int i = 0; i < 3; ++i)
        if (out.size(i) > 1 && out.stride(i) == 0) refuse("out: an output cannot be an expanded tensor");
    }
    auto stride = [](const at::Tensor& t, int i) { return t.size(i) > 1 ? t.stride(i) : 0; };
    gc_attention_kv4_t d = {};
    d.batch = small(q.size(0), "batch");
    d.queries = small(q.size(1), "queries");
    d.q_heads = small(q.size(2), "q_heads");
    d.table_width = small(table.size(1), "block_table");
    d.table_stride = stride(table, 0);
    const int64_t bound = static_cast<int64_t>(d.table_width) * c->page_size;
    d.max_length = small(given(a[5]) ? whole(a[5]) : bound, "max_length");
    d.scale = given(a[4]) ? static_cast<float>(number(a[4])) : 1.0f / std::sqrt(static_cast<float>(c->head_dim));
    d.q = q.data_ptr();
    d.q_batch_stride = stride(q, 0), d.q_query_stride = stride(q, 1), d.q_head_stride = stride(q, 2);
    d.out = out.data_ptr();
    d.o_batch_stride = stride(out, 0), d.o_query_stride = stride(out, 1), d.o_head_stride = stride(out, 2);
    d.block_table = static_cast<const int32_t*>(table.data_ptr());
    d.lengths = static_cast<const int32_t*>(vec(lengths, "lengths", d.batch, at::kInt, device));
    size_t need = 0;
    check(gc_attention_kv4_workspace_bytes(c, &d, &need));
    // from torch's allocator, so that calls on several streams or in several captured graphs never share it
    at::Tensor ws;
    if (need) ws = empty({static_cast<int64_t>(need)}, at::kByte, device);
    check(gc_attention_kv4(stream_of(c->cuda_device), c, &d, need ? ws.data_ptr() : nullptr, need));
    if (given(a[6])) written(out);
    return THPVariable_Wrap(out);
  });
}

// (q, k, v, cu_q, cu_k, causal, scale, out, status)
PyObject* attention_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &cu_q = tensor(a[3], "cu_q");
    const at::Tensor& cu_k = given(a[4]) ? tensor(a[4], "cu_k") : cu_q;
    const at::Device device = q.device();
    if (q.dim() != 3 || k.dim() != 3) refuse("q, k and v must be [tokens, heads, head_dim]");
    if (cu_q.dim() != 1 || cu_q.size(0) < 1) refuse("cu_q must be a vector of batch + 1 offsets");
    gc_attention_prompt_t d = {};
    d.cuda_device = on_cuda(q, "q");
    d.batch = small(cu_q.size(0) - 1, "cu_q");
    d.q_tokens = q.size(0);
    d.k_tokens = k.size(0);
    d.q_heads = small(q.size(1), "q");
    d.kv_heads = small(k.size(1), "k");
    d.head_dim = small(q.size(2), "head_dim");
    d.causal = truth(a[5]);
    d.scale = given(a[6]) ? static_cast<float>(number(a[6])) : 1.0f / std::sqrt(static_cast<float>(d.head_dim));
    d.q = heads(q, "q", d.q_tokens, d.q_heads, d.head_dim, at::kBFloat16, device, false);
    d.k = heads(k, "k", d.k_tokens, d.kv_heads, d.head_dim, at::kBFloat16, device, false);
    d.v = heads(v, "v", d.k_tokens, d.kv_heads, d.head_dim, at::kBFloat16, device, false);
    d.cu_q = static_cast<const int32_t*>(vec(cu_q, "cu_q", d.batch + 1LL, at::kInt, device));
    d.cu_k = static_cast<const int32_t*>(vec(cu_k, "cu_k", d.batch + 1LL, at::kInt, device));
    const at::Tensor& out = tensor(a[7], "out");
    d.out = heads(out, "out", d.q_tokens, d.q_heads, d.head_dim, at::kBFloat16, device, true);
    if (given(a[8])) d.status = const_cast<uint32_t*>(static_cast<const uint32_t*>(vec(tensor(a[8], "status"), "status", 1, at::kInt, device)));
    check(gc_attention_prompt(stream_of(d.cuda_device), &d));
    written(out);
    return Py_NewRef(a[7]);
  });
}

PyObject* set_error_class(PyObject*, PyObject* cls) {
  Py_XSETREF(g_gc_error, Py_NewRef(cls));
  Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(qk_norm_rope), FAST(kv4_append), FAST(kv4_read), FAST(kv4_attend), FAST(attention_prompt),
                         {"set_error_class", set_error_class, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving(void) {
  PyObject* m = PyModule_Create(&module);
  // which torch and Python this was compiled for: the build looks for the text and compiles again under others
  if (m && PyModule_AddStringConstant(m, "abi", SERVING_ABI)) Py_CLEAR(m);
  return m;
}
