// Native binding of the serving operators: checks the tensors of a call and forwards their addresses to libtq.
//
// A decode step calls these operators a few times per layer with kernels of a few microseconds, and marshalling the same
// arguments through ctypes took longer than the kernels (17 us per call; 3 us here).  The library's functions come in as
// addresses (attach), so that this module and tq.py use one and the same libtq.  Refusals and errors are raised by
// tq.py's own functions: refuse(where, why) and check(code, where).
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "tq.h"

namespace {

struct Library {
  decltype(&tq_pages_release) pages_release;
  decltype(&tq_pages_assign) pages_assign;
  decltype(&tq_kv8_append) kv8_append;
  decltype(&tq_kv8_gather) kv8_gather;
  decltype(&tq_sdpa_int8_decode) int8_decode;
  decltype(&tq_sdpa_prompt) prompt;
} lib;
PyObject *refuse_fn = nullptr, *check_fn = nullptr;

struct Refused {};  // a Python error is set

[[noreturn]] void refuse(const char* where, const char* why) {
  PyObject* r = PyObject_CallFunction(refuse_fn, "ss", where, why);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, why);
  throw Refused{};
}

// The tensors of one call, all on the current CUDA device.
class Call {
 public:
  explicit Call(const char* where) : where_(where) {}
  const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(where_, (std::string(name) + " must be a tensor").c_str());
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) refuse(where_, (std::string(name) + " is not on a CUDA device").c_str());
    const int dev = t.get_device();
    if (dev_ < 0) {
      dev_ = dev;
      if (c10::cuda::current_device() != dev) refuse(where_, "tensors are not on the current CUDA device");
    }
    if (dev != dev_) refuse(where_, "tensors on different devices");
    return t;
  }
  // contiguous tensor of one of two types, n elements (n < 0: any number); None gives a null address where allowed
  void* flat(PyObject* o, const char* name, at::ScalarType type, int64_t n = -1, bool optional = false,
             at::ScalarType other = at::ScalarType::Undefined) {
    if (optional && o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, name);
    if ((t.scalar_type() != type && t.scalar_type() != other) || !t.is_contiguous() || (n >= 0 && t.numel() != n))
      refuse(where_, (std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor" +
                      (n < 0 ? std::string() : " of " + std::to_string(n) + " elements")).c_str());
    return t.data_ptr();
  }
  int32_t* ints(PyObject* o, const char* name, int64_t n = -1, bool optional = false) {
    return static_cast<int32_t*>(flat(o, name, at::kInt, n, optional));
  }
  int32_t* status(PyObject* o) { return o == Py_None ? nullptr : ints(o, "status"); }
  void* stream(PyObject* o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(dev_)).stream();
    PyObject* raw = PyObject_GetAttrString(o, "cuda_stream");
    if (!raw) throw Refused{};
    void* s = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    if (PyErr_Occurred()) throw Refused{};
    return s;
  }
  // packed [n][heads][d] whose heads stand side by side; returns the distance of its rows
  int64_t rows(const at::Tensor& t, const char* name, int64_t n, int64_t heads, int64_t d) {
    if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != d || t.stride(2) != 1 ||
        (heads > 1 && t.stride(1) != d))
      refuse(where_, (std::string(name) + " must be [" + std::to_string(n) + "][" + std::to_string(heads) + "][" +
                      std::to_string(d) + "] with its heads side by side").c_str());
    return n > 1 ? t.stride(0) : heads * d;  // the stride of a single row means nothing
  }
  int dtype(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
      case at::kHalf: return TQ_FP16;
      case at::kBFloat16: return TQ_BF16;
      case at::kFloat: return TQ_FP32;
      default: refuse(where_, (std::string(name) + " must be fp16, bf16 or fp32").c_str());
    }
  }
  int32_t i32(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    if (v < INT32_MIN || v > INT32_MAX) refuse(where_, "a size beyond 32 bits");
    return static_cast<int32_t>(v);
  }
  float f32(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return static_cast<float>(v);
  }
  int64_t bytes(PyObject* o, void** p) {
    const at::Tensor& t = tensor(o, "workspace");
    if (!t.is_contiguous()) refuse(where_, "workspace must be contiguous");
    *p = t.data_ptr();
    return t.numel() * static_cast<int64_t>(t.element_size());
  }
  PyObject* done(int code) {
    if (code == TQ_OK) Py_RETURN_NONE;
    return PyObject_CallFunction(check_fn, "is", code, where_);
  }

 private:
  const char* where_;
  int dev_ = -1;
};

// An 8-bit cache: the C struct, its device, and the tensors it lives in.
struct Cache {
  tq_kv8_cache c;
  bool cuda;
  int dev;
  PyObject* keep[3];
  std::vector<int64_t> sizes[3];
  // The tensors' addresses as they are now; false if one has another type, shape or device than it came with.
  bool refresh() {
    void* at[3] = {};
    for (int i = 0; i < 3; ++i) {
      if (!keep[i]) continue;
      const at::Tensor& t = THPVariable_Unpack(keep[i]);
      if (t.scalar_type() != (i == 0 ? at::kByte : at::kInt) || t.sizes() != sizes[i] || !t.is_contiguous() || t.is_cuda() != cuda || (cuda && t.get_device() != dev)) return false;
      at[i] = t.data_ptr();
    }
    c.blocks = static_cast<uint8_t*>(at[0]);
    c.seq_lens = static_cast<int32_t*>(at[1]);
    c.page_table = static_cast<int32_t*>(at[2]);
    return true;
  }
};
const char kCache[] = "tq_kv8_cache", kMoved[] = "a tensor of the cache was resized, or has another type or device than it had";
void free_cache(PyObject* capsule) {
  auto* x = static_cast<Cache*>(PyCapsule_GetPointer(capsule, kCache));
  for (PyObject* k : x->keep) Py_XDECREF(k);
  delete x;
}

template <typename F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, want);
  return false;
}

// cache8(blocks, seq_lens, page_table or None)
PyObject* py_cache8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 3)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* w = "KV8Cache";
    for (int i = 0; i < 3; ++i)
      if (!(i == 2 && a[i] == Py_None) && !THPVariable_Check(a[i])) refuse(w, "blocks, seq_lens and page_table must be tensors");
    const at::Tensor &blocks = THPVariable_Unpack(a[0]), &lens = THPVariable_Unpack(a[1]);
    const bool paged = a[2] != Py_None;
    if (blocks.dim() != 4 || blocks.scalar_type() != at::kByte || !blocks.is_contiguous() ||
        blocks.size(3) != TQ_BLOCK8_BYTES((blocks.size(3) - 16) / 32))
      refuse(w, "blocks must be a contiguous uint8 tensor [sequences or pages][H_kv][blocks][32 d + 16]");
    if (lens.scalar_type() != at::kInt || !lens.is_contiguous() || lens.dim() != 1 || lens.device() != blocks.device())
      refuse(w, "seq_lens must be a contiguous int32 tensor [B] beside the blocks");
    Cache x = {};
    x.c.blocks = static_cast<uint8_t*>(blocks.data_ptr());
    x.c.seq_lens = static_cast<int32_t*>(lens.data_ptr());
    const int64_t B = lens.numel(), tokens = 16 * blocks.size(2);
    int64_t cap = tokens;
    if (paged) {
      const at::Tensor& table = THPVariable_Unpack(a[2]);
      if (table.scalar_type() != at::kInt || !table.is_contiguous() || table.dim() != 2 || table.size(0) != B ||
          table.device() != blocks.device())
        refuse(w, "page_table must be a contiguous int32 tensor [B][max_pages] beside the blocks");
      x.c.page_table = static_cast<int32_t*>(table.data_ptr());
      x.c.max_pages = static_cast<int32_t>(table.size(1));
      x.c.page_tokens = static_cast<int32_t>(tokens);
      x.c.num_pages = static_cast<int32_t>(blocks.size(0));
      cap = tokens * table.size(1);
    } else if (blocks.size(0) != B) {
      refuse(w, "seq_lens must have one entry per sequence of blocks");
    }
    if (cap > INT32_MAX || B > INT32_MAX || blocks.size(0) > INT32_MAX || blocks.size(1) > INT32_MAX) refuse(w, "a size beyond 32 bits");
    x.c.B = static_cast<int32_t>(B);
    x.c.H_kv = static_cast<int32_t>(blocks.size(1));
    x.c.S_cap = static_cast<int32_t>(cap);
    x.c.d = static_cast<int32_t>((blocks.size(3) - 16) / 32);
    x.cuda = blocks.is_cuda();
    x.dev = x.cuda ? blocks.get_device() : -1;
    for (int i = 0; i < (paged ? 3 : 2); ++i) {
      x.keep[i] = a[i];
      x.sizes[i] = THPVariable_Unpack(a[i]).sizes().vec();
      Py_INCREF(a[i]);
    }
    PyObject* capsule = PyCapsule_New(new Cache(x), kCache, free_cache);
    return capsule;
  });
}

// sizes(cache) -> (B, H_kv, S_cap, d, page_tokens, max_pages, num_pages); address(cache) -> that of the C struct
PyObject* py_sizes(PyObject*, PyObject* o) {
  auto* x = static_cast<Cache*>(PyCapsule_GetPointer(o, kCache));
  if (!x) return nullptr;
  return Py_BuildValue("iiiiiii", x->c.B, x->c.H_kv, x->c.S_cap, x->c.d, x->c.page_tokens, x->c.max_pages, x->c.num_pages);
}
PyObject* py_address(PyObject*, PyObject* o) {
  auto* x = static_cast<Cache*>(PyCapsule_GetPointer(o, kCache));
  if (!x) return nullptr;
  return guarded([&]() -> PyObject* {
    if (!x->refresh()) refuse("KV8Cache", kMoved);
    return PyLong_FromVoidPtr(&x->c);
  });
}

const Cache& cache_of(PyObject* o, const char* where) {
  if (!PyCapsule_IsValid(o, kCache)) refuse(where, "cache must be a KV8Cache or a PagedKV8Cache");
  auto* x = static_cast<Cache*>(PyCapsule_GetPointer(o, kCache));
  if (!x->cuda || x->dev != c10::cuda::current_device()) refuse(where, "the cache is not on the current CUDA device");
  if (!x->refresh()) refuse(where, kMoved);
  return *x;
}
void beside(const Cache& c, const at::Tensor& t, const char* where) {
  if (!t.is_cuda() || t.get_device() != c.dev) refuse(where, "tensors on different devices");
}

struct Pool {
  int32_t* table;
  int32_t cols, *free_pages, *count, *lens_out, *count_out;
};
// page_table, free_pages, free_count, free_count_out: None for contiguous caches
Pool pool_of(Call& call, const char* w, int64_t B, PyObject* table, PyObject* max_pages, PyObject* free_pages, PyObject* cnt,
             PyObject* lens_out, PyObject* cnt_out, int64_t num_pages) {
  Pool p = {};
  p.lens_out = call.ints(lens_out, "seq_lens_out", B);
  if (table == Py_None) {
    p.cols = max_pages == Py_None ? 1 : call.i32(max_pages);
    return p;
  }
  const at::Tensor& t = call.tensor(table, "page_table");
  if (t.scalar_type() != at::kInt || !t.is_contiguous() || t.dim() != 2 || t.size(0) != B || t.size(1) > INT32_MAX)
    refuse(w, "page_table must be a contiguous int32 tensor [B][max_pages]");
  p.table = static_cast<int32_t*>(t.data_ptr());
  p.cols = static_cast<int32_t>(t.size(1));
  p.free_pages = call.ints(free_pages, "free_pages");
  if (THPVariable_Unpack(free_pages).numel() < num_pages) refuse(w, "free_pages must have room for num_pages entries");
  p.count = call.ints(cnt, "free_count", 1);
  p.count_out = call.ints(cnt_out, "free_count_out", 1);
  return p;
}

// page_table, seq_lens, finished, page_tokens, num_pages, free_pages, free_count, seq_lens_out, free_count_out, status, stream, max_pages
PyObject* py_pages_release(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 12)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* w = "tq_pages_release";
    Call call(w);
    int32_t* lens = call.ints(a[1], "seq_lens");
    const int64_t B = THPVariable_Unpack(a[1]).numel();
    auto* finished = static_cast<uint8_t*>(call.flat(a[2], "finished", at::kByte, B, false, at::kBool));
    const int32_t page_tokens = call.i32(a[3]), num_pages = call.i32(a[4]);
    const Pool p = pool_of(call, w, B, a[0], a[11], a[5], a[6], a[7], a[8], num_pages);
    int32_t* status = call.status(a[9]);
    return call.done(lib.pages_release(p.table, lens, finished, static_cast<int32_t>(B), page_tokens, p.cols, num_pages, p.free_pages,
                                       p.count, p.lens_out, p.count_out, status, call.stream(a[10])));
  });
}

// page_table, seq_lens, new_lens, page_tokens, num_pages, free_pages, free_count, seq_lens_out, free_count_out, token_offsets, slots,
// workspace, status, stream, max_pages
PyObject* py_pages_assign(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 15)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* w = "tq_pages_assign";
    Call call(w);
    int32_t* lens = call.ints(a[1], "seq_lens");
    const int64_t B = THPVariable_Unpack(a[1]).numel();
    int32_t* fresh = call.ints(a[2], "new_lens", B);
    const int32_t page_tokens = call.i32(a[3]), num_pages = call.i32(a[4]);
    const Pool p = pool_of(call, w, B, a[0], a[14], a[5], a[6], a[7], a[8], num_pages);
    int32_t* offsets = call.ints(a[9], "token_offsets", B + 1);
    auto* slots = static_cast<int64_t*>(call.flat(a[10], "slots", at::kLong));
    void* ws;
    const int64_t ws_bytes = call.bytes(a[11], &ws);
    int32_t* status = call.status(a[12]);
    return call.done(lib.pages_assign(p.table, lens, fresh, static_cast<int32_t>(B), page_tokens, p.cols, num_pages, p.free_pages, p.count,
                                      p.lens_out, p.count_out, offsets, slots, THPVariable_Unpack(a[10]).numel(), ws, ws_bytes, status,
                                      call.stream(a[13])));
  });
}

// cache, k_new, v_new, slots, status, stream
PyObject* py_kv8_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 6)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* w = "tq_kv8_append";
    const Cache& c = cache_of(a[0], w);
    Call call(w);
    const at::Tensor &k = call.tensor(a[1], "k_new"), &v = call.tensor(a[2], "v_new");
    beside(c, k, w);
    auto* slots = static_cast<int64_t*>(call.flat(a[3], "slots", at::kLong));
    const int64_t rows = THPVariable_Unpack(a[3]).numel();
    if (k.scalar_type() != v.scalar_type()) refuse(w, "k_new and v_new must be of one type");
    const int64_t ks = call.rows(k, "k_new", rows, c.c.H_kv, c.c.d), vs = call.rows(v, "v_new", rows, c.c.H_kv, c.c.d);
    int32_t* status = call.status(a[4]);
    return call.done(lib.kv8_append(&c.c, k.data_ptr(), v.data_ptr(), call.dtype(k, "k_new"), ks, vs, slots, rows, status, call.stream(a[5])));
  });
}

// cache, slots, k_out, v_out, status, stream
PyObject* py_kv8_gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 6)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* w = "tq_kv8_gather";
    const Cache& c = cache_of(a[0], w);
    Call call(w);
    auto* slots = static_cast<int64_t*>(call.flat(a[1], "slots", at::kLong));
    const int64_t rows = THPVariable_Unpack(a[1]).numel();
    const at::Tensor &k = call.tensor(a[2], "k_out"), &v = call.tensor(a[3], "v_out");
    beside(c, k, w);
    call.rows(k, "k_out", rows, c.c.H_kv, c.c.d);
    call.rows(v, "v_out", rows, c.c.H_kv, c.c.d);
    if (k.scalar_type() != v.scalar_type() || !k.is_contiguous() || !v.is_contiguous())
      refuse(w, "k_out and v_out must be contiguous and of one type");
    int32_t* status = call.status(a[4]);
    return call.done(lib.kv8_gather(&c.c, slots, rows, k.data_ptr(), v.data_ptr(), call.dtype(k, "k_out"), status, call.stream(a[5])));
  });
}

// cache, q, attn_scale, window, max_seq_len, workspace, out, status, stream
PyObject* py_int8_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* w = "tq_sdpa_int8_decode";
    const Cache& c = cache_of(a[0], w);
    Call call(w);
    const at::Tensor &q = call.tensor(a[1], "q"), &out = call.tensor(a[6], "out");
    beside(c, q, w);
    if (q.dim() != 3 || !out.is_contiguous() || out.sizes() != q.sizes()) refuse(w, "q must be [B][H_q][d] and out a contiguous tensor of its shape");
    const int64_t H_q = q.size(1), stride = call.rows(q, "q", c.c.B, H_q, c.c.d);
    void* ws;
    const int64_t ws_bytes = call.bytes(a[5], &ws);
    int32_t* status = call.status(a[7]);
    return call.done(lib.int8_decode(&c.c, q.data_ptr(), call.dtype(q, "q"), stride, static_cast<int32_t>(H_q), call.f32(a[2]), call.i32(a[3]),
                                     call.i32(a[4]), ws, ws_bytes, out.data_ptr(), call.dtype(out, "out"), status, call.stream(a[8])));
  });
}

// q, k, v, q_offsets, kv_offsets, attn_scale, out, causal, window, status, stream
PyObject* py_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 11)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* w = "tq_sdpa_prompt";
    Call call(w);
    const at::Tensor &q = call.tensor(a[0], "q"), &k = call.tensor(a[1], "k"), &v = call.tensor(a[2], "v"), &out = call.tensor(a[6], "out");
    if (q.dim() != 3 || k.dim() != 3 || k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type())
      refuse(w, "q, k, v must be packed [n][heads][d] tensors of one type");
    if (!out.is_contiguous() || out.sizes() != q.sizes()) refuse(w, "out must be a contiguous tensor of q's shape");
    const int64_t n_q = q.size(0), H_q = q.size(1), d = q.size(2), n_kv = k.size(0), H_kv = k.size(1);
    const int64_t qs = call.rows(q, "q", n_q, H_q, d), ks = call.rows(k, "k", n_kv, H_kv, d), vs = call.rows(v, "v", n_kv, H_kv, d);
    int32_t* q_at = call.ints(a[3], "q_offsets");
    const int64_t B = THPVariable_Unpack(a[3]).numel() - 1;
    int32_t* k_at = call.ints(a[4], "kv_offsets", B + 1);
    const int causal = PyObject_IsTrue(a[7]);
    if (causal < 0) throw Refused{};
    if (n_q > INT32_MAX || n_kv > INT32_MAX || H_q > INT32_MAX || H_kv > INT32_MAX || d > INT32_MAX || B > INT32_MAX)
      refuse(w, "a size beyond 32 bits");
    int32_t* status = call.status(a[9]);
    return call.done(lib.prompt(q.data_ptr(), k.data_ptr(), v.data_ptr(), call.dtype(q, "q"), qs, ks, vs, static_cast<int32_t>(n_q),
                                static_cast<int32_t>(n_kv), q_at, k_at, static_cast<int32_t>(B), static_cast<int32_t>(H_q),
                                static_cast<int32_t>(H_kv), static_cast<int32_t>(d), call.f32(a[5]), causal, call.i32(a[8]), out.data_ptr(),
                                call.dtype(out, "out"), status, call.stream(a[10])));
  });
}

// attach(refuse, check, address of each function of Library in its order)
PyObject* py_attach(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 8)) return nullptr;
  void* at[6];
  for (int i = 0; i < 6; ++i) {
    at[i] = PyLong_AsVoidPtr(a[2 + i]);
    if (PyErr_Occurred()) return nullptr;
  }
  lib = {reinterpret_cast<decltype(lib.pages_release)>(at[0]), reinterpret_cast<decltype(lib.pages_assign)>(at[1]),
         reinterpret_cast<decltype(lib.kv8_append)>(at[2]),    reinterpret_cast<decltype(lib.kv8_gather)>(at[3]),
         reinterpret_cast<decltype(lib.int8_decode)>(at[4]),   reinterpret_cast<decltype(lib.prompt)>(at[5])};
  Py_XDECREF(refuse_fn);
  Py_XDECREF(check_fn);
  refuse_fn = a[0];
  check_fn = a[1];
  Py_INCREF(refuse_fn);
  Py_INCREF(check_fn);
  Py_RETURN_NONE;
}

#define TQ_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TQ_FAST(attach),     TQ_FAST(cache8),     TQ_FAST(pages_release), TQ_FAST(pages_assign),
                         TQ_FAST(kv8_append), TQ_FAST(kv8_gather), TQ_FAST(int8_decode),   TQ_FAST(prompt),
                         {"sizes", py_sizes, METH_O, nullptr},
                         {"address", py_address, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tq_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tq_bind() { return PyModule_Create(&module); }
