// Argument marshalling of the serving entry points for Python: torch tensors in, C calls of
// include/kint_serve.h out.  One step of a small batch spends a few microseconds on the GPU, so the
// checks, the output allocation and the call are made here instead of in Python.  No arithmetic.
//
// The library's functions are handed over as addresses (bind), so this module links against
// torch and Python only.
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <optional>

#include "../../include/kint_serve.h"

namespace {

struct Api {
  decltype(&kint_blocks_extend) blocks_extend;
  decltype(&kint_rope) rope;
  decltype(&kint_cache_append) append;
  decltype(&kint_cache_read) read;
  decltype(&kint_cache_attn_step) attn;
  decltype(&kint_cache_attn_workspace_bytes) attn_ws;
} api;
PyObject* kint_error = nullptr;  // KintError(code, what)

// kint_cache_attn_workspace_bytes at sizes that run in one launch, whose workspace is not touched.
constexpr size_t kUnusedWorkspace = 256;

struct Refused {};  // a Python error is set

[[noreturn]] void refuse(const char* what) {
  PyErr_SetString(PyExc_ValueError, what);
  throw Refused();
}
void need(bool ok, const char* what) {
  if (!ok) refuse(what);
}
void run(int rc, const char* what) {
  if (rc == 0) return;
  PyObject* e = PyObject_CallFunction(kint_error, "is", rc, what);
  if (e) {
    PyErr_SetObject(kint_error, e);
    Py_DECREF(e);
  }
  throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s: expected a tensor", what);
    throw Refused();
  }
  return THPVariable_Unpack(o);
}
bool none(PyObject* o) { return o == Py_None; }
int whole(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  need(v >= INT32_MIN && v <= INT32_MAX, "a whole number is out of range");
  return (int)v;
}
// A size as the C calls take it.
int size(int64_t n) {
  need(n <= INT32_MAX, "a size is past 2^31 - 1");
  return (int)n;
}
// The call's stream: the current one, or the given handle, which is then the current one while the call allocates, so that
// its memory belongs to it.
struct CallStream {
  std::optional<c10::cuda::CUDAStreamGuard> guard;
  void* handle;
  explicit CallStream(PyObject* o) {
    if (none(o)) {
      handle = c10::cuda::getCurrentCUDAStream().stream();
      return;
    }
    handle = PyLong_AsVoidPtr(o);
    if (!handle && PyErr_Occurred()) throw Refused();
    guard.emplace(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(handle), c10::cuda::current_device()));
  }
};

kint_dtype type_of(const at::Tensor& t, const char* what) {
  switch (t.scalar_type()) {
    case at::kFloat: return KINT_FP32;
    case at::kBFloat16: return KINT_BF16;
    case at::kHalf: return KINT_FP16;
    default:
      PyErr_Format(PyExc_ValueError, "%s: expected fp32, bf16 or fp16", what);
      throw Refused();
  }
}
// [..., heads, d] on the GPU with contiguous channels: (batch,) time, heads, d.
kint_heads heads(const at::Tensor& t, const char* what, int dims) {
  if (!t.is_cuda() || t.dim() != dims || !(t.stride(-1) == 1 || t.size(-1) <= 1)) {
    PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor of %d dimensions with contiguous channels", what, dims);
    throw Refused();
  }
  type_of(t, what);
  return kint_heads{t.data_ptr(), dims == 4 ? t.stride(0) : 0, t.stride(-3), t.stride(-2), size(t.size(-2))};
}
// Whole numbers on the GPU, contiguous in the last dimension.
template <class I>
I* ints(const at::Tensor& t, const char* what) {
  if (!t.is_cuda() || t.scalar_type() != (sizeof(I) == 8 ? at::kLong : at::kInt) ||
      !(t.dim() == 0 || t.stride(-1) == 1 || t.size(-1) <= 1)) {
    PyErr_Format(PyExc_ValueError, "%s: expected a contiguous CUDA tensor of int%d", what, (int)sizeof(I) * 8);
    throw Refused();
  }
  return static_cast<I*>(t.data_ptr());
}
// pages [num_blocks, kv_heads, block_size / 16, 18 d], uint8; blocks may be strided.
kint_cache pool(const at::Tensor& t) {
  need(t.is_cuda() && t.scalar_type() == at::kByte && t.dim() == 4, "pages: expected a 4-D uint8 CUDA tensor");
  const int64_t slabs = t.size(2), bytes = t.size(3);
  need(bytes % 18 == 0 && t.stride(3) == 1 && t.stride(2) == bytes && t.stride(1) == slabs * bytes,
       "pages: expected [num_blocks, kv_heads, block_size / 16, 18 d], contiguous within a block");
  need(t.size(0) <= INT32_MAX && slabs <= 4096, "pages: too many blocks or slabs");
  return kint_cache{t.data_ptr(), t.stride(0), (int)t.size(0), 16 * (int)slabs, size(t.size(1)), size(bytes / 18)};
}
struct Table {
  const float* ptr = nullptr;
  int max_pos = 0, rot = 0;
};
Table rotations(const at::Tensor& t) {
  need(t.is_cuda() && t.scalar_type() == at::kFloat && t.dim() == 3 && t.size(2) == 2 && t.is_contiguous(),
       "table: expected a contiguous fp32 CUDA tensor [max_pos, rot / 2, 2]");
  return Table{static_cast<const float*>(t.data_ptr()), size(t.size(0)), size(2 * t.size(1))};
}

// A tensor over part of `base`'s memory, `at` elements of its own type in, without a dispatched view: results that come
// together share one allocation.
at::Tensor part(const at::Tensor& base, at::ScalarType type, int64_t at, at::IntArrayRef sizes, at::IntArrayRef strides) {
  auto t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(base.storage()), base.key_set(),
                                                    c10::scalarTypeToTypeMeta(type));
  if (strides.empty())
    t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
  else
    t.unsafeGetTensorImpl()->set_sizes_and_strides(sizes, strides);
  t.unsafeGetTensorImpl()->set_storage_offset(at);
  return t;
}
int64_t up_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
// A tensor of the caller's that the call wrote into counts one change more, so that autograd notices where it was saved before.
void wrote(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// Calls whose result has no derivative here: where one is asked for, the result says so when it is needed, instead of passing for a
// constant, and a buffer for it is refused.
bool asked(const at::Tensor& x) { return x.requires_grad() && c10::GradMode::is_enabled(); }
void plain_buffer(const at::Tensor& x, const at::Tensor& out) {
  need(!asked(x) && !asked(out), "a buffer for the result is not taken where gradients are asked for");
}
void no_derivative(at::Tensor& y, const at::Tensor& x, const char* what) {
  if (asked(x))
    torch::autograd::set_history(y, std::make_shared<torch::autograd::NotImplemented>(what, torch::autograd::collect_next_edges(x)));
}
// An output like `x`: its strides where they fill its memory, else contiguous.
at::IntArrayRef like(const at::Tensor& x) { return x.is_non_overlapping_and_dense() ? x.strides() : at::IntArrayRef(); }

template <class F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t wanted, F&& body) {
  if (got != wanted) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments", wanted);
    return nullptr;
  }
  try {
    return body();
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {  // of torch (out of memory, for one)
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }

// (addresses of the six functions, KintError)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    void* f[6];
    for (int i = 0; i < 6; ++i) {
      f[i] = PyLong_AsVoidPtr(a[i]);
      if (!f[i]) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function");
        throw Refused();
      }
    }
    api.blocks_extend = (decltype(api.blocks_extend))f[0];
    api.rope = (decltype(api.rope))f[1];
    api.append = (decltype(api.append))f[2];
    api.read = (decltype(api.read))f[3];
    api.attn = (decltype(api.attn))f[4];
    api.attn_ws = (decltype(api.attn_ws))f[5];
    Py_INCREF(a[6]);
    Py_XDECREF(kint_error);
    kint_error = a[6];
    Py_RETURN_NONE;
  });
}

// lens, new, table, free, n_free, block_size, tokens, stream -> lens, cu, slots, pos, req, n_free, refused
PyObject* extend_blocks(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const at::Tensor &lens = tensor(a[0], "lens"), &add = tensor(a[1], "new"), &table = tensor(a[2], "table"),
                     &list = tensor(a[3], "free"), &n_free = tensor(a[4], "n_free");
    const int block = whole(a[5]), tokens = whole(a[6]);
    need(lens.dim() == 1 && add.sizes() == lens.sizes() && table.dim() == 2 && table.size(0) == lens.size(0) && n_free.numel() == 1,
         "lens, new, table and n_free disagree on the requests");
    need(list.dim() == 1, "free: expected one dimension");
    need(tokens >= 0, "tokens must not be negative");
    const int32_t *pl = ints<int32_t>(lens, "lens"), *pa = ints<int32_t>(add, "new"), *pf = ints<int32_t>(list, "free"),
                  *pn = ints<int32_t>(n_free, "n_free");
    int32_t* pt = ints<int32_t>(table, "table");
    const CallStream stream(a[7]);
    // one allocation: slots (8 bytes each), then pos, req, lens, cu, n_free, refused (4 bytes each), pos and req on 16 bytes
    const int64_t B = lens.size(0), places = up_to(tokens, 4), at_pos = 2 * places, at_req = at_pos + places, at_lens = at_req + places,
                  at_cu = at_lens + B, at_free = at_cu + B + 1, at_ref = at_free + 1;
    const at::Tensor out = at::empty({at_ref + 1}, lens.options());
    int32_t* o = static_cast<int32_t*>(out.data_ptr());
    run(api.blocks_extend(pl, pa, pt, size(table.stride(0)), size(table.size(1)), pf, size(list.numel()), pn, size(B), block, tokens,
                          o + at_lens, o + at_free, o + at_cu, reinterpret_cast<int64_t*>(o), o + at_pos, o + at_req, o + at_ref,
                          stream.handle),
        "kint_blocks_extend");
    wrote(table);
    auto ints_at = [&](int64_t at, int64_t n) { return wrap(part(out, at::kInt, at, {n}, {})); };
    return Py_BuildValue("(NNNNNNN)", ints_at(at_lens, B), ints_at(at_cu, B + 1), wrap(part(out, at::kLong, 0, {tokens}, {})),
                         ints_at(at_pos, tokens), ints_at(at_req, tokens), ints_at(at_free, 1), ints_at(at_ref, 1));
  });
}

// q, k, pos, table, interleaved, inverse, q_out, k_out, stream -> q', k'
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &pos = tensor(a[2], "pos");
    const at::Tensor* k = none(a[1]) ? nullptr : &tensor(a[1], "k");
    const kint_heads hq = heads(q, "q", 4), hk = k ? heads(*k, "k", 4) : kint_heads{};
    need(!k || (k->scalar_type() == q.scalar_type() && k->size(0) == q.size(0) && k->size(1) == q.size(1) && k->size(3) == q.size(3)),
         "q and k disagree on type, batch, time or channels");
    const int64_t B = q.size(0), T = q.size(1);
    need((pos.dim() == 2 && pos.size(0) == B && pos.size(1) == T) || (pos.dim() == 1 && pos.size(0) == T),
         "pos: expected [B, T] or [T]");
    const int32_t* pp = ints<int32_t>(pos, "pos");
    const Table tab = rotations(tensor(a[3], "table"));
    const CallStream stream(a[8]);
    at::Tensor qo, ko;
    if (none(a[6])) {  // both outputs in one allocation, k' on a 16-byte boundary
      const int64_t nq = k ? up_to(q.numel(), 8) : q.numel();
      const at::Tensor both = at::empty({nq + (k ? k->numel() : 0)}, q.options());
      qo = part(both, q.scalar_type(), 0, q.sizes(), like(q));
      if (k) ko = part(both, q.scalar_type(), nq, k->sizes(), like(*k));
    } else {
      qo = tensor(a[6], "out");
      plain_buffer(q, qo);
      if (k) {
        ko = tensor(a[7], "out");
        plain_buffer(*k, ko);
      }
    }
    need(qo.sizes() == q.sizes() && qo.scalar_type() == q.scalar_type() &&
             (!k || (ko.sizes() == k->sizes() && ko.scalar_type() == k->scalar_type())),
         "out disagrees with q and k");
    if (q.numel() || (k && k->numel())) {
      const kint_heads ho = heads(qo, "out", 4), hko = k ? heads(ko, "out", 4) : kint_heads{};
      run(api.rope(&hq, &ho, &hk, &hko, pp, pos.dim() == 2 ? pos.stride(0) : 0, tab.ptr, tab.max_pos, size(B), size(T), size(q.size(3)),
                   tab.rot, PyObject_IsTrue(a[4]), PyObject_IsTrue(a[5]), type_of(q, "q"), stream.handle),
          "kint_rope");
      if (!none(a[6])) {
        wrote(qo);
        if (k) wrote(ko);
      }
    }
    no_derivative(qo, q, "rope (rotary is)");
    if (k) no_derivative(ko, *k, "rope (rotary is)");
    PyObject* second = Py_None;
    if (k)
      second = wrap(ko);
    else
      Py_INCREF(second);
    return Py_BuildValue("(NN)", wrap(qo), second);
  });
}

// k, v, slots, pages, q, pos, table, interleaved, q_out, stream -> q'
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v"), &slots = tensor(a[2], "slots"), &pages = tensor(a[3], "pages");
    const kint_heads hk = heads(k, "k", 3), hv = heads(v, "v", 3);
    const kint_cache c = pool(pages);
    const int64_t tokens = k.size(0);
    need(k.sizes() == v.sizes() && k.scalar_type() == v.scalar_type() && k.size(2) == c.d && slots.dim() == 1 && slots.size(0) == tokens,
         "k, v, slots and the pages disagree");
    Table tab;
    const int32_t* pos = nullptr;
    if (!none(a[6])) {
      tab = rotations(tensor(a[6], "table"));
      need(!none(a[5]), "a rotation needs pos [tokens]");
      const at::Tensor& p = tensor(a[5], "pos");
      need(p.dim() == 1 && p.size(0) == tokens, "a rotation needs pos [tokens]");
      pos = ints<int32_t>(p, "pos");
    }
    const CallStream stream(a[9]);
    kint_heads hq{}, hqo{};
    at::Tensor qo;
    const bool has_q = !none(a[4]), turn = has_q && tab.ptr;
    need(turn || none(a[8]), "q_out: expected with q and a rotation only");
    if (has_q) {
      const at::Tensor& q = tensor(a[4], "q");
      need(q.dim() == 3 && q.size(0) == tokens && q.size(2) == c.d && q.scalar_type() == k.scalar_type(), "q and k disagree");
      if (turn) {
        qo = none(a[8]) ? at::empty_like(q) : tensor(a[8], "q_out");
        if (!none(a[8])) plain_buffer(q, qo);
        need(qo.sizes() == q.sizes() && qo.scalar_type() == q.scalar_type(), "q_out disagrees with q");
        hq = heads(q, "q", 3);
        hqo = heads(qo, "q_out", 3);
      }
    }
    if (tokens) {
      run(api.append(&c, &hk, &hv, ints<int64_t>(slots, "slots"), size(tokens), turn ? &hq : nullptr, turn ? &hqo : nullptr, pos, tab.ptr,
                     tab.max_pos, tab.rot, PyObject_IsTrue(a[7]), type_of(k, "k"), stream.handle),
          "kint_cache_append");
      wrote(pages);
      if (!none(a[8])) wrote(qo);
    }
    if (turn) {
      no_derivative(qo, tensor(a[4], "q"), "append");
      return wrap(qo);
    }
    Py_INCREF(a[4]);
    return a[4];  // q as it came, or None
  });
}

// pages, slots, dtype (0, 1, 2), stream -> k, v
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 4, [&]() -> PyObject* {
    const at::Tensor &pages = tensor(a[0], "pages"), &slots = tensor(a[1], "slots");
    const kint_cache c = pool(pages);
    const int type = whole(a[2]);
    need(type >= 0 && type <= 2, "dtype: expected fp32, bf16 or fp16");
    need(slots.dim() == 1, "slots: expected one dimension");
    const int64_t* ps = ints<int64_t>(slots, "slots");
    const auto opts = pages.options().dtype(type == 0 ? at::kFloat : type == 1 ? at::kBFloat16 : at::kHalf);
    const CallStream stream(a[3]);
    const int64_t each = slots.size(0) * c.kv_heads * c.d;
    const at::Tensor both = at::empty({2 * each}, opts);
    const at::Tensor k = part(both, both.scalar_type(), 0, {slots.size(0), c.kv_heads, c.d}, {}),
                     v = part(both, both.scalar_type(), each, {slots.size(0), c.kv_heads, c.d}, {});
    if (slots.size(0)) {
      const kint_heads hk = heads(k, "k", 3), hv = heads(v, "v", 3);
      run(api.read(&c, ps, size(slots.size(0)), &hk, &hv, (kint_dtype)type, stream.handle), "kint_cache_read");
    }
    return Py_BuildValue("(NN)", wrap(k), wrap(v));
  });
}

// q, pages, table, lens, cu, Kint, calib, tau, recon, window, sinks, max_new, max_len, out, ws, slots, stream -> out
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 17, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &pages = tensor(a[1], "pages"), &table = tensor(a[2], "table"), &lens = tensor(a[3], "lens"),
                     &cu = tensor(a[4], "cu");
    const kint_heads hq = heads(q, "q", 3);
    const kint_cache c = pool(pages);
    need(lens.dim() == 1 && q.size(2) == c.d && table.dim() == 2 && table.size(0) == lens.size(0) && cu.dim() == 1 &&
             cu.size(0) == lens.size(0) + 1,
         "q, pages, table, lens and cu disagree");
    const int32_t *pt = ints<int32_t>(table, "table"), *pl = ints<int32_t>(lens, "lens"), *pc = ints<int32_t>(cu, "cu");
    const int window = whole(a[9]), sinks = whole(a[10]), B = size(lens.size(0)), width = size(table.size(1));
    const int64_t hold = (int64_t)width * c.block_size;
    const int max_new = none(a[11]) ? size(q.size(0)) : whole(a[11]);
    const int max_len = none(a[12]) ? (int)(hold < INT32_MAX ? hold : INT32_MAX) : whole(a[12]);
    const double tau = PyFloat_AsDouble(a[7]);
    if (tau == -1.0 && PyErr_Occurred()) throw Refused();
    const int64_t* slots = nullptr;
    if (!none(a[15])) {
      const at::Tensor& t = tensor(a[15], "slots");
      need(t.dim() == 1 && t.size(0) == q.size(0), "slots: expected one for each row of q");
      slots = ints<int64_t>(t, "slots");
    }
    const CallStream stream(a[16]);
    at::Tensor out = none(a[13]) ? at::empty_like(q) : tensor(a[13], "out");
    need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type(), "out disagrees with q");
    if (!none(a[13])) plain_buffer(q, out);
    if (q.numel()) {
      const kint_heads ho = heads(out, "out", 3);
      at::Tensor ws;
      if (none(a[14])) {
        const size_t bytes = api.attn_ws(B, hq.heads, c.kv_heads, c.d, window, sinks, max_new, max_len);
        // sizes that run in one launch touch no workspace: any aligned memory of this call's will do
        if (bytes <= kUnusedWorkspace)
          ws = pages;
        else
          ws = at::empty({(int64_t)bytes}, pages.options());
      } else {
        ws = tensor(a[14], "ws");
        need(ws.is_cuda() && ws.is_contiguous(), "ws: expected a contiguous CUDA tensor");
      }
      run(api.attn(&hq, &ho, &c, pt, size(table.stride(0)), width, pl, pc, size(q.size(0)), B, window, sinks, whole(a[5]), (kint_calib)whole(a[6]),
                   (float)tau, (kint_recon)whole(a[8]), max_new, max_len, type_of(q, "q"), slots, none(a[13]), ws.data_ptr(), ws.is_same(pages) ? kUnusedWorkspace : ws.nbytes(),
                   stream.handle),
          "kint_cache_attn");
      if (!none(a[13])) wrote(out);
    }
    no_derivative(out, q, "attention over the cache");
    return wrap(out);
  });
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(bind), ENTRY(extend_blocks), ENTRY(rope), ENTRY(append), ENTRY(read), ENTRY(attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kint_serve", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kint_serve() { return PyModule_Create(&module); }
