// Argument marshalling of the token-level cache's calls (include/wk.h) for PyTorch tensors: checks, output allocation, the call.  These
// are made once per layer and token, and the kernels behind them take 2 to 20 us for small batches: marshalled in Python an
// attention call costs the host 9.6 us, a plan 11, a store 5.9; here 4.0, 5.0, 2.9.
//
// Each function returns its tensors; a str that says what is wrong with an argument; or the status of a call that failed, as an int.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <limits>
#include <optional>

#include "../../include/wk.h"

namespace {

decltype(&wk_page_plan) call_plan;
decltype(&wk_page_store) call_store;
decltype(&wk_paged_attention) call_attention;

int type_of(at::ScalarType t) {
  return t == at::kBFloat16 ? WK_BF16 : t == at::kHalf ? WK_F16 : t == at::kFloat8_e4m3fn ? WK_E4M3 : -1;
}

// One call's arguments, taken in order; the first that does not fit is remembered.
struct Arguments {
  PyObject* const* args;
  Py_ssize_t at = 0;
  const char* wrong = nullptr;
  explicit Arguments(PyObject* const* a) : args(a) {}

  bool need(bool ok, const char* what) {
    if (!ok && !wrong) wrong = what;
    return ok;
  }
  // nullptr for None, where that is allowed
  const at::Tensor* tensor(const char* what, bool optional = false) {
    PyObject* o = args[at++];
    if (optional && o == Py_None) return nullptr;
    if (!need(THPVariable_Check(o), what)) return nullptr;
    return &THPVariable_Unpack(o);
  }
  void* address() { return PyLong_AsVoidPtr(args[at++]); }
  int64_t whole() { return PyLong_AsLongLong(args[at++]); }
  int32_t whole32(const char* what) {
    const int64_t v = PyLong_AsLongLong(args[at++]);
    need(v >= std::numeric_limits<int32_t>::min() && v <= std::numeric_limits<int32_t>::max(), what);
    return static_cast<int32_t>(v);
  }
  double real() { return PyFloat_AsDouble(args[at++]); }
  void* stream(int64_t device) {
    PyObject* o = args[at++];
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
    given = c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(PyLong_AsVoidPtr(o)), static_cast<c10::DeviceIndex>(device));
    return given->stream();
  }
  std::optional<c10::cuda::CUDAStream> given;   // the caller's stream, if it is not left to be the current one
};

bool on(const at::Tensor& t, int64_t device) { return t.is_cuda() && t.get_device() == device; }
bool ints(const at::Tensor* t, int64_t size, int64_t device) {
  return t && on(*t, device) && t->scalar_type() == at::kInt && t->numel() >= size && t->is_contiguous();
}
bool table(const at::Tensor* t, int64_t rows, int64_t device) {
  return t && on(*t, device) && t->scalar_type() == at::kInt && t->dim() == 2 && t->size(0) >= rows && t->stride(1) == 1 &&
         t->size(1) <= std::numeric_limits<int32_t>::max();
}
// [n][heads][head_dim] with the heads of a row one after the other
bool rows(const at::Tensor* t, int64_t device) {
  return t && on(*t, device) && t->dim() == 3 && t->stride(2) == 1 && (t->size(1) == 1 || t->stride(1) == t->size(2)) &&
         t->size(0) <= std::numeric_limits<int32_t>::max();
}
// A contiguous tensor of x's type and device, without the way through the dispatcher.  It belongs to the stream that the call runs
// on, as if that were the current one: its memory was used on that stream only, and is used on that stream next.
at::Tensor empty(at::IntArrayRef sizes, const at::Tensor& x, const Arguments& a) {
  c10::cuda::OptionalCUDAStreamGuard guard;
  if (a.given) guard.reset_stream(*a.given);
  return at::Tensor(at::detail::empty_cuda(sizes, x.scalar_type(), x.device(), std::nullopt));
}
PyObject* said(const char* what) { return PyUnicode_FromString(what); }
PyObject* pair_of(const at::Tensor& x, const at::Tensor& y) {
  PyObject* pair = PyTuple_New(2);
  if (!pair) return nullptr;
  PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(x));
  PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(y));
  return pair;
}

// The library's calls wait where the GPU's queue is full: other Python threads run meanwhile.
template <typename F>
wk_status without_lock(F&& call) {
  PyThreadState* const state = PyEval_SaveThread();
  const wk_status st = call();
  PyEval_RestoreThread(state);
  return st;
}

// (ctx, device, n_pages, page_tokens, lens, new_tokens, lens_out|None, tables, ring, state, state_out|None, max_tokens, slots|None,
//  starts|None, stream|None) -> (slots, starts)
PyObject* page_plan(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 15) return said("wk_page_plan: 15 arguments");
  Arguments a(args);
  wk_ctx* ctx = static_cast<wk_ctx*>(a.address());
  const int64_t device = a.whole();
  const int32_t n_pages = a.whole32("wk_page_plan: n_pages"), page_tokens = a.whole32("wk_page_plan: page_tokens");
  const at::Tensor *lens = a.tensor("wk_page_plan: lens"), *more = a.tensor("wk_page_plan: new_tokens"),
                   *lens_out = a.tensor("wk_page_plan: lens_out", true), *tables = a.tensor("wk_page_plan: tables"),
                   *ring = a.tensor("wk_page_plan: ring"), *state = a.tensor("wk_page_plan: state"),
                   *state_out = a.tensor("wk_page_plan: state_out", true);
  const int32_t max_tokens = a.whole32("wk_page_plan: max_tokens");
  const at::Tensor *slots_in = a.tensor("wk_page_plan: slots_out", true), *starts_in = a.tensor("wk_page_plan: starts_out", true);
  if (PyErr_Occurred()) return nullptr;
  if (a.wrong) return said(a.wrong);
  const int64_t n = lens->numel();
  if (!a.need(n <= std::numeric_limits<int32_t>::max() && ints(lens, n, device) && ints(more, n, device) && ints(ring, n_pages, device) &&
                  ints(state, 4, device),
              "wk_page_plan: lens, new_tokens [n_req], ring [n_pages], state [4] int32, on the context's device") ||
      !a.need(!lens_out || ints(lens_out, n, device), "wk_page_plan: lens_out [n_req] int32") ||
      !a.need(!state_out || ints(state_out, 4, device), "wk_page_plan: state_out [4] int32") ||
      !a.need(table(tables, n, device), "wk_page_plan: tables [n_req, max_pages] int32") ||
      !a.need(max_tokens >= 0, "wk_page_plan: max_tokens") ||
      !a.need(!slots_in || ints(slots_in, max_tokens, device), "wk_page_plan: slots_out [max_tokens] int32") ||
      !a.need(!starts_in || ints(starts_in, n + 1, device), "wk_page_plan: starts_out [n_req + 1] int32"))
    return said(a.wrong);
  void* stream = a.stream(device);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor slots = slots_in ? *slots_in : empty({max_tokens}, *lens, a);
  const at::Tensor starts = starts_in ? *starts_in : empty({n + 1}, *lens, a);
  if (n == 0) {   // nothing to plan: no rows, and the ring as it is
    if (n_pages < 1 || page_tokens < 1) return PyLong_FromLong(WK_ERR_ARG);
    c10::cuda::OptionalCUDAStreamGuard guard;
    if (a.given) guard.reset_stream(*a.given);
    slots.view(-1).narrow(0, 0, max_tokens).fill_(-1);
    starts.view(-1).narrow(0, 0, 1).zero_();
    if (state_out && !state_out->is_same(*state)) state_out->view(-1).narrow(0, 0, 4).copy_(state->view(-1).narrow(0, 0, 4));
    return pair_of(slots, starts);
  }
  const wk_status st = without_lock([&] { return call_plan(
      ctx, n_pages, page_tokens, static_cast<int32_t>(n), lens->data_ptr<int32_t>(), more->data_ptr<int32_t>(),
      (lens_out ? lens_out : lens)->data_ptr<int32_t>(), tables->data_ptr<int32_t>(), static_cast<int32_t>(tables->size(1)),
      tables->stride(0), ring->data_ptr<int32_t>(), state->data_ptr<int32_t>(), (state_out ? state_out : state)->data_ptr<int32_t>(),
      max_tokens, slots.data_ptr<int32_t>(), starts.data_ptr<int32_t>(), stream); });
  if (st != WK_OK) return PyLong_FromLong(st);
  return pair_of(slots, starts);
  END_HANDLE_TH_ERRORS
}

// (ctx, device, cache, K_new, V_new, slots, stream|None) -> None
PyObject* page_store(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 7) return said("wk_page_store: 7 arguments");
  Arguments a(args);
  wk_ctx* ctx = static_cast<wk_ctx*>(a.address());
  const int64_t device = a.whole();
  const wk_paged_kv* cache = static_cast<const wk_paged_kv*>(a.address());
  const at::Tensor *K = a.tensor("wk_page_store: K_new"), *V = a.tensor("wk_page_store: V_new"), *slots = a.tensor("wk_page_store: slots");
  if (PyErr_Occurred()) return nullptr;
  if (a.wrong) return said(a.wrong);
  if (!a.need(cache && rows(K, device) && rows(V, device) && K->size(1) == cache->n_kv_heads && K->size(2) == cache->head_dim &&
                  K->sizes() == V->sizes() && K->strides() == V->strides() && K->scalar_type() == V->scalar_type() &&
                  type_of(K->scalar_type()) >= 0,
              "wk_page_store: K_new, V_new [n, n_kv_heads, head_dim] alike, heads contiguous") ||
      !a.need(ints(slots, K->size(0), device), "wk_page_store: slots [n] int32"))
    return said(a.wrong);
  void* stream = a.stream(device);
  if (PyErr_Occurred()) return nullptr;
  const wk_status st = without_lock([&] { return call_store(ctx, cache, K->data_ptr(), V->data_ptr(), type_of(K->scalar_type()), static_cast<int32_t>(K->size(0)),
                                  K->stride(0), slots->data_ptr<int32_t>(), stream); });
  if (st != WK_OK) return PyLong_FromLong(st);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// (ctx, device, cache, Q, tables, lens, window, sink, softmax_scale, O|None, lse_out|None, scratch, stream|None) -> O
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 13) return said("wk_paged_attention: 13 arguments");
  Arguments a(args);
  wk_ctx* ctx = static_cast<wk_ctx*>(a.address());
  const int64_t device = a.whole();
  const wk_paged_kv* cache = static_cast<const wk_paged_kv*>(a.address());
  const at::Tensor *Q = a.tensor("wk_paged_attention: Q"), *tables = a.tensor("wk_paged_attention: tables"),
                   *lens = a.tensor("wk_paged_attention: lens");
  const int32_t window = a.whole32("wk_paged_attention: window"), sink = a.whole32("wk_paged_attention: sink");
  const float scale = static_cast<float>(a.real());
  const at::Tensor *O_in = a.tensor("wk_paged_attention: O", true), *lse = a.tensor("wk_paged_attention: lse_out", true),
                   *scratch = a.tensor("wk_paged_attention: scratch");
  if (PyErr_Occurred()) return nullptr;
  if (a.wrong) return said(a.wrong);
  if (!a.need(cache && rows(Q, device) && Q->size(2) == cache->head_dim && type_of(Q->scalar_type()) >= 0 &&
                  Q->size(1) <= std::numeric_limits<int32_t>::max(),
              "wk_paged_attention: Q [n_req, n_heads, head_dim], heads contiguous"))
    return said(a.wrong);
  const int64_t n = Q->size(0), heads = Q->size(1);
  if (!a.need(ints(lens, n, device), "wk_paged_attention: lens [n_req] int32") ||
      !a.need(table(tables, n, device), "wk_paged_attention: tables [n_req, max_pages] int32") ||
      !a.need(!O_in || (on(*O_in, device) && O_in->sizes() == Q->sizes() && O_in->scalar_type() == Q->scalar_type() && O_in->is_contiguous()),
              "wk_paged_attention: O like Q, contiguous") ||
      !a.need(!lse || (on(*lse, device) && lse->dim() == 2 && lse->size(0) == n && lse->size(1) == heads &&
                       lse->scalar_type() == at::kFloat && lse->is_contiguous()),
              "wk_paged_attention: lse_out [n_req, n_heads] fp32") ||
      !a.need(on(*scratch, device) && scratch->is_contiguous(), "wk_paged_attention: scratch"))
    return said(a.wrong);
  void* stream = a.stream(device);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor O = O_in ? *O_in : empty(Q->sizes(), *Q, a);
  if (n > 0) {
    const wk_status st = without_lock([&] { return call_attention(
        ctx, cache, Q->data_ptr(), type_of(Q->scalar_type()), Q->stride(0), static_cast<int32_t>(n), static_cast<int32_t>(heads),
        tables->data_ptr<int32_t>(), static_cast<int32_t>(tables->size(1)), tables->stride(0), lens->data_ptr<int32_t>(), window, sink,
        scale, O.data_ptr(), lse ? lse->data_ptr<float>() : nullptr, scratch->data_ptr(), scratch->nbytes(), stream); });
    if (st != WK_OK) return PyLong_FromLong(st);
  }
  return THPVariable_Wrap(O);
  END_HANDLE_TH_ERRORS
}

// The addresses of wk_page_plan, wk_page_store and wk_paged_attention in the library that is in use.
PyObject* use(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 3) return said("use: 3 addresses");
  call_plan = reinterpret_cast<decltype(call_plan)>(PyLong_AsVoidPtr(args[0]));
  call_store = reinterpret_cast<decltype(call_store)>(PyLong_AsVoidPtr(args[1]));
  call_attention = reinterpret_cast<decltype(call_attention)>(PyLong_AsVoidPtr(args[2]));
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"use", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(use)), METH_FASTCALL, nullptr},
    {"page_plan", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(page_plan)), METH_FASTCALL, nullptr},
    {"page_store", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(page_store)), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(paged_attention)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_pages", "Argument marshalling of the token-level cache's calls.", -1, methods,
                          nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__pages() { return PyModule_Create(&module_def); }
