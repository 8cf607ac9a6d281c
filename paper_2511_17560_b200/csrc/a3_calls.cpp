// The decoding calls of the Python binding, compiled: a3_paged_append, a3_paged_attention and a3_token_logprobs take 2-10 us on the device, and
// looking at some ten tensors from Python took longer than that.  Each function checks its tensors, allocates the results with torch, fills
// the header's struct and makes the one call.  It is given the address of the library's function, so that it links against torch alone.
//
// Measured on the host, launch included, with the same checks in Python and here: one appended row 7.7 and 3.6 us, one short sequence 11.1 and
// 5.8, one of 5 153 slots (two launches) 15.3 and 8.6, one row of logits with five alternatives (four results) 13.3 and 7.7.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <limits.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "a3.h"

namespace {

PyObject* error_class = nullptr;  // A3Error(status, where)

struct Refused {
  int status;
  const char* where;
};
void need(bool ok, const char* where) {
  if (!ok) throw Refused{A3_EINVAL, where};
}
const at::Tensor& tensor(PyObject* o, const char* where) {
  need(THPVariable_Check(o), where);
  return THPVariable_Unpack(o);
}
const at::Tensor* tensor_or_none(PyObject* o, const char* where) { return o == Py_None ? nullptr : &tensor(o, where); }
void* address(PyObject* o) {
  void* p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
  if (PyErr_Occurred()) throw python_error();
  return p;
}
int integer(PyObject* o) {
  const long x = PyLong_AsLong(o);
  if (PyErr_Occurred()) throw python_error();
  need(x >= INT_MIN && x <= INT_MAX, "a number out of range");
  return (int)x;
}
c10::Device device_of(PyObject* o) {
  need(THPDevice_Check(o), "a device");
  return ((THPDevice*)o)->device;
}
bool indices(const at::Tensor& t, int64_t dim, c10::Device dev) {
  return t.dim() == dim && t.scalar_type() == at::kInt && t.device() == dev && t.is_contiguous();
}
// [rows][heads][d] in bf16, the heads of a row next to each other
bool rows_of(const at::Tensor& t, int64_t rows, int64_t heads, int64_t d, c10::Device dev) {
  return t.dim() == 3 && t.size(0) == rows && t.size(1) == heads && t.size(2) == d && t.scalar_type() == at::kBFloat16 && t.device() == dev &&
         (rows == 0 || (t.stride(2) == 1 && (t.stride(1) == d || heads == 1)));
}
// elements from row to row; a row alone has no next one
uint64_t row_stride(const at::Tensor& t, int64_t width) { return t.size(0) > 1 ? (uint64_t)t.stride(0) : (uint64_t)width; }
void counts(int64_t a, int64_t b = 0) { need(a <= INT_MAX && b <= INT_MAX, "a size out of range"); }

// As every call through ctypes does: other Python threads run while a launch waits for room in its queue.
template <typename F, typename... A>
void call(PyObject* fn, const char* where, A... args) {
  const F f = (F)address(fn);
  need(f != nullptr, where);
  PyThreadState* state = PyEval_SaveThread();
  const int status = f(args...);
  PyEval_RestoreThread(state);
  if (status != A3_OK) throw Refused{status, where};
}

template <typename Body>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, Body body) {
  HANDLE_TH_ERRORS
  try {
    need(given == wanted, "number of arguments");
    return body();
  } catch (const Refused& r) {
    PyObject* e = PyObject_CallFunction(error_class, "is", r.status, r.where);
    if (e) {
      PyErr_SetObject(error_class, e);
      Py_DECREF(e);
    }
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* none() { return Py_NewRef(Py_None); }

// (function, handle, cache, stream, device, Hq, Hkv, D, page_table, row_seq, row_slot, k_rows, v_rows, q_rows, row_pos, rotate, q_out) -> q_out
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 17, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[4]);
    const int64_t hq = integer(a[5]), hkv = integer(a[6]), d = integer(a[7]);
    const char* where = "a3_paged_append: contiguous int32 page table and rows on the engine's device";
    const at::Tensor &table = tensor(a[8], where), &seq = tensor(a[9], where), &slot = tensor(a[10], where);
    need(indices(table, 2, dev) && indices(seq, 1, dev) && indices(slot, 1, dev) && slot.size(0) == seq.size(0), where);
    const int64_t M = seq.size(0);
    const at::Tensor* pos = tensor_or_none(a[14], "a3_paged_append: row_pos");
    need(!pos || (indices(*pos, 1, dev) && pos->size(0) == M), "a3_paged_append: row_pos");
    where = "a3_paged_append: k_rows, v_rows: bf16 [M][Hkv][D] on the engine's device, the heads of a row next to each other";
    const at::Tensor &k = tensor(a[11], where), &v = tensor(a[12], where);
    need(rows_of(k, M, hkv, d, dev) && rows_of(v, M, hkv, d, dev), where);
    where = "a3_paged_append: q_rows, q_out: bf16 [M][Hq][D] on the engine's device, the heads of a row next to each other";
    const at::Tensor *q = tensor_or_none(a[13], where), *given = tensor_or_none(a[16], where);
    at::Tensor made;
    need(q || !given, "a3_paged_append: q_out without q_rows");
    if (q) {
      need(rows_of(*q, M, hq, d, dev) && (!given || rows_of(*given, M, hq, d, dev)), where);
      if (!given) made = at::empty({M, hq, d}, q->options());
    }
    const at::Tensor* out = given ? given : q ? &made : nullptr;
    counts(M);
    counts(table.size(0), table.size(1));
    const int rotate = PyObject_IsTrue(a[15]);
    if (rotate < 0) throw python_error();
    a3_paged_rows r{};
    r.page_table = (const int32_t*)table.data_ptr(), r.row_seq = (const int32_t*)seq.data_ptr(), r.row_slot = (const int32_t*)slot.data_ptr();
    r.row_pos = pos ? (const int32_t*)pos->data_ptr() : nullptr;
    r.k_rows = k.data_ptr(), r.v_rows = v.data_ptr();
    r.k_stride = row_stride(k, hkv * d), r.v_stride = row_stride(v, hkv * d);
    if (q) r.q_rows = q->data_ptr(), r.q_out = out->data_ptr(), r.q_stride = row_stride(*q, hq * d), r.q_out_stride = row_stride(*out, hq * d);
    r.n_seqs = (int32_t)table.size(0), r.max_pages = (int32_t)table.size(1), r.M = (int32_t)M, r.rotate = rotate;
    call<decltype(&a3_paged_append)>(a[0], "a3_paged_append", (const a3_handle*)address(a[1]), (const a3_paged_cache*)address(a[2]), (const a3_paged_rows*)&r,
                                     (a3_stream)address(a[3]));
    if (given) return Py_NewRef(a[16]);
    return q ? wrap(made) : none();
  });
}

// (function, function for the workspace, handle, cache, stream, device, Hq, D, page_table, cache_len, q_rows, scale, out, want_lse) -> (out, lse)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[5]);
    const int64_t hq = integer(a[6]), d = integer(a[7]);
    const char* where = "a3_paged_attention: contiguous int32 page table and lengths on the engine's device";
    const at::Tensor &table = tensor(a[8], where), &lens = tensor(a[9], where);
    need(indices(table, 2, dev) && indices(lens, 1, dev) && lens.size(0) == table.size(0), where);
    const int64_t n_seqs = table.size(0);
    where = "a3_paged_attention: q_rows: bf16 [n_seqs][Hq][D] on the engine's device, the heads of a row next to each other";
    const at::Tensor& q = tensor(a[10], where);
    need(rows_of(q, n_seqs, hq, d, dev), where);
    const at::Tensor* given = tensor_or_none(a[12], "a3_paged_attention: out");
    need(!given || (rows_of(*given, n_seqs, hq, d, dev) && given->is_contiguous()), "a3_paged_attention: out");
    counts(n_seqs, table.size(1));
    const double scale = PyFloat_AsDouble(a[11]);
    if (PyErr_Occurred()) throw python_error();
    const int want_lse = PyObject_IsTrue(a[13]);
    if (want_lse < 0) throw python_error();
    const at::Tensor out = given ? *given : at::empty({n_seqs, hq, d}, q.options());
    at::Tensor lse, ws;
    if (want_lse) lse = at::empty({n_seqs, hq}, q.options().dtype(at::kFloat));
    const auto* h = (const a3_handle*)address(a[2]);
    const auto* cache = (const a3_paged_cache*)address(a[3]);
    const auto room = (decltype(&a3_paged_attention_workspace_bytes))address(a[1]);
    need(room != nullptr, "a3_paged_attention");
    a3_paged_queries p{};
    p.n_seqs = (int32_t)n_seqs, p.max_pages = (int32_t)table.size(1);
    if ((p.ws_bytes = room(h, cache, p.n_seqs, p.max_pages)) > 0) {
      ws = at::empty({(int64_t)p.ws_bytes}, q.options().dtype(at::kByte));
      p.ws = ws.data_ptr();
    }
    p.page_table = (const int32_t*)table.data_ptr(), p.cache_len = (const int32_t*)lens.data_ptr();
    p.q_rows = q.data_ptr(), p.q_stride = row_stride(q, hq * d);
    p.out = out.data_ptr(), p.lse_out = want_lse ? (float*)lse.data_ptr() : nullptr;
    p.scale = (float)scale;
    call<decltype(&a3_paged_attention)>(a[0], "a3_paged_attention", h, cache, (const a3_paged_queries*)&p, (a3_stream)address(a[4]));
    return Py_BuildValue("(NN)", given ? Py_NewRef(a[12]) : wrap(out), want_lse ? wrap(lse) : none());
  });
}

// (function, handle, stream, device, logits, targets, n_top) -> (logprob, entropy, top_ids, top_logprobs)
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[3]);
    const char* where = "a3_token_logprobs: logits: fp32, bf16 or fp16 [M][vocab] on the engine's device, the logits of a row next to each other";
    const at::Tensor& x = tensor(a[4], where);
    const auto type = x.scalar_type();
    need((type == at::kFloat || type == at::kBFloat16 || type == at::kHalf) && x.dim() == 2 && x.device() == dev, where);
    const int64_t M = x.size(0), vocab = x.size(1);
    need(vocab > 0 && (x.stride(1) == 1 || vocab == 1), where);
    counts(M, vocab);
    const at::Tensor* targets = tensor_or_none(a[5], "a3_token_logprobs: targets");
    need(!targets || (indices(*targets, 1, dev) && targets->size(0) == M), "a3_token_logprobs: targets: contiguous int32 [M] on the engine's device");
    const int n_top = integer(a[6]);
    const auto fp32 = x.options().dtype(at::kFloat);
    at::Tensor logprob, entropy = at::empty({M}, fp32), ids, lps;
    a3_logit_rows r{};
    if (targets) {
      logprob = at::empty({M}, fp32);
      r.targets = (const int32_t*)targets->data_ptr(), r.logprob_out = (float*)logprob.data_ptr();
    }
    if (n_top > 0 && n_top <= A3_LOGPROBS_MAX_TOP) {  // the library refuses more
      ids = at::empty({M, n_top}, x.options().dtype(at::kInt));
      lps = at::empty({M, n_top}, fp32);
      r.top_ids_out = (int32_t*)ids.data_ptr(), r.top_logprobs_out = (float*)lps.data_ptr();
    }
    r.logits = x.data_ptr(), r.entropy_out = (float*)entropy.data_ptr();
    r.row_stride = row_stride(x, vocab);
    r.type = type == at::kFloat ? A3_LOGITS_FP32 : type == at::kBFloat16 ? A3_LOGITS_BF16 : A3_LOGITS_FP16;
    r.M = (int32_t)M, r.vocab = (int32_t)vocab, r.n_top = n_top;
    call<decltype(&a3_token_logprobs)>(a[0], "a3_token_logprobs", (const a3_handle*)address(a[1]), (const a3_logit_rows*)&r, (a3_stream)address(a[2]));
    return Py_BuildValue("(NNNN)", targets ? wrap(logprob) : none(), wrap(entropy), n_top > 0 ? wrap(ids) : none(), n_top > 0 ? wrap(lps) : none());
  });
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_XSETREF(error_class, Py_NewRef(cls));
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"paged_append", (PyCFunction)(void (*)(void))paged_append, METH_FASTCALL, nullptr},
                         {"paged_attention", (PyCFunction)(void (*)(void))paged_attention, METH_FASTCALL, nullptr},
                         {"token_logprobs", (PyCFunction)(void (*)(void))token_logprobs, METH_FASTCALL, nullptr},
                         {"set_error", set_error, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "a3_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_a3_calls() {
  PyObject* m = PyModule_Create(&module);
  // tensors are looked at through torch's own classes: of another version even what links may lie elsewhere
  if (m && PyModule_AddStringConstant(m, "torch_version", A3_TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}
