// Native half of the binding: the calls a decode loop makes per token and per round (draft_entropy, draft_step,
// verify), argument marshalling only.  At one sequence the kernels of such a call take 5 to 20 us, and building
// the argument structs in Python took 5 to 12 us of host time per call, more than a drafting kernel runs.
// Here a drafting call takes 3.3 to 4 us of host time with its launch, a verification 9 us with its three.
//
// binding.py hands over the entry points of libadasd.so as it loaded it, and the Python objects that are needed
// to raise and to allocate; keyword arguments, defaults, checks and exceptions are those of its signatures.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/core/TensorImpl.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/adasd.h"

namespace {

struct Abi {
  decltype(&adasd_draft_entropy) draft_entropy;
  decltype(&adasd_draft_step) draft_step;
  decltype(&adasd_verify) verify;
  decltype(&adasd_verify_noalloc) verify_noalloc;
  decltype(&adasd_token_logprob) token_logprob;
  decltype(&adasd_token_logprob_grad) token_logprob_grad;
  decltype(&adasd_policy_loss) policy_loss;
  decltype(&adasd_preference_loss) preference_loss;
} g_abi;
PyObject* g_error = nullptr;         // AdasdError(code, where)
PyObject* g_alloc_result = nullptr;  // alloc_verify_result(B, K, device)
PyObject* g_policy_result = nullptr, *g_preference_result = nullptr;   // PolicyResult, PreferenceResult
PyObject* g_loss_workspace = nullptr;   // LossWorkspace

struct Fail {};                      // a Python exception is set

[[noreturn]] void fail(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw Fail{};
}
void check(int rc, const char* where) {
  if (rc == 0) return;
  PyObject* e = PyObject_CallFunction(g_error, "is", rc, where);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Fail{};
}

// Positional and keyword arguments into slots; the first `required` must be there.
template <int N>
void parse(const char* fn, PyObject* const (&names)[N], int required, PyObject* const* args, Py_ssize_t nargs, PyObject* kw,
           PyObject* (&slot)[N]) {
  if (nargs > N) {
    PyErr_Format(PyExc_TypeError, "%s() takes at most %d positional arguments (%zd given)", fn, N, nargs);
    throw Fail{};
  }
  for (int i = 0; i < N; ++i) slot[i] = i < nargs ? args[i] : nullptr;
  const Py_ssize_t nk = kw ? PyTuple_GET_SIZE(kw) : 0;
  for (Py_ssize_t k = 0; k < nk; ++k) {
    PyObject* name = PyTuple_GET_ITEM(kw, k);
    int at = -1;
    for (int i = 0; i < N && at < 0; ++i)
      if (names[i] == name) at = i;              // (both interned, as a rule)
    for (int i = 0; i < N && at < 0; ++i)
      if (PyUnicode_Compare(names[i], name) == 0) at = i;
    if (at < 0) {
      PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", fn, name);
      throw Fail{};
    }
    if (slot[at]) {
      PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%U'", fn, name);
      throw Fail{};
    }
    slot[at] = args[nargs + k];
  }
  for (int i = 0; i < required; ++i)
    if (!slot[i]) {
      PyErr_Format(PyExc_TypeError, "%s() missing required argument: '%U'", fn, names[i]);
      throw Fail{};
    }
}

uint64_t integer(PyObject* o, uint64_t fallback) {       // any Python integer, taken modulo 2^64
  if (!o) return fallback;
  const uint64_t v = PyLong_CheckExact(o) ? PyLong_AsUnsignedLongLongMask(o) : [&] {
    PyObject* i = PyNumber_Index(o);
    if (!i) throw Fail{};
    const uint64_t w = PyLong_AsUnsignedLongLongMask(i);
    Py_DECREF(i);
    return w;
  }();
  if (v == (uint64_t)-1 && PyErr_Occurred()) throw Fail{};
  return v;
}

struct Ref {                                              // attribute of an object, new reference
  PyObject* o;
  Ref(PyObject* from, PyObject* name) : o(PyObject_GetAttr(from, name)) {
    if (!o) throw Fail{};
  }
  ~Ref() { Py_DECREF(o); }
  Ref(const Ref&) = delete;
};
uint64_t int_attr(PyObject* from, PyObject* name) { return integer(Ref(from, name).o, 0); }

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a torch tensor", name);
    throw Fail{};
  }
  return THPVariable_Unpack(o);
}
const char* type_name(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return "torch.float32";
    case at::kInt: return "torch.int32";
    case at::kByte: return "torch.uint8";
    default: return "torch.float64";
  }
}
void* need(PyObject* o, at::ScalarType type, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must be a contiguous CUDA tensor of %s", name, type_name(type));
    throw Fail{};
  }
  return t.data_ptr();
}
void* maybe(PyObject* o, at::ScalarType type, const char* name) { return o && o != Py_None ? need(o, type, name) : nullptr; }
void* raw(PyObject* from, PyObject* name) {               // data pointer of a tensor attribute (NULL for None)
  Ref r(from, name);
  return r.o == Py_None ? nullptr : tensor(r.o, "state and result fields").data_ptr();
}
adasd_dtype logits_type(PyObject* o) {
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() == at::kBFloat16) return ADASD_BF16;
  if (t.scalar_type() == at::kFloat) return ADASD_F32;
  PyObject* type = PyObject_GetAttrString(o, "dtype");
  if (type) {
    PyErr_Format(PyExc_TypeError, "logits must be bfloat16 or float32, got %S", type);
    Py_DECREF(type);
  }
  throw Fail{};
}
PyObject* intern(const char* s) { return PyUnicode_InternFromString(s); }

struct Names {
  PyObject *ptr = intern("ptr"), *bytes = intern("bytes"), *B = intern("B"), *cap = intern("cap"), *T_G = intern("T_G"),
           *ent_sum = intern("ent_sum"), *ent_cnt = intern("ent_cnt"), *LA = intern("LA"), *LR = intern("LR"),
           *nA = intern("nA"), *nR = intern("nR"), *mom = intern("mom"), *n_accept = intern("n_accept"),
           *next_token = intern("next_token"), *H_p = intern("H_p"), *H_q = intern("H_q"), *d_js = intern("d_js"),
           *p_accept = intern("p_accept"), *accept_mask = intern("accept_mask"), *status = intern("status"),
           *base_test = intern("base_test"), *reject_rule = intern("reject_rule"), *kde_min_n = intern("kde_min_n"),
           *bw_rule = intern("bw_rule"), *relaxed_off = intern("relaxed_off"), *d_eps = intern("d_eps"),
           *stats_path = intern("stats_path"), *apply_update = intern("apply_update"), *list_update = intern("list_update"),
           *wait_polls = intern("wait_polls"), *buf = intern("buf"), *clip_low = intern("clip_low"), *clip_high = intern("clip_high"),
           *kl_coef = intern("kl_coef"), *entropy_coef = intern("entropy_coef"), *kind = intern("kind"), *beta = intern("beta"),
           *margin = intern("margin"), *label_smoothing = intern("label_smoothing");
};
Names* N = nullptr;

// The scratch of the losses and that of all other calls are laid out differently, and each has words that must be zero between calls.
bool of_losses(PyObject* workspace) { return PyObject_TypeCheck(workspace, (PyTypeObject*)g_loss_workspace); }
struct Scratch {
  void* ptr;
  size_t bytes;
  explicit Scratch(PyObject* workspace) {
    if (of_losses(workspace)) fail(PyExc_TypeError, "workspace must be a Workspace (a LossWorkspace is laid out differently)");
    ptr = (void*)int_attr(workspace, N->ptr);
    bytes = int_attr(workspace, N->bytes);
  }
};
void* stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }

// An output: the caller's tensor, checked, or a new one.
struct Output {
  PyObject* o;
  void* ptr;
  Output(PyObject* given, int64_t n, at::ScalarType type, const at::Tensor& like, const char* name) {
    if (given && given != Py_None) {
      ptr = need(given, type, name);
      o = given;
      Py_INCREF(o);
    } else {
      at::Tensor t = at::empty({n}, like.options().dtype(type));
      ptr = t.data_ptr();
      o = THPVariable_Wrap(std::move(t));
      if (!o) throw Fail{};
    }
  }
  ~Output() { Py_XDECREF(o); }
  Output(const Output&) = delete;
  PyObject* give() {
    PyObject* r = o;
    o = nullptr;
    return r;
  }
};


const at::Tensor& draft_rows(PyObject* o) {
  const at::Tensor& x = tensor(o, "draft_logits");
  if (x.dim() != 2 || !x.is_cuda() || x.stride(1) != 1)
    fail(PyExc_ValueError, "draft_logits must be a CUDA tensor [B, V] with contiguous vocabulary");
  return x;
}

template <class F> PyObject* guarded(F f) {
  try {
    return f();
  } catch (const Fail&) {
    return nullptr;
  } catch (...) {                      // out of memory, a failed stream look-up, ...: the classes that torch's own calls raise
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

PyObject* py_draft_entropy(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  return guarded([&]() -> PyObject* {
    static PyObject* const names[] = {intern("draft_logits"), intern("workspace"), intern("T_G"), intern("active"),
                                      intern("step"), intern("k_max"), intern("H_out"), intern("stop_out")};
    PyObject* a[8];
    parse("draft_entropy", names, 2, args, nargs, kw, a);
    const at::Tensor& x = draft_rows(a[0]);
    const int B = (int)x.size(0), V = (int)x.size(1);
    Output H(a[6], B, at::kFloat, x, "H_out"), stop(a[7], B, at::kByte, x, "stop_out");
    const float* tg = (const float*)maybe(a[2], at::kFloat, "T_G");
    const uint8_t* active = (const uint8_t*)maybe(a[3], at::kByte, "active");
    const adasd_dtype dt = logits_type(a[0]);
    const int step = (int)integer(a[4], 0), k_max = (int)integer(a[5], 1 << 30);
    const int64_t stride = B > 1 ? x.stride(0) : V;
    const Scratch scratch(a[1]);
    void *ws = scratch.ptr, *st = stream(), *rows = x.data_ptr();
    const size_t ws_bytes = scratch.bytes;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_abi.draft_entropy(rows, dt, B, V, stride, tg, active, step, k_max, (float*)H.ptr, (uint8_t*)stop.ptr, ws, ws_bytes, st);
    Py_END_ALLOW_THREADS
    check(rc, "adasd_draft_entropy");
    PyObject* r = PyTuple_New(2);
    if (!r) throw Fail{};
    PyTuple_SET_ITEM(r, 0, H.give());
    PyTuple_SET_ITEM(r, 1, stop.give());
    return r;
  });
}

PyObject* py_draft_step(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  return guarded([&]() -> PyObject* {
    static PyObject* const names[] = {intern("draft_logits"), intern("workspace"), intern("T_G"), intern("active"),
                                      intern("step"), intern("k_max"), intern("seed"), intern("seq_id"), intern("rounds"),
                                      intern("round0"), intern("H_out"), intern("stop_out"), intern("token_out"),
                                      intern("status_out")};
    PyObject* a[14];
    parse("draft_step", names, 2, args, nargs, kw, a);
    const at::Tensor& x = draft_rows(a[0]);
    const int B = (int)x.size(0), V = (int)x.size(1);
    const float* tg = (const float*)maybe(a[2], at::kFloat, "T_G");
    const uint8_t* active = (const uint8_t*)maybe(a[3], at::kByte, "active");
    const uint32_t* seq = (const uint32_t*)maybe(a[7], at::kInt, "seq_id");
    const uint32_t* rounds = (const uint32_t*)maybe(a[8], at::kInt, "rounds");
    Output H(a[10], B, at::kFloat, x, "H_out"), stop(a[11], B, at::kByte, x, "stop_out"),
        token(a[12], B, at::kInt, x, "token_out"), status(a[13], B, at::kInt, x, "status_out");
    const adasd_dtype dt = logits_type(a[0]);
    const int step = (int)integer(a[4], 0), k_max = (int)integer(a[5], 1 << 30);
    const uint64_t seed = integer(a[6], 0);
    const uint32_t round0 = (uint32_t)integer(a[9], 0);
    const int64_t stride = B > 1 ? x.stride(0) : V;
    const Scratch scratch(a[1]);
    void *ws = scratch.ptr, *st = stream(), *rows = x.data_ptr();
    const size_t ws_bytes = scratch.bytes;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_abi.draft_step(rows, dt, B, V, stride, tg, active, step, k_max, seed, seq, rounds, round0, (float*)H.ptr,
                          (uint8_t*)stop.ptr, (int32_t*)token.ptr, (uint32_t*)status.ptr, ws, ws_bytes, st);
    Py_END_ALLOW_THREADS
    check(rc, "adasd_draft_step");
    PyObject* r = PyTuple_New(4);
    if (!r) throw Fail{};
    PyTuple_SET_ITEM(r, 0, H.give());
    PyTuple_SET_ITEM(r, 1, stop.give());
    PyTuple_SET_ITEM(r, 2, token.give());
    PyTuple_SET_ITEM(r, 3, status.give());
    return r;
  });
}

PyObject* py_verify(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  return guarded([&]() -> PyObject* {
    static PyObject* const names[] = {intern("target_logits"), intern("draft_logits"), intern("draft_tokens"),
                                      intern("workspace"), intern("state"), intern("draft_len"), intern("seed"),
                                      intern("seq_id"), intern("rounds"), intern("round0"), intern("options"), intern("out")};
    PyObject* a[12];
    parse("verify", names, 4, args, nargs, kw, a);
    const at::Tensor &p = tensor(a[0], "target_logits"), &q = tensor(a[1], "draft_logits");
    if (p.dim() != 3 || q.dim() != 3) fail(PyExc_ValueError, "logits must be [B, k(+1), V]");
    const int64_t B = p.size(0), K = p.size(1) - 1, V = p.size(2);
    if (q.size(0) != B || q.size(1) != K || q.size(2) != V) {
      PyErr_Format(PyExc_ValueError, "draft_logits must be [%lld, %lld, %lld]", (long long)B, (long long)K, (long long)V);
      throw Fail{};
    }
    if (p.stride(2) != 1 || (K > 0 && q.stride(2) != 1)) fail(PyExc_ValueError, "vocabulary dimension must be contiguous");
    if (p.scalar_type() != q.scalar_type()) fail(PyExc_TypeError, "target and draft logits must share a dtype");
    adasd_verify_args v{};
    v.draft_tokens = (const int32_t*)need(a[2], at::kInt, "draft_tokens");
    v.draft_len = (const int32_t*)maybe(a[5], at::kInt, "draft_len");
    v.seq_id = (const uint32_t*)maybe(a[7], at::kInt, "seq_id");
    v.round = (const uint32_t*)maybe(a[8], at::kInt, "rounds");
    v.target_logits = p.data_ptr();
    v.draft_logits = q.data_ptr();
    v.dt = logits_type(a[0]);
    v.B = (int32_t)B;
    v.k_max = (int32_t)K;
    v.V = (int32_t)V;
    v.t_seq_stride = p.stride(0);
    v.t_pos_stride = p.stride(1);
    v.d_seq_stride = K > 0 ? q.stride(0) : V;
    v.d_pos_stride = K > 0 ? q.stride(1) : V;
    v.seed = integer(a[6], 0);
    v.round0 = (uint32_t)integer(a[9], 0);
    adasd_state s{};
    if (a[4] && a[4] != Py_None) {
      PyObject* o = a[4];
      s.B = (int32_t)int_attr(o, N->B);
      s.cap = (int32_t)int_attr(o, N->cap);
      s.T_G = (float*)raw(o, N->T_G);
      s.ent_sum = (double*)raw(o, N->ent_sum);
      s.ent_cnt = (int32_t*)raw(o, N->ent_cnt);
      s.LA = (float*)raw(o, N->LA);
      s.LR = (float*)raw(o, N->LR);
      s.nA = (int32_t*)raw(o, N->nA);
      s.nR = (int32_t*)raw(o, N->nR);
      s.mom = (double*)raw(o, N->mom);
      v.state = &s;
    }
    adasd_options opt{};
    const bool has_opt = a[10] && a[10] != Py_None;
    if (has_opt) {
      PyObject* o = a[10];
      opt.base_test = (int32_t)int_attr(o, N->base_test);
      opt.reject_rule = (int32_t)int_attr(o, N->reject_rule);
      opt.kde_min_n = (int32_t)int_attr(o, N->kde_min_n);
      opt.bw_rule = (int32_t)int_attr(o, N->bw_rule);
      opt.relaxed_off = (int32_t)int_attr(o, N->relaxed_off);
      const double eps = PyFloat_AsDouble(Ref(o, N->d_eps).o);
      if (eps == -1.0 && PyErr_Occurred()) throw Fail{};
      opt.d_eps = (float)eps;
      opt.stats_path = (int32_t)int_attr(o, N->stats_path);
      opt.apply_update = (int32_t)int_attr(o, N->apply_update);
      opt.list_update = (int32_t)int_attr(o, N->list_update);
      opt.wait_polls = (int32_t)int_attr(o, N->wait_polls);
    }
    PyObject* out = a[11];
    if (out && out != Py_None) {
      Py_INCREF(out);
    } else {
      PyObject* dev = PyObject_GetAttrString(a[0], "device");
      if (!dev) throw Fail{};
      out = PyObject_CallFunction(g_alloc_result, "LLN", (long long)B, (long long)K, dev);
      if (!out) throw Fail{};
    }
    struct Drop {
      PyObject* o;
      ~Drop() { Py_XDECREF(o); }
    } drop{out};
    v.n_accept = (int32_t*)raw(out, N->n_accept);
    v.next_token = (int32_t*)raw(out, N->next_token);
    v.H_p = (float*)raw(out, N->H_p);
    v.H_q = (float*)raw(out, N->H_q);
    v.d_js = (float*)raw(out, N->d_js);
    v.p_accept = (float*)raw(out, N->p_accept);
    v.accept_mask = (uint8_t*)raw(out, N->accept_mask);
    v.status = (uint32_t*)raw(out, N->status);
    const bool noalloc = a[3] == Py_None;
    if (!noalloc) {
      const Scratch scratch(a[3]);
      v.workspace = scratch.ptr;
      v.ws_bytes = scratch.bytes;
    }
    void* st = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = (noalloc ? g_abi.verify_noalloc : g_abi.verify)(&v, has_opt ? &opt : nullptr, st);
    Py_END_ALLOW_THREADS
    check(rc, noalloc ? "adasd_verify_noalloc" : "adasd_verify");
    drop.o = nullptr;
    return out;
  });
}

// ---- log-probabilities and losses over vocabulary rows

bool given(PyObject* o) { return o && o != Py_None; }
float float_attr(PyObject* from, PyObject* name) {
  const double v = PyFloat_AsDouble(Ref(from, name).o);
  if (v == -1.0 && PyErr_Occurred()) throw Fail{};
  return (float)v;
}

// The rows of a call: logits [B, T, V] with tokens [B, T], or [B, V] with [B]; outputs are allocated in the shape of the tokens.
struct RowsCall {
  adasd_rows rows{};
  const at::Tensor* z;
  int64_t shape[2];
  int dims;
  void* stream;
  c10::Allocator* allocator;
  const at::Tensor* written[4];           // (the gradient, or the three results of a log-probability call)
  int n_written = 0;
  c10::hip::OptionalHIPGuard guard;       // the calls run on the logits' device, whatever the current one is

  RowsCall(PyObject* logits, PyObject* tokens, PyObject* workspace, bool only_sequences) {
    if (!THPVariable_Check(logits) || (z = &THPVariable_Unpack(logits), (z->dim() != 3 && (only_sequences || z->dim() != 2))) || !z->is_cuda())
      fail(PyExc_ValueError, only_sequences ? "logits must be a CUDA tensor [2P, T, V]" : "logits must be a CUDA tensor [B, T, V] or [B, V]");
    rows.dt = logits_type(logits);
    dims = (int)z->dim() - 1;
    const int64_t V = z->size(dims);
    if (V > 1 && z->stride(dims) != 1) fail(PyExc_ValueError, "vocabulary dimension must be contiguous");
    shape[0] = z->size(0);
    shape[1] = dims == 2 ? z->size(1) : 1;
    if (shape[0] > INT32_MAX || shape[1] > INT32_MAX || V > INT32_MAX) fail(PyExc_ValueError, "logits have too many positions");
    rows.B = (int32_t)shape[0];
    rows.T = (int32_t)shape[1];
    rows.V = (int32_t)V;
    rows.logits = z->data_ptr();
    rows.seq_stride = z->stride(0);
    rows.pos_stride = dims == 2 ? z->stride(1) : V;
    rows.tokens = (const int32_t*)input(tokens, at::kInt, "tokens");
    if (!of_losses(workspace)) fail(PyExc_TypeError, "workspace must be a LossWorkspace");
    Ref buf(workspace, N->buf);
    if (tensor(buf.o, "workspace.buf").device() != z->device()) fail(PyExc_ValueError, "workspace must be on the logits' device");
    allocator = THPVariable_Unpack(buf.o).storage().allocator();
    rows.workspace = (void*)int_attr(workspace, N->ptr);
    rows.ws_bytes = int_attr(workspace, N->bytes);
    guard.set_index(z->get_device());
    stream = ::stream();
  }
  // A contiguous input of this shape on the logits' device.
  void* input(PyObject* o, at::ScalarType type, const char* name, const int64_t* size, int n) const {
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous()) {
      PyErr_Format(PyExc_ValueError, "%s must be a contiguous CUDA tensor of %s", name, type_name(type));
      throw Fail{};
    }
    bool same = t.dim() == n;
    for (int i = 0; same && i < n; ++i) same = t.size(i) == size[i];
    if (!same || t.device() != z->device()) {
      PyErr_Format(PyExc_ValueError, n == 2 ? "%s must be [%lld, %lld] on the logits' device" : "%s must be [%lld] on the logits' device", name,
                   (long long)size[0], n == 2 ? (long long)size[1] : 0ll);
      throw Fail{};
    }
    return t.data_ptr();
  }
  void* input(PyObject* o, at::ScalarType type, const char* name) const { return input(o, type, name, shape, dims); }
  void* maybe(PyObject* o, at::ScalarType type, const char* name) const { return given(o) ? input(o, type, name) : nullptr; }
  const float* one(PyObject* o, int64_t n, const char* name) const { return given(o) ? (const float*)input(o, at::kFloat, name, &n, 1) : nullptr; }

  // The caller's tensors that the call writes to: torch learns of it as of its own writes in place (a backward pass that needs what was there
  // then says so).  Inference tensors keep no count.
  void written_to(const at::Tensor& t) { written[n_written++] = &t; }
  void enqueued() const {
    for (int i = 0; i < n_written; ++i)
      if (!written[i]->is_inference()) written[i]->unsafeGetTensorImpl()->bump_version();
  }

  // A new result, as at::empty makes one, from the workspace's allocator (without the dispatcher's part: calls of one token are short).
  at::Tensor result(at::IntArrayRef sizes, at::ScalarType t) const {
    if (!allocator) return at::empty(sizes, z->options().dtype(t));
    int64_t bytes = 4;                         // (every result has elements of 4 bytes)
    for (int64_t d : sizes) bytes *= d;
    auto storage = c10::make_intrusive<c10::StorageImpl>(c10::StorageImpl::use_byte_size_t(), bytes, allocator->allocate(bytes), allocator, true);
    auto made = c10::make_intrusive<c10::TensorImpl>(c10::Storage(std::move(storage)), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                     c10::scalarTypeToTypeMeta(t));
    made->set_sizes_contiguous(sizes);
    return at::Tensor(std::move(made));
  }

  // The gradient: the caller's tensor (any strides with a contiguous vocabulary), or a new one.  New reference.
  PyObject* gradient(PyObject* o) {
    if (given(o)) {
      const at::Tensor& g = tensor(o, "dlogits");
      if (g.device() != z->device() || g.scalar_type() != z->scalar_type() || g.sizes() != z->sizes() || (rows.V > 1 && g.stride(dims) != 1))
        fail(PyExc_ValueError, "dlogits must have the shape, type and device of the logits and a contiguous vocabulary");
      place(g);
      written_to(g);
      Py_INCREF(o);
      return o;
    }
    at::Tensor g = at::empty(z->sizes(), z->options());
    place(g);
    return wrap(std::move(g));
  }
  void place(const at::Tensor& g) {
    rows.dlogits = g.data_ptr();
    rows.d_seq_stride = g.stride(0);
    rows.d_pos_stride = dims == 2 ? g.stride(1) : rows.V;
  }
  static PyObject* wrap(at::Tensor t) {
    PyObject* o = THPVariable_Wrap(std::move(t));
    if (!o) throw Fail{};
    return o;
  }
};

// Results to be handed over together: the caller's tensors, or new ones, each with a storage of its own (results are kept and saved one by
// one: parts of one allocation would keep and save all of it, and torch does not save parts of different types).
template <int M> struct Results {
  RowsCall& c;
  PyObject* o[M] = {};
  int n = 0;
  explicit Results(RowsCall& call) : c(call) {}
  ~Results() {
    for (int i = 0; i < n; ++i) Py_XDECREF(o[i]);
  }
  Results(const Results&) = delete;
  int add(PyObject* p) {                       // an object as it is
    o[n] = p;
    return n++;
  }
  int make(at::IntArrayRef sizes, at::ScalarType t) { return add(RowsCall::wrap(c.result(sizes, t))); }
  int take(PyObject* given_one, at::ScalarType t, const char* name) {      // the caller's, in the shape of the tokens, or a new one
    if (!given(given_one)) return make(at::IntArrayRef(c.shape, c.dims), t);
    c.input(given_one, t, name);
    c.written_to(THPVariable_Unpack(given_one));
    Py_INCREF(given_one);
    return add(given_one);
  }
  template <class T> T* ptr(int i) const { return (T*)THPVariable_Unpack(o[i]).data_ptr(); }
  PyObject* tuple() {
    PyObject* r = PyTuple_New(n);
    if (!r) throw Fail{};
    for (int i = 0; i < n; ++i) PyTuple_SET_ITEM(r, i, o[i]);
    n = 0;
    return r;
  }
  PyObject* call(PyObject* result) {
    PyObject* r = PyObject_Vectorcall(result, o, n, nullptr);
    if (!r) throw Fail{};
    return r;
  }
};
template <class F> void enqueue(const char* where, const RowsCall& c, F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  check(rc, where);
  c.enqueued();
}
bool truth(PyObject* o, bool fallback) {
  if (!o) return fallback;
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Fail{};
  return v != 0;
}

PyObject* py_token_logprob(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  return guarded([&]() -> PyObject* {
    static PyObject* const names[] = {intern("logits"), intern("tokens"), intern("workspace"), intern("active"),
                                      intern("logprob_out"), intern("entropy_out"), intern("status_out")};
    PyObject* a[7];
    parse("token_logprob", names, 3, args, nargs, kw, a);
    RowsCall c(a[0], a[1], a[2], false);
    c.rows.active = (const uint8_t*)c.maybe(a[3], at::kByte, "active");
    Results<3> out(c);
    out.take(a[4], at::kFloat, "logprob_out");
    out.take(a[5], at::kFloat, "entropy_out");
    out.take(a[6], at::kInt, "status_out");
    c.rows.logprob = out.ptr<float>(0);
    c.rows.entropy = out.ptr<float>(1);
    c.rows.status = out.ptr<uint32_t>(2);
    enqueue("adasd_token_logprob", c, [&] { return g_abi.token_logprob(&c.rows, c.stream); });
    return out.tuple();
  });
}

PyObject* py_token_logprob_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  return guarded([&]() -> PyObject* {
    static PyObject* const names[] = {intern("logits"), intern("tokens"), intern("workspace"), intern("dlogprob"),
                                      intern("dentropy"), intern("active"), intern("dlogits")};
    PyObject* a[7];
    parse("token_logprob_grad", names, 4, args, nargs, kw, a);
    RowsCall c(a[0], a[1], a[2], false);
    const float* dlp = (const float*)c.input(a[3], at::kFloat, "dlogprob");
    const float* dent = (const float*)c.maybe(a[4], at::kFloat, "dentropy");
    c.rows.active = (const uint8_t*)c.maybe(a[5], at::kByte, "active");
    Results<1> out(c);
    out.add(c.gradient(a[6]));
    enqueue("adasd_token_logprob_grad", c, [&] { return g_abi.token_logprob_grad(&c.rows, dlp, dent, c.stream); });
    out.n = 0;
    return out.o[0];
  });
}

PyObject* py_policy_loss(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  return guarded([&]() -> PyObject* {
    static PyObject* const names[] = {intern("logits"), intern("tokens"), intern("advantage"), intern("workspace"), intern("weight"),
                                      intern("old_logprob"), intern("ref_logprob"), intern("ref_logits"), intern("options"),
                                      intern("grad_scale"), intern("need_grad"), intern("dlogits")};
    PyObject* a[12];
    parse("policy_loss", names, 4, args, nargs, kw, a);
    RowsCall c(a[0], a[1], a[3], false);
    adasd_policy_args p{};
    p.adv_per_seq = c.dims == 2 && tensor(a[2], "advantage").dim() == 1;
    p.advantage = p.adv_per_seq ? c.one(a[2], c.shape[0], "advantage") : (const float*)c.input(a[2], at::kFloat, "advantage");
    c.rows.weight = (const float*)c.maybe(a[4], at::kFloat, "weight");
    p.old_logprob = (const float*)c.maybe(a[5], at::kFloat, "old_logprob");
    p.ref_logprob = (const float*)c.maybe(a[6], at::kFloat, "ref_logprob");
    if (given(a[7])) {
      const at::Tensor& q = tensor(a[7], "ref_logits");
      if (q.device() != c.z->device() || q.scalar_type() != c.z->scalar_type() || q.sizes() != c.z->sizes() ||
          (c.rows.V > 1 && q.stride(c.dims) != 1))
        fail(PyExc_ValueError, "ref_logits must have the shape, type and device of the logits and a contiguous vocabulary");
      p.ref_logits = q.data_ptr();
      p.r_seq_stride = q.stride(0);
      p.r_pos_stride = c.dims == 2 ? q.stride(1) : c.rows.V;
    }
    p.clip_low = p.clip_high = 0.2f;
    if (given(a[8])) {
      p.clip_low = float_attr(a[8], N->clip_low);
      p.clip_high = float_attr(a[8], N->clip_high);
      p.kl_coef = float_attr(a[8], N->kl_coef);
      p.entropy_coef = float_attr(a[8], N->entropy_coef);
    }
    p.grad_scale = c.one(a[9], 1, "grad_scale");
    Results<7> out(c);
    const at::IntArrayRef size(c.shape, c.dims);
    out.make({}, at::kFloat);
    for (int i = 1; i < 5; ++i) out.make(size, at::kFloat);
    out.make(size, at::kInt);
    p.loss = out.ptr<float>(0);
    p.token_loss = out.ptr<float>(1);
    c.rows.logprob = out.ptr<float>(2);
    c.rows.entropy = out.ptr<float>(3);
    p.kl = out.ptr<float>(4);
    c.rows.status = out.ptr<uint32_t>(5);
    out.add(truth(a[10], true) ? c.gradient(a[11]) : Py_NewRef(Py_None));
    enqueue("adasd_policy_loss", c, [&] { return g_abi.policy_loss(&c.rows, &p, c.stream); });
    return out.call(g_policy_result);
  });
}

PyObject* py_preference_loss(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  return guarded([&]() -> PyObject* {
    static PyObject* const names[] = {intern("logits"), intern("tokens"), intern("workspace"), intern("weight"), intern("ref_logprob"),
                                      intern("pair_weight"), intern("options"), intern("grad_scale"), intern("need_grad"), intern("dlogits")};
    PyObject* a[10];
    parse("preference_loss", names, 3, args, nargs, kw, a);
    RowsCall c(a[0], a[1], a[2], true);
    adasd_preference_args p{};
    const int64_t P = c.shape[0] / 2;
    c.rows.weight = (const float*)c.maybe(a[3], at::kFloat, "weight");
    p.ref_logprob = (const float*)c.maybe(a[4], at::kFloat, "ref_logprob");
    p.pair_weight = c.one(a[5], P, "pair_weight");
    p.beta = 0.1f;
    if (given(a[6])) {
      static const char* const kinds[] = {"logistic", "squared", "hinge"};
      Ref kind(a[6], N->kind);
      p.kind = -1;
      for (int i = 0; i < 3; ++i)
        if (PyUnicode_Check(kind.o) && PyUnicode_CompareWithASCIIString(kind.o, kinds[i]) == 0) p.kind = i;
      if (p.kind < 0) fail(PyExc_ValueError, "kind must be 'logistic', 'squared' or 'hinge'");
      p.beta = float_attr(a[6], N->beta);
      p.margin = float_attr(a[6], N->margin);
      p.label_smoothing = float_attr(a[6], N->label_smoothing);
    }
    p.grad_scale = c.one(a[7], 1, "grad_scale");
    Results<7> out(c);
    out.make({}, at::kFloat);
    for (int i = 1; i < 3; ++i) out.make(at::IntArrayRef(&P, 1), at::kFloat);
    out.make(at::IntArrayRef(c.shape, 1), at::kFloat);
    out.make(at::IntArrayRef(c.shape, 2), at::kFloat);
    out.make(at::IntArrayRef(c.shape, 2), at::kInt);
    p.loss = out.ptr<float>(0);
    p.pair_loss = out.ptr<float>(1);
    p.pair_margin = out.ptr<float>(2);
    p.score = out.ptr<float>(3);
    c.rows.logprob = out.ptr<float>(4);
    c.rows.status = out.ptr<uint32_t>(5);
    out.add(truth(a[8], true) ? c.gradient(a[9]) : Py_NewRef(Py_None));
    enqueue("adasd_preference_loss", c, [&] { return g_abi.preference_loss(&c.rows, &p, c.stream); });
    return out.call(g_preference_result);
  });
}

// connect_losses(PolicyResult, PreferenceResult, LossWorkspace, addresses of token_logprob, token_logprob_grad, policy_loss, preference_loss)
PyObject* py_connect_losses(PyObject*, PyObject* args) {
  PyObject *policy, *preference, *workspace;
  unsigned long long f[4];
  if (!PyArg_ParseTuple(args, "OOO!KKKK", &policy, &preference, &PyType_Type, &workspace, &f[0], &f[1], &f[2], &f[3])) return nullptr;
  Py_INCREF(policy);
  Py_INCREF(preference);
  Py_XSETREF(g_policy_result, policy);
  Py_INCREF(workspace);
  Py_XSETREF(g_preference_result, preference);
  Py_XSETREF(g_loss_workspace, workspace);
  g_abi.token_logprob = (decltype(g_abi.token_logprob))f[0];
  g_abi.token_logprob_grad = (decltype(g_abi.token_logprob_grad))f[1];
  g_abi.policy_loss = (decltype(g_abi.policy_loss))f[2];
  g_abi.preference_loss = (decltype(g_abi.preference_loss))f[3];
  Py_RETURN_NONE;
}

// connect(error class, result allocator, addresses of draft_entropy, draft_step, verify, verify_noalloc)
PyObject* py_connect(PyObject*, PyObject* args) {
  PyObject *err, *alloc;
  unsigned long long f[4];
  if (!PyArg_ParseTuple(args, "OOKKKK", &err, &alloc, &f[0], &f[1], &f[2], &f[3])) return nullptr;
  Py_INCREF(err);
  Py_INCREF(alloc);
  Py_XSETREF(g_error, err);
  Py_XSETREF(g_alloc_result, alloc);
  g_abi.draft_entropy = (decltype(g_abi.draft_entropy))f[0];
  g_abi.draft_step = (decltype(g_abi.draft_step))f[1];
  g_abi.verify = (decltype(g_abi.verify))f[2];
  g_abi.verify_noalloc = (decltype(g_abi.verify_noalloc))f[3];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"draft_entropy", (PyCFunction)(void (*)(void))py_draft_entropy, METH_FASTCALL | METH_KEYWORDS, nullptr},
    {"draft_step", (PyCFunction)(void (*)(void))py_draft_step, METH_FASTCALL | METH_KEYWORDS, nullptr},
    {"verify", (PyCFunction)(void (*)(void))py_verify, METH_FASTCALL | METH_KEYWORDS, nullptr},
    {"token_logprob", (PyCFunction)(void (*)(void))py_token_logprob, METH_FASTCALL | METH_KEYWORDS, nullptr},
    {"token_logprob_grad", (PyCFunction)(void (*)(void))py_token_logprob_grad, METH_FASTCALL | METH_KEYWORDS, nullptr},
    {"policy_loss", (PyCFunction)(void (*)(void))py_policy_loss, METH_FASTCALL | METH_KEYWORDS, nullptr},
    {"preference_loss", (PyCFunction)(void (*)(void))py_preference_loss, METH_FASTCALL | METH_KEYWORDS, nullptr},
    {"connect_losses", py_connect_losses, METH_VARARGS, nullptr},
    {"connect", py_connect, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
  N = new Names;
  return PyModule_Create(&module);
}
