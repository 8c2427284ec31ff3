// Argument checks and marshalling of the verification-step operators between torch tensors and the C ABI.  These calls sit in a
// serving loop, several per layer, and the smallest kernels take 4 us: with a ctypes call of thirty arguments and a dozen tensors
// checked in Python a call cost its caller 12 - 27 us, from here, launches and the Python wrapper included, 3 - 8 us.  No arithmetic, no
// kernels: the functions of libswiftkv.so arrive as addresses through bind().
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <sstream>
#include <stdexcept>
#include <string>

#include "../../include/swiftkv.h"

namespace {

using at::Tensor;

// ---- the library's functions ---------------------------------------------------------------------------------
#define FUNCTIONS(X)                                                                                                    \
  X(swiftkv_last_error) X(swiftkv_plan_pages) X(swiftkv_qk_norm_rope) X(swiftkv_qk_norm_rope_bwd)                       \
  X(swiftkv_qk_norm_rope_bwd_scratch_bytes) X(swiftkv_tree_attention) X(swiftkv_tree_attention_scratch_bytes)           \
  X(swiftkv_token_logprobs) X(swiftkv_token_logprobs_bwd)
#define X(name) decltype(&::name) p_##name = nullptr;
FUNCTIONS(X)
#undef X
PyObject *g_error = nullptr;      // SwiftKVError

struct Refused : std::runtime_error { using std::runtime_error::runtime_error; };      // -> ValueError
struct Raised {};                                                                      // a Python error is set

void check(int32_t rc) {
  if (rc == 0) return;
  PyObject *e = PyObject_CallFunction(g_error, "is", (int)rc, p_swiftkv_last_error());
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Raised();
}

// ---- checks ----------------------------------------------------------------------------------------------------
std::string said(const Tensor &t) {
  std::ostringstream s;
  s << t.scalar_type() << " " << t.sizes() << " on " << t.device();
  return s.str();
}
[[noreturn]] void refuse(const char *name, const std::string &want, const Tensor &t) { throw Refused(std::string(name) + ": want " + want + ", got " + said(t)); }

const Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) throw Refused(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}
const Tensor *optional_tensor(PyObject *o, const char *name) { return o == Py_None ? nullptr : &tensor(o, name); }

struct On {      // the device of a call's tensors, made current for the call, and torch's current stream on it
  int index;
  std::optional<c10::cuda::CUDAGuard> guard;
  explicit On(const Tensor &t, const char *name) {
    if (!t.is_cuda()) throw Refused(std::string(name) + " must be a CUDA tensor");
    index = t.get_device();
    if (c10::cuda::current_device() != index) guard.emplace((c10::DeviceIndex)index);
  }
  void *stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream(); }
  bool holds(const Tensor &t) const { return t.is_cuda() && t.get_device() == index; }
  Tensor make(at::IntArrayRef shape, at::ScalarType type) const { return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)index)); }
};

void *vec(const On &on, const Tensor &t, const char *name, int64_t n, at::ScalarType type = at::kInt) {
  if (t.scalar_type() != type || t.dim() != 1 || (n >= 0 && t.size(0) != n) || !on.holds(t) || !t.is_contiguous()) {
    std::ostringstream s;
    s << "a contiguous " << type << " vector";
    if (n >= 0) s << " of " << n;
    s << " on cuda:" << on.index;
    refuse(name, s.str(), t);
  }
  return t.data_ptr();
}
void *whole(const On &on, const Tensor &t, const char *name, at::IntArrayRef shape, at::ScalarType type) {
  if (t.scalar_type() != type || t.sizes() != shape || !on.holds(t) || !t.is_contiguous()) {
    std::ostringstream s;
    s << "a contiguous " << type << " tensor " << shape << " on cuda:" << on.index;
    refuse(name, s.str(), t);
  }
  return t.data_ptr();
}
// [tokens, heads, head_dim] with whole heads side by side and any token stride
struct Heads { void *p; int64_t stride; };
Heads heads(const On &on, const Tensor &t, const char *name, at::ScalarType type) {
  if (t.dim() != 3 || t.scalar_type() != type || !on.holds(t)) {
    std::ostringstream s;
    s << "a " << type << " tensor [tokens, heads, head_dim] on cuda:" << on.index;
    refuse(name, s.str(), t);
  }
  const int64_t n = t.size(0), h = t.size(1), d = t.size(2);
  if ((t.stride(2) != 1 && d > 1) || (t.stride(1) != d && h > 1)) throw Refused(std::string(name) + ": the heads of a token must be contiguous");
  return {t.data_ptr(), n <= 1 && t.stride(0) < h * d ? h * d : t.stride(0)};
}
int32_t code_of(const Tensor &t, const char *name) {
  switch (t.scalar_type()) {
    case at::kFloat: return SWIFTKV_DTYPE_F32;
    case at::kBFloat16: return SWIFTKV_DTYPE_BF16;
    case at::kHalf: return SWIFTKV_DTYPE_F16;
    default: refuse(name, "fp32, bf16 or f16", t);
  }
}
int32_t i32(int64_t v, const char *name) {
  if (v < INT32_MIN || v > INT32_MAX) throw Refused(std::string(name) + " does not fit 32 bits");
  return (int32_t)v;
}
int32_t i32(PyObject *o, const char *name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return i32((int64_t)v, name);
}
float f32(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return (float)v;
}

template <typename F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd wanted", n, want);
    return nullptr;
  }
  try {
    return f();
  } catch (const Raised &) {
    return nullptr;
  } catch (const Refused &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
PyObject *none() { Py_RETURN_NONE; }

// ---- the calls ---------------------------------------------------------------------------------------------------
PyObject *plan_pages(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  return guarded(argc, 13, [&]() -> PyObject * {
    const Tensor &past = tensor(a[0], "n_past"), &table = tensor(a[3], "block_table"), &free_pages = tensor(a[4], "free_pages");
    On on(past, "n_past");
    const int64_t n = past.numel();
    if (table.dim() != 2 || table.size(0) != n) refuse("block_table", "[n_seqs, max_blocks]", table);
    const int64_t blocks = table.size(1), shape[2] = {n, blocks};
    const Tensor &slots = tensor(a[10], "out slot_map");
    const int64_t room = slots.numel();
    auto in = [&](int i, const char *name, int64_t m) { return static_cast<int32_t *>(vec(on, tensor(a[i], name), name, m)); };
    int32_t *const p_past = in(0, "n_past", n), *const p_new = in(1, "n_new", n), *const p_owned = in(2, "n_owned", n);
    check(p_swiftkv_plan_pages(p_past, p_new, p_owned, i32(n, "n_seqs"), static_cast<int32_t *>(whole(on, table, "block_table", shape, at::kInt)),
                               i32(blocks, "max_blocks"), in(4, "free_pages", -1), i32(free_pages.numel(), "free_pages"), in(5, "n_free", 1),
                               static_cast<int32_t *>(whole(on, tensor(a[6], "out block_table"), "out block_table", shape, at::kInt)), in(7, "out n_owned", n),
                               in(8, "out n_free", 1), in(9, "out cu_new", n + 1), in(10, "out slot_map", room), in(11, "out positions", room),
                               i32(room, "slot_map"), in(12, "out info", 4), on.stream()));
    return none();
  });
}

struct RopeCommon {
  at::ScalarType type;
  int32_t code, n, n_q, n_kv, hd, max_pos;
  Heads q, k;
  void *pos, *cos, *sin, *q_gain, *k_gain;
};
RopeCommon rope_common(const On &on, const Tensor &q, const Tensor &k, PyObject *pos, PyObject *cos, PyObject *sin, PyObject *qg, PyObject *kg) {
  RopeCommon r;
  r.code = code_of(q, "q");
  r.type = q.scalar_type();
  r.q = heads(on, q, "q", r.type);
  r.k = heads(on, k, "k", r.type);
  if (k.size(0) != q.size(0) || k.size(2) != q.size(2)) throw Refused("q and k must have the same tokens and head_dim");
  r.n = i32(q.size(0), "tokens");
  r.n_q = i32(q.size(1), "heads");
  r.n_kv = i32(k.size(1), "heads");
  r.hd = i32(q.size(2), "head_dim");
  const Tensor &c = tensor(cos, "cos");
  if (c.dim() != 2 || r.hd % 2) refuse("cos", "[max_pos, head_dim / 2]", c);
  r.max_pos = i32(c.size(0), "max_pos");
  const int64_t shape[2] = {r.max_pos, r.hd / 2};
  r.pos = vec(on, tensor(pos, "positions"), "positions", r.n);
  r.cos = whole(on, c, "cos", shape, at::kFloat);
  r.sin = whole(on, tensor(sin, "sin"), "sin", shape, at::kFloat);
  const Tensor *g = optional_tensor(qg, "q_gain"), *h = optional_tensor(kg, "k_gain");
  r.q_gain = g ? vec(on, *g, "q_gain", r.hd, r.type) : nullptr;
  r.k_gain = h ? vec(on, *h, "k_gain", r.hd, r.type) : nullptr;
  return r;
}

// cache planes [rows, n_kv, hd] of q's type, or codes with row scales
struct Cache { void *k, *v; float *k_scale, *v_scale; int32_t rows, n_kv; bool fp8; };
Cache cache_of(const On &on, PyObject *kc, PyObject *vc, PyObject *ks, PyObject *vs, int64_t hd, at::ScalarType type) {
  const Tensor &k = tensor(kc, "k_cache"), &v = tensor(vc, "v_cache"), *sk = optional_tensor(ks, "k_scale"), *sv = optional_tensor(vs, "v_scale");
  if (!sk != !sv) throw Refused("k_scale and v_scale go together");
  if (k.dim() != 3 || k.size(2) != hd) refuse("k_cache", "[rows, n_kv, head_dim]", k);
  Cache c;
  c.fp8 = sk != nullptr;
  const at::ScalarType want = c.fp8 ? at::kByte : type;
  const int64_t shape[3] = {k.size(0), k.size(1), hd};
  c.k = whole(on, k, "k_cache", shape, want);
  c.v = whole(on, v, "v_cache", shape, want);
  c.k_scale = sk ? static_cast<float *>(vec(on, *sk, "k_scale", shape[0], at::kFloat)) : nullptr;
  c.v_scale = sv ? static_cast<float *>(vec(on, *sv, "v_scale", shape[0], at::kFloat)) : nullptr;
  c.rows = i32(shape[0], "cache rows");
  c.n_kv = i32(shape[1], "n_kv");
  return c;
}

// q, k, v, positions, cos, sin, q_gain, k_gain, eps, slot_map, k_cache, v_cache, k_scale, v_scale, q_out
PyObject *qk_norm_rope(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  return guarded(argc, 15, [&]() -> PyObject * {
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    On on(q, "q");
    const RopeCommon r = rope_common(on, q, k, a[3], a[4], a[5], a[6], a[7]);
    const Heads hv = heads(on, v, "v", r.type);
    if (v.sizes() != k.sizes()) throw Refused("v must have k's shape");
    const Cache c = cache_of(on, a[10], a[11], a[12], a[13], r.hd, r.type);
    if (c.n_kv != r.n_kv) throw Refused("the cache must have k's heads");
    const Tensor *slots = optional_tensor(a[9], "slot_map");
    void *p_slots = slots ? vec(on, *slots, "slot_map", r.n) : nullptr;
    const Tensor out = a[14] == Py_None ? on.make(q.sizes(), r.type) : tensor(a[14], "q_out");
    const Heads ho = heads(on, out, "q_out", r.type);
    if (out.sizes() != q.sizes()) throw Refused("q_out must have q's shape");
    if (r.n == 0) return THPVariable_Wrap(out);
    check(p_swiftkv_qk_norm_rope(r.q.p, r.q.stride, r.k.p, r.k.stride, hv.p, hv.stride, r.code, r.n, r.n_q, r.n_kv, r.hd, r.q_gain, r.k_gain, f32(a[8]),
                                 static_cast<int32_t *>(r.pos), static_cast<float *>(r.cos), static_cast<float *>(r.sin), r.max_pos, ho.p, ho.stride, c.k, c.v,
                                 c.k_scale, c.v_scale, c.rows, static_cast<int32_t *>(p_slots), on.stream()));
    return THPVariable_Wrap(out);
  });
}

// dq, dk, q, k, positions, cos, sin, q_gain, k_gain, eps, out dq, out dk
PyObject *qk_norm_rope_bwd(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  return guarded(argc, 12, [&]() -> PyObject * {
    const Tensor &q = tensor(a[2], "q"), &k = tensor(a[3], "k");
    On on(q, "q");
    const RopeCommon r = rope_common(on, q, k, a[4], a[5], a[6], a[7], a[8]);
    void *dq = whole(on, tensor(a[0], "dq"), "dq", q.sizes(), r.type), *dk = whole(on, tensor(a[1], "dk"), "dk", k.sizes(), r.type);
    const Tensor oq = a[10] == Py_None ? on.make(q.sizes(), r.type) : tensor(a[10], "out[0]"), ok = a[11] == Py_None ? on.make(k.sizes(), r.type) : tensor(a[11], "out[1]");
    void *po = whole(on, oq, "out[0]", q.sizes(), r.type), *pk = whole(on, ok, "out[1]", k.sizes(), r.type);
    Tensor gq, gk;
    if (r.q_gain) gq = on.make({r.hd}, at::kFloat);
    if (r.k_gain) gk = on.make({r.hd}, at::kFloat);
    if (r.n == 0) {
      if (r.q_gain) gq.zero_();
      if (r.k_gain) gk.zero_();
      return Py_BuildValue("NNNN", THPVariable_Wrap(oq), THPVariable_Wrap(ok), r.q_gain ? THPVariable_Wrap(gq) : none(), r.k_gain ? THPVariable_Wrap(gk) : none());
    }
    const size_t bytes = p_swiftkv_qk_norm_rope_bwd_scratch_bytes(r.hd);
    const Tensor scratch = on.make({(int64_t)(bytes ? bytes : 1)}, at::kByte);
    check(p_swiftkv_qk_norm_rope_bwd(dq, dk, r.q.p, r.q.stride, r.k.p, r.k.stride, r.code, r.n, r.n_q, r.n_kv, r.hd, r.q_gain, r.k_gain, f32(a[9]),
                                     static_cast<int32_t *>(r.pos), static_cast<float *>(r.cos), static_cast<float *>(r.sin), r.max_pos, po, pk,
                                     r.q_gain ? static_cast<float *>(gq.data_ptr()) : nullptr, r.k_gain ? static_cast<float *>(gk.data_ptr()) : nullptr,
                                     scratch.data_ptr(), bytes, on.stream()));
    return Py_BuildValue("NNNN", THPVariable_Wrap(oq), THPVariable_Wrap(ok), r.q_gain ? THPVariable_Wrap(gq) : none(), r.k_gain ? THPVariable_Wrap(gk) : none());
  });
}

// q, k_cache, v_cache, n_past, cu_new, max_new, max_kv, block_table, row0, tree_mask, k_scale, v_scale, softmax_scale, out, lse
PyObject *tree_attention(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  return guarded(argc, 15, [&]() -> PyObject * {
    const Tensor &q = tensor(a[0], "q"), &past = tensor(a[3], "n_past");
    On on(q, "q");
    const int32_t code = code_of(q, "q");
    const at::ScalarType type = q.scalar_type();
    const Heads hq = heads(on, q, "q", type);
    const int64_t t = q.size(0), n_q = q.size(1), hd = q.size(2), n = past.numel();
    const Cache c = cache_of(on, a[1], a[2], a[10], a[11], hd, type);
    int32_t *p_past = static_cast<int32_t *>(vec(on, past, "n_past", n)), *p_cu = static_cast<int32_t *>(vec(on, tensor(a[4], "cu_new"), "cu_new", n + 1));
    int32_t *p_table = nullptr, *p_row0 = nullptr, *p_mask = nullptr;
    int64_t blocks = 0, words = 0;
    if (const Tensor *table = optional_tensor(a[7], "block_table")) {
      if (table->dim() != 2) refuse("block_table", "[n_seqs, max_blocks]", *table);
      blocks = table->size(1);
      p_table = static_cast<int32_t *>(whole(on, *table, "block_table", {n, blocks}, at::kInt));
    }
    if (const Tensor *row0 = optional_tensor(a[8], "row0")) p_row0 = static_cast<int32_t *>(vec(on, *row0, "row0", n));
    if (const Tensor *mask = optional_tensor(a[9], "tree_mask")) {
      if (mask->dim() != 2) refuse("tree_mask", "[tokens, words]", *mask);
      words = mask->size(1);
      p_mask = static_cast<int32_t *>(whole(on, *mask, "tree_mask", {t, words}, at::kInt));
    }
    const Tensor out = a[13] == Py_None ? on.make(q.sizes(), type) : tensor(a[13], "out");
    void *p_out = whole(on, out, "out", q.sizes(), type);
    const Tensor *lse = optional_tensor(a[14], "lse");
    float *p_lse = lse ? static_cast<float *>(whole(on, *lse, "lse", {t, n_q}, at::kFloat)) : nullptr;
    const int32_t max_new = i32(a[5], "max_new"), max_kv = i32(a[6], "max_kv");
    if (t == 0) return THPVariable_Wrap(out);
    const size_t bytes = p_swiftkv_tree_attention_scratch_bytes(i32(t, "tokens"), max_kv, i32(n_q, "heads"), i32(hd, "head_dim"));
    Tensor scratch;
    if (bytes) scratch = on.make({(int64_t)bytes}, at::kByte);
    check(p_swiftkv_tree_attention(hq.p, hq.stride, code, c.k, c.v, c.fp8 ? SWIFTKV_DTYPE_FP8_E4M3 : code, c.k_scale, c.v_scale, c.rows, p_table,
                                   i32(blocks, "max_blocks"), p_row0, p_past, p_cu, p_mask, i32(words, "mask words"), p_out, p_lse, i32(n, "n_seqs"), (int32_t)t,
                                   max_new, max_kv, (int32_t)n_q, c.n_kv, (int32_t)hd, f32(a[12]), bytes ? scratch.data_ptr() : nullptr, bytes, on.stream()));
    return THPVariable_Wrap(out);
  });
}

struct Rows { void *p; int64_t stride; int32_t code, rows, vocab; };
Rows rows_of(const On &on, const Tensor &t, const char *name) {
  const int32_t code = code_of(t, name);
  if (t.dim() != 2 || !on.holds(t) || (t.stride(1) != 1 && t.size(1) > 1)) refuse(name, "[rows, vocab] with contiguous rows on the call's device", t);
  return {t.data_ptr(), t.size(0) <= 1 && t.stride(0) < t.size(1) ? t.size(1) : t.stride(0), code, i32(t.size(0), "rows"), i32(t.size(1), "vocab")};
}

// logits, targets, top_k, temperature, logprob, entropy, lse, top_ids, top_logprobs
PyObject *token_logprobs(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  return guarded(argc, 9, [&]() -> PyObject * {
    const Tensor &x = tensor(a[0], "logits"), *targets = optional_tensor(a[1], "targets");
    On on(x, "logits");
    const Rows r = rows_of(on, x, "logits");
    const int32_t k = i32(a[2], "top_k");
    auto f = [&](int i, const char *name) { return static_cast<float *>(vec(on, tensor(a[i], name), name, r.rows, at::kFloat)); };
    int32_t *ids = nullptr;
    float *lps = nullptr;
    if (k > 0) {
      ids = static_cast<int32_t *>(whole(on, tensor(a[7], "top_ids"), "top_ids", {r.rows, k}, at::kInt));
      lps = static_cast<float *>(whole(on, tensor(a[8], "top_logprobs"), "top_logprobs", {r.rows, k}, at::kFloat));
    }
    int32_t *tgt = targets ? static_cast<int32_t *>(vec(on, *targets, "targets", r.rows)) : nullptr;
    float *logprob = f(4, "logprob"), *entropy = f(5, "entropy"), *lse = f(6, "lse");
    if (r.rows == 0) return none();
    check(p_swiftkv_token_logprobs(r.p, r.stride, r.code, tgt, r.rows, r.vocab, f32(a[3]), k, logprob, entropy, lse, ids, lps, on.stream()));
    return none();
  });
}

// logits, targets, lse, entropy, grad_logprob, grad_entropy, temperature, out
PyObject *token_logprobs_bwd(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  return guarded(argc, 8, [&]() -> PyObject * {
    const Tensor &x = tensor(a[0], "logits");
    On on(x, "logits");
    const Rows r = rows_of(on, x, "logits");
    auto f = [&](int i, const char *name) {
      const Tensor *t = optional_tensor(a[i], name);
      return t ? static_cast<float *>(vec(on, *t, name, r.rows, at::kFloat)) : nullptr;
    };
    int32_t *targets = static_cast<int32_t *>(vec(on, tensor(a[1], "targets"), "targets", r.rows));
    float *lse = f(2, "lse"), *entropy = f(3, "entropy"), *g_lp = f(4, "grad_logprob"), *g_h = f(5, "grad_entropy");
    const Tensor out = a[7] == Py_None ? on.make(x.sizes(), x.scalar_type()) : tensor(a[7], "out");
    const Rows o = rows_of(on, out, "out");
    if (o.code != r.code || o.rows != r.rows || o.vocab != r.vocab) throw Refused("out must have the logits' shape, type and device");
    if (r.rows == 0) return THPVariable_Wrap(out);
    check(p_swiftkv_token_logprobs_bwd(r.p, r.stride, r.code, targets, r.rows, r.vocab, f32(a[6]), lse, entropy, g_lp, g_h, o.p, o.stride, on.stream()));
    return THPVariable_Wrap(out);
  });
}

// bind(SwiftKVError, {name: address}): where the library's functions are
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  return guarded(argc, 2, [&]() -> PyObject * {
#define X(name)                                                                       \
  {                                                                                   \
    PyObject *v = PyDict_GetItemString(a[1], #name);                                  \
    if (!v) throw Refused("bind: " #name " is missing");                              \
    p_##name = reinterpret_cast<decltype(p_##name)>(PyLong_AsVoidPtr(v));             \
    if (PyErr_Occurred()) throw Raised();                                             \
  }
    FUNCTIONS(X)
#undef X
    Py_INCREF(a[0]);
    Py_XDECREF(g_error);
    g_error = a[0];
    return none();
  });
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(plan_pages), METHOD(qk_norm_rope), METHOD(qk_norm_rope_bwd), METHOD(tree_attention), METHOD(token_logprobs),
                         METHOD(token_logprobs_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_verify", "marshalling of the verification-step operators", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__verify(void) {
  PyObject *m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for_torch", SWIFTKV_TORCH)) Py_CLEAR(m);
  return m;
}
