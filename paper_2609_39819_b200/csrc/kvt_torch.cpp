// kvt_torch.cpp — the marshalling of append_kv and attend for Python, natively: reading a dozen tensors' types, shapes, strides
// and addresses from Python takes 4 us of a call, allocating a result 1.5 us; here it is 1 us together.
// Arguments that are exactly as the calls want them are taken here. For everything else the functions return NotImplemented,
// and the caller's own checks say what is wrong: there is one place for messages.
// No link against libkvt.so: entry points and the engine's handle come as addresses from the library the caller has loaded.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cfloat>

#include "../../include/kvt.h"

namespace {

struct Refused {};

const at::Tensor &tensor(PyObject *o) {
  if (!THPVariable_CheckExact(o)) throw Refused{};
  return THPVariable_Unpack(o);
}
uint64_t number(PyObject *o) {
  if (!PyLong_CheckExact(o)) throw Refused{};
  const unsigned long long x = PyLong_AsUnsignedLongLong(o);
  if (PyErr_Occurred()) { PyErr_Clear(); throw Refused{}; }
  return x;
}
uint32_t small(PyObject *o) {
  const uint64_t x = number(o);
  if (x > 0x7FFFFFFFu) throw Refused{};
  return (uint32_t)x;
}
void want(bool ok) { if (!ok) throw Refused{}; }

struct Place { void *p; uint64_t ts, hs; };

struct Call {
  int64_t dev, heads, dim;
  void on(const at::Tensor &x) const { want(x.is_cuda() && x.get_device() == dev); }
  Place rows(const at::Tensor &x, at::ScalarType t, int64_t n, int64_t h) const {
    want(x.scalar_type() == t && x.dim() == 3 && x.size(0) == n && x.size(1) == h && x.size(2) == dim && (x.stride(2) == 1 || dim <= 1));
    want(!x.requires_grad() || !at::GradMode::is_enabled());       // there is no backward pass
    on(x);
    return {x.data_ptr(), (uint64_t)x.stride(0), (uint64_t)x.stride(1)};
  }
  kvt_batch batch(int64_t tokens, PyObject *table, PyObject *start, PyObject *length, uint32_t most) const {
    const at::Tensor &t = tensor(table), &s = tensor(start), &l = tensor(length);
    want(t.scalar_type() == at::kInt && s.scalar_type() == at::kInt && l.scalar_type() == at::kInt && t.dim() == 2 && s.dim() == 1 && l.dim() == 1);
    const int64_t n = t.size(0), m = t.size(1);
    want(l.size(0) == n && s.size(0) == n + 1 && (t.stride(1) == 1 || m <= 1) && s.is_contiguous() && l.is_contiguous());
    want(n <= 0x7FFFFFFF && m <= 0x7FFFFFFF && tokens <= 0x7FFFFFFF);
    on(t); on(s); on(l);
    kvt_batch b{};
    b.n_seqs = (uint32_t)n; b.n_tokens = (uint32_t)tokens; b.max_blocks = (uint32_t)m; b.max_q_len = most;
    b.table_stride = (uint64_t)t.stride(0);
    b.q_start = (const uint32_t *)s.data_ptr(); b.kv_len = (const uint32_t *)l.data_ptr(); b.block_table = (const uint32_t *)t.data_ptr();
    return b;
  }
};

uint32_t code(at::ScalarType t) {
  want(t == at::kBFloat16 || t == at::kHalf);
  return t == at::kBFloat16 ? KVT_KV_BF16 : KVT_KV_FP16;
}
void not_broadcast(const Place &o, int64_t n, int64_t h) { want((o.ts || n <= 1) && (o.hs || h <= 1)); }

// Allocating and launching may have to wait: other threads go on meanwhile.
struct Unlocked {
  PyThreadState *const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
at::Tensor result(PyObject *given, const at::Tensor &like) {
  if (given != Py_None) return tensor(given);
  Unlocked u;
  return at::empty_like(like, like.options(), at::MemoryFormat::Contiguous);
}
template <class Args>
int32_t launch(PyObject *entry, PyObject *engine, PyObject *stream, const Args &a) {
  const auto f = (int32_t (*)(kvt_engine *, const Args *, void *))number(entry);
  kvt_engine *const e = (kvt_engine *)number(engine);
  void *const s = (void *)number(stream);
  Unlocked u;
  return f(e, &a, s);
}
PyObject *none() { Py_RETURN_NONE; }

// A body's answer as a Python object: its own, NotImplemented where it refused, or an exception.
template <class F>
PyObject *answer(F body) {
  try {
    return body();
  } catch (const Refused &) {
    Py_RETURN_NOTIMPLEMENTED;
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

// (entry point, engine, stream, device, KV heads, head size, layer, k, v, block_table, q_start, kv_len, rot_dim, axes, freqs,
//  axis_of, interleaved, positions, q, q_out): the rotated queries or None; a number: the call's status
PyObject *append(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return answer([&]() -> PyObject * {
    want(n == 20);
    const Call c{(int64_t)small(x[3]), (int64_t)small(x[4]), (int64_t)small(x[5])};
    const at::Tensor &k = tensor(x[7]), &v = tensor(x[8]);
    want(k.dim() == 3);
    const at::ScalarType t = k.scalar_type();
    const int64_t tokens = k.size(0);
    kvt_append_args a{};
    a.layer = small(x[6]); a.dtype = code(t);
    const Place kp = c.rows(k, t, tokens, c.heads), vp = c.rows(v, t, tokens, c.heads);
    a.k = kp.p; a.k_ts = kp.ts; a.k_hs = kp.hs; a.v = vp.p; a.v_ts = vp.ts; a.v_hs = vp.hs;
    a.b = c.batch(tokens, x[9], x[10], x[11], 0);
    a.rot_dim = small(x[12]); a.n_axes = small(x[13]); a.flags = x[16] == Py_True ? KVT_ROPE_INTERLEAVED : 0u;
    const bool rope = x[14] != Py_None;
    if (rope) {
      const at::Tensor &f = tensor(x[14]);
      want(f.scalar_type() == at::kDouble && f.is_contiguous() && f.numel() == a.rot_dim / 2);
      c.on(f);
      a.freqs = (const double *)f.data_ptr();
    }
    if (x[15] != Py_None) {
      const at::Tensor &f = tensor(x[15]);
      want(f.scalar_type() == at::kByte && f.is_contiguous() && f.numel() == a.rot_dim / 2);
      c.on(f);
      a.axis_of = (const uint8_t *)f.data_ptr();
    }
    if (x[17] != Py_None) {
      const at::Tensor &p = tensor(x[17]);
      const bool one = p.dim() == 1;
      want(rope && p.scalar_type() == at::kInt && (one || p.dim() == 2) && (one ? 1 : p.size(0)) == a.n_axes &&
           p.size(one ? 0 : 1) == tokens && (tokens <= 1 || p.stride(one ? 0 : 1) == 1));
      c.on(p);
      a.positions = (const int32_t *)p.data_ptr();
      a.pos_stride = one ? (uint64_t)tokens : (uint64_t)p.stride(0);
    } else {
      want(a.n_axes <= 1);
    }
    at::Tensor out;
    if (x[18] != Py_None) {
      const at::Tensor &q = tensor(x[18]);
      want(q.dim() == 3);
      const int64_t hq = q.size(1);
      const Place qp = c.rows(q, t, tokens, hq);
      out = result(x[19], q);
      const Place op = c.rows(out, t, tokens, hq);
      not_broadcast(op, tokens, hq);
      want(qp.p != op.p || (qp.ts == op.ts && qp.hs == op.hs));
      a.n_q_heads = (uint32_t)hq;
      a.q = qp.p; a.q_ts = qp.ts; a.q_hs = qp.hs; a.q_out = op.p; a.qo_ts = op.ts; a.qo_hs = op.hs;
    } else {
      want(x[19] == Py_None);
    }
    const int32_t rc = launch(x[0], x[1], x[2], a);
    if (rc) return PyLong_FromLong(rc);
    return out.defined() ? THPVariable_Wrap(out) : none();
  });
}

// (entry point, that of the scratch bytes, engine, stream, device, KV heads, head size, layer, q, block_table, q_start, kv_len,
//  max_q_len, causal, window, scale, out, lse): out; a number: the call's status
PyObject *attend(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return answer([&]() -> PyObject * {
    want(n == 18);
    const Call c{(int64_t)small(x[4]), (int64_t)small(x[5]), (int64_t)small(x[6])};
    const at::Tensor &q = tensor(x[8]);
    want(q.dim() == 3);
    const at::ScalarType t = q.scalar_type();
    const int64_t tokens = q.size(0), hq = q.size(1);
    kvt_attend_args a{};
    a.layer = small(x[7]); a.dtype = code(t); a.n_q_heads = (uint32_t)hq;
    const Place qp = c.rows(q, t, tokens, hq);
    a.q = qp.p; a.q_ts = qp.ts; a.q_hs = qp.hs;
    a.b = c.batch(tokens, x[9], x[10], x[11], x[12] == Py_None ? 0u : small(x[12]));
    want(x[13] == Py_True || x[13] == Py_False);
    a.flags = x[13] == Py_True ? 0u : KVT_ATTN_FULL;
    a.window = x[14] == Py_None ? 0u : small(x[14]);
    if (x[15] != Py_None) {
      want(PyFloat_CheckExact(x[15]));
      const double scale = PyFloat_AS_DOUBLE(x[15]);       // 0, which is the library's word for the default, becomes next to 0
      a.scale = scale >= 0.0 && scale < FLT_MIN ? FLT_MIN : (float)scale;
    }
    const at::Tensor out = result(x[16], q);
    const Place op = c.rows(out, t, tokens, hq);
    not_broadcast(op, tokens, hq);
    a.out = op.p; a.o_ts = op.ts; a.o_hs = op.hs;
    if (x[17] != Py_None) {
      const at::Tensor &l = tensor(x[17]);
      want(l.scalar_type() == at::kFloat && l.dim() == 2 && l.size(0) == tokens && l.size(1) == hq && l.is_contiguous() &&
           (!l.requires_grad() || !at::GradMode::is_enabled()));
      c.on(l);
      a.lse = (float *)l.data_ptr();
    }
    // scratch from the current stream's pool, or the capture's: nobody else has it while this call's kernels run
    at::Tensor scratch;
    a.scratch_bytes = ((uint64_t (*)(kvt_engine *, const kvt_attend_args *))number(x[1]))((kvt_engine *)number(x[2]), &a);
    if (a.scratch_bytes) {
      Unlocked u;
      scratch = at::empty({(int64_t)a.scratch_bytes}, q.options().dtype(at::kByte));
      a.scratch = scratch.data_ptr();
    }
    const int32_t rc = launch(x[0], x[2], x[3], a);
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  });
}

PyMethodDef methods[] = {{"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr},
                         {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvt_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvt_torch() { return PyModule_Create(&module); }
