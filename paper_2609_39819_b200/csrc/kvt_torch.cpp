// kvt_torch.cpp — the marshalling of the model-side calls for Python, natively: reading a dozen tensors' types, shapes, strides
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

// ---- choosing blocks ----
struct Rows { void *p; uint64_t stride; };
Rows table(const Call &c, const at::Tensor &x, at::ScalarType t, int64_t n, int64_t m) {
  want(x.scalar_type() == t && x.dim() == 2 && x.size(0) == n && x.size(1) == m && (x.stride(1) == 1 || m <= 1));
  want(!x.requires_grad() || !at::GradMode::is_enabled());
  c.on(x);
  return {x.data_ptr(), (uint64_t)x.stride(0)};
}
void apart(const Rows &r, int64_t n, int64_t m) { want(n <= 1 || r.stride >= (uint64_t)m); }
const float *lse_of(const Call &c, const at::Tensor &l, int64_t tokens, int64_t hq) {
  want(l.scalar_type() == at::kFloat && l.dim() == 2 && l.size(0) == tokens && l.size(1) == hq && l.is_contiguous() &&
       (!l.requires_grad() || !at::GradMode::is_enabled()));
  c.on(l);
  return (const float *)l.data_ptr();
}
kvt_key_bounds bounds_of(const Call &c, int64_t layers, const at::Tensor &codes, const at::Tensor &exps) {
  want(codes.scalar_type() == at::kChar && exps.scalar_type() == at::kByte && codes.dim() == 5 && exps.dim() == 3);
  const int64_t n = codes.size(1);
  want(codes.size(0) == layers && codes.size(2) == c.heads && codes.size(3) == 2 && codes.size(4) == (c.dim + 15) / 16 * 16 && exps.size(0) == layers &&
       exps.size(1) == n && exps.size(2) == c.heads && codes.is_contiguous() && exps.is_contiguous());
  c.on(codes); c.on(exps);
  return kvt_key_bounds{(int8_t *)codes.data_ptr(), (uint8_t *)exps.data_ptr(), (uint64_t)n};
}
float scale_of(PyObject *o) {
  if (o == Py_None) return 0.0f;
  want(PyFloat_CheckExact(o));
  const double scale = PyFloat_AS_DOUBLE(o);               // 0, which is the library's word for the default, becomes next to 0
  return scale >= 0.0 && scale < FLT_MIN ? FLT_MIN : (float)scale;
}
at::Tensor fresh(const at::Tensor &like, at::IntArrayRef shape, at::ScalarType t) {
  Unlocked u;
  return at::empty(shape, like.options().dtype(t).requires_grad(false));
}
// Scratch from the current stream's pool, or the capture's: nobody else has it while the call's kernels run.
template <class Args>
at::Tensor scratch_for(PyObject *entry, PyObject *engine, Args &a, const at::Tensor &like) {
  at::Tensor scratch;
  a.scratch_bytes = ((uint64_t (*)(kvt_engine *, const Args *))number(entry))((kvt_engine *)number(engine), &a);
  if (a.scratch_bytes) {
    scratch = fresh(like, {(int64_t)a.scratch_bytes}, at::kByte);
    a.scratch = scratch.data_ptr();
  }
  return scratch;
}

// (entry point, engine, stream, device, KV heads, head size, layers, layer, dtype code, codes, exps, block_table, q_start, kv_len, n_tokens):
// the call's status
PyObject *bound(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return answer([&]() -> PyObject * {
    want(n == 15);
    const Call c{(int64_t)small(x[3]), (int64_t)small(x[4]), (int64_t)small(x[5])};
    kvt_bound_args a{};
    a.layer = small(x[7]); a.dtype = small(x[8]);
    a.b = c.batch((int64_t)small(x[14]), x[11], x[12], x[13], 0);
    a.bounds = bounds_of(c, (int64_t)small(x[6]), tensor(x[9]), tensor(x[10]));
    return PyLong_FromLong(launch(x[0], x[1], x[2], a));
  });
}

// (entry point, that of the scratch bytes, engine, stream, device, KV heads, head size, layers, layer, dtype code, q, codes, exps, block_table,
//  q_start, kv_len, n_blocks, first, last, max_q_len, out): out; a number: the call's status
PyObject *select(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return answer([&]() -> PyObject * {
    want(n == 21);
    const Call c{(int64_t)small(x[4]), (int64_t)small(x[5]), (int64_t)small(x[6])};
    const at::Tensor &q = tensor(x[10]);
    want(q.dim() == 3);
    const int64_t tokens = q.size(0), hq = q.size(1);
    kvt_select_args a{};
    a.layer = small(x[8]); a.dtype = code(q.scalar_type()); a.n_q_heads = (uint32_t)hq;
    want(a.dtype == small(x[9]));
    const Place qp = c.rows(q, q.scalar_type(), tokens, hq);
    a.q = qp.p; a.q_ts = qp.ts; a.q_hs = qp.hs;
    a.bounds = bounds_of(c, (int64_t)small(x[7]), tensor(x[11]), tensor(x[12]));
    a.b = c.batch(tokens, x[13], x[14], x[15], x[19] == Py_None ? 0u : small(x[19]));
    a.n_blocks = small(x[16]); a.first = small(x[17]); a.last = small(x[18]);
    const at::Tensor out = x[20] != Py_None ? tensor(x[20]) : fresh(q, {tokens, c.heads, (int64_t)a.n_blocks}, at::kInt);
    want(out.scalar_type() == at::kInt && out.dim() == 3 && out.size(0) == tokens && out.size(1) == c.heads && out.size(2) == (int64_t)a.n_blocks && out.is_contiguous());
    c.on(out);
    a.out = (int32_t *)out.data_ptr();
    const at::Tensor scratch = scratch_for(x[1], x[2], a, q);
    const int32_t rc = launch(x[0], x[2], x[3], a);
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  });
}

// (entry point, engine, stream, device, KV heads, head size, layer, q, blocks, block_table, q_start, kv_len, scale, out, lse): out; a number:
// the call's status
PyObject *attend_blocks(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return answer([&]() -> PyObject * {
    want(n == 15);
    const Call c{(int64_t)small(x[3]), (int64_t)small(x[4]), (int64_t)small(x[5])};
    const at::Tensor &q = tensor(x[7]), &l = tensor(x[8]);
    want(q.dim() == 3);
    const at::ScalarType t = q.scalar_type();
    const int64_t tokens = q.size(0), hq = q.size(1);
    kvt_attend_blocks_args a{};
    a.layer = small(x[6]); a.dtype = code(t); a.n_q_heads = (uint32_t)hq;
    const Place qp = c.rows(q, t, tokens, hq);
    a.q = qp.p; a.q_ts = qp.ts; a.q_hs = qp.hs;
    want(l.scalar_type() == at::kInt && l.dim() == 3 && l.size(0) == tokens && l.size(1) == c.heads && l.size(2) <= 0x7FFFFFFF && l.is_contiguous());
    c.on(l);
    a.blocks = (const int32_t *)l.data_ptr(); a.n_blocks = (uint32_t)l.size(2);
    a.b = c.batch(tokens, x[9], x[10], x[11], 0);
    a.scale = scale_of(x[12]);
    const at::Tensor out = result(x[13], q);
    const Place op = c.rows(out, t, tokens, hq);
    not_broadcast(op, tokens, hq);
    a.out = op.p; a.o_ts = op.ts; a.o_hs = op.hs;
    if (x[14] != Py_None) a.lse = const_cast<float *>(lse_of(c, tensor(x[14]), tokens, hq));
    const int32_t rc = launch(x[0], x[1], x[2], a);
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  });
}

// (entry point, that of the scratch bytes, engine, stream, device, KV heads, head size, layer, q, lse, block_table, q_start, kv_len, max_q_len,
//  causal, window, scale, weights, keep, out): out; a number: the call's status
PyObject *weigh(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return answer([&]() -> PyObject * {
    want(n == 20);
    const Call c{(int64_t)small(x[4]), (int64_t)small(x[5]), (int64_t)small(x[6])};
    const at::Tensor &q = tensor(x[8]);
    want(q.dim() == 3);
    const int64_t tokens = q.size(0), hq = q.size(1);
    kvt_weigh_args a{};
    a.layer = small(x[7]); a.dtype = code(q.scalar_type()); a.n_q_heads = (uint32_t)hq;
    const Place qp = c.rows(q, q.scalar_type(), tokens, hq);
    a.q = qp.p; a.q_ts = qp.ts; a.q_hs = qp.hs;
    a.lse = lse_of(c, tensor(x[9]), tokens, hq);
    a.b = c.batch(tokens, x[10], x[11], x[12], x[13] == Py_None ? 0u : small(x[13]));
    const int64_t seqs = a.b.n_seqs, blocks = a.b.max_blocks;
    want(x[14] == Py_True || x[14] == Py_False);
    a.flags = x[14] == Py_True ? 0u : KVT_ATTN_FULL;
    a.window = x[15] == Py_None ? 0u : small(x[15]);
    a.scale = scale_of(x[16]);
    want(PyFloat_CheckExact(x[18]));
    a.keep = (float)PyFloat_AS_DOUBLE(x[18]);
    Rows w{nullptr, 0};
    if (x[17] != Py_None) w = table(c, tensor(x[17]), at::kFloat, seqs, blocks);
    const at::Tensor out = x[19] != Py_None ? tensor(x[19]) : fresh(q, {seqs, blocks}, at::kFloat);
    const Rows o = table(c, out, at::kFloat, seqs, blocks);
    apart(o, seqs, blocks);
    want(w.p != o.p || w.stride == o.stride || seqs <= 1);
    a.weights = (const float *)w.p; a.w_stride = w.stride; a.out = (float *)o.p; a.o_stride = o.stride;
    const at::Tensor scratch = scratch_for(x[1], x[2], a, q);
    const int32_t rc = launch(x[0], x[2], x[3], a);
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  });
}

// (entry point, engine, stream, device, KV heads, head size, weights, block_table, kv_len, n_blocks, first, last): a tuple of new tensors; a
// number: the call's status. Outputs that the caller gives are left to the caller's own marshalling.
PyObject *evict(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return answer([&]() -> PyObject * {
    want(n == 12);
    const Call c{(int64_t)small(x[3]), (int64_t)small(x[4]), (int64_t)small(x[5])};
    const at::Tensor &w = tensor(x[6]), &t = tensor(x[7]), &l = tensor(x[8]);
    want(t.dim() == 2);
    const int64_t seqs = t.size(0), blocks = t.size(1);
    want(seqs <= 0x7FFFFFFF && blocks <= 0x7FFFFFFF && l.scalar_type() == at::kInt && l.dim() == 1 && l.size(0) == seqs && l.is_contiguous());
    c.on(l);
    const Rows wr = table(c, w, at::kFloat, seqs, blocks), tr = table(c, t, at::kInt, seqs, blocks);
    at::Tensor out[4];
    {
      Unlocked u;
      const auto ints = t.options();
      out[0] = at::empty({seqs, blocks}, ints); out[1] = at::empty({seqs}, ints);
      out[2] = at::empty({seqs, blocks}, w.options().requires_grad(false)); out[3] = at::empty({seqs, blocks}, ints);
    }
    kvt_evict_args a{};
    a.n_seqs = (uint32_t)seqs; a.max_blocks = (uint32_t)blocks; a.n_blocks = small(x[9]); a.first = small(x[10]); a.last = small(x[11]);
    a.block_table = (const uint32_t *)tr.p; a.kv_len = (const uint32_t *)l.data_ptr(); a.weights = (const float *)wr.p;
    a.table_stride = tr.stride; a.w_stride = wr.stride;
    a.table_out = (uint32_t *)out[0].data_ptr(); a.kv_len_out = (uint32_t *)out[1].data_ptr();
    a.weights_out = (float *)out[2].data_ptr(); a.evicted = (uint32_t *)out[3].data_ptr();
    a.table_out_stride = a.w_out_stride = a.evicted_stride = (uint64_t)blocks;
    const int32_t rc = launch(x[0], x[1], x[2], a);
    if (rc) return PyLong_FromLong(rc);
    PyObject *const all = PyTuple_New(4);
    if (!all) return nullptr;
    for (int i = 0; i < 4; ++i) {
      PyObject *const o = THPVariable_Wrap(out[i]);
      if (!o) { Py_DECREF(all); return nullptr; }
      PyTuple_SET_ITEM(all, i, o);
    }
    return all;
  });
}

PyMethodDef methods[] = {{"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr},
                         {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
                         {"bound", (PyCFunction)(void (*)(void))bound, METH_FASTCALL, nullptr},
                         {"select", (PyCFunction)(void (*)(void))select, METH_FASTCALL, nullptr},
                         {"attend_blocks", (PyCFunction)(void (*)(void))attend_blocks, METH_FASTCALL, nullptr},
                         {"weigh", (PyCFunction)(void (*)(void))weigh, METH_FASTCALL, nullptr},
                         {"evict", (PyCFunction)(void (*)(void))evict, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvt_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvt_torch() { return PyModule_Create(&module); }
