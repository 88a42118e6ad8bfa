// Argument marshalling of binding.Block: checks its tensors, takes their addresses and the current stream, and calls the C interface.
//
// What the class does in Python costs 0.6 us a tensor (shape, type, device, layout, address, each an object), 9 us for a forward and 15 for a
// backward call, more than the kernels of a small batch take; here a call costs what the launch costs.  The same checks and messages; no arithmetic.
// The library is the one that the binding has loaded: init() gets the addresses of its functions.
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/augtree.h"

namespace {

decltype(&augtree_block_fwd) f_block_fwd;
decltype(&augtree_block_bwd) f_block_bwd;
decltype(&augtree_ckpt_pitch) f_ckpt_pitch;
decltype(&augtree_ckpt_pack) f_ckpt_pack;
decltype(&augtree_ckpt_unpack) f_ckpt_unpack;
decltype(&augtree_glu_fwd) f_glu_fwd;
decltype(&augtree_glu_bwd) f_glu_bwd;
decltype(&augtree_ckpt_wgrad) f_ckpt_wgrad;

// bits of the types that an argument may have
enum : unsigned { BF16 = 1u << AUGTREE_BF16, F16 = 1u << AUGTREE_F16, F32 = 1u << AUGTREE_F32, U8 = 1u << AUGTREE_CKPT, FLOATS = BF16 | F16 | F32 };

int code_of(at::ScalarType t) {
  switch (t) {
    case at::kBFloat16: return AUGTREE_BF16;
    case at::kHalf: return AUGTREE_F16;
    case at::kFloat: return AUGTREE_F32;
    case at::kByte: return AUGTREE_CKPT;
    default: return -1;
  }
}
std::string names(unsigned types) {
  std::string s;   // "[..]"
  for (auto [bit, name] : {std::pair{BF16, "torch.bfloat16"}, {F16, "torch.float16"}, {F32, "torch.float32"}, {U8, "torch.uint8"}})
    if (types & bit) s += (s.empty() ? "[" : ", ") + std::string(name);
  return (s.empty() ? "[" : s) + "]";
}
std::string got(PyObject *o) {
  if (!THPVariable_Check(o)) return Py_TYPE(o)->tp_name;
  const at::Tensor &t = THPVariable_Unpack(o);
  auto list = [](at::IntArrayRef v) {
    std::string s;
    for (int64_t x : v) s += (s.empty() ? "(" : ", ") + std::to_string(x);
    return (s.empty() ? "(" : s) + ")";
  };
  return list(t.sizes()) + " " + c10::toString(t.scalar_type()) + " on " + t.device().str() + " with strides " + list(t.strides());
}

struct Arg {
  void *p = nullptr;
  int code = 0;
  int64_t ld = 0;
  bool given = false;   // (a tensor of no elements has no address)
};

// The handle of a call: (address, device, hidden, bytes of a checkpoint row of `hidden`, gate)
struct Call {
  void *handle = nullptr;
  int device = -1, gate = 0;
  int64_t hidden = 0, pitch = 0;
  bool ok = true;

  explicit Call(PyObject *t) {
    ok = PyTuple_Check(t) && PyTuple_GET_SIZE(t) == 5;
    if (!ok) { PyErr_SetString(PyExc_TypeError, "handle"); return; }
    handle = PyLong_AsVoidPtr(PyTuple_GET_ITEM(t, 0));
    device = (int)PyLong_AsLong(PyTuple_GET_ITEM(t, 1));
    hidden = PyLong_AsLongLong(PyTuple_GET_ITEM(t, 2));
    pitch = PyLong_AsLongLong(PyTuple_GET_ITEM(t, 3));
    gate = (int)PyLong_AsLong(PyTuple_GET_ITEM(t, 4));
    ok = !PyErr_Occurred();
  }
  void fail(const std::string &what) {
    if (ok) PyErr_SetString(PyExc_ValueError, what.c_str());
    ok = false;
  }
  std::string shape(int64_t s0, int64_t s1) const {
    return "(" + std::to_string(s0) + (s1 < 0 ? ",)" : ", " + std::to_string(s1) + ")");
  }
  // rows and columns of an argument that has to be a matrix
  void rows(PyObject *o, const char *name, int64_t &n, int64_t &c) {
    n = c = 0;
    if (!ok) return;
    if (!THPVariable_Check(o) || THPVariable_Unpack(o).dim() != 2) return fail(std::string(name) + ": expected a tensor of two dimensions, got " + got(o));
    const auto s = THPVariable_Unpack(o).sizes();
    n = s[0]; c = s[1];
  }
  // a contiguous tensor of the given shape (s1 < 0: one dimension), or nothing for None
  Arg whole(PyObject *o, const char *name, unsigned types, int64_t s0, int64_t s1 = -1) {
    Arg a;
    if (!ok || o == Py_None) return a;
    if (THPVariable_Check(o)) {
      const at::Tensor &t = THPVariable_Unpack(o);
      a.code = code_of(t.scalar_type());
      const auto s = t.sizes();
      if (a.code >= 0 && (types >> a.code & 1) && (int64_t)s.size() == (s1 < 0 ? 1 : 2) && s[0] == s0 && (s1 < 0 || s[1] == s1) && t.is_cuda() &&
          t.get_device() == device && t.is_contiguous()) {
        a.p = t.data_ptr();
        a.given = true;
        return a;
      }
    }
    fail(std::string(name) + ": expected a contiguous tensor on cuda:" + std::to_string(device) + " of shape " + shape(s0, s1) + " and one of " +
         names(types) + ", got " + got(o));
    return a;
  }
  // a matrix whose rows are contiguous, with its leading size
  Arg strided(PyObject *o, const char *name, unsigned types, int64_t n, int64_t c) {
    Arg a;
    if (!ok) return a;
    if (THPVariable_Check(o)) {
      const at::Tensor &t = THPVariable_Unpack(o);
      a.code = code_of(t.scalar_type());
      const auto s = t.sizes();
      if (a.code >= 0 && (types >> a.code & 1) && s.size() == 2 && s[0] == n && s[1] == c && t.is_cuda() && t.get_device() == device &&
          (c <= 1 || t.stride(1) == 1)) {
        a.ld = n > 1 ? t.stride(0) : c;
        if (a.ld < c) fail(std::string(name) + ": rows overlap (" + got(o) + ")");
        a.p = t.data_ptr();
        a.given = true;
        return a;
      }
    }
    fail(std::string(name) + ": expected a tensor on cuda:" + std::to_string(device) + " of shape " + shape(n, c) + " and one of " + names(types) +
         " with contiguous rows, got " + got(o));
    return a;
  }
  // (nothing is asked of the interpreter once an exception is set)
  bool is_u8(PyObject *o) const { return ok && o != Py_None && THPVariable_Check(o) && THPVariable_Unpack(o).scalar_type() == at::kByte; }
  bool truth(PyObject *o) {
    const int r = ok ? PyObject_IsTrue(o) : 0;
    ok = ok && r >= 0;
    return r > 0;
  }
  // a saved tensor: in full, or a checkpoint
  Arg saved(PyObject *o, const char *name, int64_t n, int64_t c, int64_t row) {
    const bool u8 = is_u8(o);
    return u8 ? whole(o, name, U8, n, row) : whole(o, name, FLOATS, n, c);
  }
  Arg gate_like(PyObject *o, const char *name, unsigned types, int64_t n) {
    if (gate == AUGTREE_GATE_TOKEN) return whole(o, name, types, n);
    if (gate == AUGTREE_GATE_CHANNEL) return whole(o, name, types, hidden);
    if (gate == AUGTREE_GATE_FULL) return whole(o, name, types, n, hidden);
    if (o != Py_None) fail(std::string(name) + ": the handle has no gate");
    return {};
  }
  // two vectors of one number a channel, of one type
  int weights(PyObject *w_out, PyObject *w_in, Arg &o, Arg &i) {
    o = whole(w_out, "w_out", FLOATS, hidden);
    i = whole(w_in, "w_in", FLOATS, hidden);
    if (o.given && i.given && o.code != i.code) fail("w_out, w_in: expected one type, got " + names(1u << o.code) + " and " + names(1u << i.code));
    return o.given ? o.code : i.code;
  }
  Arg scratch(PyObject *o) {
    Arg a;
    if (!ok) return a;
    if (THPVariable_Check(o)) {
      const at::Tensor &t = THPVariable_Unpack(o);
      if (t.is_cuda() && t.get_device() == device && t.is_contiguous()) {
        a.p = t.data_ptr();
        a.given = true;
        a.ld = (int64_t)t.nbytes();
        return a;
      }
    }
    fail("ws: expected a contiguous tensor on cuda:" + std::to_string(device) + ", got " + got(o));
    return a;
  }
  int64_t pitch_of(int64_t cols) {
    int64_t p = 0;
    if (ok && f_ckpt_pitch(cols, &p)) fail("columns: expected a multiple of 8, at most 2^20, got " + std::to_string(cols));
    return p;
  }
  static unsigned like(const Arg &a) { return a.given ? 1u << a.code : 0u; }
  // the call itself, without the interpreter's lock: its return code, or null with an exception set
  template <class F>
  PyObject *run(F f) {
    if (!ok) return nullptr;
    int r = 0;
    Py_BEGIN_ALLOW_THREADS
    r = f(device < 0 ? nullptr : (void *)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream());
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
  }
};

// as torch's own functions do it: C++ exceptions become Python's
#define MARSHAL(name, count)                                                                       \
  PyObject *name##_checked(PyObject *const *a);                                                    \
  PyObject *name(PyObject *, PyObject *const *a, Py_ssize_t n) {                                   \
    if (n != count) { PyErr_SetString(PyExc_TypeError, #name ": number of arguments"); return nullptr; } \
    try {                                                                                          \
      return name##_checked(a);                                                                    \
    } catch (const std::exception &e) {                                                            \
      PyErr_SetString(PyExc_RuntimeError, e.what());                                               \
      return nullptr;                                                                              \
    }                                                                                              \
  }                                                                                                \
  PyObject *name##_checked(PyObject *const *a)

// handle, x, o, gate, w_out, w_in, y, h, r_out, r_in, ckpt_y, ckpt_o
MARSHAL(block_fwd, 12) {
  Call c(a[0]);
  int64_t n, cols;
  c.rows(a[1], "x", n, cols);
  const Arg x = c.whole(a[1], "x", FLOATS, n, c.hidden), o = c.whole(a[2], "o", FLOATS, n, c.hidden), g = c.gate_like(a[3], "gate", FLOATS, n);
  Arg wo, wi;
  const int wt = c.weights(a[4], a[5], wo, wi);
  const Arg y = c.whole(a[6], "y", Call::like(x), n, c.hidden), h = c.whole(a[7], "h", FLOATS, n, c.hidden);
  const Arg ro = c.whole(a[8], "r_out", F32, n), ri = c.whole(a[9], "r_in", F32, n);
  const Arg ky = c.whole(a[10], "ckpt_y", U8, n, c.pitch), ko = c.whole(a[11], "ckpt_o", U8, n, c.pitch);
  return c.run([&](void *st) {
    return f_block_fwd(static_cast<augtree_block_t *>(c.handle), x.p, x.code, o.p, o.code, g.p, g.code, wo.p, wi.p, wt, n, y.p, h.p, h.code,
                       static_cast<float *>(ro.p), static_cast<float *>(ri.p), ky.p, ko.p, st);
  });
}

// handle, dy, dh, y, o, gate, w_out, w_in, r_out, r_in, dx, d_o, d_gate, dw_out, dw_in, ws, accumulate
MARSHAL(block_bwd, 17) {
  Call c(a[0]);
  int64_t n, cols;
  c.rows(a[1] != Py_None ? a[1] : a[2], "dy or dh", n, cols);
  const Arg dy = c.whole(a[1], "dy", FLOATS, n, c.hidden), dh = c.whole(a[2], "dh", FLOATS, n, c.hidden);
  const Arg y = c.saved(a[3], "y", n, c.hidden, c.pitch), o = c.saved(a[4], "o", n, c.hidden, c.pitch), g = c.gate_like(a[5], "gate", FLOATS, n);
  Arg wo, wi;
  const int wt = c.weights(a[6], a[7], wo, wi);
  const Arg ro = c.whole(a[8], "r_out", F32, n), ri = c.whole(a[9], "r_in", F32, n);
  const Arg dx = c.whole(a[10], "dx", dy.given ? Call::like(dy) : FLOATS, n, c.hidden), d_o = c.whole(a[11], "d_o", FLOATS, n, c.hidden);
  const Arg dg = c.gate_like(a[12], "d_gate", Call::like(g), n);
  const Arg dwo = c.whole(a[13], "dw_out", Call::like(wo), c.hidden), dwi = c.whole(a[14], "dw_in", Call::like(wi), c.hidden);
  const Arg ws = c.scratch(a[15]);
  const int add = c.truth(a[16]);
  return c.run([&](void *st) {
    return f_block_bwd(static_cast<augtree_block_t *>(c.handle), dy.p, dy.given ? dy.code : dx.code, dh.p, dh.code, y.p, y.code, o.p, o.code, g.p, g.code,
                       wo.p, wi.p, wt, static_cast<const float *>(ro.p), static_cast<const float *>(ri.p), n, dx.p, d_o.p, d_o.code, dg.p, dwo.p, dwi.p,
                       add, ws.p, (size_t)ws.ld, st);
  });
}

// handle, x, ckpt
MARSHAL(ckpt_pack, 3) {
  Call c(a[0]);
  int64_t n, cols;
  c.rows(a[1], "x", n, cols);
  const Arg x = c.strided(a[1], "x", FLOATS, n, cols), k = c.whole(a[2], "ckpt", U8, n, c.pitch_of(cols));
  return c.run([&](void *st) { return f_ckpt_pack(static_cast<augtree_block_t *>(c.handle), x.p, x.code, x.ld, n, cols, k.p, st); });
}

// handle, ckpt, out, row, col
MARSHAL(ckpt_unpack, 5) {
  Call c(a[0]);
  int64_t n, cols;
  c.rows(a[2], "out", n, cols);
  const Arg out = c.strided(a[2], "out", FLOATS, n, cols), k = c.whole(a[1], "ckpt", U8, n, c.pitch_of(cols));
  const Arg row = c.whole(a[3], "row", F32, n), col = c.whole(a[4], "col", FLOATS, cols);
  return c.run([&](void *st) {
    return f_ckpt_unpack(static_cast<augtree_block_t *>(c.handle), k.p, n, cols, static_cast<const float *>(row.p), col.p, col.code, out.p, out.code, out.ld, st);
  });
}

// handle, g, u, a, ckpt_g, ckpt_u
MARSHAL(glu_fwd, 6) {
  Call c(a[0]);
  int64_t n, cols;
  c.rows(a[1], "g", n, cols);
  const Arg out = c.whole(a[3], "a", FLOATS, n, cols);
  if (a[3] == Py_None) c.fail("a: expected a tensor");
  const Arg g = c.strided(a[1], "g", Call::like(out), n, cols), u = c.strided(a[2], "u", Call::like(out), n, cols);
  if (g.ld != u.ld) c.fail("g, u: expected one leading size, got " + std::to_string(g.ld) + " and " + std::to_string(u.ld));
  const int64_t row = a[4] != Py_None || a[5] != Py_None ? c.pitch_of(cols) : 0;
  const Arg kg = c.whole(a[4], "ckpt_g", U8, n, row), ku = c.whole(a[5], "ckpt_u", U8, n, row);
  return c.run([&](void *st) { return f_glu_fwd(static_cast<augtree_block_t *>(c.handle), g.p, u.p, g.ld, out.code, n, cols, out.p, kg.p, ku.p, st); });
}

// handle, da, g, u, dg, du, a
MARSHAL(glu_bwd, 7) {
  Call c(a[0]);
  int64_t n, cols;
  c.rows(a[1], "da", n, cols);
  const Arg da = c.whole(a[1], "da", FLOATS, n, cols);
  const bool kept = c.is_u8(a[2]);
  Arg g, u;
  if (kept) {
    const int64_t row = c.pitch_of(cols);
    g = c.whole(a[2], "g", U8, n, row);
    u = c.whole(a[3], "u", U8, n, row);
  } else {
    g = c.strided(a[2], "g", Call::like(da), n, cols);
    u = c.strided(a[3], "u", Call::like(da), n, cols);
  }
  if (g.ld != u.ld) c.fail("g, u: expected one leading size, got " + std::to_string(g.ld) + " and " + std::to_string(u.ld));
  const Arg dg = c.strided(a[4], "dg", Call::like(da), n, cols), du = c.strided(a[5], "du", Call::like(da), n, cols);
  if (dg.ld != du.ld) c.fail("dg, du: expected one leading size, got " + std::to_string(dg.ld) + " and " + std::to_string(du.ld));
  const Arg out = c.whole(a[6], "a", Call::like(da), n, cols);
  return c.run([&](void *st) {
    return f_glu_bwd(static_cast<augtree_block_t *>(c.handle), da.p, da.code, g.p, u.p, g.ld, kept ? AUGTREE_CKPT : da.code, n, cols, dg.p, du.p, dg.ld, out.p, st);
  });
}

// handle, dy, ckpt, d_weight, ws, row, col, accumulate
MARSHAL(ckpt_wgrad, 8) {
  Call c(a[0]);
  int64_t n, m, out, cols;
  c.rows(a[1], "dy", n, m);
  c.rows(a[3], "d_weight", out, cols);
  const Arg dy = c.whole(a[1], "dy", BF16, n, m), k = c.whole(a[2], "ckpt", U8, n, c.pitch_of(cols)), dw = c.whole(a[3], "d_weight", BF16 | F32, m, cols);
  const Arg row = c.whole(a[5], "row", F32, n), col = c.whole(a[6], "col", FLOATS, cols), ws = c.scratch(a[4]);
  const int add = c.truth(a[7]);
  return c.run([&](void *st) {
    return f_ckpt_wgrad(static_cast<augtree_block_t *>(c.handle), dy.p, n, m, k.p, cols, static_cast<const float *>(row.p), col.p, col.code, dw.p, dw.code, add,
                        ws.p, (size_t)ws.ld, st);
  });
}

// addresses of the library's functions, in the order of the pointers above
PyObject *init(PyObject *, PyObject *const *a, Py_ssize_t n) {
  void *p[8];
  if (n != 8) { PyErr_SetString(PyExc_TypeError, "init: number of arguments"); return nullptr; }
  for (int i = 0; i < 8; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
  if (PyErr_Occurred()) return nullptr;
  f_block_fwd = reinterpret_cast<decltype(f_block_fwd)>(p[0]);
  f_block_bwd = reinterpret_cast<decltype(f_block_bwd)>(p[1]);
  f_ckpt_pitch = reinterpret_cast<decltype(f_ckpt_pitch)>(p[2]);
  f_ckpt_pack = reinterpret_cast<decltype(f_ckpt_pack)>(p[3]);
  f_ckpt_unpack = reinterpret_cast<decltype(f_ckpt_unpack)>(p[4]);
  f_glu_fwd = reinterpret_cast<decltype(f_glu_fwd)>(p[5]);
  f_glu_bwd = reinterpret_cast<decltype(f_glu_bwd)>(p[6]);
  f_ckpt_wgrad = reinterpret_cast<decltype(f_ckpt_wgrad)>(p[7]);
  Py_RETURN_NONE;
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(init), ENTRY(block_fwd), ENTRY(block_bwd), ENTRY(ckpt_pack), ENTRY(ckpt_unpack), ENTRY(glu_fwd), ENTRY(glu_bwd),
                         ENTRY(ckpt_wgrad), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of binding.Block.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
