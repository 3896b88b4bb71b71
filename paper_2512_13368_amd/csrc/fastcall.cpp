// Argument marshalling of binding.py in native code: the calls of a training or serving loop, with every tensor given
// by the caller.  A call through ctypes spends about 11 us in Python on its checks and conversions (each tensor's shape,
// type, layout and pointer; the parameter block; the stream), which is more than the GPU needs for a few short rows.
//
// Each function checks its arguments as binding.py does and calls the C ABI; it returns the error code, or None where an
// argument is missing or not as expected, and binding.py then takes its own path, which allocates or raises.
// Nothing is kept between calls.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/blossom.h"

namespace {

PyObject *g_fields[13];  // interned names of the parameter block's fields, in its order
PyObject *g_cuda_stream;
const char *kFields[13] = {"B", "H", "L", "d", "block", "topk", "window", "dtype", "softmax_scale", "stis_mode", "save_for_bwd", "stis_block",
                           "last_block_only"};

PyObject *g_paged_fields[13];
const char *kPagedFields[13] = {"S", "T", "H", "G", "d", "page", "n_pages", "max_pages", "dtype", "softmax_scale", "window", "max_len",
                                "table_per_head"};

PyObject *g_beam_fields[6];
const char *kBeamFields[6] = {"B", "W", "K", "V", "dtype", "eos"};

// One call's arguments, read in order; `ok` falls at the first that is not as expected.
struct Arguments {
  PyObject *const *arg;
  bool ok = true;
  at::ScalarType T{};
  void *stream = nullptr;
  int device = -1;     // of the tensors read so far
  bool mixed = false;  // they are on several

  explicit Arguments(PyObject *const *a) : arg(a) {}

  // the fields of a parameter block, the one at `real` a number, the others whole
  template <int N>
  bool fields(PyObject *const *names, int real, long (&v)[N], float *number)
  {
    PyObject *obj = *arg++;
    for (int i = 0; i < N && ok; ++i) {
      PyObject *x = PyObject_GetAttr(obj, names[i]);
      if (!x) return ok = false;
      if (i == real) *number = (float)PyFloat_AsDouble(x);
      else v[i] = PyLong_AsLong(x);
      Py_DECREF(x);
      ok = !PyErr_Occurred() && (i == real || v[i] == (int32_t)v[i]);
    }
    return ok;
  }
  void seen(const at::Tensor &t)
  {
    const int d = t.get_device();
    mixed = mixed || (device >= 0 && d != device);
    device = d;
  }
  // all of them on the current device, whose stream the call goes to
  void here() { ok = ok && !mixed && (device < 0 || c10::hip::device_count() == 0 || device == c10::hip::current_device()); }
  int32_t whole()
  {
    const long v = PyLong_AsLong(*arg++);
    ok = ok && !PyErr_Occurred() && v == (int32_t)v;
    return (int32_t)v;
  }
  float real()
  {
    const double v = PyFloat_AsDouble(*arg++);
    ok = ok && !PyErr_Occurred();
    return (float)v;
  }
  // contiguous device tensor of this shape and type (or, if `optional`, None)
  template <typename P = void>
  P *tensor(at::IntArrayRef shape, at::ScalarType type, bool optional = false)
  {
    PyObject *obj = *arg++;
    if (obj == Py_None) {
      ok = ok && optional;
      return nullptr;
    }
    if (!ok || !THPVariable_Check(obj)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor &t = THPVariable_Unpack(obj);
    ok = t.is_cuda() && t.scalar_type() == type && t.sizes() == shape && t.is_contiguous();
    if (ok) seen(t);
    return ok ? static_cast<P *>(t.data_ptr()) : nullptr;
  }
  // contiguous int32 rows [rows, *width], or [*width] where `rows` is 0
  int32_t *table(int64_t rows, int64_t *width)
  {
    PyObject *obj = *arg;
    *width = 0;
    if (ok && THPVariable_Check(obj)) {
      const at::Tensor &t = THPVariable_Unpack(obj);
      if (t.dim() == (rows ? 2 : 1)) *width = t.size(rows ? 1 : 0);
    }
    ok = ok && *width >= 1 && *width <= 0x7FFFFFFF;
    const int64_t two[2] = {rows, *width};
    return tensor<int32_t>(rows ? at::IntArrayRef(two, 2) : at::IntArrayRef(width, 1), at::kInt);
  }
  // [B, W] flags of one byte
  uint8_t *flags(at::IntArrayRef shape, bool optional)
  {
    PyObject *obj = *arg;
    const bool byte = obj != Py_None && THPVariable_Check(obj) && THPVariable_Unpack(obj).scalar_type() == at::kByte;
    return tensor<uint8_t>(shape, byte ? at::kByte : at::kBool, optional);
  }
  // a contiguous device tensor; None, or any tensor, only where `need` is 0
  void *workspace(size_t need, size_t *bytes)
  {
    PyObject *obj = *arg++;
    *bytes = 0;
    if (obj == Py_None) {
      ok = ok && need == 0;
      return nullptr;
    }
    if (!ok || !THPVariable_Check(obj)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor &t = THPVariable_Unpack(obj);
    ok = need == 0 || (t.is_cuda() && t.is_contiguous());
    if (!ok) return nullptr;
    if (need) seen(t);
    *bytes = t.nbytes();
    return t.data_ptr();
  }
  // None: torch's current stream
  void on_stream()
  {
    PyObject *obj = *arg++;
    if (!ok) return;
    if (obj == Py_None) {
      stream = (void *)c10::hip::getCurrentHIPStream().stream();
      return;
    }
    PyObject *x = PyObject_GetAttr(obj, g_cuda_stream);
    if (x) {
      stream = PyLong_AsVoidPtr(x);
      Py_DECREF(x);
    }
    ok = !PyErr_Occurred();
  }
  template <typename F>
  PyObject *run(F &&f)
  {
    if (!ok) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  }
};

// Arguments that begin with the attention layer's parameter block.
struct Call : Arguments {
  blossom_params p{};
  int64_t NB = 0;

  using Arguments::Arguments;

  bool params()
  {
    long v[13];
    if (!fields(g_fields, 8, v, &p.softmax_scale)) return false;
    p.B = (int32_t)v[0]; p.H = (int32_t)v[1]; p.L = (int32_t)v[2]; p.d = (int32_t)v[3]; p.block = (int32_t)v[4];
    p.topk = (int32_t)v[5]; p.window = (int32_t)v[6]; p.dtype = (int32_t)v[7]; p.stis_mode = (int32_t)v[9];
    p.save_for_bwd = (int32_t)v[10]; p.stis_block = (int32_t)v[11]; p.last_block_only = (int32_t)v[12];
    if (p.block < 1) return ok = false;
    NB = ((int64_t)p.L + p.block - 1) / p.block;
    T = p.dtype == 0 ? at::kFloat : at::kBFloat16;
    return true;
  }
};

// Arguments that begin with a paged cache's parameter block.
struct PagedCall : Arguments {
  blossom_paged_params p{};

  using Arguments::Arguments;

  bool params()
  {
    long v[13];
    if (!fields(g_paged_fields, 9, v, &p.softmax_scale)) return false;
    p.S = (int32_t)v[0]; p.T = (int32_t)v[1]; p.H = (int32_t)v[2]; p.G = (int32_t)v[3]; p.d = (int32_t)v[4];
    p.page = (int32_t)v[5]; p.n_pages = (int32_t)v[6]; p.max_pages = (int32_t)v[7]; p.dtype = (int32_t)v[8];
    p.window = (int32_t)v[10]; p.max_len = (int32_t)v[11]; p.table_per_head = (int32_t)v[12];
    T = p.dtype == 0 ? at::kFloat : at::kBFloat16;
    return true;
  }
  // [rows, heads, d] with contiguous heads and channels, rows that do not overlap (an expanded tensor's 0 would mean rows one after
  // another); *stride: elements from a row to the next
  void *rows(int64_t count, int64_t heads, int64_t *stride, bool optional = false)
  {
    PyObject *obj = *arg++;
    *stride = 0;
    if (obj == Py_None) {
      ok = ok && optional;
      return nullptr;
    }
    if (!ok || !THPVariable_Check(obj)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor &t = THPVariable_Unpack(obj);
    ok = t.is_cuda() && t.scalar_type() == T && t.dim() == 3 && t.size(0) == count && t.size(1) == heads && t.size(2) == p.d &&
         t.stride(2) == 1 && (heads == 1 || t.stride(1) == p.d) && (count <= 1 || t.stride(0) >= heads * p.d);
    if (!ok) return nullptr;
    seen(t);
    if (count > 1) *stride = t.stride(0);
    return t.data_ptr();
  }
};

// Arguments that begin with a beam search's parameter block.
struct BeamCall : Arguments {
  blossom_beam_params p{};

  using Arguments::Arguments;

  bool params()
  {
    long v[6];
    if (!fields(g_beam_fields, -1, v, nullptr)) return false;
    p = {(int32_t)v[0], (int32_t)v[1], (int32_t)v[2], (int32_t)v[3], (int32_t)v[4], (int32_t)v[5]};
    T = p.dtype == 0 ? at::kFloat : at::kBFloat16;
    return true;
  }
  // [B W, V], contiguous rows that do not overlap
  void *logits(int64_t *stride)
  {
    PyObject *obj = *arg++;
    *stride = 0;
    if (!ok || !THPVariable_Check(obj)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor &t = THPVariable_Unpack(obj);
    const int64_t rows = (int64_t)p.B * p.W;
    ok = t.is_cuda() && t.scalar_type() == T && t.dim() == 2 && t.size(0) == rows && t.size(1) == p.V && (p.V <= 1 || t.stride(1) == 1) &&
         (rows <= 1 || t.stride(0) >= p.V);
    if (!ok) return nullptr;
    seen(t);
    if (rows > 1) *stride = t.stride(0);
    return t.data_ptr();
  }
};

#define FASTCALL_OF(Call, name, count)                                            \
  PyObject *name##_body(Call &c);                                                 \
  PyObject *name(PyObject *, PyObject *const *args, Py_ssize_t n)                 \
  {                                                                               \
    if (n != (count)) {                                                           \
      PyErr_SetString(PyExc_TypeError, #name " takes " #count " arguments");      \
      return nullptr;                                                             \
    }                                                                             \
    try {                                                                         \
      Call c(args);                                                               \
      if (!c.params()) {                                                          \
        PyErr_Clear();                                                            \
        Py_RETURN_NONE;                                                           \
      }                                                                           \
      return name##_body(c);                                                      \
    } catch (...) { /* a tensor without storage and the like: binding.py says what is wrong */ \
      PyErr_Clear();                                                              \
      Py_RETURN_NONE;                                                             \
    }                                                                             \
  }                                                                               \
  PyObject *name##_body(Call &c)
#define FASTCALL(name, count) FASTCALL_OF(Call, name, count)

// select_blocks(p, Q, K, valid_len, sel, ws, stream)
FASTCALL(select_blocks, 7)
{
  const blossom_params &p = c.p;
  const int64_t x[4] = {p.B, p.H, p.L, p.d}, s[4] = {p.B, p.H, c.NB, p.topk}, b[1] = {p.B};
  void *Q = c.tensor(x, c.T), *K = c.tensor(x, c.T);
  int32_t *vl = c.tensor<int32_t>(b, at::kInt), *sel = c.tensor<int32_t>(s, at::kInt);
  size_t bytes;
  void *ws = c.workspace(1, &bytes);
  c.on_stream();
  return c.run([&] { return blossom_select_blocks(&p, Q, K, vl, sel, ws, bytes, c.stream); });
}

// rope_select_blocks(p, Q, K, rope_cos, rope_sin, valid_len, Q_rot, K_rot, sel, ws, stream)
FASTCALL(rope_select_blocks, 11)
{
  const blossom_params &p = c.p;
  const int64_t x[4] = {p.B, p.H, p.L, p.d}, s[4] = {p.B, p.H, c.NB, p.topk}, r[2] = {p.L, p.d / 2}, b[1] = {p.B};
  void *Q = c.tensor(x, c.T), *K = c.tensor(x, c.T);
  float *cos = c.tensor<float>(r, at::kFloat), *sin = c.tensor<float>(r, at::kFloat);
  int32_t *vl = c.tensor<int32_t>(b, at::kInt);
  void *Qr = c.tensor(x, c.T), *Kr = c.tensor(x, c.T);
  int32_t *sel = c.tensor<int32_t>(s, at::kInt);
  size_t bytes;
  void *ws = c.workspace(1, &bytes);
  c.on_stream();
  return c.run([&] { return blossom_rope_select_blocks(&p, Q, K, cos, sin, vl, Qr, Kr, sel, ws, bytes, c.stream); });
}

// select_positions(p, kv_groups, cmp_block, cmp_stride, Q, K, valid_len, score_scale, sel_pos, ws, stream)
FASTCALL(select_positions, 11)
{
  const blossom_params &p = c.p;
  const int32_t G = c.whole(), l = c.whole(), st = c.whole();
  const int64_t q[4] = {p.B, p.H, p.L, p.d}, k[4] = {p.B, G, p.L, p.d}, s[4] = {p.B, G, p.L, p.topk}, b[1] = {p.B};
  void *Q = c.tensor(q, c.T), *K = c.tensor(k, c.T);
  int32_t *vl = c.tensor<int32_t>(b, at::kInt);
  const float scale = c.real();
  int32_t *sel = c.tensor<int32_t>(s, at::kInt);
  size_t bytes;
  void *ws = c.workspace(1, &bytes);
  c.on_stream();
  return c.run([&] { return blossom_select_positions(&p, G, l, st, scale, Q, K, vl, sel, ws, bytes, c.stream); });
}

// The forward's arguments from Q on: G key/value groups, selection rows of shape `s`.
struct FwdTensors {
  void *Q, *K, *V;
  int32_t *vl, *sel;
  float *gw, *gb;
  void *O;
  float *o_lt, *o_st, *lse_lt, *lse_st;
  FwdTensors(Call &c, int64_t G, at::IntArrayRef s)
  {
    const blossom_params &p = c.p;
    const int64_t x[4] = {p.B, p.H, p.L, p.d}, k[4] = {p.B, G, p.L, p.d}, b[1] = {p.B}, w[2] = {p.H, 2 * (int64_t)p.d}, h[1] = {p.H};
    const at::IntArrayRef row(x, 3);
    Q = c.tensor(x, c.T);
    K = c.tensor(k, c.T);
    V = c.tensor(k, c.T);
    vl = c.tensor<int32_t>(b, at::kInt);
    sel = c.tensor<int32_t>(s, at::kInt);
    gw = c.tensor<float>(w, at::kFloat);
    gb = c.tensor<float>(h, at::kFloat, true);
    O = c.tensor(x, c.T);
    o_lt = c.tensor<float>(x, at::kFloat, true);
    o_st = c.tensor<float>(x, at::kFloat, true);
    lse_lt = c.tensor<float>(row, at::kFloat, true);
    lse_st = c.tensor<float>(row, at::kFloat, true);
  }
};

// attn_fwd(p, Q, K, V, valid_len, sel, gate_w, gate_b, O, o_lt, o_st, lse_lt, lse_st, ws, stream)
FASTCALL(attn_fwd, 15)
{
  const blossom_params &p = c.p;
  const int64_t s[4] = {p.B, p.H, c.NB, p.topk};
  const FwdTensors t(c, p.H, s);
  size_t bytes;
  void *ws = c.workspace(blossom_workspace_bytes(&p, BLOSSOM_WS_FWD), &bytes);
  c.on_stream();
  return c.run([&] {
    return blossom_attn_fwd(&p, t.Q, t.K, t.V, t.vl, t.sel, t.gw, t.gb, t.O, t.o_lt, t.o_st, t.lse_lt, t.lse_st, ws, bytes, c.stream);
  });
}

// attn_fwd_positions(p, kv_groups, Q, K, V, valid_len, sel_pos, gate_w, gate_b, O, o_lt, o_st, lse_lt, lse_st, stream)
FASTCALL(attn_fwd_positions, 15)
{
  const blossom_params &p = c.p;
  const int32_t G = c.whole();
  const int64_t s[4] = {p.B, G, p.L, p.topk};
  const FwdTensors t(c, G, s);
  c.on_stream();
  return c.run([&] {
    return blossom_attn_fwd_positions(&p, G, t.Q, t.K, t.V, t.vl, t.sel, t.gw, t.gb, t.O, t.o_lt, t.o_st, t.lse_lt, t.lse_st, c.stream);
  });
}

// The backward's arguments from Q on.
struct BwdTensors {
  void *Q, *K, *V;
  int32_t *vl, *sel;
  float *gw, *gb, *o_lt, *o_st, *lse_lt, *lse_st;
  void *dO, *dQ, *dK, *dV;
  float *dgw, *dgb;
  void *ws;
  size_t bytes;
  BwdTensors(Call &c, int64_t G, at::IntArrayRef s)
  {
    const blossom_params &p = c.p;
    const int64_t x[4] = {p.B, p.H, p.L, p.d}, k[4] = {p.B, G, p.L, p.d}, b[1] = {p.B}, w[2] = {p.H, 2 * (int64_t)p.d}, h[1] = {p.H};
    const at::IntArrayRef row(x, 3);
    Q = c.tensor(x, c.T);
    K = c.tensor(k, c.T);
    V = c.tensor(k, c.T);
    vl = c.tensor<int32_t>(b, at::kInt);
    sel = c.tensor<int32_t>(s, at::kInt);
    gw = c.tensor<float>(w, at::kFloat);
    gb = c.tensor<float>(h, at::kFloat, true);
    o_lt = c.tensor<float>(x, at::kFloat);
    o_st = c.tensor<float>(x, at::kFloat);
    lse_lt = c.tensor<float>(row, at::kFloat);
    lse_st = c.tensor<float>(row, at::kFloat);
    dO = c.tensor(x, c.T);
    dQ = c.tensor(x, c.T);
    dK = c.tensor(k, c.T);
    dV = c.tensor(k, c.T);
    dgw = c.tensor<float>(w, at::kFloat);
    dgb = c.tensor<float>(h, at::kFloat);
    ws = c.workspace(1, &bytes);
  }
};

// attn_bwd(p, Q, K, V, valid_len, sel, gate_w, gate_b, o_lt, o_st, lse_lt, lse_st, dO, dQ, dK, dV, d_gate_w, d_gate_b, ws,
//          rope_cos, rope_sin, stream); both tables None: blossom_attn_bwd, else blossom_attn_bwd_rope
FASTCALL(attn_bwd, 22)
{
  const blossom_params &p = c.p;
  const int64_t s[4] = {p.B, p.H, c.NB, p.topk}, r[2] = {p.L, p.d / 2};
  const BwdTensors t(c, p.H, s);
  float *cos = c.tensor<float>(r, at::kFloat, true), *sin = c.tensor<float>(r, at::kFloat, true);
  c.ok = c.ok && !cos == !sin;
  c.on_stream();
  return c.run([&] {
    if (cos)
      return blossom_attn_bwd_rope(&p, t.Q, t.K, t.V, t.vl, t.sel, t.gw, t.gb, t.o_lt, t.o_st, t.lse_lt, t.lse_st, t.dO, cos, sin,
                                   t.dQ, t.dK, t.dV, t.dgw, t.dgb, t.ws, t.bytes, c.stream);
    return blossom_attn_bwd(&p, t.Q, t.K, t.V, t.vl, t.sel, t.gw, t.gb, t.o_lt, t.o_st, t.lse_lt, t.lse_st, t.dO, t.dQ, t.dK, t.dV,
                            t.dgw, t.dgb, t.ws, t.bytes, c.stream);
  });
}

// attn_bwd_positions(p, kv_groups, Q, K, V, valid_len, sel_pos, gate_w, gate_b, o_lt, o_st, lse_lt, lse_st, dO, dQ, dK, dV,
//                    d_gate_w, d_gate_b, ws, stream)
FASTCALL(attn_bwd_positions, 21)
{
  const blossom_params &p = c.p;
  const int32_t G = c.whole();
  const int64_t s[4] = {p.B, G, p.L, p.topk};
  const BwdTensors t(c, G, s);
  c.on_stream();
  return c.run([&] {
    return blossom_attn_bwd_positions(&p, G, t.Q, t.K, t.V, t.vl, t.sel, t.gw, t.gb, t.o_lt, t.o_st, t.lse_lt, t.lse_st, t.dO, t.dQ,
                                      t.dK, t.dV, t.dgw, t.dgb, t.ws, t.bytes, c.stream);
  });
}

// out_proj_ln(p, d_model, O, W_O_t, bias, H_prev, ln_gamma, ln_beta, ln_eps, S, mean, rstd, stream)
FASTCALL(out_proj_ln, 13)
{
  const blossom_params &p = c.p;
  const int32_t dm = c.whole();
  const int64_t x[4] = {p.B, p.H, p.L, p.d}, w[2] = {dm, (int64_t)p.H * p.d}, h[3] = {p.B, p.L, dm}, g[1] = {dm};
  const at::IntArrayRef row(h, 2);
  void *O = c.tensor(x, c.T), *W = c.tensor(w, c.T);
  float *bias = c.tensor<float>(g, at::kFloat, true);
  void *prev = c.tensor(h, c.T);
  float *gamma = c.tensor<float>(g, at::kFloat), *beta = c.tensor<float>(g, at::kFloat);
  const float eps = c.real();
  void *S = c.tensor(h, c.T);
  float *mean = c.tensor<float>(row, at::kFloat, true), *rstd = c.tensor<float>(row, at::kFloat, true);
  c.on_stream();
  return c.run([&] { return blossom_out_proj_ln(&p, dm, O, W, bias, prev, gamma, beta, eps, S, mean, rstd, c.stream); });
}

// The cache's tensors as every paged call has them.
struct CacheTensors {
  int32_t *table, *cu = nullptr, *len;
  void *K, *V;
  int32_t *get_table(PagedCall &c)
  {
    const blossom_paged_params &p = c.p;
    const int64_t per_head[3] = {p.S, p.G, p.max_pages}, one[2] = {p.S, p.max_pages};
    return c.tensor<int32_t>(p.table_per_head ? at::IntArrayRef(per_head, 3) : at::IntArrayRef(one, 2), at::kInt);
  }
  void *get_cache(PagedCall &c)
  {
    const int64_t x[4] = {c.p.n_pages, c.p.G, c.p.page, c.p.d};
    return c.tensor(x, c.T);
  }
  int32_t *get_counts(PagedCall &c, int64_t n) { return c.tensor<int32_t>(at::IntArrayRef(&n, 1), at::kInt); }
};

// kv_append(p, Q, K, V, rope_cos, rope_sin, page_table, cu_seqlens, kv_len, K_cache, V_cache, Q_rot, stream)
FASTCALL_OF(PagedCall, kv_append, 13)
{
  const blossom_paged_params &p = c.p;
  const int64_t held = (int64_t)p.max_pages * p.page, cap = p.max_len > 0 && p.max_len < held ? p.max_len : held;
  const int64_t x[3] = {p.T, p.H, p.d}, r[2] = {cap, p.d / 2};
  int64_t qs, ks, vs;
  void *Q = c.rows(p.T, p.H, &qs, true), *K = c.rows(p.T, p.G, &ks), *V = c.rows(p.T, p.G, &vs);
  float *cos = c.tensor<float>(r, at::kFloat, true), *sin = c.tensor<float>(r, at::kFloat, true);
  CacheTensors t;
  t.table = t.get_table(c);
  t.cu = t.get_counts(c, (int64_t)p.S + 1);
  t.len = t.get_counts(c, p.S);
  t.K = t.get_cache(c);
  t.V = t.get_cache(c);
  void *Q_rot = c.tensor(x, c.T, true);
  c.on_stream();
  return c.run([&] { return blossom_kv_append(&p, Q, qs, K, ks, V, vs, cos, sin, t.table, t.cu, t.len, t.K, t.V, Q_rot, c.stream); });
}

// attn_decode(p, Q, K_cache, V_cache, page_table, kv_len, O, lse, ws, stream)
FASTCALL_OF(PagedCall, attn_decode, 10)
{
  const blossom_paged_params &p = c.p;
  const int64_t x[3] = {p.S, p.H, p.d};
  int64_t qs;
  void *Q = c.rows(p.S, p.H, &qs);
  CacheTensors t;
  t.K = t.get_cache(c);
  t.V = t.get_cache(c);
  t.table = t.get_table(c);
  t.len = t.get_counts(c, p.S);
  void *O = c.tensor(x, c.T);
  float *lse = c.tensor<float>(at::IntArrayRef(x, 2), at::kFloat, true);
  size_t bytes;
  void *ws = c.workspace(blossom_paged_workspace_bytes(&p, BLOSSOM_WS_DECODE), &bytes);
  c.on_stream();
  return c.run([&] { return blossom_attn_decode(&p, Q, qs, t.K, t.V, t.table, t.len, O, lse, ws, bytes, c.stream); });
}

// attn_prompt(p, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, O, lse, ws, stream)
FASTCALL_OF(PagedCall, attn_prompt, 11)
{
  const blossom_paged_params &p = c.p;
  const int64_t x[3] = {p.T, p.H, p.d};
  int64_t qs;
  void *Q = c.rows(p.T, p.H, &qs);
  CacheTensors t;
  t.K = t.get_cache(c);
  t.V = t.get_cache(c);
  t.table = t.get_table(c);
  t.cu = t.get_counts(c, (int64_t)p.S + 1);
  t.len = t.get_counts(c, p.S);
  void *O = c.tensor(x, c.T);
  float *lse = c.tensor<float>(at::IntArrayRef(x, 2), at::kFloat, true);
  size_t bytes;
  void *ws = c.workspace(blossom_paged_workspace_bytes(&p, BLOSSOM_WS_PROMPT), &bytes);
  c.on_stream();
  return c.run([&] { return blossom_attn_prompt(&p, Q, qs, t.K, t.V, t.table, t.cu, t.len, O, lse, ws, bytes, c.stream); });
}

// kv_append_tree(p, Q, K, V, rope_cos, rope_sin, page_table, cu_seqlens, kv_len, tree_mask, K_cache, V_cache, Q_rot, stream)
FASTCALL_OF(PagedCall, kv_append_tree, 14)
{
  const blossom_paged_params &p = c.p;
  const int64_t held = (int64_t)p.max_pages * p.page, cap = p.max_len > 0 && p.max_len < held ? p.max_len : held;
  const int64_t x[3] = {p.T, p.H, p.d}, r[2] = {cap, p.d / 2};
  int64_t qs, ks, vs;
  void *Q = c.rows(p.T, p.H, &qs, true), *K = c.rows(p.T, p.G, &ks), *V = c.rows(p.T, p.G, &vs);
  float *cos = c.tensor<float>(r, at::kFloat, true), *sin = c.tensor<float>(r, at::kFloat, true);
  CacheTensors t;
  t.table = t.get_table(c);
  t.cu = t.get_counts(c, (int64_t)p.S + 1);
  t.len = t.get_counts(c, p.S);
  int64_t *mask = c.tensor<int64_t>(at::IntArrayRef(x, 1), at::kLong);
  t.K = t.get_cache(c);
  t.V = t.get_cache(c);
  void *Q_rot = c.tensor(x, c.T, true);
  c.here();
  c.on_stream();
  return c.run([&] { return blossom_kv_append_tree(&p, Q, qs, K, ks, V, vs, cos, sin, t.table, t.cu, t.len, mask, t.K, t.V, Q_rot, c.stream); });
}

// attn_tree(p, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, tree_mask, O, lse, ws, stream)
FASTCALL_OF(PagedCall, attn_tree, 12)
{
  const blossom_paged_params &p = c.p;
  const int64_t x[3] = {p.T, p.H, p.d};
  int64_t qs;
  void *Q = c.rows(p.T, p.H, &qs);
  CacheTensors t;
  t.K = t.get_cache(c);
  t.V = t.get_cache(c);
  t.table = t.get_table(c);
  t.cu = t.get_counts(c, (int64_t)p.S + 1);
  t.len = t.get_counts(c, p.S);
  int64_t *mask = c.tensor<int64_t>(at::IntArrayRef(x, 1), at::kLong);
  void *O = c.tensor(x, c.T);
  float *lse = c.tensor<float>(at::IntArrayRef(x, 2), at::kFloat, true);
  size_t bytes;
  void *ws = c.workspace(blossom_paged_workspace_bytes(&p, BLOSSOM_WS_TREE), &bytes);
  c.here();
  c.on_stream();
  return c.run([&] { return blossom_attn_tree(&p, Q, qs, t.K, t.V, t.table, t.cu, t.len, mask, O, lse, ws, bytes, c.stream); });
}

// kv_accept(p, keep, K_cache, V_cache, page_table, cu_seqlens, kv_len, new_len, stream)
FASTCALL_OF(PagedCall, kv_accept, 9)
{
  const blossom_paged_params &p = c.p;
  int64_t width;
  int32_t *keep = c.table(p.S, &width);
  CacheTensors t;
  t.K = t.get_cache(c);
  t.V = t.get_cache(c);
  t.table = t.get_table(c);
  t.cu = t.get_counts(c, (int64_t)p.S + 1);
  t.len = t.get_counts(c, p.S);
  int32_t *new_len = t.get_counts(c, p.S);
  c.here();
  c.on_stream();
  return c.run([&] { return blossom_kv_accept(&p, (int32_t)width, keep, t.table, t.cu, t.len, t.K, t.V, new_len, c.stream); });
}

// kv_fork(p, parent, page_table, kv_len, refs, grow, new_table, new_len, new_refs, copies, missing, ws, stream)
FASTCALL_OF(PagedCall, kv_fork, 13)
{
  const blossom_paged_params &p = c.p;
  int64_t N;
  int32_t *parent = c.table(0, &N);
  const int64_t from[2] = {p.S, p.max_pages}, to[2] = {N, p.max_pages}, three[2] = {N, 3};
  CacheTensors t;
  t.table = c.tensor<int32_t>(from, at::kInt);
  t.len = t.get_counts(c, p.S);
  int32_t *refs = t.get_counts(c, p.n_pages);
  const int32_t grow = c.whole();
  int32_t *new_table = c.tensor<int32_t>(to, at::kInt), *new_len = t.get_counts(c, N), *new_refs = t.get_counts(c, p.n_pages);
  int32_t *copies = c.tensor<int32_t>(three, at::kInt), *missing = t.get_counts(c, 1);
  size_t bytes;
  void *ws = c.workspace(1, &bytes);
  c.here();
  c.on_stream();
  return c.run([&] {
    return blossom_kv_fork(&p, (int32_t)N, grow, parent, t.table, t.len, refs, new_table, new_len, new_refs, copies, missing, ws, bytes, c.stream);
  });
}

// kv_copy_pages(p, copies, K_cache, V_cache, stream)
FASTCALL_OF(PagedCall, kv_copy_pages, 5)
{
  const blossom_paged_params &p = c.p;
  int64_t n = 0;
  if (THPVariable_Check(*c.arg) && THPVariable_Unpack(*c.arg).dim() == 2) n = THPVariable_Unpack(*c.arg).size(0);
  c.ok = c.ok && n >= 1 && n <= 0x7FFFFFFF;
  const int64_t three[2] = {n, 3};
  int32_t *copies = c.tensor<int32_t>(three, at::kInt);
  CacheTensors t;
  t.K = t.get_cache(c);
  t.V = t.get_cache(c);
  c.here();
  c.on_stream();
  return c.run([&] { return blossom_kv_copy_pages(&p, (int32_t)n, copies, t.K, t.V, c.stream); });
}

// beam_select(p, logits, score, ended, parent, token, out_score, out_ended, ws, stream)
FASTCALL_OF(BeamCall, beam_select, 10)
{
  const blossom_beam_params &p = c.p;
  const int64_t in[2] = {p.B, p.W}, out[2] = {p.B, p.K};
  int64_t stride;
  void *logits = c.logits(&stride);
  float *score = c.tensor<float>(in, at::kFloat);
  uint8_t *ended = c.flags(in, true);
  int32_t *parent = c.tensor<int32_t>(out, at::kInt), *token = c.tensor<int32_t>(out, at::kInt);
  float *out_score = c.tensor<float>(out, at::kFloat);
  uint8_t *out_ended = c.flags(out, false);
  size_t bytes;
  void *ws = c.workspace(1, &bytes);
  c.here();
  c.on_stream();
  return c.run([&] { return blossom_beam_select(&p, logits, stride, score, ended, parent, token, out_score, out_ended, ws, bytes, c.stream); });
}

#define ENTRY(name) {#name, (PyCFunction)(void *)name, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {ENTRY(select_blocks), ENTRY(rope_select_blocks), ENTRY(select_positions), ENTRY(attn_fwd),
                          ENTRY(attn_fwd_positions), ENTRY(attn_bwd), ENTRY(attn_bwd_positions), ENTRY(out_proj_ln),
                          ENTRY(kv_append), ENTRY(attn_decode), ENTRY(attn_prompt), ENTRY(kv_append_tree), ENTRY(attn_tree),
                          ENTRY(kv_accept), ENTRY(kv_fork), ENTRY(kv_copy_pages), ENTRY(beam_select),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall()
{
  for (int i = 0; i < 13; ++i)
    if (!(g_fields[i] = PyUnicode_InternFromString(kFields[i])) || !(g_paged_fields[i] = PyUnicode_InternFromString(kPagedFields[i])))
      return nullptr;
  for (int i = 0; i < 6; ++i)
    if (!(g_beam_fields[i] = PyUnicode_InternFromString(kBeamFields[i]))) return nullptr;
  if (!(g_cuda_stream = PyUnicode_InternFromString("cuda_stream"))) return nullptr;
  return PyModule_Create(&kModule);
}
