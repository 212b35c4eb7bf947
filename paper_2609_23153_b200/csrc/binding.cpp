// Argument marshalling of the Python binding's per-layer calls, in native code: shape descriptor, output and workspace
// tensors, stream, call.  The Python functions of the same names (__init__.py) keep the interface and raise the errors;
// what is here is what they would otherwise do object by object.  No tensor data is touched.
//
// Why: a small call is bound by the host.  fwd() over 2 heads of 2,048 tokens spends 12.5 us on the device and took 16.3 us
// of host time: 5.2 in the library (two launches, three tensor maps), the rest in ctypes conversions, a Shape object, a
// workspace query and the tuples of sizes and strides behind each check.  Now 8.1, and the call takes what the device takes:
// 16.5 -> 12.6 us; selection + forward of 3 heads of 1,200 tokens 36.4 -> 19.0.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstring>
#include <initializer_list>

#include "../../include/sparkattn.h"

namespace {

// Entry points of the library that the Python side has loaded (bind()).
struct Library {
  decltype(&sparkattn_workspace_bytes) workspace_bytes;
  decltype(&sparkattn_select) select;
  decltype(&sparkattn_select_window) select_window;
  decltype(&sparkattn_select_padded) select_padded;
  decltype(&sparkattn_select_pooled) select_pooled;
  decltype(&sparkattn_quant_fp8) quant_fp8;
  decltype(&sparkattn_quant_fp8_pooled) quant_fp8_pooled;
  decltype(&sparkattn_quant_fp8_per_token) quant_fp8_per_token;
  decltype(&sparkattn_fwd) fwd;
  decltype(&sparkattn_fwd_window) fwd_window;
  decltype(&sparkattn_fwd_padded) fwd_padded;
  decltype(&sparkattn_gather_tokens) gather_tokens;
  decltype(&sparkattn_comp_workspace_bytes) comp_workspace_bytes;
  decltype(&sparkattn_comp_state) comp_state;
  decltype(&sparkattn_comp_apply) comp_apply;
  decltype(&sparkattn_fwd_gated_workspace_bytes) fwd_gated_workspace_bytes;
  decltype(&sparkattn_fwd_gated) fwd_gated;
  decltype(&sparkattn_cache_workspace_bytes) cache_workspace_bytes;
  decltype(&sparkattn_cache_append) cache_append;
  decltype(&sparkattn_cache_fwd) cache_fwd;
};
Library g_lib{};

// A stream's handle, or the current stream of the current device, asked for when the call is made.
struct Stream {
  void* handle = nullptr;
  bool given = false;
  operator void*() const { return given ? handle : c10::cuda::getCurrentCUDAStream().stream(); }
  // Memory that a call allocates for a stream of the caller's comes from that stream's: the current stream's may still be read
  // or written there, and would be handed out again before this one is through with it (a workspace: at the call's return).
  at::Tensor scratch(int64_t bytes, const at::Tensor& like) const {
    return allocate(like, [&] { return at::empty({bytes}, like.options().dtype(at::kByte)); });
  }
  // An output is read on the current stream, too: not handed out again before that one is through with it either.
  at::Tensor output(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) const {
    return read_here(allocate(like, [&] { return at::empty(sizes, like.options().dtype(type)); }));
  }
  at::Tensor output_like(const at::Tensor& like, at::ScalarType type) const {      // its strides as well
    return read_here(allocate(like, [&] { return at::empty_strided(like.sizes(), like.strides(), like.options().dtype(type)); }));
  }

 private:
  template <typename Make>
  at::Tensor allocate(const at::Tensor& like, Make make) const {
    if (!given || !like.is_cuda()) return make();
    c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(handle), like.device().index()));
    return make();
  }
  at::Tensor read_here(at::Tensor x) const {
    if (given && x.is_cuda()) x.record_stream(c10::cuda::getCurrentCUDAStream(x.device().index()));
    return x;
  }
};

// The arguments of one call, taken in order; the first one of a wrong kind raises.
class Args {
 public:
  Args(PyObject* const* args, Py_ssize_t n) : args_(args), n_(n) {}
  void expect(Py_ssize_t n) const { TORCH_CHECK_TYPE(n_ == n, "expected ", n, " arguments, got ", n_); }
  at::Tensor tensor() {
    PyObject* o = next();
    TORCH_CHECK_TYPE(THPVariable_Check(o), "expected a tensor, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
  }
  at::Tensor optional_tensor() {      // undefined for None
    if (args_[at_] == Py_None) { ++at_; return at::Tensor(); }
    return tensor();
  }
  int64_t integer() {
    const long long v = PyLong_AsLongLong(next());
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
  }
  int32_t i32() {
    const int64_t v = integer();
    TORCH_CHECK_VALUE(v == (int32_t)v, v, " does not fit 32 bits");
    return (int32_t)v;
  }
  float number() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
  }
  bool truth() {
    const int v = PyObject_IsTrue(next());
    if (v < 0) throw python_error();
    return v != 0;
  }
  Stream stream() {
    if (args_[at_] == Py_None) { ++at_; return {}; }
    return {(void*)(intptr_t)integer(), true};
  }

 private:
  PyObject* next() { return args_[at_++]; }
  PyObject* const* args_;
  Py_ssize_t n_, at_ = 0;
};

sparkattn_shape_t make_shape(const at::Tensor& x, int32_t block, float softmax_scale = 0.0f) {
  TORCH_CHECK_VALUE(x.dim() == 4 && x.stride(3) == 1, "expected a [B, H, N, d] tensor with a contiguous last dimension");
  sparkattn_shape_t s{};
  s.struct_size = sizeof(s);
  s.version = SPARKATTN_VERSION;
  s.B = (int32_t)x.size(0); s.H = (int32_t)x.size(1); s.N = (int32_t)x.size(2); s.d = (int32_t)x.size(3);
  s.block = block;
  s.stride_b = x.stride(0); s.stride_h = x.stride(1); s.stride_n = x.stride(2);
  s.softmax_scale = softmax_scale;
  return s;
}

void same_layout(const at::Tensor& a, const at::Tensor& b) {
  TORCH_CHECK_VALUE(a.sizes() == b.sizes() && a.strides() == b.strides(), "tensors of one call must share shape and strides");
}

void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
int32_t* iptr(const at::Tensor& t) { return static_cast<int32_t*>(ptr(t)); }
float* fptr(const at::Tensor& t) { return static_cast<float*>(ptr(t)); }
// Token blocks of a head.  Outputs are sized with it before the library has looked at the shape: a block size below 1,
// which the library refuses, has none.
int64_t blocks(const sparkattn_shape_t& s) { return s.block < 1 ? 0 : ((int64_t)s.N + s.block - 1) / s.block; }

// The caller's workspace, or a new one; undefined when the library does not serve the shape.
at::Tensor workspace_for(at::Tensor given, const sparkattn_shape_t& s, int32_t which, int32_t k, const at::Tensor& x, const Stream& stream) {
  if (given.defined()) return given;
  const size_t n = g_lib.workspace_bytes(&s, which, k);
  return n == 0 ? at::Tensor() : stream.scratch((int64_t)n, x);
}

PyObject* result(int rc, std::initializer_list<at::Tensor> tensors) {
  PyObject* t = PyTuple_New((Py_ssize_t)tensors.size() + 1);
  if (t == nullptr) throw python_error();
  PyTuple_SET_ITEM(t, 0, PyLong_FromLong(rc));
  Py_ssize_t i = 1;
  for (const at::Tensor& x : tensors) {
    if (x.defined()) {
      PyTuple_SET_ITEM(t, i++, THPVariable_Wrap(x));
    } else {
      Py_INCREF(Py_None);
      PyTuple_SET_ITEM(t, i++, Py_None);
    }
  }
  return t;
}
// workspace_for() found no workspace: what the Python side raises for the query that returned 0
constexpr int kNoWorkspace = 1;

// select(q, k, block, topk, kept_idx, kept_cnt, workspace, stream, frame_tokens, window, block_valid) -> rc, kept_idx, kept_cnt
PyObject* select(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(11);
  const at::Tensor q = a.tensor(), k = a.tensor();
  const int32_t block = a.i32(), topk = a.i32();
  at::Tensor idx = a.optional_tensor(), cnt = a.optional_tensor(), ws = a.optional_tensor();
  const Stream stream = a.stream();
  const int32_t frame_tokens = a.i32(), window = a.i32();
  const at::Tensor valid = a.optional_tensor();
  same_layout(q, k);
  const sparkattn_shape_t s = make_shape(q, block);
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (!idx.defined()) idx = stream.output({s.B, s.H, blocks(s), std::max(topk, 1)}, at::kInt, q);
    if (!cnt.defined()) cnt = stream.output({s.B, s.H, blocks(s)}, at::kInt, q);
    ws = workspace_for(ws, s, 0, topk, q, stream);
    if (!ws.defined()) rc = kNoWorkspace;
    else if (valid.defined())
      rc = g_lib.select_padded(&s, ptr(q), ptr(k), topk, iptr(valid), iptr(idx), iptr(cnt), ptr(ws), (size_t)ws.numel(), stream);
    else if (frame_tokens > 0)
      rc = g_lib.select_window(&s, ptr(q), ptr(k), topk, frame_tokens, window, iptr(idx), iptr(cnt), ptr(ws), (size_t)ws.numel(), stream);
    else
      rc = g_lib.select(&s, ptr(q), ptr(k), topk, iptr(idx), iptr(cnt), ptr(ws), (size_t)ws.numel(), stream);
  }
  return result(rc, {idx, cnt});
  END_HANDLE_TH_ERRORS
}

// select_pooled(ref, block, topk, workspace, kept_idx, kept_cnt, stream) -> rc, kept_idx, kept_cnt
PyObject* select_pooled(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(7);
  const at::Tensor ref = a.tensor();
  const int32_t block = a.i32(), topk = a.i32();
  const at::Tensor ws = a.tensor();
  at::Tensor idx = a.optional_tensor(), cnt = a.optional_tensor();
  const Stream stream = a.stream();
  const sparkattn_shape_t s = make_shape(ref, block);
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (!idx.defined()) idx = stream.output({s.B, s.H, blocks(s), std::max(topk, 1)}, at::kInt, ref);
    if (!cnt.defined()) cnt = stream.output({s.B, s.H, blocks(s)}, at::kInt, ref);
    rc = g_lib.select_pooled(&s, topk, iptr(idx), iptr(cnt), ptr(ws), (size_t)ws.numel(), stream);
  }
  return result(rc, {idx, cnt});
  END_HANDLE_TH_ERRORS
}

// What the three quantisation calls share: codes (laid out like x) and scales [B, H, per_head] where the caller brings none.
template <typename Call>
PyObject* quantise(const at::Tensor& x, const sparkattn_shape_t& s, int64_t per_head, at::Tensor codes, at::Tensor scales, const Stream& stream, Call call) {
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (!codes.defined()) codes = stream.output_like(x, at::kByte);
    if (!scales.defined()) scales = stream.output({s.B, s.H, per_head}, at::kFloat, x);
    rc = call(&s, ptr(x), static_cast<uint8_t*>(ptr(codes)), fptr(scales));
  }
  return result(rc, {codes, scales});
}

// quant_fp8(x, block, codes, scales, stream) -> rc, codes, scales
PyObject* quant_fp8(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(5);
  const at::Tensor x = a.tensor();
  const sparkattn_shape_t s = make_shape(x, a.i32());
  const at::Tensor codes = a.optional_tensor(), scales = a.optional_tensor();
  const Stream stream = a.stream();
  return quantise(x, s, blocks(s), codes, scales, stream, [&](auto... to) { return g_lib.quant_fp8(to..., 0, stream); });
  END_HANDLE_TH_ERRORS
}

// quant_fp8_pooled(x, block, key side, select workspace, codes, scales, stream) -> rc, codes, scales
PyObject* quant_fp8_pooled(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(7);
  const at::Tensor x = a.tensor();
  const sparkattn_shape_t s = make_shape(x, a.i32());
  const bool key_side = a.truth();
  const at::Tensor ws = a.tensor(), codes = a.optional_tensor(), scales = a.optional_tensor();
  const Stream stream = a.stream();
  return quantise(x, s, blocks(s), codes, scales, stream,
                  [&](auto... to) { return g_lib.quant_fp8_pooled(to..., key_side, ptr(ws), (size_t)ws.numel(), stream); });
  END_HANDLE_TH_ERRORS
}

// quant_fp8_per_token(x, codes, scales, stream) -> rc, codes, scales
PyObject* quant_fp8_per_token(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(4);
  const at::Tensor x = a.tensor();
  const sparkattn_shape_t s = make_shape(x, x.size(-1) == 64 ? 64 : 128);
  const at::Tensor codes = a.optional_tensor(), scales = a.optional_tensor();
  const Stream stream = a.stream();
  return quantise(x, s, s.N, codes, scales, stream, [&](auto... to) { return g_lib.quant_fp8_per_token(to..., stream); });
  END_HANDLE_TH_ERRORS
}

// fwd(q, k, v, kept_idx, kept_cnt, block, dtype, q_scale, k_scale, v_scale, softmax_scale, out, return_lse, workspace, stream,
// frame_tokens, window, block_valid) -> rc, out, lse, workspace
PyObject* fwd(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(18);
  const at::Tensor q = a.tensor(), k = a.tensor(), v = a.tensor(), idx = a.tensor(), cnt = a.optional_tensor();
  const int32_t block = a.i32(), dtype = a.i32();
  const at::Tensor sq = a.optional_tensor(), sk = a.optional_tensor(), sv = a.optional_tensor();
  const float softmax_scale = a.number();
  at::Tensor out = a.optional_tensor(), lse;
  const bool return_lse = a.truth();
  at::Tensor ws = a.optional_tensor();
  const Stream stream = a.stream();
  const int32_t frame_tokens = a.i32(), window = a.i32();
  const at::Tensor valid = a.optional_tensor();
  same_layout(q, k);
  same_layout(q, v);
  const sparkattn_shape_t s = make_shape(q, block, softmax_scale);
  const int32_t kmax = (int32_t)idx.size(-1);
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (!out.defined()) out = stream.output_like(q, at::kBFloat16);
    if (return_lse) lse = stream.output({s.B, s.H, s.N}, at::kFloat, q);
    ws = workspace_for(ws, s, 1, kmax, q, stream);
    const size_t bytes = ws.defined() ? (size_t)ws.numel() : 0;
    if (!ws.defined()) rc = kNoWorkspace;
    else if (valid.defined())
      rc = g_lib.fwd_padded(&s, dtype, ptr(q), ptr(k), ptr(v), fptr(sq), fptr(sk), fptr(sv), iptr(idx), iptr(cnt), kmax, iptr(valid),
                            ptr(out), fptr(lse), ptr(ws), bytes, stream);
    else if (frame_tokens > 0)
      rc = g_lib.fwd_window(&s, dtype, ptr(q), ptr(k), ptr(v), fptr(sq), fptr(sk), fptr(sv), iptr(idx), iptr(cnt), kmax, frame_tokens,
                            window, ptr(out), fptr(lse), ptr(ws), bytes, stream);
    else
      rc = g_lib.fwd(&s, dtype, ptr(q), ptr(k), ptr(v), fptr(sq), fptr(sk), fptr(sv), iptr(idx), iptr(cnt), kmax, ptr(out), fptr(lse),
                     ptr(ws), bytes, stream);
  }
  return result(rc, {out, lse, ws});
  END_HANDLE_TH_ERRORS
}

// gather_tokens(x, index, out, workspace, stream) -> rc, out, workspace
PyObject* gather_tokens(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(5);
  const at::Tensor x = a.tensor(), index = a.tensor();
  at::Tensor out = a.optional_tensor(), ws = a.optional_tensor();
  const Stream stream = a.stream();
  const int32_t block = x.size(-1) == 64 ? 64 : 128;
  TORCH_CHECK_VALUE(index.scalar_type() == at::kInt && index.dim() == 1 && index.is_contiguous(),
                    "index must be a contiguous 1-D int32 tensor");
  const sparkattn_shape_t src = make_shape(x, block);
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (!out.defined()) out = stream.output({src.B, src.H, index.numel(), src.d}, x.scalar_type(), x);
    const sparkattn_shape_t dst = make_shape(out, block);
    if (!ws.defined()) ws = stream.scratch(256, x);
    rc = g_lib.gather_tokens(&src, ptr(x), &dst, iptr(index), ptr(out), ptr(ws), (size_t)ws.numel(), stream);
  }
  return result(rc, {out, ws});
  END_HANDLE_TH_ERRORS
}

// What the calls of the compensation branch share: the grid and the rotary tables.
struct Rope {
  int32_t grid[3];
  at::Tensor axis, freq;
  explicit Rope(Args& a) {
    for (int32_t& g : grid) g = a.i32();
    axis = a.tensor();
    freq = a.tensor();
    TORCH_CHECK_VALUE(axis.numel() == freq.numel(), "rope axis and frequency tables must have rank/2 entries each");
  }
  // The library reads the tables on the host.  A copy from the device waits for the stream's earlier work, so this is
  // called without the interpreter lock.
  void to_host() {
    axis = axis.detach().to(at::kCPU, at::kInt).contiguous();
    freq = freq.detach().to(at::kCPU, at::kFloat).contiguous();
  }
};
bool is_contiguous(const at::Tensor& t, at::IntArrayRef sizes) { return t.is_contiguous() && t.sizes() == sizes; }
int32_t check_projection(const at::Tensor& p, const sparkattn_shape_t& s, const char* what) {
  TORCH_CHECK_VALUE(p.dim() == 3 && is_contiguous(p, {s.H, p.size(1), s.d}), what, " must be contiguous [H, rank, d]");
  return (int32_t)p.size(1);
}
void check_gate_operands(const at::Tensor& state, const at::Tensor& gate, const sparkattn_shape_t& s, int32_t rank) {
  TORCH_CHECK_VALUE(is_contiguous(state, {s.B, s.H, rank, s.d}) && state.scalar_type() == at::kFloat,
                    "state must be contiguous fp32 [B, H, rank, d]");
  TORCH_CHECK_VALUE(is_contiguous(gate, {s.B, s.H, s.N}) && gate.scalar_type() == at::kFloat, "gate must be contiguous fp32 [B, H, N]");
}
int64_t at_least_256(size_t bytes) { return (int64_t)std::max(bytes, (size_t)256); }

// comp_state(k, v, pk, T, Hg, Wg, axis, freq, state, workspace, stream) -> rc, state, workspace
PyObject* comp_state(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(11);
  const at::Tensor k = a.tensor(), v = a.tensor(), pk = a.tensor();
  same_layout(k, v);
  const sparkattn_shape_t s = make_shape(k, 128);
  Rope rope(a);
  const int32_t rank = check_projection(pk, s, "pk");
  at::Tensor state = a.optional_tensor(), ws = a.optional_tensor();
  const Stream stream = a.stream();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    rope.to_host();
    if (!state.defined()) state = stream.output({s.B, s.H, rank, s.d}, at::kFloat, k);
    if (!ws.defined()) ws = stream.scratch(at_least_256(g_lib.comp_workspace_bytes(&s, rope.grid)), k);
    rc = g_lib.comp_state(&s, ptr(k), ptr(v), ptr(pk), rank, rope.grid, iptr(rope.axis), fptr(rope.freq), fptr(state), ptr(ws),
                          (size_t)ws.numel(), stream);
  }
  return result(rc, {state, ws});
  END_HANDLE_TH_ERRORS
}

// comp_apply(q, pq, state, gate, o_sparse, T, Hg, Wg, axis, freq, eps, out, workspace, stream) -> rc, out, workspace
PyObject* comp_apply(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(14);
  const at::Tensor q = a.tensor(), pq = a.tensor(), state = a.tensor(), gate = a.tensor(), o_sparse = a.tensor();
  same_layout(q, o_sparse);
  const sparkattn_shape_t s = make_shape(q, 128);
  Rope rope(a);
  const int32_t rank = check_projection(pq, s, "pq");
  check_gate_operands(state, gate, s, rank);
  const float eps = a.number();
  at::Tensor out = a.optional_tensor(), ws = a.optional_tensor();
  const Stream stream = a.stream();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    rope.to_host();
    if (!out.defined()) out = stream.output_like(q, at::kBFloat16);
    if (!ws.defined()) ws = stream.scratch(at_least_256(g_lib.comp_workspace_bytes(&s, rope.grid)), q);
    rc = g_lib.comp_apply(&s, ptr(q), ptr(pq), rank, rope.grid, iptr(rope.axis), fptr(rope.freq), fptr(state), fptr(gate),
                          ptr(o_sparse), ptr(out), eps, ptr(ws), (size_t)ws.numel(), stream);
  }
  return result(rc, {out, ws});
  END_HANDLE_TH_ERRORS
}

// fwd_gated(q, k, v, kept_idx, kept_cnt, pq, state, gate, T, Hg, Wg, axis, freq, eps, softmax_scale, out, return_lse, workspace,
// stream) -> rc, out, lse, workspace
PyObject* fwd_gated(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(19);
  const at::Tensor q = a.tensor(), k = a.tensor(), v = a.tensor(), idx = a.tensor(), cnt = a.optional_tensor(), pq = a.tensor(),
                   state = a.tensor(), gate = a.tensor();
  same_layout(q, k);
  same_layout(q, v);
  Rope rope(a);
  const float eps = a.number(), softmax_scale = a.number();
  const sparkattn_shape_t s = make_shape(q, 128, softmax_scale);
  const int32_t rank = check_projection(pq, s, "pq"), kmax = (int32_t)idx.size(-1);
  check_gate_operands(state, gate, s, rank);
  at::Tensor out = a.optional_tensor(), lse;
  const bool return_lse = a.truth();
  at::Tensor ws = a.optional_tensor();
  const Stream stream = a.stream();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    rope.to_host();
    if (!out.defined()) out = stream.output_like(q, at::kBFloat16);
    if (return_lse) lse = stream.output({s.B, s.H, s.N}, at::kFloat, q);
    if (!ws.defined()) ws = stream.scratch(at_least_256(g_lib.fwd_gated_workspace_bytes(&s, kmax, rope.grid)), q);
    rc = g_lib.fwd_gated(&s, ptr(q), ptr(k), ptr(v), iptr(idx), iptr(cnt), kmax, ptr(pq), rank, rope.grid, iptr(rope.axis),
                         fptr(rope.freq), fptr(state), fptr(gate), eps, ptr(out), fptr(lse), ptr(ws), (size_t)ws.numel(), stream);
  }
  return result(rc, {out, lse, ws});
  END_HANDLE_TH_ERRORS
}

// The paged cache: pools, scales and the batch, as both calls take them.
struct Cache {
  at::Tensor k, v, k_scale, v_scale, table, len, start;
  sparkattn_cache_t c{};
  sparkattn_batch_t b{};
  explicit Cache(Args& a) {
    k = a.tensor();
    v = a.tensor();
    k_scale = a.optional_tensor();
    v_scale = a.optional_tensor();
    table = a.tensor();
    len = a.tensor();
    start = a.optional_tensor();
    b.max_new = a.i32();
  }
  // `rows`: a [T, heads, d] tensor of the call
  void describe(const at::Tensor& rows) {
    TORCH_CHECK_VALUE(k.dim() == 4 && k.stride(3) == 1, "expected pools [pages, H, page, d] with a contiguous last dimension");
    same_layout(k, v);
    const at::ScalarType type = k.scalar_type();
    const bool codes = type == at::kByte || type == at::kFloat8_e4m3fn;
    TORCH_CHECK_VALUE((codes || type == at::kBFloat16) && v.scalar_type() == type, "pools are bfloat16, float8_e4m3fn or uint8 (E4M3 codes)");
    TORCH_CHECK_VALUE(codes == k_scale.defined() && codes == v_scale.defined(), "E4M3 pools have scales, bf16 pools have none");
    for (const at::Tensor* x : std::initializer_list<const at::Tensor*>{&k_scale, &v_scale})
      TORCH_CHECK_VALUE(!x->defined() || (x->scalar_type() == at::kFloat && x->dim() == 2 && x->is_contiguous() && x->size(0) == k.size(0) && x->size(1) == k.size(1)),
                        "scales are contiguous float32 [pages, H]");
    TORCH_CHECK_VALUE(table.scalar_type() == at::kInt && table.dim() == 2 && table.is_contiguous(), "page_table is a contiguous int32 [B, max_pages]");
    TORCH_CHECK_VALUE(len.scalar_type() == at::kInt && len.is_contiguous() && len.dim() == 1 && len.size(0) == table.size(0), "kv_len is a contiguous int32 [B]");
    TORCH_CHECK_VALUE(!start.defined() || (start.scalar_type() == at::kInt && start.is_contiguous() && start.dim() == 1 && start.size(0) == table.size(0) + 1),
                      "q_start is a contiguous int32 [B + 1]");
    for (const at::Tensor* x : std::initializer_list<const at::Tensor*>{&v, &k_scale, &v_scale, &table, &len, &start, &rows})
      TORCH_CHECK_VALUE(!x->defined() || x->device() == k.device(), "tensors of one call must be on one device");
    c.struct_size = sizeof(c);
    c.version = SPARKATTN_VERSION;
    c.dtype = codes ? SPARKATTN_FP8_E4M3 : SPARKATTN_BF16;
    c.pages = (int32_t)k.size(0); c.H = (int32_t)k.size(1); c.page = (int32_t)k.size(2); c.d = (int32_t)k.size(3);
    c.stride_page = k.stride(0); c.stride_h = k.stride(1); c.stride_n = k.stride(2);
    b.struct_size = sizeof(b);
    b.version = SPARKATTN_VERSION;
    b.B = (int32_t)table.size(0);
    b.T = (int32_t)rows.size(0);
    if (b.max_new == 0) b.max_new = start.defined() || b.B == 0 ? b.T : b.T / b.B;
    b.max_pages = (int32_t)table.size(1);
    b.page_table = iptr(table); b.kv_len = iptr(len); b.q_start = iptr(start);
  }
  void check_device() const { TORCH_CHECK_VALUE(k.is_cuda(), "tensors of a call must be on a CUDA device"); }
  void check_workspace(const at::Tensor& ws) const { TORCH_CHECK_VALUE(ws.device() == k.device() && ws.is_contiguous() && ws.element_size() == 1, "the workspace is contiguous bytes on the call's device"); }
  // a [T, heads, d] tensor of the call as the library takes it; heads 0: any number
  sparkattn_rows_t rows(const at::Tensor& x, int64_t heads) const {
    TORCH_CHECK_VALUE(x.dim() == 3 && x.stride(2) == 1 && x.scalar_type() == at::kBFloat16 && x.size(0) == b.T && x.size(2) == c.d &&
                          (heads == 0 || x.size(1) == heads) && x.device() == k.device(),
                      "expected bfloat16 rows [T, heads, d] of the call's T and d with a contiguous last dimension");
    return {x.data_ptr(), x.stride(0), x.stride(1)};
  }
};

// cache_append(k_cache, v_cache, k_scale, v_scale, page_table, kv_len, q_start, max_new, k, v, q, q_out, cos, sin, positions, axis,
// interleaved, workspace, stream) -> rc, q_out, workspace
PyObject* cache_append(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(19);
  Cache cache(a);
  const at::Tensor k = a.tensor(), v = a.tensor(), q = a.optional_tensor();
  at::Tensor q_out = a.optional_tensor();
  const at::Tensor cos = a.optional_tensor(), sin = a.optional_tensor(), positions = a.optional_tensor(), axis = a.optional_tensor();
  const bool interleaved = a.truth();
  at::Tensor ws = a.optional_tensor();
  const Stream stream = a.stream();
  cache.describe(k);
  const sparkattn_rows_t rk = cache.rows(k, cache.c.H), rv = cache.rows(v, cache.c.H);
  sparkattn_rotary_t rotary{};
  if (cos.defined()) {
    TORCH_CHECK_VALUE(sin.defined() && cos.dim() == 2 && cos.scalar_type() == at::kFloat && sin.scalar_type() == at::kFloat && cos.is_contiguous() &&
                          sin.is_contiguous() && cos.sizes() == sin.sizes() && cos.device() == k.device() && sin.device() == k.device(),
                      "rotary tables are contiguous float32 [rows, rot / 2] on the call's device");
    TORCH_CHECK_VALUE(!positions.defined() || (positions.scalar_type() == at::kInt && positions.is_contiguous() && positions.device() == k.device() &&
                                               (positions.dim() == 1 || positions.dim() == 2) && positions.size(0) == k.size(0)),
                      "positions are contiguous int32 [T] or [T, axes] on the call's device");
    TORCH_CHECK_VALUE(!axis.defined() || (axis.scalar_type() == at::kInt && axis.is_contiguous() && axis.dim() == 1 && axis.size(0) == cos.size(1) &&
                                          axis.device() == k.device()),
                      "axis is a contiguous int32 [rot / 2] on the call's device");
    TORCH_CHECK_VALUE(axis.defined() || !positions.defined() || positions.dim() == 1 || positions.size(1) == 1, "positions over several axes need axis");
    rotary.struct_size = sizeof(rotary);
    rotary.version = SPARKATTN_VERSION;
    rotary.rot = (int32_t)(2 * cos.size(1));
    rotary.interleaved = interleaved;
    rotary.rows = (int32_t)cos.size(0);
    rotary.axes = positions.defined() && positions.dim() == 2 ? (int32_t)positions.size(1) : 1;
    rotary.cos = fptr(cos); rotary.sin = fptr(sin);
    rotary.positions = iptr(positions); rotary.axis = iptr(axis);
  }
  cache.check_device();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (q.defined() && !q_out.defined()) q_out = stream.output(q.sizes(), at::kBFloat16, q);
    if (!ws.defined()) ws = stream.scratch(256, k);
    cache.check_workspace(ws);
    sparkattn_rows_t rq{}, ro{};
    if (q.defined()) {
      rq = cache.rows(q, 0);
      ro = cache.rows(q_out, q.size(1));
    }
    rc = g_lib.cache_append(&cache.c, &cache.b, cos.defined() ? &rotary : nullptr, q.defined() ? &rq : nullptr, q.defined() ? (int32_t)q.size(1) : 0, &rk, &rv,
                            ptr(cache.k), ptr(cache.v), fptr(cache.k_scale), fptr(cache.v_scale), q.defined() ? &ro : nullptr, ptr(ws),
                            (size_t)ws.numel(), stream);
  }
  return result(rc, {q_out, ws});
  END_HANDLE_TH_ERRORS
}

// cache_fwd(k_cache, v_cache, k_scale, v_scale, page_table, kv_len, q_start, max_new, q, frame_tokens, window, softmax_scale, out, return_lse,
// workspace, stream) -> rc, out, lse, workspace
PyObject* cache_fwd(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(16);
  Cache cache(a);
  const at::Tensor q = a.tensor();
  const int32_t frame_tokens = a.i32(), window = a.i32();
  const float softmax_scale = a.number();
  at::Tensor out = a.optional_tensor(), lse;
  const bool return_lse = a.truth();
  at::Tensor ws = a.optional_tensor();
  const Stream stream = a.stream();
  cache.describe(q);
  const sparkattn_rows_t rq = cache.rows(q, 0);
  const int32_t H = (int32_t)q.size(1);
  cache.check_device();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (!out.defined()) out = stream.output(q.sizes(), at::kBFloat16, q);
    const sparkattn_rows_t ro = cache.rows(out, H);
    if (return_lse) lse = stream.output({q.size(0), q.size(1)}, at::kFloat, q);
    if (!ws.defined()) {
      const size_t bytes = g_lib.cache_workspace_bytes(&cache.c, &cache.b, H);
      ws = stream.scratch((int64_t)(bytes < 256 ? 256 : bytes), q);      // an unsupported call says why itself
    }
    cache.check_workspace(ws);
    rc = g_lib.cache_fwd(&cache.c, &cache.b, &rq, H, ptr(cache.k), ptr(cache.v), fptr(cache.k_scale), fptr(cache.v_scale), frame_tokens, window,
                         softmax_scale, &ro, fptr(lse), ptr(ws), (size_t)ws.numel(), stream);
  }
  return result(rc, {out, lse, ws});
  END_HANDLE_TH_ERRORS
}

// bind(address of each entry point, in the order of Library)
PyObject* bind(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  constexpr Py_ssize_t kEntries = sizeof(Library) / sizeof(void*);
  a.expect(kEntries);
  void* entry[kEntries];
  for (void*& e : entry) e = reinterpret_cast<void*>((intptr_t)a.integer());
  static_assert(sizeof(entry) == sizeof(Library), "one address per entry point");
  memcpy(&g_lib, entry, sizeof(entry));
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) { return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr}; }
PyMethodDef g_methods[] = {method<bind>("bind"), method<select>("select"), method<select_pooled>("select_pooled"),
                           method<quant_fp8>("quant_fp8"), method<quant_fp8_pooled>("quant_fp8_pooled"),
                           method<quant_fp8_per_token>("quant_fp8_per_token"), method<fwd>("fwd"), method<gather_tokens>("gather_tokens"),
                           method<comp_state>("comp_state"), method<comp_apply>("comp_apply"), method<fwd_gated>("fwd_gated"),
                           method<cache_append>("cache_append"), method<cache_fwd>("cache_fwd"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_sparkattn", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sparkattn(void) { return PyModule_Create(&g_module); }
