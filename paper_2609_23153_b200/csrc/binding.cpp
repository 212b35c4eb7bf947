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
  decltype(&sparkattn_cache_fwd_sink) cache_fwd_sink;
  decltype(&sparkattn_cache_append_norm) cache_append_norm;
  decltype(&sparkattn_norm_rotate) norm_rotate;
  decltype(&sparkattn_pages_workspace_bytes) pages_workspace_bytes;
  decltype(&sparkattn_pages_fork) pages_fork;
  decltype(&sparkattn_pages_reserve) pages_reserve;
  decltype(&sparkattn_pages_trim) pages_trim;
  decltype(&sparkattn_pages_compact) pages_compact;
  decltype(&sparkattn_cache_copy_pages) cache_copy_pages;
  decltype(&sparkattn_pages_reserve_len) pages_reserve_len;
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

// The library launches on the current device, in its current stream.
void check_here(const at::Tensor& x) {
  TORCH_CHECK_VALUE(x.is_cuda(), "tensors of a call must be on a CUDA device");
  TORCH_CHECK_VALUE(x.device().index() == c10::cuda::current_device(), "tensors of a call must be on the current CUDA device");
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

// The pools of a paged cache.
struct Pools {
  at::Tensor k, v, k_scale, v_scale;
  explicit Pools(Args& a) {
    k = a.tensor();
    v = a.tensor();
    k_scale = a.optional_tensor();
    v_scale = a.optional_tensor();
  }
  void describe(sparkattn_cache_t& c) const {
    TORCH_CHECK_VALUE(k.dim() == 4 && k.stride(3) == 1, "expected pools [pages, H, page, d] with a contiguous last dimension");
    same_layout(k, v);
    const at::ScalarType type = k.scalar_type();
    const bool codes = type == at::kByte || type == at::kFloat8_e4m3fn;
    TORCH_CHECK_VALUE((codes || type == at::kBFloat16) && v.scalar_type() == type, "pools are bfloat16, float8_e4m3fn or uint8 (E4M3 codes)");
    TORCH_CHECK_VALUE(codes == k_scale.defined() && codes == v_scale.defined(), "E4M3 pools have scales, bf16 pools have none");
    for (const at::Tensor* x : std::initializer_list<const at::Tensor*>{&k_scale, &v_scale})
      TORCH_CHECK_VALUE(!x->defined() || (x->scalar_type() == at::kFloat && x->dim() == 2 && x->is_contiguous() && x->size(0) == k.size(0) && x->size(1) == k.size(1)),
                        "scales are contiguous float32 [pages, H]");
    for (const at::Tensor* x : std::initializer_list<const at::Tensor*>{&v, &k_scale, &v_scale})
      TORCH_CHECK_VALUE(!x->defined() || x->device() == k.device(), "tensors of one call must be on one device");
    c.struct_size = sizeof(c);
    c.version = SPARKATTN_VERSION;
    c.dtype = codes ? SPARKATTN_FP8_E4M3 : SPARKATTN_BF16;
    c.pages = (int32_t)k.size(0); c.H = (int32_t)k.size(1); c.page = (int32_t)k.size(2); c.d = (int32_t)k.size(3);
    c.stride_page = k.stride(0); c.stride_h = k.stride(1); c.stride_n = k.stride(2);
  }
};

// The paged cache: pools, scales and the batch, as both calls take them.
struct Cache : Pools {
  at::Tensor table, len, start;
  sparkattn_cache_t c{};
  sparkattn_batch_t b{};
  explicit Cache(Args& a) : Pools(a) {
    table = a.tensor();
    len = a.tensor();
    start = a.optional_tensor();
    b.max_new = a.i32();
  }
  // `rows`: a [T, heads, d] tensor of the call
  void describe(const at::Tensor& rows) {
    Pools::describe(c);
    TORCH_CHECK_VALUE(table.scalar_type() == at::kInt && table.dim() == 2 && table.is_contiguous(), "page_table is a contiguous int32 [B, max_pages]");
    TORCH_CHECK_VALUE(len.scalar_type() == at::kInt && len.is_contiguous() && len.dim() == 1 && len.size(0) == table.size(0), "kv_len is a contiguous int32 [B]");
    TORCH_CHECK_VALUE(!start.defined() || (start.scalar_type() == at::kInt && start.is_contiguous() && start.dim() == 1 && start.size(0) == table.size(0) + 1),
                      "q_start is a contiguous int32 [B + 1]");
    for (const at::Tensor* x : std::initializer_list<const at::Tensor*>{&table, &len, &start, &rows})
      TORCH_CHECK_VALUE(!x->defined() || x->device() == k.device(), "tensors of one call must be on one device");
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

// The rotation and the norm of queries and keys, as the calls that take them do.
struct Rotation {
  at::Tensor cos, sin, positions, axis;
  sparkattn_rotary_t r{};
  explicit Rotation(Args& a) {
    cos = a.optional_tensor();
    sin = a.optional_tensor();
    positions = a.optional_tensor();
    axis = a.optional_tensor();
    r.interleaved = a.truth();
  }
  // for `tokens` tokens; NULL where nothing is rotated
  const sparkattn_rotary_t* describe(int64_t tokens, const at::Device& device) {
    if (!cos.defined()) return nullptr;
    TORCH_CHECK_VALUE(sin.defined() && cos.dim() == 2 && cos.scalar_type() == at::kFloat && sin.scalar_type() == at::kFloat && cos.is_contiguous() &&
                          sin.is_contiguous() && cos.sizes() == sin.sizes() && cos.device() == device && sin.device() == device,
                      "rotary tables are contiguous float32 [rows, rot / 2] on the call's device");
    TORCH_CHECK_VALUE(!positions.defined() || (positions.scalar_type() == at::kInt && positions.is_contiguous() && positions.device() == device &&
                                               (positions.dim() == 1 || positions.dim() == 2) && positions.size(0) == tokens),
                      "positions are contiguous int32 [T] or [T, axes] on the call's device");
    TORCH_CHECK_VALUE(!axis.defined() || (axis.scalar_type() == at::kInt && axis.is_contiguous() && axis.dim() == 1 && axis.size(0) == cos.size(1) &&
                                          axis.device() == device),
                      "axis is a contiguous int32 [rot / 2] on the call's device");
    TORCH_CHECK_VALUE(axis.defined() || !positions.defined() || positions.dim() == 1 || positions.size(1) == 1, "positions over several axes need axis");
    r.struct_size = sizeof(r);
    r.version = SPARKATTN_VERSION;
    r.rot = (int32_t)(2 * cos.size(1));
    r.rows = (int32_t)cos.size(0);
    r.axes = positions.defined() && positions.dim() == 2 ? (int32_t)positions.size(1) : 1;
    r.cos = fptr(cos); r.sin = fptr(sin);
    r.positions = iptr(positions); r.axis = iptr(axis);
    return &r;
  }
};
struct HeadNorm {
  at::Tensor q, k;
  bool on = false;
  sparkattn_norm_t n{};
  void take(Args& a) {
    on = a.truth();
    q = a.optional_tensor();
    k = a.optional_tensor();
    n.eps = a.number();
  }
  // heads -1: the call has no such tensor
  const sparkattn_norm_t* describe(int64_t q_heads, int64_t k_heads, int64_t d, const at::Device& device) {
    if (!on) return nullptr;
    n.struct_size = sizeof(n);
    n.version = SPARKATTN_VERSION;
    const at::Tensor& any = q.defined() ? q : k;
    n.weight_dtype = any.defined() && any.scalar_type() == at::kBFloat16 ? SPARKATTN_BF16 : SPARKATTN_FP32;
    n.per_head = any.defined() && any.dim() == 2;
    auto check = [&](const at::Tensor& w, int64_t heads) {
      TORCH_CHECK_VALUE(!w.defined() || ((w.scalar_type() == at::kFloat || w.scalar_type() == at::kBFloat16) && w.scalar_type() == any.scalar_type() &&
                                         w.is_contiguous() && w.dim() == any.dim() && (w.dim() == 1 || (w.dim() == 2 && (heads < 0 || w.size(0) == heads))) &&
                                         w.size(-1) == d && w.device() == device),
                        "norm weights are contiguous float32 or bfloat16 [d] or [heads, d], both alike, on the call's device");
    };
    check(q, q_heads);
    check(k, k_heads);
    n.q_weight = ptr(q); n.k_weight = ptr(k);
    return &n;
  }
};

// cache_append(k_cache, v_cache, k_scale, v_scale, page_table, kv_len, q_start, max_new, k, v, q, q_out, cos, sin, positions, axis,
// interleaved, workspace, stream) -> rc, q_out, workspace; cache_append_norm has norm, q_weight, k_weight, eps behind interleaved
template <bool NORM>
PyObject* cache_append(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(NORM ? 23 : 19);
  Cache cache(a);
  const at::Tensor k = a.tensor(), v = a.tensor(), q = a.optional_tensor();
  at::Tensor q_out = a.optional_tensor();
  Rotation rotation(a);
  HeadNorm norm;
  if constexpr (NORM) norm.take(a);
  at::Tensor ws = a.optional_tensor();
  const Stream stream = a.stream();
  cache.describe(k);
  const sparkattn_rows_t rk = cache.rows(k, cache.c.H), rv = cache.rows(v, cache.c.H);
  const sparkattn_rotary_t* rotary = rotation.describe(k.size(0), k.device());
  const sparkattn_norm_t* normed = norm.describe(q.defined() && q.dim() == 3 ? q.size(1) : -1, cache.c.H, cache.c.d, k.device());
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
    rc = g_lib.cache_append_norm(&cache.c, &cache.b, normed, rotary, q.defined() ? &rq : nullptr, q.defined() ? (int32_t)q.size(1) : 0, &rk, &rv,
                                 ptr(cache.k), ptr(cache.v), fptr(cache.k_scale), fptr(cache.v_scale), q.defined() ? &ro : nullptr, ptr(ws),
                                 (size_t)ws.numel(), stream);
  }
  return result(rc, {q_out, ws});
  END_HANDLE_TH_ERRORS
}

// norm_rotate(q, k, q_out, k_out, cos, sin, positions, axis, interleaved, norm, q_weight, k_weight, eps, workspace, stream)
// -> rc, q_out, k_out, workspace
PyObject* norm_rotate(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(15);
  const at::Tensor q = a.tensor(), k = a.optional_tensor();
  at::Tensor q_out = a.optional_tensor(), k_out = a.optional_tensor();
  Rotation rotation(a);
  HeadNorm norm;
  norm.take(a);
  at::Tensor ws = a.optional_tensor();
  const Stream stream = a.stream();
  const int32_t block = q.dim() == 4 && q.size(3) == 64 ? 64 : 128;
  const sparkattn_shape_t qs = make_shape(q, block);
  sparkattn_shape_t ks{};
  if (k.defined()) ks = make_shape(k, block);
  TORCH_CHECK_VALUE(k.defined() || !k_out.defined(), "k_out without k");
  const sparkattn_rotary_t* rotary = rotation.describe(qs.N, q.device());
  const sparkattn_norm_t* normed = norm.describe(qs.H, k.defined() ? ks.H : -1, qs.d, q.device());
  for (const at::Tensor* x : std::initializer_list<const at::Tensor*>{&q, &k, &q_out, &k_out})
    TORCH_CHECK_VALUE(!x->defined() || (x->scalar_type() == at::kBFloat16 && x->device() == q.device()), "expected bfloat16 tensors on one device");
  check_here(q);
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (!q_out.defined()) q_out = stream.output_like(q, at::kBFloat16);
    if (k.defined() && !k_out.defined()) k_out = stream.output_like(k, at::kBFloat16);
    if (!ws.defined()) ws = stream.scratch(256, q);
    TORCH_CHECK_VALUE(ws.device() == q.device() && ws.is_contiguous() && ws.element_size() == 1, "the workspace is contiguous bytes on the call's device");
    const sparkattn_shape_t qo = make_shape(q_out, block);
    sparkattn_shape_t ko{};
    if (k.defined()) ko = make_shape(k_out, block);
    rc = g_lib.norm_rotate(&qs, ptr(q), &qo, ptr(q_out), k.defined() ? &ks : nullptr, ptr(k), k.defined() ? &ko : nullptr, ptr(k_out), normed, rotary, ptr(ws),
                           (size_t)ws.numel(), stream);
  }
  return result(rc, {q_out, k_out, ws});
  END_HANDLE_TH_ERRORS
}

// cache_fwd(k_cache, v_cache, k_scale, v_scale, page_table, kv_len, q_start, max_new, q, frame_tokens, window, softmax_scale, out, return_lse,
// workspace, stream) -> rc, out, lse, workspace; cache_fwd_sink has sink behind window
template <bool SINK>
PyObject* cache_fwd(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(SINK ? 17 : 16);
  Cache cache(a);
  const at::Tensor q = a.tensor();
  const int32_t frame_tokens = a.i32(), window = a.i32(), sink = SINK ? a.i32() : 0;
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
    rc = g_lib.cache_fwd_sink(&cache.c, &cache.b, &rq, H, ptr(cache.k), ptr(cache.v), fptr(cache.k_scale), fptr(cache.v_scale), frame_tokens, window,
                              sink, softmax_scale, &ro, fptr(lse), ptr(ws), (size_t)ws.numel(), stream);
  }
  return result(rc, {out, lse, ws});
  END_HANDLE_TH_ERRORS
}

// The book of a pool of pages, as its calls take it.
struct Book {
  at::Tensor table, len, refs, table_out, refs_out, ws;
  sparkattn_book_t b{};
  bool needs_len;
  explicit Book(Args& a, bool len_too) : needs_len(len_too) {
    table = a.tensor();
    if (len_too) len = a.tensor();
    refs = a.tensor();
  }
  // int32 words [n] of the call
  void words(const at::Tensor& x, int64_t n, const char* what) const {
    TORCH_CHECK_VALUE(x.scalar_type() == at::kInt && x.dim() == 1 && x.is_contiguous() && x.size(0) == n && x.device() == table.device(), what);
  }
  void describe(int32_t page) {
    TORCH_CHECK_VALUE(table.scalar_type() == at::kInt && table.dim() == 2 && table.is_contiguous(), "page_table is a contiguous int32 [B, max_pages]");
    TORCH_CHECK_VALUE(refs.scalar_type() == at::kInt && refs.dim() == 1 && refs.is_contiguous() && refs.device() == table.device(),
                      "refs is a contiguous int32 [pages] on the table's device");
    if (needs_len) words(len, table.size(0), "kv_len is a contiguous int32 [B] on the table's device");
    b.struct_size = sizeof(b);
    b.version = SPARKATTN_VERSION;
    b.B = (int32_t)table.size(0); b.max_pages = (int32_t)table.size(1); b.pages = (int32_t)refs.size(0); b.page = page;
    b.page_table = iptr(table); b.refs = iptr(refs);
  }
  void check_device() const { check_here(table); }
  void outputs(at::Tensor given_table, at::Tensor given_refs, at::Tensor given_ws, int64_t rows, const Stream& stream) {
    table_out = given_table.defined() ? given_table : stream.output({rows, table.size(1)}, at::kInt, table);
    refs_out = given_refs.defined() ? given_refs : stream.output({refs.size(0)}, at::kInt, refs);
    TORCH_CHECK_VALUE(table_out.scalar_type() == at::kInt && table_out.dim() == 2 && table_out.is_contiguous() && table_out.size(0) == rows &&
                          table_out.size(1) == table.size(1) && table_out.device() == table.device(), "the new table is a contiguous int32 [sequences, max_pages]");
    words(refs_out, refs.size(0), "the new refs are a contiguous int32 [pages]");
    if (given_ws.defined()) {
      ws = given_ws;
    } else {
      const size_t bytes = g_lib.pages_workspace_bytes(&b);
      ws = stream.scratch((int64_t)(bytes < 256 ? 256 : bytes), table);      // an unsupported call says why itself
    }
    TORCH_CHECK_VALUE(ws.device() == table.device() && ws.is_contiguous() && ws.element_size() == 1, "the workspace is contiguous bytes on the call's device");
  }
  at::Tensor pairs(at::Tensor given, int64_t n, const Stream& stream) const {
    if (!given.defined()) return stream.output({n}, at::kInt, table);
    words(given, n, "src and dst are contiguous int32 of the call's length");
    return given;
  }
};

// pages_fork(page_table, kv_len, refs, parent, table_out, kv_len_out, refs_out, workspace, stream) -> rc, table, kv_len, refs, workspace
PyObject* pages_fork(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(9);
  Book book(a, true);
  const at::Tensor parent = a.tensor(), table_out = a.optional_tensor();
  at::Tensor len_out = a.optional_tensor();
  const at::Tensor refs_out = a.optional_tensor(), ws = a.optional_tensor();
  const Stream stream = a.stream();
  book.describe(16);      // (the call does not look at tokens)
  TORCH_CHECK_VALUE(parent.dim() == 1, "parent is a contiguous int32 [sequences] on the table's device");
  book.words(parent, parent.size(0), "parent is a contiguous int32 [sequences] on the table's device");
  book.check_device();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    book.outputs(table_out, refs_out, ws, parent.size(0), stream);
    if (!len_out.defined()) len_out = stream.output({parent.size(0)}, at::kInt, parent);
    book.words(len_out, parent.size(0), "the new lengths are a contiguous int32 [sequences]");
    rc = g_lib.pages_fork(&book.b, iptr(book.len), iptr(parent), (int32_t)parent.size(0), iptr(book.table_out), iptr(len_out), iptr(book.refs_out), ptr(book.ws),
                          (size_t)book.ws.numel(), stream);
  }
  return result(rc, {book.table_out, len_out, book.refs_out, book.ws});
  END_HANDLE_TH_ERRORS
}

// pages_reserve(page_table, kv_len, refs, kv_new, page, table_out, refs_out, src, dst, kv_len_out, workspace, stream)
// -> rc, table, refs, src, dst, workspace
PyObject* pages_reserve(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(12);
  Book book(a, true);
  const at::Tensor kv_new = a.tensor();
  const int32_t page = a.i32();
  const at::Tensor table_out = a.optional_tensor(), refs_out = a.optional_tensor();
  at::Tensor src = a.optional_tensor(), dst = a.optional_tensor();
  const at::Tensor len_out = a.optional_tensor(), ws = a.optional_tensor();
  const Stream stream = a.stream();
  book.describe(page);
  book.words(kv_new, book.b.B, "kv_new is a contiguous int32 [B] on the table's device");
  if (len_out.defined()) book.words(len_out, book.b.B, "kv_len_out is a contiguous int32 [B] on the table's device");
  book.check_device();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    book.outputs(table_out, refs_out, ws, book.b.B, stream);
    src = book.pairs(src, book.b.B, stream);
    dst = book.pairs(dst, book.b.B, stream);
    rc = len_out.defined() ? g_lib.pages_reserve_len(&book.b, iptr(book.len), iptr(kv_new), iptr(len_out), iptr(book.table_out), iptr(book.refs_out), iptr(src),
                                                     iptr(dst), ptr(book.ws), (size_t)book.ws.numel(), stream)
                           : g_lib.pages_reserve(&book.b, iptr(book.len), iptr(kv_new), iptr(book.table_out), iptr(book.refs_out), iptr(src), iptr(dst),
                                                 ptr(book.ws), (size_t)book.ws.numel(), stream);
  }
  return result(rc, {book.table_out, book.refs_out, src, dst, book.ws});
  END_HANDLE_TH_ERRORS
}

// pages_trim(page_table, kv_len, refs, page, frame_tokens, window, sink, table_out, refs_out, workspace, stream) -> rc, table, refs, workspace
PyObject* pages_trim(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(11);
  Book book(a, true);
  const int32_t page = a.i32(), frame_tokens = a.i32(), window = a.i32(), sink = a.i32();
  const at::Tensor table_out = a.optional_tensor(), refs_out = a.optional_tensor(), ws = a.optional_tensor();
  const Stream stream = a.stream();
  book.describe(page);
  book.check_device();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    book.outputs(table_out, refs_out, ws, book.b.B, stream);
    rc = g_lib.pages_trim(&book.b, iptr(book.len), frame_tokens, window, sink, iptr(book.table_out), iptr(book.refs_out), ptr(book.ws), (size_t)book.ws.numel(),
                          stream);
  }
  return result(rc, {book.table_out, book.refs_out, book.ws});
  END_HANDLE_TH_ERRORS
}

// pages_compact(page_table, refs, table_out, refs_out, src, dst, workspace, stream) -> rc, table, refs, src, dst, workspace
PyObject* pages_compact(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(8);
  Book book(a, false);
  const at::Tensor table_out = a.optional_tensor(), refs_out = a.optional_tensor();
  at::Tensor src = a.optional_tensor(), dst = a.optional_tensor();
  const at::Tensor ws = a.optional_tensor();
  const Stream stream = a.stream();
  book.describe(16);
  book.check_device();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    book.outputs(table_out, refs_out, ws, book.b.B, stream);
    src = book.pairs(src, book.b.pages / 2, stream);
    dst = book.pairs(dst, book.b.pages / 2, stream);
    rc = g_lib.pages_compact(&book.b, iptr(book.table_out), iptr(book.refs_out), iptr(src), iptr(dst), ptr(book.ws), (size_t)book.ws.numel(), stream);
  }
  return result(rc, {book.table_out, book.refs_out, src, dst, book.ws});
  END_HANDLE_TH_ERRORS
}

// cache_copy_pages(k, v, k_scale, v_scale, k_to, v_to, k_scale_to, v_scale_to, src, dst, workspace, stream) -> rc, workspace
PyObject* cache_copy_pages(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(argv, n);
  a.expect(12);
  Pools from(a), to(a);
  const at::Tensor src = a.tensor(), dst = a.tensor();
  at::Tensor ws = a.optional_tensor();
  const Stream stream = a.stream();
  sparkattn_cache_t c_from{}, c_to{};
  from.describe(c_from);
  to.describe(c_to);
  TORCH_CHECK_VALUE(src.scalar_type() == at::kInt && src.dim() == 1 && src.is_contiguous() && dst.scalar_type() == at::kInt && dst.is_contiguous() &&
                        src.sizes() == dst.sizes(), "src and dst are contiguous int32 of one length");
  for (const at::Tensor* x : std::initializer_list<const at::Tensor*>{&to.k, &src, &dst})
    TORCH_CHECK_VALUE(x->device() == from.k.device(), "tensors of one call must be on one device");
  check_here(from.k);
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    if (!ws.defined()) ws = stream.scratch(256, src);
    TORCH_CHECK_VALUE(ws.device() == src.device() && ws.is_contiguous() && ws.element_size() == 1, "the workspace is contiguous bytes on the call's device");
    rc = g_lib.cache_copy_pages(&c_from, ptr(from.k), ptr(from.v), fptr(from.k_scale), fptr(from.v_scale), &c_to, ptr(to.k), ptr(to.v), fptr(to.k_scale),
                                fptr(to.v_scale), iptr(src), iptr(dst), (int32_t)src.numel(), ptr(ws), (size_t)ws.numel(), stream);
  }
  return result(rc, {ws});
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
                           method<cache_append<false>>("cache_append"), method<cache_append<true>>("cache_append_norm"),
                           method<cache_fwd<false>>("cache_fwd"), method<cache_fwd<true>>("cache_fwd_sink"),
                           method<norm_rotate>("norm_rotate"), method<pages_fork>("pages_fork"), method<pages_reserve>("pages_reserve"),
                           method<pages_trim>("pages_trim"), method<pages_compact>("pages_compact"), method<cache_copy_pages>("cache_copy_pages"),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_sparkattn", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sparkattn(void) { return PyModule_Create(&g_module); }
