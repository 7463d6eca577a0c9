// The layers' autograd nodes in native code (host only): RunLoRAFunction, RunVeRAFunction and RunDoRAFunction of module.py without
// Python in their forward and backward.  Same buffers, same calls into librunlora, same results; what they save is host time.
//
// A training pass of a small layer is bound by its host work: with the Python node, forward + backward of 256 x 768 -> 768
// fp32 take 102-189 us of host time a pass for 75 us of GPU work (forward 30; the backward's body alone 68, because the
// autograd engine runs it on a thread of its own, where every Python object it touches comes over from another core).  With
// this node the host takes 14 us for the forward and at most the GPU's time in all: 194 -> 88 us a pass; 1024 x 4096 -> 4096
// r 64 196 -> 114, 1237 x 2056 -> 5464 197 -> 122.  Likewise VeRA (448 x 768 -> 768 r 128
// 196 -> 109, 623 x 4352 -> 4096 r 64 200 -> 117) and DoRA (765 x 1280 -> 7328 r 64 216 -> 135).
//
// ExpertsNode is the same for RunLoRAExpertsFunction and RunLoRAFp8Function (999 rows of 12 experts 1032 -> 2744 r 8, forward +
// backward: 168 us a pass with the Python node, 86 of them the GPU's).
//
// NormNode, RouteNode, GatherNode and CombineNode are RunRMSNormFunction, RunRouteFunction, RunGatherFunction and RunCombineFunction.
//
// lora(...), vera(...), dora(...), experts(...), norm(...), route(...), gather(...) and combine(...) return None where their node does not apply, and the caller then takes the Python node: tensor subclasses, torch
// function / dispatch modes, functorch transforms and tracing (all of which have to see a Python-level function), devices
// other than the current GPU, and operands that only the Python path's checks describe properly.  Forward-mode gradients are
// refused by either node, saved-tensor hooks apply to both (the same tensors are saved in the same order).
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>

#include "../../include/runlora.h"

namespace {

// entry points of librunlora (already loaded by binding.py, which hands over the addresses) and binding._check
decltype(&runlora_forward) p_forward = nullptr;
decltype(&runlora_backward) p_backward = nullptr;
decltype(&runlora_call_workspace_bytes) p_workspace_bytes = nullptr;
decltype(&runlora_vera_forward) p_vera_forward = nullptr;
decltype(&runlora_vera_backward) p_vera_backward = nullptr;
decltype(&runlora_vera_workspace_bytes) p_vera_workspace_bytes = nullptr;
decltype(&runlora_dora_forward) p_dora_forward = nullptr;
decltype(&runlora_dora_backward) p_dora_backward = nullptr;
decltype(&runlora_dora_workspace_bytes) p_dora_workspace_bytes = nullptr;
decltype(&runlora_experts_forward) p_experts_forward = nullptr;
decltype(&runlora_experts_backward) p_experts_backward = nullptr;
decltype(&runlora_experts_workspace_bytes) p_experts_workspace_bytes = nullptr;
decltype(&runlora_fp8_forward) p_fp8_forward = nullptr;
decltype(&runlora_fp8_values) p_fp8_values = nullptr;
decltype(&runlora_rmsnorm_forward) p_rmsnorm_forward = nullptr;
decltype(&runlora_rmsnorm_backward) p_rmsnorm_backward = nullptr;
decltype(&runlora_rmsnorm_workspace_bytes) p_rmsnorm_workspace_bytes = nullptr;
decltype(&runlora_route_forward) p_route_forward = nullptr;
decltype(&runlora_route_backward) p_route_backward = nullptr;
decltype(&runlora_route_workspace_bytes) p_route_workspace_bytes = nullptr;
decltype(&runlora_gather_forward) p_gather_forward = nullptr;
decltype(&runlora_gather_backward) p_gather_backward = nullptr;
decltype(&runlora_combine_forward) p_combine_forward = nullptr;
decltype(&runlora_combine_backward) p_combine_backward = nullptr;
PyObject* g_check = nullptr;

void check(int rc) {
  if (rc == RL_OK) return;
  pybind11::gil_scoped_acquire gil;
  PyObject* r = PyObject_CallFunction(g_check, "i", rc);  // raises RunLoRAError
  Py_XDECREF(r);
  if (r == nullptr) {
    python_error e;
    e.persist();
    throw std::move(e);
  }
}

int dtype_code(at::ScalarType t) {
  return t == at::kFloat ? RL_F32 : (t == at::kHalf ? RL_F16 : (t == at::kBFloat16 ? RL_BF16 : -1));
}

rl_tensor_t desc(const at::Tensor& t, int code) {
  return rl_tensor_t{t.data_ptr(), t.size(0), t.size(1), t.stride(0), code, nullptr, 0};
}

// a saved operand as the backward gets it back: a saved-tensor hook may have changed its type, layout or device, so that
// what held in the forward is checked again (types and sizes by the library, against the descriptor's own)
rl_tensor_t saved_desc(const at::Tensor& t, const at::Tensor& x) {
  TORCH_CHECK_VALUE(t.dim() == 2 && t.stride(1) == 1, "expected a 2-D tensor with contiguous rows");
  TORCH_CHECK_VALUE(t.device() == x.device(), "a saved tensor came back on another device: ", t.device(), ", not ", x.device());
  return desc(t, dtype_code(t.scalar_type()));
}

// rows as the library takes them (the same test as the Python node's)
at::Tensor rows(const at::Tensor& t, int64_t cols) {
  at::Tensor r = t.reshape({-1, cols});
  if (r.stride(-1) != 1 || r.stride(0) % 8 != 0 || r.stride(0) < cols || reinterpret_cast<uintptr_t>(r.data_ptr()) % 16 != 0)
    r = r.clone(at::MemoryFormat::Contiguous);  // (contiguous() would hand dense rows at an odd address back as they are)
  return r;
}

// scratch of one call, given back to the caching allocator behind it (stream-ordered like every tensor)
at::Tensor scratch(size_t bytes, const at::Tensor& like) {
  return at::empty({(int64_t)(bytes < 256 ? 256 : bytes)}, like.options().dtype(at::kByte));
}

struct LoRANode : public torch::autograd::Function<LoRANode> {
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& W, const at::Tensor& A,
                            const at::Tensor& B, const std::optional<at::Tensor>& bias, double scale, int64_t fwd, int64_t bwd,
                            bool keep_merged, double dropout_p, int64_t dropout_seed, bool keep_t) {
    const int64_t i = W.size(0), o = W.size(1), r = A.size(1);
    const int code = dtype_code(x.scalar_type());
    const at::Tensor x2 = rows(x, i);
    const int64_t n = x2.size(0);
    at::Tensor y = at::empty({n, o}, x.options());
    rl_saved_t saved{};
    at::Tensor T, M;
    const bool bwd_t = bwd == 1 || bwd == 5 || bwd == 6 || bwd == 7, bwd_m = bwd == 4 || bwd == 5 || bwd == 7 || bwd == 8;
    if (fwd == RL_FWD_DEFAULT || (keep_t && (fwd == RL_FWD1 || fwd == RL_FWD3) && bwd_t)) {
      T = at::empty({n, r}, x.options());
      saved.T = T.data_ptr();
      saved.ldt = r;
    }
    if (keep_merged && fwd == RL_FWD2 && bwd_m) {
      M = at::empty({i, o}, x.options());
      saved.M = M.data_ptr();
      saved.ldm = o;
    }
    const int choices = (T.defined() ? RL_CALL_T : 0) | (M.defined() ? RL_CALL_M : 0) | ((float)dropout_p != 0.f ? RL_CALL_DROPOUT : 0);
    const at::Tensor ws = scratch(p_workspace_bytes((int)fwd, -1, n, i, o, r, code, choices), x);
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(x.device().index()).stream();
    opts.workspace = ws.data_ptr();
    opts.workspace_bytes = (size_t)ws.numel();
    opts.scale = (float)scale;
    opts.bias = bias.has_value() ? bias->data_ptr() : nullptr;
    opts.dropout_p = (float)dropout_p;
    opts.dropout_seed = (uint32_t)((uint64_t)dropout_seed & 0xFFFFFFFFu);
    const rl_tensor_t dx = desc(x2, code), dw = desc(W, code), da = desc(A, code), db = desc(B, code);
    rl_tensor_t dy = desc(y, code);
    check(p_forward((int)fwd, &dx, &dw, &da, &db, &dy, &saved, &opts));
    ctx->save_for_backward({x2, W, A, B});
    ctx->saved_data["bwd"] = bwd;
    ctx->saved_data["fwd"] = (int64_t)saved.fwd_variant;
    ctx->saved_data["scale"] = (double)saved.scale;
    ctx->saved_data["thr"] = (int64_t)saved.dropout_thr;
    ctx->saved_data["seed"] = (int64_t)saved.dropout_seed;
    ctx->saved_data["x_shape"] = x.sizes().vec();
    if (T.defined()) ctx->saved_data["T"] = T;
    if (M.defined()) ctx->saved_data["M"] = M;
    std::vector<int64_t> shape = x.sizes().vec();
    shape.back() = o;
    return y.view(shape);
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto vars = ctx->get_saved_variables();
    const at::Tensor &W = vars[1], &A = vars[2], &B = vars[3];
    TORCH_CHECK_VALUE(vars[0].is_cuda(), "the saved input came back on ", vars[0].device());
    const rl_tensor_t dw = saved_desc(W, vars[0]), da = saved_desc(A, vars[0]), db = saved_desc(B, vars[0]);
    const int64_t i = W.size(0), o = W.size(1), r = A.size(1);
    const at::Tensor x2 = rows(vars[0], i);
    const int64_t n = x2.size(0);
    const int code = dtype_code(x2.scalar_type());
    const c10::OptionalDeviceGuard guard(x2.device());
    const at::Tensor dy2 = rows(grads[0], o);
    const int bwd = (int)ctx->saved_data["bwd"].toInt();
    rl_saved_t saved{};
    saved.fwd_variant = (int32_t)ctx->saved_data["fwd"].toInt();
    saved.dtype = code;
    saved.n = n; saved.i = i; saved.o = o; saved.r = r;
    saved.X = x2.data_ptr();
    saved.ldx = x2.stride(0);
    saved.scale = (float)ctx->saved_data["scale"].toDouble();
    saved.dropout_thr = (uint32_t)ctx->saved_data["thr"].toInt();
    saved.dropout_seed = (uint32_t)ctx->saved_data["seed"].toInt();
    at::Tensor T, M;
    auto it = ctx->saved_data.find("T");
    if (it != ctx->saved_data.end()) { T = it->second.toTensor(); saved.T = T.data_ptr(); saved.ldt = T.stride(0); }
    it = ctx->saved_data.find("M");
    if (it != ctx->saved_data.end()) { M = it->second.toTensor(); saved.M = M.data_ptr(); saved.ldm = M.stride(0); }
    at::Tensor dx, dA, dB;
    rl_tensor_t tx{}, ta{}, tb{};
    if (ctx->needs_input_grad(0)) { dx = at::empty({n, i}, x2.options()); tx = desc(dx, code); }
    if (ctx->needs_input_grad(2)) { dA = at::empty_like(A); ta = desc(dA, da.dtype); }
    if (ctx->needs_input_grad(3)) { dB = at::empty_like(B); tb = desc(dB, db.dtype); }
    const int choices = (T.defined() ? RL_CALL_T : 0) | (M.defined() ? RL_CALL_M : 0) | (saved.dropout_thr != 0 ? RL_CALL_DROPOUT : 0) |
                        (dx.defined() ? 0 : RL_CALL_NO_DX) | (dA.defined() ? 0 : RL_CALL_NO_DA) | (dB.defined() ? 0 : RL_CALL_NO_DB);
    const at::Tensor ws = scratch(p_workspace_bytes(-1, bwd, n, i, o, r, code, choices), x2);
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(x2.device().index()).stream();
    opts.workspace = ws.data_ptr();
    opts.workspace_bytes = (size_t)ws.numel();
    const rl_tensor_t ddy = desc(dy2, dtype_code(dy2.scalar_type()));
    check(p_backward(bwd, &ddy, &saved, &dw, &da, &db, dx.defined() ? &tx : nullptr, dA.defined() ? &ta : nullptr,
                     dB.defined() ? &tb : nullptr, &opts));
    if (dx.defined()) dx = dx.view(ctx->saved_data["x_shape"].toIntVector());
    at::Tensor none;
    return {dx, none, dA, dB, none, none, none, none, none, none, none, none};
  }
};

// a saved vector as the backward gets it back
void* saved_vec(const at::Tensor& t, int64_t count, at::ScalarType type, const at::Tensor& x, const char* name) {
  TORCH_CHECK_VALUE(t.device() == x.device(), "a saved tensor came back on another device: ", t.device(), ", not ", x.device());
  TORCH_CHECK_VALUE(t.dim() == 1 && t.numel() == count && t.scalar_type() == type && t.stride(0) == 1, name, " must be a dense vector of ",
                    count, " elements of the activation dtype");
  return t.data_ptr();
}

rl_opts_t options(const at::Tensor& x, const at::Tensor& ws, const std::optional<at::Tensor>& bias = std::nullopt, double scale = 0.0) {
  rl_opts_t o{};
  o.stream = c10::hip::getCurrentHIPStream(x.device().index()).stream();
  o.workspace = ws.data_ptr();
  o.workspace_bytes = (size_t)ws.numel();
  o.scale = (float)scale;
  o.bias = bias.has_value() ? bias->data_ptr() : nullptr;
  return o;
}

void keep_record(torch::autograd::AutogradContext* ctx, const rl_saved_t& saved, int64_t bwd, const at::Tensor& x) {
  ctx->saved_data["bwd"] = bwd;
  ctx->saved_data["fwd"] = (int64_t)saved.fwd_variant;
  ctx->saved_data["scale"] = (double)saved.scale;
  ctx->saved_data["x_shape"] = x.sizes().vec();
}

// the forward's record for the input as autograd hands it back (no dropout, T and M by the caller)
rl_saved_t record(torch::autograd::AutogradContext* ctx, const at::Tensor& x2, int code, int64_t o, int64_t r) {
  rl_saved_t s{};
  s.fwd_variant = (int32_t)ctx->saved_data["fwd"].toInt();
  s.dtype = code;
  s.n = x2.size(0); s.i = x2.size(1); s.o = o; s.r = r;
  s.X = x2.data_ptr();
  s.ldx = x2.stride(0);
  s.scale = (float)ctx->saved_data["scale"].toDouble();
  return s;
}

at::Tensor shaped(const at::Tensor& y, const at::Tensor& x) {
  std::vector<int64_t> shape = x.sizes().vec();
  shape.back() = y.size(1);
  return y.view(shape);
}

struct VeRANode : public torch::autograd::Function<VeRANode> {
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& W, const at::Tensor& A,
                            const at::Tensor& B, const at::Tensor& d, const at::Tensor& b, const std::optional<at::Tensor>& bias, double scale,
                            int64_t fwd, int64_t bwd) {
    const int64_t i = W.size(0), o = W.size(1), r = A.size(1);
    const int code = dtype_code(x.scalar_type());
    const at::Tensor x2 = rows(x, i);
    const int64_t n = x2.size(0);
    at::Tensor y = at::empty({n, o}, x.options()), T;
    rl_saved_t saved{};
    if (fwd == RL_FWD_DEFAULT) {
      T = at::empty({n, r}, x.options());
      saved.T = T.data_ptr();
      saved.ldt = r;
    }
    const at::Tensor ws = scratch(p_vera_workspace_bytes((int)fwd, -1, n, i, o, r, code), x);
    const rl_opts_t opts = options(x, ws, bias, scale);
    const rl_tensor_t dx = desc(x2, code), dw = desc(W, code), da = desc(A, code), db = desc(B, code);
    rl_tensor_t dy = desc(y, code);
    check(p_vera_forward((int)fwd, &dx, &dw, &da, &db, d.data_ptr(), b.data_ptr(), &dy, &saved, &opts));
    ctx->save_for_backward({x2, W, A, B, d, b});
    keep_record(ctx, saved, bwd, x);
    if (T.defined()) ctx->saved_data["T"] = T;
    return shaped(y, x);
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto vars = ctx->get_saved_variables();
    TORCH_CHECK_VALUE(vars[0].is_cuda(), "the saved input came back on ", vars[0].device());
    const rl_tensor_t dw = saved_desc(vars[1], vars[0]), da = saved_desc(vars[2], vars[0]), db = saved_desc(vars[3], vars[0]);
    const int64_t i = dw.rows, o = dw.cols, r = db.rows;
    const at::Tensor x2 = rows(vars[0], i);
    const int64_t n = x2.size(0);
    const int code = dtype_code(x2.scalar_type());
    const c10::OptionalDeviceGuard guard(x2.device());
    const at::Tensor dy2 = rows(grads[0], o);
    void* const d = saved_vec(vars[4], r, dy2.scalar_type(), x2, "d");
    void* const b = saved_vec(vars[5], o, dy2.scalar_type(), x2, "b");
    const int bwd = (int)ctx->saved_data["bwd"].toInt();
    rl_saved_t saved = record(ctx, x2, code, o, r);
    at::Tensor T;
    auto it = ctx->saved_data.find("T");
    if (it != ctx->saved_data.end()) { T = it->second.toTensor(); saved.T = T.data_ptr(); saved.ldt = T.stride(0); }
    at::Tensor dx, dd, dbv;
    rl_tensor_t tx{};
    if (ctx->needs_input_grad(0)) { dx = at::empty({n, i}, x2.options()); tx = desc(dx, code); }
    if (ctx->needs_input_grad(4)) dd = at::empty_like(vars[4]);
    if (ctx->needs_input_grad(5)) dbv = at::empty_like(vars[5]);
    const at::Tensor ws = scratch(p_vera_workspace_bytes(-1, bwd, n, i, o, r, code), x2);
    const rl_opts_t opts = options(x2, ws);
    const rl_tensor_t ddy = desc(dy2, dtype_code(dy2.scalar_type()));
    check(p_vera_backward(bwd, &ddy, &saved, &dw, &da, &db, d, b, dx.defined() ? &tx : nullptr, dd.defined() ? dd.data_ptr() : nullptr,
                          dbv.defined() ? dbv.data_ptr() : nullptr, &opts));
    if (dx.defined()) dx = dx.view(ctx->saved_data["x_shape"].toIntVector());
    at::Tensor none;
    return {dx, none, none, none, dd, dbv, none, none, none, none};
  }
};

struct DoRANode : public torch::autograd::Function<DoRANode> {
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& W, const at::Tensor& A,
                            const at::Tensor& B, const at::Tensor& m, const std::optional<at::Tensor>& bias, double scale, int64_t bwd) {
    const int64_t i = W.size(0), o = W.size(1), r = A.size(1);
    const int code = dtype_code(x.scalar_type());
    const at::Tensor x2 = rows(x, i);
    const int64_t n = x2.size(0);
    at::Tensor y = at::empty({n, o}, x.options());
    const at::Tensor c = at::empty({o}, x.options().dtype(at::kFloat));
    rl_saved_t saved{};
    const at::Tensor ws = scratch(p_dora_workspace_bytes(RL_FWD2, -1, n, i, o, r, code), x);
    const rl_opts_t opts = options(x, ws, bias, scale);
    const rl_tensor_t dx = desc(x2, code), dw = desc(W, code), da = desc(A, code), db = desc(B, code);
    rl_tensor_t dy = desc(y, code);
    check(p_dora_forward(RL_FWD2, &dx, &dw, &da, &db, m.data_ptr(), &dy, &saved, c.data_ptr<float>(), &opts));
    ctx->save_for_backward({x2, W, A, B, m, c, y});  // y is the tensor handed to the caller: no copy is kept
    keep_record(ctx, saved, bwd, x);
    if (bias.has_value()) ctx->saved_data["bias"] = *bias;
    return shaped(y, x);
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto vars = ctx->get_saved_variables();
    TORCH_CHECK_VALUE(vars[0].is_cuda(), "the saved input came back on ", vars[0].device());
    const at::Tensor &A = vars[2], &B = vars[3], &m = vars[4];
    const rl_tensor_t dw = saved_desc(vars[1], vars[0]), da = saved_desc(A, vars[0]), db = saved_desc(B, vars[0]), ty = saved_desc(vars[6], vars[0]);
    const int64_t i = dw.rows, o = dw.cols, r = da.cols;
    const at::Tensor x2 = rows(vars[0], i);
    const int64_t n = x2.size(0);
    const int code = dtype_code(x2.scalar_type());
    const c10::OptionalDeviceGuard guard(x2.device());
    const at::Tensor dy2 = rows(grads[0], o);
    void* const pm = saved_vec(m, db.cols, dy2.scalar_type(), x2, "m");
    const float* const c = static_cast<const float*>(saved_vec(vars[5], db.cols, at::kFloat, x2, "c"));
    const int bwd = (int)ctx->saved_data["bwd"].toInt();
    const rl_saved_t saved = record(ctx, x2, code, o, r);
    at::Tensor dx, dA, dB, dm;
    rl_tensor_t tx{}, ta{}, tb{};
    if (ctx->needs_input_grad(0)) { dx = at::empty({n, i}, x2.options()); tx = desc(dx, code); }
    if (ctx->needs_input_grad(2)) { dA = at::empty_like(A); ta = desc(dA, da.dtype); }
    if (ctx->needs_input_grad(3)) { dB = at::empty_like(B); tb = desc(dB, db.dtype); }
    if (ctx->needs_input_grad(4)) dm = at::empty_like(m);
    std::optional<at::Tensor> bias;
    auto it = ctx->saved_data.find("bias");
    if (it != ctx->saved_data.end()) bias = it->second.toTensor();
    const at::Tensor ws = scratch(p_dora_workspace_bytes(-1, bwd, n, i, o, r, code), x2);
    const rl_opts_t opts = options(x2, ws, bias);
    const rl_tensor_t ddy = desc(dy2, dtype_code(dy2.scalar_type()));
    check(p_dora_backward(bwd, &ddy, &saved, &dw, &da, &db, pm, c, &ty, dx.defined() ? &tx : nullptr, dA.defined() ? &ta : nullptr,
                          dB.defined() ? &tb : nullptr, dm.defined() ? dm.data_ptr() : nullptr, &opts));
    if (dx.defined()) dx = dx.view(ctx->saved_data["x_shape"].toIntVector());
    at::Tensor none;
    return {dx, none, dA, dB, dm, none, none, none};
  }
};

// a stack of matrices (or one): what the forward checked is checked again, as in saved_desc
rl_stack_t stack_desc(const at::Tensor& t, const at::Tensor& x, int code, int64_t cols = -1, const at::Tensor& scales = at::Tensor()) {
  TORCH_CHECK_VALUE((t.dim() == 2 || t.dim() == 3) && t.stride(-1) == 1, "expected a matrix or a stack of matrices with contiguous rows");
  TORCH_CHECK_VALUE(t.device() == x.device(), "a saved tensor came back on another device: ", t.device(), ", not ", x.device());
  const bool many = t.dim() == 3;
  const bool fp8 = scales.defined();
  if (fp8)
    TORCH_CHECK_VALUE(scales.device() == x.device() && scales.is_contiguous() && scales.element_size() == 1 && t.element_size() == 1 && t.size(-1) >= cols &&
                          scales.numel() == (many ? t.size(0) : 1) * ((t.size(-2) + 127) / 128) * ((cols + 127) / 128),
                      "an 8-bit weight came back with other bytes or scales");
  return rl_stack_t{t.data_ptr(), many ? t.size(0) : 1, t.size(-2), cols < 0 ? t.size(-1) : cols, t.stride(-2), many ? t.stride(0) : 0,
                    fp8 ? (int32_t)RL_FP8_B128 : code, fp8 ? scales.data_ptr() : nullptr, fp8 ? 128 : 0};
}

const int32_t* ends_of(const at::Tensor& ends, int64_t experts, const at::Tensor& x) {
  if (!ends.defined()) return nullptr;
  TORCH_CHECK_VALUE(ends.device() == x.device() && ends.dim() == 1 && ends.numel() == experts && ends.scalar_type() == at::kInt && ends.stride(0) == 1,
                    "ends must be a dense int32 vector with one element per expert");
  return ends.data_ptr<int32_t>();
}

// W: the stack [E, i, o] (or a matrix, one expert) in x's type, or the bytes of an 8-bit weight with `scales`; ends undefined: one expert
struct ExpertsNode : public torch::autograd::Function<ExpertsNode> {
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& A, const at::Tensor& B, const at::Tensor& W,
                            const std::optional<at::Tensor>& scales, const std::optional<at::Tensor>& ends, const std::optional<at::Tensor>& bias,
                            double scale, int64_t o, const std::optional<at::Tensor>& q, const std::optional<at::Tensor>& q_scales) {
    const int code = dtype_code(x.scalar_type());
    const at::Tensor s = scales.has_value() ? *scales : at::Tensor(), e = ends.has_value() ? *ends : at::Tensor();
    const rl_stack_t dw = stack_desc(W, x, code, o, s), da = stack_desc(A, x, code), db = stack_desc(B, x, code);
    const at::Tensor x2 = rows(x, dw.rows);
    const int64_t n = x2.size(0), r = da.cols;
    at::Tensor y = at::empty({n, o}, x.options());
    const at::Tensor T = at::empty({n, r}, x.options());
    const at::Tensor ws = scratch(p_experts_workspace_bytes(0, n, dw.experts, dw.rows, o, r, code, dw.dtype), x);
    const rl_opts_t opts = options(x, ws, bias, scale);
    const rl_tensor_t dx = desc(x2, code);
    rl_tensor_t dy = desc(y, code), dt = desc(T, code);
    if (q.has_value()) {  // (one matrix)
      const rl_tensor_t tq{q->data_ptr(), n, dw.rows, q->size(1), RL_FP8_R128, q_scales->data_ptr(), 128};
      const rl_tensor_t tw{dw.data, dw.rows, dw.cols, dw.ld, dw.dtype, dw.scales, dw.group}, ta = desc(A, code), tb = desc(B, code);
      rl_saved_t saved{};
      saved.T = T.data_ptr();
      saved.ldt = r;
      check(p_fp8_forward(&dx, &tq, &tw, &ta, &tb, &dy, &saved, &opts));
    } else {
      check(p_experts_forward(&dx, ends_of(e, dw.experts, x), &dw, &da, &db, &dy, &dt, &opts));
    }
    ctx->save_for_backward({x2, e, A, B, T, W, s});  // (the Python nodes' order; what a call lacks is skipped by both)
    ctx->saved_data["scale"] = scale;
    ctx->saved_data["o"] = o;
    ctx->saved_data["x_shape"] = x.sizes().vec();
    return shaped(y, x);
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto vars = ctx->get_saved_variables();
    TORCH_CHECK_VALUE(vars[0].is_cuda(), "the saved input came back on ", vars[0].device());
    const at::Tensor &ends = vars[1], &A = vars[2], &B = vars[3], &T = vars[4], &W = vars[5], &scales = vars[6];
    const int64_t o = ctx->saved_data["o"].toInt();
    const rl_stack_t dw = stack_desc(W, vars[0], dtype_code(W.scalar_type()), o, scales), da = stack_desc(A, vars[0], dtype_code(A.scalar_type())),
                     db = stack_desc(B, vars[0], dtype_code(B.scalar_type()));
    const rl_tensor_t dt = saved_desc(T, vars[0]);
    const at::Tensor x2 = rows(vars[0], dw.rows);
    const int64_t n = x2.size(0), i = dw.rows, r = da.cols;
    const int code = dtype_code(x2.scalar_type());
    const c10::OptionalDeviceGuard guard(x2.device());
    const at::Tensor dy2 = rows(grads[0], o);
    at::Tensor dx, dA, dB;
    rl_tensor_t tx{};
    rl_stack_t ta{}, tb{};
    if (ctx->needs_input_grad(0)) { dx = at::empty({n, i}, x2.options()); tx = desc(dx, code); }
    if (ctx->needs_input_grad(1)) { dA = at::empty(A.sizes(), A.options()); ta = stack_desc(dA, x2, da.dtype); }
    if (ctx->needs_input_grad(2)) { dB = at::empty(B.sizes(), B.options()); tb = stack_desc(dB, x2, db.dtype); }
    const at::Tensor ws = scratch(p_experts_workspace_bytes(1, n, dw.experts, i, o, r, code, dw.dtype), x2);
    const rl_opts_t opts = options(x2, ws, std::nullopt, ctx->saved_data["scale"].toDouble());
    const rl_tensor_t ddy = desc(dy2, dtype_code(dy2.scalar_type())), dx2 = desc(x2, code);
    check(p_experts_backward(&ddy, &dx2, ends_of(ends, dw.experts, x2), &dw, &da, &db, &dt, dx.defined() ? &tx : nullptr, dA.defined() ? &ta : nullptr,
                             dB.defined() ? &tb : nullptr, &opts));
    if (dx.defined()) dx = dx.view(ctx->saved_data["x_shape"].toIntVector());
    at::Tensor none;
    return {dx, dA, dB, none, none, none, none, none, none, none, none};
  }
};

// rows(), without a view where t is such a matrix already
at::Tensor matrix(const at::Tensor& t, int64_t cols) {
  if (t.dim() == 2 && t.size(1) == cols && t.stride(1) == 1 && t.stride(0) % 8 == 0 && t.stride(0) >= cols && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0) return t;
  return rows(t, cols);
}
// a dense tensor of any shape whose last dimension is `cols`, as a matrix
rl_tensor_t dense_desc(const at::Tensor& t, int64_t n, int64_t cols, int code) { return rl_tensor_t{t.data_ptr(), n, cols, cols, code, nullptr, 0}; }

// What a backward returns: where a graph of it is asked for, tensors whose own backward refuses (the library has no second derivatives).
torch::autograd::variable_list once(torch::autograd::variable_list list) {
  if (!at::GradMode::is_enabled()) return list;
  for (at::Tensor& t : list)
    if (t.defined()) t = t.detach().requires_grad_(true);
  const int64_t count = (int64_t)list.size();
  return (*std::make_shared<torch::autograd::DelayedError>("this gradient has no derivative: the operator can be differentiated once", count))(std::move(list));
}

// y, h where there is a residual, and y's rows in 8 bits (bytes and scales) where they are asked for
struct NormNode : public torch::autograd::Function<NormNode> {
  static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const std::optional<at::Tensor>& gain,
                                                const std::optional<at::Tensor>& residual, double eps, bool bytes) {
    const int code = dtype_code(x.scalar_type());
    const int64_t d = x.size(-1);
    const at::Tensor x2 = matrix(x, d), r2 = residual.has_value() ? matrix(*residual, d) : at::Tensor();
    const int64_t n = x2.size(0);
    const at::Tensor y = at::empty(x.sizes(), x.options()), h = residual.has_value() ? at::empty(x.sizes(), x.options()) : x2;
    const at::Tensor rstd = at::empty({n}, x.options().dtype(at::kFloat));
    at::Tensor q, qs;
    rl_tensor_t tq{};
    if (bytes) {
      const int64_t blocks = (d + 127) / 128;
      q = at::empty({n, blocks * 128}, x.options().dtype(at::kByte));
      qs = at::empty({blocks, (n + 15) / 16 * 16}, x.options().dtype(at::kByte));
      tq = rl_tensor_t{q.data_ptr(), n, d, blocks * 128, RL_FP8_R128, qs.data_ptr(), 128};
    }
    const rl_tensor_t tx = desc(x2, code), tr = residual.has_value() ? desc(r2, code) : rl_tensor_t{};
    rl_tensor_t ty = dense_desc(y, n, d, code), th = dense_desc(h, n, d, code);  // (th: of a residual's h alone)
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(x.device().index()).stream();
    check(p_rmsnorm_forward(&tx, residual.has_value() ? &tr : nullptr, gain.has_value() ? gain->data_ptr() : nullptr, (float)eps, &ty,
                            residual.has_value() ? &th : nullptr, rstd.data_ptr<float>(), bytes ? &tq : nullptr, &opts));
    ctx->save_for_backward({h, gain.has_value() ? *gain : at::Tensor(), rstd});
    ctx->saved_data["x_shape"] = x.sizes().vec();
    ctx->saved_data["residual"] = residual.has_value();
    ctx->saved_data["gain"] = gain.has_value();
    ctx->set_materialize_grads(false);
    torch::autograd::variable_list out{y};
    if (residual.has_value()) out.push_back(h);
    if (bytes) {
      ctx->mark_non_differentiable({q, qs});
      out.push_back(q);
      out.push_back(qs);
    }
    return out;
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto vars = ctx->get_saved_variables();
    const bool residual = ctx->saved_data["residual"].toBool(), gain = ctx->saved_data["gain"].toBool();
    // (edges are those of the tensors that there are)
    const bool need_x = ctx->needs_input_grad(0), need_gain = gain && ctx->needs_input_grad(1), need_r = residual && ctx->needs_input_grad(gain ? 2 : 1);
    const at::Tensor none, dh = residual && grads.size() > 1 ? grads[1] : none;
    if (!grads[0].defined()) return {need_x ? dh : none, none, need_r ? dh : none, none, none};  // (as it came, graph and all)
    TORCH_CHECK_VALUE(vars[0].is_cuda(), "the saved input came back on ", vars[0].device());
    const int64_t d = vars[0].size(-1);
    const at::Tensor h2 = matrix(vars[0], d);
    const c10::OptionalDeviceGuard guard(h2.device());
    const at::Tensor dy2 = matrix(grads[0], d), dh2 = dh.defined() ? matrix(dh, d) : none;
    const int64_t n = h2.size(0);
    const int code = dtype_code(h2.scalar_type());
    const float* const rstd = static_cast<const float*>(saved_vec(vars[2], n, at::kFloat, h2, "rstd"));
    const void* const w = gain ? saved_vec(vars[1], d, dy2.scalar_type(), h2, "gain") : nullptr;
    at::Tensor dx, dw;
    rl_tensor_t tx{};
    if (need_x || need_r) { dx = at::empty(ctx->saved_data["x_shape"].toIntVector(), h2.options()); tx = dense_desc(dx, n, d, code); }
    if (need_gain) dw = at::empty({d}, h2.options());
    const at::Tensor ws = need_gain ? scratch(p_rmsnorm_workspace_bytes(n, d, code), h2) : none;
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(h2.device().index()).stream();
    if (need_gain) {
      opts.workspace = ws.data_ptr();
      opts.workspace_bytes = (size_t)ws.numel();
    }
    const rl_tensor_t ty = desc(dy2, dtype_code(dy2.scalar_type())), tg = dh.defined() ? desc(dh2, dtype_code(dh2.scalar_type())) : rl_tensor_t{}, th = desc(h2, code);
    check(p_rmsnorm_backward(&ty, dh.defined() ? &tg : nullptr, &th, w, rstd, dx.defined() ? &tx : nullptr, need_gain ? dw.data_ptr() : nullptr, &opts));
    return once({need_x ? dx : none, dw, need_r ? dx : none, none, none});
  }
};

// rows of logits as the library takes them: any distance between them, which a single row may have wrong
rl_tensor_t logits_desc(const at::Tensor& t) {
  TORCH_CHECK_VALUE(t.is_cuda() && t.dim() == 2 && (t.size(1) < 2 || t.stride(1) == 1), "expected 2-D logits with contiguous rows");
  const int64_t ld = t.size(0) > 1 ? t.stride(0) : std::max(t.size(1), t.stride(0));
  return rl_tensor_t{t.data_ptr(), t.size(0), t.size(1), ld, dtype_code(t.scalar_type()), nullptr, 0};
}
template <typename V>
V* saved_table(const at::Tensor& t, at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& x, const char* name) {
  TORCH_CHECK_VALUE(t.device() == x.device() && t.sizes() == sizes && t.scalar_type() == type && t.is_contiguous(), name, " must be a dense tensor of ", sizes);
  return t.data_ptr<V>();
}

struct RouteNode : public torch::autograd::Function<RouteNode> {
  static rl_route_t plan(const std::vector<int64_t>& how, double scale, const at::Tensor& bias) {
    return rl_route_t{(int32_t)how[0], (int32_t)how[1], (int32_t)how[2], (int32_t)how[3], (int32_t)how[4], (int32_t)how[5], (int32_t)how[6], (float)scale,
                      bias.defined() ? bias.data_ptr<float>() : nullptr};
  }
  static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& logits, const std::optional<at::Tensor>& bias,
                                                std::vector<int64_t> how, double scale) {
    const rl_tensor_t tl = logits_desc(logits);
    const int64_t n = tl.rows, top = how[1];
    const at::TensorOptions ints = logits.options().dtype(at::kInt);
    const at::Tensor weight = at::empty({n, top}, logits.options().dtype(at::kFloat)), expert = at::empty({n, top}, ints), place = at::empty({n, top}, ints),
                     source = at::empty({n * top}, ints), ends = at::empty({how[0]}, ints);
    const at::Tensor ws = scratch(p_route_workspace_bytes(n, how[0], top), logits);
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(logits.device().index()).stream();
    opts.workspace = ws.data_ptr();
    opts.workspace_bytes = (size_t)ws.numel();
    const rl_route_t route = plan(how, scale, bias.has_value() ? *bias : at::Tensor());
    check(p_route_forward(&tl, &route, expert.data_ptr<int32_t>(), weight.data_ptr<float>(), place.data_ptr<int32_t>(), source.data_ptr<int32_t>(),
                          ends.data_ptr<int32_t>(), &opts));
    ctx->save_for_backward({logits, expert});
    // (the backward asks whether there is one and reads none of it: it may be updated in place before that)
    if (bias.has_value()) ctx->saved_data["bias"] = bias->detach();
    ctx->saved_data["how"] = how;
    ctx->saved_data["scale"] = scale;
    ctx->set_materialize_grads(false);  // (zeros for the four tables would be four launches)
    ctx->mark_non_differentiable({expert, place, source, ends});
    return {weight, expert, place, source, ends};
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto vars = ctx->get_saved_variables();
    const at::Tensor& logits = vars[0];
    const auto kept = ctx->saved_data.find("bias");
    const at::Tensor bias = kept != ctx->saved_data.end() ? kept->second.toTensor() : at::Tensor();
    const std::vector<int64_t> how = ctx->saved_data["how"].toIntVector();
    at::Tensor none;
    if (!grads[0].defined()) return {none, none, none, none};
    const rl_tensor_t tl = logits_desc(logits);
    const c10::OptionalDeviceGuard guard(logits.device());
    const int32_t* const expert = saved_table<int32_t>(vars[1], {tl.rows, how[1]}, at::kInt, logits, "expert");
    const at::Tensor dw = grads[0].contiguous(), dl = at::empty({tl.rows, tl.cols}, logits.options());
    rl_tensor_t td = logits_desc(dl);
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(logits.device().index()).stream();
    const rl_route_t route = plan(how, ctx->saved_data["scale"].toDouble(), bias);
    check(p_route_backward(&tl, &route, expert, saved_table<float>(dw, {tl.rows, how[1]}, at::kFloat, logits, "dweight"), &td, &opts));
    return once({dl, none, none, none});
  }
};

struct GatherNode : public torch::autograd::Function<GatherNode> {
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& place, const at::Tensor& source) {
    const int code = dtype_code(x.scalar_type());
    const at::Tensor x2 = matrix(x, x.size(-1));
    const at::Tensor out = at::empty({place.numel(), x2.size(1)}, x.options());
    const rl_tensor_t tx = desc(x2, code);
    rl_tensor_t tr = desc(out, code);
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(x.device().index()).stream();
    check(p_gather_forward(&tx, place.data_ptr<int32_t>(), source.data_ptr<int32_t>(), (int)place.size(1), &tr, &opts));
    ctx->save_for_backward({place});
    ctx->saved_data["x_shape"] = x.sizes().vec();
    return out;
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto vars = ctx->get_saved_variables();
    const at::Tensor& place = vars[0];
    const c10::OptionalDeviceGuard guard(grads[0].device());
    const at::Tensor dr = matrix(grads[0], grads[0].size(-1));
    const int code = dtype_code(dr.scalar_type());
    const at::Tensor dx = at::empty(ctx->saved_data["x_shape"].toIntVector(), dr.options());
    // (dx has the forward's rows: a table of as many entries may have others)
    TORCH_CHECK_VALUE(place.dim() == 2 && place.numel() == dr.size(0) && place.size(0) * dr.size(1) == dx.numel(), "place came back as another table");
    const rl_tensor_t tr = desc(dr, code);
    rl_tensor_t tx = dense_desc(dx, place.size(0), dr.size(1), code);
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(dr.device().index()).stream();
    check(p_gather_backward(&tr, saved_table<int32_t>(place, place.sizes(), at::kInt, dr, "place"), (int)place.size(1), &tx, &opts));
    at::Tensor none;
    return once({dx, none, none});
  }
};

struct CombineNode : public torch::autograd::Function<CombineNode> {
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& back, const at::Tensor& weight, const at::Tensor& place, const at::Tensor& source,
                            const std::optional<at::Tensor>& add) {
    const int code = dtype_code(back.scalar_type());
    const int64_t n = place.size(0), d = back.size(-1);
    const at::Tensor r2 = matrix(back, d), w = weight.contiguous(), a2 = add.has_value() ? matrix(*add, d) : at::Tensor();
    const at::Tensor y = at::empty(add.has_value() ? add->sizes() : at::IntArrayRef({n, d}), back.options());
    const rl_tensor_t tr = desc(r2, code), ta = add.has_value() ? desc(a2, code) : rl_tensor_t{};
    rl_tensor_t ty = dense_desc(y, n, d, code);
    rl_opts_t opts{};
    opts.stream = c10::hip::getCurrentHIPStream(back.device().index()).stream();
    check(p_combine_forward(&tr, place.data_ptr<int32_t>(), w.data_ptr<float>(), (int)place.size(1), add.has_value() ? &ta : nullptr, &ty, &opts));
    ctx->save_for_backward({r2, place, source, w});
    ctx->saved_data["add"] = add.has_value();
    return y;
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto vars = ctx->get_saved_variables();
    const at::Tensor &place = vars[1], &w = vars[3];
    TORCH_CHECK_VALUE(vars[0].is_cuda() && vars[0].dim() == 2, "the saved rows came back as ", vars[0].sizes(), " on ", vars[0].device());
    const int64_t d = vars[0].size(1);
    const at::Tensor r2 = matrix(vars[0], d);
    const c10::OptionalDeviceGuard guard(r2.device());
    const at::Tensor dy = matrix(grads[0], d), none;
    const int code = dtype_code(r2.scalar_type());
    const bool need_r = ctx->needs_input_grad(0), need_w = ctx->needs_input_grad(1), need_a = ctx->saved_data["add"].toBool() && ctx->needs_input_grad(4);
    at::Tensor dr, dw;
    rl_tensor_t tr{};
    if (need_r) { dr = at::empty({r2.size(0), d}, r2.options()); tr = desc(dr, code); }
    if (need_w) dw = at::empty(w.sizes(), w.options());
    if (need_r || need_w) {
      const rl_tensor_t ty = desc(dy, dtype_code(dy.scalar_type())), tb = desc(r2, code);
      rl_opts_t opts{};
      opts.stream = c10::hip::getCurrentHIPStream(r2.device().index()).stream();
      TORCH_CHECK_VALUE(place.dim() == 2 && place.numel() == r2.size(0), "place came back as another table");
      check(p_combine_backward(&ty, &tb, saved_table<int32_t>(place, place.sizes(), at::kInt, r2, "place"),
                               saved_table<int32_t>(vars[2], {place.numel()}, at::kInt, r2, "source"), saved_table<float>(w, place.sizes(), at::kFloat, r2, "weight"),
                               (int)place.size(1), need_r ? &tr : nullptr, need_w ? dw.data_ptr<float>() : nullptr, &opts));
    }
    auto out = once({dr, dw, none, none, none});
    if (need_a) out[4] = grads[0];
    return out;
  }
};

// no mode, transform or tracer that has to see a Python-level function
bool plainly_called() {
  return !(torch::jit::tracer::isTracing() || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set() ||
           c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode));
}
// a plain tensor with elements on the current GPU
const at::Tensor* plain_tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.layout() != at::kStrided || t.numel() == 0 || t.device().index() != c10::hip::current_device() || t.is_conj() || t.is_neg() || t._is_zerotensor())
    return nullptr;
  return &t;
}
bool plain_ints(const at::Tensor* t, int64_t dim) { return t != nullptr && t->scalar_type() == at::kInt && t->dim() == dim && t->is_contiguous(); }

PyObject* tuple_of(const torch::autograd::variable_list& list) {
  PyObject* out = PyTuple_New((Py_ssize_t)list.size());
  if (out == nullptr) throw python_error();
  for (size_t k = 0; k < list.size(); ++k) {
    PyObject* t = THPVariable_Wrap(list[k]);
    if (t == nullptr) {
      Py_DECREF(out);
      throw python_error();
    }
    PyTuple_SET_ITEM(out, (Py_ssize_t)k, t);
  }
  return out;
}

bool plain_2d(const at::Tensor& t, const at::Tensor& x) {
  return t.dim() == 2 && t.stride(1) == 1 && t.scalar_type() == x.scalar_type() && t.device() == x.device() && t.layout() == at::kStrided;
}

bool plain_1d(const at::Tensor& t, int64_t count, const at::Tensor& x) {
  return t.dim() == 1 && t.stride(0) == 1 && t.scalar_type() == x.scalar_type() && t.numel() == count && t.device() == x.device() && t.layout() == at::kStrided;
}

// x, W, A and B (args[0 .. 3]), vectors as long as B has rows (0) or columns (1), and a bias or None as a native node takes them; nothing
// here raises
bool operands_ok(PyObject* const* args, PyObject* bias, std::initializer_list<std::pair<PyObject*, int>> vectors) {
  for (int k = 0; k < 4; ++k)
    if (!THPVariable_CheckExact(args[k])) return false;
  if (bias != Py_None && !THPVariable_CheckExact(bias)) return false;
  for (const auto& v : vectors)
    if (!THPVariable_CheckExact(v.first)) return false;
  if (torch::jit::tracer::isTracing() || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set() ||
      c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode))
    return false;
  const at::Tensor &x = THPVariable_Unpack(args[0]), &W = THPVariable_Unpack(args[1]), &A = THPVariable_Unpack(args[2]), &B = THPVariable_Unpack(args[3]);
  if (!x.is_cuda() || x.layout() != at::kStrided || x.dim() < 1 || dtype_code(x.scalar_type()) < 0 || x.numel() == 0) return false;
  if (!plain_2d(W, x) || !plain_2d(A, x) || !plain_2d(B, x) || W.numel() == 0 || A.numel() == 0 || B.numel() == 0) return false;
  if (x.size(-1) != W.size(0) || x.device().index() != c10::hip::current_device()) return false;
  // (conjugate, negative and zero-tensor views carry their values lazily)
  auto lazy = [](const at::Tensor& t) { return t.is_conj() || t.is_neg() || t._is_zerotensor(); };
  for (const at::Tensor* t : {&x, &W, &A, &B})
    if (lazy(*t)) return false;
  for (const auto& v : vectors) {
    const at::Tensor& t = THPVariable_Unpack(v.first);
    if (!plain_1d(t, B.size(v.second), x) || lazy(t)) return false;
  }
  if (bias != Py_None) {
    const at::Tensor& t = THPVariable_Unpack(bias);
    if (t.dim() != 1 || t.stride(0) != 1 || t.scalar_type() != x.scalar_type() || t.numel() != W.size(1) || t.device() != x.device()) return false;
  }
  return true;
}

std::optional<at::Tensor> optional_tensor(PyObject* o) {
  return o == Py_None ? std::nullopt : std::optional<at::Tensor>(THPVariable_Unpack(o));
}

bool pair_of(PyObject* o, int64_t* fwd, int64_t* bwd) {
  if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 2) return false;
  PyObject *f = PyTuple_GET_ITEM(o, 0), *b = PyTuple_GET_ITEM(o, 1);
  if (!PyLong_CheckExact(f) || !PyLong_CheckExact(b)) return false;
  *fwd = PyLong_AsLongLong(f);
  *bwd = PyLong_AsLongLong(b);
  if (PyErr_Occurred()) {  // integers beyond 64 bits: the Python path has the message
    PyErr_Clear();
    return false;
  }
  return *fwd >= RL_FWD_DEFAULT && *fwd <= RL_FWD3 && *bwd >= RL_BWD_DEFAULT && *bwd <= RL_BWD8;
}

// lora(x, W, A, B, bias, scale, (fwd, bwd), keep_merged, dropout=None, keep_t=False): y, or None (see above)
PyObject* py_lora(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs < 8 || nargs > 10 || p_forward == nullptr) Py_RETURN_NONE;
  int64_t fwd = 0, bwd = 0;
  if (!PyFloat_CheckExact(args[5]) || !PyBool_Check(args[7]) || !pair_of(args[6], &fwd, &bwd)) Py_RETURN_NONE;
  double p = 0.0;
  int64_t seed = 0;
  if (nargs > 8 && args[8] != Py_None) {
    if (!PyTuple_CheckExact(args[8]) || PyTuple_GET_SIZE(args[8]) != 2) Py_RETURN_NONE;
    PyObject *dp = PyTuple_GET_ITEM(args[8], 0), *ds = PyTuple_GET_ITEM(args[8], 1);
    if (!PyFloat_CheckExact(dp) || !PyLong_CheckExact(ds)) Py_RETURN_NONE;
    p = PyFloat_AS_DOUBLE(dp);
    seed = PyLong_AsLongLong(ds);
  }
  if (PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  if (nargs > 9 && !PyBool_Check(args[9])) Py_RETURN_NONE;
  const bool keep_merged = args[7] == Py_True, keep_t = nargs > 9 && args[9] == Py_True;
  if (!operands_ok(args, args[4], {})) Py_RETURN_NONE;
  const at::Tensor &x = THPVariable_Unpack(args[0]), &W = THPVariable_Unpack(args[1]), &A = THPVariable_Unpack(args[2]), &B = THPVariable_Unpack(args[3]);
  const std::optional<at::Tensor> bias = optional_tensor(args[4]);
  at::Tensor y;
  {
    pybind11::gil_scoped_release release;
    y = LoRANode::apply(x, W, A, B, bias, PyFloat_AS_DOUBLE(args[5]), fwd, bwd, keep_merged, p, seed, keep_t);
  }
  return THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

// vera(x, W, A, B, d, b, bias, scale, (fwd, bwd)): y, or None
PyObject* py_vera(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  int64_t fwd = 0, bwd = 0;
  if (nargs != 9 || p_vera_forward == nullptr || !PyFloat_CheckExact(args[7]) || !pair_of(args[8], &fwd, &bwd)) Py_RETURN_NONE;
  if (!operands_ok(args, args[6], {{args[4], 0}, {args[5], 1}})) Py_RETURN_NONE;
  const at::Tensor &x = THPVariable_Unpack(args[0]), &W = THPVariable_Unpack(args[1]), &A = THPVariable_Unpack(args[2]), &B = THPVariable_Unpack(args[3]);
  const at::Tensor &d = THPVariable_Unpack(args[4]), &b = THPVariable_Unpack(args[5]);
  const std::optional<at::Tensor> bias = optional_tensor(args[6]);
  at::Tensor y;
  {
    pybind11::gil_scoped_release release;
    y = VeRANode::apply(x, W, A, B, d, b, bias, PyFloat_AS_DOUBLE(args[7]), fwd, bwd);
  }
  return THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

// dora(x, W, A, B, m, bias, scale, bwd): y, or None
PyObject* py_dora(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 8 || p_dora_forward == nullptr || !PyFloat_CheckExact(args[6]) || !PyLong_CheckExact(args[7])) Py_RETURN_NONE;
  const int64_t bwd = PyLong_AsLongLong(args[7]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  if (bwd < RL_BWD_DEFAULT || bwd > RL_BWD8) Py_RETURN_NONE;
  if (!operands_ok(args, args[5], {{args[4], 1}})) Py_RETURN_NONE;
  const at::Tensor &x = THPVariable_Unpack(args[0]), &W = THPVariable_Unpack(args[1]), &A = THPVariable_Unpack(args[2]), &B = THPVariable_Unpack(args[3]);
  const at::Tensor& m = THPVariable_Unpack(args[4]);
  const std::optional<at::Tensor> bias = optional_tensor(args[5]);
  at::Tensor y;
  {
    pybind11::gil_scoped_release release;
    y = DoRANode::apply(x, W, A, B, m, bias, PyFloat_AS_DOUBLE(args[6]), bwd);
  }
  return THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

// norm(x, gain, eps, residual, bytes): (y, [h,] [bytes, scales]), or None; gain and residual may be None
PyObject* py_norm(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5 || p_rmsnorm_forward == nullptr || !PyFloat_CheckExact(args[2]) || !PyBool_Check(args[4]) || !plainly_called()) Py_RETURN_NONE;
  const at::Tensor* const x = plain_tensor(args[0]);
  if (x == nullptr || x->dim() < 1 || dtype_code(x->scalar_type()) < 0) Py_RETURN_NONE;
  std::optional<at::Tensor> gain, residual;
  if (args[1] != Py_None) {
    const at::Tensor* const t = plain_tensor(args[1]);
    if (t == nullptr || t->dim() != 1 || t->numel() != x->size(-1) || t->stride(0) != 1 || t->scalar_type() != x->scalar_type()) Py_RETURN_NONE;
    gain = *t;
  }
  if (args[3] != Py_None) {
    const at::Tensor* const t = plain_tensor(args[3]);
    if (t == nullptr || t->sizes() != x->sizes() || t->scalar_type() != x->scalar_type()) Py_RETURN_NONE;
    residual = *t;
  }
  torch::autograd::variable_list out;
  {
    pybind11::gil_scoped_release release;
    out = NormNode::apply(*x, gain, residual, PyFloat_AS_DOUBLE(args[2]), args[4] == Py_True);
  }
  return tuple_of(out);
  END_HANDLE_TH_ERRORS
}

// the whole numbers of a plan; false where they are not seven of them
bool plan_of(PyObject* o, std::vector<int64_t>* how) {
  if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 7) return false;
  for (int k = 0; k < 7; ++k) {
    PyObject* const v = PyTuple_GET_ITEM(o, k);
    if (!PyLong_CheckExact(v)) return false;
    (*how)[k] = PyLong_AsLongLong(v);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      return false;
    }
    if ((*how)[k] < 0 || (*how)[k] > 1 << 30) return false;
  }
  return true;
}

// route(logits, bias, (experts, top, score, renormalise, groups, groups_kept, group_top), scale): (weight, expert, place, source, ends), or None
PyObject* py_route(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 4 || p_route_forward == nullptr || !PyFloat_CheckExact(args[3]) || !plainly_called()) Py_RETURN_NONE;
  std::vector<int64_t> how(7);
  if (!plan_of(args[2], &how)) Py_RETURN_NONE;
  const at::Tensor* const l = plain_tensor(args[0]);
  if (l == nullptr || l->dim() != 2 || dtype_code(l->scalar_type()) < 0 || (l->size(1) > 1 && l->stride(1) != 1) || (l->size(0) > 1 && l->stride(0) < l->size(1)) ||
      l->size(1) != how[0] || how[1] > how[0] || how[1] < 1)
    Py_RETURN_NONE;
  std::optional<at::Tensor> bias;
  if (args[1] != Py_None) {
    const at::Tensor* const t = plain_tensor(args[1]);
    if (t == nullptr || t->dim() != 1 || t->numel() != how[0] || t->stride(0) != 1 || t->scalar_type() != at::kFloat) Py_RETURN_NONE;
    bias = *t;
  }
  torch::autograd::variable_list out;
  {
    pybind11::gil_scoped_release release;
    out = RouteNode::apply(*l, bias, how, PyFloat_AS_DOUBLE(args[3]));
  }
  return tuple_of(out);
  END_HANDLE_TH_ERRORS
}

// gather(x, place, source): rows, or None
PyObject* py_gather(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 3 || p_gather_forward == nullptr || !plainly_called()) Py_RETURN_NONE;
  const at::Tensor *const x = plain_tensor(args[0]), *const place = plain_tensor(args[1]), *const source = plain_tensor(args[2]);
  if (x == nullptr || x->dim() < 1 || dtype_code(x->scalar_type()) < 0 || !plain_ints(place, 2) || !plain_ints(source, 1)) Py_RETURN_NONE;
  if (place->size(0) != x->numel() / x->size(-1) || source->numel() != place->numel()) Py_RETURN_NONE;
  at::Tensor out;
  {
    pybind11::gil_scoped_release release;
    out = GatherNode::apply(*x, *place, *source);
  }
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// combine(rows, place, source, weight, add): y, or None; add may be None
PyObject* py_combine(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5 || p_combine_forward == nullptr || !plainly_called()) Py_RETURN_NONE;
  const at::Tensor *const back = plain_tensor(args[0]), *const place = plain_tensor(args[1]), *const source = plain_tensor(args[2]), *const weight = plain_tensor(args[3]);
  if (back == nullptr || back->dim() != 2 || dtype_code(back->scalar_type()) < 0 || !plain_ints(place, 2) || !plain_ints(source, 1)) Py_RETURN_NONE;
  if (weight == nullptr || weight->scalar_type() != at::kFloat || weight->sizes() != place->sizes() || source->numel() != place->numel() || back->size(0) != place->numel())
    Py_RETURN_NONE;
  std::optional<at::Tensor> add;
  if (args[4] != Py_None) {
    const at::Tensor* const t = plain_tensor(args[4]);
    if (t == nullptr || t->dim() < 1 || t->size(-1) != back->size(1) || t->numel() != place->size(0) * back->size(1) || t->scalar_type() != back->scalar_type()) Py_RETURN_NONE;
    add = *t;
  }
  at::Tensor out;
  {
    pybind11::gil_scoped_release release;
    out = CombineNode::apply(*back, *weight, *place, *source, add);
  }
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// experts(x, A, B, W, scales, ends, bias, scale, d_out[, rows, row_scales]): y, or None; scales, ends, bias and the last two may be None.  W, A and B are
// stacks, or with ends None matrices; rows: x's rows in 8 bits, for an 8-bit matrix; the library's checks have the messages for sizes that do not fit
PyObject* py_experts(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if ((nargs != 9 && nargs != 11) || p_experts_forward == nullptr || !PyFloat_CheckExact(args[7]) || !PyLong_CheckExact(args[8])) Py_RETURN_NONE;
  const int64_t o = PyLong_AsLongLong(args[8]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  if (torch::jit::tracer::isTracing() || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set() ||
      c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode))
    Py_RETURN_NONE;
  for (int k = 0; k < 7; ++k) {
    if (k >= 4 && args[k] == Py_None) continue;
    if (!THPVariable_CheckExact(args[k])) Py_RETURN_NONE;
    const at::Tensor& t = THPVariable_Unpack(args[k]);
    if (!t.is_cuda() || t.layout() != at::kStrided || t.numel() == 0 || t.device().index() != c10::hip::current_device() || t.is_conj() || t.is_neg() ||
        t._is_zerotensor())
      Py_RETURN_NONE;
  }
  const at::Tensor &x = THPVariable_Unpack(args[0]), &A = THPVariable_Unpack(args[1]), &B = THPVariable_Unpack(args[2]), &W = THPVariable_Unpack(args[3]);
  const std::optional<at::Tensor> scales = optional_tensor(args[4]), ends = optional_tensor(args[5]), bias = optional_tensor(args[6]);
  const int64_t dim = ends.has_value() ? 3 : 2;
  for (const at::Tensor* t : {&A, &B, &W})
    if (t->dim() != dim || t->stride(-1) != 1) Py_RETURN_NONE;
  if (dtype_code(x.scalar_type()) < 0 || A.scalar_type() != x.scalar_type() || B.scalar_type() != x.scalar_type() || x.dim() < 1 || x.size(-1) != W.size(-2)) Py_RETURN_NONE;
  if (scales.has_value() ? (scales->dim() != dim || scales->element_size() != 1 || W.element_size() != 1 || W.size(-1) < o ||
                            scales->size(-2) != (W.size(-2) + 127) / 128 || scales->size(-1) != (o + 127) / 128 || (dim == 3 && scales->size(0) != W.size(0)))
                         : (W.scalar_type() != x.scalar_type() || W.size(-1) != o))
    Py_RETURN_NONE;
  if (ends.has_value() && (ends->dim() != 1 || ends->numel() != W.size(0) || ends->scalar_type() != at::kInt || ends->stride(0) != 1)) Py_RETURN_NONE;
  if (bias.has_value() && (bias->scalar_type() != x.scalar_type() || !bias->is_contiguous() || bias->dim() != dim - 1 || bias->size(-1) != o ||
                            (dim == 3 && bias->size(0) != W.size(0))))
    Py_RETURN_NONE;
  std::optional<at::Tensor> q, q_scales;
  if (nargs == 11 && args[9] != Py_None) {
    const at::Tensor *const t = plain_tensor(args[9]), *const u = plain_tensor(args[10]);
    const int64_t n = x.numel() / x.size(-1), blocks = (x.size(-1) + 127) / 128;
    if (t == nullptr || u == nullptr || ends.has_value() || !scales.has_value() || t->element_size() != 1 || u->element_size() != 1) Py_RETURN_NONE;
    if (t->sizes() != at::IntArrayRef({n, blocks * 128}) || u->sizes() != at::IntArrayRef({blocks, (n + 15) / 16 * 16}) || !t->is_contiguous() || !u->is_contiguous()) Py_RETURN_NONE;
    q = *t;
    q_scales = *u;
  }
  at::Tensor y;
  {
    pybind11::gil_scoped_release release;
    y = ExpertsNode::apply(x, A, B, W, scales, ends, bias, PyFloat_AS_DOUBLE(args[7]), o, q, q_scales);
  }
  return THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

// init(addresses of the library's entry points in the order below, check)
PyObject* py_init(PyObject*, PyObject* args) {
  PyObject *list, *chk;
  if (!PyArg_ParseTuple(args, "O!O", &PyTuple_Type, &list, &chk)) return nullptr;
  unsigned long long a[24];
  constexpr Py_ssize_t count = sizeof(a) / sizeof(a[0]);
  if (PyTuple_GET_SIZE(list) != count) {
    PyErr_SetString(PyExc_TypeError, "another number of entry points was expected");
    return nullptr;
  }
  for (Py_ssize_t k = 0; k < count; ++k) {
    a[k] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(list, k));
    if (PyErr_Occurred()) return nullptr;
  }
  int k = 0;
  auto take = [&](auto& p) { p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(a[k++]); };
  take(p_forward); take(p_backward); take(p_workspace_bytes);
  take(p_vera_forward); take(p_vera_backward); take(p_vera_workspace_bytes);
  take(p_dora_forward); take(p_dora_backward); take(p_dora_workspace_bytes);
  take(p_experts_forward); take(p_experts_backward); take(p_experts_workspace_bytes);
  take(p_fp8_forward); take(p_fp8_values);
  take(p_rmsnorm_forward); take(p_rmsnorm_backward); take(p_rmsnorm_workspace_bytes);
  take(p_route_forward); take(p_route_backward); take(p_route_workspace_bytes);
  take(p_gather_forward); take(p_gather_backward); take(p_combine_forward); take(p_combine_backward);
  Py_INCREF(chk);
  Py_XDECREF(g_check);
  g_check = chk;
  Py_RETURN_NONE;
}

// ---- binding.py's calls into buffers that the caller keeps ----------------------------------------------
//
// The same call as through ctypes, with the operands' descriptors made here: 3 us of host time where Python's marshalling and checks take 6 to 8 (the
// kernels of a small call take 3 to 4).  Each returns True, or None where anything is not as the call wants it: binding.py's own path has the messages.

// rows of a matrix; None where `optional`
struct RowsArg {
  rl_tensor_t t{};
  bool there = false, ok = false;
  RowsArg(PyObject* o, bool optional = false) {
    if (o == Py_None) {
      ok = optional;
      return;
    }
    const at::Tensor* const x = plain_tensor(o);
    if (x == nullptr || x->dim() != 2 || x->stride(1) != 1) return;
    const int code = dtype_code(x->scalar_type());
    if (code < 0) return;
    t = desc(*x, code);
    there = ok = true;
  }
  const rl_tensor_t* in() const { return there ? &t : nullptr; }
  rl_tensor_t* out() { return there ? &t : nullptr; }
};
// a dense tensor of `count` elements of a type; None where `optional`
struct ListArg {
  void* p = nullptr;
  int64_t last = 0;  // its last dimension
  bool ok = false;
  ListArg(PyObject* o, at::ScalarType type, int64_t dim, int64_t count, bool optional = false) {
    if (o == Py_None) {
      ok = optional;
      return;
    }
    const at::Tensor* const x = plain_tensor(o);
    if (x == nullptr || x->scalar_type() != type || x->dim() != dim || (count >= 0 && x->numel() != count) || !x->is_contiguous()) return;
    p = x->data_ptr();
    last = x->size(-1);
    ok = true;
  }
};
at::ScalarType scalar_type(int code) { return code == RL_F32 ? at::kFloat : (code == RL_F16 ? at::kHalf : at::kBFloat16); }
rl_opts_t current_options() {
  rl_opts_t o{};
  o.stream = c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream();
  return o;
}

// norm_into(X, gain, Y, eps, residual, H, rstd, bytes, scales)
PyObject* py_norm_into(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 9 || p_rmsnorm_forward == nullptr || !PyFloat_CheckExact(args[3])) Py_RETURN_NONE;
  RowsArg x(args[0]), y(args[2]), r(args[4], true), h(args[5], true);
  if (!x.ok || !y.ok || !r.ok || !h.ok) Py_RETURN_NONE;
  const int64_t n = x.t.rows, d = x.t.cols, blocks = (d + 127) / 128;
  const ListArg gain(args[1], scalar_type(x.t.dtype), 1, d, true), rstd(args[6], at::kFloat, 1, n, true), q(args[7], at::kByte, 2, n * blocks * 128, true),
      qs(args[8], at::kByte, 2, blocks * ((n + 15) / 16 * 16), true);
  if (!gain.ok || !rstd.ok || !q.ok || !qs.ok || (q.p == nullptr) != (qs.p == nullptr) || (q.p != nullptr && q.last != blocks * 128)) Py_RETURN_NONE;
  rl_tensor_t tq{q.p, n, d, blocks * 128, RL_FP8_R128, qs.p, 128};
  const rl_opts_t opts = current_options();
  check(p_rmsnorm_forward(x.in(), r.in(), gain.p, (float)PyFloat_AS_DOUBLE(args[3]), y.out(), h.out(), static_cast<float*>(rstd.p), q.p != nullptr ? &tq : nullptr, &opts));
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// route_into(logits, plan, scale, bias, weight, expert, place, source, ends, workspace)
PyObject* py_route_into(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  std::vector<int64_t> how(7);
  if (nargs != 10 || p_route_forward == nullptr || !plan_of(args[1], &how) || !PyFloat_CheckExact(args[2])) Py_RETURN_NONE;
  const at::Tensor* const l = plain_tensor(args[0]);
  if (l == nullptr || l->dim() != 2 || dtype_code(l->scalar_type()) < 0 || (l->size(1) > 1 && l->stride(1) != 1)) Py_RETURN_NONE;
  const rl_tensor_t tl = logits_desc(*l);
  const int64_t n = tl.rows, copies = n * how[1];
  const ListArg bias(args[3], at::kFloat, 1, how[0], true), weight(args[4], at::kFloat, 2, copies), expert(args[5], at::kInt, 2, copies),
      place(args[6], at::kInt, 2, copies), source(args[7], at::kInt, 1, copies), ends(args[8], at::kInt, 1, how[0]), ws(args[9], at::kByte, 1, -1, true);
  if (!bias.ok || !weight.ok || !expert.ok || !place.ok || !source.ok || !ends.ok || !ws.ok) Py_RETURN_NONE;
  if (weight.last != how[1] || expert.last != how[1] || place.last != how[1]) Py_RETURN_NONE;
  rl_opts_t opts = current_options();
  opts.workspace = ws.p;
  opts.workspace_bytes = (size_t)ws.last;
  const rl_route_t route{(int32_t)how[0], (int32_t)how[1], (int32_t)how[2], (int32_t)how[3], (int32_t)how[4], (int32_t)how[5], (int32_t)how[6],
                         (float)PyFloat_AS_DOUBLE(args[2]), static_cast<const float*>(bias.p)};
  check(p_route_forward(&tl, &route, static_cast<int32_t*>(expert.p), static_cast<float*>(weight.p), static_cast<int32_t*>(place.p),
                        static_cast<int32_t*>(source.p), static_cast<int32_t*>(ends.p), &opts));
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// gather_into(X, place, source, rows)
PyObject* py_gather_into(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 4 || p_gather_forward == nullptr) Py_RETURN_NONE;
  RowsArg x(args[0]), rows(args[3]);
  if (!x.ok || !rows.ok) Py_RETURN_NONE;
  const ListArg place(args[1], at::kInt, 2, rows.t.rows), source(args[2], at::kInt, 1, rows.t.rows);
  if (!place.ok || !source.ok || place.last * x.t.rows != rows.t.rows) Py_RETURN_NONE;
  const rl_opts_t opts = current_options();
  check(p_gather_forward(x.in(), static_cast<const int32_t*>(place.p), static_cast<const int32_t*>(source.p), (int)place.last, rows.out(), &opts));
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// combine_into(rows, place, weight, Y, add)
PyObject* py_combine_into(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5 || p_combine_forward == nullptr) Py_RETURN_NONE;
  RowsArg rows(args[0]), y(args[3]), add(args[4], true);
  if (!rows.ok || !y.ok || !add.ok) Py_RETURN_NONE;
  const ListArg place(args[1], at::kInt, 2, rows.t.rows), weight(args[2], at::kFloat, 2, rows.t.rows);
  if (!place.ok || !weight.ok || place.last != weight.last || place.last * y.t.rows != rows.t.rows) Py_RETURN_NONE;
  const rl_opts_t opts = current_options();
  check(p_combine_forward(rows.in(), static_cast<const int32_t*>(place.p), static_cast<const float*>(weight.p), (int)place.last, add.in(), y.out(), &opts));
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// values_into(bytes, scales, out)
PyObject* py_values_into(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 3 || p_fp8_values == nullptr) Py_RETURN_NONE;
  RowsArg out(args[2]);
  if (!out.ok) Py_RETURN_NONE;
  const int64_t n = out.t.rows, blocks = (out.t.cols + 127) / 128;
  const ListArg q(args[0], at::kByte, 2, n * blocks * 128), s(args[1], at::kByte, 2, blocks * ((n + 15) / 16 * 16));
  if (!q.ok || !s.ok || q.last != blocks * 128) Py_RETURN_NONE;
  const rl_tensor_t tq{q.p, n, out.t.cols, blocks * 128, RL_FP8_R128, s.p, 128};
  const rl_opts_t opts = current_options();
  check(p_fp8_values(&tq, out.out(), &opts));
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"lora", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_lora)), METH_FASTCALL, "LoRA layer as a native autograd node, or None"},
                         {"vera", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_vera)), METH_FASTCALL, "VeRA layer as a native autograd node, or None"},
                         {"dora", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_dora)), METH_FASTCALL, "DoRA layer as a native autograd node, or None"},
                         {"experts", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_experts)), METH_FASTCALL, "layer over expert stacks or an 8-bit weight as a native autograd node, or None"},
                         {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_norm)), METH_FASTCALL, "root-mean-square norm as a native autograd node, or None"},
                         {"route", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_route)), METH_FASTCALL, "routing to experts as a native autograd node, or None"},
                         {"gather", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_gather)), METH_FASTCALL, "rows to the experts as a native autograd node, or None"},
                         {"combine", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_combine)), METH_FASTCALL, "the experts' rows back as a native autograd node, or None"},
                         {"norm_into", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_norm_into)), METH_FASTCALL, "runlora_rmsnorm_forward, or None"},
                         {"route_into", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_route_into)), METH_FASTCALL, "runlora_route_forward, or None"},
                         {"gather_into", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_gather_into)), METH_FASTCALL, "runlora_gather_forward, or None"},
                         {"combine_into", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_combine_into)), METH_FASTCALL, "runlora_combine_forward, or None"},
                         {"values_into", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_values_into)), METH_FASTCALL, "runlora_fp8_values, or None"},
                         {"init", py_init, METH_VARARGS, "hand over librunlora's entry points"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_autograd", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

// read by build.py without loading the library
[[gnu::used]] const char built_for[] = "built for [" RL_BUILT_FOR "]";

}  // namespace

PyMODINIT_FUNC PyInit__autograd(void) { return PyModule_Create(&module_def); }
