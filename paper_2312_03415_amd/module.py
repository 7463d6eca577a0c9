"""torch.autograd front end of the library: a LoRA linear layer whose forward and backward run in
the computation graphs runlora_select picks for its shape (arxiv 2312.03415, Section 2), and a
helper that swaps it in for the nn.Linear modules of a model (Section 3 applies RunLoRA to every
attention and MLP linear).

Nothing is computed here: tensors are flattened to [n, d] views, buffers are allocated with torch,
and every product runs inside the HIP library through binding.runlora_forward / runlora_backward.  Each
layer's node exists twice: in native code (csrc/autograd.cpp), which ordinary calls take, and in Python below,
for the calls that have to see a Python-level function (tracing, functorch transforms, tensor subclasses, modes).

    layer = RunLoRALinear.from_linear(nn_linear, r=16, alpha=32)     # W frozen, A and B trainable
    y = layer(x)                                                     # x [..., d_in] -> [..., d_out]
    wrap_linears(model, r=16, alpha=32, targets=("q_proj", "v_proj"))
    vera = RunVeRALinear(weight, A_shared, B_shared)                 # frozen A, B; trainable vectors d, b
    layer8 = RunLoRAFp8Linear.from_linear(nn_linear, r=16, alpha=32) # the frozen W in 8 bits
    experts = RunLoRAExperts(weight_stack, r=16, alpha=32)           # one adapted layer per expert
    y = experts(x_sorted, ends)                                      # rows sorted by expert, ends[e] = where expert e's rows end
    norm = RunRMSNorm(d); h, x = norm(y, x)                          # the norm of the residual stream x + y, and the stream
    weight, _, place, source, ends = RunRouter(8, 2)(h @ router)     # every token to its two best of eight experts
    y = RunCombineFunction.apply(experts(RunGatherFunction.apply(h, place, source), ends), place, source, weight, x)
"""
import ctypes
import functools
import math

import torch
from torch import nn
from torch.autograd.function import once_differentiable

from . import binding as rl


def _workspace(device, nbytes):
    """Scratch of one call, given back to the caching allocator behind it (stream-ordered like every tensor): calls on other
    streams or from other threads may run at the same time."""
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


_native_module = None


def _native():
    """The native autograd node (built with the library, no fallback if it is missing), with the library's entry points."""
    global _native_module
    if _native_module is None:
        lib = rl.lib()
        from . import build
        if not build._ext_is_current():  # (loading it against another torch would fail later, or worse)
            raise ImportError(f"_autograd.so was not built for {build._ext_abi()}: run `python -m paper_2312_03415_amd.build`")
        from . import _autograd
        address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
        entries = (lib.runlora_forward, lib.runlora_backward, lib.runlora_call_workspace_bytes, lib.runlora_vera_forward, lib.runlora_vera_backward,
                   lib.runlora_vera_workspace_bytes, lib.runlora_dora_forward, lib.runlora_dora_backward, lib.runlora_dora_workspace_bytes,
                   lib.runlora_experts_forward, lib.runlora_experts_backward, lib.runlora_experts_workspace_bytes, lib.runlora_fp8_forward, lib.runlora_fp8_values,
                   lib.runlora_rmsnorm_forward, lib.runlora_rmsnorm_backward, lib.runlora_rmsnorm_workspace_bytes,
                   lib.runlora_route_forward, lib.runlora_route_backward, lib.runlora_route_workspace_bytes,
                   lib.runlora_gather_forward, lib.runlora_gather_backward, lib.runlora_combine_forward, lib.runlora_combine_backward)
        _autograd.init(tuple(address(f) for f in entries), rl._check)
        _native_module = _autograd
    return _native_module


def _on_inputs_gpu(forward):
    """A Python node's forward, run on its input's GPU: what it launches goes to the current device's stream.  (Backwards are run on theirs by autograd.)"""
    @functools.wraps(forward)
    def run(ctx, x, *args):
        with torch.cuda.device_of(x):
            return forward(ctx, x, *args)
    return staticmethod(run)


def _rows(x, width):
    """x as a matrix [n, width] that the library can read."""
    x2 = x.reshape(-1, width)
    if x2.stride(-1) != 1 or x2.stride(0) % 8 != 0 or x2.stride(0) < width or x2.data_ptr() % 16 != 0:
        x2 = x2.clone(memory_format=torch.contiguous_format)  # (contiguous() would hand dense rows at an odd address back as they are)
    return x2


def _reread(saved, dy, x2, *others):
    """The forward's record for the input as autograd hands it back (and that input): a saved-tensor hook may have moved it or
    laid it out anew, so the pointer the forward recorded need not be x2's."""
    device = dy.get_device()
    for t in (x2, *others):
        if t.get_device() != device:
            raise ValueError(f"a saved tensor came back on another device: {t.device}, not {dy.device}")
    if x2.data_ptr() == saved.X and x2.stride() == (saved.ldx, 1) and x2.dtype == dy.dtype:
        return saved, x2  # as it was
    x2 = _rows(x2, saved.i)
    saved = type(saved).from_buffer_copy(saved)
    saved.X, saved.ldx, saved.dtype = x2.data_ptr(), x2.stride(0), rl.dtype_code(x2.dtype)
    return saved, x2


class RunLoRAFunction(torch.autograd.Function):
    """y = x W + bias + scale (x A) B with W and bias frozen; gradients for x, A and B (Eq. 1, Eq. 3).

    pair = (forward variant, backward variant) as runlora_select returns them; keep_merged lets
    forward2 hold W + scale AB for a merged backward (i*o elements kept until the backward ran), keep_t
    lets forward1 hold scale XA for the backwards that would form it again (n*r elements);
    dropout = (p, seed) or None: LoRA dropout on the adapter's input (mask defined in runlora.h; the
    backward regenerates it from the seed the forward recorded).
    """

    @classmethod
    def apply(cls, *args):
        if cls is RunLoRAFunction:
            y = _native().lora(*args)
            if y is not None:
                return y
        return super().apply(*args)

    @_on_inputs_gpu
    def forward(ctx, x, W, A, B, bias, scale, pair, keep_merged, dropout=None, keep_t=False):
        fwd, bwd = pair
        i, o = W.shape
        r = A.shape[1]
        x2 = _rows(x, i)
        n = x2.shape[0]
        code = rl.dtype_code(x.dtype)
        y = torch.empty((n, o), dtype=x.dtype, device=x.device)
        keeps_t = fwd == rl.FWD_DEFAULT or (keep_t and fwd in (rl.FWD1, rl.FWD3) and bwd in (1, 5, 6, 7))
        T = torch.empty((n, r), dtype=x.dtype, device=x.device) if keeps_t else None
        M = None
        if keep_merged and fwd == rl.FWD2 and bwd in rl.BWD_MERGED:
            M = torch.empty((i, o), dtype=x.dtype, device=x.device)
        saved = rl.new_saved(T, M)
        p, seed = dropout if dropout else (None, 0)
        ws = _workspace(x.device, rl.runlora_call_workspace_bytes(fwd, -1, n, i, o, r, code, keep_t=T is not None, keep_merged=M is not None, dropout=bool(p)))
        rl.runlora_forward(fwd, x2, W, A, B, y, saved, workspace=ws, scale=scale, bias=bias, dropout_p=p, dropout_seed=seed)
        ctx.saved = saved
        ctx.bwd = bwd
        ctx.keep = (T, M)          # buffers *saved points into
        ctx.x_shape = x.shape
        ctx.save_for_backward(x2, W, A, B)
        return y.view(*x.shape[:-1], o)

    @staticmethod
    def backward(ctx, dy):
        x2, W, A, B = ctx.saved_tensors
        saved, x2 = _reread(ctx.saved, dy, x2, W, A, B)
        i, o = W.shape
        r = A.shape[1]
        n = x2.shape[0]
        dy2 = _rows(dy, o)
        need_x, _, need_a, need_b = ctx.needs_input_grad[:4]
        dx = torch.empty((n, i), dtype=x2.dtype, device=x2.device) if need_x else None
        dA = torch.empty_like(A) if need_a else None
        dB = torch.empty_like(B) if need_b else None
        code = rl.dtype_code(dy.dtype)
        ws = _workspace(dy.device, rl.runlora_call_workspace_bytes(-1, ctx.bwd, n, i, o, r, code, keep_t=ctx.keep[0] is not None, keep_merged=ctx.keep[1] is not None,
                                                                   dropout=saved.dropout_thr != 0, dx=need_x, da=need_a, db=need_b))
        rl.runlora_backward(ctx.bwd, dy2, saved, W, A, B, dx, dA, dB, workspace=ws)
        if dx is not None:
            dx = dx.view(ctx.x_shape)
        return dx, None, dA, dB, None, None, None, None, None, None


class RunLoRALinear(nn.Module):
    """LoRA-augmented linear layer: frozen W [d_in, d_out] (the orientation of Eq. 1, Y = XW) and
    optional frozen bias, trainable A [d_in, r] and B [r, d_out], scale = alpha / r.

    The (forward, backward) pair is chosen per token count by runlora_select the first time that
    count is seen (criterion 2 when keep_merged, 3 when keep_t), or fixed with pair=(f, b).
    """

    def __init__(self, weight, r, alpha=None, bias=None, pair=None, keep_merged=False, dropout=0.0, keep_t=False):
        super().__init__()
        d_in, d_out = weight.shape
        self.d_in, self.d_out, self.r = d_in, d_out, r
        self.scale = 1.0 if alpha is None else float(alpha) / r
        self.weight = nn.Parameter(weight.contiguous(), requires_grad=False)
        self.bias = nn.Parameter(bias.contiguous(), requires_grad=False) if bias is not None else None
        # the usual LoRA start: A random, B zero, so that the layer starts as the frozen one
        self.lora_A = nn.Parameter(torch.randn(d_in, r, dtype=weight.dtype, device=weight.device) / math.sqrt(d_in))
        self.lora_B = nn.Parameter(torch.zeros(r, d_out, dtype=weight.dtype, device=weight.device))
        self.pair = pair
        self.keep_merged = keep_merged
        self.keep_t = keep_t
        self.dropout = float(dropout)  # LoRA dropout probability, applied in training mode only
        self.last_dropout_seed = None  # seed of the most recent training-mode forward (for reproducing its mask)
        self._pairs = {}

    @classmethod
    def from_linear(cls, linear, r, alpha=None, pair=None, keep_merged=False, dropout=0.0):
        """nn.Linear keeps its weight as [d_out, d_in]; the layer holds the transposed copy."""
        w = linear.weight.detach().t().contiguous()
        b = linear.bias.detach() if linear.bias is not None else None
        return cls(w, r, alpha, b, pair, keep_merged, dropout)

    def pair_for(self, n_tokens):
        if self.pair is not None:
            return self.pair
        p = self._pairs.get(n_tokens)
        if p is None:
            code = rl.dtype_code(self.weight.dtype)
            p = rl.runlora_select(n_tokens, self.d_in, self.d_out, self.r, code, criterion=2 if self.keep_merged else (3 if self.keep_t else None))
            self._pairs[n_tokens] = p
        return p

    def forward(self, x):
        n = x.numel() // self.d_in
        if self.training and self.dropout > 0.0:
            # with dropout only forward1 / backward1 (or the default chain) exist; a fresh seed per call
            # from torch's CPU generator, so that torch.manual_seed makes runs repeatable
            self.last_dropout_seed = int(torch.randint(0, 2 ** 31 - 1, (1,)).item())
            pair = self.pair if self.pair in ((0, 0), (0, 1), (1, 1)) else (1, 1)
            return RunLoRAFunction.apply(x, self.weight, self.lora_A, self.lora_B, self.bias, self.scale, pair, False,
                                         (self.dropout, self.last_dropout_seed), self.keep_t)
        return RunLoRAFunction.apply(x, self.weight, self.lora_A, self.lora_B, self.bias, self.scale,
                                     self.pair_for(n), self.keep_merged, None, self.keep_t)

    def extra_repr(self):
        return f"d_in={self.d_in}, d_out={self.d_out}, r={self.r}, scale={self.scale:g}, bias={self.bias is not None}"


class RunVeRAFunction(torch.autograd.Function):
    """y = x W + bias + scale ((x A) diag(d)) B diag(b) with W, bias, A and B frozen; gradients for x, d and b
    (runlora_vera_forward / runlora_vera_backward: the LoRA graphs on B~ = diag(d) B diag(b))."""

    @classmethod
    def apply(cls, *args):
        if cls is RunVeRAFunction:
            y = _native().vera(*args)
            if y is not None:
                return y
        return super().apply(*args)

    @_on_inputs_gpu
    def forward(ctx, x, W, A, B, d, b, bias, scale, pair):
        fwd, bwd = pair
        i, o = W.shape
        r = A.shape[1]
        x2 = _rows(x, i)
        n = x2.shape[0]
        code = rl.dtype_code(x.dtype)
        y = torch.empty((n, o), dtype=x.dtype, device=x.device)
        T = torch.empty((n, r), dtype=x.dtype, device=x.device) if fwd == rl.FWD_DEFAULT else None
        saved = rl.new_saved(T)
        ws = _workspace(x.device, rl.runlora_vera_workspace_bytes(fwd, -1, n, i, o, r, code))
        rl.runlora_vera_forward(fwd, x2, W, A, B, d, b, y, saved, ws, scale=scale, bias=bias)
        ctx.saved = saved
        ctx.bwd = bwd
        ctx.keep = T
        ctx.x_shape = x.shape
        ctx.save_for_backward(x2, W, A, B, d, b)
        return y.view(*x.shape[:-1], o)

    @staticmethod
    def backward(ctx, dy):
        x2, W, A, B, d, b = ctx.saved_tensors
        saved, x2 = _reread(ctx.saved, dy, x2, W, A, B, d, b)
        i, o = W.shape
        r = A.shape[1]
        n = x2.shape[0]
        dy2 = _rows(dy, o)
        need = ctx.needs_input_grad
        dx = torch.empty((n, i), dtype=x2.dtype, device=x2.device) if need[0] else None
        dd = torch.empty_like(d) if need[4] else None
        db = torch.empty_like(b) if need[5] else None
        code = rl.dtype_code(dy.dtype)
        ws = _workspace(dy.device, rl.runlora_vera_workspace_bytes(-1, ctx.bwd, n, i, o, r, code))
        rl.runlora_vera_backward(ctx.bwd, dy2, saved, W, A, B, d, b, dx, dd, db, ws)
        if dx is not None:
            dx = dx.view(ctx.x_shape)
        return dx, None, None, None, dd, db, None, None, None


class RunVeRALinear(nn.Module):
    """VeRA layer: frozen W [d_in, d_out] (+ bias) and frozen random A [d_in, r], B [r, d_out] (pass the
    same tensors to every layer to share them, as VeRA does), trainable vectors d [r] (start 0.1) and
    b [d_out] (start 0, so that the layer starts as the frozen one)."""

    def __init__(self, weight, A, B, bias=None, scale=1.0, pair=None, d_init=0.1):
        super().__init__()
        d_in, d_out = weight.shape
        r = A.shape[1]
        if A.shape != (d_in, r) or B.shape != (r, d_out):
            raise ValueError("A must be [d_in, r] and B [r, d_out]")
        self.d_in, self.d_out, self.r, self.scale, self.pair = d_in, d_out, r, float(scale), pair
        self.weight = nn.Parameter(weight.contiguous(), requires_grad=False)
        self.bias = nn.Parameter(bias.contiguous(), requires_grad=False) if bias is not None else None
        self.register_buffer("vera_A", A, persistent=False)
        self.register_buffer("vera_B", B, persistent=False)
        self.vera_d = nn.Parameter(torch.full((r,), d_init, dtype=weight.dtype, device=weight.device))
        self.vera_b = nn.Parameter(torch.zeros(d_out, dtype=weight.dtype, device=weight.device))
        self._pairs = {}

    def pair_for(self, n_tokens):
        if self.pair is not None:
            return self.pair
        p = self._pairs.get(n_tokens)
        if p is None:
            p = rl.runlora_select(n_tokens, self.d_in, self.d_out, self.r, rl.dtype_code(self.weight.dtype))
            self._pairs[n_tokens] = p
        return p

    def forward(self, x):
        return RunVeRAFunction.apply(x, self.weight, self.vera_A, self.vera_B, self.vera_d, self.vera_b, self.bias,
                                     self.scale, self.pair_for(x.numel() // self.d_in))

    def extra_repr(self):
        return f"d_in={self.d_in}, d_out={self.d_out}, r={self.r}, scale={self.scale:g}, bias={self.bias is not None}"


class RunDoRAFunction(torch.autograd.Function):
    """y = x ((W + scale A B) diag(m / c)) + bias, c the column norms of W + scale A B held constant in the backward
    pass; gradients for x, A, B and m (runlora_dora_forward / runlora_dora_backward: forward2 and one of the merged
    backward graphs, the merge kernel scaling W's columns on the way)."""

    @classmethod
    def apply(cls, *args):
        if cls is RunDoRAFunction:
            y = _native().dora(*args)
            if y is not None:
                return y
        return super().apply(*args)

    @_on_inputs_gpu
    def forward(ctx, x, W, A, B, m, bias, scale, bwd):
        i, o = W.shape
        r = A.shape[1]
        x2 = _rows(x, i)
        n = x2.shape[0]
        code = rl.dtype_code(x.dtype)
        y = torch.empty((n, o), dtype=x.dtype, device=x.device)
        c = torch.empty((o,), dtype=torch.float32, device=x.device)
        saved = rl.new_saved(None)
        ws = _workspace(x.device, rl.runlora_dora_workspace_bytes(rl.FWD2, -1, n, i, o, r, code))
        rl.runlora_dora_forward(rl.FWD2, x2, W, A, B, m, y, saved, c, ws, scale=scale, bias=bias)
        ctx.saved = saved
        ctx.bwd = bwd
        ctx.bias = bias
        ctx.x_shape = x.shape
        ctx.save_for_backward(x2, W, A, B, m, c, y)  # y is the tensor handed to the caller: no copy is kept
        return y.view(*x.shape[:-1], o)

    @staticmethod
    def backward(ctx, dy):
        x2, W, A, B, m, c, y = ctx.saved_tensors
        saved, x2 = _reread(ctx.saved, dy, x2, W, A, B, m, c, y)
        i, o = W.shape
        r = A.shape[1]
        n = x2.shape[0]
        dy2 = _rows(dy, o)
        need = ctx.needs_input_grad
        dx = torch.empty((n, i), dtype=x2.dtype, device=x2.device) if need[0] else None
        dA = torch.empty_like(A) if need[2] else None
        dB = torch.empty_like(B) if need[3] else None
        dm = torch.empty_like(m) if need[4] else None
        code = rl.dtype_code(dy.dtype)
        ws = _workspace(dy.device, rl.runlora_dora_workspace_bytes(-1, ctx.bwd, n, i, o, r, code))
        rl.runlora_dora_backward(ctx.bwd, dy2, saved, W, A, B, m, c, y, dx, dA, dB, dm, ws, bias=ctx.bias)
        if dx is not None:
            dx = dx.view(ctx.x_shape)
        return dx, None, dA, dB, dm, None, None, None


class RunDoRALinear(nn.Module):
    """DoRA layer: frozen W [d_in, d_out] (+ bias), trainable A [d_in, r], B [r, d_out] (B starts at 0) and
    magnitudes m [d_out], which start at the column norms of W so that the layer starts as the frozen one.
    16-bit dtypes, r <= 128.  bwd: the merged backward graph (4, 5, 7 or 8); None = the one of the four with the
    smallest modelled time for the token count of the call (the time model of runlora_select)."""

    def __init__(self, weight, r, alpha=None, bias=None, bwd=None):
        super().__init__()
        d_in, d_out = weight.shape
        self.d_in, self.d_out, self.r, self.bwd = d_in, d_out, r, bwd
        self.scale = float(alpha) / r if alpha is not None else 1.0
        self.weight = nn.Parameter(weight.contiguous(), requires_grad=False)
        self.bias = nn.Parameter(bias.contiguous(), requires_grad=False) if bias is not None else None
        self.lora_A = nn.Parameter(torch.randn(d_in, r, dtype=weight.dtype, device=weight.device) / math.sqrt(d_in))
        self.lora_B = nn.Parameter(torch.zeros(r, d_out, dtype=weight.dtype, device=weight.device))
        self.dora_m = nn.Parameter(weight.float().norm(dim=0).to(weight.dtype))
        self._bwds = {}

    @classmethod
    def from_linear(cls, linear, r, alpha=None, bwd=None):
        """nn.Linear keeps its weight as [d_out, d_in]; the layer holds the transposed copy."""
        w = linear.weight.detach().t().contiguous()
        b = linear.bias.detach() if linear.bias is not None else None
        return cls(w, r, alpha, b, bwd)

    def bwd_for(self, n_tokens):
        if self.bwd is not None:
            return self.bwd
        b = self._bwds.get(n_tokens)
        if b is None:
            code = rl.dtype_code(self.weight.dtype)
            b = min((4, 5, 7, 8), key=lambda v: rl.runlora_model_time_us(1, v, n_tokens, self.d_in, self.d_out, self.r, code))
            self._bwds[n_tokens] = b
        return b

    def forward(self, x):
        return RunDoRAFunction.apply(x, self.weight, self.lora_A, self.lora_B, self.dora_m, self.bias, self.scale,
                                     self.bwd_for(x.numel() // self.d_in))

    def extra_repr(self):
        return f"d_in={self.d_in}, d_out={self.d_out}, r={self.r}, scale={self.scale:g}, bias={self.bias is not None}"


def _w_code(W, code):
    return rl.RL_FP8_B128 if isinstance(W, rl.Fp8Weight) else code


class RunLoRAExpertsFunction(torch.autograd.Function):
    """y_t = x_t W_e + bias_e + scale (x_t A_e) B_e over rows sorted by expert (runlora_experts_forward / _backward); gradients for x, A and
    B.  W: [experts, d_in, d_out] or an Fp8Weight stack; A = B = None: no adapter.  scale XA (n*r elements) is kept for the backward."""

    @classmethod
    def apply(cls, x, ends, W, A, B, bias, scale):
        if cls is RunLoRAExpertsFunction:
            fp8 = isinstance(W, rl.Fp8Weight)
            if A is not None:
                y = _native().experts(x, A, B, W.data if fp8 else W, W.scales if fp8 else None, ends, bias, scale, W.shape[-1])
                if y is not None:
                    return y
        return super().apply(x, ends, W, A, B, bias, scale)

    @_on_inputs_gpu
    def forward(ctx, x, ends, W, A, B, bias, scale):
        E, i, o = W.shape
        x2 = _rows(x, i)
        n, r, code = x2.shape[0], 0 if A is None else A.shape[2], rl.dtype_code(x.dtype)
        y = torch.empty((n, o), dtype=x.dtype, device=x.device)
        T = torch.empty((n, r), dtype=x.dtype, device=x.device) if r else None
        if n > 0:
            ws = _workspace(x.device, rl.runlora_experts_workspace_bytes(False, n, E, i, o, r, code, _w_code(W, code)))
            rl.runlora_experts_forward(x2, ends, W, A, B, y, T, workspace=ws, scale=scale, bias=bias)
        fp8 = isinstance(W, rl.Fp8Weight)
        ctx.scale, ctx.x_shape, ctx.w_shape = scale, x.shape, (E, i, o)
        ctx.save_for_backward(x2, ends, A, B, T, W.data if fp8 else W, W.scales if fp8 else None)
        return y.view(*x.shape[:-1], o)

    @staticmethod
    def backward(ctx, dy):
        x2, ends, A, B, T, W, scales = ctx.saved_tensors
        E, i, o = ctx.w_shape
        if scales is not None:
            W = rl.Fp8Weight(W, scales, i, o)
        n, r = x2.shape[0], 0 if A is None else A.shape[2]
        dy2, x2 = _rows(dy, o), _rows(x2, i)
        need = ctx.needs_input_grad
        dx = torch.empty((n, i), dtype=x2.dtype, device=x2.device) if need[0] else None
        make = torch.empty if n > 0 else torch.zeros
        dA = make(A.shape, dtype=A.dtype, device=A.device) if need[3] else None
        dB = make(B.shape, dtype=B.dtype, device=B.device) if need[4] else None
        if n > 0:
            for t in ctx.saved_tensors:
                if t is not None and t.device != dy.device:
                    raise ValueError(f"a saved tensor came back on another device: {t.device}, not {dy.device}")
            code = rl.dtype_code(dy.dtype)
            ws = _workspace(dy.device, rl.runlora_experts_workspace_bytes(True, n, E, i, o, r, code, _w_code(W, code)))
            rl.runlora_experts_backward(dy2, x2, ends, W, A, B, dx, dA, dB, T, workspace=ws, scale=ctx.scale)
        return dx.view(ctx.x_shape) if need[0] else None, None, None, dA, dB, None, None


class RunLoRAFp8Function(torch.autograd.Function):
    """y = Q(x) W + bias + scale (x A) B over an Fp8Weight (runlora.h); gradients for x, A and B, the large product of dx on Q(dy).
    scale XA (n*r elements) is kept for the backward.  rows: Q(x) where it is there already (an Fp8Rows, e.g. RunRMSNorm's)."""

    @classmethod
    def apply(cls, x, W, A, B, bias, scale, rows=None):
        if cls is RunLoRAFp8Function and isinstance(W, rl.Fp8Weight) and (rows is None or rows.cols == W.rows):
            y = _native().experts(x, A, B, W.data, W.scales, None, bias, scale, W.cols, *(() if rows is None else (rows.data, rows.scales)))
            if y is not None:
                return y
        return super().apply(x, W, A, B, bias, scale, rows)

    @_on_inputs_gpu
    def forward(ctx, x, W, A, B, bias, scale, rows=None):
        x2 = _rows(x, W.rows)
        n, r, code = x2.shape[0], A.shape[1], rl.dtype_code(x.dtype)
        y = torch.empty((n, W.cols), dtype=x.dtype, device=x.device)
        T = torch.empty((n, r), dtype=x.dtype, device=x.device)
        ctx.saved, ctx.w_shape, ctx.x_shape = rl.new_saved(T), W.shape, x.shape
        if n > 0:
            ws = _workspace(x.device, rl.runlora_workspace_bytes(rl.FWD1, -1, n, W.rows, W.cols, r, code, rl.RL_FP8_B128))
            if rows is None:
                rl.runlora_forward(rl.FWD1, x2, W, A, B, y, ctx.saved, workspace=ws, scale=scale, bias=bias)
            else:
                rl.runlora_fp8_forward(x2, rows, W, A, B, y, ctx.saved, workspace=ws, scale=scale, bias=bias)
        ctx.save_for_backward(x2, A, B, T, W.data, W.scales)
        return y.view(*x.shape[:-1], W.cols)

    @staticmethod
    def backward(ctx, dy):
        x2, A, B, T, data, scales = ctx.saved_tensors
        (i, o), n, r = ctx.w_shape, x2.shape[0], A.shape[1]
        W = rl.Fp8Weight(data, scales, i, o)
        dy2 = _rows(dy, o)
        need_x, _, need_a, need_b = ctx.needs_input_grad[:4]
        dx = torch.empty((n, i), dtype=x2.dtype, device=x2.device) if need_x else None
        make = torch.empty if n > 0 else torch.zeros
        dA = make(A.shape, dtype=A.dtype, device=A.device) if need_a else None
        dB = make(B.shape, dtype=B.dtype, device=B.device) if need_b else None
        if n > 0:
            saved, x2 = _reread(ctx.saved, dy2, x2, A, B, T, data, scales)
            if tuple(T.shape) != (n, r) or T.dtype != x2.dtype or T.stride(1) != 1:
                raise ValueError("scale XA came back from the saved tensors as another matrix")
            if saved.T != T.data_ptr() or saved.ldt != T.stride(0):
                saved = type(saved).from_buffer_copy(saved)
                saved.T, saved.ldt = T.data_ptr(), T.stride(0)
            code = rl.dtype_code(dy.dtype)
            ws = _workspace(dy.device, rl.runlora_workspace_bytes(-1, rl.BWD1, n, i, o, r, code, rl.RL_FP8_B128))
            rl.runlora_backward(rl.BWD1, dy2, saved, W, A, B, dx, dA, dB, workspace=ws)
        return dx.view(ctx.x_shape) if need_x else None, None, dA, dB, None, None, None


def _bytes_of_state(module, state, prefix, *_):
    for name in ("weight_data", "weight_scales"):
        t = state.get(prefix + name)
        if isinstance(t, torch.Tensor) and t.element_size() == 1:
            state[prefix + name] = t.view(torch.uint8)


def _register_bytes(module, weight):
    """An Fp8Weight as a module's buffers.  They hold whole numbers: converting a module converts its floating-point tensors, 8-bit ones among
    them; a state that holds them as such is read as bytes."""
    module.register_buffer("weight_data", weight.data.view(torch.uint8))
    module.register_buffer("weight_scales", weight.scales.view(torch.uint8))
    module.register_load_state_dict_pre_hook(_bytes_of_state)


class RunLoRAFp8Linear(nn.Module):
    """LoRA-augmented linear layer over a frozen weight kept in 8 bits (binding.Fp8Weight); otherwise as RunLoRALinear."""

    def __init__(self, weight, r, alpha=None, bias=None, dtype=torch.bfloat16):
        super().__init__()
        (self.d_in, self.d_out), self.r = weight.shape, r
        self.scale = 1.0 if alpha is None else float(alpha) / r
        device = weight.data.device
        _register_bytes(self, weight)
        self.bias = nn.Parameter(bias.contiguous(), requires_grad=False) if bias is not None else None
        self.lora_A = nn.Parameter(torch.randn(self.d_in, r, dtype=dtype, device=device) / math.sqrt(self.d_in))
        self.lora_B = nn.Parameter(torch.zeros(r, self.d_out, dtype=dtype, device=device))

    @classmethod
    def from_linear(cls, linear, r, alpha=None):
        """nn.Linear keeps its weight as [d_out, d_in]; the layer holds the transposed copy, rounded."""
        b = linear.bias.detach() if linear.bias is not None else None
        return cls(rl.Fp8Weight.quantize(linear.weight.detach().t().contiguous()), r, alpha, b, linear.weight.dtype)

    @property
    def weight(self):
        return rl.Fp8Weight(self.weight_data, self.weight_scales, self.d_in, self.d_out)

    def forward(self, x, rows=None):
        """rows: x's rows in 8 bits, where the operator in front has left them (RunRMSNorm)."""
        return RunLoRAFp8Function.apply(x, self.weight, self.lora_A, self.lora_B, self.bias, self.scale, rows)

    def extra_repr(self):
        return f"d_in={self.d_in}, d_out={self.d_out}, r={self.r}, scale={self.scale:g}, bias={self.bias is not None}"


class RunLoRAExperts(nn.Module):
    """One adapted linear layer per expert, on rows sorted by expert: frozen weight [experts, d_in, d_out] (a tensor or an Fp8Weight stack) and
    bias [experts, d_out], trainable A [experts, d_in, r] and B [experts, r, d_out]; layer(x [n, d_in], ends), ends (int32, on the
    device) = where each expert's rows end, e.g. torch.bincount(expert_of_row, minlength=experts).cumsum(0, dtype=torch.int32).
    The adapters have the weight's type, over an 8-bit weight `dtype` (bfloat16 if not given)."""

    def __init__(self, weight, r, alpha=None, bias=None, dtype=None):
        super().__init__()
        self.experts, self.d_in, self.d_out = weight.shape
        self.r, self.scale = r, 1.0 if alpha is None else float(alpha) / r
        self.fp8 = isinstance(weight, rl.Fp8Weight)
        if self.fp8:
            _register_bytes(self, weight)
            device, dtype = weight.data.device, dtype or torch.bfloat16
        else:
            self.weight = nn.Parameter(weight.contiguous(), requires_grad=False)
            device, dtype = weight.device, weight.dtype
        self.bias = nn.Parameter(bias.contiguous(), requires_grad=False) if bias is not None else None
        self.lora_A = nn.Parameter(torch.randn(self.experts, self.d_in, r, dtype=dtype, device=device) / math.sqrt(self.d_in))
        self.lora_B = nn.Parameter(torch.zeros(self.experts, r, self.d_out, dtype=dtype, device=device))

    def forward(self, x, ends):
        W = rl.Fp8Weight(self.weight_data, self.weight_scales, self.d_in, self.d_out) if self.fp8 else self.weight
        return RunLoRAExpertsFunction.apply(x, ends, W, self.lora_A, self.lora_B, self.bias, self.scale)

    def extra_repr(self):
        return f"experts={self.experts}, d_in={self.d_in}, d_out={self.d_out}, r={self.r}, scale={self.scale:g}, bias={self.bias is not None}"


class RunRMSNormFunction(torch.autograd.Function):
    """y = h / sqrt(mean h^2 + eps) * gain over the last dimension (runlora_rmsnorm_forward / _backward); without a residual h = x and y is returned, with
    one h = x + residual and (y, h) are.  rows=True appends y's rows in 8 bits: the bytes and scales of an Fp8Rows.  Gradients for x, residual and gain."""

    @classmethod
    def apply(cls, x, gain, eps, residual=None, rows=False):
        if cls is RunRMSNormFunction:
            out = _native().norm(x, gain, eps, residual, rows)
            if out is not None:
                return out if len(out) > 1 else out[0]
        return super().apply(x, gain, eps, residual, rows)

    @_on_inputs_gpu
    def forward(ctx, x, gain, eps, residual=None, rows=False):
        d = x.shape[-1]
        x2 = _rows(x, d)
        n = x2.shape[0]
        if residual is not None and (residual.shape != x.shape or residual.dtype != x.dtype):
            raise ValueError("the residual must have x's shape and type")
        r2 = None if residual is None else _rows(residual, d)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        h = x2 if residual is None else torch.empty_like(y)
        rstd = torch.empty((n,), dtype=torch.float32, device=x.device)
        q = rl.Fp8Rows.empty(n, d, x.device) if rows else None
        if n > 0:
            rl.runlora_rmsnorm_forward(x2, gain, y.view(n, d), eps, r2, None if residual is None else h.view(n, d), rstd, q)
        ctx.x_shape, ctx.residual = x.shape, residual is not None
        ctx.save_for_backward(h, gain, rstd)
        ctx.set_materialize_grads(False)
        out = (y,) if residual is None else (y, h)
        if rows:
            ctx.mark_non_differentiable(q.data, q.scales)
            out += (q.data, q.scales)
        return out if len(out) > 1 else out[0]

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh=None, *_):
        h, gain, rstd = ctx.saved_tensors
        if not ctx.residual:
            dh = None
        if dy is None:
            return (dh if ctx.needs_input_grad[0] else None), None, None, (dh if ctx.needs_input_grad[3] else None), None
        d = h.shape[-1]
        h2, dy2 = _rows(h, d), _rows(dy, d)
        n = h2.shape[0]
        need_x, need_gain = ctx.needs_input_grad[0] or ctx.needs_input_grad[3], ctx.needs_input_grad[1]
        make = torch.empty if n > 0 else torch.zeros
        dx = torch.empty((n, d), dtype=h2.dtype, device=h2.device) if need_x else None
        dgain = make((d,), dtype=h2.dtype, device=h2.device) if need_gain else None
        if n > 0 and (need_x or need_gain):
            ws = _workspace(dy.device, rl.runlora_rmsnorm_workspace_bytes(n, d, rl.dtype_code(h2.dtype))) if need_gain else None
            rl.runlora_rmsnorm_backward(dy2, h2, gain, rstd, dx, dgain, None if dh is None else _rows(dh, d), ws)
        dx = dx.view(ctx.x_shape) if need_x else None
        return (dx if ctx.needs_input_grad[0] else None), dgain, None, (dx if ctx.needs_input_grad[3] else None), None


class RunRMSNorm(nn.Module):
    """Root-mean-square norm of the last dimension with a gain [d]: norm(x) = y, norm(x, residual) = (y, x + residual).  rows=True appends y's rows in 8 bits
    (binding.Fp8Rows), which a RunLoRAFp8Linear takes next to y."""

    def __init__(self, d, eps=1e-6, dtype=torch.bfloat16, device="cuda", trainable=False):
        super().__init__()
        self.d, self.eps = d, float(eps)
        self.weight = nn.Parameter(torch.ones(d, dtype=dtype, device=device), requires_grad=trainable)

    def forward(self, x, residual=None, rows=False):
        out = RunRMSNormFunction.apply(x, self.weight, self.eps, residual, rows)
        if not rows:
            return out
        *tensors, data, scales = out
        return (*tensors, rl.Fp8Rows(data, scales, x.numel() // self.d, self.d))

    def extra_repr(self):
        return f"{self.d}, eps={self.eps:g}"


class RunRouteFunction(torch.autograd.Function):
    """(weight, expert, place, source, ends) of logits [n, experts] (runlora_route_forward / _backward); gradient of the weights for the logits."""

    @classmethod
    def apply(cls, logits, route, bias=None):
        if cls is RunRouteFunction:
            out = _native().route(logits, bias, route.how, route.scale)
            if out is not None:
                return out
        return super().apply(logits, route, bias)

    @_on_inputs_gpu
    def forward(ctx, logits, route, bias=None):
        l2 = logits if logits.dim() == 2 and (logits.shape[1] < 2 or logits.stride(1) == 1) and logits.stride(0) >= logits.shape[1] else logits.contiguous()
        n, top = l2.shape[0], route.top
        make = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=l2.device)
        weight, expert, place = make((n, top), torch.float32), make((n, top), torch.int32), make((n, top), torch.int32)
        source, ends = make((n * top,), torch.int32), make((route.experts,), torch.int32)
        if n > 0:
            ws = _workspace(l2.device, rl.runlora_route_workspace_bytes(n, route.experts, top))
            rl.runlora_route_forward(l2, route, weight, expert, place, source, ends, bias, ws)
        else:
            ends.zero_()
        ctx.route, ctx.bias = route, bias  # (the backward asks whether there is a bias and reads none of it: it may be updated in place before that)
        ctx.save_for_backward(l2, expert)
        ctx.mark_non_differentiable(expert, place, source, ends)
        ctx.set_materialize_grads(False)
        return weight, expert, place, source, ends

    @staticmethod
    @once_differentiable
    def backward(ctx, dweight, *_):
        if dweight is None:
            return None, None, None
        logits, expert = ctx.saved_tensors
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        if logits.shape[0] > 0:
            rl.runlora_route_backward(logits, ctx.route, expert, dweight.contiguous(), dlogits, ctx.bias)
        return dlogits, None, None


class RunRouter(nn.Module):
    """Routing of tokens by logits [n, experts] to `top` experts each: router(logits) = (weight, expert, place, source, ends), what RunGatherFunction,
    RunLoRAExperts and RunCombineFunction read.  balance=True: a bias [experts] (float32, a buffer that starts at 0) is added to the scores for the choice
    alone.  Options as binding.Route."""

    def __init__(self, experts, top, score="softmax", renormalise=True, groups=1, groups_kept=None, group_top=1, scale=1.0, balance=False, device="cuda"):
        super().__init__()
        self.route = rl.Route(experts, top, score, renormalise, groups, groups_kept, group_top, scale)
        self.register_buffer("bias", torch.zeros(experts, dtype=torch.float32, device=device) if balance else None)

    def forward(self, logits):
        return RunRouteFunction.apply(logits, self.route, None if self.bias is None else self.bias.float())

    def extra_repr(self):
        r = self.route
        return f"experts={r.experts}, top={r.top}, score={r.score}, renormalise={r.renormalise}, groups={r.groups}, scale={r.scale:g}"


class RunGatherFunction(torch.autograd.Function):
    """rows [n top, d] sorted by expert from x [n, d] (runlora_gather_forward / _backward); place and source as RunRouteFunction gives them."""

    @classmethod
    def apply(cls, x, place, source):
        if cls is RunGatherFunction:
            rows = _native().gather(x, place, source)
            if rows is not None:
                return rows
        return super().apply(x, place, source)

    @_on_inputs_gpu
    def forward(ctx, x, place, source):
        x2 = _rows(x, x.shape[-1])
        n, d = x2.shape
        rows = torch.empty((n * place.shape[1], d), dtype=x.dtype, device=x.device)
        if n > 0:
            rl.runlora_gather_forward(x2, place, source, rows)
        ctx.x_shape = x.shape
        ctx.save_for_backward(place)
        return rows

    @staticmethod
    @once_differentiable
    def backward(ctx, drows):
        place, = ctx.saved_tensors
        d = ctx.x_shape[-1]
        dx = torch.empty((place.shape[0], d), dtype=drows.dtype, device=drows.device)
        if place.shape[0] > 0:
            rl.runlora_gather_backward(_rows(drows, d), place, dx)
        return dx.view(ctx.x_shape), None, None


class RunCombineFunction(torch.autograd.Function):
    """y_t = add_t + sum over j of weight[t, j] rows[place[t, j]] (runlora_combine_forward / _backward); gradients for rows, weight and add."""

    @classmethod
    def apply(cls, rows, place, source, weight, add=None):
        if cls is RunCombineFunction:
            y = _native().combine(rows, place, source, weight, add)
            if y is not None:
                return y
        return super().apply(rows, place, source, weight, add)

    @_on_inputs_gpu
    def forward(ctx, rows, place, source, weight, add=None):
        r2 = _rows(rows, rows.shape[-1])
        n, d = place.shape[0], r2.shape[1]
        if add is not None and (add.shape[-1] != d or add.dtype != rows.dtype or add.numel() != n * d):
            raise ValueError("add must have one row a token, of the rows' type")
        y = torch.empty((n, d) if add is None else add.shape, dtype=rows.dtype, device=rows.device)
        weight = weight.contiguous()
        if n > 0:
            rl.runlora_combine_forward(r2, place, weight, y.view(n, d), None if add is None else _rows(add, d))
        ctx.save_for_backward(r2, place, source, weight)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        rows, place, source, weight = ctx.saved_tensors
        need = ctx.needs_input_grad
        d = rows.shape[1]
        dy2 = _rows(dy, d)
        drows = torch.empty((place.numel(), d), dtype=rows.dtype, device=rows.device) if need[0] else None
        dweight = torch.empty_like(weight) if need[3] else None
        if place.shape[0] > 0 and (need[0] or need[3]):
            rl.runlora_combine_backward(dy2, _rows(rows, d), place, source, weight, drows, dweight)
        return drows, None, None, dweight, (dy if need[4] else None)


def wrap_linears(model, r, alpha=None, targets=None, pair=None, keep_merged=False, dropout=0.0, adapter="lora"):
    """Replace nn.Linear submodules of `model` by RunLoRALinear, or by RunDoRALinear with adapter="dora" (all of
    them, or those whose attribute name is in `targets`); every other parameter of the model is frozen.
    Returns the replaced names."""
    if adapter not in ("lora", "dora"):
        raise ValueError("adapter must be 'lora' or 'dora'")
    if adapter == "dora" and (pair is not None or keep_merged or dropout):
        raise ValueError("the DoRA layer takes none of pair / keep_merged / dropout")
    replaced = []
    for name, module in list(model.named_modules()):
        for child_name, child in list(module.named_children()):
            if isinstance(child, nn.Linear) and (targets is None or child_name in targets):
                new = (RunDoRALinear.from_linear(child, r, alpha) if adapter == "dora"
                       else RunLoRALinear.from_linear(child, r, alpha, pair, keep_merged, dropout))
                setattr(module, child_name, new)
                replaced.append(f"{name}.{child_name}" if name else child_name)
    for pname, p in model.named_parameters():
        if not (pname.endswith("lora_A") or pname.endswith("lora_B") or pname.endswith("dora_m")):
            p.requires_grad_(False)
    return replaced
