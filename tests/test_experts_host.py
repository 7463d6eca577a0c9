"""Refusals of the calls over 8-bit weights and stacks of expert weights: every error is reported before any HIP call (no GPU here)."""
import ctypes
import itertools

import numpy as np
import pytest

import experts_oracle as ref
from paper_2312_03415_amd import binding as rl

ADDRESS = itertools.count(0x100000000, 0x10000000)


def tensor(rows, cols, dtype=rl.RL_BF16):
    return rl.rl_tensor_t(next(ADDRESS), rows, cols, cols, dtype, None, 0)


def stack(experts, rows, cols, dtype=rl.RL_BF16):
    fp8 = dtype == rl.RL_FP8_B128
    return rl.rl_stack_t(next(ADDRESS), experts, rows, cols, cols, rows * cols, dtype, next(ADDRESS) if fp8 else None, 128 if fp8 else 0)


def args(n=64, experts=4, i=256, o=272, r=16, w=rl.RL_BF16):
    a = dict(X=tensor(n, i), ends=next(ADDRESS), W=stack(experts, i, o, w), A=stack(experts, i, r), B=stack(experts, r, o), Y=tensor(n, o),
             T=tensor(n, r), dY=tensor(n, o), dX=tensor(n, i), dA=stack(experts, i, r), dB=stack(experts, r, o))
    a["opts"] = rl.rl_opts_t(None, next(ADDRESS), 1 << 27)
    return a


def ref_of(x):
    return ctypes.byref(x) if x is not None else None


def forward(a):
    return rl.lib().runlora_experts_forward(ref_of(a["X"]), a["ends"], ref_of(a["W"]), ref_of(a["A"]), ref_of(a["B"]), ref_of(a["Y"]), ref_of(a["T"]), ref_of(a["opts"]))


def backward(a):
    return rl.lib().runlora_experts_backward(ref_of(a["dY"]), ref_of(a["X"]), a["ends"], ref_of(a["W"]), ref_of(a["A"]), ref_of(a["B"]), ref_of(a["T"]),
                                             ref_of(a["dX"]), ref_of(a["dA"]), ref_of(a["dB"]), ref_of(a["opts"]))


def set_field(a, name, field, value):
    setattr(a[name], field, value)


@pytest.mark.parametrize("name,field,value,code", [
    ("X", "data", None, rl.RL_ERR_NULL), ("W", "data", None, rl.RL_ERR_NULL), ("W", "scales", None, rl.RL_ERR_NULL), ("B", "data", None, rl.RL_ERR_NULL),
    ("X", "dtype", 42, rl.RL_ERR_DTYPE), ("X", "dtype", rl.RL_F32, rl.RL_ERR_DTYPE), ("A", "dtype", rl.RL_F16, rl.RL_ERR_DTYPE),
    ("W", "dtype", rl.RL_INT4_G64, rl.RL_ERR_DTYPE),
    ("X", "cols", 264, rl.RL_ERR_SHAPE), ("A", "rows", 264, rl.RL_ERR_SHAPE), ("B", "cols", 264, rl.RL_ERR_SHAPE), ("B", "experts", 3, rl.RL_ERR_SHAPE),
    ("W", "experts", 0, rl.RL_ERR_SHAPE), ("W", "ld", 256, rl.RL_ERR_SHAPE), ("A", "stride", -8, rl.RL_ERR_SHAPE),
    ("X", "ld", 260, rl.RL_ERR_ALIGN), ("W", "ld", 280, rl.RL_ERR_ALIGN), ("W", "stride", 69640, rl.RL_ERR_ALIGN), ("B", "stride", 4356, rl.RL_ERR_ALIGN),
    ("W", "group", 64, rl.RL_ERR_UNSUPPORTED), ("A", "ld", 1 << 23, rl.RL_ERR_UNSUPPORTED), ("W", "experts", 70000, rl.RL_ERR_UNSUPPORTED),
])
@pytest.mark.parametrize("call", [forward, backward])
def test_inputs_are_checked(call, name, field, value, code):
    a = args(w=rl.RL_FP8_B128)
    if name == "X" and field in ("dtype",) and call is backward:
        a["dY"].dtype = value          # (the type of a call is its first tensor's)
    if name == "X" and value == rl.RL_F32:
        a["dY"].dtype, code = value, rl.RL_ERR_UNSUPPORTED
    set_field(a, name, field, value)
    assert call(a) == code


def test_outputs_options_and_workspace_are_checked():
    a = args(); a["Y"].rows = 63
    assert forward(a) == rl.RL_ERR_SHAPE
    a = args(); a["T"].cols = 24
    assert forward(a) == rl.RL_ERR_SHAPE
    a = args(); a["A"] = None
    assert forward(a) == rl.RL_ERR_NULL                 # A and B come together
    a = args(); a["A"] = a["B"] = None
    assert forward(a) == rl.RL_ERR_SHAPE                # ... and without them there is no T
    a = args(); a["ends"] = None
    assert forward(a) == rl.RL_ERR_NULL and backward(a) == rl.RL_ERR_NULL
    a = args(); a["ends"] += 2
    assert forward(a) == rl.RL_ERR_ALIGN
    a = args(); a["opts"].dropout_p = 0.1
    assert forward(a) == rl.RL_ERR_UNSUPPORTED
    a = args(); a["opts"].bias = next(ADDRESS) + 8
    assert forward(a) == rl.RL_ERR_ALIGN
    a = args(); a["opts"].workspace_bytes = 16
    assert forward(a) == rl.RL_ERR_WORKSPACE and backward(a) == rl.RL_ERR_WORKSPACE
    a = args(); a["opts"].workspace += 16
    assert forward(a) == rl.RL_ERR_ALIGN and backward(a) == rl.RL_ERR_ALIGN
    a = args(); a["opts"] = None
    assert forward(a) == rl.RL_ERR_WORKSPACE
    a = args(); a["dA"].stride = 8
    assert backward(a) == rl.RL_ERR_SHAPE               # outputs of a stack may not overlap
    a = args(); a["X"] = None
    assert backward(a) == rl.RL_ERR_NULL                # dA needs X
    a = args(); a["dB"].rows = 24
    assert backward(a) == rl.RL_ERR_SHAPE


@pytest.mark.parametrize("out,into", [("Y", "X"), ("Y", "W"), ("Y", "A"), ("Y", "B"), ("T", "X"), ("T", "Y")])
def test_forward_outputs_may_not_overlap_inputs(out, into):
    a = args()
    a[out].data = a[into].data
    assert forward(a) == rl.RL_ERR_ALIAS


@pytest.mark.parametrize("out,into", [("dX", "dY"), ("dX", "W"), ("dA", "X"), ("dA", "A"), ("dB", "T"), ("dB", "dA"), ("dA", "dX")])
def test_backward_outputs_may_not_overlap(out, into):
    a = args()
    a[out].data = a[into].data
    assert backward(a) == rl.RL_ERR_ALIAS


def test_the_layer_call_on_an_8_bit_weight_is_checked():
    W = rl.rl_tensor_t(next(ADDRESS), 256, 272, 272, rl.RL_FP8_B128, next(ADDRESS), 128)
    X, A, B, Y = tensor(64, 256), tensor(256, 16), tensor(16, 272), tensor(64, 272)
    saved, opts = rl.rl_saved_t(), rl.rl_opts_t(None, next(ADDRESS), 1 << 27)
    call = lambda v, w=W, o=opts: rl.lib().runlora_forward(v, *(ctypes.byref(t) for t in (X, w, A, B, Y, saved, o)))
    assert call(rl.FWD2) == rl.RL_ERR_UNSUPPORTED and call(rl.FWD_DEFAULT) == rl.RL_ERR_UNSUPPORTED
    bad = rl.rl_tensor_t(W.data, 256, 272, 272, rl.RL_FP8_B128, W.scales, 64)
    assert call(rl.FWD1, bad) == rl.RL_ERR_UNSUPPORTED
    bad = rl.rl_tensor_t(W.data, 256, 272, 272, rl.RL_FP8_B128, None, 128)
    assert call(rl.FWD1, bad) == rl.RL_ERR_NULL
    assert call(rl.FWD1, W, rl.rl_opts_t(None, opts.workspace, 16)) == rl.RL_ERR_WORKSPACE
    assert call(rl.FWD1, W, rl.rl_opts_t(None, opts.workspace, 1 << 27, 0.0, None, 0.1, 3)) == rl.RL_ERR_UNSUPPORTED
    saved.fwd_variant, saved.dtype, saved.n, saved.i, saved.o, saved.r, saved.X, saved.ldx = rl.FWD1, rl.RL_BF16, 64, 256, 272, 16, X.data, 256
    back = lambda v: rl.lib().runlora_backward(v, *(ctypes.byref(t) for t in (Y, saved, W, A, B, tensor(64, 256), tensor(256, 16), tensor(16, 272), rl.rl_opts_t())))
    assert back(rl.BWD4) == rl.RL_ERR_UNSUPPORTED and back(rl.BWD_DEFAULT) == rl.RL_ERR_UNSUPPORTED
    assert back(rl.BWD1) == rl.RL_ERR_WORKSPACE
    saved.n = 65
    assert back(rl.BWD1) == rl.RL_ERR_SAVED_MISMATCH
    assert rl.runlora_select(64, 256, 272, 16, rl.RL_FP8_B128) == (1, 1)


def test_the_selector_keeps_an_8_bit_weight_on_its_pair(monkeypatch):
    monkeypatch.setenv("RUNLORA_FORCE_BWD", "4")
    with pytest.raises(rl.RunLoRAError) as e:
        rl.runlora_select(64, 256, 272, 16, rl.RL_FP8_B128)
    assert e.value.code == rl.RL_ERR_UNSUPPORTED


def test_the_quantiser_is_checked():
    src, dst = tensor(200, 272), rl.rl_tensor_t(next(ADDRESS), 200, 272, 272, rl.RL_FP8_B128, next(ADDRESS), 128)
    call = lambda s, d: rl.lib().runlora_fp8_quantize(ctypes.byref(s), ctypes.byref(d), None)
    for field, value, code in (("dtype", rl.RL_BF16, rl.RL_ERR_DTYPE), ("rows", 199, rl.RL_ERR_SHAPE), ("scales", None, rl.RL_ERR_NULL),
                               ("ld", 280, rl.RL_ERR_ALIGN), ("group", 64, rl.RL_ERR_UNSUPPORTED), ("data", src.data, rl.RL_ERR_ALIAS), ("scales", src.data, rl.RL_ERR_ALIAS)):
        d = rl.rl_tensor_t.from_buffer_copy(dst)
        setattr(d, field, value)
        assert call(src, d) == code, field
    src.dtype = rl.RL_INT4_G64
    assert call(src, dst) == rl.RL_ERR_DTYPE


def test_workspace_sizes():
    w = rl.runlora_experts_workspace_bytes
    assert w(False, 64, 4, 256, 272, 16, rl.RL_BF16) > 0 and w(True, 64, 4, 256, 272, 16, rl.RL_BF16, rl.RL_FP8_B128) > w(True, 64, 4, 256, 272, 16, rl.RL_BF16)
    for bad in ((0, 4, 256, 272, 16, rl.RL_BF16), (64, 0, 256, 272, 16, rl.RL_BF16), (64, 4, 252, 272, 16, rl.RL_BF16), (64, 4, 256, 272, 12, rl.RL_BF16),
                (64, 4, 256, 272, 16, rl.RL_F32)):
        assert w(False, *bad) == 0
    assert w(False, 64, 4, 264, 272, 16, rl.RL_BF16, rl.RL_FP8_B128) == 0       # 8-bit widths come in steps of 16
    assert rl.runlora_workspace_bytes(rl.FWD1, rl.BWD1, 64, 256, 272, 16, rl.RL_BF16, rl.RL_FP8_B128) > 0
    assert rl.runlora_workspace_bytes(rl.FWD2, -1, 64, 256, 272, 16, rl.RL_BF16, rl.RL_FP8_B128) == 0


def test_weight_holders_are_checked():
    torch = pytest.importorskip("torch")
    data, scales = torch.zeros((256, 272), dtype=torch.uint8), torch.zeros((2, 3), dtype=torch.uint8)
    assert rl.Fp8Weight(data, scales, 256, 272).shape == (256, 272)
    for d, s in ((data.float(), scales), (data, scales.t()), (data, scales[:1]), (data.t(), scales), (data[:200], scales)):
        with pytest.raises(ValueError):
            rl.Fp8Weight(d, s, 256, 272)
    with pytest.raises(ValueError):
        rl.stack_desc(rl.Fp8Weight(data, scales, 256, 272))
    with pytest.raises(ValueError):
        rl._ends(torch.zeros(4, dtype=torch.int64), 4)
    with pytest.raises(ValueError):
        rl._ends(torch.zeros(8, dtype=torch.int32)[::2], 4)


# ---- the reference itself ------------------------------------------------------------------------------------------

def test_reference_rounding_is_the_nearest_value():
    values = np.unique(np.abs(ref.e4m3_value(np.arange(256).astype(np.uint8))))
    values = values[np.isfinite(values)]
    assert values.max() == 448.0 and values[1] == 2.0 ** -9 and len(values) == 127
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(0, 448, 4000), 2.0 ** rng.uniform(-12, 8, 4000), (values[1:] + values[:-1]) / 2])
    q = ref.nearest_e4m3(x)
    gap = np.abs(values[None, :] - x[:, None])
    assert np.isin(q, values).all() and np.array_equal(np.abs(q - x), gap.min(axis=1))
    ties = (gap == gap.min(axis=1, keepdims=True)).sum(axis=1) == 2
    assert ties.sum() >= 126 and (np.searchsorted(values, q[ties]) % 2 == 0).all()      # to the even neighbour


@pytest.mark.parametrize("experts,counts", [(3, [4, 0, 5]), (2, [3, 3])])
def test_reference_gradients_against_differences(experts, counts):
    """Central differences of <Y, G> over X, A and B, without rounding (exact up to fp64: Y is at most quadratic in a step of one of them)."""
    rng = np.random.default_rng(2)
    n, i, o, r, s = sum(counts) + 2, 6, 5, 3, 0.7
    ends = np.cumsum(counts)
    X, G = rng.standard_normal((n, i)), rng.standard_normal((n, o))
    W, A, B = (rng.standard_normal((experts,) + shape) for shape in ((i, o), (i, r), (r, o)))
    f = lambda x, a, b: (ref.forward(x, ends, W, a, b, None, s, False)[0][0] * G).sum()
    grads = ref.backward(G, X, ends, W, A, B, s, False)[0]
    for k, (value, grad) in enumerate(zip((X, A, B), grads)):
        for idx in np.ndindex(value.shape):
            step = np.zeros(value.shape)
            step[idx] = 1e-3
            moved = [[X, A, B], [X, A, B]]
            moved[0][k], moved[1][k] = value + step, value - step
            assert abs((f(*moved[0]) - f(*moved[1])) / 2e-3 - grad[idx]) < 1e-8
