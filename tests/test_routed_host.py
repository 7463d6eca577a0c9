"""Refusals of the calls that stand between the layers of a block with routed experts: every error is reported before any HIP call (no GPU here)."""
import ctypes
import itertools

import pytest

from paper_2312_03415_amd import binding as rl

ADDRESS = itertools.count(0x100000000, 0x10000000)
N, E, TOP, D = 100, 24, 4, 264


def tensor(rows, cols, dtype=rl.RL_BF16):
    return rl.rl_tensor_t(next(ADDRESS), rows, cols, cols, dtype, None, 0)


def rounded(rows, cols):
    return rl.rl_tensor_t(next(ADDRESS), rows, cols, (cols + 127) // 128 * 128, rl.RL_FP8_R128, next(ADDRESS), 128)


def opts():
    return rl.rl_opts_t(None, next(ADDRESS), 1 << 27)


def ref(x):
    return ctypes.byref(x) if isinstance(x, ctypes.Structure) else x


def route_args():
    return dict(logits=tensor(N, E, rl.RL_F32), route=rl.rl_route_t(E, TOP, 0, 1, 4, 2, 2, 1.0, next(ADDRESS)), expert=next(ADDRESS), weight=next(ADDRESS),
                place=next(ADDRESS), source=next(ADDRESS), ends=next(ADDRESS), opts=opts(), dweight=next(ADDRESS), dlogits=tensor(N, E, rl.RL_F32))


def route_forward(a):
    return rl.lib().runlora_route_forward(*(ref(a[k]) for k in ("logits", "route", "expert", "weight", "place", "source", "ends", "opts")))


def route_backward(a):
    return rl.lib().runlora_route_backward(*(ref(a[k]) for k in ("logits", "route", "expert", "dweight", "dlogits", "opts")))


def rows_args(dtype=rl.RL_BF16):
    return dict(X=tensor(N, D, dtype), rows=tensor(N * TOP, D, dtype), drows=tensor(N * TOP, D, dtype), add=tensor(N, D, dtype), Y=tensor(N, D, dtype),
                dY=tensor(N, D, dtype), place=next(ADDRESS), source=next(ADDRESS), weight=next(ADDRESS), dweight=next(ADDRESS), top=TOP, opts=opts())


def gather_forward(a):
    return rl.lib().runlora_gather_forward(*(ref(a[k]) for k in ("X", "place", "source", "top", "rows", "opts")))


def gather_backward(a):
    return rl.lib().runlora_gather_backward(*(ref(a[k]) for k in ("rows", "place", "top", "X", "opts")))


def combine_forward(a):
    return rl.lib().runlora_combine_forward(*(ref(a[k]) for k in ("rows", "place", "weight", "top", "add", "X", "opts")))


def combine_backward(a):
    return rl.lib().runlora_combine_backward(*(ref(a[k]) for k in ("X", "rows", "place", "source", "weight", "top", "drows", "dweight", "opts")))


def norm_args(dtype=rl.RL_BF16):
    return dict(X=tensor(N, D, dtype), R=tensor(N, D, dtype), gain=next(ADDRESS), eps=1e-6, Y=tensor(N, D, dtype), H=tensor(N, D, dtype), rstd=next(ADDRESS),
                Q=rounded(N, D), dH=tensor(N, D, dtype), dX=tensor(N, D, dtype), dgain=next(ADDRESS), opts=opts())


def norm_forward(a):
    return rl.lib().runlora_rmsnorm_forward(*(ref(a[k]) for k in ("X", "R", "gain", "eps", "Y", "H", "rstd", "Q", "opts")))


def norm_backward(a):
    return rl.lib().runlora_rmsnorm_backward(*(ref(a[k]) for k in ("X", "dH", "H", "gain", "rstd", "dX", "dgain", "opts")))


def change(a, path, value):
    if "." in path:
        name, field = path.split(".")
        setattr(a[name], field, value)
    else:
        a[path] = value


NULL, SHAPE, DTYPE, VARIANT, ALIGN, UNSUPPORTED = rl.RL_ERR_NULL, rl.RL_ERR_SHAPE, rl.RL_ERR_DTYPE, rl.RL_ERR_VARIANT, rl.RL_ERR_ALIGN, rl.RL_ERR_UNSUPPORTED


@pytest.mark.parametrize("path,value,code", [
    ("logits", None, NULL), ("route", None, NULL), ("logits.data", None, NULL), ("expert", None, NULL),
    ("logits.dtype", rl.RL_FP8_B128, DTYPE), ("logits.dtype", 42, DTYPE), ("logits.rows", 0, SHAPE), ("logits.cols", E + 1, SHAPE), ("logits.ld", E - 1, SHAPE),
    ("logits.data", 0x100000002, ALIGN), ("logits.rows", 1 << 23, UNSUPPORTED), ("logits.ld", (1 << 31) + 1, UNSUPPORTED),
    ("route.top", 0, SHAPE), ("route.top", E + 1, SHAPE), ("route.score", 2, VARIANT), ("route.score", -1, VARIANT), ("route.groups", 5, SHAPE),
    ("route.groups", -1, SHAPE), ("route.groups_kept", 5, SHAPE), ("route.groups_kept", -1, SHAPE), ("route.group_top", 3, UNSUPPORTED),
    ("route.group_top", -1, SHAPE), ("route.experts", 0, SHAPE), ("route.bias", 0x100000001, ALIGN), ("expert", 0x100000001, ALIGN)])
@pytest.mark.parametrize("call", [route_forward, route_backward])
def test_routing_is_checked(call, path, value, code):
    a = route_args()
    change(a, path, value)
    assert call(a) == code


def test_routing_limits():
    for call in (route_forward, route_backward):
        for experts, top, groups in ((1025, 4, 1), (2000, 65, 1), (520, 65, 1), (650, 4, 65)):
            a = route_args()
            a["logits"], a["dlogits"], a["route"] = tensor(N, experts, rl.RL_F32), tensor(N, experts, rl.RL_F32), rl.rl_route_t(experts, top, 0, 1, groups, 1, 1, 1.0, None)
            assert call(a) == UNSUPPORTED
    for name in ("weight", "place", "source", "ends"):
        a = route_args()
        a[name] = None
        assert route_forward(a) == NULL
    a = route_args()
    a["dweight"] = None
    assert route_backward(a) == NULL
    a = route_args()
    a["dlogits"].dtype = rl.RL_BF16
    assert route_backward(a) == DTYPE
    a = route_args()
    a["dlogits"].rows = N + 1
    assert route_backward(a) == SHAPE


def test_routing_outputs_may_not_overlap():
    base = route_args()
    for out in ("expert", "weight", "place", "source", "ends"):
        for other, at in (("logits", base["logits"].data + N * E * 4 - 4), ("bias", base["route"].bias + 4)) + tuple(
                (o, base[o] + 4) for o in ("expert", "weight", "place", "source", "ends") if o != out):
            a = dict(base)
            a[out] = at
            assert route_forward(a) == rl.RL_ERR_ALIAS, (out, other)
    for at in (base["logits"].data, base["expert"], base["dweight"]):
        a = route_args()
        for k in ("logits", "expert", "dweight", "route"):
            a[k] = base[k]
        a["dlogits"].data = at
        assert route_backward(a) == rl.RL_ERR_ALIAS


def test_routing_workspace():
    need = rl.runlora_route_workspace_bytes(10000, E, TOP)
    assert need > 0 and rl.runlora_route_workspace_bytes(4, E, TOP) == 0
    for bad in ((0, E, TOP), (1 << 23, E, TOP), (10, 0, 1), (10, 1025, 1), (10, 8, 0), (10, 8, 9), (10, 200, 65)):
        assert rl.runlora_route_workspace_bytes(*bad) == 0
    a = route_args()
    a["logits"] = tensor(10000, E, rl.RL_F32)
    for space in (rl.rl_opts_t(None, next(ADDRESS), need - 1), rl.rl_opts_t(None, None, 1 << 20), None):
        a["opts"] = space
        assert route_forward(a) == rl.RL_ERR_WORKSPACE
    assert str(need) in rl.lib().runlora_last_hip_error().decode()
    a["opts"] = rl.rl_opts_t(None, next(ADDRESS) + 64, 1 << 20)
    assert route_forward(a) == ALIGN
    # the need does not fall as the tokens grow in number up to the largest call
    sizes = [rl.runlora_route_workspace_bytes(n, E, TOP) for n in (2000, 10 ** 5, 10 ** 6, (1 << 23) - 1)]
    assert sizes == sorted(sizes) and sizes[-1] <= 512 * E * 2


@pytest.mark.parametrize("call", [gather_forward, gather_backward, combine_forward, combine_backward])
@pytest.mark.parametrize("path,value,code", [
    ("X", None, NULL), ("X.data", None, NULL), ("rows.data", None, NULL), ("place", None, NULL), ("X.dtype", 42, DTYPE), ("X.dtype", rl.RL_FP8_B128, DTYPE),
    ("rows.dtype", rl.RL_F16, DTYPE), ("X.rows", 0, SHAPE), ("X.cols", 260, ALIGN), ("X.ld", D - 8, SHAPE), ("X.ld", D + 4, ALIGN), ("rows.rows", N * TOP + 1, SHAPE),
    ("rows.cols", D + 8, SHAPE), ("top", 0, SHAPE), ("top", -3, SHAPE), ("top", 65, UNSUPPORTED), ("X.data", 0x100000008, ALIGN), ("place", 0x100000002, ALIGN)])
def test_rows_are_checked(call, path, value, code):
    a = rows_args()
    change(a, path, value)
    assert call(a) == code


def test_rows_limits_and_optional_operands():
    for call in (gather_forward, combine_backward):
        a = rows_args()
        a["source"] = None
        assert call(a) == NULL
    for call in (combine_forward, combine_backward):
        a = rows_args()
        a["weight"] = None
        assert call(a) == NULL
    a = rows_args()
    a["rows"] = None
    assert combine_backward(a) == NULL      # dweight needs them
    a = rows_args()
    a["drows"] = a["dweight"] = None
    assert combine_backward(a) == rl.RL_OK  # nothing wanted
    a = rows_args()
    a["add"].rows = N - 1
    assert combine_forward(a) == SHAPE
    a = rows_args()
    a["X"], a["rows"] = tensor(1 << 23, D), tensor((1 << 23) * TOP, D)
    assert gather_forward(a) == UNSUPPORTED


def test_rows_outputs_may_not_overlap():
    for call, outs, ins in ((gather_forward, ("rows",), ("X", "place", "source")), (gather_backward, ("X",), ("rows", "place")),
                            (combine_forward, ("X",), ("rows", "place", "weight", "add")),
                            (combine_backward, ("drows", "dweight"), ("X", "rows", "place", "source", "weight", "drows"))):
        for out, other in itertools.product(outs, ins):
            if out == other:
                continue
            a = rows_args()
            at = a[other].data if isinstance(a[other], ctypes.Structure) else a[other]
            if isinstance(a[out], ctypes.Structure):
                a[out].data = at
            else:
                a[out] = at
            assert call(a) == rl.RL_ERR_ALIAS, (call.__name__, out, other)


@pytest.mark.parametrize("call,names", [(norm_forward, ("X", "R", "Y", "H")), (norm_backward, ("X", "dH", "H", "dX"))])
def test_norm_is_checked(call, names):
    for name in names:
        for field, value, code in (("data", None, NULL), ("dtype", rl.RL_F16 if name != "X" else 42, DTYPE), ("rows", N + 1 if name != "X" else 0, SHAPE),
                                   ("cols", 260 if name == "X" else D + 8, ALIGN if name == "X" else SHAPE), ("ld", D - 8, SHAPE), ("ld", D + 4, ALIGN),
                                   ("data", 0x100000008, ALIGN)):
            a = norm_args()
            change(a, f"{name}.{field}", value)
            assert call(a) == code, (name, field)
    a = norm_args()
    a["gain"] += 8
    assert call(a) == ALIGN
    a = norm_args()
    a["rstd"] += 2
    assert call(a) == ALIGN
    for name in names:
        a = norm_args()
        a[name] = tensor(N, 32776)
    a = {k: (tensor(N, 32776) if isinstance(v, rl.rl_tensor_t) and k != "Q" else v) for k, v in norm_args().items()}
    assert call(a) == UNSUPPORTED


def test_norm_operands():
    for eps in (-1e-6, float("nan")):
        a = norm_args()
        a["eps"] = eps
        assert norm_forward(a) == SHAPE
    for field, value, code in (("data", None, NULL), ("scales", None, NULL), ("dtype", rl.RL_FP8_B128, DTYPE), ("group", 64, UNSUPPORTED), ("ld", D, SHAPE),
                               ("rows", N + 1, SHAPE), ("data", 0x100000008, ALIGN)):
        a = norm_args()
        setattr(a["Q"], field, value)
        assert norm_forward(a) == code
    a = norm_args(rl.RL_F32)
    assert norm_forward(a) == UNSUPPORTED   # 8-bit rows of 32-bit ones
    a = norm_args()
    a["rstd"] = None
    assert norm_backward(a) == NULL
    a = norm_args()
    a["dX"] = a["dgain"] = None
    assert norm_backward(a) == rl.RL_OK
    a = norm_args()
    a["opts"] = None
    assert norm_backward(a) == rl.RL_ERR_WORKSPACE
    assert rl.runlora_rmsnorm_workspace_bytes(N, D, rl.RL_BF16) > 0
    for bad in ((0, D, 2), (N, 0, 2), (N, 260, 2), (N, 32776, 2), (N, D, 42)):
        assert rl.runlora_rmsnorm_workspace_bytes(*bad) == 0


def test_norm_outputs_may_not_overlap():
    def at(a, name):
        return a["Q"].scales if name == "Qs" else (a[name].data if isinstance(a[name], ctypes.Structure) else a[name])

    def put(a, name, where):
        if name == "Qs":
            a["Q"].scales = where
        elif isinstance(a[name], ctypes.Structure):
            a[name].data = where
        else:
            a[name] = where

    forward, backward = ("Y", "H", "rstd", "Q", "Qs"), ("dX", "dgain")
    for call, outs, ins in ((norm_forward, forward, ("X", "R", "gain")), (norm_backward, backward, ("X", "dH", "H", "gain", "rstd"))):
        for out in outs:
            for other in ins + outs:
                if other == out:
                    continue
                a = norm_args()
                put(a, out, at(a, other) + 16)   # (16 bytes on: h in X's or the residual's own place is allowed)
                assert call(a) == rl.RL_ERR_ALIAS, (call.__name__, out, other)


def test_8bit_layer_on_given_rows_is_checked():
    n, i, o, r = 40, 256, 272, 16
    W = rl.rl_tensor_t(next(ADDRESS), i, o, o, rl.RL_FP8_B128, next(ADDRESS), 128)
    base = dict(X=tensor(n, i), Q=rounded(n, i), W=W, A=tensor(i, r), B=tensor(r, o), Y=tensor(n, o), saved=rl.rl_saved_t(), opts=opts())

    def call(**new):
        a = dict(base, **new)
        return rl.lib().runlora_fp8_forward(*(ref(a[k]) for k in ("X", "Q", "W", "A", "B", "Y", "saved", "opts")))

    for name in ("X", "Q", "W", "A", "B", "Y", "saved"):
        assert call(**{name: None}) == NULL
    assert call(Q=rounded(n + 1, i)) == SHAPE and call(Q=rounded(n, i + 16)) == SHAPE and call(Q=tensor(n, i)) in (NULL, DTYPE)
    assert call(W=tensor(i, o)) == DTYPE
    q = rounded(n, i)
    q.data = base["Y"].data
    assert call(Q=q) == rl.RL_ERR_ALIAS
    q = rounded(n, i)
    q.scales = base["Y"].data
    assert call(Q=q) == rl.RL_ERR_ALIAS


def test_front_end_refuses():
    torch = pytest.importorskip("torch")
    t = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    i32, f32 = torch.int32, torch.float32
    with pytest.raises(ValueError, match="on a GPU"):
        rl.runlora_rmsnorm_forward(t(4, 16), t(16), t(4, 16))
    with pytest.raises(ValueError, match="on a GPU"):
        rl.runlora_rmsnorm_backward(t(4, 16), t(4, 16), t(16), t(4, dtype=f32), t(4, 16))
    with pytest.raises(ValueError, match="on a GPU"):
        rl.runlora_route_forward(t(4, 8), rl.Route(8, 2), t(4, 2, dtype=f32), t(4, 2, dtype=i32), t(4, 2, dtype=i32), t(8, dtype=i32), t(8, dtype=i32))
    with pytest.raises(ValueError, match="on a GPU"):
        rl.runlora_gather_forward(t(4, 16), t(4, 2, dtype=i32), t(8, dtype=i32), t(8, 16))
    with pytest.raises(ValueError, match="on a GPU"):
        rl.runlora_combine_backward(t(4, 16), t(8, 16), t(4, 2, dtype=i32), t(8, dtype=i32), t(4, 2, dtype=f32), t(8, 16), t(4, 2, dtype=f32))
    with pytest.raises(ValueError, match="place"):
        rl.runlora_combine_forward(t(8, 16), t(5, 2, dtype=i32), t(4, 2, dtype=f32), t(4, 16))
    for bad in (dict(score="relu"), dict(scale=0.0), dict(scale=1e-50), dict(scale=float("inf")), dict(scale=float("nan")), dict(groups=0), dict(groups_kept=0), dict(group_top=0)):
        with pytest.raises(ValueError):
            rl.Route(8, 2, **bad)
    for experts, top in ((8, 0), ((1 << 32) + 8, 2), (8, (1 << 32) + 2)):
        with pytest.raises(ValueError):
            rl.Route(experts, top)
    for bias in (t(8), t(7, dtype=f32), t(16, dtype=f32)[::2]):
        with pytest.raises(ValueError, match="bias"):
            rl.Route(8, 2).desc(bias)
    with pytest.raises(ValueError, match="data"):
        rl.Fp8Rows(t(3, 100, dtype=torch.uint8), t(1, 16, dtype=torch.uint8), 3, 100)
    with pytest.raises(ValueError, match="scales"):
        rl.Fp8Rows(t(3, 128, dtype=torch.uint8), t(1, 3, dtype=torch.uint8), 3, 100)
    with pytest.raises(ValueError, match="on a GPU"):
        rl.Fp8Rows.empty(3, 104, "cpu").values()


def test_8bit_values_are_checked():
    call = lambda q, out: rl.lib().runlora_fp8_values(ref(q), ref(out), None)
    assert call(None, tensor(N, D)) == NULL and call(rounded(N, D), None) == NULL
    assert call(tensor(N, D), tensor(N, D)) in (NULL, DTYPE) and call(rounded(N, D), tensor(N, D, 42)) == DTYPE
    assert call(rounded(N, D), tensor(N + 1, D)) == SHAPE and call(rounded(N, D), tensor(N, D + 8)) == SHAPE
    assert call(rounded(N, 260), tensor(N, 260, rl.RL_F32)) == ALIGN
    for name in ("data", "scales"):
        q, out = rounded(N, D), tensor(N, D)
        setattr(q, name, out.data + 16)
        assert call(q, out) == rl.RL_ERR_ALIAS
