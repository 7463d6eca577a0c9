"""Corners of what stands between the layers of a block with routed experts, on the GPU against the float64 reference of routed_oracle.py."""
import contextlib
import math

import numpy as np
import pytest

import routed_oracle as ref
from helpers import to_f64, torch_dtype
from test_gpu_routed import Watching, _rl, check_route, close, gen, logits, nan, placed, route_call

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---- groups that count with their two best, nothing added to the scores ----------------------------------------------

def alike(kind, n, E, dtype, seed):
    """Logits whose 64-bit scores are the same number although they differ."""
    rand = torch.rand(n, E, generator=gen(seed), device="cuda")
    if kind == "large":         # sigmoid(38 and more) is 1
        l = 38 + 20 * rand
    elif kind == "small":       # exp(1e-17) is 1
        l = (rand - 0.5) * 1e-17
    elif kind == "neighbours":  # one step of 32 bits apart: their sigmoids differ by less than 2^-53
        l = 30 + torch.floor(8 * rand) * 2.0 ** -19
    else:                       # softmax: exp(-747) is below the smallest 64-bit number
        l = 60 * rand
        l[:, 0] = 60 + 760
    return l.to(torch_dtype(dtype))


@pytest.mark.parametrize("E,top,groups,kept", [(8, 1, 2, 1), (8, 2, 4, 2), (24, 4, 8, 3), (64, 6, 8, 3), (120, 6, 8, 3), (256, 8, 8, 4), (512, 33, 16, 9), (640, 64, 64, 20),
                                               (1024, 20, 4, 2), (1023, 9, 33, 6), (16, 4, 16, 5)])
@pytest.mark.parametrize("kind,dtype", [("large", "f32"), ("large", "bf16"), ("small", "f32"), ("neighbours", "f32"), ("far", "f32"), ("far", "f16")])
def test_groups_by_their_two_best_choose_by_the_logits(E, top, groups, kept, kind, dtype):
    """Nothing is added to the scores: the groups are ranked by them, the choice is that of the logits, also of those whose scores are the same number."""
    l = alike(kind, 70, E, dtype, E + top)
    score = "softmax" if kind == "far" else "sigmoid"
    scores = ref.Routing(to_f64(l), top, score=score).s
    assert len(np.unique(scores[:, 1:])) == 1 and len(torch.unique(l[:, 1:])) > 4
    l[11, ::3] = -math.inf
    l[12] = -math.inf
    for renormalise in (True, False):
        check_route(l, top, dtype, score=score, renormalise=renormalise, groups=groups, groups_kept=kept, group_top=2, scale=2.5)


def test_groups_by_their_two_best_of_one_row():
    l = torch.tensor([[40.0, 41, -5, -5, 0, 1, 2, 3], [0, 1, 2, 3, 40, 41, 42, 40]], device="cuda")
    want = check_route(l, 1, "f32", score="sigmoid", groups=2, groups_kept=1, group_top=2)
    assert want.expert.tolist() == [[1], [6]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_nan_and_infinity_of_one_row(dtype):
    """Without a bias they count as much, with one the NaN's expert comes first; it alone has a NaN for its weight."""
    l = logits(40, 24, dtype, 9)
    l[:, 3], l[:, 7] = math.inf, math.nan
    l[20:, 3], l[20:, 7] = math.nan, math.inf
    for bias in (None, torch.zeros(24, device="cuda")):
        _, (weight, expert, *_) = route_call(l, 2, bias, score="sigmoid", renormalise=False)
        nan_at = torch.where(torch.arange(40, device="cuda") < 20, 7, 3).int()
        first = nan_at if bias is not None else torch.full_like(nan_at, 3)
        assert torch.equal(expert[:, 0], first) and torch.equal(expert[:, 1], 10 - first)
        assert torch.equal(torch.isnan(weight), expert == nan_at[:, None]) and (weight[~torch.isnan(weight)] == 1).all()


# ---- one rounding ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,E,top", [(300, 8, 2), (300, 60, 7), (90, 256, 8), (40, 1024, 33)])
@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("sigmoid", True), ("sigmoid", False)])
def test_route_gradients_are_rounded_once(n, E, top, score, renormalise):
    """D = scale dw holds 48 bits, exp is off by 2^-31 of itself, at most three of them to a factor: the chosen experts' gradients are off by the rounding of
    the result, u (2^-24), and by 2^-28 of what q |D| and q sum |D q| come to before they cancel."""
    rl = _rl()
    l = logits(n, E, "f32", E + top, 6.0)
    how = dict(score=score, renormalise=renormalise, scale=2.7)
    want = ref.Routing(to_f64(l), top, **dict(how, scale=float(np.float32(2.7))))
    plan, (weight, expert, *_) = route_call(l, top, **how)
    dw, dl = torch.randn(n, top, generator=gen(E), device="cuda"), nan((n, E), torch.float32)
    rl.runlora_route_backward(l, plan, expert, dw, dl)
    D = want.scale * to_f64(dw)
    mean = (np.abs(D) * want.q).sum(1, keepdims=True) if renormalise else 0.0
    left = want.left if score == "sigmoid" else 1.0
    magnitude = np.zeros((n, E))
    np.put_along_axis(magnitude, want.expert, want.q * left * (np.abs(D) + mean), 1)
    exact = want.backward(to_f64(dw), "f32")[0]
    close("dlogits", dl, exact, ref.U * np.abs(exact) + 2.0 ** -28 * magnitude + 2.0 ** -149)


@pytest.mark.parametrize("n,E,top", [(300, 8, 2), (300, 60, 7), (90, 256, 8), (40, 1024, 33)])
def test_whole_row_softmax_is_rounded_once(n, E, top):
    """The same where the sum is the whole row's: weights, gradients of the chosen experts and of the others, p_e sum D q.  Masked logits, and the largest and
    lowest ones, among them."""
    rl = _rl()
    l = logits(n, E, "f32", E + top, 6.0)
    l[3, 1:] = -math.inf
    l[4, ::2] = -math.inf
    l[5, 0] = 3e38
    l[6] = torch.finfo(torch.float32).min
    l[8] = -math.inf
    how = dict(score="softmax", renormalise=False, scale=2.7)
    want = ref.Routing(to_f64(l), top, **dict(how, scale=float(np.float32(2.7))))
    plan, (weight, expert, *_) = route_call(l, top, **how)
    close("weight", weight, want.weight, (ref.U + 2.0 ** -28) * np.abs(want.weight) + 2.0 ** -149)
    dw, dl = torch.randn(n, top, generator=gen(E), device="cuda"), nan((n, E), torch.float32)
    rl.runlora_route_backward(l, plan, expert, dw, dl)
    D = want.scale * to_f64(dw)
    mean = (np.abs(D) * want.q).sum(1, keepdims=True)
    magnitude = want.s * mean
    np.put_along_axis(magnitude, want.expert, want.q * (np.abs(D) + mean), 1)
    exact = want.backward(to_f64(dw), "f32")[0]
    close("dlogits", dl, exact, ref.U * np.abs(exact) + 2.0 ** -28 * magnitude + 2.0 ** -149)


# ---- the balance bias ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("python", [False, True])
@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("softmax", False), ("sigmoid", True)])
def test_bias_may_be_updated_before_the_backward(python, score, renormalise):
    """The bias decides the choice, which the forward keeps: an update between the two leaves the gradient's bits, of a row with a NaN too."""
    from paper_2312_03415_amd.module import RunRouter
    route = RunRouter(24, 4, score, renormalise, balance=True)
    l0 = logits(33, 24, "f32", 5)
    l0[7, 3] = float("nan")
    dw = torch.randn(33, 4, generator=gen(6), device="cuda")

    def run(update):
        l = l0.clone().requires_grad_(True)
        weight = route(l)[0]
        if update:
            route.bias.add_(torch.randn(24, generator=gen(7), device="cuda"))
        return torch.autograd.grad(weight, l, dw)[0]

    with Watching() if python else contextlib.nullcontext():
        want = run(False)
        got = run(True)
    assert torch.isnan(want[7]).any() and torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("value", [-1e9, torch.finfo(torch.float32).min, 1e9, math.inf])
@pytest.mark.parametrize("E,top,groups,kept", [(16, 3, 1, 1), (64, 6, 8, 3), (120, 6, 8, 3), (256, 8, 1, 1), (1024, 20, 4, 2)])
def test_a_large_bias_on_one_expert(E, top, groups, kept, value):
    """An expert taken out, or put first, by a large bias: the others' choice is as exact as without it."""
    l = logits(200, E, "f32", E)
    l[:, 5::8] = torch.nextafter(l[:, 4::8], torch.full_like(l[:, 4::8], 9.0))  # (scores closer than 32 bits tell)
    bias = torch.randn(E, generator=gen(E), device="cuda") * 0.1
    bias[5::8] = bias[4::8]
    bias[2] = value
    for score in ("softmax", "sigmoid"):
        for group_top in (1, 2):
            check_route(l, top, "f32", bias, score=score, groups=groups, groups_kept=kept, group_top=group_top)


def test_a_large_bias_takes_no_longer():
    """It sends no row through the 64-bit scores: 16384 x 256 took 48 us with -10^9 on one expert where every row went there, 25 without."""
    rl = _rl()
    n, E, top = 16384, 256, 8
    l, bias = logits(n, E, "f32", 1, 1.0), torch.randn(E, generator=gen(2), device="cuda") * 0.1
    out_of = bias.clone()
    out_of[2] = -1e9
    plan = rl.Route(E, top, "sigmoid", groups=8, groups_kept=4, group_top=2)
    _, out = route_call(l, top, bias, score="sigmoid", groups=8, groups_kept=4, group_top=2)
    ws = torch.empty(rl.runlora_route_workspace_bytes(n, E, top), dtype=torch.uint8, device="cuda")

    def least(b):
        graph, times = torch.cuda.CUDAGraph(), []
        with torch.cuda.graph(graph):
            for _ in range(20):
                rl.runlora_route_forward(l, plan, *out, bias=b, workspace=ws)
        for _ in range(12):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            graph.replay()
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
        return min(times)

    assert least(out_of) < 1.5 * least(bias)


# ---- operands that do not belong together ----------------------------------------------------------------------------

@pytest.mark.parametrize("python", [False, True])
@pytest.mark.parametrize("shape", [(26, 1), (1, 26), (2, 13)])
def test_a_saved_table_of_another_shape_is_refused(python, shape):
    """A saved-tensor hook that hands `place` back with as many entries in other rows: the gradient has the forward's rows."""
    from paper_2312_03415_amd import module as m
    place, source = (torch.from_numpy(t).cuda() for t in placed(13, 2, 4, 3))
    x = torch.randn(13, 72, generator=gen(1), device="cuda").bfloat16().requires_grad_(True)
    with Watching() if python else contextlib.nullcontext():
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.view(shape) if t.dtype == torch.int32 else t):
            rows = m.RunGatherFunction.apply(x, place, source)
        with pytest.raises((ValueError, RuntimeError)):
            rows.sum().backward()


def test_8bit_rows_of_another_width_are_refused():
    """Rows of 120 columns lie in as many bytes as rows of 128, and are others."""
    from paper_2312_03415_amd import module as m
    rl = _rl()
    g = gen(3)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    x, W, A, B = randn(40, 128), rl.Fp8Weight.quantize(randn(128, 64)), randn(128, 8), randn(8, 64)
    y, rows = torch.empty_like(x), rl.Fp8Rows.empty(40, 128)
    rl.runlora_rmsnorm_forward(x, None, y, rows=rows)
    with pytest.raises(rl.RunLoRAError):
        rl.runlora_rmsnorm_forward(x, None, y, rows=rl.Fp8Rows(rows.data, rows.scales, 40, 120))
    with pytest.raises(rl.RunLoRAError):
        m.RunLoRAFp8Function.apply(y, W, A, B, None, 1.0, rl.Fp8Rows(rows.data, rows.scales, 40, 120))
    assert torch.isfinite(m.RunLoRAFp8Function.apply(y, W, A, B, None, 1.0, rows)).all()


# ---- plans and transforms --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,i,o,r", [(2307, 1104, 4112, 16), (2307, 1104, 4112, 64), (2049, 2064, 4368, 8), (300, 1040, 4112, 16), (17, 1104, 272, 8)])
def test_8bit_layer_on_given_rows_of_a_prompt(n, i, o, r):
    """The bits of the layer that rounds its rows itself, on 256 x 256 tiles too; scale bytes behind the last row are nobody's."""
    rl = _rl()
    g = gen(n + r)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16)
    W, A, B, bias = rl.Fp8Weight.quantize(randn(i, o) * 0.03), randn(i, r) * 0.03, randn(r, o), randn(o)
    x, w = randn(n, i), randn(i)
    h, q = torch.empty_like(x), rl.Fp8Rows.empty(n, i)
    q.scales.fill_(255)
    rl.runlora_rmsnorm_forward(x, w, h, rows=q)
    assert (q.scales[:, n:] == 255).all()
    ws = rl.new_workspace(rl.FWD1, -1, n, i, o, r, rl.RL_BF16, w_dtype=rl.RL_FP8_B128)
    got, want, T, T0 = (nan((n, k), torch.bfloat16) for k in (o, o, r, r))
    rl.runlora_forward(rl.FWD1, h, W, A, B, want, rl.new_saved(T0), workspace=ws, scale=1.5, bias=bias)
    ws.fill_(255)
    rl.runlora_fp8_forward(h, q, W, A, B, got, rl.new_saved(T), workspace=ws, scale=1.5, bias=bias)
    assert torch.isfinite(want).all() and torch.equal(got, want) and torch.equal(T, T0)


def node_calls():
    """(name, call, its differentiable input) of the four nodes."""
    from paper_2312_03415_amd import module as m
    place, source = (torch.from_numpy(t).cuda() for t in placed(13, 2, 4, 3))
    x, rows, l = (torch.randn(*s, generator=gen(k), device="cuda") for k, s in enumerate(((13, 72), (26, 72), (13, 8))))
    weight = torch.rand(13, 2, generator=gen(4), device="cuda")
    return [("norm", lambda t: m.RunRMSNormFunction.apply(t, None, 1e-5), x), ("route", lambda t: m.RunRouteFunction.apply(t, _rl().Route(8, 2))[0], l),
            ("gather", lambda t: m.RunGatherFunction.apply(t, place, source), x),
            ("combine", lambda t: m.RunCombineFunction.apply(t, place, source, weight, x), rows)]


@pytest.mark.parametrize("at", range(4))
def test_transforms_are_refused(at):
    """vmap, functional gradients and forward mode, in which no node has a rule: an error, never an answer without its tangent."""
    import torch.autograd.forward_ad as fwd
    name, call, t = node_calls()[at]
    with pytest.raises(RuntimeError):
        torch.func.vmap(call)(torch.stack((t, t)))
    with pytest.raises(RuntimeError):
        torch.func.grad(lambda v: call(v).sum())(t)
    for leaf in (t, t.clone().requires_grad_(True)):
        with fwd.dual_level(), pytest.raises((RuntimeError, NotImplementedError)):
            call(fwd.make_dual(leaf, torch.ones_like(t)))
    assert torch.isfinite(call(t)).all()
