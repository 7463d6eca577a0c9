"""What stands between the layers of a block with routed experts, on the GPU against the float64 reference of routed_oracle.py: routing, rows to the
experts and back, root-mean-square norms with the residual and 8-bit rows, and all of them together."""
import contextlib
import math

import numpy as np
import pytest

import experts_oracle
import routed_oracle as ref
from helpers import to_f64, torch_dtype

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from torch.overrides import TorchFunctionMode  # noqa: E402


def _rl():
    from paper_2312_03415_amd import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def nan(shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def junk(shape):
    return torch.full(shape, -77, dtype=torch.int32, device="cuda")


def close(name, got, want, bound):
    got = to_f64(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert np.isfinite(got).all(), f"{name}: not finite"
    over = np.abs(got - want) - bound
    assert (over <= 0).all(), f"{name}: off by {np.abs(got - want)[over > 0].max():.3e}, {(np.abs(got - want) / bound)[over > 0].max():.2f} of the bound, at {np.argwhere(over > 0)[0]}"


# ---- norm ------------------------------------------------------------------------------------------------------------

WIDTHS = [8, 64, 72, 128, 136, 256, 264, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 5120, 6152, 8192, 8200, 16384, 16392, 32768]
EPS = 1e-6


def norm_inputs(n, d, dtype, seed, residual=True):
    td, g = torch_dtype(dtype), gen(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, r = (randn(n, d) * 3).to(td), (randn(n, d) * 2).to(td) if residual else None
    return x, r, (1 + 0.2 * randn(d)).to(td), randn(n, d).to(td), randn(n, d).to(td) if residual else None


def check_norm(n, d, dtype, seed, residual=True, gain=True, rows=False):
    rl = _rl()
    td = torch_dtype(dtype)
    x, r, w, dy, dh = norm_inputs(n, d, dtype, seed, residual)
    w = w if gain else None
    y, h, rstd = nan((n, d), td), nan((n, d), td), nan((n,), torch.float32)
    q = rl.Fp8Rows.empty(n, d) if rows else None
    rl.runlora_rmsnorm_forward(x, w, y, EPS, r, h, rstd, q)
    want_h = (x.float() + r.float()).to(td) if residual else x
    assert torch.equal(h, want_h)
    wd = to_f64(w) if gain else np.ones(d)
    want, bound, want_r = ref.norm_forward(to_f64(want_h), wd, EPS, dtype)
    close("y", y, want, bound)
    close("rstd", rstd, want_r[:, 0], 64 * ref.U * want_r[:, 0])
    if rows:
        values, exps = experts_oracle.round_blocks(to_f64(y), 1, 128)
        assert np.array_equal(to_f64(q.values()), values)
        assert np.array_equal(q.scales[:, :n].cpu().numpy().T.astype(np.int64) - 127, exps)
        assert not q.data[:, d:].any()
    dx, dg = nan((n, d), td), nan((d,), td)
    ws = torch.empty(max(256, rl.runlora_rmsnorm_workspace_bytes(n, d, rl.dtype_code(td))), dtype=torch.uint8, device="cuda")
    rl.runlora_rmsnorm_backward(dy, h, w, rstd, dx, dg, dh, ws)
    (wx, wg), (bx, bg) = ref.norm_backward(to_f64(dy), to_f64(want_h), wd, EPS, to_f64(dh) if residual else None, dtype)
    close("dx", dx, wx, bx)
    close("dgain", dg, wg, bg)
    alone, dg_alone = nan((n, d), td), nan((d,), td)
    rl.runlora_rmsnorm_backward(dy, h, w, rstd, alone, None, dh)
    rl.runlora_rmsnorm_backward(dy, h, w, rstd, None, dg_alone, dh, ws)
    assert torch.equal(alone, dx) and torch.equal(dg_alone, dg)


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_norm_widths(d, dtype):
    check_norm(5, d, dtype, d, rows=True)


@pytest.mark.parametrize("d", [4, 36, 64, 68, 128, 132, 260, 516, 1028, 2052, 4100, 8192, 8196, 16388, 32768])
def test_norm_widths_f32(d):
    check_norm(5, d, "f32", d)


@pytest.mark.parametrize("n,d,dtype", [(257, 16392, "bf16"), (600, 20480, "f16"), (259, 32768, "bf16"), (300, 8196, "f32"), (258, 20484, "f32")])
def test_norm_of_wide_rows_in_turn(n, d, dtype):
    check_norm(n, d, dtype, n, rows=dtype != "f32" and d % 128 == 0)


@pytest.mark.parametrize("n,d,dtype", [(1, 4096, "bf16"), (3, 128, "bf16"), (1030, 520, "f16"), (2500, 136, "bf16"), (1025, 5120, "bf16"), (37, 24, "f32")])
@pytest.mark.parametrize("residual,gain", [(True, True), (False, True), (True, False)])
def test_norm_rows(n, d, dtype, residual, gain):
    check_norm(n, d, dtype, n, residual, gain, rows=dtype != "f32")


def test_norm_in_place_and_strided():
    """h in the residual's place, rows that lie apart, and what lies between them untouched."""
    rl = _rl()
    n, d = 19, 264
    x, r, w, dy, dh = norm_inputs(n, d, "bf16", 3)
    wide = lambda t: torch.full((n, 2 * d), 7.0, dtype=t.dtype, device="cuda")
    xs, rs, ys = wide(x), wide(x), wide(x)
    xs[:, :d], rs[:, :d] = x, r
    y0, h0, rstd = torch.empty_like(x), torch.empty_like(x), nan((n,), torch.float32)
    rl.runlora_rmsnorm_forward(x, w, y0, EPS, r, h0, rstd)
    rl.runlora_rmsnorm_forward(xs[:, :d], w, ys[:, :d], EPS, rs[:, :d], rs[:, :d])
    assert torch.equal(ys[:, :d], y0) and torch.equal(rs[:, :d], h0) and torch.equal(xs[:, :d], x)
    for t in (xs, rs, ys):
        assert (t[:, d:] == 7.0).all()
    rl.runlora_rmsnorm_forward(xs[:, :d], w, ys[:, :d], EPS, r, xs[:, :d])
    assert torch.equal(ys[:, :d], y0) and torch.equal(xs[:, :d], h0)
    dx0, dx = torch.empty_like(x), wide(x)
    rl.runlora_rmsnorm_backward(dy, h0, w, rstd, dx0, None, dh)
    rl.runlora_rmsnorm_backward(dy, rs[:, :d], w, rstd, dx[:, :d], None, dh)
    assert torch.equal(dx[:, :d], dx0) and (dx[:, d:] == 7.0).all()


def test_norm_of_rows_that_are_zero_or_not_finite():
    """A row of zeros gives zeros; a NaN or an infinity stays in its own row (and its 8-bit blocks are NaN where y is)."""
    rl = _rl()
    n, d = 6, 264
    x, _, w, dy, _ = norm_inputs(n, d, "bf16", 5, residual=False)
    x[1] = 0
    x[3, 200] = float("nan")
    x[4, 7] = float("inf")
    y, rstd, q = torch.empty_like(x), nan((n,), torch.float32), rl.Fp8Rows.empty(n, d)
    rl.runlora_rmsnorm_forward(x, w, y, EPS, rstd=rstd, rows=q)
    assert torch.isfinite(y[[0, 1, 2, 5]]).all() and not y[1].any() and torch.isnan(y[3]).all()
    assert torch.isnan(y[4, 7]) and not y[4, :7].any()   # 1 / sqrt(inf) = 0
    v = q.values()
    assert torch.isnan(v[3]).all() and torch.isnan(v[4, :128]).all() and not v[4, 128:].any() and torch.isfinite(v[[0, 1, 2, 5]]).all()
    dx = torch.empty_like(x)
    rl.runlora_rmsnorm_backward(dy, x, w, rstd, dx)
    assert torch.isfinite(dx[[0, 1, 2, 5]]).all() and torch.isnan(dx[3]).all()


def test_norm_of_more_rows_than_workgroups():
    """2^16 workgroups of 16 rows, and some more rows."""
    check_norm(65536 * 16 + 37, 8, "f16", 1)


def test_norm_rows_beyond_31_bits():
    rl = _rl()
    n, d, ld = 40, 128, 1 << 26
    g = gen(2)
    big = torch.empty(n * ld, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((n, d), (ld, 1))
    y = big.as_strided((n, d), (ld, 1), 1 << 20)
    x.copy_(torch.randn(n, d, generator=g, device="cuda"))
    assert (n - 1) * ld > 2 ** 31
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    want, rstd = torch.empty(n, d, dtype=torch.bfloat16, device="cuda"), nan((n,), torch.float32)
    rl.runlora_rmsnorm_forward(x.contiguous(), w, want, EPS, rstd=rstd)
    with pytest.raises(rl.RunLoRAError):   # (the rows interleave: their ranges overlap)
        rl.runlora_rmsnorm_forward(x, w, y, EPS)
    rl.runlora_rmsnorm_forward(x, w, want, EPS)
    y.copy_(want)
    dx, dx0 = torch.empty_like(want), torch.empty_like(want)
    rl.runlora_rmsnorm_backward(y, x, w, rstd, dx)
    rl.runlora_rmsnorm_backward(want, x.contiguous(), w, rstd, dx0)
    assert torch.equal(dx, dx0)
    z, _, _ = ref.norm_forward(to_f64(x), np.ones(d), EPS, "bf16")
    assert np.abs(to_f64(want) - z).max() < 2 ** -7 * np.abs(z).max()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_values_of_8bit_rows(dtype):
    """All 256 bytes at scale bytes from both ends, each rounded once to the type."""
    rl = _rl()
    n, d = 20, 264
    q = rl.Fp8Rows.empty(n, d)
    q.data.copy_(torch.arange(q.data.numel(), device="cuda").view_as(q.data) * 7 % 256)
    byte = np.resize([0, 1, 5, 100, 112, 120, 127, 130, 140, 230, 246, 255], (3, n))
    q.scales[:, :n] = torch.from_numpy(byte.astype(np.uint8)).cuda()
    got = q.values(torch_dtype(dtype)).cpu()
    v = experts_oracle.e4m3_value(q.data[:, :d].cpu().numpy()) * np.where(byte == 255, np.nan, np.ldexp(1.0, byte.astype(np.int64) - 127))[np.arange(d) // 128].T
    want = torch.from_numpy(v).float().to(torch_dtype(dtype))   # (exact in float32: 4 bits and an exponent of at least -127 - 9)
    assert torch.equal(torch.nan_to_num(got.float(), nan=1.5e30), torch.nan_to_num(want.float(), nan=1.5e30))


@pytest.mark.parametrize("n", [1, 40, 300])
def test_8bit_layer_on_given_rows(n):
    """The bits of the layer that rounds its rows itself."""
    rl = _rl()
    i, o, r = 272, 400, 16
    g = gen(n)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16)
    W, A, B, bias = rl.Fp8Weight.quantize(randn(i, o) * 0.06), randn(i, r) * 0.06, randn(r, o), randn(o)
    x, w = randn(n, i), randn(i)
    h, q = torch.empty_like(x), rl.Fp8Rows.empty(n, i)
    rl.runlora_rmsnorm_forward(x, w, h, rows=q)
    ws = rl.new_workspace(rl.FWD1, -1, n, i, o, r, rl.RL_BF16, w_dtype=rl.RL_FP8_B128)
    got, want, T, T0 = (nan((n, k), torch.bfloat16) for k in (o, o, r, r))
    rl.runlora_forward(rl.FWD1, h, W, A, B, want, rl.new_saved(T0), workspace=ws, scale=1.5, bias=bias)
    ws.fill_(255)
    rl.runlora_fp8_forward(h, q, W, A, B, got, rl.new_saved(T), workspace=ws, scale=1.5, bias=bias)
    assert torch.equal(got, want) and torch.equal(T, T0)


# ---- routing ---------------------------------------------------------------------------------------------------------

def route_call(l, top, bias=None, **how):
    """Runs the forward into junk; (weight, expert, place, source, ends)."""
    rl = _rl()
    n, E = l.shape
    plan = rl.Route(E, top, **how)
    out = nan((n, top), torch.float32), junk((n, top)), junk((n, top)), junk((n * top,)), junk((E,))
    ws = torch.full((max(256, rl.runlora_route_workspace_bytes(n, E, top)),), 255, dtype=torch.uint8, device="cuda")
    rl.runlora_route_forward(l, plan, *out, bias=bias, workspace=ws)
    return plan, out


def check_route(l, top, dtype, bias=None, backward=True, **how):
    rl = _rl()
    want = ref.Routing(to_f64(l), top, bias=None if bias is None else to_f64(bias), **how)
    plan, (weight, expert, place, source, ends) = route_call(l, top, bias, **how)
    for name, got in (("expert", expert), ("place", place), ("source", source), ("ends", ends)):
        assert np.array_equal(got.cpu().numpy(), getattr(want, name)), name
    close("weight", weight, want.weight, want.weight_bound())
    if backward:
        dw = torch.randn(weight.shape, generator=gen(1), device="cuda")
        dl = nan(tuple(l.shape), l.dtype)
        rl.runlora_route_backward(l, plan, expert, dw, dl, bias)
        close("dlogits", dl, *want.backward(to_f64(dw), dtype))
    return want


def logits(n, E, dtype, seed, spread=2.0):
    return (torch.randn(n, E, generator=gen(seed), device="cuda") * spread).to(torch_dtype(dtype))


@pytest.mark.parametrize("E,top", [(1, 1), (2, 1), (5, 3), (8, 2), (8, 8), (9, 4), (16, 16), (31, 5), (32, 8), (33, 2), (64, 6), (64, 64), (65, 8), (128, 8),
                                   (250, 7), (256, 8), (257, 1), (384, 8), (512, 10), (513, 64), (1000, 3), (1024, 8)])
@pytest.mark.parametrize("n", [1, 77, 1100])
def test_route_sizes(n, E, top):
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            check_route(logits(n, E, "f32", n + E), top, "f32", score=score, renormalise=renormalise, scale=2.5)


@pytest.mark.parametrize("n,E,top", [(300, 8, 2), (300, 60, 7), (90, 256, 8), (40, 1024, 33)])
@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("sigmoid", True), ("sigmoid", False), ("softmax", False)])
def test_route_weights_are_rounded_once(n, E, top, score, renormalise):
    """exp to 2^-31 of itself, at most three of them to a weight and the rest in 64 bits: u (2^-24) and 2^-28 for all else.  Softmax over the whole row: its
    sum has terms of 3 u and u |l - max| of themselves, (ln E + 3) u of the sum."""
    l = logits(n, E, "f32", E + top, 6.0)
    want = ref.Routing(to_f64(l), top, score=score, renormalise=renormalise, scale=0.75)
    weight = route_call(l, top, None, score=score, renormalise=renormalise, scale=0.75)[1][0]
    off = ref.U + 2.0 ** -28 + (0.0 if renormalise or score == "sigmoid" else (math.log(E) + 3) * ref.U)
    close("weight", weight, want.weight, off * np.abs(want.weight) + 2.0 ** -149)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("E,top,groups,kept,group_top", [(8, 2, 2, 1, 1), (24, 4, 8, 3, 2), (64, 6, 8, 3, 2), (120, 6, 8, 3, 1), (256, 8, 8, 4, 2), (63, 4, 21, 5, 2),
                                                         (64, 3, 64, 9, 1), (640, 8, 64, 2, 2), (1024, 20, 4, 1, 2), (512, 8, 64, 12, 2), (512, 33, 16, 9, 1), (256, 16, 32, 5, 2),
                                                         (96, 5, 12, 4, 2), (40, 6, 40, 17, 1), (1023, 9, 33, 6, 2), (4, 1, 4, 2, 1)])
@pytest.mark.parametrize("biased", [False, True])
def test_route_groups(dtype, E, top, groups, kept, group_top, biased):
    bias = torch.randn(E, generator=gen(E), device="cuda") * 0.1 if biased else None
    for score in ("softmax", "sigmoid"):
        check_route(logits(205, E, dtype, E + top), top, dtype, bias, score=score, groups=groups, groups_kept=kept, group_top=group_top)


@pytest.mark.parametrize("E", [8, 20, 64, 200])
@pytest.mark.parametrize("biased", [False, True])
def test_route_ties_go_to_the_lowest_index(E, biased):
    """Few distinct values, and rows of one value: the choice is that of a stable order."""
    g = gen(E)
    l = torch.randint(0, 3, (300, E), generator=g, device="cuda").float()
    l[7] = 0
    bias = torch.zeros(E, device="cuda") if biased else None
    for score in ("softmax", "sigmoid"):
        check_route(l.bfloat16(), 5, "bf16", bias, score=score)
        check_route(l.bfloat16(), 5, "bf16", bias, score=score, renormalise=False, groups=4, groups_kept=2, group_top=2)


@pytest.mark.parametrize("biased", [False, True])
def test_route_close_scores(biased):
    """Scores that differ by less than 32 bits hold: sigmoid(l) + bias with biases that undo the differences but for the last bits of a 64-bit number."""
    E, n = 48, 500
    g = gen(1)
    l = torch.randn(n, E, generator=g, device="cuda")
    l[:, 1::2] = torch.nextafter(l[:, 0::2], torch.full_like(l[:, 0::2], 9.0))
    bias = torch.randn(E // 2, generator=g, device="cuda").repeat_interleave(2) if biased else None
    for how in (dict(score="sigmoid"), dict(score="softmax"), dict(score="sigmoid", groups=6, groups_kept=3, group_top=2)):
        check_route(l, 9, "f32", bias, **how)


@pytest.mark.parametrize("n", [50, 900])
@pytest.mark.parametrize("E", [6, 40, 160])
def test_route_masked(n, E):
    """Logits of -infinity: rows without anything left, rows with fewer than `top`, whole groups; nothing of them is placed."""
    g = gen(n + E)
    l = logits(n, E, "f32", E)
    l = l.masked_fill(torch.rand(n, E, generator=g, device="cuda") < 0.8, -math.inf)
    l[3] = -math.inf
    l[n - 1] = -math.inf
    l[5] = -math.inf
    l[5, E - 1] = 1.0
    for how in (dict(), dict(score="sigmoid"), dict(renormalise=False), dict(groups=2, groups_kept=1), dict(score="sigmoid", groups=2, groups_kept=1, group_top=2)):
        for bias in (None, torch.randn(E, generator=g, device="cuda") * 0.2):
            want = check_route(l, 4, "f32", bias, **how)
            assert (want.expert[3] == -1).all() and (want.expert[5] >= 0).sum() == 1 and want.ends[-1] < 4 * n
    l[:] = -math.inf
    want = check_route(l, 4, "f32")
    assert want.ends[-1] == 0


def test_route_bias_takes_experts_out():
    bias = torch.zeros(16, device="cuda")
    bias[::2] = -math.inf
    want = check_route(logits(100, 16, "bf16", 2), 4, "bf16", bias, score="sigmoid")
    assert (want.expert % 2 == 1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_route_lowest_values_are_no_mask(dtype):
    """Logits at the type's lowest value are finite: taken last, by index; weights of a row of them are equal."""
    low = torch.finfo(torch_dtype(dtype)).min
    l = logits(64, 10, dtype, 4)
    l[:, 3:] = low
    l[9] = low
    for score in ("softmax", "sigmoid"):
        plan, (weight, expert, place, source, ends) = route_call(l, 5, score=score)
        assert (expert[:, 3:].cpu() == torch.tensor([3, 4])).all() and (place >= 0).all()
        assert expert[9].tolist() == [0, 1, 2, 3, 4] and torch.allclose(weight[9], torch.full((5,), 0.2, device="cuda"), rtol=1e-6)
        assert torch.isfinite(weight).all() and not weight[0, 3:].any() and torch.allclose(weight.sum(1), torch.ones(64, device="cuda"), rtol=1e-6)


def test_route_very_negative_scores_keep_their_ratio():
    """sigmoid of -200 is below the smallest fp32 number; the renormalised weights are not."""
    l = torch.tensor([[-200.0, -201.0, -300.0, -203.0], [-90.0, -100.0, 3.0, 80.0]], device="cuda")
    check_route(l, 3, "f32", score="sigmoid")


@pytest.mark.parametrize("E", [8, 40, 256])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("grouped", [False, True])
def test_route_nan_and_infinity(E, biased, grouped):
    """A NaN (softmax: or +infinity) makes its row's weights NaN, and only its row's; the choice stays in range, of different experts."""
    rl = _rl()
    l = logits(40, E, "f32", E)
    l[3, E - 1] = float("nan")
    l[5] = float("nan")
    l[9, 2] = float("inf")
    bias = torch.randn(E, generator=gen(3), device="cuda") * 0.1 if biased else None
    how = dict(groups=4, groups_kept=2, group_top=2) if grouped else {}
    clean = l.clone()
    clean[[3, 5, 9]] = 0
    for score in ("softmax", "sigmoid"):
        plan, (weight, expert, place, source, ends) = route_call(l, 4, bias, score=score, **how)
        _, (w0, e0, *_) = route_call(clean, 4, bias, score=score, **how)
        rest = [t for t in range(40) if t not in (3, 5, 9)]
        assert torch.equal(weight[rest], w0[rest]) and torch.equal(expert[rest], e0[rest])
        assert torch.isnan(weight[3]).all() and torch.isnan(weight[5]).all()
        assert torch.isnan(weight[9]).all() if score == "softmax" else torch.isfinite(weight[9]).all()
        assert (expert >= 0).all() and (expert < E).all() and int(ends[-1]) == 160
        assert all(len(set(row)) == 4 for row in expert.tolist())
        assert sorted(place.flatten().tolist()) == list(range(160)) and torch.equal(source[place.flatten().long()].cpu(), torch.arange(160, dtype=torch.int32))
        dl = nan(tuple(l.shape), torch.float32)
        rl.runlora_route_backward(l, plan, expert, torch.ones_like(weight), dl, bias)
        assert torch.isfinite(dl[rest]).all() and torch.isnan(dl[3]).any() and torch.isnan(dl[5]).any()


def test_route_odd_addresses_and_strides():
    """Logits and their gradient at odd addresses, with rows apart; what lies between is left."""
    rl = _rl()
    n = 131
    for dtype, E in (("bf16", 37), ("f32", 37), ("bf16", 64), ("f32", 64), ("f16", 256), ("f32", 256)):
        l = logits(n, E, dtype, 6)
        wide = nan((n + 1, 2 * E + 1), l.dtype)
        part = wide.flatten()[1:1 + n * (2 * E + 1)].view(n, 2 * E + 1)[:, :E]
        part.copy_(l)
        plan, a = route_call(l, 4)
        _, b = route_call(part, 4)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        dl0, dl = torch.empty_like(l), torch.full_like(wide, 7.0)
        to = dl.flatten()[1:1 + n * (2 * E + 1)].view(n, 2 * E + 1)[:, :E]
        dw = torch.randn(n, 4, generator=gen(1), device="cuda")
        rl.runlora_route_backward(l, plan, a[1], dw, dl0)
        rl.runlora_route_backward(part, plan, b[1], dw, to)
        assert torch.equal(to, dl0) and int((dl == 7.0).sum()) == dl.numel() - n * E
    check_route(logits(1, 5, "bf16", 1)[:, :5], 2, "bf16")


@pytest.mark.parametrize("n,E,top", [(40000, 8, 2), (100003, 64, 4), (20011, 300, 8)])
def test_route_many_tokens(n, E, top):
    check_route(logits(n, E, "bf16", n), top, "bf16", backward=False)


def test_route_foreign_choices_in_the_backward():
    """Experts outside the range count as none."""
    rl = _rl()
    l = logits(9, 12, "f32", 1)
    plan, (weight, expert, *_) = route_call(l, 3)
    bad = expert.clone()
    bad[4] = torch.tensor([-5, 12, 1 << 30], dtype=torch.int32)
    dl = nan((9, 12), torch.float32)
    rl.runlora_route_backward(l, plan, bad, torch.ones_like(weight), dl)
    assert not dl[4].any() and torch.isfinite(dl).all()


# ---- rows to the experts and back -------------------------------------------------------------------------------------

def placed(n, top, experts, seed, lost=0.1):
    """place [n, top] and source [n top] of a random choice with some copies left out."""
    rng = np.random.default_rng(seed)
    flat = rng.integers(0, experts, n * top)
    flat[rng.random(n * top) < lost] = experts
    order = np.argsort(flat, kind="stable")
    m = int((flat < experts).sum())
    place = np.full(n * top, -1, dtype=np.int32)
    place[order[:m]] = np.arange(m)
    source = np.where(np.arange(n * top) < m, order, -1).astype(np.int32)
    return place.reshape(n, top), source


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,d,top", [(1, 8, 1), (1, 4096, 8), (7, 264, 3), (5, 2048, 1), (33, 2056, 9), (130, 136, 64), (300, 520, 2), (3, 32776, 4)])
def test_rows_there_and_back(n, d, top, dtype):
    rl = _rl()
    td, g = torch_dtype(dtype), gen(n + d)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(td)
    hp, hs = placed(n, top, 5, n * d)
    place, source = torch.from_numpy(hp).cuda(), torch.from_numpy(hs).cuda()
    m = n * top
    x, drows, back, dy, add = randn(n, d), randn(m, d), randn(m, d), randn(n, d), randn(n, d)
    drows[hs < 0] = float("nan")   # rows without a copy: never read
    back[hs < 0] = float("nan")
    weight = torch.randn(n, top, generator=g, device="cuda")
    rows, dx = nan((m, d), td), nan((n, d), td)
    rl.runlora_gather_forward(x, place, source, rows)
    assert np.array_equal(to_f64(rows), ref.gather(to_f64(x), hp))
    rl.runlora_gather_backward(drows, place, dx)
    close("dx", dx, *ref.join(to_f64(drows), hp, np.ones((n, top)), None, dtype))
    for a in (None, add):
        y = nan((n, d), td)
        rl.runlora_combine_forward(back, place, weight, y, a)
        close("y", y, *ref.join(to_f64(back), hp, to_f64(weight), None if a is None else to_f64(a), dtype))
    gr, gw = nan((m, d), td), nan((n, top), torch.float32)
    rl.runlora_combine_backward(dy, back, place, source, weight, gr, gw)
    (wr, ww), (br, bw) = ref.spread(to_f64(dy), np.nan_to_num(to_f64(back)), hp, to_f64(weight), dtype)
    close("drows", gr, wr, br)
    close("dweight", gw, ww, bw)
    gr2, gw2 = nan((m, d), td), nan((n, top), torch.float32)
    rl.runlora_combine_backward(dy, None, place, source, weight, gr2, None)
    rl.runlora_combine_backward(dy, back, place, source, weight, None, gw2)
    assert torch.equal(gr2, gr) and torch.equal(gw2, gw)


def test_rows_at_strides_and_places_outside():
    """Rows apart, left alone between; places outside the rows count as none."""
    rl = _rl()
    n, top, d = 21, 3, 72
    hp, hs = placed(n, top, 4, 1, lost=0.0)
    hp[2, 1], hp[7, 0], hp[20, 2] = -9, n * top, 2 ** 31 - 1
    place, source = torch.from_numpy(hp).cuda(), torch.from_numpy(hs).cuda()
    g = gen(4)
    wide = lambda k: torch.full((k, 2 * d), 7.0, dtype=torch.bfloat16, device="cuda")
    x, rows, y = wide(n), wide(n * top), wide(n)
    x[:, :d] = torch.randn(n, d, generator=g, device="cuda")
    rl.runlora_gather_forward(x[:, :d], place, source, rows[:, :d])
    kept = np.where((hp >= 0) & (hp < n * top), hp, -1)
    want = ref.gather(to_f64(x[:, :d]), kept)
    written = np.zeros(n * top, dtype=bool)
    written[kept[kept >= 0]] = True
    assert np.array_equal(to_f64(rows[:, :d])[written], want[written]) and (rows[:, d:] == 7.0).all()
    assert (rows[torch.from_numpy(~written).cuda()] == 7.0).all()   # (their sources name copies that have no place)
    weight = torch.randn(n, top, generator=g, device="cuda")
    rl.runlora_combine_forward(rows[:, :d], place, weight, y[:, :d])
    close("y", y[:, :d], *ref.join(to_f64(rows[:, :d]), kept, to_f64(weight), None, "bf16"))
    assert (y[:, d:] == 7.0).all()
    gw, gr = nan((n, top), torch.float32), wide(n * top)
    rl.runlora_combine_backward(y[:, :d], rows[:, :d], place, source, weight, gr[:, :d], gw)
    assert gw[2, 1] == 0 and gw[7, 0] == 0 and gw[20, 2] == 0 and torch.isfinite(gw).all() and (gr[:, d:] == 7.0).all()


def test_rows_beyond_31_bits():
    rl = _rl()
    n, top, d = 70000, 4, 8192
    assert n * top * d > 2 ** 31
    hp, hs = placed(n, top, 8, 3, lost=0.01)
    place, source = torch.from_numpy(hp).cuda(), torch.from_numpy(hs).cuda()
    g = gen(7)
    x = torch.randn(n, d, generator=g, device="cuda", dtype=torch.bfloat16)
    rows = nan((n * top, d), torch.bfloat16)
    rl.runlora_gather_forward(x, place, source, rows)
    where = torch.clamp(source.long(), min=0) // top
    for lo in range(0, n * top, 40000):
        part = rows[lo:lo + 40000]
        want = torch.where((source[lo:lo + 40000] >= 0)[:, None], x[where[lo:lo + 40000]], torch.zeros((), dtype=x.dtype, device="cuda"))
        assert torch.equal(part, want)
    weight = torch.rand(n, top, generator=g, device="cuda")
    y = nan((n, d), torch.bfloat16)
    rl.runlora_combine_forward(rows, place, weight, y)
    take = np.array([0, 1, 34999, 65535, 65536, 69998, 69999])
    total = np.where(hp[take] >= 0, to_f64(weight)[take], 0.0).sum(1, keepdims=True)
    want = to_f64(x[torch.from_numpy(take).cuda()]) * total   # every placed copy is the token's own row
    assert (np.abs(to_f64(y[torch.from_numpy(take).cuda()]) - want) <= (2 ** -8 + 2 ** -20) * np.abs(want) + 1e-30).all()
    gr, gw = rows, nan((n, top), torch.float32)
    back = rows.clone()
    rl.runlora_combine_backward(x, back, place, source, weight, gr, gw)
    sq = (to_f64(x[torch.from_numpy(take).cuda()]) ** 2).sum(1, keepdims=True)
    assert (np.abs(to_f64(gw)[take] - np.where(hp[take] >= 0, sq, 0.0)) <= 2 ** -16 * sq).all()
    for t in take:
        for j in range(top):
            if hp[t, j] >= 0:
                v = to_f64(x[int(t)]) * float(weight[int(t), j])
                assert (np.abs(to_f64(gr[int(hp[t, j])]) - v) <= (2 ** -8 + 2 ** -20) * np.abs(v) + 1e-30).all()


# ---- streams and graphs -----------------------------------------------------------------------------------------------

class Chain:
    """Norm, routing, rows to the experts, a layer over them and back, into kept buffers, as a serving loop calls them."""

    def __init__(self, n, seed=0, d=272, E=6, top=2):
        rl = _rl()
        g = gen(seed)
        self.rl, self.n = rl, n
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
        bf = torch.bfloat16
        self.x, self.r, self.gain = randn(n, d).to(bf), randn(n, d).to(bf), (1 + 0.1 * randn(d)).to(bf)
        self.router = randn(d, E) / 16
        self.bias = randn(E) * 0.02
        self.W, self.A, self.B = randn(E, d, d).to(bf) / 16, randn(E, d, 8).to(bf) / 16, randn(E, 8, d).to(bf)
        self.plan = rl.Route(E, top, score="sigmoid")
        e = lambda shape, dt: torch.empty(shape, dtype=dt, device="cuda")
        i32 = torch.int32
        self.h, self.y, self.out, self.l = e((n, d), bf), e((n, d), bf), e((n, d), bf), e((n, E), torch.float32)
        self.route = e((n, top), torch.float32), e((n, top), i32), e((n, top), i32), e((n * top,), i32), e((E,), i32)
        self.rows, self.back = e((n * top, d), bf), e((n * top, d), bf)
        size = max(256, rl.runlora_route_workspace_bytes(n, E, top), rl.runlora_experts_workspace_bytes(False, n * top, E, d, d, 8, rl.RL_BF16))
        self.ws = e((size,), torch.uint8)

    def __call__(self):
        rl, (weight, expert, place, source, ends) = self.rl, self.route
        rl.runlora_rmsnorm_forward(self.x, self.gain, self.y, residual=self.r, H=self.h)
        torch.mm(self.y.float(), self.router, out=self.l)
        rl.runlora_route_forward(self.l, self.plan, weight, expert, place, source, ends, bias=self.bias, workspace=self.ws)
        rl.runlora_gather_forward(self.y, place, source, self.rows)
        rl.runlora_experts_forward(self.rows, ends, self.W, self.A, self.B, self.back, workspace=self.ws)
        rl.runlora_combine_forward(self.back, place, weight, self.out, self.h)
        return self.out

    def results(self):
        return [t.clone() for t in (self.h, self.y, *self.route, self.rows, self.back, self.out)]


@pytest.mark.parametrize("n", [5, 700])
def test_chain_on_another_stream(n):
    c = Chain(n)
    c()
    torch.cuda.synchronize()
    want = c.results()
    for t in (c.h, c.y, c.out, c.rows, c.back):
        t.fill_(float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(c.results(), want))


@pytest.mark.parametrize("n", [5, 700])
def test_two_captured_chains_share_a_workspace(n):
    """Replayed with new inputs, in turn, with eager work between: each replay gives the eager bits."""
    a, b = Chain(n, 1), Chain(n, 2)
    b.ws = a.ws
    graphs = []
    for c in (a, b):
        c()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c()
        graphs.append(graph)
    for step in range(3):
        g = gen(100 + step)
        for c, graph in zip((a, b), graphs):
            c.x.copy_(torch.randn(c.x.shape, generator=g, device="cuda"))
            c()
            torch.cuda.synchronize()
            want = c.results()
            for t in (c.h, c.y, c.out, c.rows, c.back, c.route[0]):
                t.fill_(float("nan"))
            for t in c.route[1:]:
                t.fill_(-99)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(c.results(), want)), step


# ---- the modules -------------------------------------------------------------------------------------------------------

def test_norm_module():
    from paper_2312_03415_amd.module import RunRMSNorm
    d = 264
    norm = RunRMSNorm(d, trainable=True)
    x, r, w, dy, dh = norm_inputs(30, d, "bf16", 9)
    with torch.no_grad():
        norm.weight.copy_(w)
    leaves = [t.view(5, 6, d).clone().requires_grad_(True) for t in (x, r)]
    y, h, q = norm(leaves[0], leaves[1], rows=True)
    torch.autograd.backward((y, h), (dy.view(5, 6, d), dh.view(5, 6, d)))
    hd = to_f64(h).reshape(30, d)
    want, bound, _ = ref.norm_forward(hd, to_f64(w), 1e-6, "bf16")
    close("y", y.reshape(30, d), want, bound)
    assert np.array_equal(to_f64(q.values()), experts_oracle.round_blocks(to_f64(y).reshape(30, d), 1, 128)[0])
    (wx, wg), (bx, bg) = ref.norm_backward(to_f64(dy), hd, to_f64(w), 1e-6, to_f64(dh), "bf16")
    for leaf in leaves:
        close("dx", leaf.grad.view(30, d), wx, bx)
    assert leaves[0].grad.data_ptr() != leaves[1].grad.data_ptr()   # (one gradient for both, but not one memory)
    close("dgain", norm.weight.grad, wg, bg)
    # either output alone, neither input wanted, no rows
    x1 = x.clone().requires_grad_(True)
    y, h = norm(x1, r)
    assert torch.equal(torch.autograd.grad(h, x1, dh)[0], dh)
    y, h = norm(x1, r)
    gx, = torch.autograd.grad(y, x1, dy)
    (wx, _), (bx, _) = ref.norm_backward(to_f64(dy), to_f64(h), to_f64(w), 1e-6, None, "bf16")
    close("dx of y alone", gx, wx, bx)
    with torch.no_grad():
        assert torch.equal(norm(x, r)[0], y)
    x0 = torch.empty(0, d, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y, h = norm(x0, x0.detach())
    (y.sum() + h.sum()).backward()
    assert x0.grad.shape == (0, d)


def test_gradients_of_strided_and_broadcast_upstream():
    """Gradients that arrive expanded or transposed; inputs with rows apart and at odd addresses."""
    from paper_2312_03415_amd.module import RunCombineFunction, RunGatherFunction, RunRMSNorm
    n, top, d = 12, 2, 72
    hp, hs = placed(n, top, 4, 2, lost=0.0)
    place, source = torch.from_numpy(hp).cuda(), torch.from_numpy(hs).cuda()
    g = gen(3)
    base = torch.randn(n * (2 * d) + 1, generator=g, device="cuda").bfloat16()
    odd = base[1:].view(n, 2 * d)[:, :d]
    norm = RunRMSNorm(d)
    ones = lambda *s: torch.ones(1, dtype=torch.bfloat16, device="cuda").expand(*s)
    for x in (odd, odd.contiguous()):
        x = x.detach().requires_grad_(True)
        rows = RunGatherFunction.apply(norm(x), place, source)
        weight = torch.randn(top, n, generator=gen(5), device="cuda").t().requires_grad_(True)
        y = RunCombineFunction.apply(rows, place, source, weight, None)
        gx, gw = torch.autograd.grad(y, (x, weight), ones(n, d), retain_graph=True)
        gx2, gw2 = torch.autograd.grad(y, (x, weight), torch.ones(n, d, dtype=torch.bfloat16, device="cuda"))
        assert torch.equal(gx, gx2) and torch.equal(gw, gw2)
        if x.is_contiguous():
            assert torch.equal(gx, last)
        last = gx


@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_routed_layer_gradients(score, renormalise):
    """Norm, router, rows, one linear per expert and the weighted sum, all together, in fp32, against the same in 64 bits by torch's own gradients with the same
    choice; and along a direction against a difference quotient (where no choice changes)."""
    from paper_2312_03415_amd.module import RunCombineFunction, RunGatherFunction, RunRMSNorm, RunRouter
    n, d, E, top = 50, 24, 6, 3
    g = gen(8)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, r, W, router, dy = randn(n, d), randn(n, d), randn(E, d, d) / 5, randn(d, E) / 5, randn(n, d)
    norm, route = RunRMSNorm(d, dtype=torch.float32, trainable=True), RunRouter(E, top, score, renormalise, scale=1.5, balance=True)
    with torch.no_grad():
        norm.weight.copy_(1 + 0.1 * randn(d))
        route.bias.copy_(0.01 * randn(E))
    leaves = dict(x=x, r=r, router=router)
    leaves = {k: v.clone().requires_grad_(True) for k, v in leaves.items()}

    def run(x, r, router):
        y, h = norm(x, r)
        weight, expert, place, source, ends = route(y @ router)
        rows = RunGatherFunction.apply(y, place, source)
        parts = []
        lo = 0
        for e, hi in enumerate(ends.tolist()):
            parts.append(rows[lo:hi] @ W[e])
            lo = hi
        return RunCombineFunction.apply(torch.cat(parts), place, source, weight, h), expert, ends

    out, expert, ends = run(**leaves)
    assert int(ends[-1]) == n * top
    grads = torch.autograd.grad(out, [*leaves.values(), norm.weight], dy)

    def want(x, r, router, gain):
        h = x + r
        y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * gain
        l = y @ router
        s = torch.softmax(l, 1) if score == "softmax" else torch.sigmoid(l)
        q = s.gather(1, expert.cpu().long())
        q = 1.5 * (q / q.sum(1, keepdim=True) if renormalise else q)
        z = torch.stack([y @ W[e].double().cpu() for e in range(E)], 1)   # [n, E, d]
        z = torch.gather(z, 1, expert.cpu().long()[:, :, None].expand(-1, -1, d))
        return h + (q[:, :, None] * z).sum(1)

    ref_leaves = [t.detach().double().cpu().requires_grad_(True) for t in (x, r, router, norm.weight)]
    ref_out = want(*ref_leaves)
    ref_grads = torch.autograd.grad(ref_out, ref_leaves, dy.double().cpu())
    # fp32 throughout: products of 24 terms and three operators in a row, each good to some 100 u of its terms' magnitudes: 2^-15 of the largest element
    tol = lambda t: 2.0 ** -15 * t.abs().max().item()
    assert (out.double().cpu() - ref_out).abs().max().item() < tol(ref_out.detach())
    for got, wanted, name in zip(grads, ref_grads, ("x", "r", "router", "gain")):
        assert (got.double().cpu() - wanted).abs().max().item() < tol(wanted), name
    # the 64-bit formula's gradient against differences of itself: second order in the step
    v = [torch.randn(t.shape, generator=torch.Generator().manual_seed(1), dtype=torch.float64) for t in ref_leaves]
    eps = 1e-5
    up, down = (want(*[t.detach() + s * eps * u for t, u in zip(ref_leaves, v)]) for s in (1, -1))
    slope = ((up - down) / (2 * eps) * dy.double().cpu()).sum().item()
    along = sum((gr * u).sum().item() for gr, u in zip(ref_grads, v))
    assert abs(slope - along) < 1e-6 * sum((gr * u).abs().sum().item() for gr, u in zip(ref_grads, v))


def test_captured_training_pass():
    """Forward and backward captured into a graph while an eager graph of other leaves lives; replays give the eager bits."""
    from paper_2312_03415_amd.module import RunCombineFunction, RunGatherFunction, RunRMSNorm, RunRouter
    n, d, E, top = 300, 136, 8, 2
    g = gen(4)
    norm, route = RunRMSNorm(d), RunRouter(E, top)
    x0 = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    router = torch.randn(d, E, generator=g, device="cuda") / 8
    dy = torch.randn(n, d, generator=g, device="cuda").bfloat16()

    def step(x):
        y, h = norm(x, x.detach())
        weight, _, place, source, ends = route(y.float() @ router)
        out = RunCombineFunction.apply(RunGatherFunction.apply(y, place, source), place, source, weight, h)
        return (out.detach(), *torch.autograd.grad(out, x, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x = x0.clone().requires_grad_(True)
    with torch.cuda.stream(side):
        step(x)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(x)
    for k in range(3):
        with torch.no_grad():
            x.copy_(torch.randn(n, d, generator=gen(20 + k), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        want = step(x.detach().clone().requires_grad_(True))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


class Watching(TorchFunctionMode):
    """A torch function mode: it sends calls to the Python nodes."""

    def __torch_function__(self, func, types, args=(), kwargs=None):
        return func(*args, **(kwargs or {}))


def every_node(n=14, d=72, E=6, top=2):
    """(outputs, leaves) of one call of each node, 3-D where it may be."""
    from paper_2312_03415_amd import module as m
    g = gen(12)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    bf = torch.bfloat16
    x, r, gain, l = [t.requires_grad_(True) for t in (randn(2, n // 2, d).to(bf), randn(2, n // 2, d).to(bf), randn(d).to(bf), randn(n, E))]
    y, h = m.RunRMSNormFunction.apply(x, gain, 1e-5, r)
    weight, expert, place, source, ends = m.RunRouteFunction.apply(l, _rl().Route(E, top))
    rows = m.RunGatherFunction.apply(y.detach().view(n, d).requires_grad_(True), place, source)
    out = m.RunCombineFunction.apply(rows.detach().requires_grad_(True), place, source, weight.detach().requires_grad_(True), h.detach())
    return y, h, weight, rows, out


@pytest.mark.parametrize("python", [False, True])
def test_second_derivatives_are_refused(python):
    with Watching() if python else contextlib.nullcontext():
        y, h, weight, rows, out = every_node()
        for t in (y, weight, rows, out):
            leaf = next(f[0].variable for f in t.grad_fn.next_functions if hasattr(f[0], "variable"))
            first, = torch.autograd.grad(t.float().pow(2).sum(), leaf, retain_graph=True)
            again, = torch.autograd.grad(t.float().pow(2).sum(), leaf, create_graph=True)
            assert torch.equal(first, again.detach())
            with pytest.raises(RuntimeError, match="once|twice"):
                again.float().sum().backward()


@pytest.mark.parametrize("python", [False, True])
def test_outputs_may_be_changed_in_place(python):
    """Where no gradient reads them: y and the combined rows; h is read, which autograd notices."""
    with Watching() if python else contextlib.nullcontext():
        y, h, weight, rows, out = every_node()
        for t in (y, out):
            assert not t._is_view()
            leaf = next(f[0].variable for f in t.grad_fn.next_functions if hasattr(f[0], "variable"))
            want, = torch.autograd.grad(t, leaf, 2 * torch.ones_like(t), retain_graph=True)
            t.mul_(2)
            got, = torch.autograd.grad(t, leaf, torch.ones_like(t))
            assert torch.equal(got, want)
        y, h, *_ = every_node()
        h.add_(1)
        with pytest.raises(RuntimeError, match="inplace"):
            y.sum().backward()


def test_python_nodes_give_the_native_ones_bits():
    from paper_2312_03415_amd import module as m
    rl = _rl()
    n, d, E, top = 70, 144, 12, 3
    g = gen(6)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    bf = torch.bfloat16
    x, r, gain, l = randn(n, d).to(bf), randn(n, d).to(bf), randn(d).to(bf), randn(n, E)
    W, A, B = rl.Fp8Weight.quantize(randn(d, 160).to(bf)), randn(d, 8).to(bf), randn(8, 160).to(bf)
    bias = 0.1 * randn(E)
    dy, dh = randn(n, d).to(bf), randn(n, d).to(bf)
    plan = rl.Route(E, top, "sigmoid", groups=4, groups_kept=2, group_top=2)

    def run():
        leaves = [t.clone().requires_grad_(True) for t in (x, r, gain, l, A)]
        y, h, data, scales = m.RunRMSNormFunction.apply(leaves[0], leaves[2], 1e-5, leaves[1], True)
        z, = (m.RunRMSNormFunction.apply(h, None, 1e-5),)
        weight, expert, place, source, ends = m.RunRouteFunction.apply(leaves[3], plan, bias)
        rows = m.RunGatherFunction.apply(z, place, source)
        out = m.RunCombineFunction.apply(rows, place, source, weight, h)
        q = m.RunLoRAFp8Function.apply(y, W, leaves[4], B, None, 2.0, rl.Fp8Rows(data, scales, n, d))
        grads = torch.autograd.grad((out, q), leaves, (dy, torch.ones_like(q)))
        return [y, h, data, scales[:, :n], z, weight, expert, place, source, ends, rows, out, q, *grads]

    native = run()
    with Watching():
        python = run()
    names = [t.grad_fn.name() for t in (native[0], native[5], native[10], native[11])], [t.grad_fn.name() for t in (python[0], python[5], python[10], python[11])]
    assert all("Node" in a and "Function" in b for a, b in zip(*names)), names
    for k, (a, b) in enumerate(zip(native, python)):
        assert torch.equal(a, b), k


def test_saved_tensor_hooks_and_second_use():
    """What is saved may come back laid out anew or from the host's memory and back; a second backward through a kept graph gives the same bits."""
    from paper_2312_03415_amd import module as m
    n, d, E, top = 40, 136, 8, 2
    g = gen(16)
    x0, l0 = torch.randn(n, d, generator=g, device="cuda").bfloat16(), torch.randn(n, E, generator=g, device="cuda")
    dy = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    norm, route = m.RunRMSNorm(d, trainable=True), m.RunRouter(E, top)

    def run():
        x, l = x0.clone().requires_grad_(True), l0.clone().requires_grad_(True)
        y, h = norm(x, x0)
        weight, _, place, source, _ = route(l)
        out = m.RunCombineFunction.apply(m.RunGatherFunction.apply(y, place, source), place, source, weight, h)
        first = torch.autograd.grad(out, (x, l, norm.weight), dy, retain_graph=True)
        return first, torch.autograd.grad(out, (x, l, norm.weight), dy)

    want, again = run()
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    with torch.autograd.graph.save_on_cpu():
        assert all(torch.equal(a, b) for a, b in zip(run()[0], want))
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.cpu()), pytest.raises(Exception):
        run()


def test_modules_refuse():
    from paper_2312_03415_amd import module as m
    rl = _rl()
    bf = torch.bfloat16
    t = lambda *s, dtype=bf: torch.zeros(s, dtype=dtype, device="cuda")
    norm, route = m.RunRMSNorm(64), m.RunRouter(8, 2)
    for bad in (t(3, 72), t(3, 64, dtype=torch.float16), t(3, 64).cpu()):
        with pytest.raises((ValueError, rl.RunLoRAError)):
            norm(bad)
    for residual in (t(4, 64), t(3, 64, dtype=torch.float32), t(3, 64).cpu()):
        with pytest.raises((ValueError, rl.RunLoRAError)):
            norm(t(3, 64), residual)
    for bad in (t(3, 9), t(3, 2, 8), t(3, 8).cpu()):
        with pytest.raises((ValueError, rl.RunLoRAError)):
            route(bad)
    with pytest.raises(rl.RunLoRAError):
        m.RunRouteFunction.apply(t(3, 8), rl.Route(8, 9), None)
    with pytest.raises((KeyError, ValueError, rl.RunLoRAError)):
        route(t(3, 8, dtype=torch.int32))
    weight, _, place, source, _ = route(t(5, 8))
    for bad in ((t(4, 64), place, source), (t(5, 64), place.long(), source), (t(5, 64), place, source[:-1]), (t(5, 60), place, source)):
        with pytest.raises((ValueError, rl.RunLoRAError)):
            m.RunGatherFunction.apply(*bad)
    rows = t(10, 64)
    for bad in ((rows[:9], place, source, weight, None), (rows, place, source, weight.double(), None), (rows, place, source, weight, t(4, 64)),
                (rows, place, source, weight[:, :1], None), (rows, place[:, :1].contiguous(), source, weight, None)):
        with pytest.raises((ValueError, rl.RunLoRAError)):
            m.RunCombineFunction.apply(*bad)


def test_streams_and_threads():
    """Training passes at once from several threads, each on a stream of its own, give the bits of one alone."""
    import threading
    from paper_2312_03415_amd import module as m
    n, d, E, top = 333, 264, 24, 4
    norm, route = m.RunRMSNorm(d, trainable=True), m.RunRouter(E, top, "sigmoid", groups=4, groups_kept=2, group_top=2, balance=True)
    router = torch.randn(d, E, generator=gen(2), device="cuda") / 8

    def work(seed):
        g = gen(seed)
        x, r, dy = (torch.randn(n, d, generator=g, device="cuda").bfloat16() for _ in range(3))
        out = []
        for _ in range(5):
            a, b = x.clone().requires_grad_(True), r.clone().requires_grad_(True)
            y, h, rows = norm(a, b, rows=True)
            weight, expert, place, source, ends = route(y.float() @ router)
            o = m.RunCombineFunction.apply(m.RunGatherFunction.apply(y, place, source), place, source, weight, h)
            out = [o, expert, ends, rows.values(), *torch.autograd.grad(o, (a, b, norm.weight), dy)]
        return [t.detach() for t in out]

    want = [work(s) for s in range(4)]
    torch.cuda.synchronize()
    got, streams = [None] * 4, [torch.cuda.Stream() for _ in range(4)]

    def run(k):
        with torch.cuda.stream(streams[k]):
            got[k] = work(k)
            streams[k].synchronize()

    threads = [threading.Thread(target=run, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for k in range(4):
        assert got[k] is not None and all(torch.equal(a, b) for a, b in zip(got[k], want[k])), k


def test_router_module_options():
    """What RunRouter is asked for reaches the routing; a model's conversion leaves the choice to the balance bias as it then is."""
    from paper_2312_03415_amd.module import RunRouter
    l = logits(90, 48, "f32", 12)
    how = dict(score="sigmoid", renormalise=False, groups=6, groups_kept=2, group_top=2, scale=2.5)
    route = RunRouter(48, 5, balance=True, **how)
    with torch.no_grad():
        route.bias.normal_(0, 0.1)
    assert "bias" in route.state_dict()
    for module in (route, route.bfloat16()):
        want = ref.Routing(to_f64(l), 5, bias=to_f64(module.bias), **how)
        weight, expert, place, source, ends = module(l)
        assert np.array_equal(expert.cpu().numpy(), want.expert) and np.array_equal(place.cpu().numpy(), want.place)
        close("weight", weight, want.weight, want.weight_bound())


def test_empty_batches():
    from paper_2312_03415_amd.module import RunCombineFunction, RunGatherFunction, RunRouter
    l = torch.empty(0, 8, device="cuda", requires_grad=True)
    weight, expert, place, source, ends = RunRouter(8, 2)(l)
    assert weight.shape == (0, 2) and not ends.any()
    x = torch.empty(0, 16, device="cuda", requires_grad=True)
    y = RunCombineFunction.apply(RunGatherFunction.apply(x, place, source), place, source, weight, None)
    gx, gl = torch.autograd.grad(y.sum() + weight.sum(), (x, l))
    assert gx.shape == (0, 16) and gl.shape == (0, 8)


def test_8bit_linear_takes_the_norms_rows():
    from paper_2312_03415_amd.module import RunLoRAFp8Linear, RunRMSNorm
    torch.manual_seed(0)
    layer = RunLoRAFp8Linear.from_linear(torch.nn.Linear(272, 144).bfloat16().cuda(), r=8, alpha=16)
    with torch.no_grad():
        layer.lora_B.normal_()
    norm = RunRMSNorm(272)
    for n in (3, 200):
        x = torch.randn(n, 2, 272, device="cuda").bfloat16().requires_grad_(True)
        dy = torch.randn(n, 2, 144, device="cuda").bfloat16()
        h, rows = norm(x, rows=True)
        a, b = layer(h, rows), layer(norm(x))
        assert torch.equal(a, b)
        leaves = (x, layer.lora_A, layer.lora_B)
        assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(a, leaves, dy), torch.autograd.grad(b, leaves, dy)))
    with pytest.raises(_rl().RunLoRAError):
        layer(norm(x)[:1], rows)
