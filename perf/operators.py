"""Adapted layers over a frozen weight in 8-bit floating point and over stacks of expert weights: what is timed, in plain
torch (own = False) and through the framework's entry points (own = True).

    layer    Y = Q(X) W + bias + s (X A) B                       W [i, o] e4m3, one power-of-two scale per 128 x 128 block
    experts  Y_t = X_t W_e + bias_e + s (X_t A_e) B_e            row t of expert e: rows ends[e-1] .. ends[e] - 1
             (X_t quantised like the layer's where W is e4m3)    W [E, i, o] in the activations' type or e4m3

Q(.) rounds each row's blocks of 128 columns to e4m3 with a power-of-two scale.  A training pass also returns
    dX = Q(dY) W^T + s (dY B^T) A^T      (dY itself where W is not e4m3),
    dA = s X^T (dY B^T),  dB = s (X A)^T dY      per expert.

    kind      pass     a pass returns
    layer     serve    y                       binding.runlora_forward on an Fp8Weight, into kept buffers
    layer     train    y, dx, dA, dB           RunLoRAFp8Function forward + backward
    experts   serve    y                       binding.runlora_experts_forward, into kept buffers
    experts   train    y, dx, dA, dB           RunLoRAExpertsFunction forward + backward

Values are those such layers meet: X ~ N(0, 1) with one channel in a hundred ten times as large, dY ~ N(0, 1) with one row
in eight zero (tokens the loss leaves out), W, A ~ N(0, 1/i), B ~ N(0, 0.1/r); experts' shares are uneven and some experts
may get no row at all.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _case(kind, mode, n, i, o, r, experts=1, weight="fp8", dtype="bf16", bias=False, name=None):
    c = dict(kind=kind, mode=mode, n=n, i=i, o=o, r=r, experts=experts, weight=weight, dtype=dtype, bias=bias)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token through an attention projection while generating: latency of a single small call
        _case("layer", "serve", 1, 4096, 4096, 16, name="layer_serve_1x4096x4096"),
        # 48 sequences generating one token each, the wide projection of a gated MLP
        _case("layer", "serve", 48, 4096, 11008, 32, name="layer_serve_48x4096x11008"),
        # an unpadded batch and widths that end inside a scale block, fp16, with a bias
        _case("layer", "train", 1237, 2064, 5456, 24, dtype="f16", bias=True, name="layer_train_f16_1237x2064x5456"),
        # the large workload's MLP projection
        _case("layer", "train", 8192, 4096, 11008, 32, name="layer_train_8192x4096x11008"),
        # eight tokens sent to two of eight experts each while generating
        _case("experts", "serve", 16, 2048, 8192, 16, 8, "dense", name="experts_serve_16x2048x8192_e8"),
        # a short ragged batch, more experts than tiles need, odd widths, fp16, biases
        _case("experts", "train", 999, 1032, 2744, 8, 12, "dense", "f16", True, name="experts_train_f16_999x1032x2744_e12"),
        # a training batch on the middle-sized workload's widths
        _case("experts", "train", 8192, 2048, 8192, 16, 8, "dense", name="experts_train_8192x2048x8192_e8"),
        # a large batch over square projections
        _case("experts", "train", 16384, 4096, 4096, 32, 16, "dense", name="experts_train_16384x4096x4096_e16"),
        # 32 tokens sent to two of sixteen 8-bit experts each
        _case("experts", "serve", 64, 4096, 11008, 16, 16, name="experts_fp8_serve_64x4096x11008_e16"),
        # reading a prompt of 1000 tokens, two experts each
        _case("experts", "serve", 2000, 4096, 4096, 64, 8, name="experts_fp8_serve_2000x4096x4096_e8"),
        # many experts with few rows each
        _case("experts", "train", 4096, 2048, 8192, 16, 64, name="experts_fp8_train_4096x2048x8192_e64"),
        # the largest: a training batch over the wide projection, high rank
        _case("experts", "train", 16384, 4096, 11008, 128, 8, name="experts_fp8_train_16384x4096x11008_e8"),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over its logarithm."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["layer", "experts", "experts"])
    weight = "fp8" if kind == "layer" else rng.choice(["fp8", "dense"])
    mode = rng.choice(["serve", "train", "train"])
    experts = 1 if kind == "layer" else _log(rng, 2, 64)
    step = rng.choice([16 if weight == "fp8" else 8, 256])
    i, o = _log(rng, 768, 8192, step), _log(rng, 768, 11008, step)
    n = _log(rng, 1, 3000) if mode == "serve" else _log(rng, 200, 16384)
    r = rng.choice([8, 16, 24, 32, 48, 64, 128])
    while n * i * o > 7.0e11 or experts * i * o > 1.2e9:
        if experts * i * o > 1.2e9:
            experts = max(1, experts // 2)
        else:
            n //= 2
    return _case(kind, mode, n, i, o, r, experts, weight, rng.choice(["bf16", "bf16", "f16"]), rng.random() < 0.4)


# ---- inputs ------------------------------------------------------------------------------------------

def _scale(case):
    return 2.0  # alpha / r of adapters with alpha = 2 r


def _ends(case, g):
    """Cumulative row counts of the experts: uneven shares, drawn row by row."""
    n, e = case["n"], case["experts"]
    share = torch.softmax(0.7 * torch.randn(e, generator=g), dim=0)
    return torch.bincount(torch.multinomial(share, n, replacement=True, generator=g), minlength=e).cumsum(0)


def _quantise_weight(w):
    """[E, i, o] floats -> e4m3 bytes [E, i, o] and scale bytes [E, ceil(i/128), ceil(o/128)] (value = e4m3 * 2^(byte - 127))."""
    e, i, o = w.shape
    ib, ob = (i + 127) // 128, (o + 127) // 128
    p = torch.zeros((e, ib * 128, ob * 128), device=w.device)
    p[:, :i, :o] = w
    p = p.view(e, ib, 128, ob, 128)
    m, x = torch.frexp(p.abs().amax(dim=(2, 4)))
    x = torch.where(m > 0, torch.clamp(x - torch.where(m > 0.875, 8, 9), min=-127), torch.zeros_like(x))
    q = (p * torch.exp2(-x.float())[:, :, None, :, None]).view(e, ib * 128, ob * 128)[:, :i, :o]
    return q.to(torch.float8_e4m3fn).contiguous().view(torch.uint8), (x + 127).to(torch.uint8)


def _inputs(case, seed):
    """Everything a pass reads, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, i, o, r, e = case["n"], case["i"], case["o"], case["r"], case["experts"]
    dt = DTYPES[case["dtype"]]

    def normal(shape, var):
        return torch.randn(shape, generator=g, device="cuda") * math.sqrt(var)

    x = normal((n, i), 1.0)
    x[:, torch.randint(0, i, (i // 100,), generator=g, device="cuda")] *= 10.0
    t = dict(X=x.to(dt), A=normal((e, i, r), 1.0 / i).to(dt), B=normal((e, r, o), 0.1 / r).to(dt))
    if case["weight"] == "fp8":
        q = [_quantise_weight(normal((1, i, o), 1.0 / i)) for _ in range(e)]
        t["W"], t["W_scales"] = (torch.cat([p[k] for p in q]) for k in (0, 1))
    else:
        t["W"] = torch.cat([normal((1, i, o), 1.0 / i).to(dt) for _ in range(e)])
    t["bias"] = normal((e, o), 0.01).to(dt) if case["bias"] else None
    if case["mode"] == "train":
        t["dY"] = (normal((n, o), 1.0) * (torch.rand((n, 1), generator=g, device="cuda") >= 0.125)).to(dt)
    t["ends"] = _ends(case, torch.Generator().manual_seed(seed))
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    ends = t.pop("ends")
    s = dict(case=case, t=t, rows=[0] + ends.tolist(), ends=ends.to(torch.int32).cuda())
    if case["kind"] == "layer":
        for k in ("A", "B", "W", "W_scales", "bias"):
            t[k] = t[k][0] if t[k] is not None else None
    if own:
        from paper_2312_03415_amd import binding as rl
        n, i, o, r, e = case["n"], case["i"], case["o"], case["r"], case["experts"]
        if case["weight"] == "fp8":
            t["W"] = rl.Fp8Weight(t["W"], t.pop("W_scales"), i, o)
        if case["mode"] == "serve":
            # the buffers a serving loop keeps
            s["y"] = torch.empty((n, o), dtype=t["X"].dtype, device="cuda")
            code = rl.dtype_code(t["X"].dtype)
            w_code = rl.RL_FP8_B128 if case["weight"] == "fp8" else code
            size = (rl.runlora_workspace_bytes(rl.FWD1, -1, n, i, o, r, code, w_code) if case["kind"] == "layer"
                    else rl.runlora_experts_workspace_bytes(False, n, e, i, o, r, code, w_code))
            s["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    if case["mode"] == "train":
        for k in ("X", "A", "B"):
            t[k].requires_grad_(True)
    return s


# ---- one pass ------------------------------------------------------------------------------------------

def _round_blocks(x):
    """Q(x) in 32 bits: blocks of 128 columns of a row to e4m3 times the smallest power of two that holds them."""
    n, k = x.shape
    p = torch.zeros((n, (k + 127) // 128 * 128), device=x.device)
    p[:, :k] = x
    p = p.view(n, -1, 128)
    m, e = torch.frexp(p.abs().amax(dim=2, keepdim=True))
    e = torch.clamp(e - torch.where(m > 0.875, 8, 9), min=-127).float()
    q = (p * torch.exp2(-e)).to(torch.float8_e4m3fn).float() * torch.exp2(e)
    return torch.where(m > 0, q, torch.zeros_like(q)).view(n, -1)[:, :k]


def _weight(t, e):
    """Expert e's W in 32 bits."""
    w = t["W"] if t["W"].dim() == 2 else t["W"][e]
    if "W_scales" not in t:
        return w.float()
    i, o = w.shape
    sc = t["W_scales"] if t["W_scales"].dim() == 2 else t["W_scales"][e]
    sc = torch.exp2(sc.float() - 127.0).repeat_interleave(128, 0)[:i].repeat_interleave(128, 1)[:, :o]
    return w.view(torch.float8_e4m3fn).float() * sc


def _plain(state):
    case, t, rows, s = state["case"], state["t"], state["rows"], _scale(state["case"])
    train, fp8 = case["mode"] == "train", case["weight"] == "fp8"
    dt, one = t["X"].dtype, case["kind"] == "layer"
    X = t["X"].detach().float()
    Xq = _round_blocks(X) if fp8 else X
    Y = torch.empty((case["n"], case["o"]), device="cuda")
    if train:
        dY = t["dY"].float()
        dYq = _round_blocks(dY) if fp8 else dY
        dX = torch.empty_like(X)
        dA = torch.zeros(t["A"].shape, device="cuda")
        dB = torch.zeros(t["B"].shape, device="cuda")
    for e in range(case["experts"]):
        a, b = rows[e], rows[e + 1]
        if a == b:
            continue
        W = _weight(t, e)
        A, B = (t[k].detach() if one else t[k].detach()[e] for k in ("A", "B"))
        A, B = A.float(), B.float()
        T = s * (X[a:b] @ A)
        Y[a:b] = Xq[a:b] @ W + T @ B
        if case["bias"]:
            Y[a:b] += (t["bias"] if one else t["bias"][e]).float()
        if train:
            Z = s * (dY[a:b] @ B.t())
            dX[a:b] = dYq[a:b] @ W.t() + Z @ A.t()
            (dA if one else dA[e]).copy_(X[a:b].t() @ Z)
            (dB if one else dB[e]).copy_(T.t() @ dY[a:b])
    return (Y.to(dt), dX.to(dt), dA.to(dt), dB.to(dt)) if train else Y.to(dt)


def run(state):
    if not own:
        return _plain(state)
    from paper_2312_03415_amd import binding as rl
    case, t, s = state["case"], state["t"], _scale(state["case"])
    if case["mode"] == "serve":
        if case["kind"] == "layer":
            rl.runlora_forward(rl.FWD1, t["X"], t["W"], t["A"], t["B"], state["y"], rl.new_saved(), workspace=state["ws"], scale=s,
                               bias=t["bias"])
        else:
            rl.runlora_experts_forward(t["X"], state["ends"], t["W"], t["A"], t["B"], state["y"], workspace=state["ws"], scale=s,
                                       bias=t["bias"])
        return state["y"]
    from paper_2312_03415_amd.module import RunLoRAExpertsFunction, RunLoRAFp8Function
    if case["kind"] == "layer":
        y = RunLoRAFp8Function.apply(t["X"], t["W"], t["A"], t["B"], t["bias"], s)
    else:
        y = RunLoRAExpertsFunction.apply(t["X"], state["ends"], t["W"], t["A"], t["B"], t["bias"], s)
    return (y.detach(),) + torch.autograd.grad(y, (t["X"], t["A"], t["B"]), t["dY"])


# ---- what a pass needs, and what it should give ---------------------------------------------------------

def work(case):
    n, i, o, r, e = case["n"], case["i"], case["o"], case["r"], case["experts"]
    used = e * (1.0 - (1.0 - 1.0 / e) ** n)  # experts that get a row, at even shares
    w = used * i * o * (1.0 + 1.0 / 16384 if case["weight"] == "fp8" else 2.0)
    factors = used * 2.0 * r * (i + o)
    fwd = 2.0 * n * (i * o + r * (i + o))
    if case["mode"] == "serve":
        return {"bytes": 2.0 * n * (i + o) + w + factors, "flops": fwd}
    # X, dY in, Y, dX out, the factors and their gradients; with X A kept: dY B^T, (.) A^T, dA and dB
    return {"bytes": 4.0 * n * (i + o) + w + factors + e * 2.0 * r * (i + o), "flops": fwd + 2.0 * n * (i * o + 2 * r * (i + o))}


def _nearest(v):
    """Nearest e4m3 value (ties to even) of float64 values of magnitude <= 448: steps of 2^(floor(log2 |v|) - 3), at least 2^-9."""
    step = torch.exp2(torch.clamp(torch.frexp(v)[1] - 1, min=-6).double() - 3)
    return torch.round(v / step) * step


def _blocks64(x):
    n, k = x.shape
    out = torch.empty_like(x)
    for c in range(0, k, 128):
        p = x[:, c:c + 128]
        top = p.abs().amax(dim=1, keepdim=True)
        # the smallest power of two >= top / 448, by comparison with its neighbour
        e = torch.floor(torch.log2(torch.where(top > 0, top / 448.0, torch.ones_like(top))))
        e = torch.clamp(torch.where(torch.exp2(e) * 448.0 >= top, e, e + 1), min=-127)
        out[:, c:c + 128] = _nearest(p * torch.exp2(-e)) * torch.exp2(e)
    return out


def exact(case, seed):
    t = _inputs(case, seed)
    s, n, i, o = _scale(case), case["n"], case["i"], case["o"]
    train, fp8 = case["mode"] == "train", case["weight"] == "fp8"
    X = t["X"].double()
    Xq = _blocks64(X) if fp8 else X
    Y = torch.empty((n, o), dtype=torch.float64, device="cuda")
    if train:
        dY = t["dY"].double()
        dYq = _blocks64(dY) if fp8 else dY
        dX = torch.empty_like(X)
        dA = torch.zeros(t["A"].shape, dtype=torch.float64, device="cuda")
        dB = torch.zeros(t["B"].shape, dtype=torch.float64, device="cuda")
    lo = 0
    for e, hi in enumerate(t["ends"].tolist()):
        if hi > lo:
            if fp8:
                k = torch.exp2(t["W_scales"][e].double() - 127)
                W = t["W"][e].view(torch.float8_e4m3fn).double()
                W = W * k[torch.arange(i, device="cuda") // 128][:, torch.arange(o, device="cuda") // 128]
            else:
                W = t["W"][e].double()
            A, B = t["A"][e].double(), t["B"][e].double()
            Y[lo:hi] = Xq[lo:hi] @ W + s * ((X[lo:hi] @ A) @ B)
            if case["bias"]:
                Y[lo:hi] += t["bias"][e].double()
            if train:
                dX[lo:hi] = dYq[lo:hi] @ W.t() + s * ((dY[lo:hi] @ B.t()) @ A.t())
                dA[e] = s * (X[lo:hi].t() @ (dY[lo:hi] @ B.t()))
                dB[e] = s * ((X[lo:hi] @ A).t() @ dY[lo:hi])
        lo = hi
    if not train:
        return Y
    one = case["kind"] == "layer"
    return Y, dX, dA[0] if one else dA, dB[0] if one else dB
