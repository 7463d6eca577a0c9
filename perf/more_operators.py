"""What stands between the layers of a block with routed experts: what is timed, in plain torch (own = False) and through the framework's
entry points (own = True).

    norm     h = x + residual, y = h / sqrt(mean(h^2) + eps) * gain, and y in e4m3 with a scale per 128 columns of a row
    route    logits [n, E] -> a token's experts and their weights, and the order of the rows sorted by expert
    gather   rows[place[t, j]] = x_t: every token's row to its experts
    combine  y_t = add_t + sum_j weight[t, j] rows[place[t, j]]: the experts' rows back

    kind      pass     a pass returns
    norm      serve    y, h, and the values that the 8-bit rows stand for      binding.runlora_rmsnorm_forward, into kept buffers
    norm      train    y, h, dx, d residual, d gain                            RunRMSNormFunction forward + backward
    route     serve    weight, expert, place, source, ends                     binding.runlora_route_forward, into kept buffers
    route     train    the same and d logits                                   RunRouteFunction forward + backward
    gather    serve    rows                                                    binding.runlora_gather_forward, into kept buffers
    gather    train    rows, dx                                                RunGatherFunction forward + backward
    combine   serve    y                                                       binding.runlora_combine_forward, into kept buffers
    combine   train    y, d rows, d weight                                     RunCombineFunction forward + backward

Routing.  Scores s are softmax(l) or sigmoid(l).  An expert is chosen by c = s + bias (without a bias by l, which has the order of s); a logit
of -infinity is never chosen (a padding token has nothing else).  With groups, a group of E / groups experts counts with the sum of its
`group_top` largest c, and experts outside the `kept` best groups are not chosen.  The top largest c are taken in falling order, equal ones by
index; what is missing is expert -1, weight 0, place -1.  weight = scale * s, divided by the sum over the chosen where `renorm`.  Copy (t, j) of
token t's row stands on row place[t, j] of the rows sorted by expert, in the order of t top + j within an expert; source is the inverse (-1 behind
the last row), and ends[e] is where expert e's rows end.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


def _norm(mode, n, d, dtype="bf16", residual=True, fp8=False, name=None):
    c = dict(kind="norm", mode=mode, n=n, d=d, dtype=dtype, residual=residual, fp8=fp8)
    return dict(c, name=name) if name else c


def _route(mode, n, experts, top, dtype="bf16", score="softmax", renorm=True, bias=False, groups=1, kept=1, group_top=1, scale=1.0, pad=False, name=None):
    c = dict(kind="route", mode=mode, n=n, experts=experts, top=top, dtype=dtype, score=score, renorm=renorm, bias=bias, groups=groups, kept=kept,
             group_top=group_top, scale=scale, pad=pad)
    return dict(c, name=name) if name else c


def _rows(kind, mode, n, d, top, experts, dtype="bf16", add=False, pad=False, name=None):
    c = dict(kind=kind, mode=mode, n=n, d=d, top=top, experts=experts, dtype=dtype, add=add, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token while generating, in front of 8-bit projections: latency of a single small call
        _norm("serve", 1, 4096, fp8=True, name="norm_serve_1x4096_fp8"),
        # a prompt in front of 8-bit projections
        _norm("serve", 8192, 4096, fp8=True, name="norm_serve_8192x4096_fp8"),
        # an unpadded batch of odd width in fp16, the first norm of a model: nothing to add yet
        _norm("train", 1237, 2056, "f16", residual=False, name="norm_train_f16_1237x2056"),
        # a large training batch on the wider workload's hidden size: the largest
        _norm("train", 16384, 5120, name="norm_train_16384x5120"),
        # eight tokens of a decoding batch over a few experts
        _route("serve", 8, 8, 2, name="route_serve_8x8_t2"),
        # a prompt of odd length over limited groups of experts, fp16 logits, weights that do not sum to one
        _route("serve", 1999, 120, 6, "f16", renorm=False, groups=8, kept=3, scale=16.0, name="route_serve_f16_1999x120_t6"),
        # a training batch over a middling number of experts
        _route("train", 8192, 64, 4, name="route_train_8192x64_t4"),
        # a large, padded training batch over many experts: sigmoid scores, balance bias, groups
        _route("train", 16384, 256, 8, "f32", "sigmoid", True, True, 8, 4, 2, 2.5, True, name="route_train_16384x256_t8"),
        # a decoding batch of 48 sequences sent to four of sixteen experts each
        _rows("gather", "serve", 48, 4096, 4, 16, name="gather_serve_48x4096_t4"),
        # a training batch to two of eight experts
        _rows("gather", "train", 8192, 4096, 2, 8, name="gather_train_8192x4096_t2"),
        # a prompt of odd length and width in fp16, added to the residual stream
        _rows("combine", "serve", 1237, 2056, 6, 120, "f16", add=True, name="combine_serve_f16_1237x2056_t6"),
        # a padded training batch to eight of 64 experts
        _rows("combine", "train", 8192, 2048, 8, 64, pad=True, name="combine_train_8192x2048_t8"),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over its logarithm."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["norm", "route", "gather", "combine"])
    mode = rng.choice(["serve", "train"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    n = _log(rng, 1, 4000) if mode == "serve" else _log(rng, 100, 16384)
    if kind == "norm":
        d = _log(rng, 64, 8192, rng.choice([8, 8, 128]))
        while n * d > 16384 * 5120:
            n //= 2
        return _norm(mode, n, d, dtype, rng.random() < 0.7, mode == "serve" and dtype != "f32" and rng.random() < 0.5)
    top = rng.randint(1, 8)
    pad = rng.random() < 0.3
    if kind == "route":
        score, grouped = rng.choice(["softmax", "sigmoid"]), rng.random() < 0.4
        groups = rng.choice([2, 4, 8]) if grouped else 1
        experts = _log(rng, max(top, 4 * groups), 384, groups)
        kept = rng.randint((top * groups + experts - 1) // experts, groups) if grouped else 1
        return _route(mode, n, experts, top, dtype, score, rng.random() < 0.6, rng.random() < 0.5, groups, kept, rng.choice([1, 2]) if grouped else 1,
                      rng.choice([1.0, 2.5]), pad)
    d = _log(rng, 256, 8192, rng.choice([8, 128]))
    while n * d * top > 16384 * 2048 * 8:
        n //= 2
    return _rows(kind, mode, n, d, top, _log(rng, max(top, 4), 256), dtype, kind == "combine" and rng.random() < 0.4, pad)


# ---- inputs ------------------------------------------------------------------------------------------

def _choices(case, g):
    """[n, top] different experts a token, the popular ones more often; a padding token has none (-1)."""
    n, e = case["n"], case["experts"]
    l = torch.randn((n, e), generator=g, device="cuda") + 0.7 * torch.randn((1, e), generator=g, device="cuda")
    expert = l.topk(case["top"], dim=1).indices
    if case["pad"]:
        expert[torch.rand(n, generator=g, device="cuda") < 1.0 / 16] = -1
    return expert


def _order(expert, experts):
    """place [n, top], source [n top] and ends [experts] of chosen experts (-1: none), as int32."""
    n, top = expert.shape
    flat = torch.where(expert < 0, experts, expert).flatten().long()
    rows = torch.arange(n * top, device=expert.device)
    by_expert, order = flat.sort(stable=True)
    place = torch.empty_like(order)
    place[order] = rows
    placed = by_expert < experts
    ends = torch.bincount(flat, minlength=experts + 1)[:experts].cumsum(0)
    return (torch.where(flat < experts, place, -1).view(n, top).int(), torch.where(placed, order, -1).int(), ends.int())


def _inputs(case, seed):
    """Everything a pass reads, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, dt, train = case["n"], DTYPES[case["dtype"]], case["mode"] == "train"
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    if case["kind"] == "norm":
        d = case["d"]
        x = normal(n, d)
        x[:, torch.randint(0, d, (1 + d // 100,), generator=g, device="cuda")] *= 10.0  # the few large channels of a residual stream
        t = dict(x=x.to(dt), gain=(1.0 + 0.1 * normal(d)).to(dt))
        t["residual"] = (2.0 * normal(n, d)).to(dt) if case["residual"] else None
        if train:
            t["dy"] = normal(n, d).to(dt)
            t["dh"] = normal(n, d).to(dt) if case["residual"] else None
        return t
    if case["kind"] == "route":
        e = case["experts"]
        l = 1.5 * normal(n, e) + 0.7 * normal(1, e)  # some experts are popular
        if case["pad"]:
            l[torch.rand(n, generator=g, device="cuda") < 1.0 / 16] = -math.inf
        t = dict(logits=l.to(dt), bias=0.05 * normal(e) if case["bias"] else None)
        if train:
            t["dweight"] = normal(n, case["top"])
        return t
    d, top = case["d"], case["top"]
    expert = _choices(case, g)
    place, source, _ = _order(expert, case["experts"])
    t = dict(place=place, source=source)
    if case["kind"] == "gather":
        t["x"] = normal(n, d).to(dt)
        if train:
            t["drows"] = normal(n * top, d).to(dt)
        return t
    t["rows"] = normal(n * top, d).to(dt)
    t["weight"] = torch.softmax(normal(n, top), dim=1) * (place >= 0)
    t["add"] = normal(n, d).to(dt) if case["add"] else None
    if train:
        t["dy"] = normal(n, d).to(dt)
    return t


def _plan(case):
    from paper_2312_03415_amd import binding as rl
    return rl.Route(case["experts"], case["top"], score=case["score"], renormalise=case["renorm"], groups=case["groups"], groups_kept=case["kept"],
                    group_top=case["group_top"], scale=case["scale"])


def prepare(case, seed):
    t = _inputs(case, seed)
    s = dict(case=case, t=t)
    if own:
        # the buffers a serving loop keeps
        from paper_2312_03415_amd import binding as rl
        n, kind = case["n"], case["kind"]
        empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")
        if kind == "route":
            s["route"] = _plan(case)
        if case["mode"] == "serve":
            if kind == "norm":
                s["y"] = torch.empty_like(t["x"])
                s["h"] = torch.empty_like(t["x"]) if case["residual"] else None
                s["rows8"] = rl.Fp8Rows.empty(n, case["d"], "cuda") if case["fp8"] else None
            elif kind == "route":
                top = case["top"]
                s["weight"], s["expert"], s["place"] = empty((n, top), torch.float32), empty((n, top), torch.int32), empty((n, top), torch.int32)
                s["source"], s["ends"] = empty((n * top,), torch.int32), empty((case["experts"],), torch.int32)
                s["ws"] = empty((max(256, rl.runlora_route_workspace_bytes(n, case["experts"], top)),), torch.uint8)
            elif kind == "gather":
                s["rows"] = empty((n * case["top"], case["d"]), t["x"].dtype)
            else:
                s["y"] = empty((n, case["d"]), t["rows"].dtype)
    if case["mode"] == "train":
        for k in {"norm": ("x", "residual", "gain"), "route": ("logits",), "gather": ("x",), "combine": ("rows", "weight")}[case["kind"]]:
            if t[k] is not None:
                t[k].requires_grad_(True)
    return s


# ---- one pass, in plain torch ------------------------------------------------------------------------------

def _round_blocks(x):
    """x with blocks of 128 columns of a row rounded to e4m3 times the smallest power of two that holds them."""
    n, k = x.shape
    p = torch.zeros((n, (k + 127) // 128 * 128), device=x.device)
    p[:, :k] = x
    p = p.view(n, -1, 128)
    m, e = torch.frexp(p.abs().amax(dim=2, keepdim=True))
    e = torch.clamp(e - torch.where(m > 0.875, 8, 9), min=-127).float()
    q = (p * torch.exp2(-e)).to(torch.float8_e4m3fn).float() * torch.exp2(e)
    return torch.where(m > 0, q, torch.zeros_like(q)).view(n, -1)[:, :k]


def _plain_norm(case, t):
    x, gain = t["x"].detach(), t["gain"].detach().float()
    dt = x.dtype
    # the residual stream is kept in the activations' type
    h = (x.float() + t["residual"].detach().float()).to(dt) if case["residual"] else x
    v = h.float()
    rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    xhat = v * rstd
    y = (xhat * gain).to(dt)
    if case["mode"] == "serve":
        out = (y,) + ((h,) if case["residual"] else ())
        return out + ((_round_blocks(y.float()).to(torch.bfloat16),) if case["fp8"] else ())
    dy = t["dy"].float()
    dn = dy * gain
    dx = rstd * (dn - xhat * (dn * xhat).mean(1, keepdim=True))
    dgain = (dy * xhat).sum(0).to(dt)
    if not case["residual"]:
        return y, dx.to(dt), dgain
    dx = (dx + t["dh"].float()).to(dt)
    return y, h, dx, dx, dgain


def _plain_route(case, t):
    n, e, top = case["n"], case["experts"], case["top"]
    # a choice between close scores is made in 64 bits
    l = t["logits"].detach().double()
    masked = torch.isinf(l) & (l < 0)
    some = ~masked.all(1, keepdim=True)
    if case["score"] == "softmax":
        p = torch.exp(l - torch.where(some, l.amax(1, keepdim=True), 0.0))
        s = torch.where(some, p / p.sum(1, keepdim=True), 0.0)
    else:
        s = torch.sigmoid(l)
    c = s if t["bias"] is None else s + t["bias"].double()
    c = torch.where(masked, -math.inf, c)
    key = c if t["bias"] is not None else l
    if case["groups"] > 1:
        best = c.view(n, case["groups"], -1).sort(dim=2, descending=True).values[:, :, :case["group_top"]]
        none = torch.isinf(best[:, :, 0])
        rank = torch.where(none, -math.inf, torch.where(torch.isinf(best), 0.0, best).sum(2))
        kept = rank.sort(dim=1, descending=True, stable=True).indices[:, :case["kept"]]
        out = torch.ones_like(rank, dtype=torch.bool).scatter_(1, kept, False)
        key = torch.where(out.repeat_interleave(e // case["groups"], 1), -math.inf, key)
    value, expert = (v[:, :top] for v in key.sort(dim=1, descending=True, stable=True))
    chosen = ~torch.isinf(value)
    lj, sj = l.gather(1, expert), s.gather(1, expert)
    if case["renorm"]:
        # scores over the largest of them: none vanishes
        a = lj if case["score"] == "softmax" else torch.nn.functional.logsigmoid(lj)
        a = torch.where(chosen, a, -math.inf)
        q = torch.exp(a - torch.where(chosen[:, :1], a.amax(1, keepdim=True), 0.0))
        q = torch.where(chosen, q / q.sum(1, keepdim=True), 0.0)
    else:
        q = torch.where(chosen, sj, 0.0)
    weight = (case["scale"] * q).float()
    expert = torch.where(chosen, expert, -1).int()
    place, source, ends = _order(expert, e)
    if case["mode"] == "serve":
        return weight, expert, place, source, ends
    dw = torch.where(chosen, case["scale"] * t["dweight"].double(), 0.0)
    at = torch.where(chosen, expert, 0).long()
    if case["renorm"]:
        dl = q * (dw - (dw * q).sum(1, keepdim=True))
        if case["score"] == "sigmoid":
            dl = dl * (1.0 - sj)
        dlogits = torch.zeros_like(l).scatter_add_(1, at, torch.where(chosen, dl, 0.0))
    elif case["score"] == "sigmoid":
        dlogits = torch.zeros_like(l).scatter_add_(1, at, torch.where(chosen, dw * sj * (1.0 - sj), 0.0))
    else:
        ds = torch.zeros_like(l).scatter_add_(1, at, dw)
        dlogits = s * (ds - (ds * s).sum(1, keepdim=True))
    return weight, expert, place, source, ends, dlogits.to(t["logits"].dtype)


def _plain_gather(case, t):
    x, place, top = t["x"].detach(), t["place"].long(), case["top"]
    n = case["n"]
    placed = t["source"] >= 0
    rows = torch.where(placed[:, None], x[torch.clamp(t["source"].long(), min=0) // top], 0.0)
    if case["mode"] == "serve":
        return rows
    back = t["drows"][torch.clamp(place, min=0).flatten()].float().view(n, top, -1)
    return rows, torch.where((place >= 0)[:, :, None], back, 0.0).sum(1).to(x.dtype)


def _plain_combine(case, t):
    rows, place, weight = t["rows"].detach(), t["place"].long(), t["weight"].detach()
    n, top, dt = case["n"], case["top"], t["rows"].dtype
    there = (place >= 0)[:, :, None]
    back = torch.where(there, rows[torch.clamp(place, min=0).flatten()].float().view(n, top, -1), 0.0)
    y = (back * weight[:, :, None]).sum(1)
    if case["add"]:
        y = y + t["add"].float()
    if case["mode"] == "serve":
        return y.to(dt)
    dy = t["dy"].float()
    dweight = (back * dy[:, None]).sum(2)
    source = t["source"].long()
    of = torch.clamp(source, min=0)
    drows = torch.where((source >= 0)[:, None], weight.flatten()[of][:, None] * dy[of // top], 0.0)
    return y.to(dt), drows.to(dt), dweight


_PLAIN = dict(norm=_plain_norm, route=_plain_route, gather=_plain_gather, combine=_plain_combine)


# ---- one pass --------------------------------------------------------------------------------------------

def _own_serve(state):
    from paper_2312_03415_amd import binding as rl
    case, t, s = state["case"], state["t"], state
    if case["kind"] == "norm":
        rl.runlora_rmsnorm_forward(t["x"], t["gain"], s["y"], eps=EPS, residual=t["residual"], H=s["h"], rows=s["rows8"])
        out = (s["y"],) + ((s["h"],) if case["residual"] else ())
        return out + ((s["rows8"].values(torch.bfloat16),) if case["fp8"] else ())
    if case["kind"] == "route":
        rl.runlora_route_forward(t["logits"], s["route"], s["weight"], s["expert"], s["place"], s["source"], s["ends"], bias=t["bias"], workspace=s["ws"])
        return s["weight"], s["expert"], s["place"], s["source"], s["ends"]
    if case["kind"] == "gather":
        rl.runlora_gather_forward(t["x"], t["place"], t["source"], s["rows"])
        return s["rows"]
    rl.runlora_combine_forward(t["rows"], t["place"], t["weight"], s["y"], add=t["add"])
    return s["y"]


def _own_train(state):
    from paper_2312_03415_amd import module as m
    case, t = state["case"], state["t"]
    if case["kind"] == "norm":
        if not case["residual"]:
            y = m.RunRMSNormFunction.apply(t["x"], t["gain"], EPS)
            return (y.detach(),) + torch.autograd.grad(y, (t["x"], t["gain"]), t["dy"])
        y, h = m.RunRMSNormFunction.apply(t["x"], t["gain"], EPS, t["residual"])
        return (y.detach(), h.detach()) + torch.autograd.grad((y, h), (t["x"], t["residual"], t["gain"]), (t["dy"], t["dh"]))
    if case["kind"] == "route":
        weight, expert, place, source, ends = m.RunRouteFunction.apply(t["logits"], state["route"], t["bias"])
        return (weight.detach(), expert, place, source, ends) + torch.autograd.grad(weight, t["logits"], t["dweight"])
    if case["kind"] == "gather":
        rows = m.RunGatherFunction.apply(t["x"], t["place"], t["source"])
        return (rows.detach(),) + torch.autograd.grad(rows, t["x"], t["drows"])
    y = m.RunCombineFunction.apply(t["rows"], t["place"], t["source"], t["weight"], t["add"])
    return (y.detach(),) + torch.autograd.grad(y, (t["rows"], t["weight"]), t["dy"])


def run(state):
    if own:
        return _own_serve(state) if state["case"]["mode"] == "serve" else _own_train(state)
    return _PLAIN[state["case"]["kind"]](state["case"], state["t"])


# ---- what a pass needs, and what it should give ---------------------------------------------------------

def work(case):
    n, train = case["n"], case["mode"] == "train"
    z = {"bf16": 2.0, "f16": 2.0, "f32": 4.0}[case["dtype"]]
    if case["kind"] == "norm":
        d = case["d"]
        # x and y; the residual and h; 8-bit y; dy and dx; dh
        moved = 2 + 2 * case["residual"] + (2 + case["residual"] if train else 0)
        return {"bytes": z * n * d * moved + (n * d * (1.0 + 1.0 / 128) if case["fp8"] else 0.0) + z * d * (2 if train else 1),
                "flops": n * d * (14.0 if train else 5.0)}
    top, e = case["top"], case["experts"]
    if case["kind"] == "route":
        # logits; weight, expert, place, source; the upstream gradient and that of the logits
        return {"bytes": z * n * e * (2 if train else 1) + n * top * (20.0 if train else 16.0) + 8.0 * e, "flops": n * e * (20.0 if train else 10.0)}
    d = case["d"]
    if case["kind"] == "gather":
        return {"bytes": (2 if train else 1) * z * n * d * (1 + top) + 8.0 * n * top, "flops": float(n * d * top) if train else 0.0}
    return {"bytes": z * n * d * ((1 + top + case["add"]) + (1 + top if train else 0)) + n * top * (16.0 if train else 8.0),
            "flops": n * d * top * (5.0 if train else 2.0)}


def _nearest(v):
    """Nearest e4m3 value (ties to even) of float64 values of magnitude <= 448: steps of 2^(floor(log2 |v|) - 3), at least 2^-9."""
    step = torch.exp2(torch.clamp(torch.frexp(v)[1] - 1, min=-6).double() - 3)
    return torch.round(v / step) * step


def _blocks64(x):
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], 128):
        p = x[:, c:c + 128]
        top = p.abs().amax(dim=1, keepdim=True)
        # the smallest power of two >= top / 448, by comparison with its neighbour
        e = torch.floor(torch.log2(torch.where(top > 0, top / 448.0, torch.ones_like(top))))
        e = torch.clamp(torch.where(torch.exp2(e) * 448.0 >= top, e, e + 1), min=-127)
        out[:, c:c + 128] = _nearest(p * torch.exp2(-e)) * torch.exp2(e)
    return out


def _exact_norm(case, t):
    n, d, dt = case["n"], case["d"], t["x"].dtype
    h = t["x"].double()
    if case["residual"]:
        h = (t["x"].float() + t["residual"].float()).to(dt).double()  # (the stream is kept in the activations' type)
    g = t["gain"].double()
    norm = torch.sqrt((h ** 2).sum(1) / d + EPS)[:, None]
    y = h / norm * g
    if case["mode"] == "serve":
        # the 8-bit rows are those of y as it is stored
        return (y,) + ((h,) if case["residual"] else ()) + ((_blocks64(y.to(dt).double()),) if case["fp8"] else ())
    dy = t["dy"].double()
    dx = dy * g / norm - h * ((dy * g * h).sum(1, keepdim=True) / (d * norm ** 3))
    dgain = (dy * h / norm).sum(0)
    if not case["residual"]:
        return y, dx, dgain
    dx = dx + t["dh"].double()
    return y, h, dx, dx, dgain


def _exact_route(case, t):
    n, e, top = case["n"], case["experts"], case["top"]
    l = t["logits"].double()
    open_ = l > -math.inf
    if case["score"] == "softmax":
        s = torch.nan_to_num(torch.softmax(l, 1), nan=0.0)
    else:
        s = 1.0 / (1.0 + torch.exp(-l))
    c = s.clone()
    if t["bias"] is not None:
        c += t["bias"].double()
    allowed = open_.clone()
    if case["groups"] > 1:
        size = e // case["groups"]
        rank = torch.full((n, case["groups"]), -math.inf, dtype=torch.float64, device="cuda")
        for k in range(case["groups"]):
            part, there = c[:, k * size:(k + 1) * size], open_[:, k * size:(k + 1) * size]
            left, total = there.clone(), torch.zeros(n, dtype=torch.float64, device="cuda")
            for _ in range(min(case["group_top"], size)):
                v = torch.where(left, part, -math.inf)
                m = v.amax(1)
                total += torch.where(m > -math.inf, m, 0.0)
                left &= ~((v == m[:, None]) & ((v == m[:, None]).cumsum(1) == 1))
            rank[:, k] = torch.where(there.any(1), total, -math.inf)
        # a group is kept if fewer than `kept` come before it
        index = torch.arange(case["groups"], device="cuda")
        before = (rank[:, None, :] > rank[:, :, None]) | ((rank[:, None, :] == rank[:, :, None]) & (index[None, None, :] < index[None, :, None]))
        allowed &= (before.sum(2) < case["kept"]).repeat_interleave(size, 1)
    key = c if t["bias"] is not None else l
    number = torch.arange(e, device="cuda")
    expert = torch.full((n, top), -1, dtype=torch.int64, device="cuda")
    sj = torch.zeros((n, top), dtype=torch.float64, device="cuda")
    for j in range(top):
        v = torch.where(allowed, key, -math.inf)
        first = torch.where(allowed & (v == v.amax(1, keepdim=True)), number, e).amin(1)
        ok = first < e
        at = torch.clamp(first, max=e - 1)[:, None]
        expert[:, j] = torch.where(ok, first, -1)
        sj[:, j] = torch.where(ok, s.gather(1, at)[:, 0], 0.0)
        allowed.scatter_(1, at, False)
    total = sj.sum(1, keepdim=True)
    q = torch.where(total > 0, sj / torch.where(total > 0, total, 1.0), 0.0) if case["renorm"] else sj
    weight = case["scale"] * q
    # a row stands behind all rows of lower experts and the earlier ones of its own
    flat = expert.flatten()
    one = (flat[:, None] == number).int()
    count = one.sum(0)
    start = count.cumsum(0) - count
    at = torch.clamp(flat, min=0)
    place = torch.where(flat >= 0, start[at] + one.cumsum(0).gather(1, at[:, None])[:, 0] - 1, -1)
    source = torch.full((n * top,), -1, dtype=torch.int64, device="cuda")
    source[place[place >= 0]] = torch.arange(n * top, device="cuda")[place >= 0]
    out = (weight, expert.int(), place.view(n, top).int(), source.int(), (start + count).int())
    if case["mode"] == "serve":
        return out
    dl = torch.zeros((n, e), dtype=torch.float64, device="cuda")
    dw = case["scale"] * t["dweight"].double()
    at = torch.clamp(expert, min=0)
    mean = (dw * q).sum(1, keepdim=True)
    for j in range(top):
        ok = expert[:, j] >= 0
        d = dw[:, j] * sj[:, j] if not case["renorm"] else q[:, j] * (dw[:, j] - mean[:, 0])
        if case["score"] == "sigmoid":
            d = d * (1.0 - sj[:, j])
        dl[torch.arange(n, device="cuda")[ok], at[ok, j]] += d[ok]
    if case["score"] == "softmax" and not case["renorm"]:
        dl -= s * mean
    return out + (dl,)


def _exact_rows(case, t):
    n, top = case["n"], case["top"]
    place, m = t["place"].long(), n * top
    if case["kind"] == "gather":
        x = t["x"].double()
        rows = torch.zeros((m, case["d"]), dtype=torch.float64, device="cuda")
        dx = torch.zeros_like(x)
        for j in range(top):
            ok = place[:, j] >= 0
            rows[place[ok, j]] = x[ok]
            if case["mode"] == "train":
                dx[ok] += t["drows"][place[ok, j]].double()
        return (rows, dx) if case["mode"] == "train" else rows
    y = t["add"].double() if case["add"] else torch.zeros((n, case["d"]), dtype=torch.float64, device="cuda")
    w = t["weight"].double()
    train = case["mode"] == "train"
    if train:
        dy = t["dy"].double()
        drows = torch.zeros((m, case["d"]), dtype=torch.float64, device="cuda")
        dweight = torch.zeros((n, top), dtype=torch.float64, device="cuda")
    for j in range(top):
        ok = place[:, j] >= 0
        r = t["rows"][place[ok, j]].double()
        y[ok] += w[ok, j][:, None] * r
        if train:
            drows[place[ok, j]] = w[ok, j][:, None] * dy[ok]
            dweight[ok, j] = (r * dy[ok]).sum(1)
    return (y, drows, dweight) if train else y


def exact(case, seed):
    t = _inputs(case, seed)
    return {"norm": _exact_norm, "route": _exact_route}.get(case["kind"], _exact_rows)(case, t)
