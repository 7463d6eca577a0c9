"""Long contractions over experts and 8-bit weights.  Output tiles of the large grouped kernel whose K tiles are dealt out to several workgroups, in either
direction, with experts, rows behind the last one's, adapters behind the last run only, and e4m3 runs on both sides of the 64th K tile (where a wave
changes the register that W's scales are in); and the smaller tiles, which read W's scales again every 64 K tiles.  What every case here runs on is
checked on the host (test_experts_plans.py)."""
import numpy as np
import pytest

import experts_oracle as ref
from helpers import TOL

torch = pytest.importorskip("torch")

# (rows, experts, d_in, d_out, rank, rows per expert, output that splits, weights)
CASES = [
    (4200, 3, 11280, 4112, 40, "rest", "Y", ("dense", "fp8")),
    (4200, 3, 4112, 11280, 136, "rest", "dX", ("dense", "fp8")),
    (4300, 2, 16272, 4112, 72, "uneven", "Y", ("dense", "fp8")),      # runs that begin behind K tile 64, and one that crosses it
    (4300, 2, 4112, 16272, 72, "uneven", "dX", ("dense", "fp8")),
    (1200, 2, 8208, 2576, 24, "uneven", "Y", ("dense",)),             # less than half a round of tiles: all of them split
    (1200, 2, 2576, 8208, 24, "uneven", "dX", ("dense",)),
    (700, 3, 8208, 4112, 200, "rest", "Y", ("dense",)),
    (700, 3, 4112, 8208, 200, "rest", "dX", ("dense",)),
]
PARAMS = [pytest.param(*c[:-1], w, id=f"{c[0]}x{c[2]}x{c[3]}-{c[6]}-{w}") for c in CASES for w in c[-1]]


def counts(n, experts, kind):
    return ref.counts(kind, n, experts, np.random.default_rng(n))


def rounded_rows(x):
    """Rows of float64 x rounded to e4m3 in blocks of 128 columns (no zero blocks, infinities or NaN here)."""
    n, k = x.shape
    p = torch.zeros((n, -(-k // 128) * 128), dtype=torch.float64, device="cuda")
    p[:, :k] = x
    p = p.view(n, -1, 128)
    m, e = torch.frexp(p.abs().amax(2, keepdim=True))
    e = (e - torch.where(m > 0.875, 8, 9)).double()
    return ((p * torch.exp2(-e)).float().to(torch.float8_e4m3fn).double() * torch.exp2(e)).view(n, -1)[:, :k].contiguous()


def adapted(rows, rounded, W, F, G, s, h, sums):
    """rounded W + s (rows F) G in 64 bits, and the bound of experts_oracle.py per element."""
    t = s * (rows @ F)
    at = 2.0 ** -20 * s * (rows.abs() @ F.abs())
    want = rounded @ W + t @ G
    factor = torch.minimum(h * (t.abs() @ G.abs()), 6 * h / 3 ** 0.5 * torch.sqrt((t * t) @ (G * G)))
    return want, sums * (rounded.abs() @ W.abs()) + factor + at @ G.abs()


def block_powers(g, rows, cols, block):
    """Powers of two, one for every `block` columns (and `block[0]` rows): neighbouring blocks get other scales."""
    a, b = -(-rows // block[0]), -(-cols // block[1])
    e = torch.randint(-2, 3, (a, b), generator=g, device="cuda").float()
    return torch.exp2(e).repeat_interleave(block[0], 0)[:rows].repeat_interleave(block[1], 1)[:, :cols]


def check(n, experts, i, o, r, kind, side, weight):
    """One output, every element against a 64-bit product on the device, and the same bits when called again, on scratch that holds NaN."""
    from paper_2312_03415_amd import binding as rl
    s, td, h, fp8 = 1.5, torch.bfloat16, 2.0 ** -8, weight == "fp8"
    g = torch.Generator(device="cuda").manual_seed(n + i)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    forward = side == "Y"
    rows = randn(n, i if forward else o)
    rows = (rows * block_powers(g, *rows.shape, (1, 128))).to(td)
    A, B, bias = (randn(experts, i, r) * i ** -0.5).to(td), (randn(experts, r, o) * (0.5 / r) ** 0.5).to(td), randn(experts, o).to(td)
    W = randn(experts, i, o) * i ** -0.5
    for e in range(experts):
        W[e] *= block_powers(g, i, o, (128, 128))
    W = W.to(td)
    if fp8:
        W = rl.Fp8Weight.quantize(W)
        value = lambda e: (W.data[e].view(torch.float8_e4m3fn).double() *
                           torch.exp2(W.scales[e].double() - 127).repeat_interleave(128, 0)[:i].repeat_interleave(128, 1)[:, :o])
    else:
        value = lambda e: W[e].double()
    ends_host = np.cumsum(counts(n, experts, kind))
    ends = torch.from_numpy(ends_host.astype(np.int32)).cuda()
    size = rl.runlora_experts_workspace_bytes(not forward, n, experts, i, o, r, rl.RL_BF16, rl.RL_FP8_B128 if fp8 else None)
    outs = []
    for _ in range(2):
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        out = torch.full((n, o if forward else i), float("nan"), dtype=td, device="cuda")
        if forward:
            rl.runlora_experts_forward(rows, ends, W, A, B, out, workspace=ws, scale=s, bias=bias)
        else:
            rl.runlora_experts_backward(rows, None, ends, W, A, B, out, None, None, workspace=ws, scale=s)
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
    got, lo, t = outs[0].double(), 0, lambda m: m.t().contiguous()
    for e, hi in enumerate(ends_host):
        if hi == lo:
            continue
        x = rows[lo:hi].double()
        xq = rounded_rows(x) if fp8 else x
        F, G, w = A[e].double(), B[e].double(), value(e)
        want, bound = adapted(x, xq, w if forward else t(w), F if forward else t(G), G if forward else t(F), s, h, 2.0 ** -12 if fp8 else 2.0 ** -20)
        if forward:
            want += bias[e].double()
        bound += h * want.abs()
        part = got[lo:hi]
        assert torch.isfinite(part).all()
        assert float((part - want).norm() / want.norm()) <= TOL["bf16"]
        over = (part - want).abs() > bound
        assert not bool(over.any()), (e, int(over.sum()), float(((part - want).abs() / bound).max()))
        lo = hi
    assert not bool(outs[0][lo:].any())      # rows behind the last expert's: zeros


@pytest.mark.gpu
@pytest.mark.parametrize("n,experts,i,o,r,kind,side,weight", PARAMS)
def test_split_tiles(n, experts, i, o, r, kind, side, weight):
    check(n, experts, i, o, r, kind, side, weight)


# e4m3 on the smaller tiles with more K tiles than a wave keeps scales of W for (64), and with a K that the large kernel does not take (above 16384):
# (rows, experts, d_in, d_out, rank, rows per expert, output, tile's rows; 0: few rows, in one slice)
LONG = [
    (40, 2, 8336, 5504, 16, "uneven", "Y", 0),
    (100, 1, 8336, 272, 16, "even", "Y", 32),
    (100, 3, 272, 16528, 24, "uneven", "dX", 32),
    (300, 1, 8336, 4240, 40, "even", "Y", 64),
    (300, 1, 4240, 16528, 8, "even", "dX", 64),
    (1200, 2, 8336, 4240, 16, "uneven", "Y", 128),
    (2400, 1, 16528, 4240, 72, "even", "Y", 128),
    (2400, 3, 4240, 16528, 16, "rest", "dX", 128),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n,experts,i,o,r,kind,side,tile", LONG)
def test_long_contractions_of_the_smaller_tiles(n, experts, i, o, r, kind, side, tile):
    check(n, experts, i, o, r, kind, side, "fp8")
