"""Layers over stacks of experts where rows, and experts' weights, lie more than 2^31 elements apart: sampled rows against the float64 reference
of experts_oracle.py (a row's result depends on no other row), and the sum over all rows in dA and dB against sums in 64 bits."""
import numpy as np
import pytest

import experts_oracle as ref
from helpers import TOL, to_f64
from test_gpu_experts import close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _rl():
    from paper_2312_03415_amd import binding
    return binding


def weights(rl, fp8, experts, i, o, r, g):
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)
    W = randn(experts, i, o).mul_(i ** -0.5)
    A, B = randn(experts, i, r).mul_(i ** -0.5), randn(experts, r, o).mul_((0.5 / r) ** 0.5)
    return (rl.Fp8Weight.quantize(W) if fp8 else W), A, B


def host_weight(W, e, fp8):
    if not fp8:
        return to_f64(W[e])
    return ref.weight_value(W.data[e].cpu().numpy(), W.scales[e].cpu().numpy())


@pytest.mark.parametrize("fp8", [False, True], ids=["dense", "fp8"])
def test_many_rows(fp8):
    rl = _rl()
    n, experts, i, o, r, s = 300000, 3, 8192, 144, 8, 1.5
    assert n * i > 2 ** 31
    ends_host = np.array([100000, 100000, 299990])
    g = torch.Generator(device="cuda").manual_seed(1)
    W, A, B = weights(rl, fp8, experts, i, o, r, g)
    X = torch.randn(n, i, generator=g, device="cuda", dtype=torch.bfloat16)
    dY = torch.randn(n, o, generator=g, device="cuda", dtype=torch.bfloat16)
    ends = torch.from_numpy(ends_host.astype(np.int32)).cuda()
    nan = lambda *shape: torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    Y, T, dX, dA, dB = nan(n, o), nan(n, r), nan(n, i), nan(experts, i, r), nan(experts, r, o)
    code = rl.RL_BF16
    size = max(rl.runlora_experts_workspace_bytes(b, n, experts, i, o, r, code, rl.RL_FP8_B128 if fp8 else code) for b in (False, True))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    rl.runlora_experts_forward(X, ends, W, A, B, Y, T, workspace=ws, scale=s)
    rl.runlora_experts_backward(dY, X, ends, W, A, B, dX, dA, dB, T, workspace=ws, scale=s)
    torch.cuda.synchronize()
    rows = np.array([0, 1, 99999, 100000, 100001, 262143, 262144, 262145, 299000, 299989, 299990, 299999])
    sample_ends = np.searchsorted(rows, ends_host)  # how many of the sampled rows lie before each end
    take = torch.from_numpy(rows).cuda()
    hW = np.stack([host_weight(W, e, fp8) for e in range(experts)])
    hA, hB, hX, hdY = to_f64(A), to_f64(B), to_f64(X[take]), to_f64(dY[take])
    want, bound = ref.forward(hX, sample_ends, hW, hA, hB, None, s, fp8, "bf16")
    close("Y", Y[take], want[0], bound[0], "bf16")
    close("T", T[take], want[1], bound[1], "bf16")
    want, bound = ref.backward(hdY, hX, sample_ends, hW, hA, hB, s, fp8, "bf16")
    close("dX", dX[take], want[0], bound[0], "bf16")
    # the sums: Z and T rounded to bf16 (2^-8 of an element at most), then the sum itself
    for e in range(experts):
        lo, hi = (0 if e == 0 else int(ends_host[e - 1])), int(ends_host[e])
        wA, wB = torch.zeros(i, r, dtype=torch.float64, device="cuda"), torch.zeros(r, o, dtype=torch.float64, device="cuda")
        for c in range(lo, hi, 20000):
            x, y = X[c:min(c + 20000, hi)].double(), dY[c:min(c + 20000, hi)].double()
            wA += x.t().contiguous() @ (s * (y @ B[e].double().t().contiguous()))
            wB += (s * (x @ A[e].double())).t().contiguous() @ y
        for name, got, want_sum in (("dA", dA[e], wA), ("dB", dB[e], wB)):
            if lo == hi:
                assert not got.any(), name
            else:
                assert ((got.double() - want_sum).norm() / want_sum.norm()).item() <= TOL["bf16"], name


@pytest.mark.parametrize("fp8", [False, True], ids=["dense", "fp8"])
@pytest.mark.parametrize("n", [40, 200])
def test_many_weights(n, fp8):
    rl = _rl()
    experts, i, o, r, s = 33, 8192, 8192, 8, 1.5
    assert (experts - 1) * i * o >= 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(2)
    W, A, B = weights(rl, fp8, experts, i, o, r, g)
    X = torch.randn(n, i, generator=g, device="cuda", dtype=torch.bfloat16)
    dY = torch.randn(n, o, generator=g, device="cuda", dtype=torch.bfloat16)
    first = n // 2  # half the rows are the last expert's, the others the first one's
    ends = torch.full((experts,), first, dtype=torch.int32, device="cuda")
    ends[-1] = n
    nan = lambda *shape: torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    Y, dX = nan(n, o), nan(n, i)
    code = rl.RL_BF16
    size = max(rl.runlora_experts_workspace_bytes(b, n, experts, i, o, r, code, rl.RL_FP8_B128 if fp8 else code) for b in (False, True))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    rl.runlora_experts_forward(X, ends, W, A, B, Y, None, workspace=ws, scale=s)
    rl.runlora_experts_backward(dY, X, ends, W, A, B, dX, None, None, None, workspace=ws, scale=s)
    torch.cuda.synchronize()
    rows = np.array([0, first - 1, first, n - 1])
    take = torch.from_numpy(rows).cuda()
    two = [0, experts - 1]
    hW = np.stack([host_weight(W, e, fp8) for e in two])
    hA, hB = to_f64(A)[two], to_f64(B)[two]
    hX, hdY = to_f64(X[take]), to_f64(dY[take])
    want, bound = ref.forward(hX, np.array([2, 4]), hW, hA, hB, None, s, fp8, "bf16")
    close("Y", Y[take], want[0], bound[0], "bf16")
    want, bound = ref.backward(hdY, hX, np.array([2, 4]), hW, hA, hB, s, fp8, "bf16")
    close("dX", dX[take], want[0], bound[0], "bf16")
