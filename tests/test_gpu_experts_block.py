"""A decoder block with routed experts, adapted 8-bit and 16-bit layers together: outputs and gradients of its MLP against the sum over
experts taken densely, and the timing script."""
import json

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [True, False], ids=["gated", "plain"])
@pytest.mark.parametrize("n", [1, 7, 300])
def test_routed_mlp_is_the_weighted_sum_over_experts(n, gated):
    """16-bit weights, against every expert applied to every token in 64 bits with the same choice of experts.  Each of the up to three
    products, the activation and the sum rounds to bf16 (2^-8 of an element at most): 6 roundings in a row stay below 2e-2 of the norm.
    Which side of its kink an activation is on is, like the choice of experts, taken from the run (T's rounding puts a few in ten thousand on the
    other side, and a gradient jumps there)."""
    import torch
    from paper_2312_03415_amd import experts_timing
    E, top, d, ffn, r = 5, 2, 136, 264, 8
    cfg = dict(d=d, heads=2, ffn=ffn, gated=gated, bias=True, rms=True)
    block = experts_timing.build_block(cfg, "16bit", E, top, r, 2.0 * r, torch.bfloat16, torch.device("cuda:0"), seed=3)
    mlp = block.mlp
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, d, generator=g).bfloat16().cuda().requires_grad_(True)
    dy = torch.randn(n, d, generator=g).bfloat16().cuda()
    seen = []
    mlp.up.register_forward_hook(lambda layer, args, out: seen.append(out.detach().cpu()))
    y = mlp(x)
    y.backward(dy)

    weight, expert = (x.detach().float() @ mlp.router).topk(top, dim=1)  # (the choice itself has no gradient)
    assert weight.shape == (n, top)
    sorted_expert, order = expert.flatten().cpu().sort(stable=True)
    above = torch.zeros(E, n, ffn, dtype=torch.bool)
    above[sorted_expert, order // top] = seen[0] > 0
    x64 = x.detach().double().cpu().requires_grad_(True)
    leaves = {}

    def linear(layer, name, t, e):
        A, B = (leaves.setdefault((name, k, e), getattr(layer, k)[e].detach().double().cpu().requires_grad_(True)) for k in ("lora_A", "lora_B"))
        return t @ layer.weight[e].detach().double().cpu() + layer.scale * (t @ A) @ B + layer.bias[e].detach().double().cpu()

    soft = torch.gather(x64 @ mlp.router.double().cpu(), 1, expert.cpu()).softmax(1)
    want = torch.zeros(n, d, dtype=torch.float64)
    for e in range(E):
        up = linear(mlp.up, "up", x64, e)
        hidden = torch.nn.functional.silu(linear(mlp.gate, "gate", x64, e)) * up if gated else up * above[e]
        part = linear(mlp.down, "down", hidden, e)
        want = want + part * (soft * (expert.cpu() == e)).sum(1, keepdim=True)
    want.backward(dy.double().cpu())
    rel = lambda a, b: ((a.detach().double().cpu() - b).norm() / b.norm()).item()
    assert rel(y, want.detach()) < 2e-2
    assert rel(x.grad, x64.grad) < 2e-2
    for name in ("up", "down") + (("gate",) if gated else ()):
        for k in ("lora_A", "lora_B"):
            got = getattr(getattr(mlp, name), k).grad
            ref = torch.stack([leaves[(name, k, e)].grad for e in range(E)])
            assert rel(got, ref) < 2e-2, (name, k)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_experts_timing_script(dtype, capsys):
    """Both kinds run a training step and a step of one token per sequence.  Rounding to e4m3 moves an element by 2^-4 at most, so a product
    by 9 % at the very most; a token whose expert changes moves by its MLP's output: together well below 0.3 of the block's output,
    which a wrong order of rows would exceed."""
    from paper_2312_03415_amd import experts_timing
    out = experts_timing.main(["--model", "opt1.3b", "--experts", "4", "--top", "2", "--batch", "2", "--seq", "96", "--rank", "8", "--dtype", dtype,
                               "--iters", "2", "--warmup", "1"])
    for key in ("ms_fwd_bwd", "ms_answer"):
        assert set(out[key]) == {"fp8", "16bit"} and all(v > 0 for v in out[key].values())
    assert out["frozen_bytes"]["fp8"] < 0.52 * out["frozen_bytes"]["16bit"]
    assert 0 < out["rel_diff"] < 0.3
    assert json.loads(capsys.readouterr().out.strip().splitlines()[-1])["model"] == "opt1.3b"
