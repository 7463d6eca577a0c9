"""One decoder block with a routed mixture of expert MLPs, every linear adapted, frozen weights in 8 bits or in 16: forward+backward
time of a training step, and time of a step that answers one token per sequence.

    python -m paper_2312_03415_amd.experts_timing --model opt1.3b --experts 8 --top 2 --batch 4 --seq 2048 --rank 32

Attention's projections are RunLoRAFp8Linear (kind fp8) or RunLoRALinear (kind 16bit); the MLP's are RunLoRAExperts over a stack of
8-bit or 16-bit weights.  Every token goes to its `top` best experts (RunRouter): its row is copied to the rows sorted by expert, the experts'
products run on them with the counts left on the device, and a token's rows are added to the residual stream with the router's weights.
Where the model has root-mean-square norms they are RunRMSNorm, with the residual's addition and, in front of 8-bit projections, the rows in 8 bits.

Both kinds hold the same synthetic weights (N(0, 1/d_in); the 8-bit ones rounded); inputs and the upstream gradient are N(0, 1); attention,
layer norms, the router's product and the activation are torch's own operators.  Prints one JSON line.
"""
import argparse
import json
import math

import torch
import torch.nn.functional as F
from torch import nn

from . import binding as rl
from .block_timing import MODELS, time_block
from .module import RunCombineFunction, RunGatherFunction, RunLoRAExperts, RunLoRAFp8Linear, RunLoRALinear, RunRMSNorm, RunRouter


class RoutedMLP(nn.Module):
    """x [n, d] -> sum over a token's experts of weight * expert MLP(x), added to `add` if that is given."""

    def __init__(self, router, top, gate, up, down):
        super().__init__()
        self.register_buffer("router", router)  # [d, experts]
        self.route = RunRouter(router.shape[1], top, device=router.device)
        self.top, self.gate, self.up, self.down = top, gate, up, down

    def forward(self, x, add=None):
        weight, _, place, source, ends = self.route(x.float() @ self.router)
        rows = RunGatherFunction.apply(x, place, source)
        up = self.up(rows, ends)
        hidden = F.relu(up) if self.gate is None else F.silu(self.gate(rows, ends)) * up
        return RunCombineFunction.apply(self.down(hidden, ends), place, source, weight, add)


class RoutedBlock(nn.Module):
    """Pre-norm decoder block: x + attn(norm(x)), then x + routed MLP(norm(x)); causal attention.  With a cache (keys, values of the tokens
    so far) x holds one more token of each sequence."""

    def __init__(self, cfg, experts, top, make_linear, make_experts, router, dtype, device):
        super().__init__()
        d, ffn = cfg["d"], cfg["ffn"]
        self.heads = cfg["heads"]
        norm = (lambda: RunRMSNorm(d, dtype=dtype, device=device)) if cfg["rms"] else (lambda: nn.LayerNorm(d, dtype=dtype, device=device))
        self.norm1, self.norm2 = norm(), norm()
        for p in list(self.norm1.parameters()) + list(self.norm2.parameters()):
            p.requires_grad_(False)
        self.q_proj, self.k_proj, self.v_proj, self.o_proj = (make_linear(name, d, d) for name in ("q", "k", "v", "o"))
        self.mlp = RoutedMLP(router, top, make_experts("gate", d, ffn) if cfg["gated"] else None, make_experts("up", d, ffn), make_experts("down", ffn, d))

    def forward(self, x, cache=None):
        b, s, d = x.shape
        rms = isinstance(self.norm1, RunRMSNorm)
        given = ()
        if rms and isinstance(self.q_proj, RunLoRAFp8Linear):
            h, rows = self.norm1(x, rows=True)
            given = (rows,)  # rounded once for the three projections
        else:
            h = self.norm1(x)
        split = lambda t: t.view(b, s, self.heads, d // self.heads).transpose(1, 2)
        q, k, v = (split(proj(h, *given)) for proj in (self.q_proj, self.k_proj, self.v_proj))
        if cache is not None:
            k, v = torch.cat((cache[0], k), 2), torch.cat((cache[1], v), 2)
        a = F.scaled_dot_product_attention(q, k, v, is_causal=cache is None)
        a = self.o_proj(a.transpose(1, 2).reshape(b, s, d))
        if rms:
            h, x = self.norm2(a, x)
        else:
            x = x + a
            h = self.norm2(x)
        return self.mlp(h.view(b * s, d), x).view(b, s, d)


def build_block(cfg, kind, experts, top, r, alpha, dtype, device, seed):
    """Same weights and adapters for both kinds (the generator is reseeded per layer)."""

    def draw(name, d_in, d_out, count=None):
        g = torch.Generator(device=device).manual_seed(seed + sum(map(ord, name)))
        lead = () if count is None else (count,)
        randn = lambda *shape: torch.randn(*lead, *shape, generator=g, device=device)
        W = randn(d_in, d_out).div_(math.sqrt(d_in)).to(dtype)
        bias = (randn(d_out) * 0.02).to(dtype) if cfg["bias"] else None
        A = (randn(d_in, r) / math.sqrt(d_in)).to(dtype)
        B = (randn(r, d_out) * math.sqrt(0.1 / r)).to(dtype)
        return W, bias, A, B

    def adapted(layer, A, B):
        with torch.no_grad():
            layer.lora_A.copy_(A)
            layer.lora_B.copy_(B)
        return layer

    def make_linear(name, d_in, d_out):
        W, bias, A, B = draw(name, d_in, d_out)
        if kind == "fp8":
            return adapted(RunLoRAFp8Linear(rl.Fp8Weight.quantize(W), r, alpha, bias, dtype), A, B)
        return adapted(RunLoRALinear(W, r, alpha, bias), A, B)

    def make_experts(name, d_in, d_out):
        W, bias, A, B = draw(name, d_in, d_out, experts)
        return adapted(RunLoRAExperts(rl.Fp8Weight.quantize(W) if kind == "fp8" else W, r, alpha, bias, dtype), A, B)

    g = torch.Generator(device=device).manual_seed(seed)
    router = torch.randn(cfg["d"], experts, generator=g, device=device) / math.sqrt(cfg["d"])
    return RoutedBlock(cfg, experts, top, make_linear, make_experts, router, dtype, device)


def time_answer(block, x, cache, iters, warmup):
    """Median milliseconds of one more token for every sequence."""
    times = []
    with torch.no_grad():
        for it in range(warmup + iters):
            t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            t0.record()
            block(x, cache)
            t1.record()
            t1.synchronize()
            if it >= warmup:
                times.append(t0.elapsed_time(t1))
    times.sort()
    return times[len(times) // 2]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--model", choices=sorted(MODELS), default="opt1.3b")
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--top", type=int, default=2)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--seq", type=int, default=2048)
    ap.add_argument("--rank", type=int, default=32)
    ap.add_argument("--alpha", type=float, default=None, help="LoRA alpha (default: 2 r)")
    ap.add_argument("--dtype", choices=("bf16", "f16"), default="bf16")
    ap.add_argument("--iters", type=int, default=20)
    ap.add_argument("--warmup", type=int, default=5)
    args = ap.parse_args(argv)

    if not torch.cuda.is_available():
        raise SystemExit("experts_timing needs a GPU")
    if not 1 <= args.top <= args.experts:
        raise SystemExit("--top has to lie between 1 and --experts")
    device = torch.device("cuda:0")
    dtype = torch.bfloat16 if args.dtype == "bf16" else torch.float16
    cfg = MODELS[args.model]
    d, heads = cfg["d"], cfg["heads"]
    alpha = args.alpha if args.alpha is not None else 2.0 * args.rank
    g = torch.Generator(device=device).manual_seed(20231203)
    randn = lambda *shape: torch.randn(*shape, generator=g, device=device).to(dtype)
    x0, dy = randn(args.batch, args.seq, d), randn(args.batch, args.seq, d)
    token = randn(args.batch, 1, d)
    cache = randn(args.batch, heads, args.seq, d // heads), randn(args.batch, heads, args.seq, d // heads)

    out = {"model": args.model, "experts": args.experts, "top": args.top, "batch": args.batch, "seq": args.seq, "rank": args.rank,
           "dtype": args.dtype, "data": "synthetic", "iters": args.iters, "ms_fwd_bwd": {}, "ms_answer": {}, "frozen_bytes": {}}
    ys = {}
    for kind in ("fp8", "16bit"):
        block = build_block(cfg, kind, args.experts, args.top, args.rank, alpha, dtype, device, seed=7)
        trained = {id(p) for p in block.parameters() if p.requires_grad}
        frozen = [t for t in list(block.parameters()) + list(block.buffers()) if id(t) not in trained]
        out["frozen_bytes"][kind] = sum(t.numel() * t.element_size() for t in frozen)
        x = x0.clone().requires_grad_(True)
        ms, ys[kind] = time_block(block, x, dy, args.iters, args.warmup)
        out["ms_fwd_bwd"][kind] = round(ms, 4)
        if not all(torch.isfinite(p.grad).all() for p in block.parameters() if p.requires_grad):
            raise SystemExit("a gradient is not finite")
        out["ms_answer"][kind] = round(time_answer(block, token, cache, args.iters, args.warmup), 4)
        del block, x
        torch.cuda.empty_cache()
    # the 8-bit block rounds weights and rows; some tokens also change an expert
    out["rel_diff"] = float(f"{((ys['fp8'].double() - ys['16bit'].double()).norm() / ys['16bit'].double().norm()).item():.3e}")
    print(json.dumps(out))
    return out


if __name__ == "__main__":
    main()
