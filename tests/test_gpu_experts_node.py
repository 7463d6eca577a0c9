"""The native autograd node of the layers over 8-bit weights and stacks of experts beside the Python node it stands in for: the same saved tensors, read as
a saved-tensor hook returns them, and released with the graph."""
import gc

import pytest

from paper_2312_03415_amd import binding as rl

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

N, E, I, O, R = 90, 3, 256, 272, 16
KINDS = ["experts", "experts_fp8", "fp8"]


def functions(kind):
    from paper_2312_03415_amd import module
    fn = module.RunLoRAFp8Function if kind == "fp8" else module.RunLoRAExpertsFunction
    return {"native": fn, "python": type("Python" + fn.__name__, (fn,), {})}


class Operands:
    def __init__(self, kind, seed=0, n=N):
        g = torch.Generator().manual_seed(seed)
        randn = lambda *shape: torch.randn(*shape, generator=g).div_(16.0).bfloat16().cuda()
        lead = () if kind == "fp8" else (E,)
        self.kind, self.x, self.dy = kind, randn(n, I), randn(n, O)
        self.W, self.A, self.B, self.bias = randn(*lead, I, O), randn(*lead, I, R), randn(*lead, R, O), randn(*lead, O)
        if kind != "experts":
            self.W = rl.Fp8Weight.quantize(self.W)
        self.ends = None if kind == "fp8" else torch.tensor([n // 3, n // 2, n], dtype=torch.int32, device="cuda")

    def apply(self, fn, x, A, B):
        return fn.apply(x, self.W, A, B, self.bias, 1.5) if self.kind == "fp8" else fn.apply(x, self.ends, self.W, A, B, self.bias, 1.5)

    def run(self, fn):
        x, A, B = (t.clone().requires_grad_(True) for t in (self.x, self.A, self.B))
        y = self.apply(fn, x * 1.0, A, B)
        return y, (x, A, B)


def packed(ops, fn, unpack=lambda t: t.cuda()):
    """Saved tensors by shape and type, and the gradients of a pass whose saved tensors leave as host copies and come back as unpack(t)."""
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append((tuple(t.shape), t.dtype)), t.cpu())[1], unpack):
        y, leaves = ops.run(fn)
    churn = [torch.full((1 << k,), 7.0, device="cuda", dtype=torch.bfloat16) for k in range(9, 18)]
    grads = torch.autograd.grad(y, leaves, ops.dy)
    del churn
    return seen, grads


@pytest.mark.parametrize("kind", KINDS)
def test_the_same_tensors_are_saved_in_the_same_order(kind):
    ops, fns = Operands(kind), functions(kind)
    (a, ga), (b, gb) = (packed(ops, fns[k]) for k in ("native", "python"))
    assert a == b
    assert ((N, R), torch.bfloat16) in a      # the kept product among them: it leaves and comes back as the others do
    y, leaves = ops.run(fns["native"])
    for got, want in zip(ga, torch.autograd.grad(y, leaves, ops.dy)):
        assert torch.equal(got, want)
    assert all(torch.equal(p, q) for p, q in zip(ga, gb))


@pytest.mark.parametrize("node", ["native", "python"])
@pytest.mark.parametrize("kind", KINDS)
def test_the_kept_product_goes_with_the_graph(kind, node):
    """Behind the backward a node that is still referenced (by its output) holds none of what it saved."""
    ops, fn = Operands(kind, n=4096), functions(kind)[node]
    x = ops.x.clone().requires_grad_(True)  # (one leaf for both passes: the engine's thread lets go of a graph's leaves a little behind the pass)
    gc.collect()
    for last in (False, True):
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        y = ops.apply(fn, x, ops.A, ops.B)
        g, = torch.autograd.grad(y, x, ops.dy)
        held = torch.cuda.memory_allocated() - before
        outputs = sum(t.untyped_storage().nbytes() for t in (y, g))
        assert not last or held == outputs
        del y, g


@pytest.mark.parametrize("node", ["native", "python"])
@pytest.mark.parametrize("kind", KINDS)
def test_saved_tensors_that_come_back_changed(kind, node):
    """Rows apart are read as they are; a device, layout, type or size that the forward would refuse is refused before anything is launched."""
    ops, fn = Operands(kind), functions(kind)[node]
    plain = packed(ops, fn)[1]
    wide = lambda t: torch.cat([t.cuda()] * 2, -1)[..., :t.shape[-1]] if t.dim() >= 2 and t.dtype != torch.uint8 else t.cuda()
    assert all(torch.equal(a, b) for a, b in zip(packed(ops, fn, wide)[1], plain))
    odd = lambda t: t.cuda().repeat_interleave(2, -1)[..., ::2]
    x, T, A = (N, I), (N, R), tuple(ops.A.shape)
    W = tuple((ops.W if kind == "experts" else ops.W.data).shape)
    changes = [(x, lambda t: t.cpu()), (T, lambda t: t.cpu()), (A, lambda t: t.cpu()), (W, lambda t: t.cpu()), (A, odd), (T, odd), (W, odd)]
    if kind != "fp8":
        changes += [((E,), lambda t: t.cpu()), ((E,), lambda t: t.cuda().long()), ((E,), lambda t: t.cuda()[:2])]
    if kind != "experts":
        S = tuple(ops.W.scales.shape)
        changes += [(S, lambda t: t.cpu()), (S, lambda t: t.cuda()[..., :1].contiguous()), (W, lambda t: t.cuda()[..., :I]), (W, lambda t: t.cuda().float())]
    changes += [(x, lambda t: t.cuda().float()), (T, lambda t: t.cuda().half()), (T, lambda t: t.cuda()[:-1]), (T, lambda t: t.cuda()[:, :8]),
                (A, lambda t: t.cuda().half()), (A, lambda t: t.cuda()[..., :-8].contiguous())]
    assert all(sum(s == shape for s, _ in packed(ops, fn)[0]) == 1 for shape, _ in changes)
    for k, (shape, change) in enumerate(changes):
        with pytest.raises((ValueError, rl.RunLoRAError)):
            packed(ops, fn, lambda t: change(t) if tuple(t.shape) == shape else t.cuda())
            pytest.fail(f"change {k} of a saved tensor {shape} was taken")


@pytest.mark.parametrize("kind", KINDS)
def test_a_saved_tensor_that_changes_in_place(kind):
    messages = []
    for fn in functions(kind).values():
        ops = Operands(kind)
        z = ops.x.clone().requires_grad_(True) * 1.0
        y = ops.apply(fn, z, ops.A, ops.B)
        z.add_(1.0)
        with pytest.raises(RuntimeError, match="inplace") as e:
            y.sum().backward()
        messages.append(str(e.value))
    assert messages[0] == messages[1]


@pytest.mark.parametrize("kind", KINDS)
def test_both_nodes_on_streams_and_threads(kind):
    """Four threads with a stream each: every pass gives the bits of one computed alone."""
    import threading
    for fn in functions(kind).values():
        cases = [Operands(kind, k, 300 + 40 * k) for k in range(4)]

        def one(c):
            y, leaves = c.run(fn)
            return (y.detach(),) + torch.autograd.grad(y, leaves, c.dy)
        alone = [one(c) for c in cases]
        torch.cuda.synchronize()
        out, errors = {}, []

        def work(k):
            try:
                s = torch.cuda.Stream()
                s.wait_stream(torch.cuda.default_stream())
                with torch.cuda.stream(s):
                    for _ in range(8):
                        out[k] = one(cases[k])
                s.synchronize()
            except Exception as e:   # noqa: BLE001 - reported by the main thread
                errors.append(e)
        threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not errors, errors
        assert all(torch.equal(a, b) for k in range(4) for a, b in zip(out[k], alone[k]))


@pytest.mark.parametrize("node", ["native", "python"])
@pytest.mark.parametrize("kind", KINDS)
def test_a_bias_of_another_shape_is_refused(kind, node):
    """As many elements in another order are not a bias for every expert."""
    ops, fn = Operands(kind), functions(kind)[node]
    for shape in ((1, O),) if kind == "fp8" else ((O, E), (E * O,), (E, 1, O)):
        ops.bias = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(ValueError, match="bias"):
            ops.run(fn)
