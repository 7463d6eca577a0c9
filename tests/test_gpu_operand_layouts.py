"""Rows as autograd and callers hand them over: layouts that the library does not read (rows that repeat, an odd address, an odd distance) are laid out anew by
either node of every layer, and give the bits of a dense copy."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LAYERS = ["lora", "vera", "dora", "fp8", "experts", "experts_fp8"]
D_IN, D_OUT, R = 256, 272, 16


def layer(kind, node, n):
    """f(x) of a layer with n rows a call, by its native or its Python node."""
    from paper_2312_03415_amd import binding as rl, module
    g = torch.Generator().manual_seed(3)
    randn = lambda *shape: torch.randn(*shape, generator=g).div_(16.0).bfloat16().cuda()
    name = {"lora": "RunLoRAFunction", "vera": "RunVeRAFunction", "dora": "RunDoRAFunction", "fp8": "RunLoRAFp8Function"}.get(kind, "RunLoRAExpertsFunction")
    fn = getattr(module, name)
    if node == "python":
        fn = type("Python" + name, (fn,), {})  # (a subclass's calls stay in Python)
    if kind.startswith("experts"):
        W, A, B = randn(3, D_IN, D_OUT), randn(3, D_IN, R), randn(3, R, D_OUT)
        if kind == "experts_fp8":
            W = rl.Fp8Weight.quantize(W)
        ends = torch.tensor([n // 3, n // 2, n], dtype=torch.int32, device="cuda")
        return lambda x: fn.apply(x, ends, W, A, B, None, 1.5)
    W, A, B = randn(D_IN, D_OUT), randn(D_IN, R), randn(R, D_OUT)
    if kind == "lora":
        return lambda x: fn.apply(x, W, A, B, None, 1.5, (1, 1), False)
    if kind == "vera":
        d, b = randn(R), randn(D_OUT)
        return lambda x: fn.apply(x, W, A, B, d, b, None, 1.5, (1, 1))
    if kind == "dora":
        m = W.float().norm(dim=0).bfloat16()
        return lambda x: fn.apply(x, W, A, B, m, None, 1.5, 4)
    W = rl.Fp8Weight.quantize(W)
    return lambda x: fn.apply(x, W, A, B, None, 1.5)


def rows(n, width, seed):
    return torch.randn(n, width, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


@pytest.mark.parametrize("node", ["native", "python"])
@pytest.mark.parametrize("kind", LAYERS)
@pytest.mark.parametrize("n", [2, 90])
def test_a_gradient_that_repeats_over_the_rows(kind, node, n):
    """What the sum over the rows sends back: one row, at a distance of zero from the next."""
    f, dy = layer(kind, node, n), rows(1, D_OUT, 1)[0]
    x = rows(n, D_IN, 2).requires_grad_(True)
    want, = torch.autograd.grad(f(x), x, dy.expand(n, -1).contiguous())
    got, = torch.autograd.grad(f(x).sum(0), x, dy)
    assert torch.equal(got, want)
    x3 = x.detach().view(2, n // 2, D_IN).requires_grad_(True)
    got, = torch.autograd.grad(f(x3).sum(1).sum(0), x3, dy)
    assert torch.equal(got.view(n, D_IN), want)


@pytest.mark.parametrize("node", ["native", "python"])
@pytest.mark.parametrize("kind", LAYERS)
def test_an_input_that_repeats_over_the_rows(kind, node):
    f, x, dy = layer(kind, node, 90), rows(1, D_IN, 2), rows(90, D_OUT, 1)
    y = f(x.expand(90, -1).contiguous())
    assert torch.equal(f(x.expand(90, -1)), y)
    a, b = x.clone().requires_grad_(True), x.expand(90, -1).contiguous().requires_grad_(True)
    got, = torch.autograd.grad(f(a.expand(90, -1)), a, dy)
    want, = torch.autograd.grad(f(b), b, dy)
    assert torch.equal(got, want.sum(0, keepdim=True))


def odd_address(t):
    """The same dense rows at an address that is two bytes off."""
    flat = torch.empty(t.numel() + 8, dtype=t.dtype, device=t.device)
    out = flat[1:1 + t.numel()].view(t.shape)
    out.copy_(t)
    assert out.is_contiguous() and out.data_ptr() % 16 != 0
    return out


def odd_distance(t):
    """One row of a matrix with a column more (which counts as contiguous, whatever its rows' distance)."""
    assert t.shape[0] == 1
    out = torch.empty(2, t.shape[1] + 1, dtype=t.dtype, device=t.device)[:1, :t.shape[1]]
    out.copy_(t)
    assert out.is_contiguous() and out.stride(0) % 8 != 0
    return out


@pytest.mark.parametrize("node", ["native", "python"])
@pytest.mark.parametrize("kind", LAYERS)
@pytest.mark.parametrize("n,off", [(90, odd_address), (1, odd_address), (1, odd_distance)])
def test_rows_that_only_look_dense(kind, node, n, off):
    f, x, dy = layer(kind, node, n), rows(n, D_IN, 2).requires_grad_(True), rows(n, D_OUT, 1)
    y = f(x)
    want, = torch.autograd.grad(y, x, dy)
    xo = off(x.detach()).requires_grad_(True)
    got = f(xo)
    assert torch.equal(got, y)
    assert torch.equal(torch.autograd.grad(got, xo, off(dy))[0], want)
