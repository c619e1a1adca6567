"""FP8Linear and its autograd function on the CPU, the kernels' calls replaced by
torch operations (what is tested is which of them run, and what autograd sees)."""
import pytest
import torch

from paper_2607_10611_amd import fp8
from paper_2607_10611_amd.optim import MAdam


def values(m):
    return m.dequantize(torch.float64)


def quantize(x, fmt="e4m3", rows=True, cols=False):
    """Codes that keep small integers, with scale 1."""
    def blocks(t):
        t = torch.nn.functional.pad(t.detach().float(), (0, -t.shape[1] % 128))
        q = t.to(fp8._DTYPE[fmt])
        return fp8.BlockMatrix(q, torch.full((q.shape[0], q.shape[1] // 128), 127,
                                             dtype=torch.uint8))
    x = x.reshape(-1, x.shape[-1])
    r, c = (blocks(x) if rows else None), (blocks(x.t().contiguous()) if cols else None)
    for m, n in ((r, x.shape[1]), (c, x.shape[0])):
        if m is not None:
            m.cols = n
    return r, c


@pytest.fixture
def calls(monkeypatch):
    """Names of the calls made, in order."""
    made = []

    def matmul(a, b, dtype=torch.bfloat16, out=None, accumulate=False):
        made.append("matmul")
        k = min(a.codes.shape[1], b.codes.shape[1])
        full = lambda m: fp8.BlockMatrix(m.codes, m.scales, m.fmt).dequantize(torch.float64)  # noqa: E731
        return (full(a)[:, :k] @ full(b)[:, :k].t()).to(dtype)

    def linear(x, w, dtype=torch.bfloat16, out=None):
        made.append("linear")
        y = matmul(quantize(x)[0], w, dtype)
        made.pop()
        return y.view(*x.shape[:-1], y.shape[1])

    def counted(*a, **kw):
        made.append("quantize")
        return quantize(*a, **kw)

    monkeypatch.setattr(fp8, "quantize", counted)
    monkeypatch.setattr(fp8, "matmul", matmul)
    monkeypatch.setattr(fp8, "linear", linear)
    return made


def integers(*shape, seed=0, dtype=torch.bfloat16):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=gen).to(dtype)


def layer(k=128, n=6, master=True):
    lin = fp8.FP8Linear(k, n)
    with torch.no_grad():
        lin.weight.copy_(integers(n, k, seed=1))
    if master:
        m = quantize(lin.weight)[0]
        s = torch.ones(n * k // 128, dtype=torch.float16)
        lin.use_master(m.codes.view(torch.uint8).view(-1), s)
    return lin


def test_first_derivatives(calls):
    lin, x = layer(), integers(4, 128, seed=2).requires_grad_()
    dy = integers(4, 6, seed=3)
    lin(x).backward(dy)
    assert torch.equal(x.grad.double(), dy.double() @ lin.weight.detach().double())
    assert torch.equal(lin.weight.grad.double(), dy.double().t() @ x.detach().double())


def test_second_derivatives_are_refused(calls):
    """The backward pass runs in kernels that autograd does not see: a second
    derivative through it would silently be without its terms."""
    lin, x = layer(), integers(4, 128, seed=2).requires_grad_()
    loss = lin(x).float().square().sum() + x.float().pow(3).sum()
    (dx,) = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dx.float().sum().backward()


def with_optimizer(lin):
    """MAdam over the layer's weight, its state as a first step leaves it."""
    opt, n = MAdam([lin.weight], master_format="e4m3"), lin.weight.numel()
    state = lambda *s, dtype=torch.uint8: torch.ones(*s, dtype=dtype)  # noqa: E731
    opt.state[lin.weight] = dict(step=1, m=state(n, dtype=torch.float32),
                                 v=state(n, dtype=torch.float32),
                                 ve=state(n, dtype=torch.float32), q=state(n),
                                 scales=state(n // 64))
    return opt, opt.state[lin.weight]


@pytest.mark.parametrize("shaped", [False, True])
def test_a_master_that_the_optimizer_replaced_is_not_read(calls, shaped):
    """MAdam.load_state_dict puts new tensors in place of the state's: a layer that
    still held the old ones would read a master that no step updates."""
    lin = layer(master=False)
    opt, st = with_optimizer(lin)
    lin.use_master(st["q"].view(6, 128) if shaped else st["q"], st["scales"])
    saved = opt.state_dict()
    y = lin(integers(2, 128))
    opt.load_state_dict(saved)
    with pytest.raises(RuntimeError, match="use_master"):
        lin(integers(2, 128))
    st = opt.state[lin.weight]
    lin.use_master(st["q"], st["scales"])
    assert torch.equal(lin(integers(2, 128)), y)
    assert torch.equal(saved["state"][0]["q"], st["q"])  # the saved state is as it was


def test_a_layer_whose_weight_is_loaded_reads_that_weight(calls):
    """The master is another weight's then."""
    lin, other = layer(), layer(master=False)
    x = integers(3, 128, seed=4)
    with torch.no_grad():
        other.weight.neg_()
    assert torch.equal(lin(x), -other(x))
    torch.nn.ModuleDict(dict(a=lin)).load_state_dict({"a.weight": other.weight})
    assert torch.equal(lin(x), other(x))


def test_reading_the_model_takes_the_serving_path(calls):
    """No gradient is wanted: x W^T alone runs, and x's column blocks, which only the
    weight's gradient needs, are not made."""
    lin, x = layer(), integers(4, 128, seed=2)
    want = lin(x).detach()
    assert calls == ["quantize", "matmul"]
    for mode in (torch.no_grad, torch.inference_mode):
        calls.clear()
        with mode():
            y = lin(x)
        assert calls == ["linear"] and torch.equal(y, want) and not y.requires_grad
    lin.weight.requires_grad_(False)
    calls.clear()
    assert torch.equal(lin(x), want) and calls == ["linear"]


def test_a_frozen_weight_passes_gradients_on(calls):
    lin, x = layer(), integers(4, 128, seed=2).requires_grad_()
    lin.weight.requires_grad_(False)
    dy = integers(4, 6, seed=3)
    y = lin(x)
    assert calls == ["linear"]
    y.backward(dy)
    assert torch.equal(x.grad.double(), dy.double() @ lin.weight.double())
    assert lin.weight.grad is None
