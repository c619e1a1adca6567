"""AdamW's front end on the CPU, its kernel call replaced."""
import pytest
import torch

from paper_2607_10611_amd import binding as B
from paper_2607_10611_amd.optim import AdamW


def parameter(n=4):
    p = torch.nn.Parameter(torch.zeros(n))
    p.grad = torch.ones(n)
    return p


def test_a_captured_step_is_refused(monkeypatch):
    """The step number, learning rate and draws' key go to the kernel by value: every
    replay would repeat the captured step."""
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    p = parameter()
    opt = AdamW([p])
    with pytest.raises(RuntimeError, match="captur"):
        opt.step()
    assert not opt.state[p]


@pytest.fixture
def stub(monkeypatch):
    """AdamW whose checks take CPU tensors and whose kernel call does nothing; the list
    of the (hyper-parameters, grad_scale) that it was called with."""
    made = []
    monkeypatch.setattr(AdamW, "_check_param", staticmethod(lambda p, master: None))
    monkeypatch.setattr(B, "_need", lambda *a: None)
    monkeypatch.setattr(B, "madd_adamw_step",
                        lambda al, hp, grad_scale=None, index_base=0: made.append((hp, grad_scale)))
    return made


def test_a_step_tells_autograd_that_the_parameters_changed(stub):
    """A backward pass through tensors saved before the step raises, as after torch's
    own optimizers, instead of using the new values."""
    w, other = parameter(), parameter()
    other.grad = None
    x = torch.ones(4, requires_grad=True)
    loss, loss2 = (x * w).sum(), (x * other).sum()
    AdamW([w, other]).step()
    assert len(stub) == 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    loss2.backward()  # a parameter that had no gradient is as it was


def test_refused_gradients_leave_a_list_as_it_was(stub):
    """A list's addresses belong to tensors that it keeps alive: a set that is refused
    half way must not leave addresses of tensors that nobody holds."""
    a, b = torch.ones(4), torch.ones(6)
    gl = B.GradList([a, b])
    before = list(gl.g), list(gl.gfmt), gl.format
    for bad in ([torch.ones(4), torch.ones(5)], [torch.ones(4).bfloat16(), torch.ones(6).double()]):
        with pytest.raises((ValueError, TypeError)):
            gl.set(bad)
        assert (list(gl.g), list(gl.gfmt), gl.format) == before
        assert gl._tensors[0] is a and gl._tensors[1] is b
    gl.set([a.bfloat16(), None])
    assert gl.g[0] == gl._tensors[0].data_ptr() and gl.g[1] is None


@pytest.mark.parametrize("scale", [4, 0, 1, 0.5, True])
def test_a_scale_that_is_no_tensor_is_refused(stub, scale):
    """An integer would be taken for a device address."""
    p = parameter()
    opt = AdamW([p])
    with pytest.raises(TypeError, match="grad_scale"):
        opt.step(grad_scale=scale)
    assert not stub and not opt.state[p]


def test_copies_and_scales_of_other_types_are_refused(stub):
    """bf16 codes would be written into a float16 copy, scale bytes over floats."""
    f, u8 = torch.zeros(128), torch.zeros(128, dtype=torch.uint8)
    for good in (torch.bfloat16, torch.int16, torch.uint16):
        B.AdamWList([f], [f], [f], [f], copies=[f.to(good)])
    for bad in (torch.float16, torch.float32, torch.int32):
        with pytest.raises(TypeError, match="copy"):
            B.AdamWList([f], [f], [f], [f], copies=[f.to(bad)])
    for good in (torch.uint8, torch.int8, torch.float8_e8m0fnu):
        B.AdamWList([f], [f], [u8], [u8], scales=[torch.zeros(2).to(good)])
    for bad in (torch.float16, torch.float32, torch.float8_e4m3fn):
        with pytest.raises(TypeError, match="scales"):
            B.AdamWList([f], [f], [u8], [u8], scales=[torch.zeros(2).to(bad)])
