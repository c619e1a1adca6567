"""AdamW's front end on the CPU, its kernel call replaced."""
import pytest
import torch

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
