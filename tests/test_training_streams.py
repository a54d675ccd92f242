"""Which stream the training classes take for a handle (paper_2607_05116_amd.training)."""
import contextlib

import pytest
import torch

from paper_2607_05116_amd import training


def test_handle_0_is_the_default_stream(monkeypatch):
    entered = []

    @contextlib.contextmanager
    def enter(s):
        entered.append(s)
        yield

    monkeypatch.setattr(torch.cuda, "stream", enter)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: "default")
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h: ("external", h))
    for handle in (0, 0x1000, None):
        with training._on(handle):
            pass
    assert entered == ["default", ("external", 0x1000)]


@pytest.mark.gpu
def test_a_step_on_the_default_streams_handle():
    from tests.test_gpu_training import OFFSETS, _batch, _trainer
    a, b = _trainer(), _trainer()
    offs, x = torch.tensor(OFFSETS, dtype=torch.int32, device="cuda"), _batch(4)
    a.step(x, None, offs)
    torch.cuda.synchronize()
    handle = torch.cuda.default_stream().cuda_stream
    assert handle == 0
    torch.cuda._sleep(20_000_000)                       # whatever ran on another stream would be ahead of forward
    b.forward(x, offs, stream=handle)
    b.backward(x, None, offs, stream=handle)
    b.opt.step(b.w, b.d_w, b.w_bf16, stream=handle)
    torch.cuda.synchronize()
    assert torch.equal(a.d_w, b.d_w) and torch.equal(a.w, b.w) and torch.equal(a.w_bf16, b.w_bf16)
