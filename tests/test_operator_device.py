"""The operators' tensors have to be on the current device: their kernels go to its stream, their outputs and workspace come from the tensors'
device.  The question which device is current is answered by the test."""
from types import SimpleNamespace

import pytest
import torch

from paper_2502_11058_amd import operators as O


def test_a_tensor_on_another_device_is_refused(monkeypatch):
    there = SimpleNamespace(dtype=torch.float32, is_cuda=True, device=torch.device("cuda", 1), get_device=lambda: 1)
    monkeypatch.setattr(O, "_device", lambda: 1, raising=False)
    assert O._typed(there) == 0
    monkeypatch.setattr(O, "_device", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="cuda:1.*current device"):
        O._typed(there)


@pytest.mark.gpu
def test_every_call_asks(monkeypatch):
    x, w = torch.ones(1, 4, 2, 32, device="cuda"), torch.ones(32, device="cuda")
    table, t = O.rotary_table(4, 32), torch.zeros(1, 4, 2, dtype=torch.int64, device="cuda")
    y, mean, rstd = O.norm_forward(x, w)
    o, lse = O.attention_forward(x, x, x)
    loss, lse_t = O.linear_cross_entropy_forward(x, w[None], t)
    calls = [lambda: O.norm_forward(x, w), lambda: O.norm_backward(x, x, w, mean, rstd), lambda: O.rotary_table(4, 32, device="cuda:0"), lambda: O.rotary_forward(x, x, table),
             lambda: O.rotary_backward(x, None, table), lambda: O.attention_forward(x, x, x), lambda: O.attention_backward(x, x, x, x, o, lse),
             lambda: O.linear_cross_entropy_forward(x, w[None], t), lambda: O.linear_cross_entropy_backward(loss, x, w[None], t, lse_t)]
    for call in calls:
        call()
    monkeypatch.setattr(O, "_device", lambda: 1, raising=False)
    for call in calls:
        with pytest.raises(ValueError, match="cuda:0.*current device"):
            call()
    monkeypatch.undo()
    # (backward passes run on a thread of autograd's, on which the tensors' device is current)
    x.requires_grad_(True)
    O.attention(*O.rotary(O.norm(x, w), x, table), x).sum().backward()
    assert torch.isfinite(x.grad).all()
