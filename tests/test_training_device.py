"""Kernels run on the current device: tensors on another one are refused before anything is queued."""
import math

import pytest
import torch


def test_another_device_is_refused(monkeypatch):
    from paper_2304_14463_amd import training as tr
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 77 + device, raising=False)
    assert tr._current_stream(0) == 77
    with pytest.raises(ValueError, match="cuda:1.*cuda:0"):
        tr._current_stream(1)


@pytest.mark.gpu
def test_every_call_asks_for_the_device_of_its_tensors(monkeypatch):
    from paper_2304_14463_amd import training as tr
    bf = lambda: torch.ones(64, 64, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    x, w, k, out = bf(), bf(), tr.moc_checkpoint_write(bf(), "int8"), bf().fill_(math.nan)
    mean, rstd = torch.zeros(64, device="cuda"), torch.ones(64, device="cuda")
    codes = k.codes.clone()
    calls = (lambda: tr.moc_checkpoint_write(x, "int8", out=k), lambda: tr.moc_checkpoint_read(k, torch.bfloat16, out=out), lambda: tr.moc_norm_forward(x, out=out),
             lambda: tr.moc_norm_backward(x, w, None, mean, rstd, out=out), lambda: tr.moc_linear_forward(x, w, out=out), lambda: tr.moc_linear_backward_input(x, w, out=out),
             lambda: tr.moc_linear_backward_weight(x, w, out=out))
    k.codes.zero_()
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for call in calls:
            with pytest.raises(ValueError, match="cuda:0.*cuda:1"):
                call()
    torch.cuda.synchronize()
    assert bool(out.isnan().all()) and not k.codes.any()
    for call in calls:
        call()
    tr.moc_linear_forward(x, w, out=out.zero_(), stream=torch.cuda.current_stream())
    assert torch.equal(out, torch.full_like(out, 64)) and torch.equal(k.codes, codes)
