"""Calls without a stream take the current stream of the object's device, also with a torch that lacks its short way to
that stream's handle (no GPU needed)."""
import types

import pytest
import torch

import paper_2309_16743_amd as ot
from test_binding_devices import Tensor, backward_args, forward_args


@pytest.mark.parametrize("short_way", [True, False])
def test_the_current_stream(monkeypatch, short_way):
    handles = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: handles.append(args[-1]) or ot.OT_OK

    monkeypatch.setattr(ot, "load", lambda: Library())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    stream = types.SimpleNamespace(cuda_stream=77)
    if short_way:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 77 + device, raising=False)
    else:
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream)
    bank = ot.LowRankAdapters(8, 16, 4, 2)
    clip, adam = ot.GradientClip([Tensor(5)]), ot.AdamTensors(*[[Tensor(5)]] * 4)
    del handles[:]
    bank.forward(**forward_args())
    bank.backward(**backward_args())
    clip.norm(Tensor(1))
    clip.apply(1.0)
    adam.step()
    assert handles == [77] * 5
    bank.forward(**forward_args(), stream=5)
    clip.apply(1.0, stream=types.SimpleNamespace(cuda_stream=6))
    assert handles[5:] == [5, 6]
