"""The adapters', clipping's and Adam's binding refuses tensors of another device than the object's, before the
library is called (no GPU needed: the tensors are stand-ins)."""
import pytest
import torch

import paper_2309_16743_amd as ot

F32, I32 = torch.float32, torch.int32


class Tensor:
    """What the binding asks of a tensor."""

    def __init__(self, *shape, dtype=F32, device=0):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, device
        self.is_cuda = device >= 0

    def stride(self, dim=None):
        st = []
        for i in range(len(self.shape)):
            st.append(int(torch.Size(self.shape[i + 1:]).numel()))
        return tuple(st) if dim is None else st[dim]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 4096


class Library:
    """Notes the calls that reach it."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return ot.OT_OK
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(ot, "load", lambda: lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ot, "_raw_stream", lambda *a: 0)
    return lib


def forward_args():
    return {"x": Tensor(3, 8), "w": Tensor(16, 8), "down": Tensor(2, 4, 8), "up": Tensor(2, 4, 16),
            "ids": Tensor(3, dtype=I32), "y": Tensor(3, 16), "bias": Tensor(16), "scale": Tensor(2), "t": Tensor(3, 4)}


def backward_args():
    return {"x": Tensor(3, 8), "w": Tensor(16, 8), "down": Tensor(2, 4, 8), "up": Tensor(2, 4, 16),
            "ids": Tensor(3, dtype=I32), "dy": Tensor(3, 16), "t": Tensor(3, 4), "ddown": Tensor(2, 4, 8),
            "dup": Tensor(2, 4, 16), "dx": Tensor(3, 8), "scale": Tensor(2)}


@pytest.mark.parametrize("device", [1, -1])
@pytest.mark.parametrize("name,args", [("forward", forward_args), ("backward", backward_args)])
def test_adapters(lib, name, args, device):
    bank = ot.LowRankAdapters(8, 16, 4, 2)
    getattr(bank, name)(**args())
    assert lib.calls == ["adapters_create", f"adapters_{name}"]
    for k in args():
        bad = args()
        bad[k].device, bad[k].is_cuda = device, device >= 0
        with pytest.raises(ValueError, match=k):
            getattr(bank, name)(**bad)
    assert len(lib.calls) == 2


@pytest.mark.parametrize("device", [1, -1])
def test_lists(lib, device):
    good, other = Tensor(5), Tensor(5, device=device)
    for args in (([good, other],), ([good], [other])):
        with pytest.raises(ValueError, match="cuda:0"):
            ot.GradientClip(*args)
    for i in range(4):
        arrays = [[other] if i == j else [good] for j in range(4)]
        with pytest.raises(ValueError, match="cuda:0"):
            ot.AdamTensors(*arrays)
    with pytest.raises(ValueError, match="cuda:0"):
        ot.AdamTensors([good], [good], [good], [good], copies=[Tensor(5, dtype=torch.bfloat16, device=device)])
    assert not lib.calls
    clip, adam = ot.GradientClip([good]), ot.AdamTensors([good], [good], [good], [good])
    for call in (lambda t: clip.norm(t), lambda t: clip.apply(1.0, t), lambda t: adam.step(1.0, t)):
        call(Tensor(1))
        with pytest.raises(ValueError, match="norm"):
            call(Tensor(1, device=device))
    assert lib.calls == ["clip_create", "adam_create", "clip_norm", "clip_apply", "adam_step"]
