"""The layers' binding refuses tensors of another device, type or shape than the object's before the library is
called, and passes the right pointers and strides (no GPU needed: the tensors are stand-ins)."""
import pytest
import torch

import paper_2309_16743_amd as ot
from test_binding_devices import Library, Tensor

F32, BF16, I64 = torch.float32, torch.bfloat16, torch.int64


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(ot, "load", lambda: lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ot, "_raw_stream", lambda *a: 0)
    return lib


def dense_forward():
    return {"x": Tensor(3, 8), "w": Tensor(16, 8), "y": Tensor(3, 16), "bias": Tensor(16), "residual": Tensor(3, 16),
            "pre": Tensor(3, 16)}


def dense_backward():
    return {"x": Tensor(3, 8), "w": Tensor(16, 8), "dy": Tensor(3, 16), "pre": Tensor(3, 16), "dx": Tensor(3, 8),
            "dw": Tensor(16, 8), "dbias": Tensor(16)}


def norm_forward():
    return {"x": Tensor(3, 5, 8), "y": Tensor(3, 5, 8), "weight": Tensor(8), "bias": Tensor(8), "stats": Tensor(3, 2, 2)}


def norm_backward():
    return {"x": Tensor(3, 5, 8), "stats": Tensor(3, 2, 2), "dy": Tensor(3, 5, 8), "weight": Tensor(8),
            "bias": Tensor(8), "dx": Tensor(3, 5, 8), "dweight": Tensor(8), "dbias": Tensor(8)}


def dropout_forward():
    return {"x": Tensor(3, 8), "y": Tensor(3, 8), "step": Tensor(1, dtype=I64), "residual": Tensor(3, 8)}


def dropout_backward():
    return {"dy": Tensor(3, 8), "dx": Tensor(3, 8), "step": Tensor(1, dtype=I64)}


CALLS = [(lambda: ot.DenseLayer(8, 16, activation=ot.OT_ACT_GELU), "dense", "forward", dense_forward),
         (lambda: ot.DenseLayer(8, 16, activation=ot.OT_ACT_GELU), "dense", "backward", dense_backward),
         (lambda: ot.GroupNorm(8, 2, positions=5), "norm", "forward", norm_forward),
         (lambda: ot.GroupNorm(8, 2, positions=5), "norm", "backward", norm_backward),
         (lambda: ot.Dropout(0.5, 1), "dropout", "forward", dropout_forward),
         (lambda: ot.Dropout(0.5, 1), "dropout", "backward", dropout_backward)]


@pytest.mark.parametrize("make,kind,name,args", CALLS, ids=[f"{c[1]}-{c[2]}" for c in CALLS])
def test_each_argument(lib, make, kind, name, args):
    op = make()
    getattr(op, name)(**args())
    assert lib.calls == [f"{kind}_create", f"{kind}_{name}"]
    for k in args():
        for device in (1, -1):
            bad = args()
            bad[k].device, bad[k].is_cuda = device, device >= 0
            with pytest.raises(ValueError, match=k):
                getattr(op, name)(**bad)
        bad = args()
        bad[k].dtype = torch.int16
        with pytest.raises(ValueError, match=k):
            getattr(op, name)(**bad)
        if k != "x" and not (k == "dy" and name == "backward" and kind == "dropout"):
            bad = args()
            bad[k].shape = torch.Size([n + 1 for n in bad[k].shape])
            with pytest.raises(ValueError):
                getattr(op, name)(**bad)
    assert len(lib.calls) == 2


def test_what_a_call_needs(lib):
    op = ot.DenseLayer(8, 16, activation=ot.OT_ACT_RELU)
    a = dense_backward()
    for missing, word in (("pre", "pre"), ("x", "dw needs x"), ("w", "dx needs w")):
        with pytest.raises(ValueError, match=word):
            op.backward(**{**a, missing: None})
    op.backward(None, a["w"], a["dy"], pre=a["pre"], dx=a["dx"])
    op.backward(a["x"], None, a["dy"], pre=a["pre"], dw=a["dw"])
    op.backward(None, None, a["dy"], pre=a["pre"], dbias=a["dbias"])
    ot.DenseLayer(8, 16).backward(a["x"], a["w"], a["dy"], dx=a["dx"], dw=a["dw"])
    drop = ot.Dropout(0.5, 1)
    for step in (-1, 1 << 32):
        with pytest.raises(ValueError, match="step"):
            drop.forward(Tensor(3, 8), Tensor(3, 8), step)
    for seed, site in ((-1, 0), (1 << 64, 0), (1, -1), (1, 1 << 32)):
        with pytest.raises(ValueError, match="seed"):
            ot.Dropout(0.5, seed, site=site)


def test_c_names(lib):
    """The functions with C names reach the same calls."""
    for make, kind, name, args in CALLS:
        lib.calls.clear()
        getattr(ot, f"{kind}_{name}")(make(), **args())
        assert lib.calls == [f"{kind}_create", f"{kind}_{name}"]
    for kind, a in (("dense", (8, 16)), ("norm", (8, 2)), ("dropout", (0.5, 1))):
        getattr(ot, f"{kind}_create")(*a)
