"""Refusals of the calls with an activation and of their binding that need no GPU: they return before anything is launched."""
import pytest
import torch

from paper_2502_08141_amd import lowra

P = 1 << 20           # aligned addresses that are never read


def test_act_bwd_outputs_overlap_nothing():
    """4 x 64 operands of 512 bytes on pages of their own, but for one tensor at a time.  (What is allowed launches.)"""
    f = lowra.lib().lowra_act_bwd
    page = lambda i: P + (i << 12)
    fine = dict(dY=page(0), z=page(1), mul=page(2), dZ=page(3), dmul=page(4), db=page(5))
    assert lowra.lowra_act_bwd_workspace_bytes(4, 64) == 0
    call = lambda kw: f(4, 64, 2, kw["dY"], kw["z"], kw["mul"], kw["dZ"], kw["dmul"], kw["db"], None, 0, None)
    for out in ("dZ", "dmul"):
        for other in fine:
            if other != out:
                for shift in (0, 16, -16, 496, -496):
                    if other == "db" and shift in (496, -496):
                        shift = 240 if shift > 0 else -496   # (256 bytes)
                    if (out, other, shift) != ("dZ", "dY", 0):
                        assert call(fine | {out: fine[other] + shift}) == lowra.INVALID_ARG, (out, other, shift)
    for other in ("dY", "z", "mul", "dZ", "dmul"):
        for shift in (0, 496, -240):
            assert call(fine | {"db": fine[other] + shift}) == lowra.INVALID_ARG, (other, shift)
    assert call(fine | {"dmul": fine["dY"], "dZ": fine["dY"]}) == lowra.INVALID_ARG


class OnDevice:
    """What the binding looks at of a tensor."""

    def __init__(self, shape, dtype=torch.bfloat16, index=0):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, torch.device("cuda", index), True

    def is_contiguous(self): return True
    def dim(self): return len(self.shape)
    def numel(self): return self.shape.numel()
    def data_ptr(self): return P


class Library:
    """Counts the calls that reach it."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def entry(*_):
            self.calls += 1
            return 0
        return entry


@pytest.fixture
def library(monkeypatch):
    lowra.lib()                                            # (the native calls of the binding are there, and decline these tensors)
    L = Library()
    monkeypatch.setattr(lowra, "lib", lambda: L)
    monkeypatch.setattr(lowra, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "empty_like", lambda t: OnDevice(t.shape, t.dtype, t.device.index))
    monkeypatch.setattr(torch, "empty", lambda *a, dtype, device: OnDevice([1], dtype, device.index))
    return L


@pytest.mark.parametrize("which", ["fwd", "bwd"])
def test_linear_tensors_on_another_device(library, which):
    layout = type("layout", (), {"N": 64, "K": 128, "C": 3, "packed_bytes": 2048, "scale_dtype": torch.float32, "handle": P})()
    fn = lowra.lowra_linear_fwd_act if which == "fwd" else lowra.lowra_linear_bwd_input_act
    cols_in, cols = (128, 64) if which == "fwd" else (64, 128)
    fine = {"packed": ([2048], torch.uint8), "absmax": ([64, 2], torch.float32), "mappings": ([3, 16], torch.float32), "act": ([5, cols_in], torch.bfloat16),
            "A": ([4, 128], torch.bfloat16), "B": ([64, 4], torch.bfloat16), "workspace": ([4096], torch.uint8), "mul": ([5, cols], torch.bfloat16),
            "residual": ([5, cols], torch.bfloat16), "z": ([5, cols], torch.bfloat16)}
    fine |= {"y": ([5, cols], torch.bfloat16), "bias": ([64], torch.bfloat16)} if which == "fwd" else {"dX": ([5, cols], torch.bfloat16), "dmul": ([5, cols], torch.bfloat16)}
    for other in [None, *fine]:
        t = {k: OnDevice(*v, index=int(k == other)) for k, v in fine.items()}
        args = [layout] + [t.pop(k) for k in ("packed", "absmax", "mappings", "act", "A", "B")]
        if other is None:
            fn(*args, 1.0, lowra.ACT_GELU, **t)
            assert library.calls == 1
        else:
            with pytest.raises(ValueError):
                fn(*args, 1.0, lowra.ACT_GELU, **t)
            assert library.calls == 1, other


def test_act_bwd_and_update_tensors_on_another_device(library):
    b = lambda i=0: OnDevice([5, 64], index=i)
    ws = lambda i=0: OnDevice([4096], torch.uint8, i)
    call = lambda dY=0, z=0, mul=0, w=0: lowra.lowra_act_bwd(b(dY), lowra.ACT_GELU, z=b(z), mul=b(mul), bias_grad=True, workspace=ws(w))
    call()
    assert library.calls == 1
    for kw in (dict(dY=1), dict(z=1), dict(mul=1), dict(w=1), dict(dY=1, z=1, mul=1, w=1)):
        with pytest.raises(ValueError):
            call(**kw)
    assert library.calls == 1
    f = lambda i=0: OnDevice([8, 64], torch.float32, i)
    for at, w in ((0, 1), (1, 0), (1, 1)):
        before = library.calls
        with pytest.raises(ValueError):
            lowra.MuonBatch([lowra.MuonItem(f(at), f(at), f(at))], workspace=ws(w))
        assert library.calls - before <= 1                 # (the size of the workspace is asked for)
    with pytest.raises(ValueError):
        lowra.MuonBatch([lowra.MuonItem(f(), f(), f()), lowra.MuonItem(f(), f(1), f())], workspace=ws())
