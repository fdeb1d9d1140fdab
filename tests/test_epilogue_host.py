"""Host-side refusals of the calls with an activation: they return before anything is launched, so they need no GPU."""
import ctypes as C

import pytest

from paper_2502_08141_amd import lowra
from tests.epilogue_util import ExactLayer

P = 4096              # an aligned address that is never read


def test_act_bwd_refusals():
    f = lowra.lib().lowra_act_bwd
    call = lambda M=4, N=8, act=2, dY=P, z=P, mul=None, dZ=P, dmul=None, db=None, ws=None, nb=0: f(M, N, act, dY, z, mul, dZ, dmul, db, ws, nb, None)
    for kw in (dict(M=-1), dict(N=-8), dict(act=5), dict(act=-1), dict(dZ=None), dict(dY=None), dict(z=None), dict(dmul=P), dict(mul=P, dmul=P),
               dict(act=0, mul=2 * P, dmul=3 * P, z=None)):
        assert call(**kw) == lowra.INVALID_ARG, kw
    assert call(N=12) == lowra.UNSUPPORTED
    for kw in (dict(M=(1 << 30) + 1), dict(N=(1 << 30) + 8), dict(M=0x7fffffff, db=P, ws=P, nb=1 << 40)):       # rows are rounded up in int
        assert call(**kw) == lowra.UNSUPPORTED, kw
    assert lowra.lowra_act_bwd_workspace_bytes(0x7fffffff, 8) == 0 and lowra.lowra_act_bwd_workspace_bytes(64, 12) == 0
    assert lowra.lowra_act_bwd_workspace_bytes(1 << 30, 8) > 0
    for kw in (dict(dY=P + 8), dict(z=P + 2), dict(dZ=P + 4), dict(mul=P + 2), dict(db=P + 4)):
        assert call(**kw) == lowra.MISALIGNED, kw
    need = lowra.lowra_act_bwd_workspace_bytes(4096, 1024)
    assert need > 0 and lowra.lowra_act_bwd_workspace_bytes(0, 1024) == 0
    assert call(M=4096, N=1024, db=P) == lowra.INVALID_ARG
    assert call(M=4096, N=1024, db=P, ws=P, nb=need - 1) == lowra.WORKSPACE_TOO_SMALL
    assert call(M=4096, N=1024, db=P, ws=P + 8, nb=need) == lowra.MISALIGNED
    assert call(N=0) == lowra.OK


def test_linear_refusals():
    L = lowra.lib()
    fe, be = lowra.FwdEpilogue(9, None, None, None, None), lowra.BwdEpilogue(0, None, None, None, P)
    args = lambda e: (None, P, P, P, P, 4, None, None, 0, 1.0, e, P, None, 0, None)
    assert L.lowra_linear_fwd_act(*args(None)) == lowra.INVALID_ARG and L.lowra_linear_bwd_input_act(*args(None)) == lowra.INVALID_ARG
    assert L.lowra_linear_fwd_act(*args(C.addressof(fe))) == lowra.INVALID_ARG             # unknown activation
    assert L.lowra_linear_bwd_input_act(*args(C.addressof(be))) == lowra.INVALID_ARG       # dmul without mul
    fe.act = 0
    assert L.lowra_linear_fwd_act(*args(C.addressof(fe))) == lowra.INVALID_ARG             # null layout


@pytest.mark.parametrize("size", [(8, 64, 1, 0), (264, 576, 16, 5), (520, 1024, 77, 16), (200, 1088, 33, 128)])
def test_layers_of_the_gpu_tests_are_exact(size):
    """Every product fits fp32, and the rank-r intermediates fit bf16 (which the kernels round them to)."""
    E = ExactLayer(*size, device="cpu")
    for t in (0.5 * E.x64 @ E.A64.T, 0.5 * E.dY64 @ E.B64):
        assert t.bfloat16().double().equal(t)
