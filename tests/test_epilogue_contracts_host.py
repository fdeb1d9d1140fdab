"""Refusals of the calls with an activation and of their binding that need no GPU: they return before anything is launched."""
import pytest

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
