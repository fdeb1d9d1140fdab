"""The norms' backward pass where a workgroup takes several rounds of rows, the last of them short: in every shape of workgroup (columns to 512, to 1024 with
few and with many rows, to 2048, 4096, 8192 and 16384), with both weight sums."""
import pytest
import torch

from paper_2502_08141_amd import lowra
from tests.test_gpu_norm import EPS, LAYER, RMS, formulas, inputs, near, tolerances

pytestmark = pytest.mark.gpu

SIZES = [(9000, 64), (4097, 512), (8193, 1024), (8200, 520), (16400, 776), (5000, 1024), (2049, 520), (5000, 2048), (2051, 1032), (2500, 4096), (1027, 2056), (1100, 5120),
         (513, 8192), (1030, 16384), (515, 8200)]


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("kind", [LAYER, RMS])
def test_rounds(M, N, kind):
    i = inputs(M, N, 61)
    c = {k: v.cuda() for k, v in i.items()}
    f = formulas(i, kind, True, False, True)
    t = tolerances(i, f, kind, M)
    back = lambda **kw: lowra.lowra_norm_bwd(c["dY"], c["x"], c["weight"], kind, EPS, residual=c["residual"], **kw)
    dX, dw, db = back(weight_grad=True, bias_grad=True)
    near(dX, f["dX"], t["dX"] + 2.0 ** -22 * f["dX"].abs(), "dX", 2.0 ** -8)
    near(dw, f["dweight"], t["dweight"], "dweight")
    near(db, f["dbias"], t["dbias"], "dbias")
    # without the bias, which is another kernel, and without either
    alone = back(weight_grad=True)
    assert torch.equal(alone[0], dX) and torch.equal(alone[1], dw) and torch.equal(back()[0], dX)
    again = back(weight_grad=True, bias_grad=True)
    assert all(torch.equal(a, b) for a, b in zip(again, (dX, dw, db)))
