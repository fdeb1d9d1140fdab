"""AdamW with an eps that fp32 does not hold, on elements that never had a gradient."""
import pytest
import torch

from paper_2502_08141_amd import lowra
from tests.test_gpu_adamw import check, cuda, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [1e-15, 1e-30, 1e-37, 1e-40, 1e-46, 1e-300])
@pytest.mark.parametrize("eight", [False, True])
def test_no_gradient(eps, eight):
    """0 / (sqrt(0) + eps) is zero however small eps is: what is left of the update is the decay.  The other elements go by the formula (their root is far above eps)."""
    hyper = dict(lr=1e-2, betas=(0.9, 0.99), eps=eps, weight_decay=0.1, step=3)
    s = make(1000, False, 41, loud=0.5)
    idle = torch.arange(1000) % 3 == 0
    for n in ("grad", "m", "v"):
        s[n] = torch.where(idle, torch.zeros(()), s[n])
    if eight:
        from tests.test_gpu_adamw import coded
        for n in "mv":
            s[n], s[n + "_absmax"] = coded(s[n], n == "m")
    d = cuda(s)
    lowra.AdamWBatch([lowra.AdamWItem(**d)]).run(**hyper)
    assert bool(torch.isfinite(d["weight"]).all())
    check(s, d, eight, hyper=hyper)
