"""What the loss over a vocabulary keeps of its digits: targets far below the rest."""
import pytest
import torch

from tests.test_gpu_vocab_loss import call, check, formulas

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lift", [0.0, 6.0, 12.0, -1.5, 20.0])
def test_target_far_below_small_logits(lift):
    """The other words' logits are around -20 + lift, so that their exponentials are small on a scale of their own, and the target's is 65 to 107 below
    them: smaller than an fp32 number with all its digits."""
    M, V, K = 86, 600, 64
    W, h = torch.zeros(V, K, dtype=torch.float64, device="cuda"), torch.zeros(M, K, dtype=torch.float64, device="cuda")
    W[:500, 0] = 20 + (torch.arange(500, device="cuda") % 8) / 8
    W[:500, 1] = 1.0
    W[500:586, 0] = 85 + torch.arange(86, device="cuda") / 2
    W[586:, 0] = 127.5
    h[:, 0], h[:, 1] = -1.0, lift
    assert torch.equal(h, h.bfloat16().double()) and torch.equal(W, W.bfloat16().double())
    targets = torch.arange(500, 586, dtype=torch.int32, device="cuda")
    weights = torch.ones(M, device="cuda")
    f = formulas(h, W, targets, weights)
    assert float(f["loss"].min()) > 60 and float(f["loss"].max()) > 100
    out = call(h, W, targets, weights)
    check(out, f)
    alone = call(h, W, targets, weights, grad=False)
    assert torch.equal(alone[0], out[0])
