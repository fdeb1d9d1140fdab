"""Every tile of both products of the loss over a vocabulary, with the tiles of words on one scale and on scales of their own."""
import pytest
import torch

from tests.test_gpu_vocab_loss import call, check, formulas, make
from tests.vocab_loss_sizes import TILES, UNITS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,V,K", [t[:3] for t in TILES])
def test_tiles(M, V, K):
    assert torch.cuda.get_device_properties(0).multi_processor_count == UNITS       # the sizes' tiles are those of such a card
    h, W, targets, weights = make(M, V, K, 51, known=0.3)
    h[:, -1], W[:, -1] = 0.0, 0.0
    out = call(h, W, targets, weights)
    check(out, formulas(h, W, targets, weights))
    assert all(torch.equal(a, b) for a, b in zip(out, call(h, W, targets, weights)))
    # tiles of words apart from each other by the last column: every third block of 256 words higher, every third lower, some in the middle of a block
    block = torch.arange(V, device="cuda") // 256 % 3
    W[:, -1] = torch.where(block == 1, 1.0, torch.where(block == 2, -1.0, 0.0)).double()
    W[V - V // 5:V - V // 7, -1] = 0.5
    for lift, rows in ((64.0, slice(None)), (-128.0, slice(None)), (256.0, slice(M // 2, M // 2 + 1)), (48.0, slice(0, None, 7))):
        lifted = h.clone()
        lifted[rows, -1] = lift
        check(call(lifted, W, targets, weights), formulas(lifted, W, targets, weights))
