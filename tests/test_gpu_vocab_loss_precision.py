"""What the loss over a vocabulary keeps of its digits: targets far below the rest, and gradients of probabilities that are held in bf16."""
import pytest
import torch

from tests.test_gpu_vocab_loss import REL, call, check, formulas, make

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


def close(dH, h, W, targets, weights):
    """The gradient is w sum_{v not t} p_v W_v and the target's term, the p_v made of rounded exponentials e_v (1 + d_v), |d_v| <= 2^-8, on a scale where they add up to the
    exact ones.  With s = sum p_v, D = sum p_v d_v / s and C = sum p_v W_v / s over these words it is off by w / (1 + D) sum p_v d_v (W_v - C), as sum p_v (W_v - C) = 0:
    at most 2^-8 (1 + 2^-7) w sum p_v |W_v - C|.  Beside that the exponentials themselves (REL), V fp32 sums one after another, and the output's rounding, 2^-8."""
    f = formulas(h, W, targets, weights)
    M, V = f["there"].numel(), f["V"]
    there = f["there"]
    rows = torch.arange(M, device="cuda")
    t = torch.where(there, targets, 0).long()
    p = torch.softmax(h @ W.T, 1)
    p[rows, t] = 0.0
    C = p @ W / p.sum(1, keepdim=True)
    spread = torch.empty_like(C)
    for m in range(0, M, 32):
        spread[m:m + 32] = (p[m:m + 32, :, None] * (W[None] - C[m:m + 32, None]).abs()).sum(1)
    w = (weights.double() * there)[:, None]
    off = 2.0 ** -8 * (1 + 2.0 ** -7) * w * spread + (f["size"] + f["target"]) * (2 * REL + V * 2.0 ** -24)
    ref = f["dH"]
    bad = ~((dH.double() - ref).abs() <= off * (1 + 2.0 ** -8) + ref.abs() * 2.0 ** -8 + 1.25 * V * 2.0 ** -126)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), dH.double()[bad][:4].tolist(), ref[bad][:4].tolist())


@pytest.mark.parametrize("M,V,K", [(40, 700, 64), (100, 2049, 72), (300, 520, 128), (700, 1500, 64), (1200, 300, 64)])
def test_rounded_probabilities(M, V, K):
    """Tokens whose mass is on one word that is not their target, on a few, and on many; all tokens with a weight."""
    h, W, targets, weights = make(M, V, K, 21, known=0.0, ignored=0.1)
    g = torch.Generator(device="cuda").manual_seed(M)
    sure = torch.randint(0, V, (M,), generator=g, device="cuda")
    h = h / 4 + torch.randint(0, 4, (M, 1), generator=g, device="cuda") * 4 * W[sure]          # for the others, nothing, something and all
    assert torch.equal(h, h.bfloat16().double())
    close(call(h, W, targets, weights)[2], h, W, targets, weights)
    # the same word is sure for every token, and the tiles of words are on scales of their own
    h2, W2 = h.clone(), W.clone()
    h2[:, -1], W2[:, -1] = 64.0, 0.0
    W2[256:, -1] = 1.0
    close(call(h2, W2, targets, weights)[2], h2, W2, targets, weights)
