"""Targets and weights that begin anywhere: the labels of a causal model are the tokens behind the first."""
import pytest
import torch

from paper_2502_08141_amd import lowra
from tests.test_gpu_vocab_loss import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", [1, 2, 3, 4])
@pytest.mark.parametrize("own_workspace", [False, True])
def test_shifted_targets(first, own_workspace):
    M, V, K = 61, 300, 64
    h, W, targets, weights = make(M, V, K, 31)
    h, W = h.bfloat16(), W.bfloat16()
    kw = {"workspace": torch.empty(lowra.lowra_vocab_loss_workspace_bytes(M - first, V, K), dtype=torch.uint8, device="cuda")} if own_workspace else {}
    want = lowra.lowra_vocab_loss(h[:-first], W, targets[first:].clone(), weights[first:].clone())
    for t, w in ((targets[first:], weights[first:]), (targets[first:].clone(), weights[first:]), (targets[first:], weights[first:].clone())):
        got = lowra.lowra_vocab_loss(h[:-first], W, t, w, **kw)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = lowra.lowra_vocab_loss(h[:-first], W, targets[first:], grad=False, **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_shifted_targets_in_a_graph():
    M, V, K = 40, 500, 64
    h, W, targets, weights = make(M, V, K, 32)
    h, W = h.bfloat16(), W.bfloat16()
    ws = torch.empty(lowra.lowra_vocab_loss_workspace_bytes(M - 1, V, K), dtype=torch.uint8, device="cuda")
    lowra.lowra_vocab_loss(h[:-1], W, targets[1:], weights[1:], workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lowra.lowra_vocab_loss(h[:-1], W, targets[1:], weights[1:], workspace=ws)
    for seed in (33, 34, 35):
        _, _, t, w = make(M, V, K, seed)
        targets.copy_(t); weights.copy_(w)
        graph.replay()
        torch.cuda.synchronize()
        want = lowra.lowra_vocab_loss(h[:-1], W, t[1:].clone(), w[1:].clone())
        assert all(torch.equal(a, b) for a, b in zip(out, want))
