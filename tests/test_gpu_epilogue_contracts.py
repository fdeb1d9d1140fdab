"""What include/lowra.h promises of the calls with an epilogue beyond their formulas: workspaces, tensors that share memory."""
import numpy as np
import pytest
import torch

from paper_2502_08141_amd import lowra
from tests.epilogue_util import S

pytestmark = pytest.mark.gpu


class Layer:
    """A quantized layer with values of any mantissa: two kernels that add its products in another order give other bits."""

    def __init__(self, N, K, M, r, seed=0, mix=(0.4, 0.3, 0.3)):
        rng = np.random.default_rng([seed, N, K, M, r])
        gen = torch.Generator().manual_seed(seed + 100)
        self.N, self.K, self.M, self.r = N, K, M, r
        bits = rng.choice(np.array([1, 2, 4], np.uint8), size=N, p=mix)
        self.layout = lowra.Layout(K, bits, np.searchsorted([1, 2, 4], bits).astype(np.int32), np.array([1, 2, 4], np.uint8))
        self.packed = torch.from_numpy(rng.integers(0, 256, self.layout.packed_bytes, dtype=np.uint8)).cuda()
        self.absmax = (torch.rand(N, K // 64, generator=gen) + 0.5).cuda()
        self.mp = torch.randn(3, 16, generator=gen).cuda()
        n = lambda *s: torch.randn(*s, generator=gen).bfloat16().cuda()
        self.x, self.dY = n(M, K), n(M, N)
        self.A, self.B = (n(r, K), n(N, r)) if r else (None, None)

    def state(self):
        return self.layout, self.packed, self.absmax, self.mp

    def adapters(self):
        return self.A, self.B, S


def least_workspace(L, call):
    """The fewest bytes that `call` (of a workspace) does not refuse."""
    lo, hi = 0, L.layout.workspace_bytes(lowra.OP_LINEAR_BWD_INPUT, L.M, L.r)
    big = torch.empty(hi, dtype=torch.uint8, device="cuda")
    while hi - lo > 1:
        mid = (lo + hi) // 2
        try:
            call(big[:mid])
            hi = mid
        except lowra.LowraError as e:
            assert e.status in (lowra.WORKSPACE_TOO_SMALL, lowra.INVALID_ARG)
            lo = mid
    return big[:hi]


@pytest.mark.parametrize("N,K,r", [(4096, 4096, 16), (1032, 2048, 8), (2048, 1024, 0)])
@pytest.mark.parametrize("M", [1, 4, 16])
def test_few_tokens_back_without_room_for_splits_stream(N, K, r, M):
    """The mid-token kernel is the faster one for a few tokens where its contraction is split.  Without room for that the streaming
    kernel takes the call: the bits are its own, whatever lies in the workspace."""
    L = Layer(N, K, M, r, seed=21)
    z = torch.randn(M, K, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()

    def call(ws):
        return lowra.lowra_linear_bwd_input_act(*L.state(), L.dY, *L.adapters(), lowra.ACT_SILU, z=z, residual=z, workspace=ws)[0]

    ws = least_workspace(L, call)
    ws.fill_(255)
    got = call(ws)
    lowra.lowra_set_linear_path(lowra.PATH_GEMV)
    try:
        streamed = call(ws)
    finally:
        lowra.lowra_set_linear_path(lowra.PATH_AUTO)
    assert torch.equal(got, streamed)
    whole = torch.empty(L.layout.workspace_bytes(lowra.OP_LINEAR_BWD_INPUT, M, r), dtype=torch.uint8, device="cuda")
    assert whole.numel() > ws.numel()
    # the same sums; a product's operands, the rank-r product and the result are rounded to bf16 once each (2^-8), in the streaming kernel the
    # scaled gradient and the level instead of the weight: five and four roundings
    wide = call(whole).double()
    assert float((got.double() - wide).norm() / wide.norm()) <= 9 * 2.0 ** -8
