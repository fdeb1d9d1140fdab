"""The linear calls with an epilogue and the activation's backward pass against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2502_08141_amd import lowra
from tests.epilogue_util import S, ExactLayer, act64, check, check_bwd, check_fwd, slope64

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def normal(shape, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).bfloat16().cuda()


def fwd(L, act, M=None, **kw):
    x = L.x if M is None else L.x[:M].contiguous()
    return lowra.lowra_linear_fwd_act(*L.state(), x, L.A, L.B, S, lowra.ACTS[act], **kw)


def bwd(L, act, M=None, **kw):
    dY = L.dY if M is None else L.dY[:M].contiguous()
    return lowra.lowra_linear_bwd_input_act(*L.state(), dY, L.A, L.B, S, lowra.ACTS[act], **kw)


# operands: bias, mul, residual, kept z; every activation and every operand appears with each kernel
OPERANDS = [(False, False, False, False), (True, False, False, True), (False, True, False, True), (True, False, True, False), (True, True, True, True)]


def run_both(L, act, which, seed):
    bias, mul, residual, keep = OPERANDS[which]
    fs, bs = (L.M, L.N), (L.M, L.K)
    kw = {}
    if bias: kw["bias"] = normal((L.N,), seed)
    if mul: kw["mul"] = normal(fs, seed + 1)
    if residual: kw["residual"] = normal(fs, seed + 2)
    y, z = fwd(L, act, keep_z=keep, workspace=L.workspace(lowra.OP_LINEAR_FWD), **kw)
    assert (z is not None) == keep
    check_fwd(y, z, L.v, act, **kw)
    kw = {}
    if act != "none" or mul: kw["z"] = normal(bs, seed + 3, 2.0)
    if mul: kw["mul"] = normal(bs, seed + 4)
    if residual: kw["residual"] = normal(bs, seed + 5)
    dX, dmul = bwd(L, act, workspace=L.workspace(lowra.OP_LINEAR_BWD_INPUT), **kw)
    assert (dmul is not None) == mul
    check_bwd(dX, dmul, L.g, act, **kw)


# few tokens (general and streaming kernels; K = 1024 and 4096 stream), mid-token tiles of every height, odd group counts,
# narrow and wide matrices
SIZES = [(8, 64, 1, 0), (264, 576, 1, 8), (264, 576, 16, 5), (520, 1024, 4, 16), (136, 4096, 13, 32), (256, 512, 16, 64),
         (264, 576, 17, 8), (136, 128, 40, 0), (520, 1024, 77, 16), (264, 832, 129, 64), (1032, 576, 300, 24), (200, 1088, 333, 128)]


@pytest.mark.parametrize("i,size", list(enumerate(SIZES)), ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else None)
@pytest.mark.parametrize("act", ACTS)
def test_formulas(i, size, act):
    L = ExactLayer(*size, seed=i, mix=(0.5, 0.5, 0.0) if i % 3 == 2 else (0.4, 0.3, 0.3), per_channel=i % 4 == 1, bf16_scales=i % 5 == 3)
    for which in range(len(OPERANDS)):
        run_both(L, act, which, 100 * i + 7 * which)


@pytest.mark.parametrize("mix", [(0.5, 0.5, 0.0), (0.4, 0.3, 0.3)])
@pytest.mark.parametrize("size", [(264, 576, 1, 8), (520, 1024, 300, 64), (776, 832, 270, 16)])
@pytest.mark.parametrize("act", ["gelu", "silu", "none"])
def test_256_column_kernels(size, mix, act):
    L = ExactLayer(*size, seed=3, mix=mix)
    lowra.lowra_set_linear_path(lowra.PATH_GEMM)
    try:
        for which in (1, 4):
            run_both(L, act, which, which)
    finally:
        lowra.lowra_set_linear_path(lowra.PATH_AUTO)


@pytest.mark.parametrize("path", [lowra.PATH_AUTO, lowra.PATH_GEMV])
@pytest.mark.parametrize("M", [1, 5, 16])
def test_few_tokens_back_in_either_kernel(M, path):
    """The mid-token kernel under LOWRA_PATH_AUTO, the streaming one under LOWRA_PATH_GEMV, with a whole workspace and a small one."""
    L = ExactLayer(520, 1024, M, 16, seed=15, bf16_scales=M == 5)
    z, mul, res = normal((M, L.K), 1, 2.0), normal((M, L.K), 2), normal((M, L.K), 3)
    lowra.lowra_set_linear_path(path)
    try:
        for act in ("none", "gelu", "silu"):
            dX, dmul = bwd(L, act, z=z, mul=mul, residual=res, workspace=L.workspace(lowra.OP_LINEAR_BWD_INPUT))
            check_bwd(dX, dmul, L.g, act, z=z, mul=mul, residual=res)
    finally:
        lowra.lowra_set_linear_path(lowra.PATH_AUTO)


def test_few_tokens_of_a_large_matrix_stream():
    """Where the streaming kernel is the faster one for one token (weights past 46 million)."""
    L = ExactLayer(4104, 11776, 1, 8, seed=16, mix=(0.5, 0.5, 0.0))
    z = normal((1, L.K), 1, 2.0)
    dX, _ = bwd(L, "gelu", z=z, workspace=L.workspace(lowra.OP_LINEAR_BWD_INPUT))
    check_bwd(dX, None, L.g, "gelu", z=z)


@pytest.mark.parametrize("tiling", [(256, 256, 0), (192, 192, 0), (128, 128, 0), (256, 192, 1), (256, 128, 2), (192, 128, 1)])
def test_forward_tilings(tiling):
    L = ExactLayer(776, 256, 530, 16, seed=4)
    lowra.lowra_set_fwd_tiling(*tiling)
    try:
        run_both(L, "gelu", 4, 11)
    finally:
        lowra.lowra_set_fwd_tiling()


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("rows", [32, 64, 96, 128, 192])
@pytest.mark.parametrize("mix", [(0.5, 0.5, 0.0), (0.4, 0.3, 0.3)])
def test_mid_tilings(rows, splits, mix):
    for K, seed in ((1024, 0), (832, 1)):
        L = ExactLayer(200, K, 210, 16, seed=seed, mix=mix, per_channel=seed == 1)
        lowra.lowra_set_mid_tiling(rows, splits)
        try:
            for which in (0, 4):
                run_both(L, "silu", which, 13)
        finally:
            lowra.lowra_set_mid_tiling()


def test_split_256_column_input_gradient():
    """Few 256 x 256 tiles and many channels: the contraction is split, the partial tiles' sum has the epilogue."""
    L = ExactLayer(2048, 512, 300, 16, seed=5)
    lowra.lowra_set_linear_path(lowra.PATH_GEMM)
    try:
        run_both(L, "gelu_tanh", 4, 17)
    finally:
        lowra.lowra_set_linear_path(lowra.PATH_AUTO)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N", [(1, 8), (3, 520), (48, 264), (49, 264), (64, 512), (777, 264), (801, 1032), (260, 8200), (4099, 1032)])
def test_activation_backward(M, N, act):
    dY, z, mul = normal((M, N), M), normal((M, N), M + 1, 2.0), normal((M, N), M + 2)
    for with_mul in (False, True):
        m = mul if with_mul else None
        zz = z if act != "none" or with_mul else None
        ws = torch.empty(lowra.lowra_act_bwd_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
        dZ, dmul, db = lowra.lowra_act_bwd(dY, lowra.ACTS[act], z=zz, mul=m, bias_grad=True, workspace=ws)
        assert (dZ is None) == (act == "none" and not with_mul) and (dmul is None) == (not with_mul)
        g = dY.double().cpu()
        check_bwd(dZ, dmul, g, act, z=zz, mul=m)
        # db: fp32 sums of M terms that are off by at most 2^-17 (1 + |z|) of themselves, in a tree of at most M additions
        d = g * (mul.double().cpu() if with_mul else 1.0)
        full = d * (slope64(z.cpu(), act) if act != "none" else 1.0)
        soft = 2.0 ** -17 * (1 + z.double().cpu().abs()) if act not in ("none", "relu") else torch.zeros_like(d)
        tol = (soft * d.abs()).sum(0) + 2.0 ** -21 * full.abs().sum(0) + min(M, 128) * 2.0 ** -24 * full.abs().sum(0) + 1e-30
        assert ((db.double().cpu() - full.sum(0)).abs() <= tol).all()
        again = lowra.lowra_act_bwd(dY, lowra.ACTS[act], z=zz, mul=m, bias_grad=True)       # its own workspace; the same bits
        assert torch.equal(again[2], db) and (dZ is None or torch.equal(again[0], dZ))
        if dZ is not None:
            alone = lowra.lowra_act_bwd(dY, lowra.ACTS[act], z=zz, mul=m)
            assert alone[2] is None and torch.equal(alone[0], dZ)


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_slopes_against_differences(act):
    """dZ for a gradient of ones is the slope: central differences of the activation in 64 bits."""
    z = torch.cat([torch.linspace(-9, 9, 4088), torch.tensor([-3e4, -60.0, -1e-20, 1e-20, 3e-3, 60.0, 3e4, -2.0])]).bfloat16()
    if act == "relu":
        z = z[z.abs() > 1e-3]
        z = z[:z.numel() // 8 * 8]
    ones = torch.ones(1, z.numel(), dtype=torch.bfloat16, device="cuda")
    dZ, _, _ = lowra.lowra_act_bwd(ones, lowra.ACTS[act], z=z.cuda()[None])
    h = 1e-4 * (1 + z.double().abs())
    diff = (act64(z.double() + h, act) - act64(z.double() - h, act)) / (2 * h)
    # the difference is off by h^2 / 6 times the third derivative (at most 4) and by 2^-52 |act| / h
    off = h * h + 2.0 ** -50 * z.double().abs() / h
    assert ((dZ[0].double().cpu() - diff).abs() <= diff.abs() * 2.0 ** -8 * 1.01 + 2.0 ** -17 * (1 + z.double().abs()) * (act != "relu") + off).all()


def test_infinities_and_nan():
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([[inf, -inf, nan, 0.0, 3.4e38, -3.4e38, 200.0, -200.0]], dtype=torch.float32).bfloat16().cuda()
    one = torch.ones_like(z)
    for act, tail in (("relu", 0.0), ("gelu", 0.0), ("gelu_tanh", 0.0), ("silu", 0.0)):
        dZ, dmul, _ = lowra.lowra_act_bwd(one, lowra.ACTS[act], z=z, mul=one)
        dZ, dmul = dZ[0].float().cpu(), dmul[0].float().cpu()
        assert dZ[0] == 1 and dZ[1] == tail and dZ[4] == 1 and dZ[5] == tail and dZ[6] == 1 and dZ[7] == tail, (act, dZ)
        assert dmul[0] == inf and dmul[1] == 0 and dmul[2].isnan() and dmul[3] == 0 and dmul[4] > 3e38 and dmul[5] == 0 and dmul[6] == 200, (act, dmul)
        assert act == "relu" or dZ[2].isnan()
    # an infinite gradient where a relu lets nothing through
    g = torch.full((1, 8), inf, dtype=torch.bfloat16, device="cuda")
    dZ, _, _ = lowra.lowra_act_bwd(g, lowra.ACT_RELU, z=-one)
    assert (dZ == 0).all()
    # infinities in one row of an operand stay in that row
    L = ExactLayer(264, 576, 40, 8, seed=6)
    mul, res = normal((40, 264), 1), normal((40, 264), 2)
    mul[3, :] = inf; res[5, 7] = nan
    y, _ = fwd(L, "silu", mul=mul, residual=res)
    y = y.cpu()
    assert not y[3].isfinite().all() and y[5, 7].isnan()
    y[3] = 0; y[5, 7] = 0
    assert y.isfinite().all()


@pytest.mark.parametrize("M", [1, 16, 40, 300])
def test_rows_behind_the_last_token_and_other_streams(M):
    """Outputs that are the head of a larger buffer: what lies behind stays as it was.  On a stream of the caller's."""
    L = ExactLayer(520, 1024, M, 16, seed=7)
    big = [torch.full((M + 3, c), 7.0, dtype=torch.bfloat16, device="cuda") for c in (L.N, L.N, L.K, L.K)]
    y, z, dX, dmul = (t[:M] for t in big)
    mf, mb, zb = normal((M, L.N), 1), normal((M, L.K), 2), normal((M, L.K), 3)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        fwd(L, "gelu", mul=mf, y=y, z=z)
        bwd(L, "gelu", z=zb, mul=mb, dX=dX, dmul=dmul)
    st.synchronize()
    check_fwd(y, z, L.v, "gelu", mul=mf)
    check_bwd(dX, dmul, L.g, "gelu", z=zb, mul=mb)
    for t in big:
        assert (t[M:] == 7.0).all()


@pytest.mark.parametrize("M,path", [(1, 0), (16, 0), (40, 0), (300, 0), (300, lowra.PATH_GEMM)])
def test_residual_in_place(M, path):
    """The residual may be the result's own buffer."""
    L = ExactLayer(520, 1024, M, 16, seed=13)
    rf, rb, zb = normal((M, L.N), 1), normal((M, L.K), 2), normal((M, L.K), 3)
    y, dX = rf.clone(), rb.clone()
    lowra.lowra_set_linear_path(path)
    try:
        fwd(L, "silu", residual=y, y=y)
        bwd(L, "silu", z=zb, residual=dX, dX=dX)
    finally:
        lowra.lowra_set_linear_path(lowra.PATH_AUTO)
    check_fwd(y, None, L.v, "silu", residual=rf)
    check_bwd(dX, None, L.g, "silu", z=zb, residual=rb)


def test_no_tokens():
    L = ExactLayer(264, 576, 4, 8, seed=8)
    y, z = fwd(L, "gelu", M=0, keep_z=True)
    assert tuple(y.shape) == tuple(z.shape) == (0, 264)
    e = torch.empty((0, 576), dtype=torch.bfloat16, device="cuda")
    dX, dmul = bwd(L, "silu", M=0, z=e, mul=e)
    assert tuple(dX.shape) == tuple(dmul.shape) == (0, 576)
    for ws in (None, torch.empty(16, dtype=torch.uint8, device="cuda")):
        dZ, _, db = lowra.lowra_act_bwd(e, lowra.ACT_GELU, z=e, bias_grad=True, workspace=ws)
        assert tuple(dZ.shape) == (0, 576) and tuple(db.shape) == (576,) and (db == 0).all()


@pytest.mark.parametrize("M", [4, 64])
def test_native_and_checked_calls_agree(M, monkeypatch):
    L = ExactLayer(264, 1024, M, 8, seed=9)
    b, mf, rf, zb, mb = normal((L.N,), 0), normal((M, L.N), 1), normal((M, L.N), 2), normal((M, L.K), 3), normal((M, L.K), 4)
    wf, wb = L.workspace(lowra.OP_LINEAR_FWD), L.workspace(lowra.OP_LINEAR_BWD_INPUT)
    wa = torch.empty(lowra.lowra_act_bwd_workspace_bytes(M, L.K), dtype=torch.uint8, device="cuda")

    def run():
        return [*fwd(L, "silu", bias=b, mul=mf, residual=rf, keep_z=True, workspace=wf), *bwd(L, "silu", z=zb, mul=mb, workspace=wb),
                *lowra.lowra_act_bwd(zb, lowra.ACT_SILU, z=zb, mul=mb, bias_grad=True, workspace=wa)]
    native = run()
    with monkeypatch.context() as m:
        m.setattr(lowra, "_call", type("none", (), {k: staticmethod(lambda *a: None) for k in ("linear_act", "act_bwd")}))
        plain = run()
    assert all(p.dtype == q.dtype and torch.equal(p, q) for p, q in zip(native, plain))


def test_refusals():
    L = ExactLayer(264, 576, 40, 8, seed=10)
    ok, f32 = normal((40, 264), 1), torch.zeros((40, 264), device="cuda")
    wf, wb = L.workspace(lowra.OP_LINEAR_FWD), L.workspace(lowra.OP_LINEAR_BWD_INPUT)
    zb = normal((40, 576), 2)
    for w in (None, wf):
        for kw, err in ((dict(mul=f32), TypeError), (dict(mul=ok.t()), TypeError), (dict(mul=ok[:39]), ValueError), (dict(bias=ok), ValueError),
                        (dict(residual=ok.cpu()), TypeError)):
            with pytest.raises(err):
                fwd(L, "gelu", workspace=w, **kw)
        with pytest.raises(lowra.LowraError) as e:
            lowra.lowra_linear_fwd_act(*L.state(), L.x, L.A, L.B, S, 9, workspace=w)
        assert e.value.status == lowra.INVALID_ARG
    for w in (None, wb):
        for kw in (dict(), dict(mul=zb)):                            # no z
            with pytest.raises(lowra.LowraError) as e:
                bwd(L, "gelu", workspace=w, **kw)
            assert e.value.status == lowra.INVALID_ARG
    with pytest.raises(lowra.LowraError) as e:
        fwd(L, "gelu", workspace=wf[:16])
    assert e.value.status == lowra.WORKSPACE_TOO_SMALL
    off = torch.empty(40 * 264 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(40, 264)
    with pytest.raises(lowra.LowraError) as e:
        fwd(L, "gelu", mul=off)
    assert e.value.status == lowra.MISALIGNED
    y = torch.empty_like(ok)
    for kw in (dict(y=y, z=y), dict(z=ok, mul=ok), dict(z=ok, residual=ok)):
        with pytest.raises(lowra.LowraError):
            fwd(L, "gelu", **kw)
    dX = torch.empty_like(zb)
    for kw in (dict(dX=dX, dmul=dX), dict(dmul=zb)):
        with pytest.raises(lowra.LowraError):
            bwd(L, "gelu", z=zb, mul=zb, **kw)
    with pytest.raises(lowra.LowraError):
        lowra.lowra_act_bwd(zb, lowra.ACT_GELU)
    with pytest.raises(lowra.LowraError):
        lowra.lowra_act_bwd(zb, lowra.ACT_NONE)                      # nothing asked for
    with pytest.raises(lowra.LowraError) as e:
        lowra.lowra_act_bwd(normal((4, 12), 0), lowra.ACT_NONE, bias_grad=True)
    assert e.value.status == lowra.UNSUPPORTED
    torch.cuda.synchronize()


def test_more_columns_than_a_tile_addresses():
    """256 rows of 2^22 columns reach 2^31 bytes: refused, where the call without an epilogue goes on."""
    for N, K, fn, cols_in in ((1 << 22, 64, lowra.lowra_linear_fwd_act, 64), (8, 1 << 22, lowra.lowra_linear_bwd_input_act, 8)):
        layout = lowra.Layout(K, np.full(N, 2, np.uint8), np.zeros(N, np.uint8), np.array([2], np.uint8))
        packed = torch.zeros(layout.packed_bytes, dtype=torch.uint8, device="cuda")
        absmax, mappings = torch.zeros((N, K // 64), device="cuda"), torch.zeros((1, 16), device="cuda")
        with pytest.raises(lowra.LowraError) as e:
            fn(layout, packed, absmax, mappings, torch.zeros((1, cols_in), dtype=torch.bfloat16, device="cuda"), None, None, 1.0, lowra.ACT_NONE)
        assert e.value.status == lowra.UNSUPPORTED


@pytest.mark.parametrize("M", [4, 17, 40, 300])
def test_rank_r_products_are_left_for_the_adapter_gradients(M):
    L = ExactLayer(264, 576, M, 8, seed=15)
    z = normal((M, 576), 1)
    wf, wb = L.workspace(lowra.OP_LINEAR_FWD), L.workspace(lowra.OP_LINEAR_BWD_INPUT)
    fwd(L, "gelu", mul=normal((M, 264), 2), keep_z=True, workspace=wf)
    bwd(L, "gelu", z=z, residual=z, workspace=wb)
    st, su = (lowra.lowra_linear_side_product(L.layout, op, M, 8, w) for op, w in ((lowra.OP_LINEAR_FWD, wf), (lowra.OP_LINEAR_BWD_INPUT, wb)))
    assert (st is None) == (M <= 16) and (su is None) == (M <= 16)
    if M > 16:
        want = lowra.lowra_adapter_grads(L.layout, L.x, L.dY, L.A, L.B, S)
        assert all(torch.equal(a, b) for a, b in zip(lowra.lowra_adapter_grads_from_side(L.layout, L.x, L.dY, 8, st, su), want))


def test_outputs_past_four_gigabytes():
    """The rows of a small call over and over: 138240 x 16384 values are 4.5 GB.  Every product is exact, so that the small call's bits
    come out again whichever tiles the rows fall into."""
    copies = 540
    wide, tall = ExactLayer(16384, 64, 256, 8, seed=13), ExactLayer(64, 16384, 256, 8, seed=14)
    big = lambda t: t.repeat(copies, 1)
    same = lambda t, small: bool((t.view(copies, *small.shape) == small).all())
    mul, z = normal((256, 16384), 1), normal((256, 16384), 2)
    mul_big, z_big = big(mul), big(z)

    few = fwd(wide, "silu", mul=mul, residual=z, keep_z=True)
    many = lowra.lowra_linear_fwd_act(*wide.state(), big(wide.x), wide.A, wide.B, S, lowra.ACT_SILU, mul=mul_big, residual=z_big, keep_z=True)
    assert all(same(m, f) for m, f in zip(many, few))
    del many
    few = bwd(tall, "gelu", z=z, mul=mul)
    many = lowra.lowra_linear_bwd_input_act(*tall.state(), big(tall.dY), tall.A, tall.B, S, lowra.ACT_GELU, z=z_big, mul=mul_big)
    assert all(same(m, f) for m, f in zip(many, few))
    del many
    few = lowra.lowra_act_bwd(mul, lowra.ACT_GELU_TANH, z=z, bias_grad=True)
    many = lowra.lowra_act_bwd(mul_big, lowra.ACT_GELU_TANH, z=z_big, bias_grad=True)
    assert same(many[0], few[0])
    # sums of the same fp32 terms: at most 138240 / (8 x 256 / 32) + 64 + 2048 / 32 additions in a row, 2^-24 each; |dZ| is at most its bf16 rounding up
    size = few[0].double().abs().sum(0) * 1.01
    assert ((many[2].double() / copies - few[2].double()).abs() <= 2400 * 2.0 ** -24 * size).all()


def test_graph_replays():
    L = ExactLayer(520, 1024, 64, 16, seed=11)
    few = ExactLayer(520, 1024, 4, 16, seed=12)
    mul, res, z, mb = normal((64, 520), 1), normal((64, 520), 2), normal((64, 1024), 3), normal((64, 1024), 4)
    y, zo, dX, dm = (torch.empty_like(t) for t in (mul, mul, z, z))
    y4, dX4 = torch.empty((4, 520), dtype=torch.bfloat16, device="cuda"), torch.empty((4, 1024), dtype=torch.bfloat16, device="cuda")
    z4 = z[:4].contiguous()
    ws = [torch.empty(1 << 24, dtype=torch.uint8, device="cuda") for _ in range(5)]
    out = []

    def calls():
        fwd(L, "gelu", mul=mul, residual=res, y=y, z=zo, workspace=ws[0])
        bwd(L, "gelu", z=z, mul=mb, dX=dX, dmul=dm, workspace=ws[1])
        fwd(few, "silu", y=y4, workspace=ws[2])
        bwd(few, "silu", z=z4, dX=dX4, workspace=ws[3])
        return lowra.lowra_act_bwd(dX, lowra.ACT_SILU, z=z, bias_grad=True, workspace=ws[4])

    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = calls()
    gen = torch.Generator(device="cuda").manual_seed(5)
    for rep in range(3):
        for t in (mul, res, z, mb, L.x, L.dY, few.x, few.dY):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        z4.copy_(z[:4])
        eager = calls()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, zo, dX, dm, y4, dX4, eager[0], eager[2])]
        for t in (y, zo, dX, dm, y4, dX4, captured[0], captured[2], *ws):
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip((y, zo, dX, dm, y4, dX4, captured[0], captured[2]), want):
            assert torch.equal(a, b), rep
