"""The orthogonalised adapter update against its formulas in 64 bits, and a training step of a layer that uses everything together."""
import math

import pytest
import torch

from paper_2502_08141_amd import lowra
from tests.epilogue_util import S, ExactLayer

pytestmark = pytest.mark.gpu

ABC = (3.4445, -4.7750, 2.0315)


def orthogonalised64(u, steps, abc, eps):
    X = u.double()
    X = X / (X.norm() + eps)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    for _ in range(steps):
        G = X @ X.T
        X = abc[0] * X + (abc[1] * G + abc[2] * G @ G) @ X
    return X.T if tall else X


def f32(v):
    return float(torch.tensor(v, dtype=torch.float32))


def step64(g, m, w, lr, beta, nesterov, decay, steps, scale, abc=ABC, eps=1e-7):
    lr, beta, decay, scale, eps, abc = f32(lr), f32(beta), f32(decay), f32(scale), f32(eps), [f32(v) for v in abc]
    m1 = beta * m.double() + g.double()
    u = g.double() + beta * m1 if nesterov else m1
    X = scale * orthogonalised64(u, steps, abc, eps)
    return m1, X, w.double() - lr * (X + decay * w.double()) if w is not None else None


def spectrum(rows, cols, seed, decades):
    """A gradient whose singular values fall by this many decades."""
    g = torch.Generator().manual_seed(seed)
    r = min(rows, cols)
    U, V = torch.linalg.qr(torch.randn(rows, r, generator=g, dtype=torch.float64))[0], torch.linalg.qr(torch.randn(cols, r, generator=g, dtype=torch.float64))[0]
    return ((U * 10.0 ** (-decades * torch.arange(r) / max(1, r - 1))) @ V.T).float()


# X = p(G) u in 64 bits from the fp32 momentum: what X is off by is its rounding (2^-24) and that of u, which is rounded twice
# (m', u: 2 x 2^-24) before the products grow a small direction by a^steps (485): at most 485 x 2^-23 of |u| / |u| in the norm,
# 2^-14.1, and for random gradients far less.  The Frobenius norm of X is sqrt(R) to a factor of two.
def off_by(X, X64):
    return float((X.double().cpu() - X64).norm() / X64.norm())


SHAPES = [(1, 1), (1, 64), (64, 1), (5, 7), (7, 5), (8, 256), (256, 8), (16, 300), (300, 16), (17, 1000), (1000, 17), (32, 520), (520, 32), (33, 264),
          (264, 33), (48, 4096), (4096, 48), (64, 64), (64, 11008), (11008, 64), (50, 12345), (12345, 50), (3, 4099), (4099, 3)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("decades", [0, 3])
def test_formulas(rows, cols, decades):
    for nesterov, in_place, seed in ((True, False, 1), (False, True, 2)):
        g, m = spectrum(rows, cols, seed, decades), 3 * spectrum(rows, cols, seed + 10, decades)
        w = torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)) * 0.05
        scale = math.sqrt(max(1.0, rows / cols))
        m64, X64, w64 = step64(g, m, w, 0.02, 0.95, nesterov, 0.1, 5, scale)
        gd, md, wd = g.cuda(), m.cuda(), w.cuda()
        up, bf = torch.empty_like(gd), torch.empty_like(gd, dtype=torch.bfloat16)
        mo, wo = (md, wd) if in_place else (torch.empty_like(md), torch.empty_like(wd))
        b = lowra.MuonBatch([lowra.MuonItem(gd, md, wd, bf, up, scale, None if in_place else mo, None if in_place else wo)])
        b.run(lr=0.02, momentum=0.95, nesterov=nesterov, weight_decay=0.1)
        if not in_place:
            assert torch.equal(md.cpu(), m) and torch.equal(wd.cpu(), w)
        # m': two roundings of its terms
        assert ((mo.double().cpu() - m64).abs() <= 2.0 ** -23 * (m.double().abs() + g.double().abs())).all()
        assert off_by(up, X64) <= 485 * 2.0 ** -23, off_by(up, X64)
        # w': lr times what X is off by, and roundings of its terms
        tol = 0.02 * (up.double().cpu() - X64).abs() + 2.0 ** -22 * (w.double().abs() + 0.02 * X64.abs())
        assert ((wo.double().cpu() - w64).abs() <= tol).all()
        assert torch.equal(bf, wo.bfloat16())


def test_random_gradients_are_exact_to_fp32():
    """Without small directions X is off by little more than its own rounding."""
    for rows, cols in ((16, 4096), (4096, 16), (64, 4096), (4096, 64)):
        g = torch.randn(rows, cols, generator=torch.Generator().manual_seed(3))
        zero = torch.zeros_like(g).cuda()
        up = torch.empty_like(zero)
        lowra.MuonBatch([lowra.MuonItem(g.cuda(), zero, update=up)]).run(lr=0.0, momentum=0.0, nesterov=False)
        # singular values of such a g are within a factor of 1.3: nothing grows by more than that beside the rest
        assert off_by(up, orthogonalised64(g, 5, [f32(v) for v in ABC], f32(1e-7))) <= 2.0 ** -23


@pytest.mark.parametrize("steps,abc", [(1, ABC), (2, ABC), (8, (1.5, -0.5, 0.0)), (3, (1.875, -1.25, 0.375))])
def test_steps_and_coefficients(steps, abc):
    for rows, cols in ((12, 500), (500, 40)):
        g = spectrum(rows, cols, 5, 1)
        zero = torch.zeros_like(g).cuda()
        up = torch.empty_like(zero)
        lowra.MuonBatch([lowra.MuonItem(g.cuda(), zero, update=up)]).run(lr=0.0, momentum=0.5, nesterov=False, steps=steps, coefficients=abc)
        X64 = orthogonalised64(g, steps, [f32(v) for v in abc], f32(1e-7))
        assert off_by(up, X64) <= max(1.0, abc[0]) ** steps * 2.0 ** -23


def test_orthogonal():
    """With the convergent coefficients X is orthogonal: its Gram matrix is the identity."""
    g = spectrum(32, 2000, 6, 1)
    zero, up = torch.zeros_like(g).cuda(), torch.empty_like(g).cuda()
    lowra.MuonBatch([lowra.MuonItem(g.cuda(), zero, update=up)]).run(lr=0.0, momentum=0.0, nesterov=False, steps=30, coefficients=(1.5, -0.5, 0.0))
    # quadratic convergence once near: after 30 steps of growth 1.5 from 0.018 nothing is left but rounding
    assert (up.double() @ up.double().T - torch.eye(32, device="cuda", dtype=torch.float64)).abs().max() <= 1e-5


def test_zero_tiny_huge_nan():
    """A zero gradient gives a zero update; magnitudes do not matter beyond eps; NaN and infinity stay in their matrix."""
    shapes = [(16, 512), (512, 16), (16, 512), (512, 16), (16, 512), (40, 300)]
    gs = [torch.randn(s, generator=torch.Generator().manual_seed(i)) for i, s in enumerate(shapes)]
    gs[0].zero_()
    gs[1] *= 1e-30
    gs[2] *= 1e30
    gs[3][5, 5] = float("nan")
    gs[4][5, 5] = float("inf")
    ups = [torch.empty(s, device="cuda") for s in shapes]
    ws = [torch.ones(s, device="cuda") for s in shapes]
    lowra.MuonBatch([lowra.MuonItem(g.cuda(), torch.zeros_like(g).cuda(), w, update=u) for g, u, w in zip(gs, ups, ws)]).run(
        lr=0.5, momentum=0.0, nesterov=False)
    assert (ups[0] == 0).all() and (ws[0] == 1).all()
    for i in (1, 2, 5):
        X64 = orthogonalised64(gs[i], 5, [f32(v) for v in ABC], f32(1e-7))
        assert off_by(ups[i], X64) <= 2.0 ** -22 and ws[i].isfinite().all(), i
    assert ups[3].isnan().all() and ups[4].isnan().all() and ws[3].isnan().all()


def test_batches_of_every_class_and_guards():
    """Many matrices of all short-side classes in one batch, in flat buffers with guards between them; runs repeat bit for bit."""
    shapes = [(8, 320), (320, 8), (20, 512), (264, 20), (64, 512), (512, 64), (16, 64), (33, 777), (777, 31), (5, 3000)] * 3
    sizes = [-(-a * b // 8) * 8 + 8 for a, b in shapes]           # (16-byte aligned as bf16 too)
    flat = lambda dtype=torch.float32: torch.full((sum(sizes),), 7.0, dtype=dtype, device="cuda")
    bufs = {n: flat() for n in ("grad", "momentum", "weight", "momentum_out", "weight_out", "update")} | {"weight_bf16": flat(torch.bfloat16)}
    inside = torch.zeros(sum(sizes), dtype=torch.bool)
    items, at = [], 0
    for i, ((a, b), n) in enumerate(zip(shapes, sizes)):
        v = {k: t[at:at + a * b].view(a, b) for k, t in bufs.items()}
        inside[at:at + a * b] = True
        for k in ("grad", "momentum", "weight"):
            v[k].copy_(torch.randn(a, b, generator=torch.Generator().manual_seed(i)))
        items.append(lowra.MuonItem(**v))
        at += n
    b = lowra.MuonBatch(items)
    kw = dict(lr=0.1, momentum=0.9, weight_decay=0.01)
    b.run(**kw)
    first = {k: t.clone() for k, t in bufs.items()}
    for it in items:
        m64, X64, w64 = step64(it.grad.cpu(), it.momentum.cpu(), it.weight.cpu(), 0.1, 0.9, True, 0.01, 5, 1.0)
        assert off_by(it.update, X64) <= 485 * 2.0 ** -23 and off_by(it.weight_out, w64) <= 2.0 ** -20
    for k, t in first.items():
        assert (t.cpu()[~inside] == 7.0).all(), k
    for k in ("momentum_out", "weight_out", "update", "weight_bf16"):
        bufs[k].fill_(3.0)
    b.run(**kw)
    for it, k in [(it, k) for it in items for k in ("momentum_out", "weight_out", "update", "weight_bf16")]:
        at = (getattr(it, k).data_ptr() - bufs[k].data_ptr()) // bufs[k].element_size()
        assert torch.equal(getattr(it, k), first[k][at:at + it.grad.numel()].view_as(it.grad)), k


def test_a_wide_matrix_is_a_tall_one_transposed():
    g = spectrum(24, 900, 8, 2)
    z = torch.zeros_like(g).cuda()
    ups = [torch.empty_like(z), torch.empty(900, 24, device="cuda")]
    lowra.MuonBatch([lowra.MuonItem(g.cuda(), z, update=ups[0]), lowra.MuonItem(g.T.contiguous().cuda(), torch.zeros(900, 24, device="cuda"), update=ups[1])]).run(
        lr=0.0, momentum=0.0, nesterov=False)
    assert float((ups[0] - ups[1].T).norm() / ups[0].norm()) <= 485 * 2.0 ** -23


@pytest.mark.parametrize("rows,cols", [(17, (1 << 24) + 3), ((1 << 24) + 3, 17), (64, (1 << 23) - 1), ((1 << 23) - 4, 64)])
def test_byte_offsets_up_to_two_gigabytes(rows, cols):
    """Against the 64-bit products on the device, in pieces: one library product of 64 x 8388607 left the last columns of its last row
    unwritten (they came out as a X1 + a X0, what the memory held before).  The tolerance is that of off_by's comment."""
    gen = torch.Generator(device="cuda").manual_seed(rows % 1000)
    g, m = (torch.randn(rows, cols, generator=gen, device="cuda") for _ in range(2))
    out, update = torch.full_like(m, 3.0), torch.full_like(m, 3.0)
    batch = lowra.MuonBatch([lowra.MuonItem(g, m, update=update, momentum_out=out)])
    batch.run(lr=0.0, momentum=0.5, nesterov=False, steps=2)
    assert torch.equal(out, torch.add(g, m, alpha=0.5))              # 0.5 m is exact, so one rounding either way
    a, b, c = (f32(v) for v in ABC)
    X = (out.T if rows > cols else out).double()
    X /= X.square().sum().sqrt() + f32(1e-7)
    for _ in range(2):
        G = sum(p @ p.T.contiguous() for p in X.split(1 << 20, 1))
        P = a * torch.eye(len(G), dtype=G.dtype, device="cuda") + b * G + c * G @ G
        X = torch.cat([P @ p.contiguous() for p in X.split(1 << 20, 1)], 1)
    X = X.T if rows > cols else X
    assert float(torch.linalg.vector_norm(X - update) / torch.linalg.vector_norm(X)) <= 485 * 2.0 ** -23
    for part in (slice(0, 4), slice(-4, None)):                      # the ends by themselves
        want, got = (X[part], update[part]) if rows > cols else (X[:, part], update[:, part])
        assert float((want - got).abs().max()) <= 485 * 2.0 ** -23 * float(X.abs().max())
    batch.close()


def test_streams_and_graphs():
    shapes = [(16, 512), (512, 16), (64, 300)]
    t = lambda s, i: torch.randn(s, generator=torch.Generator().manual_seed(i)).cuda()
    items = [lowra.MuonItem(t(s, i), t(s, i + 10), t(s, i + 20), update=torch.empty(s, device="cuda"), momentum_out=torch.empty(s, device="cuda"),
                            weight_out=torch.empty(s, device="cuda")) for i, s in enumerate(shapes)]
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    b = lowra.MuonBatch(items, workspace=ws)
    b.run(lr=0.1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.run(lr=0.1)
    st = torch.cuda.Stream()
    for rep in range(3):
        for i, it in enumerate(items):
            it.grad.copy_(t(it.grad.shape, 100 * rep + i))
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            b.run(lr=0.1)
        st.synchronize()
        want = [x.clone() for it in items for x in (it.update, it.momentum_out, it.weight_out)]
        for it in items:
            it.update.zero_(); it.momentum_out.zero_(); it.weight_out.zero_()
        ws.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, (x for it in items for x in (it.update, it.momentum_out, it.weight_out))))


def test_refusals():
    z = torch.zeros(16, 64, device="cuda")
    ok = dict(grad=z, momentum=z.clone(), weight=z.clone())
    with pytest.raises(ValueError):
        lowra.MuonBatch([])
    for bad, err in ((dict(grad=z.cpu()), TypeError), (dict(weight=z.half()), TypeError), (dict(momentum=z[:8]), ValueError), (dict(grad=z.t()), TypeError),
                     (dict(weight_bf16=z), TypeError), (dict(weight=None), lowra.LowraError)):
        with pytest.raises(err):
            lowra.MuonBatch([lowra.MuonItem(**(ok | bad))])
    big = torch.zeros(65, 65, device="cuda")
    with pytest.raises(lowra.LowraError) as e:
        lowra.MuonBatch([lowra.MuonItem(big, big.clone(), big.clone())])
    assert e.value.status == lowra.UNSUPPORTED
    with pytest.raises(lowra.LowraError) as e:
        lowra.MuonBatch([lowra.MuonItem(**ok)], workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == lowra.WORKSPACE_TOO_SMALL
    off = torch.zeros(16 * 64 + 1, device="cuda")[1:].view(16, 64)
    with pytest.raises(lowra.LowraError) as e:
        lowra.MuonBatch([lowra.MuonItem(**(ok | dict(grad=off)))])
    assert e.value.status == lowra.MISALIGNED
    with pytest.raises(lowra.LowraError) as e:
        lowra.MuonBatch([lowra.MuonItem(**ok), lowra.MuonItem(**ok)])
    assert e.value.status == lowra.INVALID_ARG
    shared = lowra.MuonBatch([lowra.MuonItem(**ok), lowra.MuonItem(z, z.clone(), z.clone())])       # inputs may be
    shared.close()
    b = lowra.MuonBatch([lowra.MuonItem(**ok)])
    for kw in (dict(steps=0), dict(steps=65), dict(eps=0.0), dict(eps=float("nan"))):
        with pytest.raises(lowra.LowraError) as e:
            b.run(lr=0.1, **kw)
        assert e.value.status == lowra.INVALID_ARG
    b.close()
    with pytest.raises(lowra.LowraError):
        b.run(lr=0.1)
    torch.cuda.synchronize()


@pytest.mark.parametrize("M", [4, 40, 300])
def test_training_step_of_a_gated_layer(M):
    """up, gate (silu, times up, z kept) and down (added to the input), back through all three, the adapters' gradients and their
    update: against autograd in 64 bits over the decoded weights."""
    H, F, r = 512, 1088, 8
    up, gate, down = ExactLayer(F, H, M, r, seed=1), ExactLayer(F, H, M, r, seed=2), ExactLayer(H, F, M, r, seed=3)
    layers = [up, gate, down]
    gen = torch.Generator().manual_seed(4)
    x, dOut = (torch.randn(M, H, generator=gen) * s for s in (0.5, 1.0))
    x, dOut = x.bfloat16().cuda(), dOut.bfloat16().cuda()
    lin = lambda L, t, f=lowra.lowra_linear_fwd, **kw: f(*L.state(), t, L.A, L.B, S, **kw)
    lact = lambda L, t, act, f, **kw: f(*L.state(), t, L.A, L.B, S, act, **kw)
    u = lin(up, x)
    h, z = lact(gate, x, lowra.ACT_SILU, lowra.lowra_linear_fwd_act, mul=u, keep_z=True)
    y, _ = lact(down, h, lowra.ACT_NONE, lowra.lowra_linear_fwd_act, residual=x)
    dz, du = lact(down, dOut, lowra.ACT_SILU, lowra.lowra_linear_bwd_input_act, z=z, mul=u)
    dx, _ = lact(up, du, lowra.ACT_NONE, lowra.lowra_linear_bwd_input_act, residual=dOut)
    dx, _ = lact(gate, dz, lowra.ACT_NONE, lowra.lowra_linear_bwd_input_act, residual=dx, dX=dx)
    grads = [g for L, a, d in ((up, x, du), (gate, x, dz), (down, h, dOut)) for g in lowra.lowra_adapter_grads(L.layout, a, d, L.A, L.B, S)]
    items = [lowra.MuonItem(g, torch.zeros_like(g), p.float(), p, scale=math.sqrt(max(1.0, g.shape[0] / g.shape[1])))
             for g, p in zip(grads, [p for L in layers for p in (L.A, L.B)])]
    before = [it.weight.clone() for it in items]
    batch = lowra.MuonBatch(items)
    batch.run(lr=0.02, weight_decay=0.1)
    torch.cuda.synchronize()

    ps = [p.double().requires_grad_() for L in layers for p in (L.A64, L.B64)]
    x64 = x.double().cpu().requires_grad_()
    f64 = lambda i, t: t @ layers[i].W.T + S * (t @ ps[2 * i].T) @ ps[2 * i + 1].T
    out = f64(2, torch.nn.functional.silu(f64(1, x64)) * f64(0, x64)) + x64
    want = torch.autograd.grad((out * dOut.double().cpu()).sum(), [x64, *ps])
    # every tensor between two calls is rounded to bf16 (2^-9 on average in the norm, 2^-8 at most); the longest chain has six: u, h, dz, du, dx
    # and the rank-r product in each call
    far = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())
    assert far(y, out.detach()) <= 6 * 2.0 ** -8 and far(dx, want[0]) <= 6 * 2.0 ** -8
    for g, w in zip(grads, want[1:]):
        assert far(g, w) <= 6 * 2.0 ** -8
    # the update from the gradients that the calls gave
    for it, w, g, p in zip(items, before, grads, [p for L in layers for p in (L.A, L.B)]):
        _, _, w64 = step64(g.cpu(), torch.zeros_like(g).cpu(), w.cpu(), 0.02, 0.95, True, 0.1, 5, it.scale)
        assert far(it.weight, w64) <= 0.02 * 485 * 2.0 ** -23 * float(math.sqrt(min(g.shape)) / w64.norm()) * 2 + 2.0 ** -22
        assert torch.equal(p, it.weight.bfloat16())
