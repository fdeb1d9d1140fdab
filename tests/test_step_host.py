"""Host-side refusals of the norms, rotary positions, the loss over the vocabulary and the AdamW step: they return before anything is launched or
allocated.  Frequencies of the rotary positions, which are made on the host."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2502_08141_amd import lowra

P = lambda i: (1 << 20) | i << 16      # aligned addresses 64 KiB apart that are never read
INV, UNS, MIS, SMALL = lowra.INVALID_ARG, lowra.UNSUPPORTED, lowra.MISALIGNED, lowra.WORKSPACE_TOO_SMALL


def test_norm_refusals():
    L = lowra.lib()

    def fwd(M=4, N=64, kind=0, x=P(1), w=P(2), b=P(3), eps=1e-5, y=P(4)):
        return L.lowra_norm_fwd(M, N, kind, x, w, b, eps, y, None)

    for kw in (dict(M=-1), dict(N=-8), dict(kind=2), dict(kind=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(y=None), dict(y=P(2)), dict(y=P(3)), dict(y=P(1) + 16),
               dict(y=P(1) - 16), dict(w=P(4) + 496)):
        assert fwd(**kw) == INV, kw
    for kw in (dict(N=12), dict(N=16392), dict(M=(1 << 30) + 1)):
        assert fwd(**kw) == UNS, kw
    for k in "xwby":
        assert fwd(**{k: P(9) + 8}) == MIS, k
    assert fwd(M=0, x=None, y=None) == lowra.OK and fwd(N=0, x=None, y=None) == lowra.OK

    def bwd(M=4, N=64, kind=0, dY=P(1), x=P(2), w=P(3), eps=1e-5, res=P(4), dX=P(5), dw=P(6), db=P(7), ws=P(8), nb=1 << 16):
        return L.lowra_norm_bwd(M, N, kind, dY, x, w, eps, res, dX, dw, db, ws, nb, None)

    for kw in (dict(M=-1), dict(N=-8), dict(kind=2), dict(eps=-1.0), dict(dY=None), dict(x=None), dict(res=None, dX=None, dw=None, db=None), dict(dX=None), dict(ws=None), dict(dX=P(1)),
               dict(dX=P(2)), dict(dX=P(3)), dict(dX=P(4) + 16), dict(dw=P(1)), dict(dw=P(7)), dict(db=P(5)), dict(db=P(4)), dict(ws=P(5)), dict(ws=P(2)), dict(dX=P(8))):
        assert bwd(**kw) == INV, kw
    for kw in (dict(N=12), dict(N=16392), dict(M=(1 << 30) + 1)):
        assert bwd(**kw) == UNS, kw
    for k in ("dY", "x", "w", "res", "dX", "dw", "db", "ws"):
        assert bwd(**{k: P(9) + 8}) == MIS, k
    assert bwd(nb=16) == SMALL
    size = lowra.lowra_norm_bwd_workspace_bytes
    assert size(0, 64) == 0 and size(4, 12) == 0 and 0 < size(1, 64) <= size(300, 64)
    assert size(1 << 20, 4096) < 128 << 20


def test_rope_refusals():
    L = lowra.lib()

    def rope(tensors=None, n=None, M=4, D=64, rot=64, layout=0, pos=P(1), turns=P(2), **t):
        one = dict(x=P(4), y=P(6), heads=2, x_token_stride=128, x_head_stride=64, y_token_stride=128, y_head_stride=64) | t
        tensors = [one] if tensors is None else tensors
        arr = (lowra.RopeTensor * max(len(tensors), 1))(*[lowra.RopeTensor(**k) for k in tensors])
        return L.lowra_rope(len(tensors) if n is None else n, C.addressof(arr), M, D, rot, layout, pos, turns, 1.0, 0, None)

    for kw in (dict(n=0), dict(n=-1), dict(M=-1), dict(D=0), dict(rot=0), dict(rot=-2), dict(rot=66), dict(layout=2), dict(pos=None), dict(turns=None), dict(x=None), dict(y=None),
               dict(heads=0), dict(x_token_stride=-128), dict(y_head_stride=-64), dict(y_token_stride=64), dict(y_head_stride=32), dict(y_token_stride=0), dict(y_head_stride=0),
               dict(y=P(4) + 2), dict(y=P(4), y_token_stride=256), dict(y=P(1)), dict(y=P(2)), dict(y=P(1) - 64)):
        assert rope(**kw) == INV, kw
    for kw in (dict(rot=63), dict(n=5, tensors=[dict(x=P(4), y=P(6), heads=1)] * 5), dict(M=(1 << 30) + 1), dict(D=(1 << 20) + 1), dict(M=1 << 28), dict(heads=(1 << 20) + 1)):
        assert rope(**kw) == UNS, kw
    for kw in (dict(pos=P(1) + 2), dict(turns=P(2) + 4), dict(x=P(4) + 1), dict(y=P(6) + 1)):
        assert rope(**kw) == MIS, kw
    assert L.lowra_rope(1, None, 4, 64, 64, 0, P(1), P(2), 1.0, 0, None) == INV
    assert rope(M=0, x=None, y=None, pos=None, turns=None) == lowra.OK
    # heads of two tensors between each other: rows of 6 heads, of which the first 2 and the next 3 are turned in place; refused where they meet
    row = 6 * 64
    part = lambda first, heads, base=P(4): dict(x=base + 128 * first, y=base + 128 * first, heads=heads, x_token_stride=row, x_head_stride=64, y_token_stride=row, y_head_stride=64)
    for bad in ([part(0, 2), part(1, 3)], [part(0, 6), part(5, 1)], [part(2, 3), part(0, 3)], [part(4, 2), part(0, 2, P(4) + 2 * row - 64)],
                [part(0, 2), part(2, 2) | dict(y_token_stride=row + 64)], [part(0, 2), part(0, 2) | dict(y=P(20))]):
        assert rope(bad) == INV, bad


def test_rope_frequencies():
    """Against the formulas in 64 bits: 2^-64 of a turn a unit, 53 bits of it from the frequency."""
    L = lowra.lib()

    def plan(rot, base=10000.0, scaling=0, factor=1.0, original=4096, low=1.0, high=8.0):
        out = np.zeros(max(rot // 2, 1), np.uint64)
        st = L.lowra_rope_frequencies(rot, base, scaling, factor, original, low, high, out.ctypes.data)
        return out.astype(np.float64) * 2.0 ** -64 * 2 * math.pi if st == lowra.OK else st

    for rot in (2, 4, 20, 64, 128, 130):
        for base in (10000.0, 500000.0, 7.5):
            f = np.array([base ** (-2 * j / rot) for j in range(rot // 2)])
            near = lambda got, want: np.testing.assert_allclose(got, want, rtol=1e-13, atol=1e-17)
            near(plan(rot, base), f)
            near(plan(rot, base, lowra.ROPE_SCALE_LINEAR, 4.0), f / 4)
            if rot > 2:
                stretched = plan(rot, base, lowra.ROPE_SCALE_BASE, 4.0)
                near(stretched, np.array([(base * 4.0 ** (rot / (rot - 2))) ** (-2 * j / rot) for j in range(rot // 2)]))
                near(stretched[[0, -1]], [f[0], f[-1] / 4])
            turns = 4096 * f / (2 * math.pi)
            k = np.clip((turns - 1.0) / 7.0, 0, 1)
            near(plan(rot, base, lowra.ROPE_SCALE_TURNS, 8.0), f * (k + (1 - k) / 8))
            place = lambda t: rot * math.log(4096 / (2 * math.pi * t)) / (2 * math.log(base))
            a, b = max(math.floor(place(32.0)), 0), min(math.ceil(place(1.0)), rot - 1)
            k = 1 - np.clip((np.arange(rot // 2) - a) / max(b - a, 1e-3), 0, 1)
            near(plan(rot, base, lowra.ROPE_SCALE_INDEX, 8.0, high=32.0), f * (k + (1 - k) / 8))
    for bad in (dict(rot=0), dict(rot=-2), dict(rot=4, base=1.0), dict(rot=4, base=float("inf")), dict(rot=4, scaling=5), dict(rot=4, scaling=-1), dict(rot=4, scaling=1, factor=0.5),
                dict(rot=4, scaling=1, factor=float("nan")), dict(rot=4, scaling=3, original=0), dict(rot=4, scaling=3, low=0.0), dict(rot=4, scaling=4, low=2.0, high=2.0)):
        assert plan(**bad) == INV, bad
    assert plan(3) == UNS and plan((1 << 20) + 2) == UNS and plan(2, scaling=2, factor=2.0) == UNS
    assert L.lowra_rope_frequencies(4, 10000.0, 0, 1.0, 0, 1.0, 2.0, None) == INV
    with pytest.raises(lowra.LowraError):
        lowra.lowra_rope_frequencies(3, device="cpu")
    t = lowra.lowra_rope_frequencies(8, device="cpu")
    assert t.shape == (4,) and int(t[0]) == round(2.0 ** 64 / (2 * math.pi))


def test_vocab_loss_refusals():
    L = lowra.lib()
    big = lambda i: (i + 1) << 32

    def loss(M=4, V=100, K=64, h=big(1), W=big(2), t=big(3), w=big(4), loss=big(5), lse=big(6), dH=big(7), ws=big(8), nb=1 << 30):
        return L.lowra_vocab_loss(M, V, K, h, W, t, w, loss, lse, dH, ws, nb, None)

    for kw in (dict(M=-1), dict(V=0), dict(V=-5), dict(K=0), dict(K=-8), dict(h=None), dict(W=None), dict(t=None), dict(loss=None), dict(ws=None), dict(dH=big(1)), dict(dH=big(2) + 16),
               dict(loss=big(4)), dict(lse=big(5)), dict(loss=big(3)), dict(lse=big(7)), dict(ws=big(1)), dict(ws=big(7)), dict(dH=big(8) + 1024), dict(W=big(8))):
        assert loss(**kw) == INV, kw
    for kw in (dict(K=60), dict(V=(1 << 21) + 1), dict(K=(1 << 20) + 8), dict(M=(1 << 30) + 1)):
        assert loss(**kw) == UNS, kw
    for k in ("h", "W", "t", "w", "loss", "lse", "dH", "ws"):
        assert loss(**{k: big(20) + 8}) == MIS, k
    assert loss(nb=64) == SMALL
    assert loss(M=0, h=None, W=None, t=None, loss=None, ws=None) == lowra.OK
    size = lowra.lowra_vocab_loss_workspace_bytes
    assert size(0, 100, 64) == 0 and size(4, 0, 64) == 0 and size(4, 100, 60) == 0
    assert 0 < size(4, 100, 64, False) < size(4, 100, 64)
    # tokens are taken in pieces: the workspace does not grow with the batch
    for V, K in ((32000, 4096), (128256, 8192), (50265, 1024), (257, 512), (1000, 16384)):
        assert size(1 << 20, V, K) <= (448 << 20) and size(1 << 20, V, K) == size(1 << 22, V, K)
        assert size(1 << 22, V, K, False) <= (192 << 20)


def test_adamw_refusals():
    L = lowra.lib()
    out = C.c_void_p()
    names = ("grad", "m", "v", "weight", "m_out", "v_out", "weight_out", "weight_bf16", "m_absmax", "v_absmax", "m_absmax_out", "v_absmax_out")

    def item(base, bits=32, **kw):
        d = dict(count=1000, state_bits=bits, lr_scale=1.0, decay_scale=1.0) | {n: P(base + i) for i, n in enumerate(names) if bits == 8 or "absmax" not in n}
        return d | kw

    def create(*items, n=None):
        recs = (lowra.AdamWItemRecord * max(len(items), 1))(*[lowra.AdamWItemRecord(**k) for k in items])
        return L.lowra_adamw_batch_create(len(items) if n is None else n, C.addressof(recs), C.addressof(out))

    assert create(n=0) == INV and create(n=-1) == INV and L.lowra_adamw_batch_create(1, None, C.addressof(out)) == INV and L.lowra_adamw_batch_create(1, None, None) == INV
    for bits in (32, 8):
        for n in ("grad", "m", "v", "weight", "m_out", "v_out", "weight_out"):
            assert create(item(1, bits, **{n: None})) == INV, n
        for n in names:
            if bits == 8 or "absmax" not in n:
                assert create(item(1, bits, **{n: P(30) + (2 if "absmax" in n else 8)})) == MIS, n
        assert create(item(1, bits, count=0)) == INV and create(item(1, bits, count=-5)) == INV and create(item(1, bits, count=(1 << 31) + 1)) == UNS
        assert create(item(1, bits), item(1, bits)) == INV                                  # one tensor twice
        for a in ("m_out", "v_out", "weight_out", "weight_bf16"):
            for b in ("grad", "m", "v", "weight", "weight_bf16", "v_out"):
                if a != b and a != b + "_out":
                    assert create(item(1, bits, **{a: P(1 + names.index(b))})) == INV, (a, b)
            assert create(item(1, bits, **{a: P(1) + 3984})) == INV
            assert create(item(20, bits), item(1, bits, **{a: P(20)})) == INV and create(item(1, bits, **{a: P(20)}), item(20, bits)) == INV
        assert create(item(1, bits, m_out=P(2) + 16)) == INV                                # in place means the same place
    for n in names[8:]:
        assert create(item(1, 8, **{n: None})) == INV and create(item(1, 32, **{n: P(30)})) == INV, n
    assert create(item(1, 16)) == UNS
    far = lambda i: 1 << 40 | i << 36                                                       # three items of 2^31 elements and pieces beyond what a launch has
    assert create(*[dict(count=1 << 31, state_bits=32, lr_scale=1.0, decay_scale=1.0) | {n: far(8 * i + k) for k, n in enumerate(names[:7])} for i in range(8)]) == UNS
    assert not out.value
    step = lowra.AdamWStep(1e-3, 0.9, 0.999, 1e-8, 0.0, 1)
    assert L.lowra_adamw_batch_run(None, C.addressof(step), None, None) == INV
    L.lowra_adamw_batch_destroy(None)

    def state(count=100, signed=1, q=P(1), a=P(2), o=P(3)):
        return L.lowra_adamw_state(count, signed, q, a, o, None)

    for kw in (dict(count=-1), dict(q=None), dict(a=None), dict(o=None), dict(o=P(1)), dict(o=P(2) - 32)):
        assert state(**kw) == INV, kw
    assert state(count=(1 << 33) + 1) == UNS and state(q=P(1) + 4) == MIS and state(o=P(1) + 4) == MIS and state(a=P(2) + 2) == MIS
    assert state(count=0, q=None, a=None, o=None) == lowra.OK
