"""Host-side refusals of the orthogonalised adapter update: they return before anything is launched or allocated."""
import ctypes as C

from paper_2502_08141_amd import lowra

P = 4096              # an aligned address that is never read


def test_create_refusals():
    L = lowra.lib()
    out = C.c_void_p()

    def create(n=1, ws=P, nb=1 << 20, **kw):
        rec = lowra.MuonItemRecord(**({"rows": 16, "cols": 64, "scale": 1.0, "grad": P, "momentum": P, "momentum_out": P, "weight": P, "weight_out": P} | kw))
        return L.lowra_muon_batch_create(n, C.addressof(rec), ws, nb, C.addressof(out))

    for kw in (dict(n=0), dict(n=-1), dict(rows=0), dict(cols=-3), dict(grad=None), dict(momentum=None), dict(momentum_out=None), dict(weight=None),
               dict(weight_out=None), dict(weight=None, weight_out=None), dict(weight=None, weight_out=None, update=P, weight_bf16=P), dict(ws=None)):
        assert create(**kw) == lowra.INVALID_ARG, kw
    assert create(rows=65, cols=65) == lowra.UNSUPPORTED and create(rows=65, cols=1 << 20) == lowra.UNSUPPORTED
    assert create(rows=64, cols=1 << 23) == lowra.UNSUPPORTED and create(rows=1 << 29, cols=1) == lowra.UNSUPPORTED
    for k in ("grad", "momentum", "momentum_out", "weight", "weight_out", "weight_bf16", "update"):
        assert create(**{k: P + 4}) == lowra.MISALIGNED, k
    assert create(ws=P + 8) == lowra.MISALIGNED
    assert create(nb=64) == lowra.WORKSPACE_TOO_SMALL
    assert L.lowra_muon_batch_create(1, None, P, 64, C.addressof(out)) == lowra.INVALID_ARG
    assert L.lowra_muon_batch_create(1, None, P, 64, None) == lowra.INVALID_ARG
    assert not out.value


def test_nothing_overlaps_an_output():
    """16 x 64 matrices of 4096 bytes on pages of their own, but for one tensor at a time.  (What is allowed allocates on the device.)"""
    L = lowra.lib()
    out = C.c_void_p()
    page = lambda i: 1 << 20 | i << 12

    def create(items, ws=1 << 28):
        recs = (lowra.MuonItemRecord * len(items))(*[lowra.MuonItemRecord(**({"rows": 16, "cols": 64, "scale": 1.0} | it)) for it in items])
        return L.lowra_muon_batch_create(len(items), C.addressof(recs), ws, 1 << 24, C.addressof(out))

    first = dict(grad=page(1), momentum=page(2), momentum_out=page(2), weight=page(3), weight_out=page(3), weight_bf16=page(4), update=page(5))
    second = {k: v + (16 << 12) for k, v in first.items()}
    for bad in (dict(update=page(1)), dict(update=page(3)), dict(weight_out=page(2)), dict(momentum_out=page(1)), dict(momentum_out=page(2) + 16),
                dict(weight_out=page(3) - 16), dict(weight_bf16=page(5) + 4080), dict(weight_bf16=page(6) - 16), dict(weight_bf16=page(2) + 2048)):
        assert create([first | bad]) == lowra.INVALID_ARG, bad
        assert create([second, first | bad]) == lowra.INVALID_ARG, bad
    assert create([first, first]) == lowra.INVALID_ARG                                    # one matrix twice
    for k in ("momentum_out", "weight_out", "weight_bf16", "update"):
        for other in first.values():
            assert create([first, second | {k: other}]) == lowra.INVALID_ARG, (k, other)
    for k in ("grad", "momentum", "weight"):
        assert create([first, second | {k: page(5)}]) == lowra.INVALID_ARG, k              # an input that another's output overwrites
    # the workspace: one chunk's Gram tile and one polynomial of 256 doubles each, 4096 bytes, so that at page(0) it ends where grad begins
    assert create([first], ws=page(5)) == lowra.INVALID_ARG and create([first], ws=page(0) + 16) == lowra.INVALID_ARG
    assert not out.value


def test_run_and_workspace():
    L = lowra.lib()
    step = lowra.MuonStep(0.1, 0.9, 1, 0.0, 5, 3.4, -4.8, 2.0, 1e-7)
    assert L.lowra_muon_batch_run(None, C.addressof(step), None) == lowra.INVALID_ARG
    assert L.lowra_muon_batch_workspace_bytes(0, None) == 0
    L.lowra_muon_batch_destroy(None)
    sizes = lambda *shapes: L.lowra_muon_batch_workspace_bytes(len(shapes), (lowra.MuonItemRecord * len(shapes))(*[lowra.MuonItemRecord(a, b) for a, b in shapes]))
    assert sizes((65, 65)) == 0 and sizes((0, 4)) == 0
    assert 0 < sizes((16, 64)) < sizes((16, 64), (64, 16)) and sizes((16, 64)) < sizes((64, 64))
