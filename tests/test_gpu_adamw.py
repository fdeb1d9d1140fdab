"""The AdamW step against its formulas in 64 bits, and 8-bit states code by code."""
import pytest
import torch

from paper_2502_08141_amd import lowra

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1, step=3)


def f32(v):
    return float(torch.tensor(v, dtype=torch.float32))


def make(count, eight, seed=0, loud=2.0):
    g = torch.Generator().manual_seed(seed * 1000 + count)
    r = lambda: torch.randn(count, generator=g)
    size = torch.exp(loud * r())
    s = {"grad": r() * size * 1e-3, "weight": r() * 0.05, "m": r() * size * 1e-3, "v": (r() * size * 1e-3) ** 2}
    if eight:
        for n in "mv":
            s[n], s[n + "_absmax"] = coded(s[n], n == "m")
    return s


def values(q, absmax, signed):
    """fp32, operation by operation."""
    u = q.float() * torch.tensor(1 / 127 if signed else 1 / 255, dtype=torch.float32)
    u = u * u.abs() if signed else (u * u) * (u * u)
    return u * absmax.repeat_interleave(64)[:u.numel()]


def coded(x, signed):
    """A code is the number of borders below: counted one by one, in 64 bits."""
    n = x.numel()
    pad = torch.zeros((n + 63) // 64 * 64).index_copy_(0, torch.arange(n), x.abs()).view(-1, 64)
    A = pad.amax(1)
    most, power = (127, 2) if signed else (255, 4)
    k = torch.arange(most, dtype=torch.float64) + 0.5
    border = (k * k if signed else (k * k) * (k * k))
    q = torch.empty_like(pad, dtype=torch.int64)
    for i in range(0, pad.shape[0], 256):
        q[i:i + 256] = (border * A[i:i + 256, None, None].double() < pad[i:i + 256, :, None].double() * float(most ** power)).sum(2)
    if not signed:
        q = torch.where((pad > 0) & (q < 1), 1, q)
    q = q.view(-1)[:n]
    return ((q * x.sign().long()).to(torch.int8), A) if signed else (q.to(torch.uint8), A)


def step(s, eight, clip=None, lr_scale=1.0, decay_scale=1.0, hyper=HYPER):
    """fp32 m' and v' operation by operation, w' in 64 bits with how far fp32 may be off."""
    b1, b2 = hyper["betas"]
    c = lambda v: torch.tensor(v, dtype=torch.float32)
    m, v = (values(s[n], s[n + "_absmax"], n == "m") if eight else s[n] for n in "mv")
    g = s["grad"] * c(clip) if clip is not None else s["grad"]
    m1, v1 = c(b1) * m + c(1 - b1) * g, c(b2) * v + c(1 - b2) * (g * g)
    d = lambda t: t.double()
    up = d(m1) / (1 - b1 ** hyper["step"]) / ((d(v1) / (1 - b2 ** hyper["step"])).sqrt() + hyper["eps"])
    lr, decay = hyper["lr"] * lr_scale, hyper["weight_decay"] * decay_scale
    w1 = d(s["weight"]) - lr * (up + decay * d(s["weight"]))
    # scalars, two quotients, a root and a sum: 8 roundings of the update; of its product with lr, the decay's and the difference 4
    off = 2.0 ** -20 * lr * (up.abs() + decay * d(s["weight"]).abs()) + 2.0 ** -23 * d(s["weight"]).abs()
    return m1, v1, w1, off


def cuda(s):
    return {k: v.cuda() for k, v in s.items()}


def same(a, b):
    a, b = a.cpu(), b.cpu()
    return torch.equal(a, b) or bool(((a == b) | (a.isnan() & b.isnan())).all())


def check(s, out, eight, **kw):
    m1, v1, w1, off = step(s, eight, **kw)
    if eight:
        for n, t in (("m", m1), ("v", v1)):
            q, A = coded(t, n == "m")
            assert torch.equal(out[n + "_absmax"].cpu(), A), n
            bad = out[n].cpu() != q
            assert not bad.any(), (n, bad.nonzero()[:4], out[n].cpu()[bad][:4], q[bad][:4])
            assert torch.equal(lowra.lowra_adamw_state(out[n], out[n + "_absmax"]).cpu(), values(q, A, n == "m"))
    else:
        assert torch.equal(out["m"].cpu(), m1) and torch.equal(out["v"].cpu(), v1)
    w = out["weight"].double().cpu()
    assert ((w - w1).abs() <= off).all(), float(((w - w1).abs() - off).max())
    if "weight_bf16" in out:
        assert torch.equal(out["weight_bf16"], out["weight"].bfloat16())


COUNTS = [1, 3, 4, 63, 64, 65, 127, 1000, 1023, 1024, 1025, 1088, 4099, 70000]


@pytest.mark.parametrize("count", COUNTS)
@pytest.mark.parametrize("eight", [False, True])
def test_formulas(count, eight):
    s = make(count, eight)
    d = cuda(s)
    bf = torch.empty(count, dtype=torch.bfloat16, device="cuda")
    lowra.AdamWBatch([lowra.AdamWItem(**d, weight_bf16=bf)]).run(**HYPER)              # in place
    check(s, d | {"weight_bf16": bf}, eight)
    # out of place, with a factor of the gradients on the device and others of the item's own
    d = cuda(s)
    names = ["m", "v", "weight"] + (["m_absmax", "v_absmax"] if eight else [])
    outs = {n: torch.full_like(d[n], 5) for n in names}
    b = lowra.AdamWBatch([lowra.AdamWItem(**d, **{n + "_out": outs[n] for n in names}, lr_scale=0.5, decay_scale=0.0)])
    b.run(**HYPER, grad_scale=torch.full((1,), 0.3, device="cuda"))
    check(s, outs, eight, clip=0.3, lr_scale=0.5, decay_scale=0.0)
    assert all(torch.equal(d[n].cpu(), s[n]) for n in s)
    first = {n: t.clone() for n, t in outs.items()}
    b.run(**HYPER, grad_scale=torch.full((1,), 0.3, device="cuda"))
    assert all(torch.equal(first[n], outs[n]) for n in names)


@pytest.mark.parametrize("hyper", [dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, step=1), dict(lr=1e-3, betas=(0.0, 0.0), eps=1e-6, weight_decay=0.01, step=1),
                                   dict(lr=1e-3, betas=(0.95, 0.9999), eps=1e-8, weight_decay=0.01, step=1000000)])
def test_steps_and_betas(hyper):
    for eight in (False, True):
        s = make(3000, eight, 1)
        d = cuda(s)
        lowra.AdamWBatch([lowra.AdamWItem(**d)]).run(**hyper)
        check(s, d, eight, hyper=hyper)


def test_against_torch():
    """Ten steps from zero states beside torch's own AdamW in 64 bits."""
    g = torch.Generator().manual_seed(5)
    w = torch.randn(5000, generator=g)
    p = torch.nn.Parameter(w.double().clone())
    opt = torch.optim.AdamW([p], lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    d = {"grad": torch.empty(5000), "weight": w.clone(), "m": torch.zeros(5000), "v": torch.zeros(5000)}
    d = cuda(d)
    b = lowra.AdamWBatch([lowra.AdamWItem(**d)])
    for t in range(1, 11):
        grad = torch.randn(5000, generator=g) * 0.01
        p.grad = grad.double()
        opt.step()
        d["grad"].copy_(grad)
        b.run(lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1, step=t)
    # ten steps' roundings of the weights, and 2^-20 of ten updates of at most a few lr
    assert float((d["weight"].double().cpu() - p.detach()).abs().max()) <= 10 * (2.0 ** -24 * 5 + 2.0 ** -20 * 4e-3)


def test_borders_go_to_the_lower_code():
    """Magnitudes on a border exactly (a quarter of the largest is 63.5 squared), next to it on both sides, and a v far below its group's largest."""
    A = torch.tensor(2.0 ** -7)
    up, down = torch.nextafter(A / 4, A), torch.nextafter(A / 4, torch.tensor(0.0))
    m = torch.zeros(64)
    m[:8] = torch.stack([A, A / 4, up, down, -A / 4, -up, -down, torch.tensor(0.0)])
    s = {"grad": torch.zeros(64), "weight": torch.ones(64), "m": torch.zeros(64, dtype=torch.int8), "v": torch.zeros(64, dtype=torch.uint8), "m_absmax": torch.zeros(1), "v_absmax": torch.zeros(1)}
    s["grad"] = m.clone()
    d = cuda(s)
    lowra.AdamWBatch([lowra.AdamWItem(**d)]).run(lr=0.0, betas=(0.0, 0.0), step=1)                  # m' = g, v' = g^2
    assert d["m"][:8].tolist() == [127, 63, 64, 63, -63, -64, -63, 0]
    check(s, d, True, hyper=dict(lr=0.0, betas=(0.0, 0.0), eps=1e-8, weight_decay=0.01, step=1))
    # exact borders of every code, as far as fp32 has them, and their neighbours
    k = torch.arange(127, dtype=torch.float64) + 0.5
    x = ((k / 127) ** 2).float()
    for shift in (0, 1, -1):
        y = x if shift == 0 else torch.nextafter(x, torch.full_like(x, float(shift)))
        g = torch.zeros(8 * 64)
        for j in range(0, 127, 16):
            part = y[j:j + 16]
            g[(j // 16) * 64:(j // 16) * 64 + part.numel()] = part
            g[(j // 16) * 64 + 63] = 1.0
        s = {"grad": g, "weight": torch.ones(512), "m": torch.zeros(512, dtype=torch.int8), "v": torch.zeros(512, dtype=torch.uint8), "m_absmax": torch.zeros(8), "v_absmax": torch.zeros(8)}
        d = cuda(s)
        lowra.AdamWBatch([lowra.AdamWItem(**d)]).run(lr=0.0, betas=(0.0, 0.0), step=1)
        check(s, d, True, hyper=dict(lr=0.0, betas=(0.0, 0.0), eps=1e-8, weight_decay=0.01, step=1))
    g = torch.full((64,), 1e-12)
    g[0] = 1.0
    s = {"grad": g, "weight": torch.ones(64), "m": torch.zeros(64, dtype=torch.int8), "v": torch.zeros(64, dtype=torch.uint8), "m_absmax": torch.zeros(1), "v_absmax": torch.zeros(1)}
    d = cuda(s)
    lowra.AdamWBatch([lowra.AdamWItem(**d)]).run(**HYPER)
    assert bool((d["v"][1:] == 1).all()) and int(d["v"][0]) == 255


@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1e-10, 1e10, 1e18])
def test_tiny_and_huge_gradients(scale):
    for eight in (False, True):
        s = make(700, False, 2, loud=1.0)
        s["m"], s["v"] = torch.zeros(700), torch.zeros(700)
        s["grad"] = (s["grad"].double() * 1e3 * scale).float()
        if eight:
            for n in "mv":
                s[n], s[n + "_absmax"] = coded(s[n], n == "m")
        d = cuda(s)
        lowra.AdamWBatch([lowra.AdamWItem(**d)]).run(**HYPER)
        m1, v1, _, _ = step(s, eight)
        if eight:
            for n, t in (("m", m1), ("v", v1)):
                q, A = coded(t, n == "m")
                assert torch.equal(d[n].cpu(), q) and torch.equal(d[n + "_absmax"].cpu(), A)
        else:
            assert torch.equal(d["m"].cpu(), m1) and torch.equal(d["v"].cpu(), v1)
        assert bool(torch.isfinite(d["weight"]).all())


def test_many_items_of_both_widths():
    """Items do not touch each other or what lies between them: the bits of each are those that it has in a batch of its own."""
    counts = [1, 64, 100, 2048, 5000, 333, 16384, 7]
    pool = {}
    items, alone = [], []
    for i, n in enumerate(counts):
        eight = i % 2 == 0
        s = make(n, eight, 10 + i)
        a, b = cuda(s), {}
        for k, t in s.items():                                    # 64 bytes of guard on both sides
            e, have = 64 // t.element_size(), t.numel()
            pool[i, k] = torch.full((have + 2 * e,), 77, dtype=t.dtype, device="cuda")
            b[k] = pool[i, k][e:e + have]
            b[k].copy_(t)
        alone.append(a); items.append(b)
    lowra.AdamWBatch([lowra.AdamWItem(**b, lr_scale=1 + i) for i, b in enumerate(items)]).run(**HYPER)
    for i, (a, b) in enumerate(zip(alone, items)):
        lowra.AdamWBatch([lowra.AdamWItem(**a, lr_scale=1 + i)]).run(**HYPER)
        for k in a:
            assert torch.equal(a[k], b[k]), (i, k)
            e = 64 // a[k].element_size()
            assert bool((pool[i, k][:e] == 77).all() and (pool[i, k][e + a[k].numel():] == 77).all()), (i, k)


def test_past_32_bit_offsets():
    """An item whose tensors are larger than 4 GB, and whose last groups are short: as the same elements in a batch of their own."""
    count = (1 << 30) + 4099
    for eight in (False, True):
        g = torch.Generator(device="cuda").manual_seed(7)
        d = {"grad": torch.empty(count, device="cuda").normal_(generator=g), "weight": torch.empty(count, device="cuda").normal_(generator=g)}
        if eight:
            d |= {"m": torch.randint(-127, 128, (count,), generator=g, device="cuda", dtype=torch.int8), "v": torch.randint(0, 256, (count,), generator=g, device="cuda", dtype=torch.uint8),
                  "m_absmax": torch.rand((count + 63) // 64, generator=g, device="cuda"), "v_absmax": torch.rand((count + 63) // 64, generator=g, device="cuda")}
        else:
            d |= {"m": torch.empty(count, device="cuda").normal_(generator=g), "v": torch.rand(count, generator=g, device="cuda")}
        spans = [(0, 3000), ((1 << 30) - 64, (1 << 30) + 4099)]
        parts = [{k: (t[a // 64:(b + 63) // 64] if "absmax" in k else t[a:b]).clone() for k, t in d.items()} for a, b in spans]
        lowra.AdamWBatch([lowra.AdamWItem(**d)]).run(**HYPER)
        for (a, b), q in zip(spans, parts):
            lowra.AdamWBatch([lowra.AdamWItem(**q)]).run(**HYPER)
            whole = b - a if b == count else (b - a) // 64 * 64                     # (a group that the part cuts has another largest magnitude)
            for k, t in q.items():
                n = (whole + 63) // 64 if "absmax" in k else whole
                first = a // 64 if "absmax" in k else a
                assert torch.equal(d[k][first:first + n], t[:n]), k
        if eight:
            values = lowra.lowra_adamw_state(d["m"], d["m_absmax"])
            assert torch.equal(values[-4099:], lowra.lowra_adamw_state(d["m"][-4099:].clone(), d["m_absmax"][-65:].clone()))
        del d


def test_not_finite_stays_where_it_is():
    for eight in (False, True):
        s = make(256, eight, 3)
        s["grad"][70], s["grad"][140] = float("nan"), float("inf")
        d = cuda(s)
        lowra.AdamWBatch([lowra.AdamWItem(**d)]).run(**HYPER)
        clean = make(256, eight, 3)
        e = cuda(clean)
        lowra.AdamWBatch([lowra.AdamWItem(**e)]).run(**HYPER)
        touched = [70, 140]
        keep = [i for i in range(256) if i not in touched]
        assert torch.equal(d["weight"][keep], e["weight"][keep]) and bool(d["weight"][70].isnan())
        if eight:
            groups = [0, 3]
            for n in "mv":
                assert torch.equal(d[n].view(4, 64)[groups], e[n].view(4, 64)[groups]) and torch.equal(d[n + "_absmax"][groups], e[n + "_absmax"][groups])
                assert not bool(torch.isfinite(d[n + "_absmax"][1:3]).any())
                assert bool(lowra.lowra_adamw_state(d[n], d[n + "_absmax"]).view(4, 64)[1].isnan().all())


def test_graph_and_stream():
    """A captured run repeats its scalars: three replays are three eager runs."""
    for eight in (False, True):
        s = make(5000, eight, 4)
        a, b = cuda(s), cuda(s)
        scale = torch.full((1,), 0.5, device="cuda")
        ba, bb = lowra.AdamWBatch([lowra.AdamWItem(**a)]), lowra.AdamWBatch([lowra.AdamWItem(**b)])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ba.run(**HYPER, grad_scale=scale)
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            bb.run(**HYPER, grad_scale=scale)
            torch.cuda.synchronize()
            assert all(torch.equal(a[k], b[k]) for k in a)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            ba.run(**HYPER)
        st.synchronize()
        bb.run(**HYPER)
        assert all(torch.equal(a[k], b[k]) for k in a)


def test_binding_refusals():
    good = cuda(make(100, False))
    eight = cuda(make(100, True))
    for bad in (good | {"m": good["m"].double()}, good | {"m": eight["m"]}, eight | {"v": good["v"]}, eight | {"m_absmax": None}):
        with pytest.raises((TypeError, AttributeError)):
            lowra.AdamWBatch([lowra.AdamWItem(**bad)])
    for bad in (good | {"v": good["v"][:64].contiguous()}, eight | {"m_absmax": torch.zeros(3, device="cuda")}, good | {"m_absmax": torch.zeros(2, device="cuda")}):
        with pytest.raises(ValueError):
            lowra.AdamWBatch([lowra.AdamWItem(**bad)])
    for bad in ([good, good], [good | {"m": good["grad"]}], [good | {"v": good["m"]}]):
        with pytest.raises(lowra.LowraError) as e:
            lowra.AdamWBatch([lowra.AdamWItem(**b) for b in bad])
        assert e.value.status == lowra.INVALID_ARG
    with pytest.raises(ValueError):
        lowra.AdamWBatch([])
    b = lowra.AdamWBatch([lowra.AdamWItem(**good)])
    for kw in (dict(step=0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(betas=(float("nan"), 0.9))):
        with pytest.raises(lowra.LowraError) as e:
            b.run(lr=0.1, **kw)
        assert e.value.status == lowra.INVALID_ARG
    with pytest.raises(TypeError):
        b.run(lr=0.1, grad_scale=torch.ones(1, device="cuda", dtype=torch.float64))
    with pytest.raises(ValueError):
        b.run(lr=0.1, grad_scale=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        lowra.lowra_adamw_state(eight["m"], torch.zeros(3, device="cuda"))


@pytest.mark.parametrize("eight", [False, True])
def test_large_batch_is_its_items(eight):
    """A batch past the caches, in pieces of four rounds with ragged ends, gives the bits of its items in batches of their own."""
    counts = [1200003, 64, 1, 4095, 4096, 4097, 1000000, 63, 1023, 8193, 1300000, 900001, 1100032, 1250000, 777777, 1000001]
    items = [cuda(make(1000, eight, seed=i)) for i in range(len(counts))]
    for s, n in zip(items, counts):                                     # the same thousand elements over and over (960: whole groups)
        for k, t in list(s.items()):
            if "absmax" in k:
                s[k] = t[:15].repeat((n + 959) // 960)[:(n + 63) // 64].contiguous()
            else:
                s[k] = t[:960].repeat((n + 959) // 960)[:n].contiguous()
    def run(which):
        sets = [{k: v.clone() for k, v in items[i].items()} for i in which]
        copies = [torch.empty(counts[i], dtype=torch.bfloat16, device="cuda") for i in which]
        batch = lowra.AdamWBatch([lowra.AdamWItem(weight_bf16=c, **s) for s, c in zip(sets, copies)])
        batch.run(**HYPER)
        torch.cuda.synchronize()
        return [dict(s, copy=c) for s, c in zip(sets, copies)]
    assert sum(counts) * (18 if eight else 30) > 1 << 27 and max(counts) * 30 < 1 << 27
    for i, out in enumerate(run(range(len(counts)))):
        alone, = run([i])
        assert all(torch.equal(out[k], alone[k]) for k in out), (i, counts[i])
