"""A fine-tuning step of a decoder block with everything that the library has for one: norms, quantized LoRA linears with their epilogues, rotary
positions, the loss over a vocabulary, the way back through all of them, and the AdamW step on adapters and norm weights -- against autograd in 64 bits over
the decoded weights.  Attention stands between the library's calls as plain fp32 products with their gradient written out."""
import math

import pytest
import torch

from paper_2502_08141_amd import lowra, synth
from tests.gpu_util import DeviceLayer

pytestmark = pytest.mark.gpu

H, F, HEADS, D, ROT, V, R, S = 256, 512, 4, 64, 48, 1003, 8, 2.0
SEQ, BATCH = 24, 3
M = SEQ * BATCH
NAMES = {"q": (H, H), "k": (H, H), "v": (H, H), "o": (H, H), "up": (F, H), "gate": (F, H), "down": (H, F)}
NORM, EPS = lowra.NORM_RMS, 1e-5


class Model:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, k=1.0: (torch.randn(*s, generator=g) * k)
        self.lin, self.W, self.master = {}, {}, {}
        for i, (n, (N, K)) in enumerate(NAMES.items()):
            d = DeviceLayer(synth.make_custom(N, K, 1, R, seed=40 + i))
            d.quantize()
            # (the layer's weights have deviations of their own: the scales bring the products to order one)
            scale = 1.0 / (float(lowra.lowra_dequantize(d.layout, d.packed, d.absmax, d.mp).float().std()) * math.sqrt(K))
            d.absmax = (d.absmax * 2.0 ** round(math.log2(scale))).contiguous()
            self.W[n] = lowra.lowra_dequantize(d.layout, d.packed, d.absmax, d.mp).double().cpu()
            self.lin[n] = d
            self.master[n + ".A"], self.master[n + ".B"] = r(R, K, k=1 / math.sqrt(K)), r(N, R, k=0.1)
        for n in ("n1", "n2", "n3"):
            self.master[n] = 1 + r(H, k=0.1)
        self.master = {n: t.bfloat16().float().cuda() for n, t in self.master.items()}
        self.p = {n: t.bfloat16() for n, t in self.master.items()}
        self.head = r(V, H, k=1 / math.sqrt(H)).bfloat16().cuda()
        self.x = r(M, H).bfloat16().cuda()
        self.targets = torch.where(torch.rand(M, generator=g) < 0.9, torch.randint(0, V, (M,), generator=g), -100).int().cuda()
        self.weights = ((self.targets >= 0).float() / float((self.targets >= 0).sum())).contiguous()
        self.positions = torch.arange(SEQ).repeat(BATCH).int().cuda()
        self.turns = lowra.lowra_rope_frequencies(ROT)
        self.ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def args(self, n):
        d = self.lin[n]
        return d.layout, d.packed, d.absmax, d.mp

    def fwd(self, n, x, act=None, **kw):
        f = lowra.lowra_linear_fwd if act is None else lowra.lowra_linear_fwd_act
        return f(*self.args(n), x, self.p[n + ".A"], self.p[n + ".B"], S, *(() if act is None else (act,)), workspace=self.ws, **kw)

    def bwd(self, n, dY, act=lowra.ACT_NONE, **kw):
        return lowra.lowra_linear_bwd_input_act(*self.args(n), dY, self.p[n + ".A"], self.p[n + ".B"], S, act, workspace=self.ws, **kw)

    def norm(self, n, x):
        return lowra.lowra_norm_fwd(x, self.p[n], None, NORM, EPS)

    def norm_back(self, n, dY, x, residual=None):
        dX, dw, _ = lowra.lowra_norm_bwd(dY, x, self.p[n], NORM, EPS, residual=residual, weight_grad=True, workspace=self.ws)
        return dX, dw


def heads(t):
    return t.float().view(BATCH, SEQ, HEADS, D).transpose(1, 2).contiguous()


def flat(t):
    return t.transpose(1, 2).reshape(M, HEADS, D)


MASK = torch.triu(torch.full((SEQ, SEQ), float("-inf")), 1)


def attention(q, k, v):
    p = torch.softmax(heads(q) @ heads(k).transpose(2, 3).contiguous() / math.sqrt(D) + MASK.cuda(), 3)
    return p, flat(p @ heads(v)).reshape(M, H).bfloat16()


def attention_back(dO, q, k, v, p):
    g = heads(dO)
    dV = p.transpose(2, 3).contiguous() @ g
    dP = g @ heads(v).transpose(2, 3).contiguous()
    dS = p * (dP - (dP * p).sum(3, keepdim=True)) / math.sqrt(D)
    return (flat(t).bfloat16() for t in (dS @ heads(k), dS.transpose(2, 3).contiguous() @ heads(q), dV))


def upper_half(m, ctx):
    """From attention's output to the loss, and back."""
    t = {}
    t["h1"], _ = m.fwd("o", ctx, lowra.ACT_NONE, residual=m.x)
    t["n2"] = m.norm("n2", t["h1"])
    t["u"] = m.fwd("up", t["n2"])
    t["a"], t["z"] = m.fwd("gate", t["n2"], lowra.ACT_SILU, mul=t["u"], keep_z=True)
    t["h2"], _ = m.fwd("down", t["a"], lowra.ACT_NONE, residual=t["h1"])
    t["n3"] = m.norm("n3", t["h2"])
    t["loss"], t["lse"], dn3 = lowra.lowra_vocab_loss(t["n3"], m.head, m.targets, m.weights, workspace=m.ws)
    t["dh2"], t["g.n3"] = m.norm_back("n3", dn3, t["h2"])
    t["dz"], t["du"] = m.bwd("down", t["dh2"], lowra.ACT_SILU, z=t["z"], mul=t["u"])
    dn2, _ = m.bwd("up", t["du"])
    dn2, _ = m.bwd("gate", t["dz"], residual=dn2)
    t["dh1"], t["g.n2"] = m.norm_back("n2", dn2, t["h1"], residual=t["dh2"])
    t["dctx"], _ = m.bwd("o", t["dh1"])
    for n, x, dY in (("o", ctx, t["dh1"]), ("up", t["n2"], t["du"]), ("gate", t["n2"], t["dz"]), ("down", t["a"], t["dh2"])):
        t["g." + n + ".A"], t["g." + n + ".B"] = lowra.lowra_adapter_grads(m.lin[n].layout, x, dY, m.p[n + ".A"], m.p[n + ".B"], S, workspace=m.ws)
    return t


def step(m):
    n1 = m.norm("n1", m.x)
    q, k, v = (m.fwd(n, n1).view(M, HEADS, D) for n in "qkv")
    q, k = lowra.lowra_rope([q, k], m.positions, m.turns)
    p, ctx = attention(q, k, v)
    t = upper_half(m, ctx)
    dq, dk, dv = attention_back(t["dctx"].view(M, HEADS, D), q, k, v, p)
    dq, dk = lowra.lowra_rope([dq, dk], m.positions, m.turns, inverse=True)
    dn1 = None
    for n, dY in (("q", dq), ("k", dk), ("v", dv)):
        dY = dY.reshape(M, H).contiguous()
        dn1, _ = m.bwd(n, dY, residual=dn1)
        t["g." + n + ".A"], t["g." + n + ".B"] = lowra.lowra_adapter_grads(m.lin[n].layout, n1, dY, m.p[n + ".A"], m.p[n + ".B"], S, workspace=m.ws)
    t["dx"], t["g.n1"] = m.norm_back("n1", dn1, m.x, residual=t["dh1"])
    return t, ctx


def exact(m, p, x):
    """The loss in 64 bits as a function of the parameters."""
    norm = lambda n, t: t / torch.sqrt(t.square().mean(1, keepdim=True) + EPS) * p[n]
    lin = lambda n, t: t @ m.W[n].T + S * (t @ p[n + ".A"].T) @ p[n + ".B"].T
    angle = m.positions.cpu().double()[:, None] * torch.tensor([10000.0 ** (-2 * j / ROT) for j in range(ROT // 2)], dtype=torch.float64)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    def turn(t):
        a, b = t[..., :ROT // 2], t[..., ROT // 2:ROT]
        return torch.cat([a * c - b * s, a * s + b * c, t[..., ROT:]], 2)
    n1 = norm("n1", x)
    q, k, v = (lin(n, n1).view(M, HEADS, D) for n in "qkv")
    split = lambda t: t.view(BATCH, SEQ, HEADS, D).transpose(1, 2)
    a = torch.softmax(split(turn(q)) @ split(turn(k)).transpose(2, 3) / math.sqrt(D) + MASK.double(), 3) @ split(v)
    h1 = lin("o", a.transpose(1, 2).reshape(M, H)) + x
    n2 = norm("n2", h1)
    h2 = lin("down", torch.nn.functional.silu(lin("gate", n2)) * lin("up", n2)) + h1
    z = norm("n3", h2) @ m.head.double().cpu().T
    loss = torch.nn.functional.cross_entropy(z, m.targets.cpu().long(), ignore_index=-100, reduction="none")
    return loss, (loss * m.weights.double().cpu()).sum()


def test_gradients_and_update():
    m = Model(1)
    t, _ = step(m)
    names = list(m.p)
    p = {n: m.p[n].double().cpu().requires_grad_() for n in names}
    x = m.x.double().cpu().requires_grad_()
    loss, total = exact(m, p, x)
    want = dict(zip(names + ["x"], torch.autograd.grad(total, [p[n] for n in names] + [x])))
    # Every tensor between two calls is rounded to bf16, by 2^-8 of a value at most and 2^-9 in the norm; with the rank-r products the longest way (from the
    # loss down to the first norm's weight and up to it) has 12 tensors up and 10 down.  A softmax, a silu gate and a norm may double what reaches them.
    far = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())
    off = 22 * 2.0 ** -9 * 2
    assert far(t["loss"], loss.detach()) <= off and far(t["dx"], want["x"]) <= off, (far(t["loss"], loss.detach()), far(t["dx"], want["x"]))
    for n in names:
        assert far(t["g." + n], want[n]) <= off, (n, far(t["g." + n], want[n]))
    # and along a direction, against differences of the 64-bit loss
    g = torch.Generator().manual_seed(5)
    way = {n: torch.randn(p[n].shape, generator=g, dtype=torch.float64) * p[n].detach().std() for n in names}
    moved = lambda e: float(exact(m, {n: p[n].detach() + e * way[n] for n in names}, x.detach())[1])
    slope = (moved(1e-5) - moved(-1e-5)) / 2e-5
    got = sum(float((t["g." + n].double().cpu() * way[n]).sum()) for n in names)
    size = math.sqrt(sum(float((want[n] * way[n]).square().sum()) for n in names))
    assert abs(got - slope) <= off * max(size, abs(slope)) * 2

    # the step on all of them, norm weights without decay: against torch's own in 64 bits from the gradients that the calls gave
    for bits in (32, 8):
        w = {n: m.master[n].clone() for n in names}
        items = []
        for n in names:
            grad = t["g." + n]
            extra = {} if bits == 32 else {"m_absmax": torch.zeros((grad.numel() + 63) // 64, device="cuda"), "v_absmax": torch.zeros((grad.numel() + 63) // 64, device="cuda")}
            items.append(lowra.AdamWItem(grad=grad, m=torch.zeros_like(grad, dtype=torch.float32 if bits == 32 else torch.int8),
                                         v=torch.zeros_like(grad, dtype=torch.float32 if bits == 32 else torch.uint8), weight=w[n],
                                         weight_bf16=torch.empty_like(w[n], dtype=torch.bfloat16), decay_scale=0.0 if n in ("n1", "n2", "n3") else 1.0, **extra))
        norm = torch.sqrt(sum(t["g." + n].square().sum() for n in names))
        clip = (0.5 / norm).clamp(max=1.0).reshape(1)                       # stays on the device
        lowra.AdamWBatch(items).run(lr=1e-3, weight_decay=0.1, step=1, grad_scale=clip)
        for n, it in zip(names, items):
            q = torch.nn.Parameter(m.master[n].double().clone())
            q.grad = t["g." + n].double() * clip.double()
            torch.optim.AdamW([q], lr=1e-3, weight_decay=0.0 if n in ("n1", "n2", "n3") else 0.1).step()
            # 2^-20 of an update of at most lr, three roundings of the weight (test_gpu_adamw.py)
            assert bool(((it.weight.double() - q.detach()).abs() <= 2.0 ** -20 * 1e-3 * 1.2 + 2.0 ** -22 * q.detach().abs()).all()), n
            assert torch.equal(it.weight_bf16, it.weight.bfloat16())


def test_captured_half_and_update():
    """From attention's output to the loss and back, and the update, as one captured graph: replays with new inputs give the eager calls' bits."""
    m = Model(2)
    _, ctx = step(m)
    names = [n for n in m.p if n.split(".")[0] in ("o", "up", "gate", "down", "n2", "n3")]
    t = upper_half(m, ctx)
    torch.cuda.synchronize()

    def build(t, master):
        out = {n: torch.empty_like(m.p[n]) for n in names}
        state = {n: (torch.zeros_like(t["g." + n]), torch.zeros_like(t["g." + n])) for n in names}
        return out, state, lowra.AdamWBatch([lowra.AdamWItem(grad=t["g." + n], m=state[n][0], v=state[n][1], weight=master[n], weight_bf16=out[n]) for n in names])

    live = ctx.clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    upper_half(m, live)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        captured = upper_half(m, live)
    for seed in (1, 2, 3):
        live.copy_(ctx * (1 + seed))
        graph.replay()
        torch.cuda.synchronize()
        eager = upper_half(m, live)
        assert all(torch.equal(captured[n], eager[n]) for n in eager)
        # the update behind it, from the graph's gradients and from the eager ones
        a, b = ({n: m.master[n].clone() for n in names} for _ in range(2))
        for grads, master in ((captured, a), (eager, b)):
            _, _, batch = build(grads, master)
            for step_number in (1, 2):
                batch.run(lr=1e-3, step=step_number)
        assert all(torch.equal(a[n], b[n]) for n in names)
