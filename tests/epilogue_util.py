"""Quantized layers whose products are exact in fp32, and the epilogues' formulas in 64 bits.

Levels, scales, activations and adapters are small multiples of powers of two: every decoded weight, every rank-r product and
every partial sum is then exact in the type it is held in, whatever the order, so that what a call's outputs differ by from the
formulas is its epilogue's alone."""
import numpy as np
import torch

from oracle import lowra_oracle as orc
from paper_2502_08141_amd import lowra

LEVELS = {1: np.array([-1.0, 0.5]), 2: np.array([-1.0, -0.5, 0.25, 1.0]), 4: np.arange(-8, 8) / 8.0}
S = 0.5


class ExactLayer:
    def __init__(self, N, K, M, r, seed=0, mix=(0.4, 0.3, 0.3), per_channel=False, bf16_scales=False, device="cuda"):
        rng = np.random.default_rng([seed, N, K, M, r])
        self.N, self.K, self.M, self.r = N, K, M, r
        bits = rng.choice(np.array([1, 2, 4], np.uint8), size=N, p=mix)
        if per_channel:
            cb, widths = np.arange(N, dtype=np.int32), bits
        else:
            cb, widths = np.searchsorted([1, 2, 4], bits).astype(np.int32), np.array([1, 2, 4], np.uint8)
        mp = np.zeros((widths.size, 16), np.float32)
        for c, b in enumerate(widths):
            mp[c, :1 << b] = LEVELS[int(b)]
        absmax = rng.choice(np.array([0.015625, 0.03125, 0.0625], np.float32), size=(N, K // 64))
        packed = rng.integers(0, 256, int(bits.astype(np.int64).sum()) * K // 8, dtype=np.uint8)
        W = orc.dequantize(packed, absmax, bits, cb, mp, K)
        self.W = torch.from_numpy(W.astype(np.uint16).view(np.int16)).view(torch.bfloat16).double()
        x, dY = rng.integers(-2, 3, (M, K)), rng.integers(-2, 3, (M, N))
        A, B = np.zeros((r, K)), np.zeros((N, r))
        for j in range(r):                                 # sixteen entries each: the rank-r products are small integers times S
            A[j, rng.choice(K, 16, replace=K < 16)] = rng.choice([-1.0, 1.0], 16)
            B[rng.choice(N, 16, replace=N < 16), j] = rng.choice([-1.0, 1.0], 16)
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).double()
        self.x64, self.dY64, self.A64, self.B64 = t(x), t(dY), t(A), t(B)
        self.v = self.x64 @ self.W.T + S * (self.x64 @ self.A64.T) @ self.B64.T
        self.g = self.dY64 @ self.W + S * (self.dY64 @ self.B64) @ self.A64
        for e in (self.v, self.g):
            assert torch.equal(e, e.float().double())
        if device == "cuda":
            self.layout = lowra.Layout(K, bits, cb, widths)
            if bf16_scales:
                self.layout.set_scale_dtype(torch.bfloat16)
            self.packed, self.mp = torch.from_numpy(packed).cuda(), torch.from_numpy(mp).cuda()
            self.absmax = torch.from_numpy(absmax).cuda().to(torch.bfloat16 if bf16_scales else torch.float32)
            b = lambda a: a.bfloat16().cuda()
            self.x, self.dY, self.A, self.B = b(self.x64), b(self.dY64), b(self.A64) if r else None, b(self.B64) if r else None

    def state(self):
        return self.layout, self.packed, self.absmax, self.mp

    def workspace(self, op):
        return torch.empty(self.layout.workspace_bytes(op, self.M, self.r), dtype=torch.uint8, device="cuda")


def act64(z, act):
    f = torch.nn.functional
    return {"none": lambda t: t, "relu": f.relu, "gelu": f.gelu, "gelu_tanh": lambda t: f.gelu(t, approximate="tanh"), "silu": f.silu}[act](z.double())


def slope64(z, act):
    z = z.double().clone().requires_grad_()
    return torch.autograd.grad(act64(z, act).sum(), z)[0]


# Tolerances.  A result is rounded to bf16 once: half a step, 2^-8 of it.  Before that it is fp32: the activations and their slopes
# are within 2^-17 of |z| and 1 + |z| (gelu: 4e-6 relatively in the distribution function, 2^-18; exp2 of an argument below 2^7
# rounded to 24 bits: 2^-17 relatively at |z| = 90, where only the product with z counts), products and sums 2^-22 of their terms.
def bf16_off(ref, terms):
    return ref.abs() * 2.0 ** -8 * (1 + 2.0 ** -8) + terms + 1e-30


def check(got, ref, terms, what):
    got = got.double().cpu()
    bad = ~((got - ref).abs() <= bf16_off(ref, terms))
    bad &= ~((got == ref) | (got.isnan() & ref.isnan()))
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist())


def check_fwd(y, z, v, act, bias=None, mul=None, residual=None):
    """y and z of a forward call against the formulas; v: the exact products."""
    c = lambda t: t.double().cpu()
    v = v + c(bias) if bias is not None else v
    a = act64(v, act)
    m = c(mul) if mul is not None else torch.ones_like(v)
    ref = a * m + (c(residual) if residual is not None else 0.0)
    terms = (0.0 if act in ("none", "relu") else 2.0 ** -17) * v.abs() * m.abs() + 2.0 ** -22 * (a * m).abs() + 2.0 ** -22 * ref.abs() + 2.0 ** -23 * v.abs() * m.abs()
    check(y, ref, terms, "y")
    if z is not None:
        check(z, v, 2.0 ** -23 * v.abs(), "z")


def check_bwd(dX, dmul, g, act, z=None, mul=None, residual=None):
    c = lambda t: t.double().cpu()
    size = g.abs() + (c(residual).abs() if residual is not None else 0.0)
    g = g + (c(residual) if residual is not None else 0.0)
    soft = 0.0 if act in ("none", "relu") else 2.0 ** -17
    slope = slope64(c(z), act) if act != "none" else torch.ones_like(g)
    za = c(z).abs() if z is not None else torch.zeros_like(g)
    m = c(mul) if mul is not None else torch.ones_like(g)
    if dX is not None:
        ref = g * m * slope
        check(dX, ref, soft * (1 + za) * (g * m).abs() + 2.0 ** -21 * size * m.abs() * (1 + slope.abs()), "dX")
    if dmul is not None:
        ref = g * act64(c(z), act)
        check(dmul, ref, soft * za * g.abs() + 2.0 ** -21 * size * za, "dmul")
