"""Operators of a fine-tuning step beside the quantized LoRA linear, as measurable cases: the norms around a layer, the rotary
positions of its queries and keys, the loss over the vocabulary with its gradient, and the adaptive step on the adapters.

`run` computes a case in elementary torch operations where `own` is false, and by the library's calls where it is true.

  norm     forward   xh = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)  (rms: mean = 0)    y = xh weight + bias
           backward  g = dY weight    dX = rstd (g - mean(g) - xh mean(g xh)) + residual  (rms: without mean(g))
                     dweight = sum of dY xh, dbias = sum of dY over the tokens
  rope     angle = position f_j, f_j = base^(-2 j / rot) scaled for a longer context; the pair (a, b) of x becomes
           (a cos - b sin, a sin + b cos); inverse: by -angle, which is also the way back of a gradient
  loss     z = h W^T    loss = log(sum exp z) - z_target    dH = weight (softmax(z) - e_target) W;  no target: zero
  adamw    g = clip grad    m' = b1 m + (1 - b1) g    v' = b2 v + (1 - b2) g^2
           w' = w - lr ((m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps) + decay w)
           8 bits: groups of 64, each with its largest magnitude A.  m: a signed code q for sgn(q) (q / 127)^2 A; v: q for
           (q / 255)^4 A, and above zero where v is.  A code counts the borders (k + 1/2) that lie below, on the scale of q.

Shapes are those of the models the repository names (LLaMA-2 7B and 13B, BART-large) and, for the drawn cases, generic ones.

A case is a dict of plain values:
  kind     norm | rope | loss | adamw
  M, N, K  tokens, columns (norm), head width (rope), vocabulary (loss), MLP width of a layer (adamw); K: model width
  back     norm: the backward pass; rope: the inverse; loss: with the gradient
  rms, bias, residual      norm: which, and the operands that are there
  heads, kv_heads, rot, interleaved, scaling, factor, far      rope: heads of the two tensors, rotated columns, the pairs' order,
                           how the frequencies are scaled, by what; the largest position
  r, layers, bits, clip, step      adamw: adapter rank, decoder layers stepped together, bits of the states, a device factor
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
BASE, ORIGINAL, LOW, HIGH = 10000.0, 4096, 1.0, 8.0
LR, BETAS, ADAM_EPS, DECAY = 2e-4, (0.9, 0.999), 1e-8, 0.01
GROUP = 64


def _norm(name, M, N, back=False, rms=False, bias=False, residual=False):
    return {"name": name, "kind": "norm", "M": M, "N": N, "back": back, "rms": rms, "bias": bias, "residual": residual}


def _rope(name, M, heads, kv_heads, N, rot, interleaved=False, back=False, scaling="none", factor=1.0, far=4096):
    return {"name": name, "kind": "rope", "M": M, "heads": heads, "kv_heads": kv_heads, "N": N, "rot": rot, "interleaved": interleaved,
            "back": back, "scaling": scaling, "factor": factor, "far": far}


def _loss(name, M, N, K, back=True):
    return {"name": name, "kind": "loss", "M": M, "N": N, "K": K, "back": back}


def _adamw(name, N, K, r, layers, bits, clip=False, step=100):
    return {"name": name, "kind": "adamw", "N": N, "K": K, "r": r, "layers": layers, "bits": bits, "clip": clip, "step": step}


def listed():
    return [
        # one decoded token of the 7B model: all latency
        _norm("norm_one_token", 1, 4096, rms=True),
        # training step of BART-large, a ragged batch: back through a layer norm behind a residual sum, with its weights' gradients
        _norm("norm_bart_back", 777, 1024, back=True, bias=True, residual=True),
        # training step of the 7B model, batch 8 x 512: back through the norm in front of a block, and the residual stream's gradient
        _norm("norm_7b_back", 4096, 4096, back=True, rms=True, residual=True),
        # four sequences decode a token each, at positions far beyond the trained context
        _rope("rope_tokens_far", 4, 32, 8, 128, 128, scaling="turns", factor=8.0, far=1 << 20),
        # part of each head, neighbours as pairs, an odd number of tokens
        _rope("rope_part_odd", 777, 16, 16, 80, 20, interleaved=True, scaling="linear", factor=2.0),
        # training step of the 7B model: the gradients of queries and keys turned back
        _rope("rope_7b_back", 4096, 32, 32, 128, 128, back=True),
        # a few labelled tokens over a small odd vocabulary
        _loss("loss_small_odd", 19, 1003, 512),
        # evaluation of a prompt with the 7B model: the loss alone
        _loss("loss_eval", 333, 32000, 4096, back=False),
        # training step of BART-large, ragged batch, a vocabulary of an odd size
        _loss("loss_bart", 777, 50265, 1024),
        # training step of the 7B model, batch 8 x 512
        _loss("loss_7b", 4096, 32000, 4096),
        # the adapters of one 7B layer at rank 16, states in 32 bits
        _adamw("adamw_layer", 11008, 4096, 16, 1, 32),
        # the adapters of a whole 7B model at rank 64, states in 8 bits, gradients clipped by a factor that is on the device
        _adamw("adamw_model_8", 11008, 4096, 64, 32, 8, clip=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


WIDTHS = [512, 1024, 2048, 4096, 5120, 8192]
MOST_LOSS = 4096 * 32000 * 4096


def draw(rng):
    kind = rng.choice(["norm", "norm", "rope", "loss", "loss", "adamw"])
    if kind == "norm":
        N = rng.choice(WIDTHS) if rng.random() < 0.5 else 8 * _log(rng, 8, 1376)
        rms, back = rng.random() < 0.5, rng.random() < 0.6
        c = _norm("", min(_log(rng, 1, 16384), (1 << 25) // N), N, back, rms, rng.random() < 0.5, back and rng.random() < 0.5)
    elif kind == "rope":
        N = rng.choice([64, 128, 256, 80, 96, 8 * rng.randint(2, 32)])
        heads = _log(rng, 1, 64)
        rot = N if rng.random() < 0.6 else 2 * rng.randint(2, N // 2)
        scaling = rng.choice(["none", "none", "linear", "base", "turns", "index"])
        c = _rope("", min(_log(rng, 1, 8192), (1 << 25) // (2 * heads * N)), heads, rng.choice([heads, max(1, heads // 4), 1]), N, rot, rng.random() < 0.4,
                  rng.random() < 0.4, scaling, 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]), _log(rng, 512, 1 << 20))
    elif kind == "loss":
        K = rng.choice(WIDTHS) if rng.random() < 0.5 else 8 * _log(rng, 32, 640)
        N = rng.choice([32000, 50265, 128256]) if rng.random() < 0.4 else _log(rng, 257, 130000)
        c = _loss("", max(1, min(_log(rng, 1, 8192), MOST_LOSS // (N * K))), N, K, rng.random() < 0.7)
    else:
        r = rng.choice([4, 8, 16, 32, 64, rng.randint(1, 64)])
        N, K = rng.choice([(2816, 1024), (5504, 2048), (11008, 4096)]) if rng.random() < 0.6 else (8 * _log(rng, 32, 1376), 8 * _log(rng, 32, 512))
        most = 32 * 64 * (9 * 4096 + 3 * 11008) // (r * (9 * K + 3 * N))
        c = _adamw("", N, K, r, _log(rng, 1, max(1, min(32, most))), rng.choice([8, 32]), rng.random() < 0.5, _log(rng, 1, 10000))
    del c["name"]
    return c


# ---- inputs: tensors on the GPU from the seed alone ---------------------------------------------------------------

def _layer_shapes(c):
    """Rows and columns of the adapters of a decoder layer's seven matrices: A [r, in], B [out, r] of each."""
    h, f, r = c["K"], c["N"], c["r"]
    out = []
    for o, i in [(h, h)] * 4 + [(f, h)] * 2 + [(h, f)]:
        out += [(r, i), (o, r)]
    return out


def _spans(c):
    """(first, count) of every adapter in the flat buffers, each at the start of a group of 64; and the buffers' length."""
    spans, at = [], 0
    for rows, cols in _layer_shapes(c) * c["layers"]:
        spans.append((at, rows * cols))
        at += -(-rows * cols // GROUP) * GROUP
    return spans, at


def _frequencies(c):
    """Radians a position for every pair, in 64 bits."""
    j, rot, how, s = torch.arange(c["rot"] // 2, dtype=torch.float64), c["rot"], c["scaling"], c["factor"]
    f = BASE ** (-2 * j / rot)
    if how == "linear":
        return f / s
    if how == "base":
        return (BASE * s ** (rot / (rot - 2))) ** (-2 * j / rot)
    if how == "turns":                                    # as it is where a pair turns HIGH times in the trained context, slowed below LOW
        keep = ((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
    elif how == "index":                                  # the same borders as places in the list of pairs, a ramp between them
        place = [rot * math.log(ORIGINAL / (2 * math.pi * t)) / (2 * math.log(BASE)) for t in (HIGH, LOW)]
        first, last = max(math.floor(place[0]), 0), min(math.ceil(place[1]), rot - 1)
        keep = 1 - ((j - first) / max(last - first, 1e-3)).clamp(0, 1)
    else:
        return f
    return f * (keep + (1 - keep) / s)


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)

    kind, m = c["kind"], {"case": c}
    if kind == "norm":
        M, N = c["M"], c["N"]
        m["x"] = (normal(M, N, dtype=torch.float32) * (1 + 4 * (torch.rand(N, generator=g, device="cuda") < 0.01)) + 0.25).bfloat16()   # a few loud columns
        m["weight"] = (1 + normal(N, std=0.2, dtype=torch.float32)).bfloat16()
        if c["bias"]:
            m["bias"] = normal(N, std=0.1)
        if c["back"]:
            m["dY"] = normal(M, N, std=1e-3)
            if c["residual"]:
                m["residual"] = normal(M, N, std=1e-3)
    elif kind == "rope":                                  # queries and keys as a projection of all three left them
        M, D, h, kv = c["M"], c["N"], c["heads"], c["kv_heads"]
        qkv = normal(M, (h + 2 * kv) * D)
        m["q"], m["k"] = qkv[:, :h * D].view(M, h, D), qkv[:, h * D:(h + kv) * D].view(M, kv, D)
        m["positions"] = torch.randint(0, c["far"], (M,), generator=g, device="cuda", dtype=torch.int32)
        m["frequencies"] = _frequencies(c).cuda()
    elif kind == "loss":
        M, V, K = c["M"], c["N"], c["K"]
        m["W"] = normal(V, K, std=0.02)
        t = torch.randint(0, V, (M,), generator=g, device="cuda")
        known = 16 * torch.rand(M, 1, generator=g, device="cuda") / (0.02 ** 2 * K)      # how far the model knows the token: logits up to 16
        m["h"] = (normal(M, K, dtype=torch.float32) + known * m["W"][t].float()).bfloat16()
        there = torch.rand(M, generator=g, device="cuda") < 0.9                          # the others are padding
        there[0] = True
        m["targets"] = torch.where(there, t, -100).int()
        m["weights"] = (there / there.sum()).float()
    else:
        spans, total = _spans(c)
        there = torch.zeros(total, dtype=torch.bool, device="cuda")
        for first, count in spans:
            there[first:first + count] = True
        t = c["step"]
        loud = torch.exp(2 * torch.randn(total, generator=g, device="cuda"))             # gradients of very different sizes
        m["grad"] = normal(total, std=1e-3, dtype=torch.float32) * loud * there
        m["m"] = normal(total, std=3e-4 if t > 1 else 0.0, dtype=torch.float32) * loud * there
        m["v"] = (1e-3 * loud).square() * (1 - BETAS[1] ** (t - 1)) * (0.5 + torch.rand(total, generator=g, device="cuda")) * there
        m["weight"] = normal(total, std=0.02, dtype=torch.float32) * there
        if c["clip"]:
            m["clip"] = torch.rand(1, generator=g, device="cuda") * 0.5 + 0.5
        if c["bits"] == 8:
            for n in "mv":
                m[n], m[n + "_absmax"] = _coded(m[n], n == "m")
    return m


def prepare(c, seed):
    m = _inputs(c, seed)
    kind = c["kind"]
    if kind == "adamw":                                   # the step is written beside what it reads, so that a pass can be repeated
        for n in ("m", "v", "weight") + (("m_absmax", "v_absmax") if c["bits"] == 8 else ()):
            m[n + "_out"] = torch.zeros_like(m[n])
        m["weight_bf16"] = torch.zeros_like(m["weight"], dtype=torch.bfloat16)
    if own:                                               # the handles, plans and workspaces that a program keeps
        from paper_2502_08141_amd import lowra

        if kind == "norm" and c["back"]:
            m["workspace"] = torch.empty(lowra.lowra_norm_bwd_workspace_bytes(c["M"], c["N"]), dtype=torch.uint8, device="cuda")
        elif kind == "rope":
            m["plan"] = lowra.lowra_rope_frequencies(c["rot"], BASE, lowra.ROPE_SCALINGS[c["scaling"]], c["factor"], ORIGINAL, LOW, HIGH)
        elif kind == "loss":
            m["workspace"] = torch.empty(lowra.lowra_vocab_loss_workspace_bytes(c["M"], c["N"], c["K"], c["back"]), dtype=torch.uint8, device="cuda")
        elif kind == "adamw":
            items = []
            for first, count in _spans(c)[0]:
                part = lambda n: m[n][first:first + count]
                groups = lambda n: m[n][first // GROUP:first // GROUP + -(-count // GROUP)]
                more = {n: groups(n) for n in ("m_absmax", "v_absmax", "m_absmax_out", "v_absmax_out")} if c["bits"] == 8 else {}
                items.append(lowra.AdamWItem(**{n: part(n) for n in ("grad", "m", "v", "weight", "m_out", "v_out", "weight_out", "weight_bf16")}, **more))
            m["batch"] = lowra.AdamWBatch(items)
    return m


# ---- the plain forms: elementary operations in 32 bits ------------------------------------------------------------

def _values(q, absmax, signed):
    """What 8-bit states stand for."""
    u = q.float() * (1 / 127 if signed else 1 / 255)
    u = u * u.abs() if signed else (u * u) * (u * u)
    return (u.view(-1, GROUP) * absmax[:, None]).view(-1)


def _coded(x, signed):
    """8-bit codes and the groups' largest magnitudes; next to a border in 64 bits."""
    absmax = x.abs().view(-1, GROUP).amax(1)
    most, power = (127.0, 2) if signed else (255.0, 4)
    A, a = absmax.double()[:, None], x.abs().double().view(-1, GROUP)
    full = a * most ** power
    q = torch.floor(most * (a / A.clamp(min=1e-300)) ** (1 / power) + 0.5).clamp(0, most)      # within one of the count
    border = lambda k: (k * k if signed else (k * k) * (k * k)) * A
    q = torch.where((q > 0) & (full <= border(q - 0.5)), q - 1, q)
    q = torch.where((q < most) & (full > border(q + 0.5)), q + 1, q)
    if signed:
        return (q.view(-1) * x.sign()).to(torch.int8), absmax
    return torch.where(a > 0, q.clamp(min=1), q).view(-1).to(torch.uint8), absmax


def _plain_norm(m):
    c, x, w = m["case"], m["x"].float(), m["weight"].float()
    d = x if c["rms"] else x - x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(d.square().mean(1, keepdim=True) + EPS)
    xh = d * rstd
    if not c["back"]:
        return {"y": (xh * w + m["bias"].float() if c["bias"] else xh * w).bfloat16()}
    dY = m["dY"].float()
    g = dY * w
    dX = g - xh * (g * xh).mean(1, keepdim=True)
    dX = rstd * (dX if c["rms"] else dX - g.mean(1, keepdim=True))
    dX = dX + m["residual"].float() if c["residual"] else dX
    return {"dX": dX.bfloat16(), "dweight": (dY * xh).sum(0)} | ({"dbias": dY.sum(0)} if c["bias"] else {})


def _turned(x, cos, sin, c):
    n = c["rot"]
    x, y = x.float(), x.float().clone()
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if c["interleaved"] else (x[..., :n // 2], x[..., n // 2:n])
    first, second = (slice(0, n, 2), slice(1, n, 2)) if c["interleaved"] else (slice(0, n // 2), slice(n // 2, n))
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    return y.bfloat16()


def _plain_rope(m):
    c = m["case"]
    angle = m["positions"].double()[:, None] * m["frequencies"][None]                    # a far position's angle needs 64 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(-angle if c["back"] else angle).float()[:, None]
    return {"q": _turned(m["q"], cos, sin, c), "k": _turned(m["k"], cos, sin, c)}


def _plain_loss(m):
    c, t = m["case"], m["targets"].long()
    W = m["W"].float()
    z = m["h"].float() @ W.T
    there, at = (t >= 0)[:, None], t.clamp(min=0)[:, None]
    zt = z.gather(1, at)
    most = z.amax(1, keepdim=True)
    lse = most + torch.log(torch.exp(z - most).sum(1, keepdim=True))
    out = {"loss": torch.where(there, lse - zt, 0.0)[:, 0], "lse": lse[:, 0]}
    if c["back"]:
        p = torch.exp(z - lse)
        p.scatter_add_(1, at, torch.full_like(zt, -1.0))
        out["dH"] = torch.where(there, (m["weights"][:, None] * p) @ W, 0.0).bfloat16()
    return out


def _plain_adamw(m):
    c, (b1, b2), t = m["case"], BETAS, m["case"]["step"]
    eight = c["bits"] == 8
    m0, v0 = (_values(m[n], m[n + "_absmax"], n == "m") if eight else m[n] for n in "mv")
    g, w = m["grad"] * m["clip"] if c["clip"] else m["grad"], m["weight"]
    m1, v1 = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * (g * g)
    w1 = w - LR * ((m1 / (1 - b1 ** t)) / (torch.sqrt(v1 / (1 - b2 ** t)) + ADAM_EPS) + DECAY * w)
    m["weight_out"].copy_(w1)
    m["weight_bf16"].copy_(w1)
    if eight:                                             # the states are kept in 8 bits and given as what they stand for
        for n, s in (("m", m1), ("v", v1)):
            q, a = _coded(s, n == "m")
            m[n + "_out"].copy_(q)
            m[n + "_absmax_out"].copy_(a)
        m1, v1 = (_values(m[n + "_out"], m[n + "_absmax_out"], n == "m") for n in "mv")
    else:
        m["m_out"].copy_(m1)
        m["v_out"].copy_(v1)
    return {"m": m1, "v": v1, "weight": m["weight_out"], "weight_bf16": m["weight_bf16"]}


def run(m):
    c = m["case"]
    kind = c["kind"]
    if not own:
        return {"norm": _plain_norm, "rope": _plain_rope, "loss": _plain_loss, "adamw": _plain_adamw}[kind](m)
    from paper_2502_08141_amd import lowra

    if kind == "norm":
        norm = lowra.NORM_RMS if c["rms"] else lowra.NORM_LAYER
        if not c["back"]:
            return {"y": lowra.lowra_norm_fwd(m["x"], m["weight"], m.get("bias"), norm, EPS)}
        dX, dw, db = lowra.lowra_norm_bwd(m["dY"], m["x"], m["weight"], norm, EPS, residual=m.get("residual"), weight_grad=True, bias_grad=c["bias"],
                                          workspace=m["workspace"])
        return {"dX": dX, "dweight": dw} | ({"dbias": db} if c["bias"] else {})
    if kind == "rope":
        q, k = lowra.lowra_rope([m["q"], m["k"]], m["positions"], m["plan"], lowra.ROPE_INTERLEAVED if c["interleaved"] else lowra.ROPE_HALF, inverse=c["back"])
        return {"q": q, "k": k}
    if kind == "loss":
        loss, lse, dH = lowra.lowra_vocab_loss(m["h"], m["W"], m["targets"], m["weights"] if c["back"] else None, grad=c["back"], workspace=m["workspace"])
        return {"loss": loss, "lse": lse} | ({"dH": dH} if c["back"] else {})
    m["batch"].run(lr=LR, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, step=c["step"], grad_scale=m.get("clip"))
    m1, v1 = m["m_out"], m["v_out"]
    if c["bits"] == 8:                                    # the states are given as what they stand for
        m1, v1 = lowra.lowra_adamw_state(m1, m["m_absmax_out"]), lowra.lowra_adamw_state(v1, m["v_absmax_out"])
    return {"m": m1, "v": v1, "weight": m["weight_out"], "weight_bf16": m["weight_bf16"]}


def work(c):
    kind = c["kind"]
    if kind == "norm":
        M, N = c["M"], c["N"]
        if not c["back"]:
            return {"bytes": 4 * M * N + 2 * N * (1 + c["bias"]), "flops": 6 * M * N}
        return {"bytes": 2 * M * N * (3 + c["residual"]) + 2 * N + 4 * N * (1 + c["bias"]), "flops": 14 * M * N}
    if kind == "rope":
        size = c["M"] * (c["heads"] + c["kv_heads"]) * c["N"]
        return {"bytes": 4 * size + 4 * c["M"] + 4 * c["rot"], "flops": 3 * size}
    if kind == "loss":
        M, V, K = c["M"], c["N"], c["K"]
        return {"bytes": 2 * V * K + 2 * M * K * (1 + c["back"]) + (12 + 4 * c["back"]) * M, "flops": 2 * M * V * K * (1 + c["back"])}
    count = sum(n for _, n in _spans(c)[0])
    # gradient and weight in, weight and its bf16 copy out, the states in and out; in 8 bits also as what they stand for
    state = 16 if c["bits"] == 32 else 4 * (1 + 4 / GROUP) + 8
    return {"bytes": int(count * (14 + state)), "flops": 16 * count}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_norm(c, m):
    x, w = m["x"].double().requires_grad_(), m["weight"].double().requires_grad_()
    b = (m["bias"].double() if c["bias"] else torch.zeros_like(w.detach())).requires_grad_()
    if c["rms"]:
        y = x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + EPS) * w + b
    else:
        y = torch.nn.functional.layer_norm(x, (c["N"],), w, b, EPS)
    if not c["back"]:
        return {"y": y.detach()}
    dX, dw, db = torch.autograd.grad(y, [x, w, b], m["dY"].double())
    dX = dX + m["residual"].double() if c["residual"] else dX
    return {"dX": dX, "dweight": dw} | ({"dbias": db} if c["bias"] else {})


def _exact_rope(c, m):
    rot, s, out = c["rot"], c["factor"], {}
    base = BASE * s ** (rot / (rot - 2)) if c["scaling"] == "base" else BASE
    pairs = []
    for j in range(rot // 2):
        f = math.exp(-2 * j / rot * math.log(base))
        if c["scaling"] == "linear":
            f /= s
        elif c["scaling"] == "turns":
            turns = ORIGINAL * f / math.tau
            part = 1.0 if turns >= HIGH else 0.0 if turns <= LOW else (turns - LOW) / (HIGH - LOW)
            f = f * part + f / s * (1 - part)
        elif c["scaling"] == "index":
            at = lambda turns: rot / 2 * math.log(ORIGINAL / (math.tau * turns), base)
            first, last = max(math.floor(at(HIGH)), 0), min(math.ceil(at(LOW)), rot - 1)
            part = 0.0 if j <= first else 1.0 if j >= last else (j - first) / (last - first)
            f = f * (1 - part) + f / s * part
        pairs.append(f)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       m["positions"].double()[:, None] * torch.tensor(pairs, dtype=torch.float64, device="cuda") * (-1 if c["back"] else 1))[:, None]
    for n in "qk":
        x = m[n].double().clone()
        M, heads, _ = x.shape
        part = x[..., :rot]
        part = part.reshape(M, heads, rot // 2, 2) if c["interleaved"] else part.reshape(M, heads, 2, rot // 2).transpose(2, 3)
        part = torch.view_as_real(torch.complex(part[..., 0], part[..., 1]) * turn)
        x[..., :rot] = (part if c["interleaved"] else part.transpose(2, 3)).reshape(M, heads, rot)
        out[n] = x
    return out


def _exact_loss(c, m):
    h, W, t = m["h"].double(), m["W"].double(), m["targets"].long()
    if c["M"] * c["N"] * 8 > 8 << 30:
        return None
    logp = torch.log_softmax(h @ W.T, 1)
    there = t >= 0
    rows = torch.nonzero(there)[:, 0]
    loss = torch.zeros(c["M"], dtype=torch.float64, device="cuda")
    loss[rows] = -logp[rows, t[rows]]
    out = {"loss": loss, "lse": h @ W[0] - logp[:, 0]}
    if c["back"]:
        p = logp.exp_()
        p[rows, t[rows]] = torch.expm1(-loss[rows])
        out["dH"] = (p * (m["weights"].double() * there)[:, None]) @ W
    return out


def _exact_values(q, absmax, signed):
    u = q.double().view(-1, GROUP) / (127 if signed else 255)
    return ((u * u.abs() if signed else u ** 4) * absmax.double()[:, None]).view(-1)


def _exact_coded(x, signed):
    """The value that is left of a state in 8 bits: on the scale of the codes, halves go down."""
    most, power = (127, 2) if signed else (255, 4)
    A = x.abs().view(-1, GROUP).amax(1, keepdim=True)
    u = most * (x.abs().view(-1, GROUP) / torch.where(A > 0, A, 1.0)).pow(1 / power)
    q = torch.ceil(u - 0.5)
    q = q if signed else torch.where((u > 0) & (q < 1), 1.0, q)
    return (x.sign().view(-1, GROUP) * (q / most) ** power * A).view(-1)


def _exact_adamw(c, m):
    (b1, b2), t, eight = BETAS, c["step"], c["bits"] == 8
    m0, v0 = (_exact_values(m[n], m[n + "_absmax"], n == "m") if eight else m[n].double() for n in "mv")
    g, w = m["grad"].double() * (m["clip"].double() if c["clip"] else 1.0), m["weight"].double()
    m1, v1 = torch.lerp(g, m0, b1), torch.lerp(g.square(), v0, b2)
    w1 = w * (1 - LR * DECAY) - LR / (1 - b1 ** t) * m1 / ((v1 / (1 - b2 ** t)).sqrt() + ADAM_EPS)
    if eight:
        m1, v1 = _exact_coded(m1, True), _exact_coded(v1, False)
    return {"m": m1, "v": v1, "weight": w1, "weight_bf16": w1}


def exact(c, seed):
    m = _inputs(c, seed)
    return {"norm": _exact_norm, "rope": _exact_rope, "loss": _exact_loss, "adamw": _exact_adamw}[c["kind"]](c, m)
