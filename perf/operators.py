"""Operators around the quantized LoRA linear, as measurable cases: the linear with bias, activation, gate and residual in
its epilogue, forward and input gradient; the activation's backward pass with the bias gradient; and the optimiser step
on the adapters whose update is orthogonalised by Newton-Schulz products.

`run` computes a case in elementary torch operations where `own` is false, and by the library's calls where it is true.

  forward         v = x What^T + s (x A^T) B^T + bias      y = act(v) mul + residual      z = v, kept for the backward pass
  input gradient  g = dY What + s (dY B) A + residual      dX = g mul act'(z)             dmul = g act(z)
  activation      dZ = dY mul act'(z)                      dmul = dY act(z)               db = sum of dZ over the tokens
  update          m' = beta m + g    u = g + beta m' (Nesterov) or m'    X = u / (|u| + eps), then five times
                  X = a X + (b X X^T + c (X X^T)^2) X      w' = w - lr (scale X + decay w)

Shapes are those of the linear layers the repository names (256 x 512 of its smallest test, BART-large, LLaMA-2 7B and
13B) and, for the drawn cases, generic ones between them.

A case is a dict of plain values:
  kind    fwd | bwd | act | update
  N, K    output channels and input features (act: N columns; update: model width `K` and MLP width `N` of a layer)
  M, r    tokens and adapter rank
  act     none | relu | gelu | gelu_tanh | silu
  bias, mul, residual, z    truth values: the operand is there (z: is kept; act with bias: the bias gradient is asked for)
  mix, tables, scales       the quantized matrix: percent of 1-, 2- and 4-bit channels; one table per width ("shared") or
                            per channel ("channel"); group scales "fp32" or "bf16"
  layers, nesterov          update: decoder layers whose adapters are stepped together
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

GROUP = 64
SCALE = 2.0
WIDTHS = (1, 2, 4)
BETA, LR, DECAY, EPS = 0.95, 0.02, 0.1, 1e-7
COEFFICIENTS, STEPS = (3.4445, -4.7750, 2.0315), 5


def _case(name, kind, N, K, M=0, r=0, act="none", bias=False, mul=False, residual=False, z=False, mix="50/25/25", tables="shared",
          scales="fp32", layers=0, nesterov=False):
    return {"name": name, "kind": kind, "N": N, "K": K, "M": M, "r": r, "act": act, "bias": bias, "mul": mul, "residual": residual,
            "z": z, "mix": mix, "tables": tables, "scales": scales, "layers": layers, "nesterov": nesterov}


def listed():
    return [
        # the smallest layer there is, sixteen tokens: all latency
        _case("fwd_tiny", "fwd", 256, 512, 16, 8, "gelu", bias=True, mix="25/50/25"),
        # one decoded token through the 7B gate projection: silu(gate) times the up projection's output
        _case("fwd_one_token", "fwd", 11008, 4096, 1, 16, "silu", mul=True),
        # prefill of an odd number of tokens through the 7B down projection, added to the residual stream
        _case("fwd_prefill_odd", "fwd", 4096, 11008, 333, 16, "none", residual=True),
        # training step of BART-large's first feed-forward layer, ragged batch, one table per channel
        _case("fwd_bart", "fwd", 4096, 1024, 777, 64, "gelu", bias=True, z=True, mix="50/50/0", tables="channel"),
        # training step of the 7B gate projection, batch 8 x 512, 1.5 bits
        _case("fwd_gate", "fwd", 11008, 4096, 4096, 64, "silu", mul=True, z=True, mix="50/50/0"),
        # the gradient of a few tokens through an attention projection, added to the residual stream's
        _case("bwd_few_tokens", "bwd", 4096, 4096, 4, 16, "none", residual=True),
        # back through BART-large's second feed-forward layer into the activation of the first
        _case("bwd_bart", "bwd", 1024, 4096, 777, 64, "gelu", mix="50/50/0"),
        # back through the 7B down projection into the gated activation, batch 8 x 512
        _case("bwd_down", "bwd", 4096, 11008, 4096, 64, "silu", mul=True, mix="50/50/0"),
        # a gradient that comes from outside: through a GELU, with the gradient of BART-large's bias
        _case("act_bart", "act", 4096, 0, 777, 0, "gelu", bias=True),
        # the bias gradient by itself, wide and long
        _case("act_bias", "act", 11008, 0, 4096, 0, "none", bias=True),
        # the adapters of one 7B decoder layer, rank 64
        _case("update_layer", "update", 11008, 4096, 0, 64, layers=1, nesterov=True),
        # the adapters of a whole 7B model, rank 16
        _case("update_model", "update", 11008, 4096, 0, 16, layers=32, nesterov=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


SHAPES = [(1024, 1024), (4096, 1024), (1024, 4096), (4096, 4096), (11008, 4096), (4096, 11008), (5120, 5120)]
MIXES = ["25/50/25", "50/25/25", "34/33/33", "50/50/0", "85/15/0"]
LAYERS = [(2816, 1024), (5504, 2048), (11008, 4096)]
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "fwd", "bwd", "bwd", "act", "update"])
    if kind == "update":
        N, K = rng.choice(LAYERS) if rng.random() < 0.6 else (8 * _log(rng, 32, 1376), GROUP * _log(rng, 8, 64))
        r = rng.choice([4, 8, 16, 32, 64, rng.randint(1, 64)])
        most = 32 * 16 * (9 * 4096 + 3 * 11008) // (r * (9 * K + 3 * N))
        c = _case("", kind, N, K, 0, r, layers=_log(rng, 1, max(1, min(32, most))), nesterov=rng.random() < 0.5)
    elif kind == "act":
        act, M = rng.choice(ACTS), _log(rng, 1, 4096)
        c = _case("", kind, 8 * _log(rng, 32, 1376), 0, M, 0, act, bias=act == "none" or rng.random() < 0.7,
                  mul=act != "none" and rng.random() < 0.4)
    else:
        N, K = rng.choice(SHAPES) if rng.random() < 0.6 else (8 * _log(rng, 32, 1376), GROUP * _log(rng, 8, 172))
        M = min(_log(rng, 1, 4096), 4096 * 11008 * 4096 // (N * K))
        if rng.random() < 0.3:
            M = rng.randint(1, 16)
        act = rng.choice(ACTS)
        c = _case("", kind, N, K, M, rng.choice([0, 8, 16, 32, 64, rng.randint(1, 64)]), act,
                  bias=kind == "fwd" and rng.random() < 0.5, mul=rng.random() < 0.4, residual=rng.random() < 0.4,
                  z=kind == "fwd" and rng.random() < 0.4, mix=rng.choice(MIXES), tables="channel" if rng.random() < 0.25 else "shared",
                  scales="bf16" if rng.random() < 0.2 else "fp32")
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


def _levels(b):
    """2^b levels for normal weights that are scaled by the largest of 64 (which is 2.4 deviations on average)."""
    q = (torch.arange(1 << b, dtype=torch.float64) + 0.5) / (1 << b)
    return (torch.special.ndtri(q) * (1.25 if b == 1 else 1.15) / 2.4).float()


def _quantized(c, normal, g, seed):
    """The state of a quantized matrix: random codes (the frozen base is whatever it is), scales, tables, widths."""
    N, K = c["N"], c["K"]
    f1, f2, _ = (int(v) / 100 for v in c["mix"].split("/"))
    rng = np.random.default_rng([seed, 1])
    bits = np.full(N, 4, np.uint8)
    perm, n1, n2 = rng.permutation(N), round(f1 * N), round((f1 + f2) * N)
    bits[perm[:n1]], bits[perm[n1:n2]] = 1, 2
    cb, widths = (np.arange(N, dtype=np.int32), bits) if c["tables"] == "channel" else \
        (np.searchsorted(WIDTHS, bits).astype(np.int32), np.array(WIDTHS, np.uint8))
    mappings = torch.zeros(widths.size, 16)
    for b in WIDTHS:
        at = np.nonzero(widths == b)[0]
        if at.size:
            mappings[at, :1 << b] = _levels(b) * torch.from_numpy(1 + 0.05 * rng.standard_normal((at.size, 1))).float()
    m = {"bits": bits, "cb": cb, "widths": widths, "mappings": mappings.cuda()}
    m["packed"] = torch.randint(0, 256, (int(bits.astype(np.int64).sum()) * K // 8,), generator=g, device="cuda", dtype=torch.uint8)
    absmax = normal(N, K // GROUP, std=0.3, dtype=torch.float32).add_(2.4).clamp_(1.2).mul_(0.02)
    m["absmax"] = absmax.bfloat16() if c["scales"] == "bf16" else absmax
    return m


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)

    kind, M, N, K, r = c["kind"], c["M"], c["N"], c["K"], c["r"]
    m = {"case": c}
    if kind == "update":                                  # gradients of a few tokens: a falling spectrum, and their momentum
        sizes = [a * b for a, b in _layer_shapes(c)] * c["layers"]
        total = sum(sizes)
        m["grad"], m["momentum"] = normal(total, std=1e-3, dtype=torch.float32), normal(total, std=4e-3, dtype=torch.float32)
        m["weight"] = normal(total, std=0.02, dtype=torch.float32)
        at, fall = 0, 0.02 ** (torch.arange(r, device="cuda", dtype=torch.float32) / r)
        shapes = _layer_shapes(c)
        for _ in range(c["layers"]):
            for rows, cols in shapes:
                scale = fall[:, None] if rows == r and cols != r else fall
                for t in ("grad", "momentum"):
                    m[t][at:at + rows * cols].view(rows, cols).mul_(scale)
                at += rows * cols
        return m
    if kind == "act":
        m["dY"] = normal(M, N)
        cols = N
    else:
        m |= _quantized(c, normal, g, seed)
        if r:
            m["A"], m["B"] = normal(r, K, std=0.01), normal(N, r, std=0.01)
        cols = N if kind == "fwd" else K
        m["x" if kind == "fwd" else "dY"] = normal(M, K if kind == "fwd" else N)
    if c["bias"] and kind == "fwd":
        m["bias"] = normal(N, std=0.5)
    if c["mul"]:
        m["mul"] = normal(M, cols)
    if c["residual"]:
        m["residual"] = normal(M, cols)
    if kind != "fwd" and c["act"] != "none" or (kind == "bwd" and c["mul"]):
        m["z"] = normal(M, cols, std=1.5)
    return m


def prepare(c, seed):
    m = _inputs(c, seed)
    kind = c["kind"]
    if kind == "update":                                  # the step is written beside what it reads, so that a pass can be repeated
        m["momentum_out"], m["weight_out"] = torch.empty_like(m["momentum"]), torch.empty_like(m["weight"])
        m["weight_bf16"] = torch.empty_like(m["weight"], dtype=torch.bfloat16)
    if own:                                               # the handles and workspaces that a program keeps
        from paper_2502_08141_amd import lowra

        if kind in ("fwd", "bwd"):
            m["layout"] = lowra.Layout(c["K"], m["bits"], m["cb"], m["widths"])
            if c["scales"] == "bf16":
                m["layout"].set_scale_dtype(torch.bfloat16)
            op = lowra.OP_LINEAR_FWD if kind == "fwd" else lowra.OP_LINEAR_BWD_INPUT
            m["workspace"] = torch.empty(m["layout"].workspace_bytes(op, c["M"], c["r"]), dtype=torch.uint8, device="cuda")
        elif kind == "act":
            m["workspace"] = torch.empty(lowra.lowra_act_bwd_workspace_bytes(c["M"], c["N"]), dtype=torch.uint8, device="cuda")
        else:
            items, at = [], 0
            for rows, cols in _layer_shapes(c) * c["layers"]:
                v = {t: m[t][at:at + rows * cols].view(rows, cols)
                     for t in ("grad", "momentum", "weight", "momentum_out", "weight_out", "weight_bf16")}
                items.append(lowra.MuonItem(scale=_update_scale(rows, cols), **v))
                at += rows * cols
            m["batch"] = lowra.MuonBatch(items)
    return m


def _update_scale(rows, cols):
    return math.sqrt(max(1.0, rows / cols))


# ---- the plain forms: elementary operations in 32 bits ------------------------------------------------------------

def _decoded(m):
    """What [N, K]: a row's codes, low bits first, through its table, times its groups' scales."""
    c, bits = m["case"], torch.from_numpy(m["bits"].astype(np.int64)).cuda()
    K, cb = c["K"], torch.from_numpy(m["cb"].astype(np.int64)).cuda()
    first = torch.cumsum(bits * (K // 8), 0) - bits * (K // 8)
    W = torch.empty(c["N"], K, device="cuda")
    for b in WIDTHS:
        rows = torch.nonzero(bits == b)[:, 0]
        if not rows.numel():
            continue
        bytes_ = m["packed"][first[rows, None] + torch.arange(K * b // 8, device="cuda")]
        codes = (bytes_[:, :, None] >> torch.arange(0, 8, b, device="cuda", dtype=torch.uint8)) & ((1 << b) - 1)
        level = torch.gather(m["mappings"][cb[rows]], 1, codes.view(rows.numel(), K).long())
        W[rows] = (level.view(rows.numel(), K // GROUP, GROUP) * m["absmax"][rows].float()[:, :, None]).view(rows.numel(), K)
    return W


def _act(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "gelu":
        return 0.5 * v * torch.erfc(-v * math.sqrt(0.5))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v


def _act_slope(v, act):
    if act == "relu":
        return (v > 0).float()
    if act == "gelu":
        return 0.5 * torch.erfc(-v * math.sqrt(0.5)) + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
        return 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)
    if act == "silu":
        s = 1 / (1 + torch.exp(-v))
        return s * (1 + v * (1 - s))
    return torch.ones_like(v)


def _float(m, name):
    return m[name].float() if name in m else None


def _back(g, m, bias):
    """A gradient through y = act(z) mul: {dZ | dX, dmul, db} as asked for."""
    act, mul, z, out = m["case"]["act"], _float(m, "mul"), _float(m, "z"), {}
    if mul is not None:
        out["dmul"] = (g * _act(z, act)).bfloat16()
        g = g * mul
    if act != "none":
        g = g * _act_slope(z, act)
    if bias:
        out["db"] = g.sum(0)
    return g, out


def _orthogonalised(u):
    """Newton-Schulz products of every matrix of a stack, u / |u|, with the short side's Gram matrix."""
    a, b, c = COEFFICIENTS
    X = u / (u.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = X.shape[1] > X.shape[2]
    X = X.transpose(1, 2).contiguous() if tall else X
    for _ in range(STEPS):
        G = X @ X.transpose(1, 2).contiguous()
        X = a * X + (b * G + c * (G @ G)) @ X
    return X.transpose(1, 2) if tall else X


def _plain(m):
    c = m["case"]
    if c["kind"] == "update":
        m["momentum_out"].copy_(BETA * m["momentum"] + m["grad"])
        u, at = m["grad"] + BETA * m["momentum_out"] if c["nesterov"] else m["momentum_out"], 0
        u, w, new = (t.view(c["layers"], -1) for t in (u, m["weight"], m["weight_out"]))
        for rows, cols in _layer_shapes(c):               # the same factor of all layers at a time
            here = slice(at, at + rows * cols)
            X = _orthogonalised(u[:, here].reshape(-1, rows, cols)).reshape(-1, rows * cols)
            new[:, here] = w[:, here] - LR * (_update_scale(rows, cols) * X + DECAY * w[:, here])
            at += rows * cols
        m["weight_bf16"].copy_(m["weight_out"])
        return {"momentum": m["momentum_out"], "weight": m["weight_out"], "weight_bf16": m["weight_bf16"]}
    if c["kind"] == "act":
        g, out = _back(m["dY"].float(), m, c["bias"])
        return out | ({"dZ": g.bfloat16()} if c["act"] != "none" or c["mul"] else {})
    W, A, B = _decoded(m), _float(m, "A"), _float(m, "B")
    if c["kind"] == "bwd":
        g = m["dY"].float() @ W
        if A is not None:
            g = g + SCALE * ((m["dY"].float() @ B) @ A)
        if "residual" in m:
            g = g + m["residual"].float()
        g, out = _back(g, m, False)
        return out | {"dX": g.bfloat16()}
    x = m["x"].float()
    v = x @ W.T
    if A is not None:
        v = v + SCALE * ((x @ A.T) @ B.T)
    if "bias" in m:
        v = v + m["bias"].float()
    y = _act(v, c["act"])
    if "mul" in m:
        y = y * m["mul"].float()
    if "residual" in m:
        y = y + m["residual"].float()
    return {"y": y.bfloat16()} | ({"z": v.bfloat16()} if c["z"] else {})


def run(m):
    if not own:
        return _plain(m)
    from paper_2502_08141_amd import lowra

    c = m["case"]
    if c["kind"] == "update":
        m["batch"].run(lr=LR, momentum=BETA, nesterov=c["nesterov"], weight_decay=DECAY, steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)
        return {"momentum": m["momentum_out"], "weight": m["weight_out"], "weight_bf16": m["weight_bf16"]}
    act, get = lowra.ACTS[c["act"]], m.get
    if c["kind"] == "act":
        dZ, dmul, db = lowra.lowra_act_bwd(m["dY"], act, z=get("z"), mul=get("mul"), bias_grad=c["bias"], workspace=m["workspace"])
        return {n: t for n, t in (("dZ", dZ), ("dmul", dmul), ("db", db)) if t is not None}
    state = (m["layout"], m["packed"], m["absmax"], m["mappings"])
    if c["kind"] == "bwd":
        dX, dmul = lowra.lowra_linear_bwd_input_act(*state, m["dY"], get("A"), get("B"), SCALE, act, z=get("z"), mul=get("mul"),
                                                    residual=get("residual"), workspace=m["workspace"])
        return {n: t for n, t in (("dX", dX), ("dmul", dmul)) if t is not None}
    y, z = lowra.lowra_linear_fwd_act(*state, m["x"], get("A"), get("B"), SCALE, act, bias=get("bias"), mul=get("mul"),
                                      residual=get("residual"), keep_z=c["z"], workspace=m["workspace"])
    return {n: t for n, t in (("y", y), ("z", z)) if t is not None}


def work(c):
    M, N, K, r = c["M"], c["N"], c["K"], c["r"]
    if c["kind"] == "update":
        count = c["layers"] * sum(a * b for a, b in _layer_shapes(c))
        # gradient, momentum and weight read; momentum, weight and its bf16 copy written; the Gram matrix and its polynomial's product
        return {"bytes": 22 * count, "flops": 3 * r * count + 14 * c["layers"] * (4 * STEPS - 2) * 2 * r ** 3}
    cols = N if c["kind"] != "bwd" else K
    slots = c["mul"] + c["residual"] + c["z"]
    if c["kind"] == "act":
        through = c["act"] != "none" or c["mul"]
        return {"bytes": 2 * M * N * (1 + 2 * through + 2 * c["mul"]) + 4 * N * c["bias"], "flops": 0}
    if c["kind"] == "bwd":
        slots += c["mul"] + (c["act"] != "none" or c["mul"])          # dmul out, z in
    f1, f2, f4 = (int(v) / 100 for v in c["mix"].split("/"))
    code = (f1 + 2 * f2 + 4 * f4) / 8 + (2 if c["scales"] == "bf16" else 4) / GROUP
    return {"bytes": N * K * code + 2 * (M * (K + N) + r * (K + N) + M * cols * slots + N * c["bias"]),
            "flops": 2 * M * N * K + 2 * M * r * (N + K)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _weights64(m):
    """What from its bits: bit i of a row's stream is bit i % 8 of byte i / 8; a code is its bits, lowest first."""
    c = m["case"]
    stream = (m["packed"][:, None] >> torch.arange(8, device="cuda", dtype=torch.uint8)).bitwise_and_(1).view(-1, c["K"])
    a = m["absmax"].double().repeat_interleave(GROUP, dim=1)
    first = np.concatenate([[0], np.cumsum(m["bits"].astype(np.int64))])[:-1]      # in pieces of K bits
    W = torch.empty(c["N"], c["K"], device="cuda", dtype=torch.float64)
    for b in WIDTHS:
        rows = np.nonzero(m["bits"] == b)[0]
        if rows.size:
            own_bits = stream[torch.from_numpy((first[rows][:, None] + np.arange(b)).ravel()).cuda()].view(rows.size, c["K"], b)
            code = (own_bits.int() << torch.arange(b, device="cuda", dtype=torch.int32)).sum(2)
            at = torch.from_numpy(rows).cuda()
            tables = m["mappings"].double()[torch.from_numpy(m["cb"][rows].astype(np.int64)).cuda()]
            W[at] = torch.gather(tables, 1, code.long()) * a[at]
    return W


def _act64(v, act):
    f = torch.nn.functional
    return {"none": lambda t: t, "relu": f.relu, "gelu": f.gelu, "gelu_tanh": lambda t: f.gelu(t, approximate="tanh"), "silu": f.silu}[act](v)


def _back64(g, m, bias):
    c, out = m["case"], {}
    z = m["z"].double().requires_grad_() if "z" in m else None
    if z is None:
        d = g
    else:
        mul = m["mul"].double().requires_grad_() if "mul" in m else None
        y = _act64(z, c["act"])
        y = y * mul if mul is not None else y
        got = torch.autograd.grad(y, [z] + ([mul] if mul is not None else []), g)
        d = got[0]
        if mul is not None:
            out["dmul"] = got[1]
    if bias:
        out["db"] = d.sum(0)
    return d, out


def exact(c, seed):
    m = _inputs(c, seed)
    if c["kind"] == "update":
        a, b, cc = COEFFICIENTS
        mom = BETA * m["momentum"].double() + m["grad"].double()
        u, w, at = m["grad"].double() + BETA * mom if c["nesterov"] else mom, m["weight"].double(), 0
        new, spans, grams = torch.empty_like(w), [], []
        for rows, cols in _layer_shapes(c) * c["layers"]:
            U = u[at:at + rows * cols].view(rows, cols)
            spans.append((at, rows, cols, U))
            grams.append((U @ U.T if rows <= cols else U.T @ U).cpu())
            at += rows * cols
        for (at, rows, cols, U), G in zip(spans, grams):              # the polynomial on the eigenvalues of the Gram matrix
            norm = float(G.trace().sqrt()) + EPS
            ev, V = torch.linalg.eigh(G / norm ** 2)
            p, lam = torch.ones_like(ev), ev.clamp(min=0)
            for _ in range(STEPS):
                q = a + b * lam + cc * lam ** 2
                p, lam = p * q, lam * q ** 2
            P = ((V * p) @ V.T / norm).cuda()
            X = P @ U if rows <= cols else U @ P
            W = w[at:at + rows * cols].view(rows, cols)
            new[at:at + rows * cols] = (W - LR * (_update_scale(rows, cols) * X + DECAY * W)).reshape(-1)
        return {"momentum": mom, "weight": new, "weight_bf16": new}
    if c["kind"] == "act":
        d, out = _back64(m["dY"].double(), m, c["bias"])
        return out | ({"dZ": d} if "z" in m else {})
    W = _weights64(m)
    if "A" in m:
        W = W + SCALE * m["B"].double() @ m["A"].double()
    if c["kind"] == "bwd":
        g = m["dY"].double() @ W
        d, out = _back64(g + m["residual"].double() if "residual" in m else g, m, False)
        return out | {"dX": d}
    v = m["x"].double() @ W.T
    v = v + m["bias"].double() if "bias" in m else v
    y = _act64(v, c["act"])
    y = y * m["mul"].double() if "mul" in m else y
    y = y + m["residual"].double() if "residual" in m else y
    return {"y": y} | ({"z": v} if c["z"] else {})
