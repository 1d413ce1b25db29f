"""Workloads the layer norm, the gated feed-forward products and the Muon step
are timed on, with 64-bit references for their outputs.

Three families of calls around a linear layer and the optimizer step:

  norm      layer norm of rows of activations, forward, backward (the weight's
            and the bias's gradients reduced over the rows), or both
  gated     the wide half of a gated feed-forward block, h = act(x g') * (x u')
            for two weights g and u: forward (down to one token), backward from
            the input alone, or a training step's forward and backward
  ortho     orthogonalising matrices by Newton-Schulz products
  muon      the optimizer step made of it: replica gradients averaged, momentum,
            orthogonalised, weights updated, for many matrices of a flat buffer

A case is a dict of plain values:
  op        "norm", "gated", "ortho" or "muon"
  norm:     rows, cols, dtype, part ("forward", "backward", "both"), affine
  gated:    m (tokens), k (inputs), n (hidden units), act ("silu", "gelu"),
            part ("forward", "backward", "both")
  ortho:    batch, rows, cols, dtype (of the input), rank (0: a gradient of full
            rank; else that of its strong part)
  muon:     layout ("resnet50", "vgg16-classifier", or "drawn" with `matrices`
            and `shape_seed`), K, dtype (of the replicas), nesterov
`run` computes the plain form in 32 bits from elementary torch operations, or,
with `own` set, calls the package.
"""
from __future__ import annotations

import math
import random

import torch

#: False: `run` computes the plain form; True: it calls the package.
own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5                            # of the layer norm
STEPS = 5                             # Newton-Schulz steps
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
NORM_EPS = 1e-7                       # added to a matrix's norm
MOMENTUM, LR, DECAY = 0.95, 1e-3, 0.1
PAD = 64                              # a matrix of the flat buffers starts at a multiple of this
#: the most a drawn case may cost: the largest listed ones
MOST_ELEMENTS = 16384 * 8192
MOST_GATED = 12 * 8192 * 4096 * 16384
MOST_ORTHO = 1 << 42


def _norm(name, rows, cols, dtype, part, affine=True):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "part": part,
            "affine": affine}


def _gated(name, m, k, n, act, part):
    return {"name": name, "op": "gated", "m": m, "k": k, "n": n, "act": act, "part": part}


def _ortho(name, batch, rows, cols, dtype, rank):
    return {"name": name, "op": "ortho", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype,
            "rank": rank}


def _muon(name, layout, K, dtype, nesterov=True, matrices=0, shape_seed=0):
    return {"name": name, "op": "muon", "layout": layout, "K": K, "dtype": dtype, "nesterov": nesterov,
            "matrices": matrices, "shape_seed": shape_seed}


def listed():
    return [
        # one token before a linear layer: latency
        _norm("norm-token", 1, 4096, "bf16", "forward"),
        # a batch of tokens on the way to a layer's products
        _norm("norm-forward", 8192, 4096, "bf16", "forward"),
        # fp32 rows of a classifier's width, both passes, sizes that fill nothing
        _norm("norm-ragged", 5001, 1000, "f32", "both"),
        # the largest: the backward pass of a long batch of wide rows
        _norm("norm-backward", 16384, 8192, "bf16", "backward"),
        # one token through a square block: the weights' bytes, latency
        _gated("gated-token", 1, 4096, 4096, "silu", "forward"),
        # a few requests through a wide block
        _gated("gated-tokens-24", 24, 4096, 16384, "silu", "forward"),
        # a training step of a batch whose sizes fill no tile
        _gated("gated-ragged", 1000, 2047, 1001, "gelu", "both"),
        # the largest: a training step of a wide block on 8192 tokens
        _gated("gated-step", 8192, 4096, 16384, "silu", "both"),
        # one matrix, the classifier of ResNet-18: fifteen dependent products
        _ortho("ortho-small", 1, 1000, 512, "f32", 0),
        # the stacked 1 x 1 convolutions of one of ResNet-50's stages, the
        # gradients of low rank that few examples leave
        _ortho("ortho-stack", 8, 2048, 512, "bf16", 64),
        # the optimizer step of all of ResNet-50's matrices, sixteen bf16 replicas
        _muon("muon-resnet50", "resnet50", 16, "bf16"),
        # the largest: VGG-16's three classifier matrices, fp32 replicas
        _muon("muon-vgg16", "vgg16-classifier", 4, "f32"),
    ]


def _log(rng, lo, hi, unit=1):
    """A whole number (a multiple of `unit`) between lo and hi, spread over its
    logarithm."""
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, unit * int(round(x / unit))))


def draw(rng):
    op = rng.choice(["norm", "norm", "gated", "gated", "ortho", "muon"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "norm":
        cols = _log(rng, 16, 32768, rng.choice([1, 8]))
        rows = _log(rng, 1, min(65536, MOST_ELEMENTS // cols))
        c = _norm("", rows, cols, dtype, rng.choice(["forward", "backward", "both"]), rng.random() < 0.8)
    elif op == "gated":
        part = rng.choice(["forward", "forward", "backward", "both"])
        m = _log(rng, 1, 8192) if part == "forward" else _log(rng, 16, 8192)
        unit = rng.choice([1, 128])     # any width, or a multiple of 128
        c = _gated("", m, _log(rng, max(32, unit), 8192, unit), _log(rng, max(32, unit), 16384, unit),
                   rng.choice(["silu", "gelu"]), part)
        while work(c)["flops"] > MOST_GATED:
            c["m"] = (c["m"] + 1) // 2
    elif op == "ortho":
        rows, cols = _log(rng, 1, 4096), _log(rng, 1, 8192)
        if rng.random() < 0.5:
            rows, cols = cols, rows
        c = _ortho("", _log(rng, 1, 24), rows, cols, dtype, rng.choice([0, 0, 1, 16]))
        while work(c)["flops"] > MOST_ORTHO:
            c["batch"] = (c["batch"] + 1) // 2
    else:
        c = _muon("", "drawn", _log(rng, 1, 16), dtype, rng.random() < 0.7, _log(rng, 1, 24),
                  rng.randrange(1 << 20))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs --


def _resnet50():
    """The convolutions as matrices [out, in * k * k], and the classifier."""
    shapes, inner, wide = [(64, 147)], 64, 64
    for blocks, width in ((3, 64), (4, 128), (6, 256), (3, 512)):
        for b in range(blocks):
            shapes += [(width, wide), (width, 9 * width), (4 * width, width)]
            if b == 0:
                shapes.append((4 * width, wide))
            wide = 4 * width
    return shapes + [(1000, 2048)]


def _shapes(case):
    """[(rows, cols)] of a step's matrices."""
    if case["layout"] == "resnet50":
        return _resnet50()
    if case["layout"] == "vgg16-classifier":
        return [(4096, 25088), (4096, 4096), (1000, 4096)]
    r = random.Random(case["shape_seed"])
    return [(_log(r, 1, 2048), _log(r, 1, 4608)) for _ in range(case["matrices"])]


def _layers(case):
    """([(offset, rows, cols)], elements of the flat buffers)."""
    out, o = [], 0
    for rows, cols in _shapes(case):
        out.append((o, rows, cols))
        o += -(-rows * cols // PAD) * PAD
    return out, o


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * int(seed) + 31)
    return gen


def _randn(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _activations(gen, rows, cols, dtype):
    """Rows with an offset and channels of a log-normal spread, some rows
    (padding) zero."""
    x = _randn(gen, rows, cols).mul_(_randn(gen, cols).mul_(0.5).exp_()).add_(_randn(gen, rows, 1).mul_(0.3))
    if rows > 1:
        x *= torch.rand(rows, 1, device="cuda", generator=gen) > 0.05
    return x.to(DTYPES[dtype])


def _norm_inputs(case, seed):
    """x, the output gradient, weight, bias."""
    gen, rows, cols = _generator(seed), case["rows"], case["cols"]
    x = _activations(gen, rows, cols, case["dtype"])
    dy = _activations(gen, rows, cols, case["dtype"])
    dy *= 1.0 / 256
    if not case["affine"]:
        return x, dy, None, None
    return x, dy, _randn(gen, cols).mul_(0.2).add_(1.0), _randn(gen, cols).mul_(0.1)


def _gated_inputs(case, seed):
    """x [m, k], the weights [n, k], the output gradient [m, n], all bf16."""
    gen, m, k, n = _generator(seed), case["m"], case["k"], case["n"]
    x = _activations(gen, m, k, "bf16")
    gate = _randn(gen, n, k).mul_(1.0 / math.sqrt(k)).bfloat16()
    up = _randn(gen, n, k).mul_(1.0 / math.sqrt(k)).bfloat16()
    dh = _activations(gen, m, n, "bf16") * (1.0 / 256) if case["part"] != "forward" else None
    return x, gate, up, dh


def _gradient(gen, batch, rows, cols, rank):
    """Gradients: noise, under it a strong part of low rank."""
    g = _randn(gen, batch, rows, cols)
    if rank:
        r = min(rank, rows, cols)
        g = g.mul_(0.05) + torch.bmm(_randn(gen, batch, rows, r), _randn(gen, batch, r, cols)).mul_(r ** -0.5)
    return g.mul_(1e-3)


def _ortho_inputs(case, seed):
    gen = _generator(seed)
    return _gradient(gen, case["batch"], case["rows"], case["cols"], case["rank"]).to(DTYPES[case["dtype"]])


def _muon_inputs(case, seed):
    """Flat weights and momentum, the stack of replica gradients."""
    gen, (layers, total) = _generator(seed), _layers(case)
    w, m = torch.zeros(total, device="cuda"), torch.zeros(total, device="cuda")
    grads = torch.zeros(case["K"], total, device="cuda", dtype=DTYPES[case["dtype"]])
    for o, rows, cols in layers:
        n = rows * cols
        w[o:o + n] = _randn(gen, n).mul_(cols ** -0.5)
        m[o:o + n] = _gradient(gen, 1, rows, cols, 16).view(-1).mul_(5.0)
        base = _gradient(gen, 1, rows, cols, 16).view(-1)
        for k in range(case["K"]):
            grads[k, o:o + n] = (base + _randn(gen, n).mul_(1e-3)).to(grads.dtype)
    return w, m, grads


def prepare(case, seed):
    """What a training or serving program holds before the call: weights laid out
    once after an optimizer step, the statistics that a forward pass left, the
    optimizer's handle."""
    state = {"case": case}
    if case["op"] == "norm":
        state["x"], state["dy"], state["weight"], state["bias"] = _norm_inputs(case, seed)
        if case["part"] == "backward":
            x = state["x"].float()
            mean = x.mean(dim=1)
            state["saved"] = torch.stack([mean, ((x - mean[:, None]).square().mean(dim=1) + EPS).rsqrt()])
    elif case["op"] == "gated":
        state["x"], gate, up, state["dh"] = _gated_inputs(case, seed)
        if own:
            from paper_2603_18112_amd import glu
            state["w"] = glu.Weight(gate, up)
        else:
            state["w"] = gate, up
    elif case["op"] == "ortho":
        state["x"] = _ortho_inputs(case, seed)
    else:
        state["w"], state["m"], state["grads"] = _muon_inputs(case, seed)
        if own:
            from paper_2603_18112_amd import muon
            state["opt"] = muon.Muon(_layers(case)[0], state["w"], state["m"], case["K"],
                                     grad_dtype=case["dtype"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY,
                                     nesterov=case["nesterov"], steps=STEPS, coefficients=COEFFICIENTS,
                                     eps=NORM_EPS)
    return state


# --------------------------------------------------------------- plain form --


def _plain_norm(state):
    case, x, weight = state["case"], state["x"].float(), state["weight"]
    out = {}
    if case["part"] == "backward":
        mean, rstd = state["saved"][0][:, None], state["saved"][1][:, None]
    else:
        mean = x.mean(dim=1, keepdim=True)
        rstd = ((x - mean).square().mean(dim=1, keepdim=True) + EPS).rsqrt()
    xh = (x - mean) * rstd
    if case["part"] != "backward":
        y = xh if weight is None else xh * weight + state["bias"]
        out["y"], out["mean"], out["rstd"] = y.to(state["x"].dtype), mean[:, 0], rstd[:, 0]
    if case["part"] != "forward":
        dy = state["dy"].float()
        g = dy if weight is None else dy * weight
        dx = rstd * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))
        out["dx"] = dx.to(state["x"].dtype)
        if weight is not None:
            out["dweight"], out["dbias"] = (dy * xh).sum(dim=0), dy.sum(dim=0)
    return out


def _act(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1.0 + g * (1.0 - s))
    c = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * c, c + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_gated(state):
    case, x = state["case"], state["x"].float()
    gate, up = (t.float() for t in state["w"])
    g, u = x @ gate.t(), x @ up.t()
    a, da = _act(g, case["act"])
    out = {}
    if case["part"] != "backward":
        out["h"] = (a * u).bfloat16()
    if case["part"] != "forward":
        dh = state["dh"].float()
        dg, du = dh * u * da, dh * a
        out["dx"] = (dg @ gate + du @ up).bfloat16()
        out["dgate"], out["dup"] = (dg.t() @ x).bfloat16(), (du.t() @ x).bfloat16()
    return out


def _plain_ortho(x):
    """Newton-Schulz steps of [..., rows, cols] in fp32."""
    a, b, c = COEFFICIENTS
    x = x.float()
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-2, -1).contiguous()
    norm = x.double().square().sum(dim=(-2, -1), keepdim=True).sqrt()
    x = (x.double() / (norm + NORM_EPS)).float()
    for _ in range(STEPS):
        s = x @ x.transpose(-2, -1).contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.transpose(-2, -1).contiguous() if tall else x


def _plain_muon(state):
    case, w, m, grads = state["case"], state["w"], state["m"], state["grads"]
    for o, rows, cols in _layers(case)[0]:
        n = rows * cols
        g = grads[:, o:o + n].float().mean(dim=0)
        buf = m[o:o + n]
        buf.mul_(MOMENTUM).add_(g)
        u = g + MOMENTUM * buf if case["nesterov"] else buf
        step = _plain_ortho(u.view(rows, cols)).reshape(-1)
        w[o:o + n].mul_(1.0 - LR * DECAY).sub_(step, alpha=LR * math.sqrt(max(1.0, rows / cols)))
    return {"w": w, "m": m}


# ------------------------------------------------------------ package calls --


def _own_norm(state):
    from paper_2603_18112_amd import norm
    case, x, weight = state["case"], state["x"], state["weight"]
    out, saved = {}, state.get("saved")
    if case["part"] != "backward":
        out["y"], saved = norm.layer_norm(x, weight, state["bias"], eps=EPS, save=True)
        out["mean"], out["rstd"] = saved[0], saved[1]
    if case["part"] != "forward":
        dx, dw, db = norm.layer_norm_backward(state["dy"], x, saved, weight, need_dw=weight is not None,
                                              need_db=weight is not None)
        out["dx"] = dx
        if weight is not None:
            out["dweight"], out["dbias"] = dw, db
    return out


def _own_gated(state):
    from paper_2603_18112_amd import glu
    case, x, dh, w = state["case"], state["x"], state["dh"], state["w"]
    if case["part"] == "forward":
        return {"h": glu.gated_linear(x, w, act=case["act"])}
    out, saved = {}, None
    if case["part"] == "both":
        out["h"], saved = glu.gated_linear(x, w, act=case["act"], save=True)
    out["dx"], out["dgate"], out["dup"] = glu.gated_linear_backward(dh, x, w, saved=saved, act=case["act"],
                                                                    dw_dtype="bf16")
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        if op == "norm":
            return _own_norm(state)
        if op == "gated":
            return _own_gated(state)
        if op == "ortho":
            from paper_2603_18112_amd import muon
            return {"o": muon.orthogonalize(state["x"], steps=STEPS, coefficients=COEFFICIENTS, eps=NORM_EPS,
                                            dtype="bf16")}
        state["opt"].step(state["grads"])
        return {"w": state["w"], "m": state["m"]}
    if op == "norm":
        return _plain_norm(state)
    if op == "gated":
        return _plain_gated(state)
    if op == "ortho":
        return {"o": _plain_ortho(state["x"]).bfloat16()}
    return _plain_muon(state)


def _ortho_flops(rows, cols):
    """Each step's three products; two of them are symmetric, and half of each is
    enough."""
    s, l = min(rows, cols), max(rows, cols)
    return STEPS * (s * s * l + s * s * s + 2 * s * s * l)


def work(case):
    """A norm reads x (and dy) and writes y (or dx).  A gated product reads the
    activations, the output gradient and the weights and writes its results; what a
    step keeps between its passes is written and read by choice.  An
    orthogonalisation reads and writes its matrices; a step of it reads the
    replicas, the weights and the momentum and writes the last two."""
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "norm":
        n, e, passes = case["rows"] * case["cols"], size[case["dtype"]], {"forward": 2, "backward": 3, "both": 4}
        return {"bytes": n * e * passes[case["part"]] + (case["cols"] * 8 if case["affine"] else 0),
                "flops": n * {"forward": 7, "backward": 13, "both": 20}[case["part"]]}
    if case["op"] == "gated":
        m, k, n = case["m"], case["k"], case["n"]
        b = {"forward": m * k + 2 * n * k + m * n, "backward": 2 * m * k + 4 * n * k + m * n,
             "both": 2 * m * k + 4 * n * k + 2 * m * n}
        return {"bytes": 2 * b[case["part"]], "flops": m * k * n * {"forward": 4, "backward": 12, "both": 12}[case["part"]]}
    if case["op"] == "ortho":
        n = case["batch"] * case["rows"] * case["cols"]
        return {"bytes": n * (size[case["dtype"]] + 2), "flops": case["batch"] * _ortho_flops(case["rows"], case["cols"])}
    shapes = _shapes(case)
    n = sum(r * c for r, c in shapes)
    return {"bytes": n * (case["K"] * size[case["dtype"]] + 16), "flops": sum(_ortho_flops(r, c) for r, c in shapes)}


# --------------------------------------------------------- 64-bit reference --


def _exact_ortho(g):
    """Each step is X times a polynomial of its Gram matrix on the shorter side,
    by Horner's rule, in 64 bits."""
    x = g.double()
    x = x / (torch.linalg.vector_norm(x) + NORM_EPS)
    eye = torch.eye(min(x.shape), dtype=torch.float64, device=x.device)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        wide = x.shape[0] <= x.shape[1]
        xt = x.t().contiguous()
        gram = torch.mm(x, xt) if wide else torch.mm(xt, x)
        p = a * eye + torch.mm(gram, b * eye + c * gram)
        x = torch.mm(p, x) if wide else torch.mm(x, p)
    return x


def exact(case, seed):
    if case["op"] == "norm":
        x, dy, weight, bias = _norm_inputs(case, seed)
        x, dy = x.double(), dy.double()
        n = case["cols"]
        gamma = torch.ones(n, dtype=torch.float64, device="cuda") if weight is None else weight.double()
        mean = x.sum(dim=1) / n
        var = torch.var(x, dim=1, correction=0) if n > 1 else torch.zeros_like(mean)
        std = torch.sqrt(var + EPS)
        z = (x - mean.unsqueeze(1)) / std.unsqueeze(1)
        out = {}
        if case["part"] != "backward":
            out["y"] = z * gamma + (0.0 if bias is None else bias.double())
            out["mean"], out["rstd"] = mean, 1.0 / std
        if case["part"] != "forward":
            v = dy * gamma
            s1, s2 = v.sum(dim=1, keepdim=True), torch.linalg.vecdot(v, z).unsqueeze(1)
            out["dx"] = (n * v - s1 - z * s2) / (n * std.unsqueeze(1))
            if weight is not None:
                out["dweight"], out["dbias"] = torch.linalg.vecdot(dy, z, dim=0), dy.sum(dim=0)
        return out
    if case["op"] == "gated":
        x, gate, up, dh = _gated_inputs(case, seed)
        x, both = x.double(), torch.cat([gate, up]).double()
        n = case["n"]
        z = torch.mm(x, both.t().contiguous())
        g, u = z[:, :n], z[:, n:]
        if case["act"] == "silu":
            a = g / (1.0 + torch.exp(-g))
            da = (a * torch.exp(-g) + 1.0) / (1.0 + torch.exp(-g))
        else:
            a = 0.5 * g * torch.erfc(-g / math.sqrt(2.0))
            da = 0.5 * torch.erfc(-g / math.sqrt(2.0)) + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)
        out = {}
        if case["part"] != "backward":
            out["h"] = a * u
        if case["part"] != "forward":
            d = torch.cat([dh.double() * u * da, dh.double() * a], dim=1)
            out["dx"] = torch.mm(d, both)
            dw = torch.mm(d.t().contiguous(), x)
            out["dgate"], out["dup"] = dw[:n], dw[n:]
        return out
    if case["op"] == "ortho":
        return {"o": torch.stack([_exact_ortho(g) for g in _ortho_inputs(case, seed)])}
    w, m, grads = (t.double() for t in _muon_inputs(case, seed))
    mean = grads.sum(dim=0) / case["K"]
    buf = m * MOMENTUM + mean
    u = buf * MOMENTUM + mean if case["nesterov"] else buf
    new = w * (1.0 - LR * DECAY)
    flat = torch.zeros_like(w, dtype=torch.bool)
    for o, rows, cols in _layers(case)[0]:
        scale = math.sqrt(rows / cols) if rows > cols else 1.0
        new[o:o + rows * cols] -= LR * scale * _exact_ortho(u[o:o + rows * cols].view(rows, cols)).reshape(-1)
        flat[o:o + rows * cols] = True
    return {"w": torch.where(flat, new, w), "m": torch.where(flat, buf, m)}
