"""Workloads the 4-bit and gradient-clipping operators are timed on, with
64-bit references for their outputs.

Three families of calls that a training program makes around the AGS step:

  clip      the norm over many gradient tensors and their clipping to a bound,
            on the way into the replica stack of the step
  quantize  microscaled 4-bit floating point (E2M1 elements, one E8M0 scale
            for 32 of them): a tensor stored in 4 bits and read back, along
            its rows, its columns or both, rounded to nearest or with given
            random bytes
  linear    the products of a linear layer whose operands are held that way:
            forward (down to one token), backward (input and weight
            gradients), and both in one training step

A case is a dict of plain values:
  op        "clip", "quantize" or "linear"
  clip:     kind      "inplace": tensors clipped where they are
                      "pack":    one worker's tensors clipped into its row of
                                 the flat replica stack
                      "stack":   every row of a replica stack clipped to its
                                 own norm, into a stack of another type
            tensors, elements, shape_seed: how many tensors, parameters in
                      all, and the seed their sizes come from
            K, dtype, out_dtype, bound: replicas, types, the largest norm
  quantize: rows, cols, dtype, axis ("rows", "cols", "both"), noise
  linear:   m, k, n, dtype, part ("forward", "backward", "both"), noise (on
            the output gradient), dw_dtype
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
EPS = 1e-6            # added to the norm in the clip coefficient
PAD = 64              # a layer of the flat buffers starts at a multiple of this
GAP = 2048            # elements between the rows of a replica stack
BLOCK = 32            # elements that share one scale
#: the most a drawn case may cost: the largest listed ones
MOST_ELEMENTS = 8 * 25_557_032
MOST_FLOPS = 6 * 8192 ** 3


def _clip(name, kind, tensors, elements, shape_seed, K, dtype, out_dtype, bound):
    return {"name": name, "op": "clip", "kind": kind, "tensors": tensors, "elements": elements,
            "shape_seed": shape_seed, "K": K, "dtype": dtype, "out_dtype": out_dtype, "bound": bound}


def _quantize(name, rows, cols, dtype, axis, noise):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "axis": axis,
            "noise": noise}


def _linear(name, m, k, n, dtype, part, noise=False, dw_dtype="f32"):
    return {"name": name, "op": "linear", "m": m, "k": k, "n": n, "dtype": dtype, "part": part,
            "noise": noise, "dw_dtype": dw_dtype}


def listed():
    return [
        # a small model's gradients, nothing to clip: launches and host work
        _clip("clip-small", "inplace", 10, 24_234, 1, 1, "f32", "f32", 1e6),
        # one worker's bf16 gradients (ResNet-50's count and size) into its row
        _clip("clip-pack", "pack", 161, 25_557_032, 2, 1, "bf16", "bf16", 1.0),
        # eight workers' fp32 gradients, each clipped to its own norm, to bf16
        _clip("clip-stack", "stack", 161, 25_557_032, 3, 8, "f32", "bf16", 1.0),
        # a large model's usual step: the norm is taken, nothing is clipped
        _clip("clip-large", "inplace", 32, 138_357_544, 4, 1, "f32", "f32", 1e6),
        # the activations of a small batch before a classifier
        _quantize("quantize-small", 64, 1000, "f32", "rows", False),
        # fp32 weights of odd sizes for the transposed product
        _quantize("quantize-cols", 5001, 2047, "f32", "cols", False),
        # an output gradient for both products of the backward pass
        _quantize("quantize-both", 8192, 4096, "bf16", "both", True),
        # one token through a square layer: latency
        _linear("token", 1, 4096, 4096, "bf16", "forward"),
        # a few requests through VGG-16's first classifier layer: the weights' bytes
        _linear("tokens-24", 24, 25088, 4096, "bf16", "forward"),
        # a batch through ResNet-50's classifier, sizes that fill no tile
        _linear("forward-ragged", 1000, 2048, 1000, "f32", "forward"),
        # the backward pass of a wide layer, rounded with random bytes, the
        # weight gradient as a replica stack holds it
        _linear("backward-wide", 4096, 4096, 16384, "bf16", "backward", True, "bf16"),
        # the largest: forward and backward of a square layer on 8192 tokens
        _linear("step-square", 8192, 8192, 8192, "bf16", "both", True, "f32"),
    ]


def _log(rng, lo, hi, unit=1):
    """A whole number (a multiple of `unit`) between lo and hi, spread over its
    logarithm."""
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, unit * int(round(x / unit))))


def draw(rng):
    op = rng.choice(["clip", "quantize", "linear", "linear"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "clip":
        kind = rng.choice(["inplace", "pack", "stack"])
        tensors = _log(rng, 1, 600)
        K = _log(rng, 2, 16) if kind == "stack" else 1
        elements = _log(rng, 2_000, 138_357_544 if K == 1 else MOST_ELEMENTS // K)
        out = dtype if kind == "inplace" else rng.choice(["f32", "bf16"])
        # in place, a bound that clips would find other gradients on the next pass
        bound = 1e6 if kind == "inplace" else rng.choice([1.0, 1.0, 1e6])
        c = _clip("", kind, tensors, elements, rng.randrange(1 << 20), K, dtype, out, bound)
    elif op == "quantize":
        rows = _log(rng, 1, 25_088)
        cols = _log(rng, 1, min(25_088, 8192 * 4096 // rows))
        c = _quantize("", rows, cols, dtype, rng.choice(["rows", "cols", "both"]),
                      rng.random() < 0.4)
    else:
        part = rng.choice(["forward", "forward", "backward", "both"])
        m = _log(rng, 1, 8192) if part == "forward" else _log(rng, 16, 8192)
        unit = rng.choice([1, 640])     # any width, or a multiple of 128
        k, n = _log(rng, max(32, unit), 25_088, unit), _log(rng, max(32, unit), 16_384, unit)
        c = _linear("", m, k, n, dtype, part, rng.random() < 0.5, rng.choice(["f32", "bf16"]))
        while work(c)["flops"] > MOST_FLOPS:
            c["m"] = (c["m"] + 1) // 2
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs --


def _numels(case):
    """Tensor sizes of a model: weights of very different sizes, each followed
    by two small vectors, no size a multiple of anything."""
    r = random.Random(case["shape_seed"])
    n = case["tensors"]
    share = [math.exp(r.uniform(0.0, 6.0)) if i % 3 == 0 else 0.0 for i in range(n)]
    total = sum(share)
    return [max(1, int(case["elements"] * s / total)) if s else r.randint(1, 700) for s in share]


def _flat(case):
    """(offset of each layer, row stride of the replica stack)."""
    offsets, o = [], 0
    for x in _numels(case):
        offsets.append(o)
        o += -(-x // PAD) * PAD
    return offsets, o + GAP


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * int(seed) + 29)
    return gen


def _clip_inputs(case, seed):
    """Gradients of a log-uniform scale per tensor: the tensors of one flat
    gradient buffer, or a replica stack whose rows differ by up to a factor of
    ten."""
    gen, r, dt = _generator(seed), random.Random(int(seed)), DTYPES[case["dtype"]]
    numels = _numels(case)
    sigma = [10.0 ** r.uniform(-4.0, -1.0) for _ in numels]
    offsets, stride = _flat(case)
    g = torch.zeros(case["K"], stride, device="cuda", dtype=dt)
    for k in range(case["K"]):
        f = 10.0 ** r.uniform(-1.0, 0.0)
        for o, n, s in zip(offsets, numels, sigma):
            g[k, o:o + n] = torch.randn(n, device="cuda", generator=gen).mul_(s * f).to(dt)
    return g


def _matrix(rows, cols, dtype, gen, spread):
    """A matrix whose columns have scales of a log-normal spread (activations
    have wide channels), some of its rows masked to zero."""
    scale = torch.randn(cols, device="cuda", generator=gen).mul_(spread).exp_()
    x = torch.randn(rows, cols, device="cuda", generator=gen).mul_(scale)
    if rows > 1:
        x *= (torch.rand(rows, 1, device="cuda", generator=gen) > 0.05)
    return x.to(DTYPES[dtype])


def _noise(rows, cols, gen):
    return torch.randint(0, 256, (rows, cols), dtype=torch.uint8, device="cuda", generator=gen)


def _quantize_inputs(case, seed):
    gen = _generator(seed)
    x = _matrix(case["rows"], case["cols"], case["dtype"], gen, 1.0)
    return x, _noise(case["rows"], case["cols"], gen) if case["noise"] else None


def _linear_inputs(case, seed):
    """Activations x [m, k], fp32 master weights w [n, k], the output gradient
    dy [m, n] and its random bytes."""
    gen, m, k, n = _generator(seed), case["m"], case["k"], case["n"]
    x = _matrix(m, k, case["dtype"], gen, 0.7)
    w = torch.randn(n, k, device="cuda", generator=gen).mul_(1.0 / math.sqrt(k))
    if case["part"] == "forward":
        return x, w, None, None
    dy = _matrix(m, n, case["dtype"], gen, 0.5)
    dy *= 1.0 / 1024
    return x, w, dy, _noise(m, n, gen) if case["noise"] else None


def prepare(case, seed):
    """What a training program holds before the call.  The weights of a linear
    layer are laid out once after each optimizer step, so they are here."""
    state = {"case": case}
    if case["op"] == "clip":
        g = _clip_inputs(case, seed)
        offsets, stride = _flat(case)
        if case["kind"] != "stack":
            state["flat"] = g
            g = [g[0, o:o + n] for o, n in zip(offsets, _numels(case))]
        state["g"] = g
        out_dt = DTYPES[case["out_dtype"]]
        if case["kind"] == "pack":
            state["out"] = torch.zeros(stride, device="cuda", dtype=out_dt)
        elif case["kind"] == "stack":
            state["out"] = torch.zeros(case["K"], stride, device="cuda", dtype=out_dt)
        if own:
            from paper_2603_18112_amd import clip
            layers = [(o, n, 0) for o, n in zip(offsets, _numels(case))]
            if case["kind"] == "inplace":
                state["plan"] = clip.GradClip.for_tensors(g)
            elif case["kind"] == "pack":
                state["plan"] = clip.GradClip.for_tensors(g, layers=layers, out_dtype=case["out_dtype"])
            else:
                state["plan"] = clip.GradClip.for_stack(layers, case["K"], stride, dtype=case["dtype"],
                                                        out_dtype=case["out_dtype"])
    elif case["op"] == "quantize":
        state["x"], state["noise"] = _quantize_inputs(case, seed)
    else:
        state["x"], w, state["dy"], state["noise"] = _linear_inputs(case, seed)
        forward, backward = case["part"] != "backward", case["part"] != "forward"
        if own:
            from paper_2603_18112_amd import mx
            state["w"] = mx.Weight(w, forward=forward, backward=backward)
        else:
            state["w"] = _plain_rows(w, None) if forward else None
            state["wt"] = _plain_rows(w.t().contiguous(), None) if backward else None
    return state


# --------------------------------------------------------------- plain form --


def _plain_rows(x, noise):
    """The values that x's elements stand for once its rows are held in 4 bits:
    blocks of 32 along the last axis, fp32."""
    rows, cols = x.shape
    pad = -cols % BLOCK
    x = torch.nn.functional.pad(x.float(), (0, pad)).view(rows, -1, BLOCK)
    amax = x.abs().amax(dim=-1, keepdim=True)
    bits = amax.view(torch.int32)
    e = (bits >> 23) - 129
    if noise is not None:       # a scale under which nothing is clipped
        e = e + ((bits & 0x7FFFFF) > 0x400000)
    e = e.clamp(-127, 125)
    y = x.abs() * ((127 - e) << 23).view(torch.float32)
    if noise is None:
        q = 0.5 * ((y > 0.25).float() + (y >= 0.75) + (y > 1.25) + (y >= 1.75))
        q += (y > 2.5).float() + (y >= 3.5) + 2.0 * (y > 5.0)
    else:
        r = torch.nn.functional.pad(noise, (0, pad)).view(rows, -1, BLOCK).float()
        step = 0.5 + 0.5 * (y >= 2.0) + (y >= 4.0)
        u = y / step
        lo = u.floor()
        q = ((lo + ((u - lo) * 256.0 + r + 0.5 >= 256.0)) * step).clamp(max=6.0)
    # 2^e in two factors: 2^-127 has no normal fp32 value
    half = (e >> 1)
    q = q * ((127 + half) << 23).view(torch.float32) * ((127 + e - half) << 23).view(torch.float32)
    q = torch.where(x < 0, -q, q)
    return q.view(rows, -1)[:, :cols]


def _plain_cols(x, noise):
    return _plain_rows(x.t(), None if noise is None else noise.t()).t()


def _plain_clip(state):
    case, g = state["case"], state["g"]
    numels = _numels(case)
    if case["kind"] == "stack":
        offsets, _ = _flat(case)
        out, norms = state["out"], []
        for k in range(case["K"]):
            parts = [g[k, o:o + n].float() for o, n in zip(offsets, numels)]
            norm = torch.stack([p.square().sum() for p in parts]).sum().sqrt()
            c = (case["bound"] / (norm + EPS)).clamp(max=1.0)
            for p, o, n in zip(parts, offsets, numels):
                out[k, o:o + n] = (p * c).to(out.dtype)
            norms.append(norm)
        return {"norms": torch.stack(norms), "out": out}
    parts = [t.float() for t in g]
    norm = torch.stack([p.square().sum() for p in parts]).sum().sqrt()
    c = (case["bound"] / (norm + EPS)).clamp(max=1.0)
    if case["kind"] == "inplace":
        for t, p in zip(g, parts):
            t.copy_(p * c)
        return {"norms": norm.view(1), "out": state["flat"]}
    out = state["out"]
    for p, o, n in zip(parts, _flat(case)[0], numels):
        out[o:o + n] = (p * c).to(out.dtype)
    return {"norms": norm.view(1), "out": out}


def _plain_quantize(state):
    case, x, noise = state["case"], state["x"], state["noise"]
    out = {}
    if case["axis"] != "cols":
        out["rows"] = _plain_rows(x, noise).to(torch.bfloat16)
    if case["axis"] != "rows":
        # read back as it is stored: the transpose
        out["cols"] = _plain_rows(x.t(), None if noise is None else noise.t()).to(torch.bfloat16)
    return out


def _plain_linear(state):
    case, x, dy = state["case"], state["x"], state["dy"]
    out = {}
    if case["part"] != "backward":
        out["y"] = (_plain_rows(x, None) @ state["w"].t()).to(x.dtype)
    if case["part"] != "forward":
        out["dx"] = (_plain_rows(dy, state["noise"]) @ state["wt"].t()).to(dy.dtype)
        dw = _plain_cols(dy, state["noise"]).t() @ _plain_cols(x, None)
        out["dw"] = dw.to(DTYPES[case["dw_dtype"]])
    return out


# ------------------------------------------------------------ package calls --


def _own_clip(state):
    case, g = state["case"], state["g"]
    if case["kind"] == "inplace":
        return {"norms": state["plan"].clip(g, case["bound"]), "out": state["flat"]}
    bases = [g] if case["kind"] == "stack" else g
    return {"norms": state["plan"].clip(bases, case["bound"], out=[state["out"]]), "out": state["out"]}


def _own_quantize(state):
    from paper_2603_18112_amd import mx
    case, x, noise = state["case"], state["x"], state["noise"]
    if case["axis"] == "rows":
        return {"rows": mx.dequantize(mx.quantize(x, noise=noise), "bf16")}
    if case["axis"] == "cols":
        return {"cols": mx.dequantize(mx.quantize_t(x, noise=noise), "bf16")}
    q, qt = mx.quantize_both(x, noise=noise)
    return {"rows": mx.dequantize(q, "bf16"), "cols": mx.dequantize(qt, "bf16")}


def _own_linear(state):
    from paper_2603_18112_amd import mx
    case, x, dy, w = state["case"], state["x"], state["dy"], state["w"]
    if case["part"] == "forward":
        return {"y": mx.linear(x, w)}
    if case["part"] == "backward":
        dx, dw = mx.linear_backward(dy, x, w, noise=state["noise"], dw_dtype=case["dw_dtype"])
        return {"dx": dx, "dw": dw}
    y, saved = mx.linear(x, w, save=True)
    dx, dw = mx.linear_backward(dy, saved, w, noise=state["noise"], dw_dtype=case["dw_dtype"])
    return {"y": y, "dx": dx, "dw": dw}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"clip": _own_clip, "quantize": _own_quantize, "linear": _own_linear}[op](state)
    return {"clip": _plain_clip, "quantize": _plain_quantize, "linear": _plain_linear}[op](state)


def work(case):
    """Clipping reads the gradients once for the norm, and where they are
    written elsewhere writes them once.  Quantizing reads the matrix (and the
    random bytes) and writes the values read back.  A linear layer reads the
    activations, the output gradient and the weights' 4.25 bits an element,
    and writes its results."""
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "clip":
        n, e = case["K"] * sum(_numels(case)), size[case["dtype"]]
        o = 0 if case["kind"] == "inplace" else size[case["out_dtype"]]
        return {"bytes": n * (e + o), "flops": n * (2 if o == 0 else 3)}
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        sides = 2 if case["axis"] == "both" else 1
        return {"bytes": n * (size[case["dtype"]] + (1 if case["noise"] else 0) + 2 * sides),
                "flops": n * 4 * sides}
    m, k, n, e = case["m"], case["k"], case["n"], size[case["dtype"]]
    w = n * k * 17 // 32
    b, f = m * k * e, 0
    if case["part"] != "backward":
        b, f = b + w + m * n * e, f + 2 * m * n * k
    if case["part"] != "forward":
        b += m * n * (e + (1 if case["noise"] else 0)) + w + m * k * e + n * k * size[case["dw_dtype"]]
        f += 4 * m * n * k
    return {"bytes": b, "flops": f}


# --------------------------------------------------------- 64-bit reference --


def _power(e):
    """2^e in 64 bits (pow of the math library is not exact)."""
    return ((e + 1023) << 52).view(torch.float64)


def _exact_rows(x, noise):
    """The stored values in 64 bits, from the definition: the block's scale is
    2^(floor(log2 of its largest magnitude) - 2), doubled with random bytes if
    6 of it is less than that magnitude; a value goes to a neighbour on the
    grid 0, 1/2, 1, 3/2, 2, 3, 4, 6 of the scale."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    z = torch.zeros(rows, blocks * BLOCK, dtype=torch.float64, device=x.device)
    z[:, :cols] = x
    z = z.reshape(rows, blocks, BLOCK)
    top = z.abs().max(dim=2, keepdim=True).values
    e = torch.frexp(top).exponent.long() - 3
    e = torch.where(top > 0, e, -127)
    if noise is not None:
        e = torch.where(top > 6.0 * _power(e), e + 1, e)
    scale = _power(e.clamp(-127, 125))
    a = (z / scale).abs()
    width = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0)).double()
    if noise is None:
        v = torch.round(a / width) * width            # ties to the even neighbour
    else:
        r = torch.zeros(rows, blocks * BLOCK, dtype=torch.float64, device=x.device)
        r[:, :cols] = noise
        v = torch.floor(a / width + (r.reshape(rows, blocks, BLOCK) + 0.5) / 256.0) * width
    v = v.clamp(max=6.0) * scale * torch.sign(z)
    return v.reshape(rows, blocks * BLOCK)[:, :cols]


def _exact_t(x, noise):
    return _exact_rows(x.t(), None if noise is None else noise.t())


def exact(case, seed):
    if case["op"] == "quantize":
        x, noise = _quantize_inputs(case, seed)
        out = {}
        if case["axis"] != "cols":
            out["rows"] = _exact_rows(x, noise)
        if case["axis"] != "rows":
            out["cols"] = _exact_t(x, noise)
        return out
    if case["op"] == "linear":
        x, w, dy, noise = _linear_inputs(case, seed)
        out = {}
        if case["part"] != "backward":
            out["y"] = torch.mm(_exact_rows(x, None), _exact_rows(w, None).t().contiguous())
        if case["part"] != "forward":
            out["dx"] = torch.mm(_exact_rows(dy, noise), _exact_t(w, None).t().contiguous())
            out["dw"] = torch.mm(_exact_t(dy, noise), _exact_t(x, None).t().contiguous())
        return out
    g = _clip_inputs(case, seed)
    numels, (offsets, stride) = _numels(case), _flat(case)

    def scaled(parts):
        norm = math.sqrt(math.fsum(float(p.double().pow(2).sum()) for p in parts))
        f = min(1.0, case["bound"] / (norm + EPS))
        return norm, [p.double() * f for p in parts]

    def row(parts):
        flat = torch.zeros(stride, dtype=torch.float64, device="cuda")
        for p, o, n in zip(parts, offsets, numels):
            flat[o:o + n] = p
        return flat

    rows = [scaled([g[k, o:o + n] for o, n in zip(offsets, numels)]) for k in range(case["K"])]
    out = torch.stack([row(p) for _, p in rows])
    return {"norms": torch.tensor([n for n, _ in rows], dtype=torch.float64),
            "out": out[0] if case["kind"] == "pack" else out}
