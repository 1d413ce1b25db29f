"""A gated block trained as one would: layer norm, gated products, a 4-bit product
down and their backward passes into the rows of a replica stack, each row clipped
by its norm, the vectors updated by AGS and the matrices by Muon.  Each operator is
held against its 64-bit form at the values it was given there; the whole step replayed from a
graph gives what eager steps give.
"""
import pytest
import torch

import muon_reference
import norm_reference
import test_gpu_glu as gated

pytestmark = pytest.mark.gpu

from paper_2603_18112_amd import ags, clip, glu, muon, mx, norm  # noqa: E402

F, B = torch.float32, torch.bfloat16
ROWS, D, N, K = 150, 200, 330, 3
SHAPES = [(D,), (D,), (N, D), (N, D), (D, N)]       # norm's weight and bias, gate, up, down


class Block:
    """out = x + down(silu(gate y) * up y), y the layer norm of x."""

    def __init__(self, seed):
        gen = torch.Generator().manual_seed(seed)
        self.at, end = [], 0
        for s in SHAPES:
            self.at.append(end)
            end = -(-(end + torch.Size(s).numel()) // 8) * 8
        self.flat, self.m = torch.zeros(end).cuda(), torch.zeros(end).cuda()
        self.vw, self.vb, self.gate, self.up, self.down = self.views(self.flat)
        self.vw.fill_(1.0)
        self.vb.copy_(torch.randn(D, generator=gen) * 0.1)
        for w in (self.gate, self.up, self.down):
            w.copy_(torch.randn(w.shape, generator=gen) / w.shape[1] ** 0.5)
        self.w, self.q = glu.Weight(self.gate, self.up), mx.Weight(self.down)
        self.x = torch.randn(K, ROWS, D, generator=gen).to(B).cuda()
        self.target = torch.randn(K, ROWS, D, generator=gen).cuda()
        self.noise = torch.randint(0, 256, (K, ROWS, D), dtype=torch.uint8, generator=gen).cuda()
        self.grads = torch.zeros(K, end).cuda()
        layers = [(o, torch.Size(s).numel(), 0) for o, s in zip(self.at, SHAPES)]
        self.clipper = clip.GradClip.for_stack(layers, K, end)
        self.vectors = ags.AGS(layers[:2], self.flat, self.m, K, lr=0.05, momentum=0.9)
        self.matrices = muon.Muon([(o, *s) for o, s in zip(self.at[2:], SHAPES[2:])], self.flat, self.m, K, lr=0.02)

    def views(self, row):
        return [row[o:o + torch.Size(s).numel()].view(s) for o, s in zip(self.at, SHAPES)]

    def gradients(self, k):
        """One worker's forward and backward pass into its row; what went in and
        out of the operators."""
        gw, gb, ggate, gup, gdown = self.views(self.grads[k])
        x = self.x[k]
        y, stats = norm.layer_norm(x, self.vw, self.vb, save=True)
        h, saved = glu.gated_linear(y, self.w, save=True)
        o, kept = mx.linear(h, self.q, dtype="f32", save=True)
        dout = ((x + o - self.target[k]) / ROWS).to(B)
        dh, _ = mx.linear_backward(dout, kept, self.q, self.noise[k], dw=gdown)
        dy, _, _ = glu.gated_linear_backward(dh, y, self.w, saved=saved, dgate=ggate, dup=gup)
        dx, _, _ = norm.layer_norm_backward(dy, x, stats, self.vw, dweight=gw, dbias=gb)
        return {"y": y, "stats": stats, "h": h, "dh": dh, "dy": dy, "dx": dx}

    def step(self):
        for k in range(K):
            t = self.gradients(k)
        norms = self.clipper.clip([self.grads], 0.05)
        self.vectors.step(self.grads)
        self.matrices.step(self.grads)
        self.w.update(self.gate, self.up)
        self.q.update(self.down)
        return t["dx"], norms


def _within(got, want, tol, what):
    off = (got.double().cpu() - want).abs() - tol
    assert torch.isfinite(got).all() and (off <= 0).all(), f"{what}: {float(off.max()):.3g} beyond its bound"


def test_each_operator_at_the_values_of_a_step():
    b = Block(1)
    for k in range(K):
        t = {key: v.cpu() for key, v in b.gradients(k).items()}
        x, vw, vb = b.x[k].cpu(), b.vw.cpu(), b.vb.cpu()
        (y, mean, rstd), (e_y, e_mean, e_rstd) = norm_reference.forward(x, vw, vb, 1e-5, B)
        _within(t["y"], y, e_y, "y")
        _within(t["stats"][0], mean, e_mean, "mean")
        _within(t["stats"][1], rstd, e_rstd, "rstd")
        gate, up = b.gate.cpu().to(B), b.up.cpu().to(B)
        want = gated._results(t["y"], gate, up, t["dh"], "silu", True)
        gw, gb, ggate, gup, _ = b.views(b.grads[k])
        for got, w, what in zip((t["h"], t["dy"], ggate, gup), want, ("h", "dy", "dgate", "dup")):
            gated._within(got, *w, what)
        got = t["dx"], gw, gb
        want = norm_reference.backward(t["dy"], x, t["stats"], vw, B, F)
        for g, w, e, what in zip(got, want[0], want[1], ("dx", "dweight", "dbias")):
            _within(g, w, e, what)
    # the matrices' step on what clipping left; the vectors and the gaps are AGS's
    norms = b.clipper.clip([b.grads], 0.05)
    assert (norms > 0.05).all()
    old_w, old_m, grads = b.flat.cpu(), b.m.cpu(), b.grads.cpu()
    b.matrices.step(b.grads)
    scaled = [(o, r, c, muon.spectral_scale(r, c)) for o, (r, c) in zip(b.at[2:], SHAPES[2:])]
    want_w, want_m, tols = muon_reference.step(old_w, old_m, grads, scaled, 0.02, 0.95, 0.0, True)
    for (o, r, c, _), tol in zip(scaled, tols):
        at = slice(o, o + r * c)
        assert float((b.flat.double().cpu()[at] - want_w[at]).norm()) <= tol
        assert ((b.m.double().cpu()[at] - want_m[at]).abs() <=
                (K + 3) * 2.0 ** -24 * grads[:, at].double().abs().mean(dim=0)).all()
    first = b.at[2]
    assert torch.equal(b.flat[:first].cpu(), old_w[:first]) and torch.equal(b.m[:first].cpu(), old_m[:first])


def test_steps_replayed_from_a_graph():
    eager, other = Block(2), Block(2)
    stream = torch.cuda.Stream()
    start = [t.clone() for t in (other.flat, other.m)]
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other.step()                                     # every handle's last stream is the capturing one
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        dx, norms = other.step()
    # both from the same state
    eager.step()
    torch.cuda.synchronize()
    assert torch.equal(eager.flat, other.flat) and torch.equal(eager.m, other.m)
    assert not torch.equal(other.flat, start[0]) and not torch.equal(other.m, start[1])
    for seed in (3, 4, 5):
        x = torch.randn(K, ROWS, D, generator=torch.Generator().manual_seed(seed)).to(B).cuda()
        for b in (eager, other):
            b.x.copy_(x)
        if seed == 5:
            for b in (eager, other):
                b.vectors.set_lr(0.01)
                b.matrices.set_lr(0.004)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want_dx, want_norms = eager.step()
        torch.cuda.synchronize()
        assert torch.equal(dx, want_dx) and torch.equal(norms, want_norms)
        assert torch.equal(eager.flat, other.flat) and torch.equal(eager.m, other.m)
        assert torch.equal(eager.w.data, other.w.data) and torch.equal(eager.grads, other.grads)


def test_block_gradients_against_autograd():
    """The gradients of the norm and the gated products together against autograd's
    in 64 bits.  The operators round y, h, dy and what lies between them to bf16, half a
    step of 2^-8 each and at most five one after the other: 5 2^-8 of the norm."""
    b = Block(6)
    t = b.gradients(0)
    x, vw, vb, gate, up = (v.double().cpu().requires_grad_() for v in
                           (b.x[0], b.vw, b.vb, b.gate.to(B), b.up.to(B)))
    y = torch.nn.functional.layer_norm(x, (D,), vw, vb, 1e-5)
    h = torch.nn.functional.silu(y @ gate.t()) * (y @ up.t())
    h.backward(t["dh"].double().cpu())
    gw, gb, ggate, gup, _ = b.views(b.grads[0])
    for got, want in ((t["h"], h.detach()), (t["dx"], x.grad), (gw, vw.grad), (gb, vb.grad), (ggate, gate.grad),
                      (gup, up.grad)):
        assert float((got.double().cpu() - want).norm() / want.norm()) <= 5 * 2.0 ** -8
