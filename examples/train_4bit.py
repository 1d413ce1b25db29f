"""Training with 4-bit products, clipped replica gradients and the AGS step.

K workers of a data-parallel step train a two-layer classifier on one GPU.
Each worker multiplies in 4 bits (both layers, forward and backward, the
output gradient rounded stochastically) and writes its weight gradients into
its row of the replica stack; each row is clipped by its own norm; the AGS
step averages the rows, takes its statistics and decision and updates the
fp32 weights, which are then stored in 4 bits again.  Inputs are random
points labelled by a fixed random network, drawn afresh every step.

    python examples/train_4bit.py [--steps 100] [--workers 8] [--batch 128]

prints the loss, the largest gradient norm and the AGS decision as it goes,
then the accuracy (of 40 classes) on fresh points: one batch, and the same points one at a
time, the way a server would be asked.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_18112_amd import ags, clip, mx  # noqa: E402


class Classifier:
    """x [rows, features] -> relu(x w1' + b1) w2' + b2 with 4-bit weights.

    The parameters live in one flat fp32 buffer, laid out as `layers`
    ((offset, numel, flags) of w1, b1, w2, b2, offsets multiples of 8)."""

    def __init__(self, features, hidden, classes, generator):
        self.sizes = [(hidden, features), (hidden,), (classes, hidden), (classes,)]
        self.layers, end = [], 0
        for shape in self.sizes:
            numel = torch.Size(shape).numel()
            weight = ags.AGS_LAYER_SCALE | ags.AGS_LAYER_DECAY if len(shape) == 2 else 0
            self.layers.append((end, numel, weight))
            end = -(-(end + numel) // 8) * 8
        self.stride = end
        self.flat = torch.zeros(end, device="cuda")
        self.w1, self.b1, self.w2, self.b2 = self.views(self.flat)
        for w in (self.w1, self.w2):
            w.copy_(torch.randn(w.shape, generator=generator, device="cuda") / w.shape[1] ** 0.5)
        self.q1, self.q2 = mx.Weight(self.w1), mx.Weight(self.w2)

    def views(self, row):
        """Views of a flat row (the parameters, or a replica's gradients)."""
        return [row[o:o + n].view(shape) for (o, n, _), shape in zip(self.layers, self.sizes)]

    def store(self):
        """After a step: the new weights in 4 bits."""
        self.q1.update(self.w1)
        self.q2.update(self.w2)

    def logits(self, x):
        h = torch.relu(mx.linear(x, self.q1) + self.b1.to(x.dtype))
        return mx.linear(h, self.q2, dtype="f32") + self.b2

    def gradients(self, x, labels, row, generator):
        """Loss of one worker's batch; its gradients go into `row`."""
        g1, gb1, g2, gb2 = self.views(row)
        h, saved1 = mx.linear(x, self.q1, save=True)
        h = torch.relu(h + self.b1.to(h.dtype))
        logits, saved2 = mx.linear(h, self.q2, dtype="f32", save=True)
        logits += self.b2
        loss = F.cross_entropy(logits, labels)
        dy = torch.softmax(logits, 1)
        dy[torch.arange(len(labels), device="cuda"), labels] -= 1
        dy = (dy / len(labels)).to(x.dtype)
        gb2.copy_(dy.sum(0))
        dh, _ = mx.linear_backward(dy, saved2, self.q2, noise(dy, generator), dw=g2)
        dh = torch.where(h > 0, dh, 0)
        gb1.copy_(dh.sum(0))
        mx.linear_backward(dh, saved1, self.q1, noise(dh, generator), dw=g1, need_dx=False)
        return loss


def noise(x, generator):
    """Random bytes for stochastic rounding, one for each element."""
    return torch.randint(0, 256, x.shape, dtype=torch.uint8, device="cuda", generator=generator)


def train(steps=100, workers=8, batch=128, features=512, hidden=1024, classes=40, lr=0.2,
          max_norm=1.0, seed=0, log=lambda line: None):
    """Returns (losses, norms [steps, workers], model, a function that draws
    points and labels)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    teacher = [torch.randn(hidden, features, generator=gen, device="cuda") / features ** 0.5,
               torch.randn(classes, hidden, generator=gen, device="cuda")]

    def draw(rows):
        x = torch.randn(rows, features, generator=gen, device="cuda")
        return x.to(torch.bfloat16), (torch.relu(x @ teacher[0].t()) @ teacher[1].t()).argmax(1)

    model = Classifier(features, hidden, classes, gen)
    grads = torch.zeros(workers, model.stride, device="cuda")  # the replica stack
    opt = ags.AGS(model.layers, model.flat, torch.zeros_like(model.flat), workers, lr=lr,
                  momentum=0.9, weight_decay=1e-5, delta=0.5)
    clipper = clip.GradClip.for_stack(model.layers, workers, model.stride)
    losses, norms = [], []
    for step in range(steps):
        opt.set_lr(lr * (1 - step / steps))
        losses.append(sum(model.gradients(*draw(batch), grads[k], gen) for k in range(workers)) / workers)
        norms.append(clipper.clip([grads], max_norm))
        opt.step(grads)
        model.store()
        if step % 20 == 0 or step == steps - 1:
            st = opt.read_stats()
            log(f"step {step:4d}  loss {losses[-1].item():.4f}  largest norm {norms[-1].max().item():.3f}  "
                f"sensitive {int(st.glob['sensitive'])}")
    opt.close()
    clipper.close()
    return torch.stack(losses), torch.stack(norms), model, draw


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--batch", type=int, default=128)
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args()
    if not torch.cuda.is_available():
        sys.exit("needs a GPU")
    _, _, model, draw = train(args.steps, args.workers, args.batch, seed=args.seed,
                              log=lambda line: print(line, flush=True))
    x, labels = draw(256)
    together = model.logits(x)
    single = torch.cat([model.logits(x[i:i + 1]) for i in range(len(x))])
    for name, y in (("one batch", together), ("one at a time", single)):
        print(f"accuracy, {name}: {(y.argmax(1) == labels).float().mean().item():.3f}")


if __name__ == "__main__":
    main()
