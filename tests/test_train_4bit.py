"""The training example that runs the 4-bit products, the clipping of replica
gradients and the AGS step together (examples/train_4bit.py)."""
import importlib.util
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import mx_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PATH = os.path.join(ROOT, "examples", "train_4bit.py")


def _example():
    spec = importlib.util.spec_from_file_location("train_4bit", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_help_and_refusal_without_a_gpu():
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1")
    r = subprocess.run([sys.executable, PATH, "--help"], env=env, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "--workers" in r.stdout
    r = subprocess.run([sys.executable, PATH, "--steps", "1"], env=env, capture_output=True, text=True, timeout=120)
    assert r.returncode == 1 and "needs a GPU" in r.stderr


@pytest.mark.gpu
@pytest.mark.parametrize("workers,batch,features,hidden,classes", [(4, 96, 200, 330, 20), (1, 33, 64, 96, 5)])
def test_training_learns_and_stores_what_the_step_left(workers, batch, features, hidden, classes):
    # A loss below 0.8 ln(classes) is one that guessing the labels can't reach.
    losses, norms, model, draw = _example().train(60, workers, batch, features, hidden, classes, seed=3)
    assert norms.shape == (60, workers) and torch.isfinite(norms).all() and torch.isfinite(losses).all()
    assert losses[-10:].mean().item() < 0.8 * np.log(classes)
    # The 4-bit forms are those of the weights after the last step, and the
    # gaps of the flat row stay zero.
    for q, w in ((model.q1, model.w1), (model.q2, model.w2)):
        w = w.double().cpu().numpy()
        for form, x in ((q.rows, w), (q.cols, np.ascontiguousarray(w.T))):
            got = ref.unpack(form.codes.cpu().numpy(), form.scales.cpu().numpy(), *x.shape)[:, :x.shape[1]]
            assert np.array_equal(got, ref.store_rows(x)[0])
    used = torch.zeros(model.stride, dtype=torch.bool)
    for o, n, _ in model.layers:
        used[o:o + n] = True
    assert not model.flat.cpu()[~used].any()
    # Asked together or one at a time the answers differ by the order of fp32
    # sums alone, which can move a stored 4-bit input by a step: few labels flip.
    x, _ = draw(64)
    together = model.logits(x).argmax(1)
    single = torch.cat([model.logits(x[i:i + 1]) for i in range(len(x))]).argmax(1)
    assert (together == single).sum().item() >= 58


@pytest.mark.gpu
def test_each_row_is_clipped_by_its_own_norm():
    from paper_2603_18112_amd import clip
    ex = _example()
    gen = torch.Generator(device="cuda").manual_seed(1)
    model = ex.Classifier(128, 160, 24, gen)
    grads = torch.zeros(3, model.stride, device="cuda")
    for k in range(3):
        x = torch.randn(40, 128, generator=gen, device="cuda").to(torch.bfloat16) * (k + 1)
        model.gradients(x, torch.randint(0, 24, (40,), generator=gen, device="cuda"), grads[k], gen)
    before = grads.double().cpu()
    want = before.norm(dim=1)
    bound = want.sort().values[1].item() * 0.999  # two rows above it, one below
    c = clip.GradClip.for_stack(model.layers, 3, model.stride)
    got = c.clip([grads], bound)
    c.close()
    assert torch.allclose(got.double().cpu(), want, rtol=2.0 ** -23, atol=0)
    scale = torch.clamp(bound / (want + 1e-6), max=1.0)
    assert (scale < 1).sum().item() == 2
    # one rounding of the coefficient, one of the norm in it, one of the product
    assert torch.allclose(grads.double().cpu(), before * scale[:, None], rtol=4 * 2.0 ** -24, atol=0)
