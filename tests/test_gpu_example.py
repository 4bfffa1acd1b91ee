"""The example runs its operators together as they would be used: top logits, distillation loss, scan backward, compression
and the sparse step.  Run with `-m gpu` on an MI355X."""

import importlib.util
import os

import numpy as np
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("distill_lm", os.path.join(ROOT, "examples", "distill_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_student_learns_from_pairs_and_sparse_gradients():
    losses = example().train(steps=30, workers=2, vocab=500, width=128, report=say)
    assert np.all(np.isfinite(losses))
    assert np.mean(losses[-5:]) < 0.8 * np.mean(losses[:5]), losses


def test_gradient_of_the_whole_model():
    """The flat gradient that a pass leaves, against torch's own of the same model in binary32.  Activations are rounded to
    bfloat16 (2^-9 of each on average, a handful of them in a row): 3 % of the gradient's norm."""
    import torch
    E = example()
    from paper_1712_01887_amd import binding as B
    vocab, width, sequences, length, k, T, hard = 300, 64, 3, 21, 16, 2.0, 0.25
    model, rows = E.Model(vocab, width, 5), 63
    gen = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    idx = torch.stack([torch.randperm(vocab, generator=gen, device="cuda")[:k] for _ in range(rows)]).to(torch.int32)
    val = torch.randn(rows, k, generator=gen, device="cuda")
    run = E.Pass(model, sequences, length)
    logits = run.forward(tokens)
    loss, grad = torch.empty(rows, device="cuda"), torch.empty_like(model.theta)
    B.Distillation(rows, vocab, torch.bfloat16).dgc_distill_loss(logits, idx, val, loss, logits, labels=labels,
                                                                 temperature=T, hard_weight=hard)
    run.backward(logits, grad)
    theta = model.theta.cpu().clone().requires_grad_(True)
    w = {name: model.of(theta, name) for name in model.shapes}
    p = w["embed"][tokens.cpu()] @ w["w_in"]
    a, x = torch.sigmoid(p[:, :width]).view(sequences, length, width), p[:, width:].view(sequences, length, width)
    h, out = torch.zeros(sequences, width), []
    for t in range(length):
        h = a[:, t] * h + (1 - a[:, t]) * x[:, t]
        out.append(h)
    z = torch.stack(out, 1).view(rows, width) @ w["w_out"]
    target = torch.softmax(val.cpu() / T, 1)
    kl = (target * (target.log() - torch.log_softmax(z / T, 1).gather(1, idx.cpu().long()))).sum(1)
    ce = torch.nn.functional.cross_entropy(z, labels.cpu().long(), reduction="none")
    want = (1 - hard) * T * T * kl + hard * ce
    want.sum().backward()
    assert torch.allclose(loss.cpu(), want.detach(), rtol=0.03)
    for name in model.shapes:
        got, expect = model.of(grad.cpu(), name), model.of(theta.grad, name)
        assert float((got - expect).norm()) < 0.03 * float(expect.norm()), name
