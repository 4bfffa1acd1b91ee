"""The example that runs rotary positions, linear attention, the vocabulary loss and the compression together.  Run with
`-m gpu` on an MI355X."""

import importlib.util
import os

import numpy as np
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("attention_lm", os.path.join(ROOT, "examples", "attention_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_trains_and_generates():
    import torch
    E = example()
    model, losses = E.train(steps=4, workers=2, vocab=300, width=64, heads=2, sequences=4, length=33, report=say)
    assert np.all(np.isfinite(losses))
    tokens = E.generate(model, torch.arange(15, device="cuda").view(3, 5), 7)
    assert tokens.shape == (3, 7) and int(tokens.min()) >= 0 and int(tokens.max()) < 300


def plain(E, model, theta, tokens, labels, sequences, length):
    """The losses of the same model in binary32 with torch alone, on the CPU."""
    import torch
    heads, dim, width = model.heads, model.dim, model.width
    w = {name: model.of(theta, name) for name in model.shapes}
    x = w["embed"][tokens]
    q, k, v = (y.view(sequences, length, heads, dim) for y in (x @ w["w_in"]).split(width, dim=1))
    f = 10000.0 ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64) / dim)
    angle = (torch.arange(length, dtype=torch.float64)[:, None] * f)[None, :, None]
    c, s = torch.cos(angle).float(), torch.sin(angle).float()
    turn = lambda y: torch.cat((y[..., :dim // 2] * c - y[..., dim // 2:] * s, y[..., :dim // 2] * s + y[..., dim // 2:] * c), -1)
    q, k = turn(q), turn(k)
    t = torch.arange(length)
    apart = (t[:, None] - t).clamp_min(0).float()
    decay = torch.exp(model.log_decay.cpu()[:, None, None] * apart) * (t[:, None] >= t)
    shares = torch.einsum("bthd,bshd->bhts", q, k) * decay
    o = torch.einsum("bhts,bshd->bthd", shares, v).reshape(-1, width) * dim ** -0.5
    z = (x + o @ w["w_o"]) @ w["w_out"].t()
    return torch.nn.functional.cross_entropy(z, labels.long(), reduction="none")


def test_gradient_of_the_whole_model():
    """The flat gradient that a pass leaves, against torch's own of the same model in binary32.  Parameters and activations are
    rounded to bfloat16 (2^-9 of each on average, a dozen of them in a row): 4 % of the gradient's norm."""
    import torch
    E = example()
    vocab, width, heads, sequences, length = 300, 64, 2, 3, 70
    model, n = E.Model(vocab, width, heads, 5), sequences * length
    gen = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    labels = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    run, grad = E.Pass(model, sequences, length), torch.empty_like(model.theta)
    run.forward(tokens)
    loss = run.losses(labels)
    run.backward(grad)
    theta = model.theta.cpu().clone().requires_grad_(True)
    want = plain(E, model, theta, tokens.cpu(), labels.cpu(), sequences, length)
    want.sum().backward()
    assert float((loss.cpu() - want.detach()).norm()) < 0.04 * float(want.detach().norm())
    for name in model.shapes:
        got, expect = model.of(grad.cpu(), name), model.of(theta.grad, name)
        assert float((got - expect).norm()) < 0.04 * float(expect.norm()), name


def test_single_steps_go_on_from_a_prompt():
    """The inputs of the output layer of tokens that come one by one, against those of the same tokens in one call.  Both are
    rounded to bfloat16 a few times, in other sums: 2 % of their norm."""
    import torch
    E = example()
    model, sequences, prompt, more = E.Model(200, 64, 2, 3), 3, 40, 5
    gen = torch.Generator(device="cuda").manual_seed(4)
    tokens = torch.randint(0, 200, (sequences, prompt + more), generator=gen, device="cuda")
    whole = E.Pass(model, sequences, prompt + more, train=False).forward(tokens.reshape(-1)).view(sequences, prompt + more, -1)
    run, step = E.Pass(model, sequences, prompt, train=False), E.Pass(model, sequences, 1, train=False)
    step.state = run.state
    run.forward(tokens[:, :prompt].reshape(-1))
    for i in range(more):
        got = step.forward(tokens[:, prompt + i], first_position=prompt + i, carry=True).float()
        want = whole[:, prompt + i].float()
        assert float((got - want).norm()) < 0.02 * float(want.norm()), i
