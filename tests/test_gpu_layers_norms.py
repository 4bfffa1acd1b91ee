"""The layers of models with matrix states, forward and backward, by the norms of whole results: element-by-element bounds
(tests/layers_reference.py) add up roundings that are all as large as they can be and all of one sign, which leaves room for a
part of an operand that was forgotten.  Here they are counted as what they are, independent: n of them are sqrt(n) of one.
Run with `-m gpu` on an MI355X.

In binary32 a step is U = 2^-23 of a partial sum (an addition inside a matrix unit need not round to the nearest).  Sums go by
matrix products of 16 terms, six of them for the parts of three times eight bits: 6 / 16 additions a term.  Beside these at
most 16 U: products of parts that are left out (three times at most), weights and exponentials, whose arguments of up to 8 or so are
rounded.  Results in 16 bits are off by what rounding the exact ones leaves, 5 % more for the sample."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import layers_reference as L
from tests.parity import say
from tests.test_gpu_attention import inputs
from tests.test_gpu_rotary import dtype_of, rounded_inputs
from tests.test_gpu_vocab_range import run

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


def near(got, value, exact, additions, dtype, also=0.0):
    """`value`: the exact result with the roundings that the operator documents, to `dtype` in the end not yet."""
    norm = np.linalg.norm
    last = rounded_inputs(value, dtype) if dtype != "f32" else value
    bound = 1.05 * norm(last - exact) + ((16.0 + np.sqrt(additions)) * U + also) * norm(exact)
    off = norm(got.detach().cpu().double().numpy() - exact)
    say(f"  off by {off / norm(exact):.2e} of the norm, bound {bound / norm(exact):.2e}")
    assert off <= bound, (off / norm(exact), bound / norm(exact))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("length,count,heads,dk,dv", [(70, 5, 3, 64, 64), (300, 2, 2, 128, 128), (2000, 1, 2, 64, 64), (200, 3, 2, 50, 100),
                                                      (260, 2, 1, 200, 40), (3, 40, 4, 64, 128)])
def test_attention(length, count, heads, dk, dv, dtype):
    """Additions: a chunk of 32 steps adds two products of 16 terms to the state, six parts each, and a row of a state is one more sum of
    dk or dv terms.  For 16-bit results shares and the state that is read are two bfloat16 parts, the first cut off: 2^-16 of
    either is left out on average."""
    import torch
    say(f"[attention] {count} x {length} x {heads} x {dk} x {dv} {dtype} by norms")
    n, t = count * length, dtype_of(dtype)
    x = inputs(n, count, heads, dk, dv, dtype, length)
    decay = np.resize(np.array([-0.003, -0.03, 0.0, -0.3], np.float32), heads)
    dev = {name: torch.from_numpy(v).to(torch.float32 if "state" in name else t).cuda() for name, v in x.items()}
    out = {name: torch.empty_like(dev[like]) for name, like in
           (("o", "v"), ("dq", "q"), ("dk", "k"), ("dv", "v"), ("state_last", "state0"), ("dstate0", "state0"))}
    plan = B.LinearAttention(count, length, heads, dk, dv, t, scale=0.7)
    rates = torch.from_numpy(decay).cuda()
    plan.dgc_linear_attention_forward(dev["q"], dev["k"], dev["v"], rates, dev["state0"], out["o"], out["state_last"])
    plan.dgc_linear_attention_backward(dev["q"], dev["k"], dev["v"], rates, dev["state0"], dev["do"], dev["dstate_last"], out["dq"],
                                       out["dk"], out["dv"], out["dstate0"])
    want = L.attention(x["q"], x["k"], x["v"], decay, x["state0"], 0.7, [length] * count, x["do"], x["dstate_last"], dtype)
    additions = 12 * -(-length // 32) + 6 * max(dk, dv) / 16 + 12
    for name, got in out.items():
        state = "state" in name
        near(got, want[name][0], want[name][0], additions, "f32" if state else dtype, 0.0 if state or dtype == "f32" else 2 * 2.0 ** -16)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,width", [(700, 77, 1500), (300, 1000, 96), (64, 10000, 128), (1000, 3000, 256)])
def test_vocabulary_loss(rows, vocab, width, dtype):
    """A share is off by its logit's error besides its own: logits of standard deviation 2, some eight of them in a sum's steps."""
    say(f"[vocabulary loss] {rows} x {vocab} x {width} {dtype} by norms")
    rng = np.random.default_rng(rows + width)
    hidden = rounded_inputs(rng.normal(size=(rows, width)), dtype)
    weight = rounded_inputs(rng.normal(size=(vocab, width)) * 2.0 * width ** -0.5, dtype)
    labels = rng.integers(0, vocab, rows)
    w = np.full(rows, np.float32(64.0 / rows))
    got = run(hidden, weight, labels, w, dtype)
    want = L.vocab_loss(hidden, weight, labels, w, dtype)
    logit = 2 * np.sqrt(6 * width / 16)
    for name in ("lse", "loss"):
        near(got[name], want[name][0], want[name][0], logit ** 2 + vocab / 16, "f32")
    z = hidden @ weight.T
    share = np.exp(z - z.max(1, keepdims=True))
    share /= share.sum(1, keepdims=True)
    share[np.arange(rows), labels] -= 1.0
    if dtype != "f32":
        share = rounded_inputs(share, dtype)
    near(got["dhidden"], w[:, None] * (share @ weight), want["dhidden"][0], 6 * vocab / 16 + logit ** 2, dtype)
    near(got["dweight"], (w[:, None] * share).T @ hidden, want["dweight"][0], 6 * rows / 16 + logit ** 2, dtype)
