"""The layers of models with matrix states where a call has more threads than one launch may have, 2^32: the same results at
both sides of the seams, and nothing left out.  Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import layers_reference as L
from tests.parity import say
from tests.test_gpu_rotary import close, dtype_of

pytestmark = pytest.mark.gpu


def room(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"{gib} GiB of device memory wanted")


@pytest.mark.parametrize("length,train", [(1, False), (2, True), (5, True)])
def test_attention_of_very_many_sequences(length, train):
    """2^24 pairs of sequence and head and more, one workgroup each: step by step and by chunks."""
    import torch
    room(24)
    count, heads, dk, dv, dtype = (1 << 20) + 3, 16, 4, 8, "bf16"
    say(f"[attention] {count} sequences of {length} steps, {heads} heads of {dk} x {dv}")
    gen, n, t = torch.Generator(device="cuda").manual_seed(length), count * length, dtype_of(dtype)

    def normal(*shape, to=t):
        x = torch.empty(*shape, dtype=to, device="cuda")
        return x.normal_(generator=gen)

    q, k, v = normal(n, heads, dk), normal(n, heads, dk), normal(n, heads, dv)
    state0 = normal(count, heads, dk, dv, to=torch.float32)
    rates = torch.full((heads,), -0.1, device="cuda")
    plan = B.LinearAttention(count, length, heads, dk, dv, t, scale=0.5, backward=train)
    out = dict(o=torch.full_like(v, float("nan")), state_last=torch.full_like(state0, float("nan")))
    plan.dgc_linear_attention_forward(q, k, v, rates, state0, out["o"], out["state_last"])
    do = flow = None
    if train:
        do, flow = normal(n, heads, dv), normal(count, heads, dk, dv, to=torch.float32)
        for name, x in (("dq", q), ("dk", k), ("dv", v), ("dstate0", state0)):
            out[name] = torch.full_like(x, float("nan"))
        plan.dgc_linear_attention_backward(q, k, v, rates, state0, do, flow, out["dq"], out["dk"], out["dv"], out["dstate0"])
    # (2^24 - 1) workgroups of one, two or three walks to a launch, of 16 sequences' heads each
    seams = [(1 << 20) * i // walks for walks in (1, 2, 3) for i in range(1, walks + 1)]
    some = sorted({min(max(s + d, 0), count - 1) for s in [0, count - 1] + seams for d in (-2, -1, 0, 1, 2)})
    at = torch.tensor(some, device="cuda")
    rows = (at[:, None] * length + torch.arange(length, device="cuda")).flatten()
    host = lambda x, which: None if x is None else x[which].cpu().double().numpy()
    want = L.attention(host(q, rows), host(k, rows), host(v, rows), rates.cpu().numpy(), host(state0, at), 0.5,
                       [length] * len(some), host(do, rows), host(flow, at), dtype)
    for name, x in out.items():
        state = "state" in name
        close(x[at if state else rows], *want[name], "f32" if state else dtype, name)
        assert all(bool(torch.isfinite(part).all()) for part in x.split(1 << 18)), name


@pytest.mark.parametrize("rows,dim,heads,dtype,gib", [((1 << 25) + 5, 8, (2, 1), "f32", 8), ((1 << 31) - 1, 3, (1,), "bf16", 36)])
def test_rotary_of_very_many_rows(rows, dim, heads, dtype, gib):
    """More rows than a launch takes; 2^31 - 1 of them in two pieces each are 2^32 threads.  All heads of all rows share a vector."""
    import torch
    room(gib)
    say(f"[rotary] {rows} rows of {heads} heads of {dim} {dtype}")
    turned, t = dim // 2 * 2, dtype_of(dtype)
    rng = np.random.default_rng(1)
    one = torch.from_numpy(rng.normal(size=(len(heads), dim))).to(t).cuda()
    x = [v.expand(rows, h, dim) for v, h in zip(one, heads)]
    out = [torch.full((rows, h, dim), float("nan"), dtype=t, device="cuda") for h in heads]
    positions = torch.arange(rows, device="cuda")
    plan = B.Rotary(dim, t, half=True)
    plan.dgc_rotary(positions, x, out)
    most = (1 << 24) - 1
    some = sorted({min(max(s + d, 0), rows - 1) for s in [0, rows // 2, rows - 1, 1 << 30] + [most * i for i in (1, 2, 3, 127, 128)]
                   for d in (-2, -1, 0, 1, 2)})
    at = torch.tensor(some, device="cuda")
    for i, h in enumerate(heads):
        want = L.rotary(one[i].cpu().double().expand(len(some), h, dim).numpy(), np.array(some), L.frequencies(turned), True, 1.0, False)
        close(out[i][at], *want, dtype, i)
        assert all(bool(torch.isfinite(part).all()) for part in out[i].split(1 << 26)), i


def test_vocabulary_loss_of_very_many_logits():
    """2^39 logits: a thread for each 128 of them in the largest tiles, 2^32."""
    import torch
    room(40)
    rows, vocab, width, t = (1 << 24) - 1, 1 << 15, 2, torch.bfloat16
    say(f"[vocabulary loss] {rows} x {vocab} x {width} bf16, the loss alone")
    gen = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn(rows, width, generator=gen, device="cuda").to(t)
    m = torch.randn(vocab, width, generator=gen, device="cuda").to(t)
    y = torch.randint(-1, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    loss, lse = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    plan = B.VocabularyLoss(rows, vocab, width, t, backward=False)
    plan.dgc_vocab_loss_forward(h, m, y, loss, lse)
    at = torch.tensor([0, 1, 255, 256, rows // 2, rows - 257, rows - 2, rows - 1], device="cuda")
    want = L.vocab_loss(h[at].cpu().double().numpy(), m.cpu().double().numpy(), y[at].cpu().numpy(), None, "bf16", alone=True)
    close(lse[at], *want["lse"], "f32", "lse")
    close(loss[at], *want["loss"], "f32", "loss")
    assert bool(torch.isfinite(lse).all()) and bool(torch.isfinite(loss).all())
