"""The vocabulary loss and its gradients against their definition in 64 bits (tests/layers_reference.py), element by element.
Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import layers_reference as L
from tests.parity import capture, say
from tests.test_gpu_rotary import SENTINEL, close, dtype_of, rounded_inputs

pytestmark = pytest.mark.gpu


def matrix(rows, columns, dtype, values=None, gap=0, lead=0, beyond=SENTINEL):
    import torch
    buffer = torch.full((rows * (columns + gap) + lead + 16,), beyond, dtype=dtype_of(dtype), device="cuda")
    view = buffer[lead:lead + rows * (columns + gap)].view(rows, columns + gap)[:, :columns]
    if values is not None:
        view.copy_(torch.from_numpy(values))
    return buffer, view


def outside(buffer, view):
    keep = view.clone()
    view.fill_(SENTINEL)
    same = bool((buffer == SENTINEL).all())
    view.copy_(keep)
    return same


def check(rows, vocab, width, dtype, weighted=True, masks=False, gap=0, lead=0, seed=0, scale=1.0, plan_rows=None):
    import torch
    say(f"[vocabulary loss] {rows} x {vocab} x {width} {dtype} weighted={weighted} masks={masks} gap={gap} lead={lead}")
    rng = np.random.default_rng(seed + rows + vocab + width)
    hidden = rounded_inputs(rng.normal(size=(rows, width)), dtype)
    weight = rounded_inputs(rng.normal(size=(vocab, width)) * 2.0 * scale * width ** -0.5, dtype)
    labels = rng.integers(0, vocab, rows)
    w = (rng.random(rows) + 0.5).astype(np.float32) * np.float32(4.0 / max(rows, 1)) if weighted else None
    flags = 0
    if masks:
        labels[::3] = -1
        w[1::4] = 0.0
        hidden[1::4] = np.nan                                          # a row of weight zero counts nothing
        if rows > 5:
            labels[5], flags = vocab + 3, B.DGC_DIAG_BAD_INDEX
    plan = B.VocabularyLoss(plan_rows or rows, vocab, width, dtype_of(dtype))
    _, h = matrix(rows, width, dtype, hidden, gap, lead, float("nan"))
    _, m = matrix(vocab, width, dtype, weight, gap, lead, float("nan"))
    y = torch.from_numpy(labels.astype(np.int32)).cuda()
    row_weight = torch.from_numpy(w).cuda() if weighted else None
    loss, lse = torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
    diag = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan.dgc_vocab_loss_forward(h, m, y, loss, lse, row_weight=row_weight, diag_flags=diag)
    assert int(diag) == flags
    diag.zero_()
    dh, dm = matrix(rows, width, dtype, None, gap, lead), matrix(vocab, width, dtype, None, gap, lead)
    plan.dgc_vocab_loss_backward(h, m, y, lse, dh[1], dm[1], row_weight=row_weight, diag_flags=diag)
    assert int(diag) == flags
    want = L.vocab_loss(hidden, weight, labels, w, dtype)
    seen = np.isfinite(hidden).all(1)
    assert not seen.size or bool(torch.isnan(lse).cpu().numpy()[~seen].all())
    close(lse[torch.from_numpy(seen).cuda()], want["lse"][0][seen], want["lse"][1][seen], "f32", "lse")
    close(loss, *want["loss"], "f32", "loss")
    close(dh[1], *want["dhidden"], dtype, "dhidden")
    close(dm[1], *want["dweight"], dtype, "dweight")
    assert outside(*dh) and outside(*dm)
    # either alone, and the loss alone
    one, two = torch.full_like(dh[1], 3.0), torch.full_like(dm[1], 3.0)
    plan.dgc_vocab_loss_backward(h, m, y, lse, one, None, row_weight=row_weight)
    plan.dgc_vocab_loss_backward(h, m, y, lse, None, two, row_weight=row_weight)
    assert torch.equal(one, dh[1]) and torch.equal(two, dm[1])
    again = torch.empty_like(loss)
    plan.dgc_vocab_loss_forward(h, m, y, again, None, row_weight=row_weight)
    assert torch.equal(again, loss)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,width", [(1, 1, 1), (1, 29, 32), (3, 100, 7), (20, 500, 64), (65, 129, 63), (64, 64, 64),
                                              (128, 256, 128), (129, 257, 65), (300, 1000, 96), (257, 511, 200), (5, 20000, 40),
                                              (700, 77, 1500), (33, 8193, 72)])
def test_sizes(rows, vocab, width, dtype):
    check(rows, vocab, width, dtype)


@pytest.mark.parametrize("rows,vocab,width,dtype", [(2100, 20000, 64, "f32"), (2100, 20000, 64, "bf16"), (10, 5000, 16385, "bf16"),
                                                    (10, 5000, 16385, "f32"), (5000, 300, 64, "f16"), (3, 100001, 40, "f32")])
def test_several_pieces(rows, vocab, width, dtype):
    """More shares than are kept at a time, more of the weight than is packed at a time, and more rows than sums are kept in
    parts for."""
    check(rows, vocab, width, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap,lead", [(0, 0), (8, 8), (3, 1), (64, 0), (1, 0), (8, 1)])
def test_strides_and_masks(gap, lead, dtype):
    check(90, 333, 128, dtype, masks=True, gap=gap, lead=lead)
    check(40, 70, 50, dtype, weighted=False, gap=gap, lead=lead)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_fewer_rows_than_the_plan(dtype):
    check(7, 300, 64, dtype, plan_rows=500)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_logits(dtype):
    """Logits of some 60: exponentials that only a running maximum keeps finite."""
    check(50, 400, 64, dtype, scale=12.0)


def test_no_rows():
    import torch
    plan = B.VocabularyLoss(0, 40, 16, torch.float32)
    h, m = torch.empty(0, 16, device="cuda"), torch.ones(40, 16, device="cuda")
    y, none = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    dm = torch.full((40, 16), 5.0, device="cuda")
    plan.dgc_vocab_loss_forward(h, m, y, none, none)
    plan.dgc_vocab_loss_backward(h, m, y, none, torch.empty_like(h), dm)
    assert bool((dm == 0).all())


def test_all_rows_masked():
    import torch
    for dtype in ("f32", "bf16"):
        plan = B.VocabularyLoss(30, 100, 64, dtype_of(dtype))
        h = torch.full((30, 64), float("inf"), dtype=dtype_of(dtype), device="cuda")
        m = torch.randn(100, 64, device="cuda").to(dtype_of(dtype))
        loss, lse = torch.empty(30, device="cuda"), torch.empty(30, device="cuda")
        for labels, w in ((torch.full((30,), -1), None), (torch.zeros(30), torch.zeros(30, device="cuda"))):
            y = labels.to(torch.int32).cuda()
            dh, dm = torch.full_like(h, 2.0), torch.full_like(m, 2.0)
            plan.dgc_vocab_loss_forward(h, m, y, loss, lse, row_weight=w)
            plan.dgc_vocab_loss_backward(h, m, y, lse, dh, dm, row_weight=w)
            assert bool((loss == 0).all()) and bool((dh == 0).all()) and bool((dm == 0).all())


def test_weights_of_any_size_in_binary16():
    """Row weights far below and above what binary16 holds: shares are scaled by powers of two that are taken off again."""
    import torch
    rows, vocab, width = 100, 200, 64
    rng = np.random.default_rng(1)
    hidden = rounded_inputs(rng.normal(size=(rows, width)), "f16")
    weight = rounded_inputs(rng.normal(size=(vocab, width)) * 0.2, "f16")
    labels = rng.integers(0, vocab, rows)
    for size in (2.0 ** -20, 2.0 ** -3, 2.0 ** 10):
        w = np.full(rows, size, np.float32)
        plan = B.VocabularyLoss(rows, vocab, width, torch.float16)
        h, m = torch.from_numpy(hidden).half().cuda(), torch.from_numpy(weight).half().cuda()
        y, wt = torch.from_numpy(labels.astype(np.int32)).cuda(), torch.from_numpy(w).cuda()
        loss, lse, dh, dm = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(m)
        plan.dgc_vocab_loss_forward(h, m, y, loss, lse, row_weight=wt)
        plan.dgc_vocab_loss_backward(h, m, y, lse, dh, dm, row_weight=wt)
        want = L.vocab_loss(hidden, weight, labels, w, "f16")
        close(dh, *want["dhidden"], "f16", size)
        close(dm, *want["dweight"], "f16", size)


def test_gradients_against_differences():
    """Central differences along the gradients, in 32 bits, of steps that change the loss by some 1 %: off by the third
    derivative's share, below 1e-3 of the slope at such steps, and by the roundings of the loss, 2^-20 of it."""
    import torch
    rows, vocab, width = 60, 150, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    h, m = torch.randn(rows, width, generator=gen, device="cuda"), torch.randn(vocab, width, generator=gen, device="cuda") * 0.2
    y = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    plan = B.VocabularyLoss(rows, vocab, width, torch.float32)
    loss, lse, dh, dm = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(m)
    plan.dgc_vocab_loss_forward(h, m, y, loss, lse)
    plan.dgc_vocab_loss_backward(h, m, y, lse, dh, dm)
    total = float(loss.double().sum())
    for which, g in ((0, dh), (1, dm)):
        slope = float(g.double().norm())
        step = (g / slope) * (0.01 * total / slope)
        sums = []
        for sign in (1.0, -1.0):
            plan.dgc_vocab_loss_forward(h + sign * step if which == 0 else h, m + sign * step if which else m, y, loss)
            sums.append(float(loss.double().sum()))
        assert abs((sums[0] - sums[1]) / (2 * 0.01 * total) - 1.0) < 5e-3, which


def test_refusals_of_the_plan():
    import torch
    for a in ((-1, 10, 8), (4, 0, 8), (4, 10, 0)):
        with pytest.raises(B.DgcError):
            B.VocabularyLoss(*a, torch.float32)
    plan = B.VocabularyLoss(4, 10, 8, torch.float32)
    h, m, y, f = torch.zeros(4, 8, device="cuda"), torch.zeros(10, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    plan.dgc_vocab_loss_forward(h, m, y, f, f.clone())
    for a in ((h[:, :7], m, y, f), (h, m[:9], y, f), (h, m, y.long(), f), (h, m, y[:3], f), (h, m, y, f[:3]), (h.half(), m, y, f),
              (h, m.t().contiguous().t(), y, f), (h, m.cpu(), y, f), (torch.zeros(5, 8, device="cuda"), m, y, f)):
        with pytest.raises(B.DgcError):
            plan.dgc_vocab_loss_forward(*a)
    with pytest.raises(B.DgcError):
        plan.dgc_vocab_loss_forward(h, m, y, None, None)
    with pytest.raises(B.DgcError):
        plan.dgc_vocab_loss_backward(h, m, y, f, None, None)
    for dh, dm in ((h, None), (None, m), (m[:4], m)):
        with pytest.raises(B.DgcError):
            plan.dgc_vocab_loss_backward(h, m, y, f, dh, dm)
    small = B.VocabularyLoss(4, 10, 8, torch.float32, backward=False)
    small.dgc_vocab_loss_forward(h, m, y, f)
    if small._ws_bytes < plan._ws_bytes:
        with pytest.raises(B.DgcError):
            small.dgc_vocab_loss_backward(h, m, y, f, torch.empty_like(h), None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_on_another_stream(dtype):
    import torch
    rows, vocab, width = 80, 9000, 96
    t = dtype_of(dtype)
    gen = torch.Generator(device="cuda").manual_seed(6)
    h, m = torch.empty(rows, width, dtype=t, device="cuda"), torch.empty(vocab, width, dtype=t, device="cuda")
    y, w = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")

    class Side:
        def __init__(self):
            self.plan = B.VocabularyLoss(rows, vocab, width, t)
            self.loss, self.lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            self.dh, self.dm = torch.empty_like(h), torch.empty_like(m)

        def run(self):
            self.plan.dgc_vocab_loss_forward(h, m, y, self.loss, self.lse, row_weight=w)
            self.plan.dgc_vocab_loss_backward(h, m, y, self.lse, self.dh, self.dm, row_weight=w)

        def all(self):
            return [self.loss, self.lse, self.dh, self.dm]

    def renew():
        h.copy_(torch.randn(rows, width, generator=gen, device="cuda"))
        m.copy_(torch.randn(vocab, width, generator=gen, device="cuda") * 0.2)
        y.copy_(torch.randint(-1, vocab, (rows,), generator=gen, device="cuda"))
        w.copy_(torch.rand(rows, generator=gen, device="cuda"))

    renew()
    eager, first, second, other = Side(), Side(), Side(), Side()
    graphs = []
    for side in (first, second):
        side.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with capture(graph):
            side.run()
        graphs.append(graph)
    stream = torch.cuda.Stream()
    for _ in range(3):
        renew()
        eager.run()
        for side in (first, second, other):
            for x in side.all():
                x.fill_(float("nan"))
        for graph in graphs:
            graph.replay()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            other.run()
        stream.synchronize()
        torch.cuda.synchronize()
        for side in (first, second, other):
            for x, z in zip(side.all(), eager.all()):
                assert torch.equal(x, z)
