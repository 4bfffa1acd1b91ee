"""A teacher's top logits and the distillation loss with its gradient, against their definitions in 64 bits
(tests/operators_reference.py).  Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import operators_reference as R
from tests.parity import capture, say

pytestmark = pytest.mark.gpu
SENTINEL = 12345.0


def dtype_of(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def place(values, dtype, stride=None, shift=0):
    """(buffer, view) of the values as rows `stride` apart in a buffer of NaN."""
    import torch
    rows, vocab = values.shape
    stride = stride or vocab
    buffer = torch.full((rows * stride + shift + 64,), float("nan"), dtype=dtype_of(dtype), device="cuda")
    view = buffer[shift:shift + rows * stride].view(rows, stride)[:, :vocab]
    view.copy_(torch.from_numpy(values))
    return buffer, view


def cast(values, dtype):
    """As they are in the element type."""
    import torch
    return torch.from_numpy(np.asarray(values, np.float32)).to(dtype_of(dtype)).double().numpy()


def logits(rows, vocab, dtype, seed, kind="plain"):
    rng = np.random.default_rng([seed, rows, vocab])
    z = rng.normal(size=(rows, vocab)) * 2.5
    low = {"f32": np.finfo(np.float32).min, "f16": np.finfo(np.float16).min, "bf16": -3.3895313892515355e38}[dtype]
    if kind == "ties":
        z = np.round(z)
    elif kind == "equal":
        z[:] = 1.25
    elif kind == "zeros":                                             # of both signs
        z = np.where(rng.random(z.shape) < 0.5, 0.0, -0.0)
    elif kind == "masked":
        z[:, rng.random(vocab) < 0.7] = -np.inf
        z[rows // 2] = -np.inf
    elif kind == "lowest":
        z[:, rng.random(vocab) < 0.95] = low
        z[rows // 2] = low
    elif kind == "few":                                               # fewer than k that can be chosen
        keep = rng.random(z.shape) < 5.0 / vocab
        z[~keep] = -np.inf
    elif kind == "rising":
        z = np.sort(z, axis=1)
    elif kind == "falling":
        z = -np.sort(-z, axis=1)
    elif kind == "crowded":                                           # the largest in one stretch of each row
        z[:, vocab // 3:vocab // 3 + 300] += 30.0
    return cast(z, dtype)


# ---------------------------------------------------------------------------
# Top logits
# ---------------------------------------------------------------------------
def check_top(z, k, dtype, stride=None, shift=0, temperature=1.0):
    import torch
    rows, vocab = z.shape
    say(f"[top] {rows} x {vocab} {dtype} k={k} stride={stride} shift={shift}")
    buffer, view = place(z, dtype, stride, shift)
    plan = B.Distillation(rows, vocab, dtype_of(dtype))
    idx, val, lse = plan.alloc_top_logits(k)
    idx.fill_(-7)
    plan.dgc_top_logits(view, idx, val, lse, temperature=temperature)
    torch.cuda.synchronize()
    want_idx, want_val = R.top(z, k)
    assert np.array_equal(idx.cpu().numpy(), want_idx)
    assert np.array_equal(val.double().cpu().numpy(), want_val)
    want, got = R.lse(z, temperature), lse.double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(np.isneginf(want), np.isneginf(got))
    assert np.array_equal(np.isnan(want) | np.isposinf(want), np.isnan(got))
    assert np.all(np.abs(got - want)[fine] <= R.lse_bound(z, temperature)[fine])
    again = plan.alloc_top_logits(k)
    plan.dgc_top_logits(view, again[0], again[1], None, temperature=temperature)
    assert torch.equal(again[0], idx) and torch.equal(again[1], val)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 29, 64, 255, 1000, 4097, 10000, 40001])
def test_top_sizes(vocab, dtype):
    for k in (1, 7, 64, 256):
        check_top(logits(5, vocab, dtype, k), k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", ["ties", "equal", "zeros", "masked", "lowest", "few", "rising", "falling", "crowded"])
@pytest.mark.parametrize("vocab", [1500, 33001])
def test_top_values(vocab, kind, dtype):
    for k in (3, 100, 256):
        check_top(logits(6, vocab, dtype, k, kind), k, dtype, temperature=2.0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("stride,shift", [(5003, 0), (5008, 1), (5003, 5), (5064, 8)])
def test_top_strides(stride, shift, dtype):
    check_top(logits(9, 5001, dtype, stride), 20, dtype, stride=stride, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_top_large_vocabularies(dtype):
    check_top(logits(3, 131072, dtype, 1), 64, dtype)
    check_top(logits(2, 131075, dtype, 2, "crowded"), 256, dtype)
    check_top(logits(2, 262145, dtype, 3), 33, dtype)
    check_top(logits(2, 300000, dtype, 4, "equal"), 33, dtype)
    check_top(logits(2, 300000, dtype, 4, "lowest"), 256, dtype)


def test_top_many_rows():
    check_top(logits(2500, 130, "bf16", 1), 40, "bf16")
    check_top(logits(700, 2000, "f32", 2), 16, "f32")


@pytest.mark.parametrize("vocab,k", [(65, 65), (128, 127), (224, 210), (256, 256), (500, 193), (511, 256)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_top_most_of_a_row(vocab, k, dtype):
    check_top(logits(300, vocab, dtype, vocab), k, dtype)
    check_top(logits(3, vocab, dtype, k, "ties"), k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_top_nan_and_infinity(dtype):
    for vocab in (500, 20000):
        z = logits(6, vocab, dtype, 3)
        z[0, 10] = np.nan
        z[1, 17] = np.inf
        z[2, ::2] = np.nan
        z[3, :] = np.nan
        z[4, 5], z[4, 6], z[4, 400] = np.inf, np.inf, -np.inf
        check_top(z, 12, dtype)


# ---------------------------------------------------------------------------
# Distillation
# ---------------------------------------------------------------------------
def teacher(z, k, seed, missing=False):
    rng = np.random.default_rng([seed, 7])
    rows, vocab = z.shape
    idx = np.full((rows, k), -1, np.int32)
    val = np.full((rows, k), -np.inf, np.float32)
    for r in range(rows):
        usable = np.flatnonzero(z[r] > -1e4)                          # a teacher masks what its student masks
        m = min(k, len(usable))
        if missing and r % 3 == 1:
            m = int(rng.integers(0, m + 1))
        idx[r, :m] = rng.choice(usable, m, replace=False)
        val[r, :m] = -np.sort(-(rng.normal(size=m) * 1.5 + 9.0))
        if missing:                                                   # absent pairs anywhere, not only behind the others
            order = rng.permutation(k)
            idx[r], val[r] = idx[r][order], val[r][order]
    return idx, val


def check_distill(z, k, dtype, stride=None, shift=0, temperature=1.0, hard=0.0, tail=False, missing=False, weighted=True,
                  in_place=False, seed=0, labels=None, dead=()):
    import torch
    rows, vocab = z.shape
    say(f"[distill] {rows} x {vocab} {dtype} k={k} T={temperature} hard={hard} tail={tail} stride={stride} shift={shift} "
        f"in place={in_place}")
    rng = np.random.default_rng([seed, 9])
    idx, val = teacher(z, k, seed, missing)
    top_lse = None
    if tail:
        shifted = np.where(idx >= 0, val.astype(np.float64) / temperature, -np.inf)
        top_lse = (R.lse(np.concatenate([shifted, np.zeros((rows, 1))], 1), 1.0) + rng.random(rows)).astype(np.float32)
    if hard > 0.0 and labels is None:
        labels = np.array([rng.choice(np.flatnonzero(z[r] > -1e4)) if (z[r] > -1e4).any() else -1 for r in range(rows)], np.int32)
        labels[rng.random(rows) < 0.2] = -1
        named = (idx[:, 0] >= 0) & (rng.random(rows) < 0.3)            # now and then the label is one of the pairs
        labels[named] = idx[named, 0]
    weight = None
    if weighted:
        weight = (rng.random(rows) * 2.0).astype(np.float32)
        weight[rng.random(rows) < 0.2] = 0.0
    for r in dead:
        weight[r] = 0.0
    _, view = place(z, dtype, stride, shift)
    buffer, grad = place(np.full_like(z, SENTINEL), dtype, stride, shift)
    if in_place:
        buffer, grad = None, view
    up = lambda w: None if w is None else torch.from_numpy(w).cuda()
    loss = torch.full((rows,), SENTINEL, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = B.Distillation(rows, vocab, dtype_of(dtype))
    kw = dict(top_lse=up(top_lse), labels=up(labels), row_weight=up(weight), temperature=temperature, hard_weight=hard,
              diag_flags=flags)
    alone = torch.empty_like(loss)
    plan.dgc_distill_loss(view, up(idx), up(val), alone, None, **kw)
    plan.dgc_distill_loss(view, up(idx), up(val), loss, grad, **kw)
    torch.cuda.synchronize()
    assert torch.equal(alone, loss) and int(flags) == 0
    want_loss, want_grad, loss_bound, grad_bound = R.distill(z, idx, val, temperature, hard, labels, top_lse, weight)
    off = np.abs(loss.double().cpu().numpy() - want_loss) - loss_bound
    assert off.max(initial=-1.0) <= 0.0, ("loss", off.max(), int(off.argmax()))
    off = np.abs(grad.double().cpu().numpy() - want_grad) - R.rounded(grad_bound, want_grad, dtype)
    assert not np.isnan(off).any()
    assert off.max(initial=-1.0) <= 0.0, ("grad", off.max(), np.unravel_index(off.argmax(), off.shape))
    if buffer is not None:                                            # nothing between the rows or around them
        inside = torch.zeros_like(buffer, dtype=torch.bool)
        inside[shift:shift + rows * (stride or vocab)].view(rows, stride or vocab)[:, :vocab] = True
        assert bool(torch.isnan(buffer[~inside]).all())
        only = torch.full_like(view, SENTINEL)                        # the gradient in a call of its own
        plan.dgc_distill_loss(view, up(idx), up(val), None, only, **kw)
        assert torch.equal(only, grad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 29, 255, 1000, 4097, 10000, 32771])
def test_distill_sizes(vocab, dtype):
    for k, hard, temperature in ((1, 0.0, 1.0), (8, 0.5, 2.0), (64, 0.1, 1.0), (256, 0.3, 4.0)):
        check_distill(logits(4, vocab, dtype, k), min(k, vocab), dtype, temperature=temperature, hard=hard, seed=vocab + k)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", ["masked", "lowest", "equal", "ties", "crowded"])
def test_distill_values(kind, dtype):
    for vocab in (700, 21001):
        z = logits(9, vocab, dtype, 2, kind)
        check_distill(z, 40, dtype, temperature=2.0, hard=0.2, missing=True, seed=vocab)
        check_distill(z, 40, dtype, temperature=1.0, hard=0.2, tail=True, missing=True, seed=vocab + 1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("stride,shift", [(5003, 0), (5008, 1), (5003, 5), (5064, 8)])
def test_distill_strides(stride, shift, dtype):
    check_distill(logits(7, 5001, dtype, stride), 16, dtype, stride=stride, shift=shift, hard=0.1, temperature=2.0)
    check_distill(logits(7, 5001, dtype, stride), 16, dtype, stride=stride, shift=shift, in_place=True, hard=0.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_large_vocabularies(dtype):
    check_distill(logits(2, 131072, dtype, 1), 64, dtype, temperature=2.0, hard=0.1, weighted=False)
    check_distill(logits(2, 131075, dtype, 2), 64, dtype, in_place=True, weighted=False)
    check_distill(logits(2, 300001, dtype, 3), 256, dtype, hard=0.5, weighted=False)
    check_distill(logits(2, 300001, dtype, 3), 256, dtype, temperature=3.0, in_place=True, hard=0.5, weighted=False)


def test_distill_many_rows():
    check_distill(logits(3000, 130, "bf16", 1), 20, "bf16", hard=0.1, temperature=2.0, missing=True)
    check_distill(logits(600, 2000, "f32", 2), 20, "f32", hard=0.1, temperature=2.0, tail=True)


def test_hard_labels_alone_and_soft_ones_alone():
    import torch
    z = logits(6, 3001, "f32", 4)
    check_distill(z, 10, "f32", hard=1.0)
    labels = np.array([5, -1, 3000, 7, -100, 0], np.int32)
    want_loss, want_grad, lb, gb = R.distill(z, np.full((6, 0), -1), np.zeros((6, 0)), 1.0, 1.0, labels)
    plan = B.Distillation(6, 3001, torch.float32)
    _, view = place(z, "f32")
    loss, grad = torch.empty(6, device="cuda"), torch.empty(6, 3001, device="cuda")
    plan.dgc_distill_loss(view, None, None, loss, grad, labels=torch.from_numpy(labels).cuda(), hard_weight=1.0)
    assert np.all(np.abs(loss.double().cpu().numpy() - want_loss) <= lb)
    assert np.all(np.abs(grad.double().cpu().numpy() - want_grad) <= R.rounded(gb, want_grad, "f32"))


def test_rows_that_do_not_count_hold_anything():
    import torch
    for vocab in (600, 30000):
        z = logits(5, vocab, "f32", 6)
        idx, val = teacher(z, 9, 6)
        _, view = place(z, "f32")
        view[1] = float("nan")
        view[2, 5] = float("inf")
        view[3] = float("-inf")
        weight = torch.tensor([1.0, 0.0, 0.0, 1.0, 1.0], device="cuda")
        val[1] = np.nan
        loss, grad = torch.empty(5, device="cuda"), torch.full((5, vocab), SENTINEL, device="cuda")
        plan = B.Distillation(5, vocab, torch.float32)
        up = lambda w: torch.from_numpy(w).cuda()
        plan.dgc_distill_loss(view, up(idx), up(val), loss, grad, row_weight=weight)
        assert bool((loss[1:4] == 0).all()) and bool((grad[1:4] == 0).all())
        assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(grad).all()) and bool((grad[0] != 0).any())
        weight.fill_(1.0)
        plan.dgc_distill_loss(view, up(idx), up(val), loss, grad, row_weight=weight)
        assert bool(torch.isnan(loss[1:3]).all()) and bool(torch.isnan(grad[1:3]).any(1).all())
        assert float(loss[3]) == 0.0 and bool(torch.isfinite(grad[[0, 3, 4]]).all())


def test_indices_outside_the_vocabulary_are_flagged():
    import torch
    z = logits(4, 1000, "f32", 8)
    idx, val = teacher(z, 6, 8)
    labels = np.array([3, 1000, 5, 6], np.int32)
    bad_idx = idx.copy()
    bad_idx[2, 4] = 1000
    bad_idx[3, 0] = 2 ** 31 - 1
    plan = B.Distillation(4, 1000, torch.float32)
    _, view = place(z, "f32")
    up = lambda w: torch.from_numpy(w).cuda()
    loss, grad = torch.empty(4, device="cuda"), torch.empty(4, 1000, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan.dgc_distill_loss(view, up(bad_idx), up(val), loss, grad, labels=up(labels), hard_weight=0.5, diag_flags=flags)
    assert int(flags) == B.DGC_DIAG_BAD_INDEX
    want_loss, want_grad, lb, gb = R.distill(z, bad_idx, val, 1.0, 0.5, labels)
    assert np.all(np.abs(loss.double().cpu().numpy() - want_loss) <= lb)
    assert np.all(np.abs(grad.double().cpu().numpy() - want_grad) <= R.rounded(gb, want_grad, "f32"))


def test_gradient_against_differences():
    """Central differences of the loss in single logits, steps of e = 2^-4: the third derivative of a log-sum-exp at
    temperature T is at most T^-3 q_j, so that the difference is off by e^2 / 6 of (1 - a) T^2 T^-3 q + a q1, plus the rounding
    of two losses over 2 e."""
    import torch
    e = 2.0 ** -4
    z = logits(3, 400, "f32", 9)
    idx, val = teacher(z, 12, 9)
    labels = np.array([4, idx[1, 3], -1], np.int32)
    T, a = 2.0, 0.25
    plan = B.Distillation(3, 400, torch.float32)
    up = lambda w: torch.from_numpy(w).cuda()
    kw = dict(labels=up(labels), temperature=T, hard_weight=a)
    _, view = place(z, "f32")
    loss, grad = torch.empty(3, device="cuda"), torch.empty(3, 400, device="cuda")
    plan.dgc_distill_loss(view, up(idx), up(val), loss, grad, **kw)
    q, q1 = np.exp(z / T - R.lse(z, T)[:, None]), np.exp(z - R.lse(z, 1.0)[:, None])
    bound = R.distill(z, idx, val, T, a, labels)[2]
    for j in {4, 9, 399, int(z[0].argmax()), int(z[1].argmax()), *idx[:, 0].tolist(), int(idx[1, 3])}:
        at = []
        for sign in (1, -1):
            w = z.copy()
            w[:, j] = (w[:, j] + sign * e).astype(np.float32)
            _, v = place(w, "f32")
            out = torch.empty(3, device="cuda")
            plan.dgc_distill_loss(v, up(idx), up(val), out, None, **kw)
            at.append((out.double().cpu().numpy(), w[:, j]))
        slope = (at[0][0] - at[1][0]) / (at[0][1] - at[1][1])
        grown = np.exp(e)                                             # q at the step's far end
        curve = e * e / 6 * grown * ((1 - a) / T * q[:, j] + a * q1[:, j])
        got = grad[:, j].double().cpu().numpy()
        assert np.all(np.abs(slope - got) <= curve + 4 * bound / (2 * e) + 1e-6 * np.abs(got)), j


def test_capture_and_another_stream():
    import torch
    for vocab in (3000, 140000):
        z = logits(6, vocab, "bf16", 10)
        idx, val = teacher(z, 30, 10)
        up = lambda w: torch.from_numpy(w).cuda()
        _, view = place(z, "bf16")
        idx, val = up(idx), up(val)
        plan = B.Distillation(6, vocab, torch.bfloat16)
        out = list(plan.alloc_top_logits(30)) + [torch.empty(6, device="cuda"), torch.empty_like(view)]

        def both():
            plan.dgc_top_logits(view, *out[:3])
            plan.dgc_distill_loss(view, idx, val, out[3], out[4])

        both()
        torch.cuda.synchronize()
        want = [o.clone() for o in out]
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for o in out:
                o.zero_()
            both()
        stream.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(out, want))
        graph = torch.cuda.CUDAGraph()
        with capture(graph):
            both()
        for _ in range(4):
            for o in out:
                o.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip(out, want))
