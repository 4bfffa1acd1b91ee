"""The vocabulary loss over the whole range of its inputs' values, against its definition in 64 bits
(tests/layers_reference.py).  Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import layers_reference as L
from tests.parity import say
from tests.test_gpu_rotary import close, dtype_of, rounded_inputs

pytestmark = pytest.mark.gpu


def run(hidden, weight, labels, row_weight, dtype):
    """{name: tensor} of both calls."""
    import torch
    t, (rows, width), vocab = dtype_of(dtype), hidden.shape, weight.shape[0]
    plan = B.VocabularyLoss(rows, vocab, width, t)
    h, m = torch.from_numpy(hidden).to(t).cuda(), torch.from_numpy(weight).to(t).cuda()
    y = torch.from_numpy(labels.astype(np.int32)).cuda()
    w = None if row_weight is None else torch.from_numpy(row_weight.astype(np.float32)).cuda()
    out = dict(loss=torch.full((rows,), 9.0, device="cuda"), lse=torch.full((rows,), 9.0, device="cuda"),
               dhidden=torch.full_like(h, 9.0), dweight=torch.full_like(m, 9.0))
    plan.dgc_vocab_loss_forward(h, m, y, out["loss"], out["lse"], row_weight=w)
    plan.dgc_vocab_loss_backward(h, m, y, out["lse"], out["dhidden"], out["dweight"], row_weight=w)
    return out


def kind(name, dtype):
    return dtype if name.startswith("d") else "f32"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(5, 1), (20, 29), (20, 64), (70, 65), (20, 10000), (300, 10000), (1400, 10000)])
@pytest.mark.parametrize("centre", [-90.0, -110.0, -500.0, 90.0])
def test_logits_far_from_zero(centre, rows, vocab, dtype):
    """All logits of all rows about `centre`, in tiles of every size, whose last one has wavefronts without a column."""
    say(f"[vocabulary loss] {rows} x {vocab} {dtype} logits about {centre}")
    rng = np.random.default_rng(rows + vocab)
    width = 32
    hidden, weight = rng.normal(size=(rows, width)), rng.normal(size=(vocab, width)) * 2.0 * width ** -0.5
    hidden[:, 7], weight[:, 7] = 1.0, centre
    hidden, weight = rounded_inputs(hidden, dtype), rounded_inputs(weight, dtype)
    labels = rng.integers(-1, vocab, rows)
    w = np.full(rows, 1.0 / rows, np.float32)
    want = L.vocab_loss(hidden, weight, labels, w, dtype)
    for name, got in run(hidden, weight, labels, w, dtype).items():
        close(got, *want[name], kind(name, dtype), name)


def small(rows, vocab, width, dtype, seed):
    rng = np.random.default_rng(seed)
    hidden = rounded_inputs(rng.normal(size=(rows, width)), dtype)
    weight = rounded_inputs(rng.normal(size=(vocab, width)) * 2.0 * width ** -0.5, dtype)
    return hidden, weight, rng.integers(0, vocab, rows), np.full(rows, 1.0 / rows, np.float32)


HUGE = [("f16", 6e4), ("bf16", 1e12), ("bf16", -3e38), ("f32", 1e12), ("f32", 1e30), ("f32", -3e38)]


@pytest.mark.parametrize("dtype,huge", HUGE)
@pytest.mark.parametrize("rows,vocab", [(20, 500), (300, 9000)])
def test_rows_without_a_weight_hold_anything(rows, vocab, dtype, huge):
    """Large finite numbers in rows without a label or of weight zero: the others are as they are without these rows."""
    say(f"[vocabulary loss] {rows} x {vocab} {dtype} rows of {huge} that count nothing")
    hidden, weight, labels, w = small(rows, vocab, 48, dtype, 3)
    dead = np.zeros(rows, bool)
    dead[1::7] = dead[4::7] = True
    labels[1::7], w[4::7] = -1, 0.0
    hidden[dead] = rounded_inputs(np.full(1, huge), dtype)
    got = run(hidden, weight, labels, w, dtype)
    want = L.vocab_loss(hidden[~dead], weight, labels[~dead], w[~dead], dtype, alone=True)
    import torch
    for name in ("lse", "loss", "dhidden"):
        close(got[name][torch.from_numpy(~dead).cuda()], *want[name], kind(name, dtype), name)
    close(got["dweight"], *want["dweight"], dtype, "dweight")
    dead = torch.from_numpy(dead).cuda()
    assert bool((got["loss"][dead] == 0).all()) and bool((got["dhidden"][dead] == 0).all())


@pytest.mark.parametrize("dtype,huge", [("f16", 3e4), ("bf16", 1e12), ("bf16", 1e30), ("f32", 2.0 ** 20), ("f32", 1e12), ("f32", 1e30)])
@pytest.mark.parametrize("rows,vocab", [(20, 500), (300, 9000)])
def test_one_row_of_the_weight_far_larger(rows, vocab, dtype, huge):
    """A row of the weight whose logits are all far below the others': its share is zero, and nothing else changes."""
    say(f"[vocabulary loss] {rows} x {vocab} {dtype} a row of the weight of {huge}")
    hidden, weight, labels, w = small(rows, vocab, 48, dtype, 5)
    hidden[:, 7] = 1.0
    weight[11] = 0.0
    weight[11, 7] = rounded_inputs(np.full(1, -huge), dtype)[0]
    labels[labels == 11] = 12
    want = L.vocab_loss(hidden, weight, labels, w, dtype, alone=True)
    for name, got in run(hidden, weight, labels, w, dtype).items():
        close(got, *want[name], kind(name, dtype), name)


@pytest.mark.parametrize("rows,vocab", [(40, 500), (300, 9000)])
def test_rows_of_many_sizes(rows, vocab):
    """Rows of hidden, rows of the weight and row weights from 2^-40 of the largest to the largest, in 32 bits: losses and
    dhidden are as near as the row alone would be; of dweight too, each element by the rows that it is made of."""
    say(f"[vocabulary loss] {rows} x {vocab} f32 rows of many sizes")
    hidden, weight, labels, w = small(rows, vocab, 48, "f32", 7)
    rng = np.random.default_rng(8)
    hidden *= np.exp2(-rng.integers(0, 41, rows))[:, None]
    weight *= np.exp2(-rng.integers(0, 41, vocab))[:, None]
    w *= np.exp2(-rng.integers(0, 41, rows)).astype(np.float32)
    want = L.vocab_loss(hidden, weight, labels, w, "f32", alone=True)
    for name, got in run(hidden, weight, labels, w, "f32").items():
        close(got, *want[name], "f32", name)


@pytest.mark.parametrize("rows,vocab,width,dtype", [(8192, 131072, 32, "bf16"), (4096, 256000, 64, "f16"), (16384, 131072, 16, "f32")])
def test_large_plans_run_both_calls(rows, vocab, width, dtype):
    """Shapes whose forward call wants more workspace than their backward call.  lse against torch's, in 64 bits, of some rows;
    a row's gradient against the products of its shares."""
    import torch
    say(f"[vocabulary loss] {rows} x {vocab} x {width} {dtype}, one plan for both calls")
    t, gen = dtype_of(dtype), torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn(rows, width, generator=gen, device="cuda").to(t)
    m = (torch.randn(vocab, width, generator=gen, device="cuda") * 2.0 * width ** -0.5).to(t)
    y = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    plan = B.VocabularyLoss(rows, vocab, width, t)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dh, dm = torch.empty_like(h), torch.empty_like(m)
    plan.dgc_vocab_loss_forward(h, m, y, loss, lse)
    plan.dgc_vocab_loss_backward(h, m, y, lse, dh, dm)
    some = torch.tensor([0, 1, rows // 2, rows - 1])
    hidden, weight, labels = h[some].cpu().double().numpy(), m.cpu().double().numpy(), y[some].cpu().numpy()
    want = L.vocab_loss(hidden, weight, labels, None, dtype, alone=True)
    close(lse[some], *want["lse"], "f32", "lse")
    close(loss[some], *want["loss"], "f32", "loss")
    close(dh[some], *want["dhidden"], dtype, "dhidden")
    assert bool(torch.isfinite(dm).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(40, 700), (300, 20000)])
def test_row_weights_of_many_sizes(rows, vocab, dtype):
    """Weights from 1e-8 of the largest to the largest: a row's dhidden is as near as if it were alone, also in binary16, where
    most of its shares times its weight would be subnormal; either gradient alone is the same."""
    import torch
    say(f"[vocabulary loss] {rows} x {vocab} {dtype} row weights of many sizes")
    hidden, weight, labels, _ = small(rows, vocab, 64, dtype, 9)
    w = (65536.0 * 10.0 ** np.random.default_rng(2).uniform(-8.0, 0.0, rows)).astype(np.float32)
    w[3::11] = 0.0
    want = L.vocab_loss(hidden, weight, labels, w, dtype, alone=True)
    got = run(hidden, weight, labels, w, dtype)
    for name in got:
        value, bound = want[name]
        # binary16 ends at 65504: what is 65520 and more, by more than the bound, is infinite there, and what may be is not looked at
        most = 65520.0 if kind(name, dtype) == "f16" else np.inf
        beyond, inside = np.abs(value) - bound >= most, np.abs(value) + bound < most
        here = got[name].cpu().double().numpy()
        assert np.array_equal(here[beyond], np.copysign(np.inf, value[beyond])), name
        close(got[name][torch.from_numpy(inside).cuda()], value[inside], bound[inside], kind(name, dtype), name)
    t = dtype_of(dtype)
    h, m = torch.from_numpy(hidden).to(t).cuda(), torch.from_numpy(weight).to(t).cuda()
    y, row_weight = torch.from_numpy(labels.astype(np.int32)).cuda(), torch.from_numpy(w).cuda()
    plan, one, two = B.VocabularyLoss(rows, vocab, 64, t), torch.empty_like(h), torch.empty_like(m)
    plan.dgc_vocab_loss_backward(h, m, y, got["lse"], one, None, row_weight=row_weight)
    plan.dgc_vocab_loss_backward(h, m, y, got["lse"], None, two, row_weight=row_weight)
    assert torch.equal(one, got["dhidden"]) and torch.equal(two, got["dweight"])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_equal_weights_round_the_shares_themselves(dtype):
    """A mean over 20 rows, whose weight 1 / 20 has no short form in the type: both gradients are 1 / 20 of those of weight one,
    up to a rounding of the results (half a step each) and four of binary32."""
    rows, vocab = 20, 10000
    hidden, weight, labels, _ = small(rows, vocab, 96, dtype, 4)
    size = np.float32(1.0 / rows)
    one = run(hidden, weight, labels, None, dtype)
    mean = run(hidden, weight, labels, np.full(rows, size), dtype)
    for name in ("dhidden", "dweight"):
        a, b = one[name].cpu().double().numpy() * float(size), mean[name].cpu().double().numpy()
        unit = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
        tiny = 2.0 ** -25 * 1.05 if dtype == "f16" else 0.0
        assert np.all(np.abs(a - b) <= (2 * unit + unit ** 2 + 2.0 ** -21) * np.abs(a) + 2 * tiny), name


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_no_rows_leave_zeros(dtype):
    """No rows: dweight is zero, whatever the workspace holds."""
    import torch
    t = dtype_of(dtype)
    plan = B.VocabularyLoss(9, 70, 24, t)
    plan.workspace.fill_(255)                                          # NaN in every type
    h, m = torch.empty(0, 24, dtype=t, device="cuda"), torch.ones(70, 24, dtype=t, device="cuda")
    y, none = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    dm = torch.full_like(m, 5.0)
    plan.dgc_vocab_loss_backward(h, m, y, none, torch.empty_like(h), dm, row_weight=none)
    assert bool((dm == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,width", [(1, 29, 8), (90, 300, 65), (640, 9000, 130)])
def test_workspaces_that_hold_anything(rows, vocab, width, dtype):
    """Nothing is read from the workspace that the call has not written: the same bits after it was filled with NaN."""
    import torch
    t, gen = dtype_of(dtype), torch.Generator(device="cuda").manual_seed(3)
    h, m = torch.randn(rows, width, generator=gen, device="cuda").to(t), torch.randn(vocab, width, generator=gen, device="cuda").to(t)
    y = torch.randint(-1, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    w = torch.rand(rows, generator=gen, device="cuda")
    plan, seen = B.VocabularyLoss(rows, vocab, width, t), []
    for fill in (0, 255):
        plan.workspace.fill_(fill)
        loss, lse, dh, dm = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(m)
        plan.dgc_vocab_loss_forward(h, m, y, loss, lse, row_weight=w)
        plan.workspace.fill_(fill)
        plan.dgc_vocab_loss_backward(h, m, y, lse, dh, dm, row_weight=w)
        seen.append((loss, lse, dh, dm))
    assert all(torch.equal(a, b) for a, b in zip(*seen)) and all(bool(torch.isfinite(a).all()) for a in seen[1])
