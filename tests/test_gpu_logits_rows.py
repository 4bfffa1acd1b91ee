"""More rows than workgroups: each takes several, the next one on its way while the present one is finished, with registers and
LDS used again, whatever the rows before held.  A compute unit has at most 2048 threads, so that `MANY` rows are more than
twice what 256 of them hold of workgroups of that many threads, whatever their registers.  Every row has to come out as in
calls of few rows, where a workgroup has one, bit by bit; some also against the definition.  Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import operators_reference as R
from tests.parity import say
from tests.test_gpu_distill import SENTINEL, dtype_of

pytestmark = pytest.mark.gpu
MANY = {64: 17003, 256: 4501, 512: 2203, 1024: 1101}


def mixed_rows(rows, vocab, dtype, seed, stride):
    """Plain rows, and among them rows of -inf, of few values, of one value, with a NaN, mostly masked, and rising ones."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    buffer = torch.full((rows, stride), float("nan"), dtype=dtype_of(dtype), device="cuda")
    z = torch.randn(rows, vocab, generator=gen, device="cuda") * 2.5
    z[1::7] = float("-inf")
    z[2::7] = z[2::7].round()
    z[3::21] = 1.25
    z[4::7, vocab // 2] = float("nan")
    z[5::7] = torch.where(torch.rand(z[5::7].shape, generator=gen, device="cuda") < 0.7, torch.full_like(z[5::7], float("-inf")), z[5::7])
    z[6::21] = z[6::21].sort(dim=1).values
    view = buffer[:, :vocab]
    view.copy_(z)
    return buffer, view


def some(rows, seed, count=90):
    """The first and the last rows, and others."""
    return np.unique(np.concatenate([np.arange(10), np.arange(rows - 20, rows), np.random.default_rng(seed).integers(0, rows, count)]))


@pytest.mark.parametrize("threads,vocab,dtype,k", [(64, 130, "bf16", 40), (64, 255, "f32", 200), (256, 900, "f32", 16), (256, 2001, "f16", 64),
                                                   (256, 8003, "bf16", 100), (256, 4001, "f32", 256), (512, 9001, "bf16", 64),
                                                   (512, 40003, "f16", 33), (512, 17001, "f32", 256)])
def test_top_of_many_rows(threads, vocab, dtype, k):
    import torch
    rows, stride = MANY[threads], vocab + 3
    say(f"[top rows] {rows} x {vocab} {dtype} k={k}")
    _, z = mixed_rows(rows, vocab, dtype, vocab, stride)
    plan = B.Distillation(rows, vocab, dtype_of(dtype))
    out = plan.alloc_top_logits(k)
    plan.dgc_top_logits(z, *out, temperature=2.0)
    parts = plan.alloc_top_logits(k)
    few = 600 if threads == 512 else 256                              # with fewer, longer pieces and so other sums
    for lo in range(0, rows, few):
        lo = min(lo, rows - few)
        plan.dgc_top_logits(z[lo:lo + few], *(t[lo:lo + few] for t in parts), temperature=2.0)
    torch.cuda.synchronize()
    for a, b in zip(out, parts):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
    at = some(rows, k)
    there = torch.from_numpy(at).cuda()
    chosen = z[there].double().cpu().numpy()
    idx, val = R.top(chosen, k)
    assert np.array_equal(out[0][there].cpu().numpy(), idx) and np.array_equal(out[1][there].double().cpu().numpy(), val)
    want, got = R.lse(chosen, 2.0), out[2][there].double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(want), np.isnan(got)) and np.array_equal(np.isneginf(want), np.isneginf(got))
    assert np.all(np.abs(got[fine] - want[fine]) <= R.lse_bound(chosen, 2.0)[fine])


@pytest.mark.parametrize("temperature", [1.0, 2.0, 3.0])
@pytest.mark.parametrize("threads,vocab,dtype", [(64, 130, "bf16"), (64, 255, "f32"), (256, 900, "f32"), (256, 2001, "f16"), (256, 8003, "bf16"),
                                                 (256, 4001, "f32"), (512, 9001, "bf16"), (512, 20003, "f32"), (512, 30001, "f16"),
                                                 (512, 41001, "bf16"), (512, 57343, "f16"), (1024, 60001, "bf16"), (1024, 40001, "f32"),
                                                 (1024, 131077, "bf16"), (1024, 65539, "f32")])
def test_loss_of_many_rows(threads, vocab, dtype, temperature):
    import torch
    rows, stride, k = MANY[threads], vocab + 3, 24
    say(f"[distill rows] {rows} x {vocab} {dtype} T={temperature}")
    buffer, z = mixed_rows(rows, vocab, dtype, vocab + 1, stride)
    z[4::7, vocab // 2] = 0.0                                         # here only rows of weight zero hold a NaN
    z[5::7, 3] = 1.0                                                  # the label of these, not masked
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    weight = torch.rand(rows, generator=gen, device="cuda") + 0.5
    weight[::5] = 0.0
    z[::35] = float("nan")
    step = 7 if vocab % 7 else 11
    idx = ((torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda") + torch.arange(k, device="cuda") * step) % vocab).to(torch.int32)
    idx[3::4, k // 2:] = -1
    idx = torch.where(z.gather(1, idx.clamp_min(0).long()) > float("-inf"), idx, torch.full_like(idx, -1))
    val = torch.randn(rows, k, generator=gen, device="cuda") * 1.5 + 9.0
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    labels[5::7] = 3
    labels[6::7] = idx[6::7, 0]
    plan = B.Distillation(rows, vocab, dtype_of(dtype))
    args = lambda lo, hi: dict(labels=labels[lo:hi], row_weight=weight[lo:hi], temperature=temperature, hard_weight=0.25)
    loss, alone, parts = (torch.full((rows,), SENTINEL, device="cuda") for _ in range(3))
    grad, grad_parts = (torch.full_like(buffer, SENTINEL) for _ in range(2))
    plan.dgc_distill_loss(z, idx, val, alone, None, **args(0, rows))
    plan.dgc_distill_loss(z, idx, val, loss, grad[:, :vocab], **args(0, rows))
    few = 203
    for lo in range(0, rows, few):
        hi = min(rows, lo + few)
        plan.dgc_distill_loss(z[lo:hi], idx[lo:hi], val[lo:hi], parts[lo:hi], grad_parts[lo:hi, :vocab], **args(lo, hi))
    at = some(rows, k)
    there = torch.from_numpy(at).cuda()
    chosen = z[there].double().cpu().numpy()
    plan.dgc_distill_loss(z, idx, val, None, z, **args(0, rows))      # in the logits' place
    torch.cuda.synchronize()
    assert torch.equal(loss, alone) and torch.equal(loss, parts) and bool(torch.isfinite(loss).all())
    assert torch.equal(grad[:, :vocab], grad_parts[:, :vocab]) and torch.equal(grad[:, :vocab], z)
    assert bool((grad[:, vocab:] == torch.tensor(SENTINEL).to(grad.dtype).item()).all()) and bool(torch.isnan(buffer[:, vocab:]).all())
    assert bool((z[::5] == 0).all()) and bool((z[1::7] == 0).all())
    pick = lambda t: t[there].cpu().numpy()
    want_loss, want_grad, loss_bound, grad_bound = R.distill(chosen, pick(idx), pick(val), temperature, 0.25, pick(labels), None, pick(weight))
    assert np.all(np.abs(pick(loss).astype(np.float64) - want_loss) <= loss_bound)
    off = np.abs(z[there].double().cpu().numpy() - want_grad) - R.rounded(grad_bound, want_grad, dtype)
    assert not np.isnan(off).any() and off.max() <= 0.0, np.unravel_index(off.argmax(), off.shape)
