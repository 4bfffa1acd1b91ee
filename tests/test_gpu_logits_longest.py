"""Rows of the most logits that are accepted, 2^31 - 1: no index passes 32 bits on the way.  Run with `-m gpu` on an MI355X.

A few logits stand so far above the others that these add less than 2^31 exp(-55) < 1e-14 to any sum: the definition over
the few alone is the reference."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import operators_reference as R
from tests.parity import say

pytestmark = pytest.mark.gpu
VOCAB = (1 << 31) - 1
FEW = np.array([0, 5, VOCAB // 2, VOCAB - 9, VOCAB - 8, VOCAB - 2, VOCAB - 1])
HIGH = 62.0 - 0.5 * np.array([3, 0, 5, 1, 6, 4, 2])
EDGE = 1 << 16                                                        # of the buffer, on both sides of the row


def row(dtype):
    import torch
    buffer = torch.empty(VOCAB + 2 * EDGE, dtype=dtype, device="cuda")
    buffer.normal_()
    buffer[:EDGE] = float("inf")                                      # would be the largest, and spoil every sum
    buffer[-EDGE:] = float("inf")
    view = buffer[EDGE:EDGE + VOCAB].view(1, VOCAB)
    view[0, torch.from_numpy(FEW).cuda()] = torch.from_numpy(HIGH).cuda().to(dtype)
    return buffer, view


def edges_untouched(buffer):
    import torch
    return bool(torch.isposinf(buffer[:EDGE]).all()) and bool(torch.isposinf(buffer[-EDGE:]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_longest_row(dtype):
    import torch
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    buffer, view = row(t)
    say(f"[longest] {VOCAB} {dtype}")
    plan = B.Distillation(1, VOCAB, t)
    idx, val, lse = plan.alloc_top_logits(5)
    plan.dgc_top_logits(view, idx, val, lse)
    torch.cuda.synchronize()
    order = np.argsort(-HIGH)[:5]
    assert np.array_equal(idx.cpu().numpy()[0], FEW[order])
    assert np.array_equal(val.cpu().numpy()[0], HIGH[order])
    few = HIGH[None, :]
    assert abs(float(lse) - R.lse(few, 1.0)[0]) <= R.lse_bound(few, 1.0)[0]
    say("[longest] distillation")
    pairs, values = np.array([[6, 1, 0, 4]]), np.array([[9.0, 8.5, 7.0, 6.5]], np.float32)
    want_loss, want_grad, loss_bound, grad_bound = R.distill(few, pairs, values, 1.0, 0.25, np.array([5]))
    loss = torch.empty(1, device="cuda")
    top_idx = torch.from_numpy(FEW[pairs].astype(np.int32)).cuda()
    label = torch.from_numpy(FEW[5:6].astype(np.int32)).cuda()
    plan.dgc_distill_loss(view, top_idx, torch.from_numpy(values).cuda(), loss, view, labels=label, hard_weight=0.25)
    torch.cuda.synchronize()
    assert abs(float(loss) - want_loss[0]) <= loss_bound[0]
    at = torch.from_numpy(FEW).cuda()
    got = view[0, at].double().cpu().numpy()
    assert np.all(np.abs(got - want_grad[0]) <= R.rounded(grad_bound[0], want_grad[0], dtype))
    view[0, at] = 0.0
    assert float(view.max()) < 1e-20 and float(view.min()) >= 0.0
    assert edges_untouched(buffer)
    say("[longest] nothing but -inf")
    view.fill_(float("-inf"))
    plan.dgc_distill_loss(view, top_idx, torch.from_numpy(values).cuda(), loss, view, labels=label, hard_weight=0.25)
    torch.cuda.synchronize()
    assert float(loss) == 0.0 and bool((view[0, ::4095] == 0).all()) and float(view.max()) == 0.0 and float(view.min()) == 0.0
    assert edges_untouched(buffer)
