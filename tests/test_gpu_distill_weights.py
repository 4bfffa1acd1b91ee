"""The ends of the hard labels' weight: a term without weight counts nothing, whatever it holds.  Run with `-m gpu` on an
MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import operators_reference as R
from tests.test_gpu_distill import SENTINEL, logits, place

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [300, 9001, 70001])
def test_pairs_without_weight_may_hold_anything(vocab, dtype):
    """hard_weight = 1 is the loss of the labels alone: also where a pair names a logit of -inf (its divergence is infinite), or
    holds an infinity or NaN, in the row's own or the teacher's sum."""
    import torch
    rows, k = 6, 5
    z = logits(rows, vocab, dtype, 41)
    z[1, 10:20] = -np.inf
    z[5, 10:20] = -np.inf
    idx = np.tile(np.arange(8, 8 + k, dtype=np.int32), (rows, 1))
    val = np.tile(np.array([9.0, 8.0, 7.0, 6.0, 5.0], np.float32), (rows, 1))
    val[2, 1], val[3, 2], val[4, 3] = np.inf, np.nan, -np.inf
    idx[5, 0], idx[5, 4] = vocab, -1
    labels = np.array([9, 25, 8, 3, -1, 40], np.int32)
    up = lambda w: torch.from_numpy(w).cuda()
    for temperature in (1.0, 2.0, 3.0):
        for top_lse in (None, np.array([9.5, 9.5, np.nan, np.inf, -np.inf, 9.5], np.float32)):
            _, view = place(z, dtype)
            grad = torch.full_like(view, SENTINEL)
            loss, flags = torch.full((rows,), SENTINEL, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
            B.Distillation(rows, vocab, view.dtype).dgc_distill_loss(
                view, up(idx), up(val), loss, grad, top_lse=None if top_lse is None else up(top_lse), labels=up(labels),
                temperature=temperature, hard_weight=1.0, diag_flags=flags)
            assert int(flags) == B.DGC_DIAG_BAD_INDEX                 # (of row 5)
            want_loss, want_grad, lb, gb = R.distill(z, np.full((rows, 0), -1), np.zeros((rows, 0)), temperature, 1.0, labels)
            assert np.all(np.abs(loss.double().cpu().numpy() - want_loss) <= lb)
            assert np.all(np.abs(grad.double().cpu().numpy() - want_grad) <= R.rounded(gb, want_grad, dtype))


def test_labels_without_weight_may_hold_anything():
    """hard_weight = 0 is the divergence alone, with labels as without, and they are not looked at."""
    import torch
    z = logits(4, 2000, "f32", 42)
    z[1, 7] = -np.inf
    idx, val = np.tile(np.arange(3, dtype=np.int32), (4, 1)), np.tile(np.array([3.0, 2.0, 1.0], np.float32), (4, 1))
    labels = torch.tensor([5, 7, 2000, -1], dtype=torch.int32, device="cuda")
    out = []
    for given in (None, labels):
        _, view = place(z, "f32")
        loss, grad, flags = torch.empty(4, device="cuda"), torch.empty_like(view), torch.zeros(1, dtype=torch.int32, device="cuda")
        B.Distillation(4, 2000, torch.float32).dgc_distill_loss(view, torch.from_numpy(idx).cuda(), torch.from_numpy(val).cuda(), loss, grad,
                                                                labels=given, temperature=2.0, diag_flags=flags)
        assert int(flags) == 0 and bool(torch.isfinite(loss).all())
        out.append((loss, grad))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
