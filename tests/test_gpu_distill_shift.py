"""What is added to all of a teacher's pairs does not change their softmax: where the addition is exact, not by a bit.  Run with
`-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import operators_reference as R
from tests.test_gpu_distill import logits, place

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temperature", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("vocab,k", [(200, 3), (3001, 64), (20001, 256)])
def test_pairs_that_are_all_larger(vocab, k, temperature):
    """Values are multiples of 2^-9 below 2^13, so that sums with 4096, and differences, are exact in binary32."""
    import torch
    rows = 64
    z = logits(rows, vocab, "f32", 51)
    rng = np.random.default_rng(52)
    idx = np.stack([rng.choice(vocab, k, replace=False) for _ in range(rows)]).astype(np.int32)
    val = (np.round(rng.normal(size=(rows, k)) * 1.5 * 512) / 512).astype(np.float32)
    plan = B.Distillation(rows, vocab, torch.float32)
    _, view = place(z, "f32")
    out = []
    for more in (0.0, 9.0, 1000.0, -4096.0):
        loss, grad = torch.empty(rows, device="cuda"), torch.empty_like(view)
        plan.dgc_distill_loss(view, torch.from_numpy(idx).cuda(), torch.from_numpy(val + np.float32(more)).cuda(), loss, grad,
                              temperature=temperature)
        out.append((loss, grad))
    for loss, grad in out[1:]:
        assert torch.equal(loss, out[0][0]) and torch.equal(grad, out[0][1])
    want_loss, want_grad, lb, gb = R.distill(z, idx, val, temperature, 0.0)
    assert np.all(np.abs(out[0][0].double().cpu().numpy() - want_loss) <= lb)
    assert np.all(np.abs(out[0][1].double().cpu().numpy() - want_grad) <= R.rounded(gb, want_grad, "f32"))
