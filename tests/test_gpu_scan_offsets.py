"""Row offsets that hold anything: rows outside the arrays are left out.  Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests.test_gpu_scan import SENTINEL, array, untouched

pytestmark = pytest.mark.gpu
LEAST, MOST = -(1 << 63), (1 << 63) - 1


@pytest.mark.parametrize("max_length", [4, 20, 300])                  # each of the kernels
@pytest.mark.parametrize("offsets", [[0, 10, LEAST, 40, MOST], [LEAST, 10, 60, LEAST, LEAST], [90, LEAST, LEAST + 1, 0, 3],
                                     [MOST, LEAST, 5, MOST, 7]])
def test_offsets_at_the_ends_of_their_type(offsets, max_length):
    """Only the rows that two offsets enclose are written, in both directions.  (Where sequences overlap, which of them a row
    is left by is not told.)"""
    import torch
    rows, d = 100, 48
    want = np.zeros(rows, bool)
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        lo, hi = min(max(lo, 0), rows), min(max(hi, 0), rows)
        want[lo:max(lo, min(hi, lo + max_length))] = True
    gate, x, dh = torch.zeros(rows, d, device="cuda"), torch.ones(rows, d, device="cuda"), torch.ones(rows, d, device="cuda")
    plan = B.GatedScan(4, max_length, d, torch.float32, row_offsets=torch.tensor(offsets, device="cuda"), rows=rows)
    out = {name: array(rows, d, "f32", d, 0) for name in ("h", "dgate", "dx")}
    states = torch.zeros(plan.state_rows + 2, d, device="cuda").fill_(SENTINEL)
    kept = states[1:-1]
    plan.dgc_gated_scan_forward(gate, x, None, out["h"][1], None, kept)
    plan.dgc_gated_scan_backward(gate, x, kept, dh, None, out["dgate"][1], out["dx"][1])
    torch.cuda.synchronize()
    assert bool((states[0] == SENTINEL).all()) and bool((states[-1] == SENTINEL).all())
    for name, (buffer, view) in out.items():
        written = (view != SENTINEL).all(1).cpu().numpy()
        if max_length <= 128:                                         # tiles may leave rows out when offsets do not ascend
            assert np.array_equal(written, want), name
        assert not np.any(written & ~want), name
        assert untouched(buffer, view, rows, d, d, 0), name
