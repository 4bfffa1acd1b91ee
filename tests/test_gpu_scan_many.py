"""More short sequences than a launch has workgroups of 256 threads for.  Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import operators_reference as R
from tests.parity import say
from tests.test_gpu_scan import SENTINEL, close

pytestmark = pytest.mark.gpu
LAUNCH = (1 << 32) // 256


@pytest.mark.parametrize("length", [1, 5])                            # a thread to a channel, and tiles
def test_more_sequences_than_a_launch_takes(length):
    import torch
    n = LAUNCH + 5
    say(f"[scan] {n} sequences of {length}")
    gen = torch.Generator(device="cuda").manual_seed(length)
    gate, x, dh = (torch.randn(n * length, 1, generator=gen, device="cuda") for _ in range(3))
    h0, dh_last = (torch.randn(n, 1, generator=gen, device="cuda") for _ in range(2))
    h, dgate, dx = (torch.full((n * length, 1), SENTINEL, device="cuda") for _ in range(3))
    h_last, dh0 = (torch.full((n, 1), SENTINEL, device="cuda") for _ in range(2))
    plan = B.GatedScan(n, length, 1, torch.float32)
    states = plan.alloc_states()
    plan.dgc_gated_scan_forward(gate, x, h0, h, h_last, states)
    plan.dgc_gated_scan_backward(gate, x, states, dh, dh_last, dgate, dx, dh0)
    torch.cuda.synchronize()
    for t in (h, dgate, dx, h_last, dh0):
        assert not bool((t == SENTINEL).any())
    # sequences at both ends of both launches, and some in between, as the channels of one sequence
    picked = np.unique(np.concatenate([np.arange(64), np.arange(LAUNCH - 64, n), np.random.default_rng(1).integers(0, n, 2000)]))
    at = torch.from_numpy(picked).cuda()
    steps = lambda t: t.view(n, length)[at].t().contiguous()
    once = lambda t: t.view(1, n)[:, at]
    v = {k: steps(t).cpu().numpy() for k, t in (("gate", gate), ("x", x), ("dh", dh))}
    start, end = once(h0).cpu().numpy(), once(dh_last).cpu().numpy()
    f = R.scan_forward(v["gate"], v["x"], [length], start, False)
    b = R.scan_backward(v["gate"], v["x"], [length], start, v["dh"], end, False)
    close(steps(h), f["h"], f["h_bound"], "f32", "h")
    close(once(h_last), f["last"], f["last_bound"], "f32", "h_last")
    close(steps(dx), b["dx"], b["dx_bound"], "f32", "dx")
    close(steps(dgate), b["dgate"], b["dgate_bound"], "f32", "dgate")
    close(once(dh0), b["dh0"], b["dh0_bound"], "f32", "dh0")
