"""Rotary positions against their definition in 64 bits (tests/layers_reference.py), element by element.  Run with `-m gpu`
on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import layers_reference as L
from tests import operators_reference as R
from tests.parity import capture, say

pytestmark = pytest.mark.gpu
SENTINEL = 12345.0


def dtype_of(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def array(rows, heads, dim, dtype, values=None, gap=0, lead=0, by_head=False):
    """A [rows, heads, dim] tensor inside a buffer of sentinels: heads `gap` elements further apart than they are long, the
    first one `lead` elements in; with `by_head`, a head's rows behind each other."""
    import torch
    buffer = torch.full((rows * heads * (dim + gap) + lead + 16,), SENTINEL, dtype=dtype_of(dtype), device="cuda")
    inner = buffer[lead:lead + rows * heads * (dim + gap)]
    view = inner.view(heads, rows, dim + gap).transpose(0, 1) if by_head else inner.view(rows, heads, dim + gap)
    view = view[..., :dim]
    if values is not None:
        view.copy_(torch.from_numpy(values))
    return buffer, view


def rounded_inputs(values, dtype):
    import torch
    return torch.from_numpy(values).to(dtype_of(dtype)).double().numpy()


def close(got, value, bound, dtype, what):
    got = got.detach().cpu().double().numpy()
    off = np.abs(got - value) - R.rounded(bound, value, dtype)
    assert got.shape == value.shape and np.all(np.isfinite(got)), what
    assert off.size == 0 or off.max() <= 0.0, (what, off.max(), np.unravel_index(np.argmax(off), off.shape))


def outside_untouched(buffer, view):
    import torch
    keep = view.clone()
    view.fill_(SENTINEL)
    same = bool((buffer == SENTINEL).all())
    view.copy_(keep)
    return same


CASES = [  # rows, heads of each array, head_dim, rotary_dim
    (1, (1,), 2, 2), (1, (3, 1), 64, 64), (64, (16, 16), 64, 64), (7, (5, 2), 75, 50), (33, (4,), 128, 128),
    (130, (2, 2, 1, 1), 256, 256), (19, (3,), 13, 12), (19, (3,), 13, 0), (300, (1, 1), 1, 0), (257, (2,), 96, 32),
    (11, (40, 10), 80, 78), (2, (300,), 8, 8)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("rows,heads,dim,turned", CASES)
def test_heads_of_many_sizes(rows, heads, dim, turned, half, dtype):
    import torch
    say(f"[rotary] {rows} x {heads} x {dim} of which {turned} half={half} {dtype}")
    rng = np.random.default_rng(rows + dim)
    positions = rng.integers(-(1 << 20), 1 << 20, rows)
    for layout, inverse, magnitude in ((dict(), False, 1.0), (dict(gap=3, lead=1), True, 1.25), (dict(gap=8, by_head=True), False, -0.5)):
        plan = B.Rotary(dim, dtype_of(dtype), rotary_dim=turned, half=half, magnitude=magnitude)
        values = [rounded_inputs(rng.normal(size=(rows, h, dim)), dtype) for h in heads]
        x = [array(rows, h, dim, dtype, v, **layout) for h, v in zip(heads, values)]
        out = [array(rows, h, dim, dtype, **layout) for h in heads]
        plan.dgc_rotary(torch.from_numpy(positions).cuda(), [t for _, t in x], [t for _, t in out], inverse=inverse)
        for i, v in enumerate(values):
            close(out[i][1], *L.rotary(v, positions, L.frequencies(turned), half, magnitude, inverse), dtype, i)
            assert outside_untouched(*out[i])
            assert np.array_equal(x[i][1].cpu().double().numpy(), v)
        separate = [t.clone() for _, t in out]
        plan.dgc_rotary(torch.from_numpy(positions).cuda(), [t for _, t in x], [t for _, t in x], inverse=inverse)   # in place
        for i in range(len(heads)):
            assert torch.equal(x[i][1], separate[i])
            assert outside_untouched(*x[i])


@pytest.mark.parametrize("start", [0, -(1 << 31), 1 << 20, 1 << 31, (1 << 40) - 5])
def test_far_positions(start):
    """The angle of a position of 2^40 in 64-bit floats is off by 2^-12 of a radian at most: the reference takes its turns
    in whole numbers of Python's instead."""
    import math
    import torch
    n, rows = 32, 9
    positions = start + np.arange(rows)
    plan = B.Rotary(n, torch.float32, half=True)
    table = [int(x) for x in plan.frequencies.cpu().tolist()]
    x = np.zeros((rows, 1, n))
    x[..., :n // 2] = 1.0
    _, t = array(rows, 1, n, "f32", x)
    plan.dgc_rotary(torch.from_numpy(positions).cuda(), [t], [t])
    got = t.cpu().double().numpy()[:, 0]
    f = L.frequencies(n)
    for r in range(rows):
        for i in range(n // 2):
            assert abs(table[i] * 2.0 ** -64 * math.tau - f[i]) < 1e-13 * f[i] + 1e-18
            angle = (int(positions[r]) * table[i] % (1 << 64)) * 2.0 ** -64 * math.tau
            assert abs(got[r, i] - math.cos(angle)) < 11 * R.EPS and abs(got[r, i + n // 2] - math.sin(angle)) < 11 * R.EPS


@pytest.mark.parametrize("factor,context", [(4.0, 0), (8.0, 8192), (2.0, 100)])
def test_scaled_frequencies(factor, context):
    import torch
    rows, dim = 50, 64
    plan = B.Rotary(dim, torch.float32, base=5e5, factor=factor, context=context, low_turns=1.0, high_turns=4.0, magnitude=1.1)
    values = np.random.default_rng(1).normal(size=(rows, 2, dim)).astype(np.float32).astype(np.float64)
    positions = np.arange(rows) * 37
    _, x = array(rows, 2, dim, "f32", values)
    plan.dgc_rotary(torch.from_numpy(positions).cuda(), [x], [x])
    close(x, *L.rotary(values, positions, L.frequencies(dim, 5e5, factor, context, 1.0, 4.0), False, 1.1, False), "f32", "x")


def test_inverse_is_the_gradient():
    """sum of (turned x) y = sum of x (y turned back), and differences along an element."""
    import torch
    rows, h, dim = 40, 3, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, y = (torch.randn(rows, h, dim, generator=gen, device="cuda") for _ in range(2))
    positions = torch.arange(rows, device="cuda") * 1000
    plan = B.Rotary(dim, torch.float32, magnitude=1.3)
    fx, by = torch.empty_like(x), torch.empty_like(y)
    plan.dgc_rotary(positions, [x], [fx])
    plan.dgc_rotary(positions, [y], [by], inverse=True)
    # each of the two sums has rows * h * dim terms that are off by 11 EPS * 1.3 * 2 of their size, taken with every sign alike
    size = 11 * R.EPS * 1.3 * 2 * float((x.abs().double() * y.abs().double()).sum() * 2)
    assert abs(float((fx.double() * y.double()).sum() - (x.double() * by.double()).sum())) < size


def test_shared_and_strided_inputs():
    """A vector that all heads share (a stride of 0), a projection's slices, and more rows than a launch has workgroups for."""
    import torch
    rows, h, dim = 1000, 6, 32
    plan = B.Rotary(dim, torch.bfloat16, half=True)
    rng = np.random.default_rng(2)
    one = rounded_inputs(rng.normal(size=(rows, 1, dim)), "bf16")
    _, base = array(rows, 1, dim, "bf16", one)
    positions = rng.integers(0, 1 << 16, rows)
    out = torch.empty(rows, h, dim, dtype=torch.bfloat16, device="cuda")
    plan.dgc_rotary(torch.from_numpy(positions).cuda(), [base.expand(rows, h, dim)], [out])
    close(out, *L.rotary(np.repeat(one, h, 1), positions, L.frequencies(dim), True, 1.0, False), "bf16", "shared")
    with pytest.raises(B.DgcError):
        plan.dgc_rotary(torch.from_numpy(positions).cuda(), [out], [base.expand(rows, h, dim)])


def test_refusals_of_the_plan():
    import torch
    for kw in (dict(head_dim=0), dict(head_dim=257), dict(head_dim=8, rotary_dim=10), dict(head_dim=8, rotary_dim=3),
               dict(head_dim=8, base=0.0), dict(head_dim=8, device="cpu")):
        with pytest.raises(B.DgcError):
            B.Rotary(kw.pop("head_dim"), torch.float32, **kw)
    with pytest.raises(B.DgcError):
        B.Rotary(8, torch.float64)
    plan = B.Rotary(8, torch.float32)
    x = torch.zeros(4, 2, 8, device="cuda")
    at = torch.arange(4, device="cuda")
    for positions, src, dst in ((at.int(), [x], [x]), (at.cpu(), [x], [x]), (at[:3], [x], [x]), (at, [x.half()], [x]),
                                (at, [x], [x.cpu()]), (at, [x], []), (at, [], []), (at, [x] * 5, [x] * 5),
                                (at, [x[..., ::2]], [x[..., :4]]), (at, [x.transpose(1, 2)], [x])):
        with pytest.raises(B.DgcError):
            plan.dgc_rotary(positions, src, dst)
    empty = torch.zeros(0, 2, 8, device="cuda")
    plan.dgc_rotary(at[:0], [empty], [empty])


def test_captured_and_on_another_stream():
    import torch
    rows, h, dim = 70, 4, 64
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(rows, h, dim, generator=gen, device="cuda").half()
    positions = torch.arange(rows, device="cuda")
    plan = B.Rotary(dim, torch.float16)
    want, out = torch.empty_like(x), torch.zeros_like(x)
    plan.dgc_rotary(positions, [x], [want])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan.dgc_rotary(positions, [x], [out])
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with capture(graph):
        plan.dgc_rotary(positions, [x], [out])
    for step in range(3):
        positions += 1000 * step
        x.copy_(torch.randn(rows, h, dim, generator=gen, device="cuda"))
        out.zero_()
        graph.replay()
        plan.dgc_rotary(positions, [x], [want])
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,heads,key_heads,dim,turned", [(9000, 6, 2, 80, 64), (3, 6, 2, 75, 50), (70000, 1, 1, 64, 64)])
def test_slices_of_one_projection(rows, heads, key_heads, dim, turned, dtype):
    """q and k as parts of q | k | v, turned in place; rows enough that a thread takes all heads, and few."""
    import torch
    say(f"[rotary] q | k | v of {rows} x {heads} + 2 x {key_heads} x {dim} {dtype}")
    rng = np.random.default_rng(rows)
    values = rounded_inputs(rng.normal(size=(rows, heads + 2 * key_heads, dim)), dtype)
    whole = torch.from_numpy(values).to(dtype_of(dtype)).cuda()
    q, k = whole[:, :heads], whole[:, heads:heads + key_heads]
    positions = rng.integers(0, 1 << 18, rows)
    plan = B.Rotary(dim, dtype_of(dtype), rotary_dim=turned, half=True)
    plan.dgc_rotary(torch.from_numpy(positions).cuda(), [q, k], [q, k])
    want = L.rotary(values[:, :heads + key_heads], positions, L.frequencies(turned), True, 1.0, False)
    close(whole[:, :heads + key_heads], *want, dtype, "q | k")
    assert np.array_equal(whole[:, heads + key_heads:].cpu().double().numpy(), values[:, heads + key_heads:])
