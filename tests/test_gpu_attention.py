"""Linear attention with a decay for each head, forward and backward, against its definition in 64 bits
(tests/layers_reference.py), element by element.  Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import layers_reference as L
from tests.parity import capture, say
from tests.test_gpu_rotary import array, close, dtype_of, outside_untouched, rounded_inputs

pytestmark = pytest.mark.gpu
DECAYS = np.array([0.0, -0.003, -0.05, -1.0, -np.inf, -20.0, -0.3], np.float32)


def inputs(n, sequences, heads, dk, dv, dtype, seed):
    rng = np.random.default_rng(seed)
    v = {name: rounded_inputs(rng.normal(size=(n, heads, d)) * size, dtype)
         for name, d, size in (("q", dk, 1.0), ("k", dk, dk ** -0.5), ("v", dv, 1.0), ("do", dv, 0.5))}
    for name in ("state0", "dstate_last"):
        v[name] = rng.normal(size=(sequences, heads, dk, dv)).astype(np.float32)
    return v


def check(lengths, heads, dk, dv, dtype, packed=True, max_length=None, carried=True, train=True, seed=0, gap=0, scale=0.7,
          layout=None, decays=None):
    import torch
    n, count = sum(lengths), len(lengths)
    total = n + gap
    layout = layout or {}
    say(f"[attention] lengths {lengths[:6]}{'...' if count > 6 else ''} heads {heads} x {dk} x {dv} {dtype} packed={packed} "
        f"carried={carried} {layout}")
    x = inputs(n, count, heads, dk, dv, dtype, seed)
    decay = np.resize(DECAYS if decays is None else np.asarray(decays, np.float32), heads)
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    plan = B.LinearAttention(count, max(lengths, default=0) if max_length is None else max_length, heads, dk, dv,
                             dtype_of(dtype), scale=scale, row_offsets=torch.from_numpy(offsets).cuda() if packed else None,
                             rows=total, backward=train)
    pad = lambda w: np.concatenate([w, np.full((gap, *w.shape[1:]), np.nan)]) if gap else w
    t = {name: array(total, heads, x[name].shape[2], dtype, pad(x[name]), **layout)[1] for name in ("q", "k", "v", "do")}
    out = {name: array(total, heads, d, dtype, **layout) for name, d in (("o", dv), ("dq", dk), ("dk", dk), ("dv", dv))}
    state0 = torch.from_numpy(x["state0"]).cuda() if carried else None
    dlast = torch.from_numpy(x["dstate_last"]).cuda() if carried else None
    last, d0 = (torch.full((count, heads, dk, dv), 7.0, device="cuda") for _ in range(2))
    rates = torch.from_numpy(decay).cuda()
    plan.dgc_linear_attention_forward(t["q"], t["k"], t["v"], rates, state0, out["o"][1], last)
    want = L.attention(x["q"], x["k"], x["v"], decay, x["state0"] if carried else None, scale, lengths,
                       x["do"] if train else None, x["dstate_last"] if carried else None, dtype)
    names = ["o"]
    if train:
        plan.dgc_linear_attention_backward(t["q"], t["k"], t["v"], rates, state0, t["do"], dlast, out["dq"][1],
                                           out["dk"][1], out["dv"][1], d0)
        names += ["dq", "dk", "dv"]
        close(d0, *want["dstate0"], "f32", "dstate0")
    close(last, *want["state_last"], "f32", "state_last")
    for name in names:
        buffer, view = out[name]
        close(view[:n], *want[name], dtype, name)
        if gap:
            view[:n] = 12345.0
        assert outside_untouched(buffer, view[:0] if gap else view), name


DIMS = [(64, 64), (128, 128), (1, 1), (5, 100), (100, 5), (50, 100), (33, 65), (256, 256), (130, 200), (16, 256), (256, 16),
        (32, 96)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dk,dv", DIMS)
def test_heads_of_many_sizes(dk, dv, dtype):
    check([70, 0, 1, 131], 2, dk, dv, dtype, seed=dk + dv, decays=[-0.003, -0.3])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("length", [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257])
def test_lengths(length, dtype):
    check([length] * 3, 2, 24, 40, dtype, packed=False, carried=length % 2 == 0, seed=length, decays=[-0.05, 0.0])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 128), (72, 66), (33, 256), (129, 130), (256, 256), (64, 65), (200, 7)])
def test_single_steps_of_many_sizes(dk, dv, dtype):
    check([1] * 5, 3, dk, dv, dtype, packed=False, seed=dk, decays=[-0.05, -2.0, 0.0])
    check([3, 0, 4, 1], 2, dk, dv, dtype, seed=dv, decays=[-0.05, -0.7], layout=dict(gap=1))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_every_decay(dtype):
    check([150, 3, 40], 7, 20, 24, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", [dict(gap=3, lead=1), dict(gap=8, lead=8), dict(by_head=True), dict(by_head=True, gap=5, lead=3)])
def test_strides(layout, dtype):
    check([100, 37], 3, 32, 64, dtype, layout=layout, decays=[-0.01])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,heads,dk,dv", [([2000], 2, 64, 64), ([3000, 5, 0, 1200], 1, 32, 32), ([1] * 300, 3, 16, 16),
                                                 ([0, 0], 2, 8, 8), ([1500], 1, 128, 128), ([700] * 4, 1, 40, 128)])
def test_long_and_many(lengths, heads, dk, dv, dtype):
    check(lengths, heads, dk, dv, dtype, decays=[-0.02, -0.001])


def test_rows_behind_the_last_sequence_stay():
    """Rows that no sequence has are neither read (they hold NaN) nor written."""
    for dtype in ("f32", "bf16"):
        check([70, 20, 65], 2, 32, 48, dtype, gap=40, decays=[-0.1])
        check([3, 1], 2, 32, 48, dtype, gap=3, decays=[-0.1])


def test_offsets_outside_the_arrays_are_left_out():
    """Offsets are read on the device: rows outside [0, rows) and beyond max_length are never touched."""
    import torch
    heads, dk, dv = 1, 16, 16
    for lo, hi, begin, end in ((-5, 10, 0, 10), (15, 1 << 40, 15, 20), (30, 40, 20, 20), (10, 5, 5, 5), (0, 20, 0, 12)):
        plan = B.LinearAttention(1, 12, heads, dk, dv, torch.float32, row_offsets=torch.tensor([lo, hi]).cuda(), rows=20)
        x = inputs(20, 1, heads, dk, dv, "f32", 3)
        t = {name: array(20, heads, 16, "f32", x[name])[1] for name in ("q", "k", "v", "do")}
        outs = {name: array(20, heads, 16, "f32") for name in ("o", "dq", "dk", "dv")}
        rates = torch.full((1,), -0.1, device="cuda")
        plan.dgc_linear_attention_forward(t["q"], t["k"], t["v"], rates, None, outs["o"][1])
        plan.dgc_linear_attention_backward(t["q"], t["k"], t["v"], rates, None, t["do"], None, outs["dq"][1], outs["dk"][1],
                                           outs["dv"][1])
        if hi - lo > 12:
            end = min(end, begin + 12)
        end = max(begin, end)
        part = {k: v[begin:end] for k, v in x.items()}
        want = L.attention(part["q"], part["k"], part["v"], np.float32([-0.1]), None, 1.0, [end - begin], part["do"])
        for name, (buffer, view) in outs.items():
            close(view[begin:end], *want[name], "f32", (lo, hi, name))
            view[begin:end] = 12345.0
            assert bool((buffer == 12345.0).all()), (lo, hi, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_then_single_tokens(dtype):
    """A prompt in one call, then token by token with the states in one array: the same as the whole in one call."""
    import torch
    heads, dk, dv, count, prompt, more = 3, 64, 80, 5, 90, 6
    x = inputs(count * (prompt + more), count, heads, dk, dv, dtype, 9)
    rates = torch.from_numpy(np.resize(DECAYS, heads)).cuda()
    want = L.attention(x["q"], x["k"], x["v"], np.resize(DECAYS, heads), None, 0.5, [prompt + more] * count,
                       dtype=dtype)
    part = lambda name, lo, hi: torch.from_numpy(
        x[name].reshape(count, prompt + more, heads, -1)[:, lo:hi].reshape(count * (hi - lo), heads, -1)).to(dtype_of(dtype)).cuda()
    of = lambda r, lo, hi: r.reshape(count, prompt + more, heads, dv)[:, lo:hi].reshape(-1, heads, dv)
    state = torch.zeros(count, heads, dk, dv, device="cuda")
    spans = [(0, prompt)] + [(prompt + i, prompt + i + 1) for i in range(more)]
    for lo, hi in spans:
        plan = B.LinearAttention(count, hi - lo, heads, dk, dv, dtype_of(dtype), scale=0.5, backward=False)
        o = torch.empty(count * (hi - lo), heads, dv, dtype=dtype_of(dtype), device="cuda")
        plan.dgc_linear_attention_forward(part("q", lo, hi), part("k", lo, hi), part("v", lo, hi), rates, state, o, state)
        close(o, of(want["o"][0], lo, hi), of(want["o"][1], lo, hi), dtype, (lo, hi))
    close(state, *want["state_last"], "f32", "state")


def test_heads_that_share_keys():
    """k and v of one head for all of them: gradients come for each head, and add up to the shared vector's."""
    import torch
    heads, n, d = 4, 77, 32
    x = inputs(n, 1, heads, d, d, "f32", 5)
    x["k"], x["v"] = np.repeat(x["k"][:, :1], heads, 1), np.repeat(x["v"][:, :1], heads, 1)
    rates = torch.full((heads,), -0.02, device="cuda")
    t = {name: array(n, heads, d, "f32", x[name])[1] for name in ("q", "do")}
    for name in ("k", "v"):
        t[name] = array(n, 1, d, "f32", x[name][:, :1])[1].expand(n, heads, d)
    plan = B.LinearAttention(1, n, heads, d, d, torch.float32)
    o, dq, dk, dv = (torch.empty(n, heads, d, device="cuda") for _ in range(4))
    plan.dgc_linear_attention_forward(t["q"], t["k"], t["v"], rates, None, o)
    plan.dgc_linear_attention_backward(t["q"], t["k"], t["v"], rates, None, t["do"], None, dq, dk, dv)
    want = L.attention(x["q"], x["k"], x["v"], np.full(heads, -0.02, np.float32), None, 1.0, [n], x["do"])
    for name, got in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        close(got, *want[name], "f32", name)
    with pytest.raises(B.DgcError):
        plan.dgc_linear_attention_forward(t["q"], t["k"], t["v"], rates, None, t["v"])


def test_large_values_in_sixteen_bits():
    """States beyond what binary16 holds, behind outputs that it does hold."""
    import torch
    n, d = 300, 32
    x = inputs(n, 1, 1, d, d, "f16", 8)
    x["k"] = rounded_inputs(np.abs(x["k"]) * 300.0, "f16")
    x["v"] = rounded_inputs(np.abs(x["v"]) * 300.0, "f16")
    x["q"] = rounded_inputs(x["q"] * 2.0 ** -12, "f16")
    t = {name: array(n, 1, d, "f16", x[name])[1] for name in ("q", "k", "v")}
    o, last = torch.empty(n, 1, d, dtype=torch.float16, device="cuda"), torch.empty(1, 1, d, d, device="cuda")
    plan = B.LinearAttention(1, n, 1, d, d, torch.float16, backward=False)
    plan.dgc_linear_attention_forward(t["q"], t["k"], t["v"], torch.zeros(1, device="cuda"), None, o, last)
    want = L.attention(x["q"], x["k"], x["v"], np.zeros(1, np.float32), None, 1.0, [n], dtype="f16")
    assert np.abs(want["state_last"][0]).max() > 1e6 and np.abs(want["o"][0]).max() < 65504
    close(o, *want["o"], "f16", "o")
    close(last, *want["state_last"], "f32", "state_last")


def test_gradients_against_differences():
    """Along a direction: the 32-bit loss sum (o . do) at two points, against the gradients in 32 bits.  With steps of h the
    difference is off by h^2 times a third derivative, none here (each input enters linearly), and by the roundings of two
    sums of n terms: 2^-24 * (sum of |terms|) * 64 / h, far below the 2 % asked for."""
    import torch
    n, heads, d = 200, 2, 32
    x = inputs(n, 1, heads, d, d, "f32", 11)
    t = {name: array(n, heads, d, "f32", x[name])[1] for name in ("q", "k", "v", "do")}
    rates = torch.tensor([-0.01, -0.1], device="cuda")
    plan = B.LinearAttention(1, n, heads, d, d, torch.float32)
    grads = {name: torch.empty(n, heads, d, device="cuda") for name in ("q", "k", "v")}
    o = torch.empty(n, heads, d, device="cuda")
    plan.dgc_linear_attention_backward(t["q"], t["k"], t["v"], rates, None, t["do"], None, *grads.values())
    for name in grads:
        step = grads[name] / grads[name].norm()
        loss = []
        for sign in (1.0, -1.0):
            moved = dict(t, **{name: t[name] + sign * step})
            plan.dgc_linear_attention_forward(moved["q"], moved["k"], moved["v"], rates, None, o)
            loss.append(float((o.double() * t["do"].double()).sum()))
        assert abs((loss[0] - loss[1]) / 2 / float(grads[name].norm()) - 1.0) < 0.02, name


def test_refusals_of_the_plan():
    import torch
    for a in ((1, 4, 0, 8, 8), (1, 4, 1, 0, 8), (1, 4, 1, 8, 257), (-1, 4, 1, 8, 8)):
        with pytest.raises(B.DgcError):
            B.LinearAttention(*a, torch.float32)
    with pytest.raises(B.DgcError):
        B.LinearAttention(1, 4, 1, 8, 8, torch.float32, rows=5)
    with pytest.raises(B.DgcError):
        B.LinearAttention(1, 4, 1, 8, 8, torch.float32, row_offsets=torch.tensor([0, 4]).cuda())
    plan = B.LinearAttention(2, 4, 2, 8, 16, torch.float32)
    k, v, rates = torch.zeros(8, 2, 8, device="cuda"), torch.zeros(8, 2, 16, device="cuda"), torch.zeros(2, device="cuda")
    state = torch.zeros(2, 2, 8, 16, device="cuda")
    good = [k, k, v, rates, state, torch.empty_like(v), state]
    plan.dgc_linear_attention_forward(*good)
    for i, bad in ((0, v), (1, k[:4]), (2, v.half()), (2, v.cpu()), (3, rates[:1]), (3, rates.double()), (4, state[:1]),
                   (4, state.transpose(2, 3)), (5, k), (5, v), (6, state.half()), (0, k.transpose(1, 2))):
        with pytest.raises(B.DgcError):
            plan.dgc_linear_attention_forward(*[bad if j == i else x for j, x in enumerate(good)])


@pytest.mark.parametrize("length", [1, 300])
def test_captured_and_on_another_stream(length):
    """Two plans' calls in two graphs, replayed with eager work between: states and gradients of every replay."""
    import torch
    heads, d, count = 2, 64, 3
    gen = torch.Generator(device="cuda").manual_seed(6)
    n = count * length
    rates = torch.tensor([-0.01, -0.2], device="cuda")
    new = lambda: torch.randn(n, heads, d, generator=gen, device="cuda")
    q, k, v, do = new().bfloat16(), new().bfloat16(), new().bfloat16(), new().bfloat16()
    state = torch.zeros(count, heads, d, d, device="cuda")

    class Side:
        def __init__(self):
            self.plan = B.LinearAttention(count, length, heads, d, d, torch.bfloat16)
            self.o, self.dq, self.dk, self.dv = (torch.empty_like(q) for _ in range(4))
            self.last, self.d0 = torch.empty_like(state), torch.empty_like(state)

        def run(self):
            self.plan.dgc_linear_attention_forward(q, k, v, rates, state, self.o, self.last)
            self.plan.dgc_linear_attention_backward(q, k, v, rates, state, do, self.last, self.dq, self.dk, self.dv, self.d0)

        def all(self):
            return [self.o, self.last, self.dq, self.dk, self.dv, self.d0]

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
    for step in range(3):
        for x in (q, k, v, do):
            x.copy_(new())
        state.normal_(generator=gen)
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
            for x, y in zip(side.all(), eager.all()):
                assert torch.equal(x, y)


@pytest.mark.parametrize("lengths", [[5000], [2049, 0, 1], [700, 3], [2, 1]])
def test_states_left_in_place(lengths):
    """state_last in state0's place and dstate0 in dstate_last's, also where sequences are cut into segments that run at the same
    time: what arrays of their own hold, to the bit."""
    import torch
    heads, d, n = 2, 64, sum(lengths)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v, do = (torch.randn(n, heads, d, generator=gen, device="cuda").bfloat16() for _ in range(4))
    rates = torch.tensor([-0.0001, -0.002], device="cuda")
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(lengths)])).cuda()
    plan = B.LinearAttention(len(lengths), max(lengths), heads, d, d, torch.bfloat16, row_offsets=offsets, rows=n)
    first, flow = (torch.randn(len(lengths), heads, d, d, generator=gen, device="cuda") for _ in range(2))
    want, got = [torch.empty_like(q) for _ in range(4)], [torch.empty_like(q) for _ in range(4)]
    last, d0 = torch.empty_like(first), torch.empty_like(first)
    plan.dgc_linear_attention_forward(q, k, v, rates, first, want[0], last)
    plan.dgc_linear_attention_backward(q, k, v, rates, first, do, flow, *want[1:], d0)
    plan.dgc_linear_attention_backward(q, k, v, rates, first, do, flow, *got[1:], flow)
    plan.dgc_linear_attention_forward(q, k, v, rates, first, got[0], first)
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and torch.equal(first, last) and torch.equal(flow, d0)


def test_same_bits_on_every_run():
    import torch
    heads, d, n = 3, 64, 5000
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v, do = (torch.randn(n, heads, d, generator=gen, device="cuda") for _ in range(4))
    rates = torch.tensor([-0.01, 0.0, -0.002], device="cuda")
    plan = B.LinearAttention(1, n, heads, d, d, torch.float32)
    seen = None
    for _ in range(4):
        out = [torch.empty_like(q) for _ in range(4)]
        plan.dgc_linear_attention_forward(q, k, v, rates, None, out[0])
        plan.dgc_linear_attention_backward(q, k, v, rates, None, do, None, *out[1:])
        assert seen is None or all(torch.equal(x, y) for x, y in zip(seen, out))
        seen = out
