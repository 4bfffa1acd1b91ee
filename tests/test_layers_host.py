"""Refusals and host arithmetic of the layers of recurrent language models with matrix states (no GPU: every check comes
before the first HIP call), and their 64-bit definitions against differences."""

import ctypes as C

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import layers_reference as L

P = 1 << 20                                                           # an address that is never followed
BAD, BIG, ODD = B.DGC_ERR_INVALID_ARG, B.DGC_ERR_CAPACITY, B.DGC_ERR_ALIGNMENT


def ref(x):
    return None if x is None else C.byref(x)


def heads(data=P, row=64, head=8):
    return B.DgcHeads(data, row, head)


def rotary_shape(**kw):
    return B.DgcRotaryShape(*dict(dict(dtype=B.DGC_BF16, flags=0, rows=10, head_dim=8, rotary_dim=8), **kw).values())


def rotary(lib, shape, **kw):
    a = dict(positions=P, frequencies=P, magnitude=1.0, count=1, heads=(C.c_int32 * 1)(8), x=heads(), out=heads(2 * P))
    a.update(kw)
    return lib.dgc_rotary(ref(shape), *a.values(), None)


def attention_shape(**kw):
    d = dict(dtype=B.DGC_F32, heads=8, key_dim=8, value_dim=8, rows=20, sequences=4, max_length=5, row_offsets=None,
             scale=1.0, reserved=0)
    return B.DgcAttention(*dict(d, **kw).values())


def forward(lib, shape, **kw):
    a = dict(q=heads(), k=heads(2 * P), v=heads(3 * P), decay=P, state0=None, o=heads(4 * P), last=None, ws=P, bytes=1 << 50)
    a.update(kw)
    return lib.dgc_linear_attention_forward(ref(shape), *a.values(), None)


def backward(lib, shape, **kw):
    a = dict(q=heads(), k=heads(2 * P), v=heads(3 * P), decay=P, state0=None, do=heads(4 * P), dlast=None, dq=heads(5 * P),
             dk=heads(6 * P), dv=heads(7 * P), d0=None, ws=P, bytes=1 << 50)
    a.update(kw)
    return lib.dgc_linear_attention_backward(ref(shape), *a.values(), None)


def vocab_shape(**kw):
    d = dict(dtype=B.DGC_F16, reserved=0, rows=20, vocab=50, width=32, hidden_stride=32, weight_stride=32)
    return B.DgcVocab(*dict(d, **kw).values())


def loss_forward(lib, shape, **kw):
    a = dict(hidden=P, weight=2 * P, labels=P, row_weight=None, loss=P, lse=P, flags=None, ws=P, bytes=1 << 50)
    a.update(kw)
    return lib.dgc_vocab_loss_forward(ref(shape), *a.values(), None)


def loss_backward(lib, shape, **kw):
    a = dict(hidden=P, weight=2 * P, labels=P, row_weight=None, lse=P, dhidden=3 * P, hs=32, dweight=4 * P, ws_=32, flags=None,
             ws=P, bytes=1 << 50)
    a.update(kw)
    return lib.dgc_vocab_loss_backward(ref(shape), *a.values(), None)


def test_struct_layout():
    assert C.sizeof(B.DgcHeads) == 24 and C.sizeof(B.DgcRotaryShape) == 24 and C.sizeof(B.DgcAttention) == 56
    assert C.sizeof(B.DgcVocab) == 48


def test_rotary_refusals(dgc_lib):
    for kw, status in ((dict(dtype=3), BAD), (dict(flags=4), BAD), (dict(rows=-1), BAD), (dict(head_dim=0), BAD),
                       (dict(head_dim=257), BAD), (dict(rotary_dim=7), BAD), (dict(rotary_dim=10), BAD),
                       (dict(rotary_dim=-2), BAD), (dict(rows=1 << 31), BIG)):
        assert rotary(dgc_lib, rotary_shape(**kw)) == status, kw
    assert rotary(dgc_lib, None) == BAD
    for kw, status in ((dict(positions=None), BAD), (dict(frequencies=None), BAD), (dict(magnitude=float("inf")), BAD),
                       (dict(magnitude=float("nan")), BAD), (dict(count=0), BAD), (dict(count=5), BAD),
                       (dict(heads=(C.c_int32 * 1)(0)), BAD), (dict(heads=(C.c_int32 * 1)(65536)), BIG), (dict(x=None), BAD),
                       (dict(out=None), BAD), (dict(x=heads(None)), BAD), (dict(out=heads(None)), BAD),
                       (dict(x=heads(row=-1)), BAD), (dict(x=heads(P + 1)), ODD), (dict(out=heads(P + 1)), ODD),
                       (dict(positions=P + 4), ODD), (dict(frequencies=P + 4), ODD), (dict(x=heads(row=1 << 60)), BIG),
                       (dict(out=heads(row=63)), BAD), (dict(out=heads(head=7)), BAD), (dict(out=heads(head=0)), BAD),
                       (dict(out=heads(row=0)), BAD), (dict(out=heads(row=8, head=79)), BAD),
                       (dict(x=heads(row=72), out=heads(row=64)), BAD)):
        assert rotary(dgc_lib, rotary_shape(), **kw) == status, kw
    empty = rotary_shape(rows=0)
    assert rotary(dgc_lib, empty, positions=None, x=heads(None), out=heads(None)) == B.DGC_OK


def test_frequencies(dgc_lib):
    out = (C.c_uint64 * 128)()
    call = lambda n, *a: dgc_lib.dgc_rotary_frequencies(n, *a, out)
    for a in ((7, 1e4, 1, 0, 1, 32), (-2, 1e4, 1, 0, 1, 32), (258, 1e4, 1, 0, 1, 32), (8, 0.5, 1, 0, 1, 32),
              (8, float("inf"), 1, 0, 1, 32), (8, float("nan"), 1, 0, 1, 32), (8, 1e4, 0.5, 0, 1, 32),
              (8, 1e4, 1, -1, 1, 32), (8, 1e4, 1, 0, 32, 32), (8, 1e4, 1, 0, -1, 32), (8, 1e4, 1, 0, 1, float("inf"))):
        assert call(*a) == BAD, a
    assert dgc_lib.dgc_rotary_frequencies(8, 1e4, 1, 0, 1, 32, None) == BAD
    assert dgc_lib.dgc_rotary_frequencies(0, 1e4, 1, 0, 1, 32, None) == B.DGC_OK
    for n, base, factor, context in ((8, 1e4, 1.0, 0.0), (256, 5e5, 8.0, 8192.0), (2, 1.0, 4.0, 0.0), (50, 1e4, 2.0, 100.0)):
        assert call(n, base, factor, context, 1.0, 32.0) == B.DGC_OK
        got = np.array([out[i] for i in range(n // 2)], np.float64) * 2.0 ** -64 * 2 * np.pi
        # a whole number of 2^-64 turns: off by half of one, 2^-65 turns of 2 pi, besides the roundings of 64 bits
        assert np.allclose(got, L.frequencies(n, base, factor, context), rtol=1e-13, atol=2 * np.pi * 2.0 ** -65)


def test_attention_refusals(dgc_lib):
    size = C.c_size_t()
    for call in (forward, backward):
        assert call(dgc_lib, None) == BAD
        for kw, status in ((dict(dtype=3), BAD), (dict(heads=0), BAD), (dict(heads=65536), BIG), (dict(key_dim=0), BAD),
                           (dict(value_dim=257), BAD), (dict(rows=21), BAD), (dict(rows=-1), BAD), (dict(sequences=-1), BAD),
                           (dict(max_length=-1), BAD), (dict(row_offsets=P + 4), ODD), (dict(scale=float("nan")), BAD),
                           (dict(reserved=1), BAD), (dict(rows=1 << 40, row_offsets=P), BIG),
                           (dict(sequences=1 << 30, rows=0, max_length=0), BIG)):
            assert call(dgc_lib, attention_shape(**kw)) == status, kw
            assert dgc_lib.dgc_linear_attention_workspace_bytes(ref(attention_shape(**kw)), 0, C.byref(size)) == status, kw
        s = attention_shape()
        for kw, status in ((dict(q=None), BAD), (dict(k=heads(None)), BAD), (dict(v=heads(P + 2)), ODD), (dict(decay=None), BAD),
                           (dict(decay=P + 1), ODD), (dict(state0=P + 2), ODD), (dict(q=heads(row=-8)), BAD),
                           (dict(k=heads(head=1 << 60)), BIG), (dict(v=heads(row=1 << 24)), BIG)):
            assert call(dgc_lib, s, **kw) == status, kw
    for name in ("o",):
        for x, status in ((None, BAD), (heads(None), BAD), (heads(row=56), BAD), (heads(head=0), BAD), (heads(P), BAD),
                          (heads(3 * P), BAD), (heads(9 * P + 1), ODD)):
            assert forward(dgc_lib, attention_shape(), **{name: x}) == status
    for name in ("dq", "dk", "dv"):
        for x, status in ((None, BAD), (heads(None), BAD), (heads(row=56), BAD), (heads(head=0), BAD), (heads(P), BAD),
                          (heads(4 * P), BAD), (heads(9 * P + 1), ODD)):
            assert backward(dgc_lib, attention_shape(), **{name: x}) == status
    assert backward(dgc_lib, attention_shape(), dq=heads(6 * P)) == BAD
    assert dgc_lib.dgc_linear_attention_workspace_bytes(ref(attention_shape()), 0, None) == BAD
    assert dgc_lib.dgc_linear_attention_workspace_bytes(ref(attention_shape()), 2, C.byref(size)) == BAD
    nothing = attention_shape(rows=0, sequences=0)
    none = heads(None)
    assert forward(dgc_lib, nothing, q=none, k=none, v=none, o=none) == B.DGC_OK


@pytest.mark.parametrize("kw", [dict(rows=100000, sequences=1, max_length=100000, heads=2), dict()])
def test_attention_workspaces(dgc_lib, kw):
    for back, call in ((0, forward), (1, backward)):
        size = C.c_size_t()
        assert dgc_lib.dgc_linear_attention_workspace_bytes(ref(attention_shape(**kw)), back, C.byref(size)) == B.DGC_OK
        if size.value:
            assert call(dgc_lib, attention_shape(**kw), ws=None) == BAD
            assert call(dgc_lib, attention_shape(**kw), ws=P + 128) == ODD
            assert call(dgc_lib, attention_shape(**kw), bytes=size.value - 1) == BIG


def test_vocab_refusals(dgc_lib):
    size = C.c_size_t()
    for back, call in ((0, loss_forward), (1, loss_backward)):
        assert call(dgc_lib, None) == BAD
        for kw, status in ((dict(dtype=-1), BAD), (dict(reserved=1), BAD), (dict(rows=-1), BAD), (dict(vocab=0), BAD),
                           (dict(width=0), BAD), (dict(hidden_stride=31), BAD), (dict(weight_stride=31), BAD),
                           (dict(rows=1 << 24), BIG), (dict(vocab=1 << 24), BIG), (dict(width=1 << 20, hidden_stride=1 << 20, weight_stride=1 << 20), BIG),
                           (dict(hidden_stride=1 << 24), BIG), (dict(weight_stride=1 << 24), BIG)):
            assert call(dgc_lib, vocab_shape(**kw)) == status, kw
            assert dgc_lib.dgc_vocab_loss_workspace_bytes(ref(vocab_shape(**kw)), back, C.byref(size)) == status, kw
        assert dgc_lib.dgc_vocab_loss_workspace_bytes(ref(vocab_shape()), back, C.byref(size)) == B.DGC_OK
        for kw, status in ((dict(hidden=None), BAD), (dict(weight=None), BAD), (dict(labels=None), BAD), (dict(hidden=P + 1), ODD),
                           (dict(weight=P + 1), ODD), (dict(labels=P + 2), ODD), (dict(row_weight=P + 2), ODD),
                           (dict(flags=P + 2), ODD), (dict(lse=P + 2), ODD), (dict(ws=None), BAD), (dict(ws=P + 128), ODD),
                           (dict(bytes=size.value - 1), BIG)):
            assert call(dgc_lib, vocab_shape(), **kw) == status, kw
    assert dgc_lib.dgc_vocab_loss_workspace_bytes(ref(vocab_shape()), 0, None) == BAD
    assert dgc_lib.dgc_vocab_loss_workspace_bytes(ref(vocab_shape()), 2, C.byref(size)) == BAD
    assert loss_forward(dgc_lib, vocab_shape(), loss=None, lse=None) == BAD
    for kw, status in ((dict(dhidden=None, dweight=None), BAD), (dict(hs=31), BAD), (dict(ws_=31), BAD), (dict(hs=1 << 24), BIG),
                       (dict(lse=None), BAD), (dict(dhidden=P), BAD), (dict(dweight=2 * P), BAD), (dict(dhidden=4 * P), BAD),
                       (dict(dhidden=3 * P + 1), ODD), (dict(dweight=4 * P + 1), ODD)):
        assert loss_backward(dgc_lib, vocab_shape(), **kw) == status, kw
    none = dict(hidden=None, weight=None, labels=None)
    assert loss_forward(dgc_lib, vocab_shape(rows=0), **none) == B.DGC_OK
    assert loss_backward(dgc_lib, vocab_shape(rows=0), dweight=None, **none) == B.DGC_OK


def test_vocab_workspaces_grow_with_the_rows(dgc_lib):
    """A plan's workspace is asked for at its most rows."""
    for dtype in (B.DGC_F32, B.DGC_F16, B.DGC_BF16):
        for vocab, width in ((29, 32), (10000, 1500), (131072, 2048), (50001, 1203)):
            for back in (0, 1):
                before = 0
                for rows in list(range(0, 300)) + [511, 512, 513, 700, 1000, 1024, 1025, 2047, 2048, 2049, 4096, 10000, 70000]:
                    size = C.c_size_t()
                    shape = vocab_shape(dtype=dtype, rows=rows, vocab=vocab, width=width, hidden_stride=width, weight_stride=width)
                    assert dgc_lib.dgc_vocab_loss_workspace_bytes(ref(shape), back, C.byref(size)) == B.DGC_OK
                    assert size.value >= before, (dtype, rows, vocab, width, back)
                    before = size.value


def test_vocab_statistics_take_what_their_tiles_leave(dgc_lib):
    """Two floats a row and tile of 256 columns where there are many of both, beside the packed arrays; and enough of them for
    the smaller tiles of fewer rows."""
    def forward_bytes(rows, vocab, width, dtype):
        size = C.c_size_t()
        shape = vocab_shape(dtype=dtype, rows=rows, vocab=vocab, width=width, hidden_stride=width, weight_stride=width)
        assert dgc_lib.dgc_vocab_loss_workspace_bytes(ref(shape), 0, C.byref(size)) == B.DGC_OK
        return size.value

    rows, vocab, width = 8192, 131072, 1024
    packed = 2 * rows * width + 2 * (1 << 26)
    assert forward_bytes(rows, vocab, width, B.DGC_BF16) <= packed + rows * (vocab // 256) * 8 + rows * 4 + 4096
    for dtype, parts in ((B.DGC_F32, 3), (B.DGC_F16, 1), (B.DGC_BF16, 1)):
        for vocab in (29, 300, 10000, 25600, 60000, 131072):
            for rows in (1, 60, 64, 128, 200, 500, 1000, 1279, 1280, 5000):
                tiles = lambda side: -(-rows // side) * -(-vocab // side)
                side = 256 if parts == 1 and tiles(256) >= 200 else 128 if tiles(128) >= 200 else 64
                packed = parts * 64 * 2 * rows + parts * 64 * 2 * -(-vocab // 256) * 256
                assert forward_bytes(rows, vocab, 64, dtype) >= packed + rows * -(-vocab // side) * 8 + rows * 4


def test_definitions_against_differences():
    """The gradients that the GPU tests compare with, against central differences of the definitions themselves."""
    rng = np.random.default_rng(4)
    n, h, dk, dv, lengths, scale = 9, 2, 3, 4, [4, 0, 5], 0.7
    x = dict(q=rng.normal(size=(n, h, dk)), k=rng.normal(size=(n, h, dk)), v=rng.normal(size=(n, h, dv)),
             state0=rng.normal(size=(3, h, dk, dv)))
    decay, do, dlast = np.log(np.array([0.9, 0.5])), rng.normal(size=(n, h, dv)), rng.normal(size=(3, h, dk, dv))

    def value():
        r = L.attention(x["q"], x["k"], x["v"], decay, x["state0"], scale, lengths)
        return (r["o"][0] * do).sum() + (r["state_last"][0] * dlast).sum()

    got = L.attention(x["q"], x["k"], x["v"], decay, x["state0"], scale, lengths, do, dlast)
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("state0", "dstate0")):
        for _ in range(6):
            at = tuple(rng.integers(0, s) for s in x[name].shape)
            keep, step = x[name][at], 1e-5
            x[name][at] = keep + step
            up = value()
            x[name][at] = keep - step
            down = value()
            x[name][at] = keep
            assert abs((up - down) / (2 * step) - got[grad][0][at]) < 1e-7, (name, at)
    rows, vocab, width = 6, 11, 5
    y = dict(hidden=rng.normal(size=(rows, width)), weight=rng.normal(size=(vocab, width)))
    labels, w = np.array([0, 10, -1, 3, 3, 12]), rng.random(rows)
    value = lambda: L.vocab_loss(y["hidden"], y["weight"], labels, w, "f32")["loss"][0].sum()
    got = L.vocab_loss(y["hidden"], y["weight"], labels, w, "f32")
    for name in y:
        for _ in range(8):
            at = tuple(rng.integers(0, s) for s in y[name].shape)
            keep, step = y[name][at], 1e-5
            y[name][at] = keep + step
            up = value()
            y[name][at] = keep - step
            down = value()
            y[name][at] = keep
            assert abs((up - down) / (2 * step) - got["d" + name][0][at]) < 1e-7, (name, at)


def test_rotary_refuses_an_array_twice(dgc_lib):
    """An array that is listed twice would be turned by two workgroups at once."""
    def call(x, out, rows=10):
        return rotary(dgc_lib, rotary_shape(rows=rows), count=2, heads=(C.c_int32 * 2)(8, 8), x=(B.DgcHeads * 2)(*x), out=(B.DgcHeads * 2)(*out))

    a, b, c = heads(P), heads(2 * P), heads(3 * P)
    assert call((a, a), (b, b)) == BAD and call((a, a), (a, a)) == BAD
    assert call((a, b), (b, c)) == BAD and call((a, b), (c, a)) == BAD and call((a, b), (a, a)) == BAD
    assert call((a, a), (b, b), rows=0) == B.DGC_OK


def test_attention_refuses_gradients_in_the_first_states(dgc_lib):
    """dq's walk reads the first states while dv's leaves dstate0."""
    assert backward(dgc_lib, attention_shape(), state0=8 * P, d0=8 * P) == BAD
    assert backward(dgc_lib, attention_shape(), state0=8 * P, dlast=8 * P, d0=8 * P) == BAD
