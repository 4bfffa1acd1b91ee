"""Refusals and host arithmetic of the operators on logits and sequences (no GPU: every check comes before the first
HIP call), and their 64-bit definitions against independent forms."""

import ctypes as C

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import operators_reference as R

P = 1 << 20                                                           # an address that is never followed


def logits(**kw):
    d = dict(dtype=B.DGC_BF16, reserved=0, rows=4, vocab=100, row_stride=100)
    d.update(kw)
    return B.DgcLogits(**d)


def scan(**kw):
    d = dict(dtype=B.DGC_F32, flags=0, rows=20, sequences=4, max_length=5, channels=8, row_offsets=None)
    d.update(kw)
    return B.DgcScan(**d)


def top(lib, shape, **kw):
    a = dict(logits=P, temperature=1.0, k=4, idx=P, val=P, lse=P, ws=P, bytes=1 << 40)
    a.update(kw)
    return lib.dgc_top_logits(C.byref(shape) if shape else None, *a.values(), None)


def distill(lib, shape, **kw):
    a = dict(logits=P, k=4, idx=P, val=P, lse=None, labels=P, weight=None, temperature=1.0, hard=0.5, loss=P, grad=P,
             stride=100, flags=None, ws=P, bytes=1 << 40)
    a.update(kw)
    return lib.dgc_distill_loss(C.byref(shape) if shape else None, *a.values(), None)


def forward(lib, shape, **kw):
    a = dict(gate=P, gs=8, x=2 * P, xs=8, h0=None, h=3 * P, hs=8, last=None, states=None, ws=P, bytes=1 << 40)
    a.update(kw)
    return lib.dgc_gated_scan_forward(C.byref(shape) if shape else None, *a.values(), None)


def backward(lib, shape, **kw):
    a = dict(gate=P, gs=8, x=2 * P, xs=8, states=P, dh=3 * P, dhs=8, dh_last=None, dgate=4 * P, dgs=8, dx=5 * P, dxs=8,
             dh0=None, ws=P, bytes=1 << 40)
    a.update(kw)
    return lib.dgc_gated_scan_backward(C.byref(shape) if shape else None, *a.values(), None)


def test_struct_layout():
    assert C.sizeof(B.DgcLogits) == 32 and C.sizeof(B.DgcScan) == 48


def test_shapes_that_are_refused(dgc_lib):
    bad, big = B.DGC_ERR_INVALID_ARG, B.DGC_ERR_CAPACITY
    for call in (top, distill):
        assert call(dgc_lib, None) == bad
        for kw, status in ((dict(dtype=3), bad), (dict(dtype=-1), bad), (dict(reserved=1), bad), (dict(rows=-1), bad),
                           (dict(vocab=0), bad), (dict(row_stride=99), bad), (dict(rows=1 << 31), big),
                           (dict(vocab=1 << 31, row_stride=1 << 31), big), (dict(row_stride=1 << 60), big)):
            assert call(dgc_lib, logits(**kw)) == status, kw
    size = C.c_size_t()
    assert dgc_lib.dgc_logits_workspace_bytes(None, C.byref(size)) == bad
    assert dgc_lib.dgc_logits_workspace_bytes(C.byref(logits()), None) == bad
    assert dgc_lib.dgc_logits_workspace_bytes(C.byref(logits()), C.byref(size)) == B.DGC_OK
    for call in (forward, backward):
        assert call(dgc_lib, None) == bad
        for kw, status in ((dict(dtype=3), bad), (dict(flags=2), bad), (dict(rows=-1), bad), (dict(sequences=-1), bad),
                           (dict(max_length=-1), bad), (dict(channels=0), bad), (dict(rows=21), bad),
                           (dict(row_offsets=P + 4), B.DGC_ERR_ALIGNMENT), (dict(channels=1 << 31), big),
                           (dict(rows=1 << 41, row_offsets=P), big)):
            assert call(dgc_lib, scan(**kw)) == status, kw
    n = C.c_int64()
    assert dgc_lib.dgc_gated_scan_state_rows(C.byref(scan()), None) == bad
    assert dgc_lib.dgc_gated_scan_workspace_bytes(C.byref(scan(channels=0)), C.byref(size)) == bad
    for rows, sequences in ((20, 4), (640, 1), (0, 3)):
        assert dgc_lib.dgc_gated_scan_state_rows(C.byref(scan(rows=rows, sequences=sequences, row_offsets=P)), C.byref(n)) == 0
        assert n.value == rows // B.DGC_SCAN_STATE_ROWS + sequences


def test_arguments_that_are_refused(dgc_lib):
    bad, off = B.DGC_ERR_INVALID_ARG, B.DGC_ERR_ALIGNMENT
    nan, inf = float("nan"), float("inf")
    for kw, status in ((dict(k=0), bad), (dict(k=257), bad), (dict(temperature=0.0), bad), (dict(temperature=-1.0), bad),
                       (dict(temperature=nan), bad), (dict(temperature=inf), bad), (dict(logits=None), bad),
                       (dict(idx=None), bad), (dict(val=None), bad), (dict(logits=P + 1), off), (dict(idx=P + 2), off),
                       (dict(lse=P + 2), off)):
        assert top(dgc_lib, logits(), **kw) == status, kw
    for kw, status in ((dict(k=-1), bad), (dict(k=257), bad), (dict(temperature=nan), bad), (dict(hard=-0.1), bad),
                       (dict(hard=1.1), bad), (dict(hard=nan), bad), (dict(labels=None), bad), (dict(idx=None), bad),
                       (dict(val=None), bad), (dict(loss=None, grad=None), bad), (dict(stride=99), bad),
                       (dict(stride=101), bad), (dict(logits=None), bad), (dict(logits=P + 1), off),
                       (dict(grad=P + 1), off), (dict(labels=P + 2), off), (dict(loss=P + 2), off), (dict(flags=P + 2), off)):
        assert distill(dgc_lib, logits(), **kw) == status, kw                # (grad is the logits, with stride 101)
    for kw, status in ((dict(gs=7), bad), (dict(xs=7), bad), (dict(hs=7), bad), (dict(gate=None), bad), (dict(x=None), bad),
                       (dict(h=None), bad), (dict(h=P, hs=9), bad), (dict(gate=P + 2), off), (dict(h0=P + 2), off),
                       (dict(states=P + 2), off), (dict(xs=1 << 60), B.DGC_ERR_CAPACITY)):
        assert forward(dgc_lib, scan(), **kw) == status, kw
    for kw, status in ((dict(gs=7), bad), (dict(dxs=7), bad), (dict(states=None), bad), (dict(dh=None), bad),
                       (dict(dgate=None), bad), (dict(dx=None), bad), (dict(dx=4 * P), bad), (dict(dx=3 * P, dxs=9), bad),
                       (dict(dgate=4 * P + 2), off), (dict(dh0=P + 2), off)):
        assert backward(dgc_lib, scan(), **kw) == status, kw


def test_workspaces_that_are_too_small(dgc_lib):
    size = C.c_size_t()
    shapes = [logits(rows=r, vocab=v, row_stride=v) for r, v in ((1, 200000), (4, 131072), (300, 5000))]
    for shape in shapes:
        assert dgc_lib.dgc_logits_workspace_bytes(C.byref(shape), C.byref(size)) == B.DGC_OK
        if size.value:
            for call in (top, distill):
                kw = dict(stride=shape.vocab) if call is distill else {}
                assert call(dgc_lib, shape, ws=None, **kw) == B.DGC_ERR_INVALID_ARG
                assert call(dgc_lib, shape, ws=P + 4, **kw) == B.DGC_ERR_ALIGNMENT
                assert call(dgc_lib, shape, bytes=size.value - 1, **kw) == B.DGC_ERR_CAPACITY
    for kw in (dict(rows=100000, sequences=1, max_length=100000, channels=64), dict(rows=4096, sequences=2, max_length=2048)):
        shape = scan(**kw)
        assert dgc_lib.dgc_gated_scan_workspace_bytes(C.byref(shape), C.byref(size)) == B.DGC_OK
        if size.value:
            strides = dict(gs=64, xs=64)
            assert forward(dgc_lib, shape, hs=64, ws=None, **strides) == B.DGC_ERR_INVALID_ARG
            assert forward(dgc_lib, shape, hs=64, bytes=size.value - 1, **strides) == B.DGC_ERR_CAPACITY
            assert backward(dgc_lib, shape, dhs=64, dgs=64, dxs=64, ws=P + 4, **strides) == B.DGC_ERR_ALIGNMENT


def test_nothing_to_do_is_no_error(dgc_lib):
    assert top(dgc_lib, logits(rows=0), logits=None, idx=None, val=None, lse=None) == B.DGC_OK
    assert distill(dgc_lib, logits(rows=0), logits=None, idx=None, val=None, loss=P, grad=None) == B.DGC_OK
    assert forward(dgc_lib, scan(rows=0, sequences=0), gate=None, x=None, h=None) == B.DGC_OK
    assert backward(dgc_lib, scan(rows=0, sequences=0), gate=None, x=None, states=None, dh=None, dgate=None, dx=None) == B.DGC_OK


def test_binding_refuses_other_tensors():
    import torch
    with pytest.raises(B.DgcError):
        B._dtype_code(torch.float64)
    t = torch.zeros(4, 10)
    here = t.get_device()                                             # -1: not a GPU
    f32 = torch.float32
    for tensor, dtype, shape, index in ((t, f32, (4, 9), here), (t, f32, (5, 10), here), (t, torch.bfloat16, (4, 10), here),
                                        (t, f32, (4, 10), 0), (torch.zeros(10, 4).t(), f32, (4, 10), here),
                                        (torch.zeros(1, 10).expand(4, 10), f32, (4, 10), here),
                                        (torch.zeros(40), f32, (4, 10), here)):
        with pytest.raises(B.DgcError) as err:
            B._rows_of(tensor, "t", dtype, shape, index)
        assert err.value.status == B.DGC_ERR_INVALID_ARG
    for tensor, shape in ((torch.zeros(4, 10)[:, :5], (4, 5)), (t, (40,))):
        with pytest.raises(B.DgcError):
            B._dense(tensor, "t", f32, shape, here)
    assert B._rows_of(torch.zeros(4, 30)[:, 5:15], "t", f32, (4, 10), here) == 30
    assert B._rows_of(torch.zeros(1, 10).expand(1, 10), "t", f32, (1, 10), here) == 10
    assert B._dense(None, "t", f32, (4,), here) == 0


# --- the definitions themselves ----------------------------------------------------------
def test_definition_of_the_loss_by_differences():
    rng = np.random.default_rng(1)
    z = rng.normal(size=(3, 17))
    idx = np.stack([rng.permutation(17)[:5] for _ in range(3)]).astype(np.int32)
    idx[1, 2] = -1
    val = rng.normal(size=(3, 5))
    labels = np.array([2, -1, idx[2, 1]])
    for kw in (dict(temperature=1.0, hard=0.0), dict(temperature=2.0, hard=0.3),
               dict(temperature=2.0, hard=0.3, top_lse=np.array([2.0, 2.5, 3.0]))):
        def f(w):
            return R.distill(w, idx, val, labels=labels, weight=np.array([1.0, 0.5, 2.0]), **kw)
        loss, grad = f(z)[:2]
        assert np.all(np.isfinite(loss))
        for j in range(17):
            up, down = z.copy(), z.copy()
            up[:, j] += 1e-5
            down[:, j] -= 1e-5
            assert np.allclose((f(up)[0] - f(down)[0]) / 2e-5, grad[:, j], atol=1e-8)


def test_definition_of_the_recurrence_by_differences():
    rng = np.random.default_rng(2)
    lengths = [4, 0, 7]
    v = dict(gate=rng.normal(size=(11, 3)), x=rng.normal(size=(11, 3)), h0=rng.normal(size=(3, 3)))
    dh, dl = rng.normal(size=(11, 3)), rng.normal(size=(3, 3))
    for free in (False, True):
        def f(w):
            out = R.scan_forward(w["gate"], w["x"], lengths, w["h0"], free)
            return (out["h"] * dh).sum() + (out["last"] * dl).sum()
        g = R.scan_backward(v["gate"], v["x"], lengths, v["h0"], dh, dl, free)
        for name, key in (("gate", "dgate"), ("x", "dx"), ("h0", "dh0")):
            for i in np.ndindex(v[name].shape):
                up, down = ({k: w.copy() for k, w in v.items()} for _ in range(2))
                up[name][i] += 1e-5
                down[name][i] -= 1e-5
                assert abs((f(up) - f(down)) / 2e-5 - g[key][i]) < 1e-8
