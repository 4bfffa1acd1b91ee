"""Workspaces of the operators on logits and sequences: what they need, and what is refused (no GPU: every check comes before
the first HIP call)."""

import ctypes as C

import pytest

from paper_1712_01887_amd import binding as B
from tests.test_operators_host import P, backward, distill, forward, logits, scan, top


@pytest.mark.parametrize("rows,vocab", [(0, 100), (1, 200000), (4, 131072), (300, 5000), ((1 << 31) - 1, 29)])
def test_logits_need_none(dgc_lib, rows, vocab):
    shape, size = logits(rows=rows, vocab=vocab, row_stride=vocab), C.c_size_t(99)
    assert dgc_lib.dgc_logits_workspace_bytes(C.byref(shape), C.byref(size)) == B.DGC_OK
    assert size.value == 0
    if rows == 0:
        for ws, have in ((None, 0), (P + 4, 0), (None, 1 << 40)):
            assert top(dgc_lib, shape, ws=ws, bytes=have) == B.DGC_OK
            assert distill(dgc_lib, shape, ws=ws, bytes=have) == B.DGC_OK


# (shape, tiles of 128 steps that leave a row of words each): one of 256 bytes and those words, in whole 256 bytes
SCANS = [(dict(rows=100000, sequences=1, max_length=100000, channels=64), 782),
         (dict(rows=4096, sequences=2, max_length=2048), 32),
         (dict(rows=129, sequences=1, max_length=129, channels=3), 2),
         (dict(rows=5000, sequences=7, max_length=3000, channels=1500, row_offsets=P), 5000 // 128 + 7)]


@pytest.mark.parametrize("kw,tiles", SCANS)
def test_tiles_side_by_side_need_their_words(dgc_lib, kw, tiles):
    shape, size = scan(**kw), C.c_size_t()
    assert dgc_lib.dgc_gated_scan_workspace_bytes(C.byref(shape), C.byref(size)) == B.DGC_OK
    assert size.value == 256 + -(-tiles * shape.channels * 8 // 256) * 256
    d = shape.channels
    ways = ((forward, dict(gs=d, xs=d, hs=d)), (backward, dict(gs=d, xs=d, dhs=d, dgs=d, dxs=d)))
    for call, strides in ways:
        assert call(dgc_lib, shape, ws=None, **strides) == B.DGC_ERR_INVALID_ARG
        assert call(dgc_lib, shape, ws=P + 4, **strides) == B.DGC_ERR_ALIGNMENT
        assert call(dgc_lib, shape, ws=P + 128, **strides) == B.DGC_ERR_ALIGNMENT
        assert call(dgc_lib, shape, bytes=size.value - 1, **strides) == B.DGC_ERR_CAPACITY


@pytest.mark.parametrize("kw", [dict(), dict(rows=128, sequences=1, max_length=128), dict(rows=4 * 128, sequences=4, max_length=128),
                                dict(rows=400 * 200, sequences=400, max_length=200), dict(rows=0, sequences=3, max_length=4, row_offsets=P)])
def test_other_scans_need_none(dgc_lib, kw):
    size = C.c_size_t(99)
    assert dgc_lib.dgc_gated_scan_workspace_bytes(C.byref(scan(**kw)), C.byref(size)) == B.DGC_OK
    assert size.value == 0
