"""A plan that several threads call: each call's sizes are its own (no GPU: the library is replaced by one that looks at what
it is given after another call has begun)."""

import ctypes as C

import pytest

from paper_1712_01887_amd import binding as B


class Late:
    """A library whose first call is overtaken by a second one before it reads its arguments."""

    def __init__(self):
        self.meanwhile, self.seen = None, []

    def _call(self, shape, logits, *_):
        run, self.meanwhile = self.meanwhile, None
        if run is not None:
            run()
        s = C.cast(shape, C.POINTER(B.DgcLogits)).contents
        self.seen.append((logits, s.dtype, s.rows, s.vocab, s.row_stride))
        return B.DGC_OK

    dgc_top_logits = dgc_distill_loss = _call

    def dgc_logits_workspace_bytes(self, shape, size):
        return B.DGC_OK


def plan(rows, vocab, monkeypatch):
    import torch
    lib = Late()
    monkeypatch.setattr(B, "load", lambda: lib)
    monkeypatch.setattr(B._Plan, "_on", lambda self, device: self.__dict__.update(
        _index=-1, device=torch.device("cpu"), _f32=torch.float32, _i32=torch.int32, _raw_stream=lambda i: 0, _current=lambda: -1))
    return B.Distillation(rows, vocab, torch.float32), lib


@pytest.mark.parametrize("op", ["top", "distill"])
@pytest.mark.parametrize("first,second", [((6, 40), (2, 57)), ((2, 57), (6, 40)), ((3, 41), (5, 40)), ((6, 41), (6, 42))])
def test_sizes_of_a_call_are_its_own(first, second, op, monkeypatch):
    import torch
    p, lib = plan(6, 40, monkeypatch)

    def call(rows, stride):
        z = torch.zeros(rows, stride)[:, :40]
        i, v = torch.zeros(rows, 4, dtype=torch.int32), torch.zeros(rows, 4)
        if op == "top":
            p.dgc_top_logits(z, i, v)
        else:
            p.dgc_distill_loss(z, i, v, torch.zeros(rows))
        return z

    keep = []
    lib.meanwhile = lambda: keep.append(call(*second))
    z = call(*first)
    assert lib.seen == [(keep[0].data_ptr(), B.DGC_F32, second[0], 40, second[1]), (z.data_ptr(), B.DGC_F32, first[0], 40, first[1])]
