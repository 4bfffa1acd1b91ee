"""Temperatures that the operators on logits accept (no GPU: the check comes before the first HIP call)."""

import ctypes as C

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B

SMALLEST = np.float32(1.44269504) / np.finfo(np.float32).max          # below it, log2(e) / temperature is infinite


def calls(lib, temperature):
    shape = B.DgcLogits(B.DGC_F32, 0, 0, 100, 100)                    # no rows: nothing is launched
    p = 1 << 20
    return (lib.dgc_top_logits(C.byref(shape), p, temperature, 4, p, p, p, None, 0, None),
            lib.dgc_distill_loss(C.byref(shape), p, 4, p, p, None, p, None, temperature, 0.5, p, p, 100, None, None, 0, None))


@pytest.mark.parametrize("temperature", [1e-45, 1e-40, 2.9e-39, float(SMALLEST) * 0.999])
def test_so_cold_that_the_scale_is_infinite(dgc_lib, temperature):
    assert calls(dgc_lib, temperature) == (B.DGC_ERR_INVALID_ARG, B.DGC_ERR_INVALID_ARG)


@pytest.mark.parametrize("temperature", [float(SMALLEST) * 1.001, 1e-38, 1e-3, 1.0, 1e30])
def test_accepted(dgc_lib, temperature):
    assert calls(dgc_lib, temperature) == (B.DGC_OK, B.DGC_OK)
