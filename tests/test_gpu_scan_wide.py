"""Scans whose rows lie far apart or are wide: what lanes without work ask for stays behind every buffer's end, so that nothing
between the rows is written and nothing foreign comes into the sums.  Run with `-m gpu` on an MI355X."""

import pytest

from tests.test_gpu_scan import check

pytestmark = pytest.mark.gpu
MOST = (1 << 24) - 1


@pytest.mark.parametrize("dtype,stride", [("f32", 4473925), ("f32", 4500001), ("f32", 9586982), ("f32", MOST), ("f32", MOST - 1),
                                          ("f16", 8947849), ("bf16", 8947850), ("bf16", MOST), ("f16", MOST - 1), ("bf16", MOST - 3)])
def test_rows_far_apart(dtype, stride):
    check([5], 4 if stride % 2 == 0 else 3, dtype, packed=False, stride=stride, seed=30)
    check([11, 7], 2, dtype, free=True, stride=stride, seed=31)


@pytest.mark.parametrize("stride", [4500001, 9586982])
def test_tiles_of_rows_far_apart(stride):
    check([135], 4 if stride % 2 == 0 else 3, "f32", packed=False, stride=stride, seed=32)


def test_wide_rows():
    check([5], 4500001, "f32", packed=False, seed=33)
