"""The vocabulary loss over the whole range of its inputs' values, against its definition in 64 bits
(tests/layers_reference.py).  Run with `-m gpu` on an MI355X."""

import numpy as np
import pytest

from paper_1712_01887_amd import binding as B
from tests import layers_reference as L
from tests.parity import say
from tests.test_gpu_rotary import close, dtype_of, rounded_inputs

pytestmark = pytest.mark.gpu


def run(hidden, weight, labels, row_weight, dtype):
    """{name: tensor} of both calls."""
    import torch
    t, (rows, width), vocab = dtype_of(dtype), hidden.shape, weight.shape[0]
    plan = B.VocabularyLoss(rows, vocab, width, t)
    h, m = torch.from_numpy(hidden).to(t).cuda(), torch.from_numpy(weight).to(t).cuda()
    y = torch.from_numpy(labels.astype(np.int32)).cuda()
    w = None if row_weight is None else torch.from_numpy(row_weight.astype(np.float32)).cuda()
    out = dict(loss=torch.full((rows,), 9.0, device="cuda"), lse=torch.full((rows,), 9.0, device="cuda"),
               dhidden=torch.full_like(h, 9.0), dweight=torch.full_like(m, 9.0))
    plan.dgc_vocab_loss_forward(h, m, y, out["loss"], out["lse"], row_weight=w)
    plan.dgc_vocab_loss_backward(h, m, y, out["lse"], out["dhidden"], out["dweight"], row_weight=w)
    return out


def kind(name, dtype):
    return dtype if name.startswith("d") else "f32"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(5, 1), (20, 29), (20, 64), (70, 65), (20, 10000), (300, 10000), (1400, 10000)])
@pytest.mark.parametrize("centre", [-90.0, -110.0, -500.0, 90.0])
def test_logits_far_from_zero(centre, rows, vocab, dtype):
    """All logits of all rows about `centre`, in tiles of every size, whose last one has wavefronts without a column."""
    say(f"[vocabulary loss] {rows} x {vocab} {dtype} logits about {centre}")
    rng = np.random.default_rng(rows + vocab)
    width = 32
    hidden, weight = rng.normal(size=(rows, width)), rng.normal(size=(vocab, width)) * 2.0 * width ** -0.5
    hidden[:, 7], weight[:, 7] = 1.0, centre
    hidden, weight = rounded_inputs(hidden, dtype), rounded_inputs(weight, dtype)
    labels = rng.integers(-1, vocab, rows)
    w = np.full(rows, 1.0 / rows, np.float32)
    want = L.vocab_loss(hidden, weight, labels, w, dtype)
    for name, got in run(hidden, weight, labels, w, dtype).items():
        close(got, *want[name], kind(name, dtype), name)
