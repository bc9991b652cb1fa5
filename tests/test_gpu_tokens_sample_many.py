"""olive_sample on so many rows that a workgroup counts a whole row of up to 65024 bf16 tokens by
itself, in counts of 16 bits: the same answers as calls of few rows give, whose rows are counted in
parts, and as the fp64 definition does (which test_gpu_tokens_sample.py states)."""
import numpy as np
import pytest
import torch

from paper_2609_36246_amd import _lib as L
from tests.test_gpu_tokens_sample import Sample, uniform
from tests.tokens_harness import BF16

pytestmark = pytest.mark.gpu
ROWS = 1100


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    L.load()


def logits(vocab):
    """Rows of normal values; among them rows of one value (a count of `vocab`) and of two whose bins share a
    word (neighbours: their last bits differ), in parts of every share."""
    gen = torch.Generator().manual_seed(vocab)
    z = (torch.randn(ROWS, vocab, generator=gen) * 2.0).to(BF16)
    z[3], z[4], z[5], z[6] = 1.5, 1.5078125, -1.5, 0.0
    for i, (a, b) in enumerate(((1.5, 1.5078125), (1.5078125, 1.5), (1.5078125, 1.515625), (-1.5, -1.5078125))):
        z[10 + i], z[20 + i], z[30 + i] = a, a, a
        z[10 + i, -1], z[20 + i, ::2], z[30 + i, 1:] = b, b, b
    z[40] = torch.finfo(BF16).min
    z[40, vocab // 2] = 1.0
    z[41] = -float("inf")
    z[41, -1] = -3.0
    z[42] *= 1e-15                                     # values without a bin
    return z.cuda()


@pytest.mark.parametrize("vocab", [16385, 40001, 65023, 65024])
@pytest.mark.parametrize("settings", [dict(top_p=0.9301), dict(top_k=32513), dict(top_k=60, top_p=0.9, min_p=0.011),
                                      dict(min_p=0.05, temperature=1.3)], ids=str)
def test_rows_that_one_workgroup_counts(vocab, settings):
    z, u = logits(vocab), uniform(ROWS, vocab)
    u[43], u[44] = 0.0, 1.0
    whole = Sample(z, u, **settings)
    assert len(whole.work) == 0
    got = whole.run()
    few = [np.concatenate(t) for t in zip(*(
        tuple(a.copy() for a in Sample(z[i:i + 100], u[i:i + 100], **settings).run()) for i in range(0, ROWS, 100)))]
    assert np.array_equal(got[0], few[0]) and np.array_equal(got[2], few[2])
    assert np.all(np.abs(got[1] - few[1]) <= 2.0 ** -23 * np.abs(few[1]) + 2.0 ** -39 * (1 + np.abs(few[1])))
    rows = [0, 3, 4, 5, 6, 10, 11, 12, 13, 20, 21, 22, 23, 30, 31, 32, 33, 40, 41, 42, 43, 44, 1099]
    some = Sample(z[rows], u[rows], **settings)
    some.run = lambda: tuple(a[rows] for a in got)
    some.check()
