"""Beam selection where its sums are at an end of what they can be, against the definition in 64 bits as in test_beams.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_beams import BF16, F32, TORCH, check, gpu, scores


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab,some", [(4096, 4096), (5000, 5000), (9001, 4000), (70000, 40000), (300, 300)])
@pytest.mark.parametrize("out", [3, 64])
@pytest.mark.parametrize("groups", [1, 60])
def test_many_logits_of_the_largest_finite_number(dtype, vocab, some, out, groups):
    """More than LDS holds candidates, with nothing above them that could be a bound; also beside what is lower, below it by a step, and -inf.
    A row's log sum is the largest number + log(some), which in 64 bits is that number: all are worth the row's score"""
    rng, beams, top = np.random.default_rng(some), 3, float(torch.finfo(TORCH[dtype]).max)
    x = np.full((groups * beams, vocab), top, np.float64)
    for r, low in zip(range(len(x)), (1.0, -np.inf, top * (1 - torch.finfo(TORCH[dtype]).eps), -top)):
        x[r, rng.permutation(vocab)[: vocab - some]] = low
    check(x.astype(np.float32), scores(rng, len(x)), None, 0, beams, out, dtype)
