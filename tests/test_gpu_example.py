"""The example program trains: its loss falls from the logarithm of the vocabulary towards the entropy of its data."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("eight", [False, True])
def test_training_with_moments_in_either_form(eight):
    import train_bigram
    vocab = 300
    losses, theta, t_perp = train_bigram.train(rounds=12, vocab=vocab, eight=eight)
    assert all(math.isfinite(x) for x in losses) and all(torch.isfinite(t).all() for t in theta + [t_perp])
    # four followers at 0.7, 0.1, 0.1, 0.1: 0.94; a model that has learnt nothing: 5.70; one that knows the followers but not
    # which is the frequent one: 1.39
    assert losses[0] < math.log(vocab) + 0.5
    assert losses[-1] < 1.39, losses


def test_the_same_run_gives_the_same_bits():
    import train_bigram
    a, b = (train_bigram.train(rounds=2, inner=5, eight=True) for _ in range(2))
    assert all(torch.equal(x, y) for x, y in zip(a[1] + [a[2]], b[1] + [b[2]]))
