"""Siblings that were not sampled, asked after likely ones were refused: how far the border between keeping and refusing
may be off does not grow as less is left.

p of a token and what is left of the row are sums of weights, none negative, each off by at most 2e-14 of itself; what is left loses
at most half to refused tokens before it is summed anew, so that it is off by at most (2 x 2e-14 + 2 x 2e-14) of itself, and p by as much as
its weight and the row's sum, 4e-14: in all 1.2e-13 of the border.  The random numbers lie at least 1e-12 from it and at most the half
step of their type, 2^-25."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify import call
from tests.verify_model import verify

pytestmark = pytest.mark.gpu

MOST = 1 - 2.0 ** -24


def siblings(refused, V, count, seed, places):
    """`count` sequences whose first tokens have all but little: refused[i] the share of what is left that is the i-th's.  The next
    sibling's random number is the float next to its border, above or below it."""
    gen = torch.Generator().manual_seed(seed)
    m = len(refused) + 2
    rows, tokens, uniform = [], [], []
    for _ in range(count):
        row = torch.randn(V, generator=gen)
        ids = torch.tensor(places) if places else torch.randperm(V, generator=gen)[:len(refused) + 1]
        rest = torch.ones(V, dtype=torch.bool)
        rest[ids[:-1]] = False
        row[ids[-1]] = torch.logsumexp(row[rest], 0) - 1.0            # some tenths of what is left
        left = torch.logsumexp(row[rest].double(), 0)
        for i, share in reversed(list(zip(ids[:-1].tolist(), refused))):
            row[i] = left + np.log(share / (1 - share))
            left = torch.logaddexp(left, row[i].double())
        keep = rest.clone()
        border = float(torch.exp(row[ids[-1]].double() - torch.logsumexp(row[keep].double(), 0)))
        near = np.float32(border)
        for other in (near, np.nextafter(near, np.float32(0)), np.nextafter(near, np.float32(1))):
            if abs(float(other) - border) > 2e-12:
                near = other
                break
        rows += [row] * m
        tokens += [0] + ids.tolist()
        uniform += [0.5] + [MOST] * len(refused) + [float(near)]
    n = m * count
    return dict(logits=torch.stack(rows), tokens=torch.tensor(tokens, dtype=torch.int32), uniform=torch.tensor(uniform),
                starts=list(range(0, n + 1, m)), parent=torch.tensor([-1] + [0] * (m - 1), dtype=torch.int32).repeat(count),
                draft=None, temperature=None)


@pytest.mark.parametrize("refused", [[0.4], [0.9], [0.999], [0.99999], [0.99, 0.99], [0.999, 0.999, 0.999], [0.9999] * 4, [0.7] * 20])
@pytest.mark.parametrize("V,places", [(64, None), (9000, None), (9000, "near")])
def test_borders_behind_refused_tokens(refused, V, places):
    """Somewhere in the vocabulary, or all in one chunk of it."""
    a = siblings(refused, V, 64, len(refused), [11 * i + 1 for i in range(len(refused) + 1)] if places else None)
    m = len(refused) + 2
    *want, near = verify(max_keep=2, **a)
    assert near > 1e-12
    kept = want[1]
    assert 10 < kept.count(2) < 54 and kept.count(1) + kept.count(2) == 64         # both sides of the border
    assert all(row[1] in (-1, m - 1) for row in want[0])
    assert call(a, 2) == tuple(want)
