"""Ids of probability 0 in flashd_draft_verify: masked logits (-infinity, NaN) are neither kept nor drawn, whatever the random
numbers and the drafts' probabilities.  Results by hand, from the definition."""
import math

import pytest
import torch

from tests.test_gpu_verify import call

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
MOST = 1 - 2.0 ** -24                     # the largest random number below 1
MASKS = [-math.inf, math.nan]


def sequences(rows, tokens, uniform, parent=None, draft=None, heat=None, dtype=F32):
    """One sequence of len(tokens) new tokens, `rows` the logits behind each."""
    n = len(tokens)
    return dict(logits=torch.stack(rows).to(dtype), tokens=torch.tensor(tokens, dtype=torch.int32), uniform=torch.tensor(uniform),
                starts=[0, n], parent=None if parent is None else torch.tensor(parent, dtype=torch.int32),
                draft=None if draft is None else torch.stack(draft), temperature=None if heat is None else torch.tensor([heat]))


def allowed(V, ids, mask, seed=0):
    """Logits of which only `ids` are not masked."""
    row = torch.full((V,), mask)
    row[ids] = torch.randn(len(ids), generator=torch.Generator().manual_seed(seed))
    return row


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("heat", [None, 0.7, 1e-30, math.inf])
@pytest.mark.parametrize("V,first", [(1000, 1), (1000, 999), (5000, 17), (5000, 4096), (9000, 4097), (9000, 8999)])
def test_the_first_and_the_last_allowed_id_are_drawn(dtype, mask, heat, V, first):
    ids = sorted({first, min(first + 3, V - 1), min(first + 300, V - 1)})
    row = allowed(V, ids, mask)
    row[ids] = 1.0                        # (all alike, so that a temperature of 1e-30 leaves all of them)
    for draft in (None, [torch.full((V,), 1.0 / V)]):
        for u, want in ((0.0, ids[0]), (MOST, ids[-1])):
            assert call(sequences([row], [0], [u], draft=draft, heat=heat, dtype=dtype), 1) == ([[0]], [1], [want])


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("tree", [False, True])
def test_a_masked_draft_is_refused(mask, tree):
    """Its random number is 0, or its own probability as a draft is, so that u q(x) is 0; 0 is not below 0."""
    V = 6000
    row = allowed(V, [5, 4500], mask)
    parent = [-1, 0, 0] if tree else None
    for u in (0.0, 0.5, MOST):
        for x in (0, 6, 4499, 5999):
            for q in (None, 0.0, -1.0, math.nan, 1e-9):
                if u > 0 and q is None:
                    continue
                draft = None
                if q is not None:
                    draft = [torch.zeros(V) for _ in range(3)]
                    for r in draft:
                        r[x] = q
                for u0, want in ((0.0, 5), (MOST, 4500)):
                    a = sequences([row] * 3, [0, x, x], [u0, u, u], parent, draft)
                    assert call(a, 3) == ([[0, -1, -1]], [1], [want]), (u, x, q, u0)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("draft", [F32, F16])
def test_nothing_is_left_but_masked_ids(mask, draft):
    """p is 1/2 at two ids and 0 elsewhere, q a little more at both: after the refusal nothing is left, r stays p, and the same draft
    asked once more is kept by u = 0.9."""
    V = 5000
    row = torch.full((V,), mask)
    row[[7, 4200]] = 0.0
    q = torch.zeros(V)
    q[[7, 4200]] = 0.501                  # 0.99999994 x 0.501 is not below 0.5, 0.9 x 0.501 is
    q = q.to(draft)
    rows, drafts, parent = [row] * 3, [q] * 3, [-1, 0, 0]
    for x in (7, 4200):
        assert call(sequences(rows, [0, x, x], [0.5, MOST, 0.9], parent, drafts), 3)[:2] == ([[0, 2, -1]], [2])
        for u0, want in ((0.0, 7), (0.49, 7), (0.51, 4200), (MOST, 4200)):
            assert call(sequences(rows, [0, x, x], [u0, MOST, MOST], parent, drafts), 3) == ([[0, -1, -1]], [1], [want])


@pytest.mark.parametrize("mask", MASKS)
def test_siblings_up_to_the_last_allowed_id(mask):
    """Not sampled: three ids have a third each; the two of them that are refused are not drawn, nor is a masked one."""
    V = 4099
    row = torch.full((V,), mask)
    row[[3, 4000, 4098]] = 2.0
    for u0 in (0.0, 0.5, MOST):
        for x, y, left in ((3, 4000, 4098), (4098, 3, 4000), (4000, 4098, 3)):
            a = sequences([row] * 4, [0, x, y, 11], [u0, MOST, MOST, 0.0], [-1, 0, 0, 0])
            assert call(a, 4) == ([[0, -1, -1, -1]], [1], [left])
