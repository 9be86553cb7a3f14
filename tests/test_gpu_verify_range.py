"""What flashd_draft_verify does with numbers at and past the ends of their ranges: the next token is one that the target allows."""
import math

import pytest
import torch

from tests.test_gpu_verify import BF16, F32, call
from tests.verify_model import random_call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [1, 2, 1000, 4097, 5000, 8191])
@pytest.mark.parametrize("draft", [None, F32])
@pytest.mark.parametrize("u", [1.0, math.nan, 2.0, math.inf, -1.0])
def test_a_random_number_that_is_none(V, draft, u):
    """The next token is in the vocabulary and not masked, behind chains and trees, whatever has been refused."""
    for tree in (False, True):
        a = random_call([1, 4, 9], V, BF16, tree, draft, seed=V)
        a["logits"][:, 1::2] = -math.inf
        a["logits"][:, V // 2 + 1:] = math.nan
        a["uniform"][:] = u
        _, n, then = call(a, 9)
        for b in range(3):
            assert 1 <= n[b] <= 9 and 0 <= then[b] <= V // 2 and then[b] % 2 == 0, (b, then)
        a["uniform"][1:] = 0.9
        a["uniform"][torch.tensor(a["starts"][:-1])] = u
        assert all(0 <= x <= V // 2 and x % 2 == 0 for x in call(a, 9)[2])


@pytest.mark.parametrize("u", [1.0, math.nan])
def test_every_allowed_id_refused(u):
    """Random numbers that refuse what has probability 1: what was left before the last refusal stays."""
    V = 5000
    for ids in ([9], [9, 4500], [9, 10, 4500]):
        row = torch.full((V,), -math.inf)
        row[ids] = 0.0
        n = len(ids) + 2
        a = dict(logits=row.repeat(n, 1), tokens=torch.tensor([0] + ids + [ids[0]], dtype=torch.int32),
                 uniform=torch.full((n,), u), starts=[0, n], parent=torch.tensor([-1] + [0] * (n - 1), dtype=torch.int32),
                 draft=None, temperature=None)
        _, _, then = call(a, n)
        assert then[0] in ids
