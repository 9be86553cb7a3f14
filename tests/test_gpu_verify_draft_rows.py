"""Rows of `draft` that flashd_draft_verify does not read: those of tokens that no token continues."""
import math

import pytest

from tests.test_gpu_verify import BF16, F16, F32, call, check
from tests.verify_model import random_call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [1000, 5000])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("junk", [math.inf, math.nan, -math.inf, 3.0])
def test_draft_rows_that_no_token_continues_may_hold_anything(V, dtype, junk):
    for tree in (False, True):
        a = random_call([1, 5, 9, 2], V, F32, tree, dtype, seed=V + 1)
        continued = {s + int(p) for s, e in zip(a["starts"], a["starts"][1:])
                     for p in (a["parent"][s + 1:e].tolist() if tree else range(e - s - 1))}
        others = sorted(set(range(17)) - continued)
        assert len(others) >= 4
        for most in (9, 1):
            for u in (1.0, 2.0 ** -10):
                b = dict(a, uniform=a["uniform"] * u, draft=a["draft"].clone())
                want = check(b, most)
                b["draft"][others] = junk
                assert call(b, most) == want
