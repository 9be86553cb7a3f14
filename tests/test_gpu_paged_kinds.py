"""What infinities and NaN do where they are seen, kind by kind: in values, and in keys whose scores become infinite."""
import math

import pytest
import torch

from tests import paged_util as pu
from tests.test_gpu_tree import run

pytestmark = pytest.mark.gpu

HINTS = (1, 6, 12, 20)          # 4 rows to a token: 16, 32, 64 and 128 rows to a tile (f32: 16 and 32)
TYPES = [("bf16", 128), ("f16", 128), ("bf16", 64), ("f16", 64), ("f32", 128), ("f32", 64)]
INF, NAN = math.inf, math.nan


def same_kind(got, want):
    return torch.isnan(got) if math.isnan(want) else got == want


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("first,second", [(-INF, 0.0), (INF, 0.0), (NAN, 0.0), (-INF, -INF), (INF, INF), (INF, -INF), (-INF, NAN)])
def test_kinds_of_values(first, second, hint, dtype, d):
    """Tokens 7 and 13 of a tree with such values in column 3: a row that sees them has their sum there, of its kind and sign; all else
    is as without them."""
    c = pu.make([75, 3], [21, 9], 2, d, 16, dtype, seed=95)
    q = pu.queries(c, 8, dtype, seed=96)
    bits, seen = pu.random_tree(c.some, 1, seed=97, holes=True)
    o, mass, size = pu.attention(c, q, d ** -0.5, seen)
    bound = pu.attention_bound(c, dtype, o, mass, size)
    p = c.table[0].long()
    for i, x in ((7, first), (13, second)):
        if x != 0.0:
            c.v[p[(75 + i) // 16], :, (75 + i) % 16, 3] = x
    got = run(c, q, d ** -0.5, bits, max_q=hint).double()
    kinds = set()
    for t in range(c.starts[-1]):
        values = [x for i, x in ((7, first), (13, second)) if t < 21 and i in seen[t] and x != 0.0]
        fine = torch.ones(d, dtype=torch.bool)
        if values:
            fine[3] = False
            assert same_kind(got[t, :, 3], sum(values)).all(), (t, values, got[t, :, 3])
            kinds.add(str(sum(values)))
        assert ((got[t] - o[t]).abs() <= bound[t])[:, fine].all(), t
    assert kinds


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("bad", [INF, -INF])
@pytest.mark.parametrize("at", [10, 74, 75, 75 + 13])
def test_keys_of_infinite_score(at, bad, hint, dtype, d):
    """A key that is infinite in one column, among the cached ones or the new: to queries on whose side its score is -inf it weighs nothing,
    to the others the output is NaN (inf - inf), and rows that do not see it are as they were."""
    c = pu.make([75, 3], [21, 9], 2, d, 16, dtype, seed=98)
    q = pu.queries(c, 8, dtype, seed=99)
    bits, seen = pu.random_tree(c.some, 1, seed=100, holes=True)
    p = c.table[0].long()
    c.k[p[at // 16], :, at % 16, 5] = 0.0
    o, mass, size = pu.attention(c, q, d ** -0.5, seen)
    all_bound = pu.attention_bound(c, dtype, o, mass, size)
    # without the key: its page column is left out by a score of -inf, which is what the formula gives
    ref, out = o.clone(), torch.zeros(c.starts[-1], 8, dtype=torch.bool)
    k, v, _ = c.keys(0)
    for t in range(21):
        js = [j for j in list(range(75)) + [75 + i for i in seen[t]] if j != at]
        if at < 75 or at - 75 in seen[t]:
            for h in range(8):
                if q[t, h, 5].sign() * math.copysign(1, bad) > 0:
                    out[t, h] = True
                else:
                    w = torch.softmax(k[h // 4][js] @ q[t, h].double() * d ** -0.5, 0)
                    ref[t, h] = w @ v[h // 4][js]
                    all_bound[t, h] = pu.attention_bound(c, dtype, ref[t:t + 1, h:h + 1], (w @ v[h // 4][js].abs()).view(1, 1, d),
                                                         size[t:t + 1, h:h + 1])[0, 0]
    c.k[p[at // 16], :, at % 16, 5] = bad
    got = run(c, q, d ** -0.5, bits, max_q=hint).double()
    assert torch.isnan(got[out]).all()
    assert ((got - ref).abs() <= all_bound)[~out].all()
    assert at == 75 + 13 or bool(out.any())
