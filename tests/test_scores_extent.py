"""Scores whose last row ends before its stride does: what lies behind the last key's score is not the call's."""
import pytest
import torch

from paper_2505_14201_amd import flashd
from tests.test_abi import NO_GPU
from tests.test_evict_refusals import S, evict, score
from tests.test_paged_refusals import E_HIP, E_OVERLAP, cache

PLACES = 64                               # of a row: max_pages * page of cache()
STRIDE = 100
LAST = S + 5 * STRIDE * 4                 # the last of 3 x 2 rows


@pytest.mark.skipif(not NO_GPU, reason="a valid call would launch a kernel on made-up pointers")
def test_what_lies_behind_the_last_row_is_taken():
    end = LAST + PLACES * 4
    for name in ("lse", "weight", "bits", "table", "lens", "start"):
        assert score(**{name: end}, stride=STRIDE) == E_HIP
    assert score(lse=S + 6 * PLACES * 4, stride=PLACES) == E_HIP
    for name in ("out", "budgets", "refs", "table", "lens"):
        assert evict(**{name: end}, stride=STRIDE) == E_HIP
    two = cache(layers=2, layer_stride=10 * 2 * 16 * 64)
    assert evict(two, layer_stride=5000, stride=STRIDE, out=end + 5000 * 4) == E_HIP


def test_the_last_row_itself_is_not():
    for name in ("lse", "weight"):
        assert score(**{name: LAST + PLACES * 4 - 4}, stride=STRIDE) == E_OVERLAP
    assert score(lse=S + 6 * PLACES * 4 - 4, stride=PLACES) == E_OVERLAP
    for name in ("out", "budgets", "refs"):
        assert evict(**{name: LAST + PLACES * 4 - 4}, stride=STRIDE) == E_OVERLAP
        assert evict(**{name: LAST}, stride=STRIDE) == E_OVERLAP
    two = cache(layers=2, layer_stride=10 * 2 * 16 * 64)
    assert evict(two, layer_stride=5000, stride=STRIDE, out=LAST + (5000 + PLACES) * 4 - 4) == E_OVERLAP


@pytest.mark.gpu
def test_rows_that_begin_inside_of_a_buffer():
    """Rows that are the ends of longer ones, and right behind the last of them another argument."""
    z = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t, device="cuda")       # noqa: E731
    pool = torch.randn(6, 2, 16, 64, device="cuda")
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    lens, starts = z(3) + 30, torch.arange(4, dtype=torch.int32, device="cuda")
    q = torch.randn(3, 4, 64, device="cuda")
    plain = torch.zeros(3, 2, 32, device="cuda")
    flashd.cache_score(q, pool, table, lens, starts, torch.ones(3, 4, device="cuda"), plain, 0.125)
    base = torch.zeros(3 * 2 * 50 + 12, device="cuda")
    lse = base[300:].view(3, 4)
    lse.fill_(1.0)
    rows = base[:300].view(3, 2, 50)[..., 18:]
    flashd.cache_score(q, pool, table, lens, starts, lse, rows, 0.125)
    assert torch.equal(rows, plain) and bool((lse == 1).all()) and not bool(base[:300].view(3, 2, 50)[..., :18].any())
    out = base[300:303].view(torch.int32)
    value = torch.randn_like(pool)
    k, v, kk, vv = pool.clone(), value.clone(), pool.clone(), value.clone()
    want = z(3)
    flashd.cache_evict(k, v, z(6) + 1, table, lens, plain, want, 20)
    flashd.cache_evict(kk, vv, z(6) + 1, table, lens, rows, out, 20)
    assert out.tolist() == want.tolist() == [20] * 3
    assert torch.equal(k, kk) and torch.equal(v, vv) and torch.equal(rows, plain)
