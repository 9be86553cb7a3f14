"""draft_verify, cache_score and cache_evict where offsets pass 32 bits, and at the largest vocabulary: the same bits as with
the same numbers close together, or the plain model's."""
import pytest
import torch

from paper_2505_14201_amd import flashd
from tests import paged_util as pu
from tests.test_gpu_verify import check, random_call

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def far_apart(x, stride):
    """x [rows, ...] with its rows `stride` elements apart; what lies between is not written."""
    row = x[0].numel()
    base = torch.empty((x.shape[0] - 1) * stride + row, dtype=x.dtype, device="cuda")
    out = base.as_strided(x.shape, (stride,) + x[0].contiguous().stride())
    out.copy_(x)
    return out


@pytest.mark.parametrize("n", [2, 40])
def test_pages_far_behind_the_first(n):
    """Keys in the last pages of pools of 9 GB."""
    c = pu.make([700, 33, 2500], [n, 1, n], 1, 128, 256, "bf16", seed=n)
    P = 140000
    far = (c.table + torch.where(c.table >= 0, P - c.k.shape[0], 0)).to(torch.int32)
    used = c.table[c.table >= 0].long()
    pools = []
    for x in (c.k, c.v):
        big = torch.empty(1, P, *x.shape[1:], dtype=BF16, device="cuda")
        big[0, (used + P - c.k.shape[0]).cuda()] = x[used].cuda()
        pools.append(big)
    q = pu.queries(c, 4, "bf16", seed=3).cuda()
    k, v, table, lens, starts = c.gpu()
    lse = torch.full((c.starts[-1], 4), 6.0, device="cuda")
    scores = []
    for kk, t in ((k, table), (pools[0][0], far.cuda())):
        score = torch.ones(3, 1, table.shape[1] * 256, device="cuda")
        flashd.cache_score(q, kk, t, lens, starts, lse, score, 0.05, decay=0.5)
        scores.append(score)
    assert torch.equal(scores[0], scores[1])
    refs = torch.zeros(c.k.shape[0], dtype=torch.int32)
    refs[used] = 1
    big_refs = torch.zeros(P, dtype=torch.int32)
    big_refs[used + P - c.k.shape[0]] = 1
    outs = []
    for kk, vv, t, r, s in ((k[None], v[None], table, refs, scores[0]), (*pools, far.cuda(), big_refs, scores[1])):
        out = torch.zeros(3, dtype=torch.int32, device="cuda")
        flashd.cache_evict(kk, vv, r.cuda(), t, lens, s, out, 512, first=2, recent=30)
        outs.append(out)
    assert outs[0].tolist() == outs[1].tolist() == [512, 33, 512]
    assert torch.equal(scores[0], scores[1])
    for small, big in ((k, pools[0][0]), (v, pools[1][0])):
        assert torch.equal(small[used.cuda()], big[(used + P - c.k.shape[0]).cuda()])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 30, 120])
def test_queries_far_apart(dtype, n):
    """So far that a tile's rows lie in one token, and rows pass 2^31 elements."""
    c = pu.make([300, 64], [n, 5], 2, 64, 64, dtype, seed=n)
    q = pu.queries(c, 10, dtype, seed=4).cuda()
    k, _, table, lens, starts = c.gpu()
    lse = torch.full((n + 5, 10), 5.0, device="cuda")
    scores = []
    for x in (q, far_apart(q, (1 << 25) + 640)):
        score = torch.ones(2, 2, table.shape[1] * 64, device="cuda")
        flashd.cache_score(x, k, table, lens, starts, lse, score, 0.125, decay=0.5)
        scores.append(score)
    # (other tiles, and so other orders of sums: each of 5 rows a token is added once, all are positive)
    assert bool(((scores[0] - scores[1]).abs() <= 2 * (5 * n + 3) * pu.EPS32 * scores[0]).all())
    again = torch.ones_like(scores[1])
    flashd.cache_score(x, k, table, lens, starts, lse, again, 0.125, decay=0.5)
    assert torch.equal(again, scores[1])


def test_logits_far_apart():
    a = random_call([9, 4, 30], 5000, BF16, True, F32, seed=11)
    stride = 110_000_000
    check(a, 8, logits=far_apart(a["logits"], stride), draft=far_apart(a["draft"], stride // 2))


@pytest.mark.parametrize("draft", [None, BF16])
def test_the_largest_vocabulary(draft):
    check(random_call([3, 1], 1 << 24, BF16, False, draft, seed=13), 3)
