"""flashd_cache_score against its definition in fp64."""
import math

import pytest
import torch

from paper_2505_14201_amd import flashd
from tests.paged_util import DT, EPS32, ints, make, queries, random_tree

pytestmark = pytest.mark.gpu


def log_sum_exp(c, q, scale, seen=None):
    """fp64 log-sum-exps [T, Hq] of the visible scores, rounded to fp32; -inf without a key."""
    T, Hq, _ = q.shape
    out = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    for t, h, x, at, _ in each_row(c, q, scale, seen):
        if len(at):
            out[t, h] = torch.logsumexp(x, 0)
    return out.float()


def each_row(c, q, scale, seen):
    """Token row, head, its visible scores, their keys, and the largest sum of absolute products."""
    Hkv = c.k.shape[1]
    for b, (l, m) in enumerate(zip(c.lens, c.some)):
        k, _, there = c.keys(b)
        for i in range(m):
            t = c.starts[b] + i
            js = range(i + 1) if seen is None else seen[t]
            at = torch.tensor(list(range(l)) + [l + j for j in js if j < m], dtype=torch.long)
            at = at[there[at]]
            for h in range(q.shape[1]):
                kh = k[h // (q.shape[1] // Hkv)][at]
                size = float((kh.abs() @ q[t, h].double().abs()).max()) * abs(scale) if len(at) else 0.0
                yield t, h, kh @ q[t, h].double() * scale, at, size


def model(c, q, scale, lse, score, decay, weight=None, seen=None):
    """fp64 scores and how far the operator may be from them.

    A weight's exponent in powers of 2: a sum of d products and its scaling, (d + 2) e of the sum of their absolute values (e = 2^-24);
    lse times log2 e, less log2 w (1 ulp of the hardware's logarithm): 4 e of their sizes; their difference: e of the larger.  In
    fp32 that is an absolute error of the exponent and so a relative one of the weight; 2 e more for the exponential.  The sum
    of n weights: n e of it at most; a product and a sum with the old score: 2 e."""
    out, bound = score.double().clone(), torch.zeros_like(score, dtype=torch.float64)
    fresh = torch.zeros_like(out)
    d, Hq = q.shape[2], q.shape[1]
    G = Hq // c.k.shape[1]
    of = [b for b, m in enumerate(c.some) for _ in range(m)]
    for t, h, x, at, size in each_row(c, q, scale, seen):
        l, w = float(lse[t, h]), 1.0 if weight is None else float(weight[t])
        if not math.isfinite(l) or not w > 0:
            continue
        p = w * torch.exp(x - l)
        off = ((d + 4) * size + 5 * (abs(l) + abs(math.log(w))) + 4) * EPS32
        fresh[of[t], h // G, at] += p
        bound[of[t], h // G, at] += p * off
    for b, (l, m) in enumerate(zip(c.lens, c.some)):
        if m:
            old = out[b, :, :l] * decay if decay else torch.zeros_like(out[b, :, :l])
            out[b, :, :l] = old + fresh[b, :, :l]
            out[b, :, l:l + m] = fresh[b, :, l:l + m]
            bound[b, :, :l + m] += (m * G + 3) * EPS32 * out[b, :, :l + m].abs() + 1e-37
    return out, bound


def check(c, Hq, dtype, decay=1.0, weight=None, tree=None, seen=None, scale=None, std=1.5, q=None, extra=0, bad_ok=False):
    q = queries(c, Hq, dtype, std=std, extra=extra) if q is None else q
    d = q.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    lse = log_sum_exp(c, q, scale, seen)
    B, Hkv, page = len(c.lens), c.k.shape[1], c.k.shape[2]
    S = c.table.shape[1] * page + 12
    old = torch.rand(B, Hkv, S, generator=torch.Generator().manual_seed(5))
    want, bound = model(c, q, scale, lse, old, decay, weight, seen)
    k, _, table, lens, start = c.gpu()
    if decay == 0.0:
        old = torch.where(bound > 0, math.nan, old.double()).float()         # is not read
    for b, (l, m) in enumerate(zip(c.lens, c.some)):
        old[b, :, l:l + m] = math.nan                                        # nor are these
    got = old.cuda()
    flashd.cache_score(q.cuda(), k, table, lens, start, lse.cuda(), got, scale, tree=None if tree is None else tree.cuda(),
                       row_weight=None if weight is None else weight.cuda(), decay=decay, kscale=c.kscale)
    got = got.cpu().double()
    left = bound == 0                                                        # the scores of no key of a sequence that grows
    assert torch.equal(got[left].nan_to_num(-1), old.double()[left].nan_to_num(-1))
    off = (got - want).abs()[~left]
    assert bool((off <= bound[~left]).all()), float((off / bound[~left]).max())
    return got


@pytest.mark.parametrize("dtype,fp8", [("f32", False), ("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 3])
def test_tokens(dtype, fp8, d, n):
    c = make([0, 1, 63, 64, 65, 257, 700, 31], [n, 1, n, 0, n, n, 1, n], 2, d, 16, dtype, fp8, seed=d + n)
    check(c, 8, dtype, decay=0.9)
    check(c, 2, dtype, decay=0.0)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (5, 5), (12, 4), (7, 1), (32, 2)])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_heads_and_pages(Hq, Hkv, page):
    check(make([300, 17, 129], [2, 5, 1], Hkv, 64, page, "bf16", seed=Hq), Hq, "bf16")


@pytest.mark.parametrize("dtype,fp8", [("f32", False), ("bf16", False), ("f16", True)])
@pytest.mark.parametrize("n", [9, 40, 150])
def test_chunks(dtype, fp8, n):
    """More rows than a group of them in LDS, keys that only the later rows see."""
    check(make([40, 0, 190], [n, n // 2, 2 * n], 2, 64, 32, dtype, fp8, seed=n), 8, dtype)


@pytest.mark.parametrize("Hq,n", [(130, 3), (257, 2), (129, 1), (128, 3), (127, 2), (65, 4), (7, 40), (3, 100)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_heads_to_one(Hq, n, dtype):
    """Groups of 64 or 128 rows are of whole tokens, or of a token's heads where those are more."""
    c = make([70, 5, 130], [n, 1, n], 1, 64, 16, dtype, seed=Hq)
    check(c, Hq, dtype)
    tree, seen = random_tree([n, 1, n], 2, holes=True)
    check(c, Hq, dtype, tree=tree, seen=seen, weight=torch.arange(2 * n + 1.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("words,some", [(1, [7, 33, 1, 0, 64]), (2, [70, 100, 5]), (1, [90])])
@pytest.mark.parametrize("holes", [False, True])
def test_trees(dtype, words, some, holes):
    c = make([45, 63, 0, 10, 200][:len(some)], some, 2, 64, 16, dtype, seed=words)
    tree, seen = random_tree(some, words, holes=holes)
    check(c, 4, dtype, tree=tree, seen=seen)


def test_a_key_that_begins_a_wavefronts_last_place():
    """The first new key behind 63, 127 and 255 old ones, which only one token of a tree sees."""
    some = [3, 3, 3]
    c = make([63, 127, 255], some, 1, 64, 16, "bf16", seed=2)
    tree = torch.tensor([[0], [1], [6]] * 3)
    check(c, 2, "bf16", tree=tree, seen=[[], [0], [1, 2]] * 3)


def test_weights_of_tokens():
    c = make([100, 300], [6, 40], 2, 128, 16, "bf16", seed=3)
    w = torch.rand(46, generator=torch.Generator().manual_seed(1)) + 0.01
    w[::3] = 0.0
    w[7] = -1.0
    w[8] = 1e-30
    check(c, 8, "bf16", weight=w)
    check(c, 8, "bf16", weight=torch.zeros(46))


def test_what_does_not_count_may_be_anything():
    """Tokens of weight 0 and without a key, pages that nobody has, keys that nobody sees: NaN and infinities."""
    some = [6, 5]
    c = make([100, 37], some, 2, 64, 16, "bf16", seed=4)
    q = queries(c, 4, "bf16")
    w = torch.ones(11)
    w[2] = 0.0
    tree, seen = random_tree(some, 1, seed=9, holes=True)
    for t in range(11):
        seen[t] = [j for j in seen[t] if j != 4]                     # token 4 of each sequence is seen by nobody
        tree[t] = sum(1 << j for j in seen[t])
    clean = check(c, 4, "bf16", weight=w, tree=tree, seen=seen, q=q)
    k = c.k.clone()
    for b in range(2):
        j = c.lens[b] + 4
        k[int(c.table[b, j // 16]), :, j % 16] = math.nan
    k[int(c.table[1, 2]), :, 37 + 5 - 32:] = math.inf                # behind the sequence
    free = set(range(k.shape[0])) - set(c.table.flatten().tolist())
    k[sorted(free)] = math.nan
    q[2] = math.inf
    scale = 0.125
    lse = log_sum_exp(c, queries(c, 4, "bf16"), scale, seen)
    _, _, table, lens, start = c.gpu()
    S = c.table.shape[1] * 16 + 12
    got = torch.rand(2, 2, S, generator=torch.Generator().manual_seed(5))
    for b in range(2):
        got[b, :, c.lens[b]:c.lens[b] + some[b]] = math.nan
    got = got.cuda()
    flashd.cache_score(q.cuda(), k.cuda(), table, lens, start, lse.cuda(), got, scale, tree=tree.cuda(), row_weight=w.cuda())
    assert torch.equal(got.cpu().double().nan_to_num(-1), clean.nan_to_num(-1))


def test_pages_that_are_none():
    c = make([100, 200], [3, 2], 2, 64, 16, "bf16", seed=6)
    c.table[0, 2] = -1
    c.table[1, 5] = -1
    check(c, 4, "bf16", decay=0.5)
    c.table[1, 7] = -9                       # held back
    check(c, 4, "bf16")


@pytest.mark.parametrize("dtype,fp8,d,n", [("bf16", False, 128, 88), ("f32", False, 128, 24), ("bf16", False, 64, 128),
                                           ("bf16", True, 128, 104), ("f32", False, 64, 88), ("f16", True, 64, 128)])
@pytest.mark.parametrize("more", [0, 1])
def test_rows_that_fit_on_the_chip_and_that_do_not(dtype, fp8, d, n, more):
    some = [n + more, 5, n + more - 1, 33]
    c = make([70, 900, 1500, 3], some, 2, d, 64, dtype, fp8, seed=n)
    check(c, 8, dtype, decay=0.9, weight=torch.arange(sum(some)) % 3 * 0.5)


@pytest.mark.parametrize("tree", [False, True])
def test_many_units_of_a_few_turns(tree):
    gen = torch.Generator().manual_seed(17)
    some = torch.randint(4, 30, (60,), generator=gen).tolist()
    c = make(torch.randint(0, 700, (60,), generator=gen).tolist(), some, 3, 64, 32, "bf16", seed=18)
    words, seen = random_tree(some, 1) if tree else (None, None)
    check(c, 15, "bf16", tree=words, seen=seen)


def test_long_and_many():
    gen = torch.Generator().manual_seed(7)
    some = torch.randint(0, 3, (700,), generator=gen).tolist()
    check(make(torch.randint(0, 90, (700,), generator=gen).tolist(), some, 1, 64, 16, "bf16", seed=8), 2, "bf16", extra=5)
    check(make([40000], [1], 1, 64, 256, "f16", seed=9), 3, "f16")


def test_strides_and_a_pool_of_layers():
    c = make([70, 20], [4, 3], 2, 64, 16, "f16", seed=10)
    q = queries(c, 4, "f16")
    lse = log_sum_exp(c, q, 0.125)
    k, _, table, lens, start = c.gpu()
    S = table.shape[1] * 16
    plain = torch.zeros(2, 2, S, device="cuda")
    flashd.cache_score(q.cuda(), k, table, lens, start, lse.cuda(), plain, 0.125)
    both = torch.full((3, k.shape[0], 2, *k.shape[1:]), math.nan, dtype=k.dtype, device="cuda")     # K and V side by side
    both[1, :, 0] = k
    wide = torch.full((7, 9, 64), math.nan, dtype=q.dtype, device="cuda")
    wide[:, 2:6] = q.cuda()
    far = torch.zeros(2, 2, S + 20, device="cuda")
    flashd.cache_score(wide[:, 2:6], both[1, :, 0], table, lens, start, lse.cuda(), far[..., :S], 0.125)
    assert torch.equal(far[..., :S], plain) and bool((far[..., S:] == 0).all())


def test_a_captured_call_is_replayed_with_other_numbers():
    c = make([70, 20, 0], [4, 3, 5], 2, 128, 16, "bf16", seed=11)
    q = queries(c, 4, "bf16")
    k, _, table, lens, start = c.gpu()
    lse, qg = log_sum_exp(c, q, 0.1).cuda(), q.cuda()
    score = torch.zeros(3, 2, table.shape[1] * 16, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    flashd.cache_score(qg, k, table, lens, start, lse, score, 0.1, decay=0.5, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flashd.cache_score(qg, k, table, lens, start, lse, score, 0.1, decay=0.5)
    for less in (0, 3, 1):
        lens.copy_(ints([70 - less, 20 - less, 0]))
        score.fill_(1.0)
        want = score.clone()
        flashd.cache_score(qg, k, table, lens, start, lse, want, 0.1, decay=0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(score, want)


def test_weights_of_a_row_sum_to_one():
    c = make([1000], [1], 1, 128, 16, "bf16", seed=12)
    got = check(c, 1, "bf16", decay=0.0)
    assert abs(float(got[0, 0, :1001].sum()) - 1) < 1e-4
