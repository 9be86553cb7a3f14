"""The log-sum-exps that flashd_attn_fwd_tree_lse leaves beside its output."""
import math

import pytest
import torch

from paper_2505_14201_amd import flashd
from tests.paged_util import EPS32, make, queries, random_tree
from tests.test_abi import E_ALIGN, E_NULL
from tests.test_gpu_score import each_row

pytestmark = pytest.mark.gpu


def check(c, Hq, dtype, tree=None, seen=None, hint=None, extra=0, scale=None):
    """Against fp64: each score is off by at most (d + 8) e of its sum of absolute products (e = 2^-24), and so is the log-sum-exp; the
    sum of n weights by n e of itself, and an exponential and a logarithm by some e of theirs; the results in powers of 2, and their product with ln
    2, by 4 e of their sizes (the reference lies at most 60 below the largest score)."""
    q = queries(c, Hq, dtype, std=1.5, extra=extra)
    T, _, d = q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    k, v, table, lens, start = c.gpu()
    o, plain = (torch.full((T, Hq, d), 7.0, dtype=q.dtype, device="cuda") for _ in range(2))
    lse = torch.full((T, Hq), 7.0, device="cuda")
    args = dict(tree=None if tree is None else tree.cuda(), kscale=c.kscale, vscale=c.vscale)
    hint = hint or max(max(c.some), 1)
    flashd.attn_fwd_tree(q.cuda(), k, v, o, table, lens, start, hint, scale, lse=lse, **args)
    flashd.attn_fwd_tree(q.cuda(), k, v, plain, table, lens, start, hint, scale, **args)
    assert torch.equal(o, plain)
    got = lse.cpu().double()
    for t, h, x, at, size in each_row(c, q, scale, seen):
        if len(at) == 0:
            assert float(got[t, h]) == -math.inf
            continue
        want = float(torch.logsumexp(x, 0))
        bound = EPS32 * ((d + 8) * size + len(at) + 16 + 4 * (abs(want) + 60))
        assert abs(float(got[t, h]) - want) <= bound, (t, h, float(got[t, h]), want, bound)
    assert bool((got[c.starts[-1]:] == 7).all())             # rows of nobody
    return lse


@pytest.mark.parametrize("dtype,fp8", [("f32", False), ("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 4, 14, 40])
def test_types_and_tiles(dtype, fp8, d, n):
    c = make([0, 1, 65, 700, 31], [n, n, 0, 1, n], 2, d, 16, dtype, fp8, seed=d + n)
    check(c, 8, dtype, extra=3)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("L,n", [(20000, 1), (9000, 12), (5000, 70)])
def test_units_that_are_split(dtype, L, n):
    check(make([L], [n], 1, 64, 64, dtype, seed=n), 3, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_trees_with_rows_that_see_nothing(dtype):
    some = [7, 33, 1, 0, 64]
    c = make([45, 0, 0, 10, 200], some, 2, 64, 16, dtype, seed=1)
    tree, seen = random_tree(some, 1, holes=True)
    check(c, 4, dtype, tree=tree, seen=seen)
    check(c, 4, dtype, tree=tree, seen=seen, scale=-0.3, hint=1)


def test_peaked_scores():
    for dtype in ("f16", "bf16", "f32"):
        check(make([300, 2000], [3, 20], 1, 64, 16, dtype, seed=2, qk_std=6.0), 4, dtype, scale=1.0)


def test_refusals():
    from tests.test_paged_refusals import AUX, O, Q, START, cache
    call = lambda **kw: flashd.raw().flashd_attn_fwd_tree_lse(     # noqa: E731
        cache(), 0, Q, 256, O, 256, 5, 3, 4, START, AUX, 1, 0.1, flashd.BF16, kw["lse"], None, None, 0)
    assert call(lse=None) == E_NULL and call(lse=0x200000000002) == E_ALIGN
    for at in (Q, O, START, AUX, O + 5 * 4 * 64 * 2 - 4):
        assert call(lse=at) == -12


def test_captured():
    c = make([300, 20, 4000], [3, 5, 1], 2, 128, 16, "bf16", seed=3)
    q = queries(c, 8, "bf16").cuda()
    k, v, table, lens, start = c.gpu()
    o, lse = torch.zeros_like(q), torch.zeros(9, 8, device="cuda")
    ws = torch.empty(flashd.tree_workspace_bytes(8, 2, 5, 128, flashd.BF16), dtype=torch.uint8, device="cuda")
    want = check(c, 8, "bf16")
    q = queries(c, 8, "bf16", std=1.5).cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flashd.attn_fwd_tree(q, k, v, o, table, lens, start, 5, 1 / math.sqrt(128), lse=lse, workspace=ws)
    for _ in range(3):
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(lse, want)
