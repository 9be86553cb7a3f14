"""flashd_attn_fwd_tree against fp64: lengths from none to several pages and more than one workgroup's
share, row counts around the tile, pages that end inside a block, chains and trees whose rows may see nothing, the types
and the strides, and what infinities and NaN do where they are not seen."""
import pytest
import torch

from paper_2505_14201_amd import flashd
from tests import paged_util as pu

pytestmark = pytest.mark.gpu


def run(c, q, scale, bits=None, max_q=None, ws=None, o=None, **kw):
    k, v, table, lens, start = c.gpu()
    if o is None:
        o = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    flashd.attn_fwd_tree(q.cuda(), k, v, o, table, lens, start, max_q or max(c.some), scale,
                         tree=None if bits is None else bits.cuda(), kscale=c.kscale, vscale=c.vscale,
                         workspace=ws, **kw)
    torch.cuda.synchronize()
    return o.cpu()


def check(c, q, dtype, scale, bits=None, seen=None, got=None, rows=None, **kw):
    got = run(c, q, scale, bits, **kw) if got is None else got
    o, mass, size = pu.attention(c, q, scale, seen)
    bound = pu.attention_bound(c, dtype, o, mass, size)
    rows = slice(None) if rows is None else rows
    err = (got.double() - o).abs()[rows]
    worst = (err / bound[rows]).max().item() if err.numel() else 0.0
    assert torch.isfinite(got[rows].double()).all()
    assert worst <= 1.0, f"{worst:.2f} times the bound, off by {err.max():.2e}"
    return got


# (lens, new tokens, Hq, Hkv, page)
SHAPES = [([0], [1], 1, 1, 16), ([1], [1], 4, 1, 16), ([15], [1], 4, 2, 16), ([16], [1], 8, 2, 16),
          ([31, 0, 5], [1, 1, 1], 4, 4, 16), ([33, 100], [2, 0], 6, 2, 32), ([0, 129, 64], [0, 3, 5], 8, 2, 64),
          ([200, 1, 77, 300], [4, 9, 1, 2], 16, 1, 128), ([700], [17], 5, 1, 256), ([1025, 3], [1, 33], 12, 2, 16)]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("shape", SHAPES)
def test_chains_and_trees(shape, dtype, d):
    lens, some, Hq, Hkv, page = shape
    c = pu.make(lens, some, Hkv, d, page, dtype, seed=len(lens) + lens[0])
    q = pu.queries(c, Hq, dtype, seed=3)
    check(c, q, dtype, d ** -0.5)
    for holes in (False, True):
        bits, seen = pu.random_tree(some, 1, seed=lens[0], holes=holes)
        got = check(c, q, dtype, d ** -0.5, bits, seen)
        if lens[0] == 0:
            none = [t for t in range(some[0]) if not seen[t]]
            assert torch.count_nonzero(got[none]) == 0
    check(c, q, dtype, -d ** -0.5)
    check(c, q, dtype, 0.0)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("lens,some,page", [([40, 0, 333], [3, 1, 6], 16), ([1500], [20], 64)])
def test_fp8_cache(lens, some, page, dtype, d):
    c = pu.make(lens, some, 2, d, page, fp8=True, seed=5)
    q = pu.queries(c, 8, dtype, seed=6)
    check(c, q, dtype, d ** -0.5)
    bits, seen = pu.random_tree(some, 1, seed=7)
    check(c, q, dtype, d ** -0.5, bits, seen)


@pytest.mark.parametrize("words,n", [(1, 64), (1, 70), (2, 70), (2, 128), (3, 129)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_words_of_a_tree(words, n, dtype):
    """Tokens up to the last bit of a row's words; those past it are not seen."""
    c = pu.make([45], [n], 1, 64, 16, dtype, seed=n)
    q = pu.queries(c, 2, dtype, seed=8)
    bits, seen = pu.random_tree([n], words, seed=9)
    check(c, q, dtype, 0.125, bits, seen)


@pytest.mark.parametrize("lens,some", [([20000], [1]), ([9000, 10, 4100, 0, 777], [3, 1, 2, 1, 5])])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_long_sequences(lens, some, dtype):
    """Units that many workgroups share, next to short ones."""
    c = pu.make(lens, some, 2, 64, 64, dtype, seed=11)
    q = pu.queries(c, 4, dtype, seed=12)
    check(c, q, dtype, 0.125)


def test_many_sequences():
    """More sequences than threads, most of them without new tokens."""
    lens = [(7 * b) % 50 for b in range(700)]
    some = [b % 3 == 1 for b in range(700)]
    some = [int(x) for x in some]
    c = pu.make(lens, some, 1, 64, 16, "bf16", seed=13)
    check(c, pu.queries(c, 4, "bf16", seed=14), "bf16", 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_scores_that_keep_growing(dtype):
    """Keys that grow along the sequence: every block lies far above what was seen before."""
    c = pu.make([900], [4], 1, 128, 32, dtype, seed=15, qk_std=4.0)
    j = torch.arange(904)
    c.k[c.table[0].long()[j // 32], :, j % 32] *= torch.linspace(0.05, 4.0, 904).view(-1, 1, 1).to(c.k.dtype)
    check(c, pu.queries(c, 8, dtype, seed=16, std=4.0), dtype, 128 ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), float("-inf")])
def test_what_is_not_seen_may_hold_anything(dtype, bad):
    """New tokens that only some rows see, with a value and a key that are no numbers: the others keep
    their output.  The keys behind a sequence's last one are no numbers either."""
    lens, some = [70, 5], [6, 4]
    c = pu.make(lens, some, 2, 64, 16, dtype, seed=17)
    q = pu.queries(c, 8, dtype, seed=18)
    bits, seen = pu.random_tree(some, 1, seed=19, holes=False)
    o, mass, size = pu.attention(c, q, 0.125, seen)
    bound = pu.attention_bound(c, dtype, o, mass, size)
    for b, (l, m) in enumerate(zip(lens, some)):
        p = c.table[b].long()
        for key in range(l + m, len(p) * 16):
            if p[key // 16] >= 0:
                c.v[p[key // 16], :, key % 16] = bad
                c.k[p[key // 16], :, key % 16] = bad
        at = l + m - 2                                  # token m - 2: seen by itself and maybe m - 1
        c.v[p[at // 16], :, at % 16, 3] = bad
        c.k[p[at // 16], :, at % 16, 5] = bad
    got = run(c, q, 0.125, bits)
    for b, m in enumerate(some):
        for i in range(m):
            t = c.starts[b] + i
            if m - 2 not in seen[t]:
                assert ((got[t].double() - o[t]).abs() <= bound[t]).all(), (b, i)
            else:
                assert not torch.isfinite(got[t].double()[:, 3]).any() or bad == float("-inf")


def test_fp8_nan_that_is_not_seen():
    c = pu.make([33], [3], 1, 64, 16, fp8=True, seed=20)
    q = pu.queries(c, 4, "bf16", seed=21)
    bits = torch.tensor([[1], [3], [4]])
    o, mass, size = pu.attention(c, q, 0.125, [[0], [0, 1], [2]])
    c.v.view(torch.uint8)[c.table[0, 2].long(), :, 2, 7] = 0x7f       # key 34, token 1
    got = run(c, q, 0.125, bits)
    bound = pu.attention_bound(c, "bf16", o, mass, size)
    for t in (0, 2):
        assert ((got[t].double() - o[t]).abs() <= bound[t]).all()
    assert torch.isnan(got[1, :, 7]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64])
def test_missing_pages_weigh_nothing(dtype, page):
    c = pu.make([300, 90], [2, 1], 2, 64, page, dtype, seed=22)
    c.table[0, 1] = -1
    q = pu.queries(c, 4, dtype, seed=23)
    check(c, q, dtype, 0.125)
    c.table[1] = -1                                     # a sequence without any page
    got = check(c, q, dtype, 0.125)
    assert torch.count_nonzero(got[2]) == 0
    bad = pu.Paged(c.k, c.v, c.table.clone(), c.lens, c.some)
    bad.table[0, 1] = c.k.shape[0]                      # a number behind the pool is no page
    bad.table[1] = -7
    assert torch.equal(run(bad, q, 0.125), got)


def test_strides_and_rows_behind_the_last():
    """Queries inside a projection's output, outputs with a gap, K and V of a page side by side, rows behind
    the last sequence left as they were."""
    c = pu.make([50, 7], [3, 2], 2, 64, 16, "bf16", seed=24)
    q = pu.queries(c, 4, "bf16", seed=25, extra=3)
    pool = torch.zeros(c.k.shape[0], 2, *c.k.shape[1:], dtype=torch.bfloat16)
    pool[:, 0], pool[:, 1] = c.k, c.v
    pool = pool.cuda()
    wide = torch.zeros(8, 7, 64, dtype=torch.bfloat16, device="cuda")
    wide[:, 1:5] = q.cuda()
    out = torch.full((8, 5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    flashd.attn_fwd_tree(wide[:, 1:5], pool[:, 0], pool[:, 1], out[:, :4], c.table.cuda(), pu.ints(c.lens).cuda(),
                         pu.ints(c.starts).cuda(), 3, 0.125)
    torch.cuda.synchronize()
    check(c, q[:5], "bf16", 0.125, got=out[:5, :4].cpu())
    assert (out[5:] == 7).all() and (out[:, 4] == 7).all()


def test_any_hint_and_a_workspace_between_canaries():
    from tests.gpu_util import Guarded
    c = pu.make([2000, 30], [9, 2], 2, 128, 64, "bf16", seed=26)
    q = pu.queries(c, 8, "bf16", seed=27)
    for hint in (1, 2, 9, 40, 1000):
        need = flashd.tree_workspace_bytes(8, 2, hint, 128, flashd.BF16)
        ws = Guarded(need)
        check(c, q, "bf16", 0.09, max_q=hint, ws=ws.payload)
        assert ws.intact()
        assert torch.equal(run(c, q, 0.09, max_q=hint), run(c, q, 0.09, max_q=hint, ws=ws.payload))


def test_a_page_beyond_32_bits():
    """Page numbers times their size pass 2^32 bytes: one layer of a pool of 4.3 GB, used at its ends."""
    P, page, d = 66000, 256, 128
    k = torch.zeros(P, 1, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    c = pu.make([500], [1], 1, d, page, "bf16", seed=28)
    ids = [P - 1, 1, P - 2][:c.table.shape[1]]
    for at, p in enumerate(ids):
        k[p], v[p] = c.k[c.table[0, at]].cuda(), c.v[c.table[0, at]].cuda()
    q = pu.queries(c, 4, "bf16", seed=29)
    o = torch.empty_like(q, device="cuda")
    flashd.attn_fwd_tree(q.cuda(), k, v, o, pu.ints([ids]).cuda(), pu.ints([500]).cuda(), pu.ints([0, 1]).cuda(), 1, 0.09)
    torch.cuda.synchronize()
    check(c, q, "bf16", 0.09, got=o.cpu())
