"""The paged cache's operators where what they find on the device is no program's: every output lies between canaries."""
import pytest
import torch

from paper_2505_14201_amd import flashd
from tests import paged_util as pu
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu

HINTS = (1, 6, 12, 20)          # 4 rows to a token: 16, 32, 64 and 128 rows to a tile (f32: 16 and 32)
INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1
WILD = [([-5, 1 << 30, 7], [0, 3, 1, 9]), ([0, 0, 0], [0, -4, 2, 1 << 30]), ([190, 192, 500], [0, 3, 4, 9]),
        ([3, 0, 0], [1, INT_MIN, 4, 9]), ([0, 5, 9], [8, INT_MIN, INT_MIN + 1, INT_MAX]), ([INT_MIN, INT_MAX, 17], [INT_MIN, INT_MAX, 1, INT_MIN]),
        ([0, 0, 0], [INT_MAX, INT_MAX, INT_MAX, INT_MAX])]


class Fenced:
    """Tensors between canaries, by name."""

    def __init__(self):
        self.fences = {}

    def put(self, name, t):
        g = Guarded(t.numel() * t.element_size())
        x = g.view(t.dtype, t.shape)
        x.copy_(t)
        self.fences[name] = g
        return x

    def check(self, what):
        torch.cuda.synchronize()
        for name, g in self.fences.items():
            assert g.intact(), f"{what}: written outside {name}"


def rows_of(lens, starts, T, most):
    """Rows of the packed tensors that are some sequence's tokens with a key."""
    rows = set()
    for l, a, e in zip(lens, starts, starts[1:]):
        a, e = max(a, 0), min(max(e, 0), T)
        n = min(max(e - a, 0), most - min(max(l, 0), most))
        rows |= set(range(a, a + n))
    return rows


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("lens,starts", WILD)
def test_wild_numbers_write_nothing_outside(lens, starts, dtype, d):
    """Starts that fall, as far as a whole number goes, lengths below zero and past the table, pages behind the pool: every call ends,
    nothing outside its outputs is written, and of o no row but those of tokens with a key."""
    P, Hkv, Hq, page, cols, T, layers = 40, 2, 8, 16, 12, 9, 2
    gen = torch.Generator().manual_seed(90)
    dt = pu.DT[dtype]
    f = Fenced()
    z = lambda *s: torch.randn(*s, generator=gen).to(dt)        # noqa: E731
    k, v = f.put("k", z(layers, P, Hkv, page, d)), f.put("v", z(layers, P, Hkv, page, d))
    table = torch.arange(36, dtype=torch.int32).view(3, 12)
    table[0, 0], table[1, 2], table[2, 5] = 1 << 20, -9, INT_MIN
    table, refs = f.put("table", table), f.put("refs", torch.ones(P, dtype=torch.int32))
    refs[36:] = 0
    lens_g, starts_g = pu.ints(lens).cuda(), pu.ints(starts).cuda()
    x = [z(T, n, d).cuda() for n in (Hq, Hkv, Hkv)]
    q, o = f.put("q_out", z(T, Hq, d)), f.put("o", torch.full((T, Hq, d), 7.0, dtype=dt))
    after, report = f.put("lens_out", torch.zeros(3, dtype=torch.int32)), f.put("report", torch.zeros(4, dtype=torch.int32))
    inv = torch.ones(d // 2, device="cuda")
    bits = torch.full((T, 1), -1, dtype=torch.int64, device="cuda")
    keep = pu.ints([[0, 1], [0, 0], [0, 2]]).cuda()
    flashd.cache_append(*x, q, k[0], v[0], table, lens_g, starts_g, inv_freq=inv)
    f.check("append")
    mine = rows_of(lens, starts, T, cols * page)
    other = [t for t in range(T) if t not in mine]
    for hint in HINTS:
        ws = Guarded(flashd.tree_workspace_bytes(Hq, Hkv, hint, d, flashd._DTYPE[dt]))
        for tree in (None, bits):
            flashd.attn_fwd_tree(x[0], k[0], v[0], o, table, lens_g, starts_g, hint, 0.125, tree=tree, workspace=ws.payload)
            f.check(f"attention, hint {hint}")
            assert ws.intact()
            assert (o[other] == 7).all()
    flashd.cache_commit(k, v, table, lens_g, starts_g, after, keep=keep)
    f.check("commit")
    tout, lout = f.put("table_out", torch.zeros(5, cols, dtype=torch.int32)), f.put("forked lens", torch.zeros(5, dtype=torch.int32))
    flashd.cache_fork(pu.ints([2, INT_MIN, 0, 3, INT_MAX]).cuda(), refs, table, lens_g, tout, lout)
    f.check("fork")
    assert tout[1].tolist() == [-1] * cols and lout.tolist() == [lens[2], 0, lens[0], 0, 0]
    flashd.cache_reserve(k, v, refs, table, lens_g, starts_g, report)
    f.check("reserve")


def test_columns_beyond_the_table_are_counted_without_overflow():
    """Many sequences that claim 2^31 tokens: the count of missing pages stays at the largest number."""
    B = 64
    k, v = (torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    refs = torch.zeros(4, dtype=torch.int32, device="cuda")
    table = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    starts = pu.ints([0, INT_MAX] * (B // 2) + [0]).cuda()
    report = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    flashd.cache_reserve(k, v, refs, table, lens, starts, report)
    assert report.tolist() == [INT_MAX] + [-1] * B
    lens[:] = 16                        # no room at all: every one of them is beyond
    flashd.cache_reserve(k, v, refs, table, lens, pu.ints([0, INT_MAX] + [0] * (B - 1)).cuda(), report)
    assert report.tolist() == [1 << 27] + [-1] * B
    assert not refs.any() and (table == -1).all()
