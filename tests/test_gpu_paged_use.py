"""The operators on a paged cache as a program meets them: every row count the attention has a kernel for with
the same hard cases, steps recorded into graphs and replayed, other streams, calls that overlap, shared pages."""
import pytest
import torch

from paper_2505_14201_amd import flashd
from tests import paged_util as pu
from tests.test_gpu_tree import check, run

pytestmark = pytest.mark.gpu

# hints whose rows, 4 to a token, choose 16, 32, 64 and 128 rows to a tile
HINTS = (1, 6, 12, 20)
TYPES = [("bf16", 128, False), ("f16", 128, False), ("bf16", 64, False), ("f16", 64, False), ("bf16", 128, True),
         ("f16", 64, True), ("f16", 128, True), ("bf16", 64, True), ("f32", 128, False), ("f32", 64, False)]


def small(dtype, d, fp8, seed, lens=(150, 3, 97), some=(21, 1, 13), page=16, **kw):
    return pu.make(list(lens), list(some), 2, d, page, dtype, fp8=fp8, seed=seed, **kw)


@pytest.mark.parametrize("dtype,d,fp8", TYPES)
@pytest.mark.parametrize("hint", HINTS)
def test_rows_of_every_kernel(hint, dtype, d, fp8):
    """Chains, trees with rows that see nothing, scales of either sign and zero, and a page missing in the middle."""
    c = small(dtype, d, fp8, seed=50)
    q = pu.queries(c, 8, dtype, seed=51)
    bits, seen = pu.random_tree(c.some, 1, seed=52, holes=True)
    for scale in (d ** -0.5, -d ** -0.5, 0.0):
        check(c, q, dtype, scale, max_q=hint)
        check(c, q, dtype, scale, bits, seen, max_q=hint)
    c.table[0, 4] = -1
    c.table[2] = -1                                     # tokens 22 .. 34 see nothing
    got = check(c, q, dtype, d ** -0.5, max_q=hint)
    assert torch.count_nonzero(got[22:]) == 0
    check(c, q, dtype, d ** -0.5, bits, seen, max_q=hint)


@pytest.mark.parametrize("dtype,d,fp8", TYPES)
@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_numbers_that_are_none(bad, hint, dtype, d, fp8):
    """A drafted token whose key and value are no numbers: who does not see it keeps its output, whose
    value column it spoils are those that see it.  Pages behind the last key hold such numbers throughout."""
    c = small(dtype, d, fp8, seed=53, lens=(75, 3), some=(21, 9))
    q = pu.queries(c, 8, dtype, seed=54)
    bits, seen = pu.random_tree(c.some, 1, seed=55, holes=False)
    o, mass, size = pu.attention(c, q, d ** -0.5, seen)
    bound = pu.attention_bound(c, dtype, o, mass, size)
    at = 75 + 13                                        # token 13 of sequence 0
    p = c.table[0].long()
    if fp8:
        c.v.view(torch.uint8)[p[at // 16], :, at % 16, 3] = 0x7f
    else:
        c.v[p[at // 16], :, at % 16, 3] = bad
    for b, (l, m) in enumerate(zip(c.lens, c.some)):
        for key in range(l + m, -(-(l + m) // 16) * 16):
            for x in (c.k, c.v):
                if fp8:
                    x.view(torch.uint8)[c.table[b, key // 16].long(), :, key % 16] = 0xff
                else:
                    x[c.table[b, key // 16].long(), :, key % 16] = bad
    got = run(c, q, d ** -0.5, bits, max_q=hint).double()
    for b, m in enumerate(c.some):
        for i in range(m):
            t = c.starts[b] + i
            spoilt = b == 0 and 13 in seen[t]
            fine = torch.ones(d, dtype=torch.bool)
            fine[3] = not spoilt
            assert ((got[t] - o[t]).abs() <= bound[t])[:, fine].all(), (b, i)
            assert not spoilt or not torch.isfinite(got[t, :, 3]).any(), (b, i)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hint", HINTS)
def test_growing_scores_of_every_kernel(hint, dtype):
    c = pu.make([900], [4], 1, 128, 32, dtype, seed=56, qk_std=4.0)
    j = torch.arange(904)
    c.k[c.table[0].long()[j // 32], :, j % 32] *= torch.linspace(0.05, 4.0, 904).view(-1, 1, 1).to(c.k.dtype)
    check(c, pu.queries(c, 4, dtype, seed=57, std=4.0), dtype, 128 ** -0.5, max_q=hint)


@pytest.mark.parametrize("Hq,Hkv,some", [(3, 1, [50, 0, 17]), (7, 1, [90]), (128, 1, [3, 5]), (5, 5, [200, 1])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_groups_that_do_not_divide_a_tile(Hq, Hkv, some, dtype):
    """Chains of many row tiles whose last rows are in the middle of a token."""
    c = pu.make([70 * (b + 1) for b in range(len(some))], some, Hkv, 64, 64, dtype, seed=58)
    check(c, pu.queries(c, Hq, dtype, seed=59), dtype, 0.125)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f32", 64)])
def test_a_shared_page_counts_for_each_who_holds_it(dtype, d):
    """One page in the tables of two sequences, and twice in one."""
    c = pu.make([64, 40], [2, 1], 2, d, 16, dtype, seed=60)
    c.table[1, :2] = c.table[0, :2]
    c.table[0, 3] = c.table[0, 1]
    check(c, pu.queries(c, 4, dtype, seed=61), dtype, d ** -0.5)


@pytest.mark.parametrize("hint", (1, 12, 20))
def test_ragged_chunks_far_longer_than_the_chip_is_wide(hint):
    """More row tiles than workgroups, of sequences that differ in length: some rows against fp64."""
    lens, some = [900, 0, 63, 2000], [700, 1000, 1, 333]
    c = pu.make(lens, some, 4, 64, 64, "bf16", seed=62)
    q = pu.queries(c, 16, "bf16", seed=63)
    got = run(c, q, 0.125, max_q=hint)
    few = [0, 1, 31, 32, 699, 700, 701, 1234, 1699, 1700, 1701, 2033]
    for t in few:                                       # a token by itself: the keys up to its own
        b = max(x for x in range(4) if c.starts[x] <= t and c.some[x] > 0)
        i = t - c.starts[b]
        one = pu.Paged(c.k, c.v, c.table[b:b + 1], [lens[b] + i], [1])
        o, mass, size = pu.attention(one, q[t:t + 1], 0.125)
        assert ((got[t:t + 1].double() - o).abs() <= pu.attention_bound(one, "bf16", o, mass, size)).all(), t


def test_as_many_sequences_as_are_allowed():
    lens = [(13 * b) % 40 for b in range(4096)]
    some = [int(b % 2 == 0) for b in range(4096)]
    c = pu.make(lens, some, 1, 64, 16, "bf16", seed=64)
    check(c, pu.queries(c, 2, "bf16", seed=65), "bf16", 0.125)


def test_reserve_in_a_pool_of_more_than_a_million_pages():
    P, page = 1 << 20 | 4097, 16
    k = torch.zeros(P, 1, page, 64, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros(P, 1, page, 64, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    refs = torch.ones(P, dtype=torch.int32, device="cuda")
    free = [5, 1 << 20, (1 << 20) + 1, P - 1]
    refs[torch.tensor(free, device="cuda")] = 0
    table = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    lens, starts = pu.ints([0, 0, 0]).cuda(), pu.ints([0, 1, 18, 19]).cuda()
    report = torch.empty(4, dtype=torch.int32, device="cuda")
    flashd.cache_reserve(k, v, refs, table, lens, starts, report)
    assert report.tolist() == [0, -1, -1, -1]
    assert table.tolist() == [[5, -1], [1 << 20, (1 << 20) + 1], [P - 1, -1]]
    assert int(refs.sum()) == P


class Loop:
    """A serving loop's tensors, fixed in place: what a recorded step reads and writes."""

    def __init__(self, seed, dtype=torch.bfloat16, layers=2, P=80, page=16, Hq=8, Hkv=2, d=64, some=(3, 1, 5)):
        gen = torch.Generator().manual_seed(seed)
        self.layers, self.some, T = layers, list(some), sum(some)
        z = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t, device="cuda")       # noqa: E731
        self.k, self.v = z(layers, P, Hkv, page, d, t=dtype), z(layers, P, Hkv, page, d, t=dtype)
        self.refs, self.lens, self.after = z(P), z(len(some)), z(len(some))
        self.table = torch.full((len(some), 12), -1, dtype=torch.int32, device="cuda")
        self.report = z(len(some) + 1)
        starts = [0]
        for m in some:
            starts.append(starts[-1] + m)
        self.starts = pu.ints(starts).cuda()
        self.x = [torch.randn(T, n, d, generator=gen).to(dtype).cuda() for n in (Hq, Hkv, Hkv)]
        self.q, self.o = z(T, Hq, d, t=dtype), z(layers, T, Hq, d, t=dtype)
        self.bits = pu.random_tree(self.some, 1, seed=seed, holes=False)[0].cuda()
        self.keep = pu.ints([[0, 1], [0, 0], [0, 2]]).cuda()
        self.n_keep = pu.ints([2, 1, 2]).cuda()
        self.inv = (100.0 ** (-torch.arange(0, d, 2).double() / d)).float().cuda()
        self.ws = z(flashd.tree_workspace_bytes(Hq, Hkv, max(some), d, flashd.BF16), t=torch.uint8)

    def step(self, stream=None):
        kw = {} if stream is None else {"stream": stream}
        flashd.cache_reserve(self.k, self.v, self.refs, self.table, self.lens, self.starts, self.report, **kw)
        for y in range(self.layers):
            flashd.cache_append(*self.x, self.q, self.k[y], self.v[y], self.table, self.lens, self.starts,
                                inv_freq=self.inv, **kw)
            flashd.attn_fwd_tree(self.q, self.k[y], self.v[y], self.o[y], self.table, self.lens, self.starts,
                                 max(self.some), 0.125, tree=self.bits, workspace=self.ws, **kw)
        flashd.cache_commit(self.k, self.v, self.table, self.lens, self.starts, self.after, keep=self.keep,
                            n_keep=self.n_keep, **kw)

    def go_on(self):
        """Between steps: the lengths, and other tokens."""
        self.lens.copy_(self.after)
        for x in self.x:
            x.copy_(x.roll(1, 0))

    def state(self):
        torch.cuda.synchronize()
        return [x.cpu().clone() for x in (self.k.view(torch.int16), self.v.view(torch.int16), self.refs, self.table,
                                          self.lens, self.after, self.report, self.o.view(torch.int16))]


def test_a_recorded_step_is_the_step():
    """Replays with other tokens and growing lengths, eager work between them, against the same steps
    one by one; two graphs of two loops replayed at once on two streams."""
    for x in (Loop(70), Loop(71)):                      # (first launches load the kernels)
        x.step()
    eager, loops = [Loop(70), Loop(71)], [Loop(70), Loop(71)]
    graphs = []
    for x in loops:
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            x.step()
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for x in eager:
            x.step()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for x, y in zip(eager, loops):
            for a, b in zip(x.state(), y.state()):
                assert torch.equal(a, b)
            x.go_on()
            y.go_on()
    assert eager[0].lens.tolist() == [10, 5, 10]


def test_a_graph_brings_its_workspace():
    x = Loop(72)
    x.step()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        with pytest.raises(flashd.FlashdError) as e:
            flashd.attn_fwd_tree(x.q, x.k[0], x.v[0], x.o[0], x.table, x.lens, x.starts, 5, 0.125)
        x.o.zero_()
    assert e.value.status == -7
    g.replay()
    torch.cuda.synchronize()


def test_other_streams_and_calls_that_overlap():
    """The same loops on streams of their own at once, the stream given or current, and workspaces of the
    library's: all as alone."""
    want = Loop(73)
    for _ in range(3):
        want.step()
        want.go_on()
    want = want.state()
    for given in (False, True):
        loops = [Loop(73) for _ in range(4)]
        streams = [torch.cuda.Stream() for _ in loops]
        torch.cuda.synchronize()
        for x in loops:
            x.ws = None
        for _ in range(3):
            for x, s in zip(loops, streams):
                if given:
                    x.step(stream=s)
                    with torch.cuda.stream(s):
                        x.go_on()
                else:
                    with torch.cuda.stream(s):
                        x.step()
                        x.go_on()
        for x in loops:
            for a, b in zip(want, x.state()):
                assert torch.equal(a, b)


@pytest.mark.parametrize("hint", HINTS)
def test_the_same_bits_again(hint):
    c = pu.make([3000, 17, 800], [5, 1, 9], 2, 128, 64, "bf16", seed=74)
    q = pu.queries(c, 8, "bf16", seed=75)
    first = run(c, q, 0.09, max_q=hint)
    for _ in range(5):
        assert torch.equal(run(c, q, 0.09, max_q=hint), first)


def test_steps_without_tokens():
    """No tokens at all, and rows of a padded batch behind the last one: they stay as they are."""
    x = Loop(76)
    x.starts.zero_()
    x.o.fill_(3)
    x.q.fill_(5)
    x.after.fill_(-1)
    x.n_keep.zero_()
    x.step()
    torch.cuda.synchronize()
    assert (x.o == 3).all() and (x.q == 5).all() and x.after.tolist() == [0, 0, 0]
    assert not x.refs.any() and not x.k.any() and x.report.tolist() == [0, -1, -1, -1]
    empty = [t[:0] for t in (x.x[0], x.x[1], x.x[2], x.q)]
    flashd.cache_append(*empty, x.k[0], x.v[0], x.table, x.lens, x.starts)
    flashd.attn_fwd_tree(empty[3], x.k[0], x.v[0], x.o[0][:0], x.table, x.lens, x.starts, 1, 0.1)
    torch.cuda.synchronize()


def test_tokens_behind_the_end_of_the_table():
    """Two columns of 16 keys: of 5 tokens behind 30 keys two have a key, as reserve says; the others' queries are
    formed, their outputs left as they were."""
    c = pu.make([30, 3], [2, 2], 2, 64, 16, "bf16", seed=78)
    q = pu.queries(pu.Paged(c.k, c.v, c.table, [30, 3], [5, 2]), 4, "bf16", seed=79)
    k, v, table, lens, _ = c.gpu()
    starts = pu.ints([0, 5, 7]).cuda()
    refs = torch.zeros(k.shape[0], dtype=torch.int32, device="cuda")
    refs[table[table >= 0].long()] = 1
    report = torch.empty(3, dtype=torch.int32, device="cuda")
    flashd.cache_reserve(k, v, refs, table, lens, starts, report)
    assert int(report[0]) == 1
    qg, out = q.cuda(), torch.full((7, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    for hint in HINTS:
        o = torch.full_like(out, 7)
        flashd.attn_fwd_tree(qg, k, v, o, table, lens, starts, hint, 0.125)
        torch.cuda.synchronize()
        assert (o[2:5] == 7).all()
        check(c, torch.cat([q[:2], q[5:]]), "bf16", 0.125, got=torch.cat([o[:2], o[5:]]).cpu())
    new = torch.ones(7, 2, 64, dtype=torch.bfloat16, device="cuda")
    flashd.cache_append(qg, new, new, out, k, v, table, lens, starts)
    torch.cuda.synchronize()
    assert torch.equal(out, qg)


def test_wild_numbers_on_the_device_stay_inside():
    """Lengths, starts and pages that no program should leave there: nothing outside the tensors is touched and the
    call ends.  (Starts that fall, lengths below zero and past the table, pages behind the pool.)"""
    for lens, starts in (([-5, 1 << 30, 7], [0, 3, 1, 9]), ([0, 0, 0], [0, -4, 2, 1 << 30]), ([190, 192, 500], [0, 3, 4, 9])):
        x = Loop(77)
        x.step()
        x.lens.copy_(pu.ints(lens))
        x.starts.copy_(pu.ints(starts))
        x.table[0, 0] = 1 << 20
        x.table[1, 2] = -9
        flashd.cache_append(*x.x, x.q, x.k[0], x.v[0], x.table, x.lens, x.starts, inv_freq=x.inv)
        for hint in HINTS:
            flashd.attn_fwd_tree(x.q, x.k[0], x.v[0], x.o[0], x.table, x.lens, x.starts, hint, 0.125, tree=x.bits)
        flashd.cache_commit(x.k, x.v, x.table, x.lens, x.starts, x.after, keep=x.keep, n_keep=x.n_keep)
        torch.cuda.synchronize()
