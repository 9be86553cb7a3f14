"""Sequences that branch, grow, keep part of what was drafted and are set back: pages and counts as the list model has them, every page
that is written to named once, and every sequence's keys and values its own."""
import random

import pytest
import torch

from paper_2505_14201_amd import flashd
from tests import paged_util as pu
from tests.pages_model import Pages, check_own

pytestmark = pytest.mark.gpu

LAYERS, HKV, D = 2, 1, 64


class World:
    """Pools whose rows hold a token's number (K) and its negative (V), and per sequence the list of its tokens."""

    def __init__(self, B, page, P, max_pages):
        self.page, self.max_pages = page, max_pages
        z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")                # noqa: E731
        self.k, self.v = (torch.zeros(LAYERS, P, HKV, page, D, device="cuda") for _ in "kv")
        self.refs, self.lens = z(P), z(B)
        self.table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
        self.model = Pages(self.table.cpu(), [0] * B, P)
        self.held = [[] for _ in range(B)]
        self.next = 1

    def fork(self, parent):
        t, l = torch.full((len(parent), self.max_pages), -9, dtype=torch.int32, device="cuda"), torch.zeros(len(parent), dtype=torch.int32, device="cuda")
        flashd.cache_fork(pu.ints(parent).cuda(), self.refs, self.table, self.lens, t, l)
        self.table, self.lens = t, l
        self.held = [list(self.held[p]) if 0 <= p < len(self.held) else [] for p in parent]
        self.model.fork(parent)
        self.agrees()

    def set_back(self, lens):
        self.model.lens = list(lens)
        self.lens = pu.ints(lens).cuda()
        self.held = [h[:l] for h, l in zip(self.held, lens)]

    def reserve(self, some):
        self.some, starts = some, [0]
        for m in some:
            starts.append(starts[-1] + m)
        self.starts, self.q_start = starts, pu.ints(starts).cuda()
        report = torch.full((len(some) + 1,), -9, dtype=torch.int32, device="cuda")
        flashd.cache_reserve(self.k, self.v, self.refs, self.table, self.lens, self.q_start, report)
        want, _ = self.model.reserve(some, self.page)
        assert report.tolist() == want
        self.agrees()
        return want[0]

    def append(self):
        """A number of its own for every new token, into every layer."""
        T = self.starts[-1]
        self.new = list(range(self.next, self.next + T))
        self.next += T
        if T:
            ids = torch.tensor(self.new, dtype=torch.float32, device="cuda").view(T, 1, 1).expand(T, HKV, D).contiguous()
            for y in range(LAYERS):
                flashd.cache_append(ids.clone(), ids + 0.25 * y, -ids - 0.25 * y, torch.empty_like(ids), self.k[y], self.v[y], self.table,
                                    self.lens, self.q_start)

    def commit(self, keep):
        most = max([len(x) for x in keep] + [1])
        out = torch.full_like(self.lens, -9)
        flashd.cache_commit(self.k, self.v, self.table, self.lens, self.q_start, out,
                            keep=pu.ints([x + [0] * (most - len(x)) for x in keep]).cuda(), n_keep=pu.ints([len(x) for x in keep]).cuda())
        self.lens = out
        for b, x in enumerate(keep):
            self.held[b] += [self.new[self.starts[b] + i] for i in x]
        self.model.lens = [len(h) for h in self.held]

    def agrees(self):
        assert self.table.tolist() == self.model.table.tolist()
        assert self.lens.tolist() == self.model.lens
        assert self.refs.tolist() == self.model.refs

    def contents(self, new=False, without=()):
        """Every sequence's tokens (with those just appended) are in its pages."""
        b = [x for x, h in enumerate(self.held) for _ in range(len(h) + new * self.some[x]) if x not in without]
        j = [i for x, h in enumerate(self.held) for i in range(len(h) + new * self.some[x]) if x not in without]
        ids = [t for x, h in enumerate(self.held) if x not in without
               for t in h + (self.new[self.starts[x]:self.starts[x + 1]] if new else [])]
        b, j, ids = (torch.tensor(x, dtype=torch.long, device="cuda") for x in (b, j, ids))
        p = self.table.long()[b, j // self.page]
        assert (p >= 0).all()
        for y in range(LAYERS):
            assert (self.k[y, p, :, j % self.page] == (ids + 0.25 * y).view(-1, 1, 1)).all()
            assert (self.v[y, p, :, j % self.page] == -(ids + 0.25 * y).view(-1, 1, 1)).all()


def fails(w, some):
    """Reserving finds too few pages, and the rest of the step runs on: nobody's keys change."""
    assert w.reserve(some) > 0
    check_own(w.table.tolist(), w.refs.tolist(), w.lens.tolist(), some, w.page, missing=True)
    w.append()
    w.contents(without=w.model.held_back(w.page))
    q = torch.randn(max(w.starts[-1], 1), HKV, D, device="cuda")
    for hint in (1, 20):
        flashd.attn_fwd_tree(q, w.k[0], w.v[0], torch.empty_like(q), w.table, w.lens, w.q_start, hint, 0.1)
    flashd.cache_commit(w.k, w.v, w.table, w.lens, w.q_start, torch.empty_like(w.lens),
                        keep=torch.tensor([[0, 1]] * len(some), dtype=torch.int32, device="cuda") + 1)
    w.contents(without=w.model.held_back(w.page))


def step(w, some, keep):
    assert w.reserve(some) == 0
    check_own(w.table.tolist(), w.refs.tolist(), w.lens.tolist(), some, w.page)
    w.append()
    w.contents(new=True)
    w.commit(keep)
    w.contents()


@pytest.mark.parametrize("B,page,P,max_pages", [(3, 16, 80, 8), (17, 32, 500, 20), (70, 16, 9000, 30), (1500, 16, 70000, 25)])
def test_lives_of_sequences(B, page, P, max_pages):
    rng = random.Random(B + 1)
    w = World(B, page, P, max_pages)
    for turn in range(8):
        if turn:
            parent = [rng.choice([b, b, b, rng.randrange(B), -1]) for b in range(B)]
            if turn == 3:
                parent = [rng.randrange(B) for _ in range(B + 5)]
                B += 5
            w.fork(parent)
        if turn % 3 == 2:
            w.set_back([rng.randint(0, l) if rng.random() < 0.3 else l for l in w.model.lens])
        some = [rng.choice([0, 1, 1, 2, rng.randint(0, 2 * page)]) for _ in range(B)]
        some = [min(m, max_pages * page - l) for m, l in zip(some, w.model.lens)]
        step(w, some, [sorted(rng.sample(range(m), rng.randint(0, m))) for m in some])


@pytest.mark.parametrize("keys,drafts,kept,then", [(15, 4, 1, 1), (16, 4, 0, 2), (20, 30, 1, 16), (20, 16, 0, 16), (33, 40, 0, 7), (0, 40, 0, 5), (48, 1, 0, 1)])
def test_twins_of_a_sequence_with_pages_left_over(keys, drafts, kept, then):
    """Branching right after part of the drafts was dropped: what is left over is nobody's to share."""
    w = World(2, 16, 40, 8)
    step(w, [keys, 3], [list(range(keys)), [0, 1, 2]])
    step(w, [drafts, 1], [list(range(kept)), []])
    w.fork([0, 1, 0, 0])
    step(w, [then, 1, then, 0], [list(range(then)), [0], list(range(then)), []])
    step(w, [1, 1, 1, 1], [[0], [0], [0], [0]])


def test_a_twin_that_is_set_back():
    """One twin's length falls to an earlier page, and to the middle of the page both are in: it must not write over the other's keys."""
    w = World(1, 16, 40, 8)
    step(w, [70], [list(range(70))])
    w.fork([0, 0, 0, 0])
    w.set_back([70, 32, 20, 66])
    step(w, [1, 40, 40, 9], [[0], list(range(0, 40, 3)), [], list(range(9))])
    w.fork([3, 2, 1, 0])
    w.set_back([0, 5, 16, 70])
    step(w, [100, 3, 20, 1], [[0], [0], list(range(20)), []])


def test_shared_pages_behind_the_keys_of_long_rows():
    """Hundreds of left-over columns, the first shared one in their middle."""
    w = World(2, 16, 3000, 520)
    step(w, [5, 8000], [[0], list(range(8000))])
    w.fork([0, 1, 1])
    w.set_back([1, 8000, 3000])
    w.reserve([0, 0, 1000])                     # sequence 2 takes pages of its own behind key 3000
    w.fork([0, 1, 2, 2])
    w.set_back([1, 8000, 3000, 40])
    step(w, [1, 1, 4000, 6000], [[0], [0], list(range(0, 4000, 7)), []])


def test_a_failed_reserve_holds_shared_pages_back():
    """Three twins of 20 keys and one free page: none writes to the page they share, however often the step is run; without the third
    there is enough, and all keys are there."""
    w = World(1, 16, 3, 3)
    step(w, [20], [list(range(20))])
    w.fork([0, 0, 0])
    was = w.k.clone(), w.v.clone()
    for _ in range(3):
        fails(w, [1, 2, 3])
        assert w.table.tolist() == [[0, -3, -1]] * 3
        assert torch.equal(w.k, was[0]) and torch.equal(w.v, was[1])
    w.fork([0, 1, -1])
    step(w, [1, 1, 0], [[0], [0], []])


def test_a_twin_that_rests_keeps_its_keys_beside_a_failed_reserve():
    """No free page: a twin set back into the middle of the page would write over a key of the one that rests."""
    w = World(1, 16, 2, 3)
    step(w, [20], [list(range(20))])
    w.fork([0, 0])
    w.set_back([20, 18])
    fails(w, [0, 1])
    w.contents(without={1})
    w.reserve([0, 0])                           # taken up again without new tokens
    w.contents()
    w.fork([-1, 1])
    step(w, [0, 3], [[], [0, 2]])


def test_pages_held_back_branch_and_go_back_like_others():
    w = World(2, 16, 4, 5)
    step(w, [20, 5], [list(range(20)), list(range(5))])
    w.fork([0, 0, 1])
    fails(w, [1, 1, 30])
    w.fork([1, 0, 0, 2])
    fails(w, [1, 1, 20, 1])
    w.set_back([10, 20, 0, 5])                  # the held back column lies behind the keys, or all of them go
    w.reserve([0, 1, 0, 1])
    w.contents()
    w.fork([1, 3])
    step(w, [14, 1], [[0], [0]])
    w.fork([0, 0])
    fails(w, [0, 100])                          # columns are missing: the page that both hold is held back as well
    assert w.model.held_back(16) == {1}
    step(w, [0, 1], [[], [0]])


@pytest.mark.parametrize("B,page,P,max_pages", [(6, 16, 7, 6), (40, 32, 42, 8), (1100, 16, 1200, 8)])
def test_lives_in_a_pool_that_is_too_small(B, page, P, max_pages):
    rng = random.Random(B + 2)
    w, failed = World(B, page, P, max_pages), 0
    for _ in range(14):
        w.fork([rng.choice([b, b, b, rng.randrange(B), -1]) for b in range(B)])
        if rng.random() < 0.3:
            w.set_back([rng.randint(0, l) if rng.random() < 0.3 else l for l in w.model.lens])
        some = [rng.choice([0, 1, 2, rng.randint(0, 2 * page)]) for _ in range(B)]
        some = [min(m, max_pages * page - l + rng.choice([0, 0, 0, 5])) for m, l in zip(some, w.model.lens)]
        trial = Pages(w.table.cpu(), w.model.lens, P)
        trial.rows = [list(r) for r in w.model.rows]
        if trial.reserve(some, page)[0][0]:
            failed += 1
            fails(w, some)
        else:
            step(w, some, [sorted(rng.sample(range(m), rng.randint(0, m))) for m in some])
    assert 3 < failed < 14


def test_keys_without_pages_get_them():
    """Lengths that the rows have no pages for: a sequence that grows gets the pages of its keys as well, and its tokens have one."""
    P, page, lens, some = 40, 16, [20, 32, 5, 0, 64, 50, 49, 3, 16], [5, 1, 0, 3, 40, 2, 1, 2, 0]
    table = torch.full((9, 8), -1, dtype=torch.int32)
    table[4, :2], table[5, :3], table[6, :4] = pu.ints([30, 31]), pu.ints([32, 33, 34]), pu.ints([35, 36, 37, 38])
    model = Pages(table, lens, P)
    starts = [0]
    for m in some:
        starts.append(starts[-1] + m)
    k, v = (torch.zeros(1, P, HKV, page, D, device="cuda") for _ in "kv")
    refs, tab, lens_g, q_start = pu.ints(model.refs).cuda(), table.cuda(), pu.ints(lens).cuda(), pu.ints(starts).cuda()
    report = torch.zeros(10, dtype=torch.int32, device="cuda")
    flashd.cache_reserve(k, v, refs, tab, lens_g, q_start, report)
    want, _ = model.reserve(some, page)
    assert report.tolist() == want == [0] + [-1] * 9
    assert tab.tolist() == model.table.tolist() and refs.tolist() == model.refs
    check_own(tab.tolist(), refs.tolist(), lens, some, page)
    x = torch.ones(starts[-1], HKV, D, device="cuda")
    flashd.cache_append(x, x.clone(), x.clone(), torch.empty_like(x), k[0], v[0], tab, lens_g, q_start)
    assert int(k.sum()) == starts[-1] * HKV * D and int(v.sum()) == starts[-1] * HKV * D
