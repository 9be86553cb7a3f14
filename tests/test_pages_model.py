"""The list model of the paged cache on the CPU: what has to hold whatever the numbers are, over many random lives."""
import random

import pytest

from tests import paged_util as pu
from tests.pages_model import Pages, check_own


def life(model, B, page, max_pages, seed, steps=12):
    rng = random.Random(seed)
    for _ in range(steps):
        parent = [rng.choice([b, b, rng.randrange(B), -1]) for b in range(B)]
        model.fork(parent)
        if rng.random() < 0.5:                          # some lengths are set back
            model.lens = [rng.randint(0, l) if rng.random() < 0.3 else l for l in model.lens]
        some = [rng.choice([0, 1, 2, rng.randint(0, 3 * page)]) for _ in range(B)]
        some = [min(m, max_pages * page - l) for m, l in zip(some, model.lens)]
        was = list(model.lens)
        report, copies = model.reserve(some, page)
        yield report, copies, was, some
        if report[0] == 0:
            model.lens = [l + rng.randint(0, m) for l, m in zip(model.lens, some)]


@pytest.mark.parametrize("seed", range(20))
def test_what_is_written_to_is_the_sequences_own(seed):
    page, max_pages, B = 16, 12, 6
    model = Pages(pu.ints([[-1] * max_pages] * B), [0] * B, 200)
    for report, copies, lens, some in life(model, B, page, max_pages, seed):
        assert report[0] == 0
        check_own(model.table.tolist(), model.refs, lens, some, page)
        assert {b for b, *_ in copies} == {b for b in range(B) if report[1 + b] >= 0}


def test_twins_of_a_sequence_with_pages_left_over():
    """15 keys, 4 drafted, 1 kept: a page is left over.  Two twins that both go on get one each."""
    model = Pages(pu.ints([[-1] * 3]), [0], 12)
    model.reserve([15], 16)
    model.lens = [15]
    model.reserve([4], 16)
    model.lens = [16]
    model.fork([0, 0])
    report, copies = model.reserve([1, 1], 16)
    assert report == [0, -1, -1] and copies == [] and model.rows == [[0, 1], [0, 2]] and model.refs[:4] == [2, 1, 1, 0]


@pytest.mark.parametrize("seed", range(20))
def test_nothing_shared_is_written_to_where_pages_are_missing(seed):
    """A pool that is too small most of the time: sequences end at random and calls are made again."""
    page, max_pages, B = 16, 6, 6
    model = Pages(pu.ints([[-1] * max_pages] * B), [0] * B, 7)
    failed = held = 0
    for report, copies, lens, some in life(model, B, page, max_pages, seed, steps=40):
        failed += report[0] > 0
        held += len(model.held_back(page))
        assert not model.held_back(page) or report[0] > 0
        check_own(model.table.tolist(), model.refs, lens, some, page, missing=report[0] > 0)
    assert failed > 3


def test_a_shared_page_is_held_back_until_there_are_enough():
    """Three twins of 20 keys and one free page, two copies wanted: all three are held back; without the third there is enough."""
    model = Pages(pu.ints([[-1] * 3]), [0], 3)
    model.reserve([20], 16)
    model.lens = [20]
    model.fork([0, 0, 0])
    for _ in range(2):
        assert model.reserve([1, 1, 1], 16) == ([1, -1, -1, -1], [])
        assert model.rows == [[0, -3]] * 3 and model.refs == [3, 3, 0] and model.held_back(16) == {0, 1, 2}
    model.fork([0, 1, -1])
    assert model.refs == [2, 2, 0]
    assert model.reserve([1, 1, 0], 16) == ([0, -1, 1, -1], [(1, 1, 2, 4)])
    assert model.rows == [[0, 1], [0, 2], []] and model.refs == [2, 1, 1]
