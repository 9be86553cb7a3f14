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
