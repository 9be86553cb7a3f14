"""The bookkeeping of a paged cache in Python lists, as flashd.h describes it, and what has to hold whatever the numbers are: the pages
that a sequence is about to write to are its own."""
from __future__ import annotations

from tests import paged_util as pu


class Pages(pu.Pages):
    """As pu.Pages, but reserving also takes back, from the first one on that another row names too, the pages behind a growing
    sequence's keys.  (pu.Pages counts those as the sequence's own, so that twins write to one page.)"""

    def room(self, b, m, page):
        """New tokens of sequence b that have a key."""
        return max(0, min(m, self.max_pages * page - self.lens[b]))

    def reserve(self, some, page):
        for b, m in enumerate(some):
            self.rows[b] = self.rows[b][:-(-(self.lens[b] + self.room(b, m, page)) // page)]
        refs = self.refs
        for b, m in enumerate(some):
            if self.room(b, m, page) > 0:
                first = -(-self.lens[b] // page)
                shared = [col for col in range(first, len(self.rows[b])) if refs[self.rows[b][col]] > 1]
                self.rows[b] = self.rows[b][:shared[0]] if shared else self.rows[b]
        return super().reserve(some, page)


def written(lens, some, page, max_pages):
    """(sequence, column) of every page that new tokens are about to be written to."""
    for b, (l, m) in enumerate(zip(lens, some)):
        last = min(l + m, max_pages * page)
        for col in range(l // page, -(-last // page) if last > l else 0):
            yield b, col


def check_own(table, refs, lens, some, page):
    """table and refs as lists: refs counts the table's entries, and no page that is about to be written to is named twice."""
    count = [0] * len(refs)
    for row in table:
        for p in row:
            if p >= 0:
                count[p] += 1
    assert count == refs
    for b, col in written(lens, some, page, len(table[0])):
        assert table[b][col] >= 0 and count[table[b][col]] == 1, (b, col, table[b])
