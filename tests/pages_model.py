"""The bookkeeping of a paged cache in Python lists, as flashd.h describes it, and what has to hold whatever the numbers are: the pages
that a sequence is about to write to are its own."""
from __future__ import annotations

from tests import paged_util as pu


def named(entry):
    """The page that an entry of the table names: held back ones are -2 - page."""
    return -2 - entry if entry < -1 else entry


class Pages(pu.Pages):
    """As pu.Pages, but reserving also takes back, from the first one on that another row names too, the pages behind a growing
    sequence's keys (pu.Pages counts those as the sequence's own, so that twins write to one page), and where it fails holds back the
    shared part-filled pages of those that would write to them."""

    @property
    def refs(self):
        n = [0] * self.P
        for row in self.rows:
            for p in row:
                n[named(p)] += 1
        return n

    def held_back(self, page):
        """The sequences whose last page is held back."""
        return {b for b, l in enumerate(self.lens) if l % page and l // page < len(self.rows[b]) and self.rows[b][l // page] < -1}

    def room(self, b, m, page):
        """New tokens of sequence b that have a key."""
        return max(0, min(m, self.max_pages * page - self.lens[b]))

    def reserve(self, some, page):
        for b in self.held_back(page):
            self.rows[b][self.lens[b] // page] = named(self.rows[b][self.lens[b] // page])
        for b, m in enumerate(some):
            self.rows[b] = self.rows[b][:-(-(self.lens[b] + self.room(b, m, page)) // page)]
        refs = self.refs
        for b, m in enumerate(some):
            if self.room(b, m, page) > 0:
                first = -(-self.lens[b] // page)
                shared = [col for col in range(first, len(self.rows[b])) if self.rows[b][col] < 0 or refs[self.rows[b][col]] > 1]
                self.rows[b] = self.rows[b][:shared[0]] if shared else self.rows[b]
        report, copies = super().reserve(some, page)
        if report[0]:
            refs = self.refs
            for b, m in enumerate(some):
                l = self.lens[b]
                if self.room(b, m, page) > 0 and l % page and l // page < len(self.rows[b]) and refs[self.rows[b][l // page]] > 1:
                    self.rows[b][l // page] = -2 - self.rows[b][l // page]
        return report, copies


def written(lens, some, page, max_pages):
    """(sequence, column) of every page that new tokens are about to be written to."""
    for b, (l, m) in enumerate(zip(lens, some)):
        last = min(l + m, max_pages * page)
        for col in range(l // page, -(-last // page) if last > l else 0):
            yield b, col


def check_own(table, refs, lens, some, page, missing=False):
    """table and refs as lists: refs counts the table's entries, and no page that is about to be written to is named twice.  missing:
    reserve has reported so, and some have no page to write to."""
    count = [0] * len(refs)
    for row in table:
        for p in row:
            if p != -1:
                count[named(p)] += 1
    assert count == refs
    for b, col in written(lens, some, page, len(table[0])):
        assert missing if table[b][col] < 0 else count[table[b][col]] == 1, (b, col, table[b])
