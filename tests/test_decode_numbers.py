"""Numbers that a decode-step call cannot take as they are given: refused, and neither wrapped nor cut."""

import numpy as np
import pytest

import paper_2609_38095_amd as zo


def holed_book():
    """A book whose compaction takes four moves: pages 4 .. 7 are in use, 0 .. 3 are free."""
    book = zo.ZoPages(8, 4)
    low, high = book.add(16), book.add(16)
    book.drop(low)
    return book, high


def test_compact_takes_the_room_that_it_is_given():
    """Moves are written to an array of `room` rows: none of a negative number, no more than the pages of the book."""
    for room in (-1, -2, -2 ** 31, -2 ** 32 + 1):
        book, high = holed_book()
        before = book.table([high])[0]
        with pytest.raises(zo.ZoError) as e:
            book.compact(room)
        assert e.value.status == zo.ZO_ERR_ARG and np.array_equal(book.table([high])[0], before)
    for room, moved in ((0, 0), (1, 1), (3, 3), (8, 4), (2 ** 32, 4), (2 ** 32 + 1, 4), (2 ** 62, 4)):
        book, high = holed_book()
        src, dst, rows = book.compact(room)
        assert len(src) == len(dst) == len(rows) == moved and rows.tolist() == [4] * moved
