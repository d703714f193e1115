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


def refused(call, *args, **kw):
    with pytest.raises(zo.ZoError) as e:
        call(*args, **kw)
    assert e.value.status == zo.ZO_ERR_ARG


def test_page_ids_are_whole_numbers_of_32_bits():
    """2^32 + 1 is not page 1, and neither is 1.5 (a call without caches copies nothing, and is checked all the same)."""
    for bad in ([2 ** 32 + 1], np.array([2 ** 32 + 1]), np.array([-2 ** 32]), np.array([2 ** 31]), np.array([2 ** 64 - 1], np.uint64), [2 ** 70],
                [1.5], np.array([1.5]), np.array([2.0 ** 32]), [float("nan")], [float("inf")]):
        for args in ((bad, [2]), ([2], bad), ([2], [3], bad)):
            refused(zo.zo_cache_copy, [], [], *args)
    for good in ([1], (1,), np.array([1]), np.array([1], np.uint8), np.array([1, 7])[:1], np.array([1.0]), range(1, 2), []):
        zo.zo_cache_copy([], [], good, good, good)
    zo.zo_cache_copy([], [], [1], [2])


def test_counts_and_sequences_fit_32_bits():
    book = zo.ZoPages(8, 4)
    a = book.add(6)
    for wide in (2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 64 + 1, -1):
        for call in (book.add, book.fork, book.drop, book.extend, lambda n: book.extend(a, n), lambda n: book.table([n]),
                     lambda n: book.table(np.array([n])), lambda n: book.table([a, n], width=4)):
            refused(call, wide)
        assert book.length(wide) == -1 and book.length(a) == 6 and book.left() == 6
        for args in ((wide, 4), (8, wide)):
            with pytest.raises(ValueError):
                zo.ZoPages(*args)
        refused(zo.zo_rotary_turns, wide + 64)
    refused(book.table, [0.5])
    ids, lengths = book.table(np.array([a], np.int64))
    assert lengths.tolist() == [6] and book.table([])[0].shape == (0, 1)


def test_host_arrays_may_be_strided():
    """Columns of an array of moves, every other frequency: taken as numbers, whatever lies between them."""
    moves = np.array([[1, 2, 4], [3, 5, 4]], np.int32)
    zo.zo_cache_copy([], [], *moves.T)
    zo.zo_cache_copy([], [], moves[::-1, 0], moves[::-1, 1])
    from paper_2609_38095_amd import decode
    turns = np.arange(8.0)
    for view in (turns[::2], turns[::-1]):
        got = decode._doubles(view)
        assert np.array_equal(got, view) and got.flags.c_contiguous
        memoryview(got).cast("B")  # as the binding reads it
    assert decode._doubles(turns) is turns
    assert all(decode._int32s(c).flags.c_contiguous and np.array_equal(decode._int32s(c), c) for c in moves.T)
