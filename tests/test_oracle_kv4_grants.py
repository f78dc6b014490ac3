"""Who is granted what when the pool is full: written out by hand, not taken from the oracle's own rule."""
import numpy as np
import pytest

from oracle import kv4


def tables(lens, n_pages, max_pages):
    """Rows with pages 0, 1, 2, ... in turn; (page_of, len, refs)."""
    page_of, refs, at = np.full((len(lens), max_pages), -1, np.int32), np.zeros(n_pages, np.int32), 0
    for r, n in enumerate(lens):
        for c in range(-(-n // 64)):
            page_of[r, c], refs[at] = at, 1
            at += 1
    return page_of, np.array(lens, np.int32), refs


# lengths, pages, requests, offsets -> ok, slots
EXTEND = [
    ([64, 6, 6], 3, [0, 1, 2], [0, 1, 2, 3], [0, 1, 1], [-1, 1 * 64 + 6, 2 * 64 + 6]),          # a page boundary stops its own row only
    ([64, 6, 64], 3, [2, 0, 1], [0, 1, 2, 2], [0, 0, 1], [-1, -1]),                             # no tokens: nothing to refuse
    ([64, 63, 64, 1], 5, [0, 1, 2, 3], [0, 65, 66, 67, 68], [0, 1, 0, 1], [-1] * 65 + [1 * 64 + 63, -1, 3 * 64 + 1]),   # one page free, two wanted in front of row 2
    ([64, 63, 64, 1], 5, [1, 2, 0, 3], [0, 1, 2, 3, 4], [1, 1, 0, 1], [1 * 64 + 63, 4 * 64, -1, 3 * 64 + 1]),
]


@pytest.mark.parametrize("lens,n_pages,row,off,ok,slots", EXTEND)
def test_extend(lens, n_pages, row, off, ok, slots):
    page_of, length, refs = tables(lens, n_pages, 4)
    slot, got = kv4.extend(page_of, length, refs, row, off, off[-1])
    assert got.tolist() == ok and slot.tolist() == slots
    assert length.tolist() == [n + sum(b - a for r2, a, b, o in zip(row, off[:-1], off[1:], ok) if r2 == r and o) for r, n in enumerate(lens)]


# rows 0 .. 2 of lengths 64, 70, 128 in five pages, rows 3 .. 5 empty
FORK = [(5, [1, 0, 2], [3, 4, 5], [0, 1, 1]), (6, [1, 1, 2], [3, 4, 5], [1, 0, 1])]


@pytest.mark.parametrize("n_pages,src,dst,ok", FORK)
def test_fork(n_pages, src, dst, ok):
    page_of, length, refs = tables([64, 70, 128, 0, 0, 0], n_pages, 4)
    pages = np.zeros((n_pages, 1, 80 * 64), np.uint8)
    assert kv4.fork(pages, page_of, length, refs, src, dst).tolist() == ok
    held = np.bincount(page_of[page_of >= 0], minlength=n_pages)
    assert (held == refs).all()
