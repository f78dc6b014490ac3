"""Grants of pages on the GPU when the pool is full, against results written out by hand."""
import gc

import pytest
import torch

from tests.test_oracle_kv4_grants import EXTEND, FORK, tables
from tests.test_serving_kv4 import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def cache(lens, n_pages):
    c = Cache(n_pages, 1, 64, len(lens), 4)
    c.page_of[:], c.len[:], c.refs[:] = tables(lens, n_pages, 4)
    c.push()
    return c


@pytest.mark.parametrize("lens,n_pages,row,off,ok,slots", EXTEND)
def test_extend(lens, n_pages, row, off, ok, slots):
    c = cache(lens, n_pages)
    want, slot = c.extend(row, off)                 # (compares ok and slots with the oracle's, which the hand-written ones pin)
    assert want.tolist() == slots and slot.cpu().tolist()[:len(slots)] == slots
    c.check()


@pytest.mark.parametrize("n_pages,src,dst,ok", FORK)
def test_fork(n_pages, src, dst, ok):
    c = cache([64, 70, 128, 0, 0, 0], n_pages)
    assert c.fork(src, dst).tolist() == ok
    c.check()


def test_a_decode_step_with_a_full_pool():
    """1024 rows, one token each: those on a page's edge are refused, wherever they stand in the call, all others go on."""
    lens = [64 if i % 3 == 0 else 5 + i % 50 for i in range(1024)]
    c = cache(lens, 1024)
    c.extend(range(1024), range(1025))
    assert c.len.tolist() == [n + (n != 64) for n in lens]
    c.check()
