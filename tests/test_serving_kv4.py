"""The paged 4-bit key/value cache on the GPU against its oracle: codes and tables equal bit for bit."""
import gc

import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2609_24270_b200 import binding as ag
from paper_2609_24270_b200 import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()



def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy((a.view(np.int16) if a.dtype == np.uint16 else a).copy()).cuda()


class Cache:
    """Pages and tables on both sides."""

    def __init__(self, n_pages, H_kv, D, rows, max_pages, seed=0):
        rng = np.random.default_rng(seed)
        self.D = D
        self.pages = rng.integers(0, 256, (n_pages, H_kv, 80 * D)).astype(np.uint8)
        self.page_of = np.full((rows, max_pages), -1, np.int32)
        self.len = np.zeros(rows, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.d = {k: dev(getattr(self, k)) for k in ("pages", "page_of", "len", "refs")}
        self.bind()

    def bind(self):
        d = self.d
        self.pool = ag.KV4Pool(d["pages"].data_ptr(), self.pages.shape[0], self.pages.shape[1], self.D)
        self.table = ag.KV4Table(d["page_of"].data_ptr(), d["len"].data_ptr(), d["refs"].data_ptr(), *self.page_of.shape)

    def push(self):
        """The host's state to the device."""
        for k in self.d:
            self.d[k].copy_(torch.from_numpy(getattr(self, k)))

    def check(self):
        torch.cuda.synchronize()
        for k in ("page_of", "len", "refs", "pages"):
            assert (self.d[k].cpu().numpy() == getattr(self, k)).all(), k

    def extend(self, row, new_off, n_tokens=None, stream=0):
        n_tokens = int(new_off[-1]) if n_tokens is None else n_tokens
        d_row, d_off = dev(np.asarray(row, np.int32)), dev(np.asarray(new_off, np.int32))
        slot = torch.full((max(n_tokens, 1),), -7, dtype=torch.int32, device="cuda")
        ok = torch.full((len(row),), -7, dtype=torch.int32, device="cuda")
        ag.kv4_extend(self.pool, self.table, d_row.data_ptr(), d_off.data_ptr(), len(row), slot.data_ptr(), n_tokens, ok.data_ptr(), stream)
        torch.cuda.synchronize()
        want_slot, want_ok = kv4.extend(self.page_of, self.len, self.refs, list(row), list(new_off), n_tokens)
        assert (ok.cpu().numpy() == want_ok).all()
        assert (slot.cpu().numpy()[:n_tokens] == want_slot).all()
        return want_slot, slot

    def fork(self, src, dst):
        d_src, d_dst = dev(np.asarray(src, np.int32)), dev(np.asarray(dst, np.int32))
        ok = torch.full((len(src),), -7, dtype=torch.int32, device="cuda")
        ag.kv4_fork(self.pool, self.table, d_src.data_ptr(), d_dst.data_ptr(), len(src), ok.data_ptr())
        torch.cuda.synchronize()
        want = kv4.fork(self.pages, self.page_of, self.len, self.refs, src, dst)
        assert (ok.cpu().numpy() == want).all()
        return want

    def free(self, row):
        d_row = dev(np.asarray(row, np.int32))
        ag.kv4_free(self.pool, self.table, d_row.data_ptr(), len(row))
        torch.cuda.synchronize()
        kv4.free(self.page_of, self.len, self.refs, row)

    def compact(self):
        moved = torch.full((self.pages.shape[0],), -7, dtype=torch.int32, device="cuda")
        ag.kv4_compact(self.pool, self.table, moved.data_ptr())
        torch.cuda.synchronize()
        assert (moved.cpu().numpy() == kv4.compact(self.pages, self.page_of, self.refs)).all()


def special_rows(n, H, D, seed):
    """Rows with wide and narrow groups, equal elements, halves of steps, values that are not finite, the largest bf16."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, H, D)).astype(np.float32) * np.exp(rng.standard_normal((n, H, 1)) * 4).astype(np.float32)
    if n > 4:
        x[0, 0, :32] = 2.5
        x[1, 0, :32] = np.arange(32) * 0.5          # steps of one: every second value is half way between two codes
        x[2, H - 1, 3] = np.inf
        x[3, H - 1, 5] = np.nan
        x[4, 0, :32] = 3.3e38 * np.sign(rng.standard_normal(32))
        x[4, 0, 32:] *= 1e-38
    return kv4.bf16_bits(kv4.f32_to_bf16_value(x))


@pytest.mark.parametrize("H_kv,D,n", [(2, 128, 1), (2, 128, 67), (1, 64, 5), (3, 64, 130), (8, 128, 33)])
def test_store_and_load_bit_for_bit(H_kv, D, n):
    c = Cache(5, H_kv, D, 1, 1)
    K, V = special_rows(n, H_kv, D, 1), special_rows(n, H_kv, D, 2)
    rng = np.random.default_rng(3)
    slot = rng.permutation(5 * 64)[:n].astype(np.int32)
    if n > 10:
        slot[[3, 7, 9]] = [-1, 5 * 64, 1 << 30]     # skipped
    width = H_kv * D
    fused = dev(np.concatenate([K.reshape(n, width), np.zeros((n, 8), np.uint16), V.reshape(n, width)], 1))   # parts of a wider row
    d_slot = dev(slot)
    stride = 2 * width + 8
    ag.kv4_store(c.pool, fused.data_ptr(), fused.data_ptr() + 2 * (width + 8), d_slot.data_ptr(), n, stride, stride)
    kv4.store(c.pages, D, K, V, slot)
    c.check()
    back = torch.full((2, n, H_kv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    ag.kv4_load(c.pool, d_slot.data_ptr(), n, back[0].data_ptr(), back[1].data_ptr())
    torch.cuda.synchronize()
    live = [i for i in range(n) if 0 <= slot[i] < 5 * 64]
    for got, want in zip(back.float().cpu().numpy(), kv4.load(c.pages, D, slot[live])):
        with np.errstate(over="ignore"):
            # s * code + lo is rounded to 32 bits (the product is exact) and then to bf16
            want = kv4.f32_to_bf16_value(np.where(np.isnan(want), 0, want).astype(np.float32)) + np.where(np.isnan(want), np.nan, 0)
        assert np.array_equal(got[live], want.astype(np.float32), equal_nan=True)
        assert (np.delete(got, live, 0) == 7.0).all()


@pytest.mark.parametrize("D", [64, 128])
def test_large_calls_equal_small_ones(D):
    """Calls with several rows per lane (the last block not full) against the same rows in small calls, which the test above pins."""
    H, n_pages = 2, 600
    n = n_pages * 64 - 5
    c = Cache(n_pages, H, D, 1, 1)
    gen = torch.Generator(device="cuda").manual_seed(D)
    K, V = (torch.randn(n, H, D, device="cuda", generator=gen).bfloat16() for _ in range(2))
    slot = torch.randperm(n_pages * 64, device="cuda", generator=gen)[:n].int()
    slot[::97] = -1
    ag.kv4_store(c.pool, K.data_ptr(), V.data_ptr(), slot.data_ptr(), n)
    once = c.d["pages"].clone()
    c.d["pages"].copy_(torch.from_numpy(c.pages))
    step = 1000
    for i in range(0, n, step):
        ag.kv4_store(c.pool, K[i:].data_ptr(), V[i:].data_ptr(), slot[i:].data_ptr(), min(step, n - i))
    assert torch.equal(once, c.d["pages"])
    back, parts = torch.full((2, n, H, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((2, n, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    ag.kv4_load(c.pool, slot.data_ptr(), n, back[0].data_ptr(), back[1].data_ptr())
    for i in range(0, n, step):
        ag.kv4_load(c.pool, slot[i:].data_ptr(), min(step, n - i), parts[0, i:].data_ptr(), parts[1, i:].data_ptr())
    assert torch.equal(back, parts) and (back[:, ::97] == 7.0).all() and (back[0, 1:90] - K[1:90]).abs().max() < 0.6


def test_tables_follow_the_oracle_through_a_long_history():
    rng = np.random.default_rng(5)
    c = Cache(40, 2, 64, 12, 9)
    for step in range(40):
        kind = rng.integers(0, 4)
        if kind <= 1:
            n = int(rng.integers(1, 6))
            rows = rng.integers(-1, 13, n) if step % 5 == 0 else rng.permutation(12)[:n]      # now and then bad rows and repeats
            c.extend(rows, np.concatenate([[0], np.cumsum(rng.integers(0, 200, n))]))
        elif kind == 2:
            n = int(rng.integers(1, 5))
            c.fork(rng.integers(-1, 13, n) if step % 5 == 0 else rng.integers(0, 12, n), rng.integers(0, 12, n))
        else:
            c.free(rng.integers(-1, 13, int(rng.integers(1, 4))) if step % 2 else rng.permutation(12)[:2])
        c.check()
        if step % 4 == 3:
            c.compact()
            c.check()


def test_the_first_and_last_page_and_a_full_pool():
    c = Cache(3, 1, 64, 4, 3)
    c.extend([0, 1], [0, 64, 193])          # one page and three: four are not there, the second is refused
    assert c.len.tolist() == [64, 0, 0, 0]
    c.extend([1], [0, 128])                 # the last two
    c.extend([2], [0, 1])                   # none left
    c.extend([2, 0], [0, 1, 1])             # refused, and granted without tokens
    c.check()
    assert c.fork([1, 0], [2, 3]).tolist() == [1, 1]       # full pages only: nothing to copy
    c.free([0, 0, 1])                       # named twice: given up once
    c.check()
    c.extend([0], [0, 64])                  # still no page: the forks hold them
    c.free([2, 3])
    c.compact()
    c.check()
    assert not c.refs.any()
    c.extend([3], [5, 70], n_tokens=80)     # tokens in front of and behind the requests have no slot
    c.check()


def test_many_pages_rows_and_tokens():
    """More pages than threads of the allocating block, 1024 requests in a call, slots written by the second kernel, long rows."""
    rng = np.random.default_rng(9)
    c = Cache(5000, 1, 64, 1200, 300)
    c.refs[rng.permutation(5000)[:2000]] = 1
    c.push()
    rows = rng.permutation(1200)[:1024]
    c.extend(rows, np.concatenate([[0], np.cumsum(rng.integers(0, 100, 1024))]))
    c.check()
    c.extend(rows[:3], [0, 9000, 9000, 19000])
    c.check()
    empty = [r for r in range(1200) if c.len[r] == 0]
    c.fork(rng.choice(rows, len(empty)), empty)
    c.check()
    c.refs[c.refs == 1] = 0                  # the pages set aside above leave holes; so do some rows
    held = np.bincount(c.page_of[c.page_of >= 0], minlength=5000).astype(np.int32)
    c.refs[:] = held
    c.push()
    c.free(rows[100:700])
    c.compact()
    c.check()


@pytest.mark.parametrize("n_pages", [31, 32, 33, 1023, 4097, 131072, 131073, 200000])
def test_pools_of_every_size(n_pages):
    """Free pages scattered over small and large pools: dealt in ascending order, and closed up again.  Contents: a page's first word is its number."""
    rng = np.random.default_rng(n_pages)
    rows, max_pages = 40, n_pages // 8 + 2
    pages = torch.zeros(n_pages, ag.kv4_page_bytes(1, 64) // 4, dtype=torch.int32, device="cuda")
    pages[:, 0] = torch.arange(n_pages, device="cuda")
    pages[:, -1] = -pages[:, 0]
    refs = (rng.random(n_pages) < 0.6).astype(np.int32)
    refs[n_pages // 3: n_pages // 2] = 0
    page_of, length = np.full((rows, max_pages), -1, np.int32), np.zeros(rows, np.int32)
    used = np.flatnonzero(refs)[: max_pages]
    page_of[0, : len(used)] = used
    length[0] = 64 * len(used)
    want_page_of, want_len, want_refs = page_of.copy(), length.copy(), refs.copy()
    d_page_of, d_len, d_refs = dev(page_of), dev(length), dev(refs)
    pool, table = ag.KV4Pool(pages.data_ptr(), n_pages, 1, 64), ag.KV4Table(d_page_of.data_ptr(), d_len.data_ptr(), d_refs.data_ptr(), rows, max_pages)
    grow = np.arange(1, rows, dtype=np.int32)
    off = np.concatenate([[0], np.cumsum(rng.integers(0, 64 * max(2, n_pages // 150), rows - 1))]).astype(np.int32)
    d_row, d_off, slot, ok = dev(grow), dev(off), torch.empty(int(off[-1]), dtype=torch.int32, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    ag.kv4_extend(pool, table, d_row.data_ptr(), d_off.data_ptr(), rows - 1, slot.data_ptr(), int(off[-1]), ok.data_ptr())
    want_slot, want_ok = kv4.extend(want_page_of, want_len, want_refs, list(grow), list(off), int(off[-1]))
    torch.cuda.synchronize()
    assert (ok.cpu().numpy()[: rows - 1] == want_ok).all() and (slot.cpu().numpy() == want_slot).all()
    for d, w in ((d_page_of, want_page_of), (d_len, want_len), (d_refs, want_refs)):
        assert (d.cpu().numpy() == w).all()
    moved = torch.full((n_pages,), -7, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    ag.kv4_compact(pool, table, moved.data_ptr())
    torch.cuda.synchronize()
    held = np.flatnonzero(want_refs > 0)
    n_used = len(held)
    want = np.full(n_pages, -1, np.int32)
    want[held[held < n_used]] = held[held < n_used]
    holes = np.flatnonzero(want_refs[:n_used] <= 0)
    want[held[held >= n_used]] = holes
    assert (moved.cpu().numpy() == want).all()
    back = np.zeros(n_pages, np.int64)
    back[want[held]] = held
    assert (pages[:n_used, 0].cpu().numpy() == back[:n_used]).all() and (pages[:n_used, -1].cpu().numpy() == -back[:n_used]).all()
    want_page_of[want_page_of >= 0] = want[want_page_of[want_page_of >= 0]]
    assert (d_page_of.cpu().numpy() == want_page_of).all()
    after = np.zeros(n_pages, np.int32)
    after[:n_used] = want_refs[back[:n_used]]
    assert (d_refs.cpu().numpy() == after).all()


@pytest.mark.parametrize("H_kv,D", [(1, 64), (8, 128)])
def test_other_layers_follow_by_copies(H_kv, D):
    """Two buffers under one table: what fork and compact do to the first, ag_kv4_copy does to the second."""
    c, other = Cache(30, H_kv, D, 6, 6, seed=1), Cache(30, H_kv, D, 1, 1, seed=2)
    c.extend([0, 1, 2, 3], [0, 100, 164, 400, 420])
    before = other.pages.copy()
    c.fork([0, 2, 2], [4, 5, 0])                    # (row 0 is not empty: refused)
    src = [int(c.page_of[0, 1]), int(c.page_of[2, 3]), -1, 30, 7]
    dst = [int(c.page_of[4, 1]), int(c.page_of[5, 3]), 5, 6, 7]
    d_src, d_dst = dev(np.array(src, np.int32)), dev(np.array(dst, np.int32))
    ag.kv4_copy(other.pool, d_src.data_ptr(), d_dst.data_ptr(), 5)
    for a, b in list(zip(src, dst))[:2]:
        other.pages[b] = before[a]
    c.free([1])
    refs = c.refs.copy()
    moved = torch.empty(30, dtype=torch.int32, device="cuda")
    ag.kv4_compact(c.pool, c.table, moved.data_ptr())
    ag.kv4_copy(other.pool, None, moved.data_ptr(), 30)
    want = kv4.compact(c.pages, c.page_of, c.refs)
    c.check()
    for p in range(30):
        if refs[p] > 0 and want[p] != p:
            other.pages[want[p]] = other.pages[p]
    assert (moved.cpu().numpy() == want).all()
    other.check()


def test_on_a_side_stream_and_in_a_graph():
    """A decode step's bookkeeping (extend, store) captured once and replayed: every replay appends the next token."""
    c = Cache(12, 2, 128, 3, 4)
    c.extend([0, 1, 2], [0, 62, 63, 191])
    c.check()
    row, off = dev(np.array([2, 0], np.int32)), dev(np.array([0, 1, 2], np.int32))
    slot, ok = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    K, V = torch.zeros(2, 2, 128, dtype=torch.int16, device="cuda"), torch.zeros(2, 2, 128, dtype=torch.int16, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        at = torch.cuda.current_stream().cuda_stream
        ag.kv4_extend(c.pool, c.table, row.data_ptr(), off.data_ptr(), 2, slot.data_ptr(), 2, ok.data_ptr(), at)
        ag.kv4_store(c.pool, K.data_ptr(), V.data_ptr(), slot.data_ptr(), 2, stream=at)
    c.check()                                # capturing ran nothing
    for step in range(4):
        k, v = special_rows(2, 2, 128, 20 + step), special_rows(2, 2, 128, 30 + step)
        K.copy_(torch.from_numpy(k.view(np.int16)))
        V.copy_(torch.from_numpy(v.view(np.int16)))
        graph.replay()
        want, want_ok = kv4.extend(c.page_of, c.len, c.refs, [2, 0], [0, 1, 2], 2)
        kv4.store(c.pages, 128, k, v, want)
        torch.cuda.synchronize()
        assert (slot.cpu().numpy() == want).all() and (ok.cpu().numpy() == want_ok).all()
        c.check()
