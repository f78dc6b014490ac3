"""Compaction of large pools: where the pages go, and that the work grows with the pool, not with its square."""
import gc

import pytest
import torch

from paper_2609_24270_b200 import binding as ag

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def compact(n, refs, row):
    """(moved, refs, row's pages, contents by page, best ms of compaction, best ms of the same copies alone)"""
    words = ag.kv4_page_bytes(1, 64) // 4
    pages = torch.zeros(n, words, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    ln = torch.tensor([64 * len(row)], dtype=torch.int32, device="cuda")
    moved = torch.empty(n, dtype=torch.int32, device="cuda")
    pool = ag.KV4Pool(pages.data_ptr(), n, 1, 64)
    best = [float("inf")] * 2
    for _ in range(3):
        pages[:, 0] = torch.arange(n, device="cuda")
        pages[:, -1] = -pages[:, 0]
        live, held = refs.clone(), row.clone()
        table = ag.KV4Table(held.data_ptr(), ln.data_ptr(), live.data_ptr(), 1, len(row))
        for i, call in enumerate((lambda: ag.kv4_compact(pool, table, moved.data_ptr(), stream), lambda: ag.kv4_copy(pool, None, moved.data_ptr(), n, stream))):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            torch.cuda.synchronize()
            e[0].record()
            call()
            e[1].record()
            torch.cuda.synchronize()
            best[i] = min(best[i], e[0].elapsed_time(e[1]))
    return moved, live, held, pages[:, 0].clone(), pages[:, -1].clone(), best


@pytest.mark.parametrize("n", [1 << 17, (1 << 20) + 33])
@pytest.mark.parametrize("part", [0.02, 0.5, 0.98])
def test_pages_in_use_at_random(n, part):
    gen = torch.Generator(device="cuda").manual_seed(n)
    refs = (torch.rand(n, device="cuda", generator=gen) < part).int() * torch.randint(1, 4, (n,), device="cuda", generator=gen, dtype=torch.int32)
    used = refs > 0
    ids = torch.arange(n, device="cuda")
    row = ids[used][torch.randperm(int(used.sum()), device="cuda", generator=gen)[:1000]].int()
    moved, live, held, first, last, (took, copies) = compact(n, refs, row)
    n_used = int(used.sum())
    want = torch.where(used, ids, -1)
    want[ids[used & (ids >= n_used)]] = ids[~used & (ids < n_used)]
    assert torch.equal(moved.long(), want) and torch.equal(held.long(), want[row.long()])
    back = torch.full((n,), -1, device="cuda")
    back[want[used]] = ids[used]
    assert torch.equal(first[:n_used].long(), back[:n_used]) and torch.equal(last[:n_used].long(), -back[:n_used])
    assert torch.equal(live[:n_used], refs[back[:n_used]]) and not live[n_used:].any()
    print(f"{n} pages, {part}: {took * 1000:.0f} us, copies {copies * 1000:.0f}")
    assert took < 0.5 + 4 * copies                  # half a millisecond for the counts of a million pages


@pytest.mark.parametrize("n", [1, 131073])
@pytest.mark.parametrize("kind", ["none", "all", "front", "back"])
def test_nothing_or_everything_moves(n, kind):
    ids = torch.arange(n, device="cuda")
    refs = {"none": ids < 0, "all": ids >= 0, "front": ids < n // 2, "back": ids >= n // 2}[kind].int()
    moved, live, _, first, _, _ = compact(n, refs, torch.full((1,), -1, dtype=torch.int32, device="cuda"))
    n_used = int(refs.sum())
    want = torch.where(refs > 0, ids, -1)
    want[ids[(refs > 0) & (ids >= n_used)]] = ids[(refs <= 0) & (ids < n_used)]
    assert torch.equal(moved.long(), want) and (live[:n_used] == 1).all() and not live[n_used:].any()
