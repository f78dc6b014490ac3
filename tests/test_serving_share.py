"""Prompts on part of the chip while something else keeps SMs busy, or with fewer blocks than SMs: every launch ends, either with the right outputs or with the
documented AG_ERR_UNMANNED_SM (no block came to a planned SM: nothing has run), and the plan can be used again."""
import gc

import pytest
import torch

from paper_2609_24270_b200 import binding as ag
from tests.gpu_util import device_topo
from tests.test_serving_kv4_decode import make, queries
from tests.test_serving_prompt import dev, offsets, plan_for, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def give_memory_back():
    """Tests that look at addresses or at free memory find torch's allocator without blocks of these."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


class Prompt:
    def __init__(self, lens, H_q=8, H_kv=2, D=128):
        n = sum(lens)
        self.n, self.n_seq, self.shape = n, len(lens), (H_q, H_kv, D)
        self.q, self.k, self.v = (dev(rows(n, h, D, i)) for i, h in enumerate((H_q, H_kv, H_kv)))
        self.off = dev(offsets(lens))
        self.o = torch.zeros(n, H_q, D, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()

    def run(self, plan, stream):
        ag.attention_prompt(self.q.data_ptr(), self.k.data_ptr(), self.v.data_ptr(), self.o.data_ptr(), *self.shape, self.off.data_ptr(), None, self.n_seq, self.n, self.n,
                            plan, stream=stream.cuda_stream)


@pytest.mark.parametrize("elsewhere", [False, True])
def test_fewer_blocks_than_planned_sms(elsewhere):
    """One to nine blocks land where the hardware puts them: on SMs of the plan, or on others, where they wait for a while and leave."""
    p, s, topo = Prompt([500, 130]), torch.cuda.Stream(), device_topo()
    first = ag.sched_build(topo, None, topo.n_sm - 20, ag.make_policy(kind=ag.AG_OBLIVIOUS, M=128, N=256, K=64))
    avoid = first.parsed()["sm_list"].tolist() if elsewhere else []
    plan = ag.sched_build(topo, None, 20, ag.make_policy(kind=ag.AG_OBLIVIOUS, M=128, N=256, K=64, avoid=avoid))
    p.run(plan, s)
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK
    want, seen = p.o.clone(), []
    for i in range(60):
        plan.set_grid(1 + i % 9)
        p.o.zero_()
        torch.cuda.synchronize()
        p.run(plan, s)
        torch.cuda.synchronize()
        seen.append(plan.last_status())
        assert torch.equal(p.o, want) if seen[-1] == ag.AG_OK else (seen[-1] == ag.AG_ERR_UNMANNED_SM and not p.o.any())
    plan.set_grid(0)
    p.run(plan, s)
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK and torch.equal(p.o, want)
    print({k: seen.count(k) for k in set(seen)})


def test_beside_long_decodes():
    """Decode steps over long rows fill the whole chip, one behind the other, on another stream."""
    c = make([30000, 30000], 8, 64, seed=3)
    Q = dev(queries(2, 32, 64, 4))
    size = ag.attention_decode_kv4_workspace(2, 32, 8, 64, c.page_of.shape[1])
    ws, out = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(2, 32, 64, dtype=torch.bfloat16, device="cuda")
    p, plan = Prompt([700, 300, 64]), plan_for(74)
    main, other = torch.cuda.Stream(), torch.cuda.Stream()

    def step():
        ag.attention_decode_kv4(Q.data_ptr(), c.pool, c.table, None, out.data_ptr(), 2, 32, ws.data_ptr(), size, main.cuda_stream)

    p.run(plan, other)
    step()
    torch.cuda.synchronize()
    assert plan.last_status() == ag.AG_OK
    want = p.o.clone(), out.clone()
    for i in range(8):
        p.o.zero_()
        out.zero_()
        torch.cuda.synchronize()
        for _ in range(8):
            step()
        p.run(plan, other)
        for _ in range(8):
            step()
        torch.cuda.synchronize()
        st = plan.last_status()
        assert torch.equal(out, want[1])
        assert torch.equal(p.o, want[0]) if st == ag.AG_OK else (st == ag.AG_ERR_UNMANNED_SM and not p.o.any())
