"""Cases that measure the serving operators: attention over prompts, the paged 4-bit key/value cache (store, decode attention) and
its pages (fork, free, compact).

`own = False` computes every operator in elementary torch operations (32 bits, rounded once at the end); `own = True` makes the
library calls.  Both take the same state.  The cache layout that both read is the documented one of the 4-bit pages:

page = 64 tokens x all KV heads; per KV head a block of 80 D bytes:
    [0, 32 D)    codes of K     [32 D, 64 D)  codes of V
    [64 D, 72 D) (scale, base) of K as bf16 pairs, [64 tokens][D / 32 groups]     [72 D, 80 D)  the same for V
Codes lie in four runs of 16 tokens, 8 D bytes each; the low nibble of a byte comes first:
    K: token 8 h + g of the run, element 32 grp + 8 t + i  -> byte h 4 D + (4 g + t) D / 8 + 4 grp + i / 2
    V: token 8 h + 2 t + e of the run, element 16 i + 8 hi + g -> byte h 4 D + (4 g + t) D / 8 + e D / 16 + hi D / 32 + i / 2
An element stands for scale * code + base.
"""
import math
import random

import torch

own = False
PAGE = 64
BF16 = torch.bfloat16


# ---- cases ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one short turn of a chat on a small model: latency
        dict(name="prompt_turn", op="prompt", n_seq=1, q_min=77, q_max=77, past=0, H_q=8, H_kv=2, D=64, fused=True, len_seed=1),
        # a mixed batch of a server: prompts of all lengths, some of them later chunks of longer prompts
        dict(name="prompt_mixed_batch", op="prompt", n_seq=16, q_min=33, q_max=1024, past=2048, H_q=32, H_kv=8, D=128, fused=False, len_seed=2),
        # one long prompt from its beginning, projections in one fused buffer
        dict(name="prompt_8192", op="prompt", n_seq=1, q_min=8192, q_max=8192, past=0, H_q=32, H_kv=8, D=128, fused=True, len_seed=3),
        # one request, a few hundred tokens in: the latency of a single stream
        dict(name="decode_one", op="decode", B=1, len_min=300, len_max=300, H_q=32, H_kv=8, D=128, len_seed=4),
        # the serving batch: 128 requests of uneven lengths
        dict(name="decode_batch", op="decode", B=128, len_min=200, len_max=1024, H_q=32, H_kv=8, D=128, len_seed=5),
        # few requests with very long contexts
        dict(name="decode_long", op="decode", B=4, len_min=120000, len_max=131072, H_q=32, H_kv=8, D=128, len_seed=6),
        # one decode step's new tokens, one per request
        dict(name="store_step", op="store", n=128, new_min=1, new_max=1, len_max=1024, H_kv=8, D=128, len_seed=7),
        # the keys and values of whole prompts
        dict(name="store_prompts", op="store", n=16, new_min=2000, new_max=4096, len_max=100, H_kv=8, D=128, len_seed=8),
        # a beam step: four requests branch four ways, the parents leave
        dict(name="fork_beams", op="fork", parents=4, children=4, len_min=50, len_max=700, H_kv=8, D=128, len_seed=9),
        # many samples of shared prompts start at once
        dict(name="fork_samples", op="fork", parents=32, children=16, len_min=100, len_max=4096, H_kv=8, D=128, len_seed=10),
        # a small pool with holes
        dict(name="compact_small", op="compact", n_pages=300, rows=12, used=0.5, H_kv=2, D=64, len_seed=11),
        # a large pool after many requests have left
        dict(name="compact_large", op="compact", n_pages=8192, rows=200, used=0.5, H_kv=8, D=128, len_seed=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "decode", "decode", "store", "fork", "compact"])
    H_kv = rng.choice([1, 2, 4, 8])
    D = rng.choice([64, 128, 128])
    seed = rng.randrange(1 << 30)
    if op == "prompt":
        H_q = min(32, H_kv * rng.choice([1, 2, 3, 4, 5, 8, 16]) if H_kv < 8 else 8 * rng.choice([1, 2, 4]))
        H_q -= H_q % H_kv
        q_max = _log(rng, 1, 8192)
        past = rng.choice([0, 0, _log(rng, 1, 8000)])
        most = max(1, (1 << 31) // (H_q * q_max * (q_max + past)))   # scores of the plain form, padded
        n_seq = min(_log(rng, 1, 64), most)
        return dict(op=op, n_seq=n_seq, q_min=_log(rng, 1, q_max), q_max=q_max, past=past, H_q=H_q, H_kv=H_kv, D=D,
                    fused=past == 0 and rng.random() < 0.5, len_seed=seed)
    if op == "decode":
        H_q = H_kv * rng.choice([1, 2, 3, 4, 7, 8, 16] if H_kv < 8 else [1, 4, 8])
        len_max = _log(rng, 1, 131072)
        B = min(_log(rng, 1, 256), max(1, 524288 // len_max))
        return dict(op=op, B=B, len_min=_log(rng, 1, len_max), len_max=len_max, H_q=H_q, H_kv=H_kv, D=D, len_seed=seed)
    if op == "store":
        new_max = rng.choice([1, _log(rng, 2, 4096)])
        return dict(op=op, n=min(_log(rng, 1, 256), max(1, 65536 // new_max)), new_min=_log(rng, 1, new_max), new_max=new_max,
                    len_max=_log(rng, 1, 2048), H_kv=H_kv, D=D, len_seed=seed)
    if op == "fork":
        return dict(op=op, parents=_log(rng, 1, 32), children=rng.randint(1, 16), len_min=1, len_max=_log(rng, 1, 4096), H_kv=H_kv, D=D, len_seed=seed)
    return dict(op=op, n_pages=_log(rng, 40, 8192), rows=_log(rng, 1, 200), used=round(rng.uniform(0.1, 0.9), 2), H_kv=H_kv, D=D, len_seed=seed)


def _lens(case, n, lo, hi):
    r = random.Random(case["len_seed"])
    return [hi] + [_log(r, lo, hi) for _ in range(n - 1)]


def _prompt_lens(case):
    q = _lens(case, case["n_seq"], case["q_min"], case["q_max"])
    r = random.Random(case["len_seed"] + 1)
    return q, [a + (r.randint(0, case["past"]) if case["past"] else 0) for a in q]


def _pages(n):
    return (n + PAGE - 1) // PAGE


def work(case):
    op, D = case["op"], case["D"]
    head_block = 80 * D
    if op == "prompt":
        q, k = _prompt_lens(case)
        pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(q, k))
        return {"bytes": 4 * D * (case["H_q"] * sum(q) + case["H_kv"] * sum(k)), "flops": 4 * D * case["H_q"] * pairs}
    if op == "decode":
        n = _lens(case, case["B"], case["len_min"], case["len_max"])
        return {"bytes": sum(n) * case["H_kv"] * 5 * D // 4 + 4 * case["B"] * case["H_q"] * D, "flops": 4 * D * case["H_q"] * sum(n)}
    if op == "store":      # rows in, pages out, pages in, rows back out
        n = sum(_lens(case, case["n"], case["new_min"], case["new_max"]))
        return {"bytes": n * case["H_kv"] * D * (4 + 4) + 2 * n * case["H_kv"] * 5 * D // 4, "flops": 0}
    if op == "fork":
        n = _lens(case, case["parents"], case["len_min"], case["len_max"])
        open_pages = case["children"] * sum(1 for x in n if x % PAGE)
        return {"bytes": 2 * open_pages * case["H_kv"] * head_block + 8 * case["children"] * sum(_pages(x) for x in n), "flops": 0}
    used = int(case["n_pages"] * case["used"])
    return {"bytes": 2 * used * (case["n_pages"] - used) // case["n_pages"] * case["H_kv"] * head_block + 12 * case["n_pages"], "flops": 0}


# ---- states -----------------------------------------------------------------------------------------------------------
_topo, _plans = {}, {}


def _plan(stream):
    """A plan of the whole chip for each stream (of each device), since calls of one plan must not run at the same time; found once."""
    key = stream.device_index, stream.cuda_stream
    plan = _plans.get(key)
    if plan is None:
        from paper_2609_24270_b200 import binding as ag
        if key[0] not in _topo:
            _topo[key[0]] = ag.topo_discover(ag.AG_TOPO_CENSUS | ag.AG_TOPO_CLUSTER | ag.AG_TOPO_LATENCY)
        topo = _topo[key[0]]
        plan = _plans[key] = ag.sched_build(topo, None, topo.n_sm, ag.make_policy(kind=ag.AG_DIE_COMPACT, M=128, N=256, K=64))
    return plan


def _random_pages(gen, n_pages, H_kv, D):
    """Pages as a cache holds them: random codes, scales around 0.25, bases around the middle of the range."""
    pages = torch.randint(0, 256, (n_pages, H_kv, 80 * D), dtype=torch.uint8, device="cuda", generator=gen)
    sb = pages[:, :, 64 * D:].view(BF16)                                   # [n_pages][H_kv][2 x 64 x D / 32 pairs]
    scale = 0.25 * torch.exp(0.3 * torch.randn(n_pages, H_kv, 4 * D, device="cuda", generator=gen))
    base = scale * (-7.5 + torch.randn(n_pages, H_kv, 4 * D, device="cuda", generator=gen))
    sb[..., 0::2] = scale.to(BF16)
    sb[..., 1::2] = base.to(BF16)
    return pages


def _random_table(gen, lens, n_pages, n_rows, max_pages, span=None):
    """Rows of distinct pages at random places among the first `span` pages; (page_of, len, refs)."""
    page_of = torch.full((n_rows, max_pages), -1, dtype=torch.int32)
    order = torch.randperm(span or n_pages, generator=torch.Generator().manual_seed(gen.initial_seed())).to(torch.int32)
    at = 0
    for i, n in enumerate(lens):
        p = _pages(n)
        page_of[i, :p] = order[at:at + p]
        at += p
    length = torch.zeros(n_rows, dtype=torch.int32)
    length[:len(lens)] = torch.tensor(lens, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[order[:at].long()] = 1
    return page_of.cuda(), length.cuda(), refs.cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, D = case["op"], case["D"]
    st = dict(op=op, case=case)

    def rows(n, heads, stretch=1.0):
        return (stretch * torch.randn(n, heads, D, device="cuda", generator=gen)).to(BF16)

    if op == "prompt":
        H_q, H_kv = case["H_q"], case["H_kv"]
        q, k = _prompt_lens(case)
        if case["fused"]:
            qkv = rows(sum(q), H_q + 2 * H_kv, 1.2)
            st.update(Q=qkv[:, :H_q], K=qkv[:, H_q:H_q + H_kv], V=qkv[:, H_q + H_kv:])
        else:
            st.update(Q=rows(sum(q), H_q, 1.2), K=rows(sum(k), H_kv, 1.2), V=rows(sum(k), H_kv))
        off = lambda v: torch.tensor([0] + list(torch.tensor(v).cumsum(0)), dtype=torch.int32).cuda()  # noqa: E731
        st.update(q_off=off(q), kv_off=off(k), q_max=max(q), kv_max=max(k), O=torch.empty(sum(q), H_q, D, dtype=BF16, device="cuda"))
        if own:
            _plan(torch.cuda.current_stream())
    elif op == "decode":
        n = _lens(case, case["B"], case["len_min"], case["len_max"])
        max_pages = _pages(max(n))
        n_pages = sum(_pages(x) for x in n) + 3
        st.update(pages=_random_pages(gen, n_pages, case["H_kv"], D), Q=rows(case["B"], case["H_q"]),
                  O=torch.empty(case["B"], case["H_q"], D, dtype=BF16, device="cuda"))
        st["page_of"], st["len"], st["refs"] = _random_table(gen, n, n_pages, case["B"], max_pages)
    elif op == "store":
        new = _lens(case, case["n"], case["new_min"], case["new_max"])
        r = random.Random(case["len_seed"] + 2)
        old = [r.randint(0, case["len_max"]) for _ in new]
        max_pages = _pages(max(a + b for a, b in zip(old, new)))
        n_pages = sum(_pages(a + b) for a, b in zip(old, new)) + 5
        H_kv, total = case["H_kv"], sum(new)
        st.update(pages=torch.zeros(n_pages, H_kv, 80 * D, dtype=torch.uint8, device="cuda"), K=rows(total, H_kv, 1.5), V=rows(total, H_kv),
                  row=torch.arange(case["n"], dtype=torch.int32).flip(0).cuda(), total=total,
                  new_off=torch.tensor([0] + list(torch.tensor(new).cumsum(0)), dtype=torch.int32).cuda(),
                  slot=torch.empty(total, dtype=torch.int32, device="cuda"), ok=torch.empty(case["n"], dtype=torch.int32, device="cuda"),
                  K_back=torch.empty(total, H_kv, D, dtype=BF16, device="cuda"), V_back=torch.empty(total, H_kv, D, dtype=BF16, device="cuda"))
        st["page_of"], st["len"], st["refs"] = _random_table(gen, old[::-1], n_pages, case["n"], max_pages)
    elif op == "fork":
        n = _lens(case, case["parents"], case["len_min"], case["len_max"])
        kids = case["parents"] * case["children"]
        n_pages = sum(_pages(x) for x in n) + kids + 7
        st.update(pages=_random_pages(gen, n_pages, case["H_kv"], D),
                  src=torch.arange(case["parents"], dtype=torch.int32).repeat(case["children"]).cuda(),
                  dst=(case["parents"] + torch.arange(kids, dtype=torch.int32)).cuda(),
                  gone=torch.arange(case["parents"], dtype=torch.int32).cuda(), ok=torch.empty(kids, dtype=torch.int32, device="cuda"))
        st["page_of"], st["len"], st["refs"] = _random_table(gen, n, n_pages, case["parents"] + kids, max(_pages(x) for x in n))
    else:
        used, n_rows = int(case["n_pages"] * case["used"]), case["rows"]
        r = random.Random(case["len_seed"])
        cuts = sorted(r.randint(0, used) for _ in range(n_rows - 1))
        n = [max(0, (b - a) * PAGE - r.randint(0, PAGE - 1)) for a, b in zip([0] + cuts, cuts + [used])]
        st.update(pages=_random_pages(gen, case["n_pages"], case["H_kv"], D), moved=torch.empty(case["n_pages"], dtype=torch.int32, device="cuda"))
        st["page_of"], st["len"], st["refs"] = _random_table(gen, n, case["n_pages"], n_rows, max(1, max(_pages(x) for x in n)))
    if own and op != "prompt":
        from paper_2609_24270_b200 import binding as ag
        st["pool"] = ag.KV4Pool(st["pages"].data_ptr(), st["pages"].shape[0], case["H_kv"], D)
        if op == "decode":
            size = ag.attention_decode_kv4_workspace(case["B"], case["H_q"], case["H_kv"], D, st["page_of"].shape[1])
            st["workspace"] = torch.empty(max(1, size), dtype=torch.uint8, device="cuda")
            st["table"] = ag.KV4Table(st["page_of"].data_ptr(), st["len"].data_ptr(), st["refs"].data_ptr(), *st["page_of"].shape)
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(st):
    return (_own if own else _plain)[st["op"]](st)


def _own_prompt(st):
    from paper_2609_24270_b200 import binding as ag
    c, stream = st["case"], torch.cuda.current_stream()
    ag.attention_prompt(st["Q"].data_ptr(), st["K"].data_ptr(), st["V"].data_ptr(), st["O"].data_ptr(), c["H_q"], c["H_kv"], c["D"],
                        st["q_off"].data_ptr(), st["kv_off"].data_ptr(), c["n_seq"], st["Q"].shape[0], st["K"].shape[0], _plan(stream),
                        q_stride=st["Q"].stride(0), k_stride=st["K"].stride(0), v_stride=st["V"].stride(0), stream=stream.cuda_stream)
    return st["O"]


def _own_decode(st):
    from paper_2609_24270_b200 import binding as ag
    c = st["case"]
    ag.attention_decode_kv4(st["Q"].data_ptr(), st["pool"], st["table"], None, st["O"].data_ptr(), c["B"], c["H_q"],
                            st["workspace"].data_ptr(), st["workspace"].numel(), stream=torch.cuda.current_stream().cuda_stream)
    return st["O"]


def _tables(st):
    """The state's tables once more, since a pass changes them."""
    return st["page_of"].clone(), st["len"].clone(), st["refs"].clone()


def _own_store(st):
    from paper_2609_24270_b200 import binding as ag
    page_of, length, refs = _tables(st)
    table = ag.KV4Table(page_of.data_ptr(), length.data_ptr(), refs.data_ptr(), *page_of.shape)
    stream = torch.cuda.current_stream().cuda_stream
    n, total = st["case"]["n"], st["total"]
    ag.kv4_extend(st["pool"], table, st["row"].data_ptr(), st["new_off"].data_ptr(), n, st["slot"].data_ptr(), total, st["ok"].data_ptr(), stream)
    ag.kv4_store(st["pool"], st["K"].data_ptr(), st["V"].data_ptr(), st["slot"].data_ptr(), total, stream=stream)
    ag.kv4_load(st["pool"], st["slot"].data_ptr(), total, st["K_back"].data_ptr(), st["V_back"].data_ptr(), stream=stream)
    return dict(K=st["K_back"], V=st["V_back"], slot=st["slot"], ok=st["ok"], page_of=page_of, len=length, refs=refs)


def _own_fork(st):
    from paper_2609_24270_b200 import binding as ag
    page_of, length, refs = _tables(st)
    table = ag.KV4Table(page_of.data_ptr(), length.data_ptr(), refs.data_ptr(), *page_of.shape)
    stream = torch.cuda.current_stream().cuda_stream
    ag.kv4_fork(st["pool"], table, st["src"].data_ptr(), st["dst"].data_ptr(), st["src"].numel(), st["ok"].data_ptr(), stream)
    ag.kv4_free(st["pool"], table, st["gone"].data_ptr(), st["gone"].numel(), stream)
    return dict(pages=st["pages"], ok=st["ok"], page_of=page_of, len=length, refs=refs)


def _own_compact(st):
    from paper_2609_24270_b200 import binding as ag
    page_of, length, refs = _tables(st)
    table = ag.KV4Table(page_of.data_ptr(), length.data_ptr(), refs.data_ptr(), *page_of.shape)
    ag.kv4_compact(st["pool"], table, st["moved"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return dict(pages=st["pages"], moved=st["moved"], page_of=page_of, refs=refs)


_own = dict(prompt=_own_prompt, decode=_own_decode, store=_own_store, fork=_own_fork, compact=_own_compact)


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _attend(q, k, v, visible):
    """q [B][n][H_q][D], k and v [B][m][H_kv][D] in 32 bits, visible [B][n][m]; rows that see nothing give zeros."""
    B, n, H_q, D = q.shape
    m, H_kv = k.shape[1:3]
    s = q.view(B, n, H_kv, H_q // H_kv, D).permute(0, 2, 3, 1, 4).reshape(B, H_kv, -1, D) @ k.permute(0, 2, 3, 1)   # [B][H_kv][G n][m]
    s = s.view(B, H_kv, H_q // H_kv, n, m).mul_(1 / math.sqrt(D))
    s.masked_fill_(~visible[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = p.view(B, H_kv, -1, m) @ v.permute(0, 2, 1, 3)
    o = o.view(B, H_kv, H_q // H_kv, n, D) / total.masked_fill(total == 0, 1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, H_q, D)


def _plain_prompt(st):
    q_off, kv_off = st["q_off"].long(), st["kv_off"].long()
    n, m = (q_off[1:] - q_off[:-1])[:, None], (kv_off[1:] - kv_off[:-1])[:, None]
    i, j = torch.arange(st["q_max"], device="cuda")[None], torch.arange(st["kv_max"], device="cuda")[None]
    at = (q_off[:-1, None] + i).clamp(max=st["Q"].shape[0] - 1)
    seen = (kv_off[:-1, None] + j).clamp(max=st["K"].shape[0] - 1)
    visible = (j < m)[:, None, :] & (j[:, None, :] <= (m - n + i)[:, :, None])
    o = _attend(st["Q"].float()[at], st["K"].float()[seen], st["V"].float()[seen], visible)
    return o[i < n].to(BF16)


def _values(pages, D):
    """What pages [..., H_kv, 80 D] hold: K and V as [..., 64, H_kv, D] in 32 bits."""
    lead = pages.shape[:-1]
    z = len(lead)
    nib = torch.stack((pages[..., :64 * D] & 15, pages[..., :64 * D] >> 4), -1)
    k = nib[..., :32 * D, :].reshape(*lead, 4, 2, 8, 4, D // 32, 8)                 # run, h, g, t, grp, i
    k = k.permute(*range(z), z, z + 1, z + 2, z + 4, z + 3, z + 5).reshape(*lead, PAGE, D // 32, 32)
    v = nib[..., 32 * D:, :].reshape(*lead, 4, 2, 8, 4, 2, 2, D // 16)              # run, h, g, t, e, hi, i
    v = v.permute(*range(z), z, z + 1, z + 3, z + 4, z + 6, z + 5, z + 2).reshape(*lead, PAGE, D // 32, 32)
    sb = pages[..., 64 * D:].contiguous().view(BF16).float().reshape(*lead, 2, PAGE, D // 32, 2)
    out = []
    for which, codes in enumerate((k, v)):
        x = codes.float() * sb[..., which, :, :, 0:1] + sb[..., which, :, :, 1:2]
        out.append(x.reshape(*lead, PAGE, D).movedim(z - 1, z))
    return out


def _plain_decode(st):
    B, max_pages = st["page_of"].shape
    D = st["case"]["D"]
    k, v = _values(st["pages"][st["page_of"].long().clamp(min=0)], D)               # [B][max_pages][64][H_kv][D]
    k, v = (x.reshape(B, max_pages * PAGE, -1, D) for x in (k, v))
    visible = torch.arange(max_pages * PAGE, device="cuda")[None] < st["len"][:, None]
    return _attend(st["Q"].float()[:, None], k, v, visible[:, None])[:, 0].to(BF16)


def _quantised(x):
    """The values that bf16 rows [n][H_kv][D] have after four bits: groups of 32, scale rounded to bf16."""
    g = x.float().view(*x.shape[:-1], -1, 32)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    scale = ((hi - lo) / 15).to(BF16).float()
    code = torch.where(scale > 0, (g - lo) / scale, torch.zeros_like(g)).round().clamp(0, 15)
    return (code * scale + lo).view(x.shape).to(BF16)


def _plain_store(st):
    page_of, length, refs = _tables(st)
    row, off = st["row"].long(), st["new_off"].long()
    old, new = length[row].long(), off[1:] - off[:-1]
    first, last = _pages(old), _pages(old + new)
    before = (last - first).cumsum(0) - (last - first)
    free = torch.argsort((refs > 0).int(), stable=True)
    ok = (before + last - first <= (refs == 0).sum()) & (last <= page_of.shape[1])
    c = torch.arange(page_of.shape[1], device="cuda")[None]
    fresh = (c >= first[:, None]) & (c < last[:, None]) & ok[:, None]
    page = free[(before[:, None] + c - first[:, None]).clamp(0, free.numel() - 1)].int()
    page_of[row] = torch.where(fresh, page, page_of[row])
    refs.index_add_(0, page.flatten(), fresh.flatten().int())
    length[row] = torch.where(ok, old + new, old).int()
    token = torch.arange(st["total"], device="cuda")
    i = torch.searchsorted(off, token, right=True) - 1
    at = old[i] + token - off[i]
    slot = torch.where(ok[i], page_of[row[i], at // PAGE] * PAGE + at % PAGE, -1).int()
    return dict(K=_quantised(st["K"]), V=_quantised(st["V"]), slot=slot, ok=ok.int(), page_of=page_of, len=length, refs=refs)


def _plain_fork(st):
    page_of, length, refs = _tables(st)
    src, dst = st["src"].long(), st["dst"].long()
    n = length[src].long()
    full, is_open = n // PAGE, (n % PAGE > 0).long()
    before = is_open.cumsum(0) - is_open
    free = torch.argsort((refs > 0).int(), stable=True)
    ok = (before + is_open <= (refs == 0).sum()) & (length[dst] == 0)
    c = torch.arange(page_of.shape[1], device="cuda")[None]
    fresh = (c == full[:, None]) & (is_open * ok > 0)[:, None]
    shared = (c < full[:, None]) & ok[:, None]
    page = free[before.clamp(max=free.numel() - 1)][:, None].int().expand(-1, c.numel())
    old = page_of[src]
    page_of[dst] = torch.where(fresh, page, torch.where(shared, old, page_of[dst]))
    refs.index_add_(0, old.clamp(min=0).flatten(), shared.flatten().int())
    refs.index_add_(0, page.flatten(), fresh.flatten().int())
    length[dst] = torch.where(ok, n.int(), length[dst])
    st["pages"][page[fresh].long()] = st["pages"][old[fresh].long()]
    gone = st["gone"].long()
    held = page_of[gone]
    refs.index_add_(0, held.clamp(min=0).flatten(), -(held >= 0).flatten().int())
    page_of[gone] = -1
    length[gone] = 0
    return dict(pages=st["pages"], ok=ok.int(), page_of=page_of, len=length, refs=refs)


def _plain_compact(st):
    page_of, length, refs = _tables(st)
    used = refs > 0
    ids = torch.arange(refs.numel(), device="cuda")
    low = ids < used.sum()
    frm, to = ids[used & ~low], ids[~used & low]
    moved = torch.where(used, ids, -1)
    moved[frm] = to
    st["pages"][to] = st["pages"][frm]
    page_of = torch.where(page_of >= 0, moved[page_of.clamp(min=0).long()], -1).int()
    count = torch.zeros_like(refs)
    count[moved[used]] = refs[used]
    return dict(pages=st["pages"], moved=moved.int(), page_of=page_of, refs=count)


_plain = dict(prompt=_plain_prompt, decode=_plain_decode, store=_plain_store, fork=_plain_fork, compact=_plain_compact)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------
def _softmax64(q, k, v, first):
    """One sequence, one KV head: q [n][D] rows, row r sees keys 0 .. first[r]; 64 bits."""
    s = (q @ k.T) / math.sqrt(q.shape[1])
    s = torch.where(torch.arange(k.shape[0], device=q.device)[None] <= first[:, None], s, -math.inf)
    w = torch.softmax(s, 1)
    return torch.where(first[:, None] >= 0, w, 0) @ v


def exact(case, seed):
    st = prepare(case, seed)
    D = case["D"]
    if case["op"] == "prompt":
        G = case["H_q"] // case["H_kv"]
        q_off, kv_off = st["q_off"].tolist(), st["kv_off"].tolist()
        out = torch.empty(st["O"].shape, dtype=torch.float64, device="cuda")
        for a, b, c, d in zip(q_off[:-1], q_off[1:], kv_off[:-1], kv_off[1:]):
            first = (d - c) - (b - a) + torch.arange(b - a, device="cuda")
            for h in range(case["H_q"]):
                out[a:b, h] = _softmax64(st["Q"][a:b, h].double(), st["K"][c:d, h // G].double(), st["V"][c:d, h // G].double(), first)
        return out
    if case["op"] == "decode":
        G = case["H_q"] // case["H_kv"]
        raw = st["pages"]
        out = torch.empty(st["O"].shape, dtype=torch.float64, device="cuda")
        # where element d of token r of a page lies, written out from the layout's formulas
        r, d = torch.arange(PAGE, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
        run, h, g = r // 16, (r % 16) // 8, r % 8
        k_byte = run * 8 * D + h * 4 * D + (4 * g + d % 32 // 8) * (D // 8) + 4 * (d // 32) + d % 8 // 2
        k_high = (d % 2).expand(PAGE, D)
        t, e = r % 8 // 2, r % 2
        v_byte = 32 * D + run * 8 * D + h * 4 * D + (4 * (d % 8) + t) * (D // 8) + e * (D // 16) + (d % 16 // 8) * (D // 32) + d // 32
        v_high = (d // 16 % 2).expand(PAGE, D)
        for b, n in enumerate(st["len"].tolist()):
            ids = st["page_of"][b, :_pages(n)].long()
            for hk in range(case["H_kv"]):
                block = raw[ids, hk]
                vals = []
                for byte, high, at in ((k_byte, k_high, 64 * D), (v_byte, v_high, 72 * D)):
                    codes = (block[:, byte.reshape(-1)].view(-1, PAGE, D) >> (4 * high)) & 15
                    sb = block[:, at:at + 8 * D].contiguous().view(BF16).double().view(-1, PAGE, D // 32, 2)
                    vals.append((codes.double() * sb[..., 0].repeat_interleave(32, -1) + sb[..., 1].repeat_interleave(32, -1)).view(-1, D)[:n])
                out[b, hk * G:(hk + 1) * G] = _softmax64(st["Q"][b, hk * G:(hk + 1) * G].double(), vals[0], vals[1], torch.full((G,), n, device="cuda"))
        return out
    if case["op"] == "store":
        res = {}
        for name in ("K", "V"):
            x = st[name].double().unflatten(-1, (-1, 32))
            lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
            s = ((hi - lo) / 15).to(BF16).double()
            u = torch.round((x - lo) / torch.where(s > 0, s, 1.0)).clamp(max=15)
            res[name] = (lo + s * u).flatten(-2)
        return dict(K=res["K"], V=res["V"], slot=None, ok=None, page_of=None, len=None, refs=None)
    return None
