"""Cases that measure a drafted step of a server: rotary positions, new keys and values appended to the 4-bit cache with their rotation,
attention of a tree of drafted tokens over that cache, and the verification of the drafts.

`own = False` computes every operator in elementary torch operations (32 bits, 64 for angles and for sums that decide, rounded once at the
end); `own = True` makes the library calls.  Both take the same state.

rotary     pair (a, b) of a head becomes (a c - b s, b c + a s), c and s = magnitude * cos, sin (position * frequency), in 32 bits; the
           pairs are (i, i + rot / 2) ("halves") or (2 i, 2 i + 1) ("pairs") of the head's first rot elements, the others stay
append     K rotated and rounded to bf16, then K and V in four bits: groups of 32 with lowest value lo and scale s = bf16((hi - lo) / 15),
           code = rint((x - lo) / s), an element stands for s * code + lo; the rotated queries beside it
tree       token i sees all of its request's cache, its ancestors among the request's drafted tokens and itself
verify     from the root on: child x of the token in hand is accepted when u q(x) < r(x), r = p at first; a rejected one leaves r =
           max(r - q, 0) / sum; where no child is left the next token is the first v with cumsum(r)(v) > u sum(r)

Cache layout: page = 64 tokens x all KV heads; per KV head a block of 80 D bytes:
    [0, 32 D)    codes of K     [32 D, 64 D)  codes of V
    [64 D, 72 D) (scale, base) of K as bf16 pairs, [64 tokens][D / 32 groups]     [72 D, 80 D)  the same for V
Codes lie in four runs of 16 tokens, 8 D bytes each; the low nibble of a byte comes first:
    K: token 8 h + g of the run, element 32 grp + 8 t + i  -> byte h 4 D + (4 g + t) D / 8 + 4 grp + i / 2
    V: token 8 h + 2 t + e of the run, element 16 i + 8 hi + g -> byte h 4 D + (4 g + t) D / 8 + e D / 16 + hi D / 32 + i / 2
"""
import math
import random

import torch

own = False
PAGE = 64
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


# ---- cases ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the drafted tokens of eight requests, far into long contexts: latency
        dict(name="rotary_drafts", op="rotary", n=64, H_q=32, H_kv=8, D=128, rot=128, pairs=True, fused=True, far=131072, scaling="bands", len_seed=1),
        # whole prompts, half of each head rotated
        dict(name="rotary_prompts", op="rotary", n=16384, H_q=32, H_kv=8, D=128, rot=64, pairs=False, fused=True, far=4096, scaling="none", len_seed=2),
        # one decode step of a batch: one token a request
        dict(name="append_step", op="append", n=128, H_q=32, H_kv=8, D=128, rot=128, pairs=False, fused=True, far=8192, scaling="ramp", gather=False, len_seed=3),
        # the tokens of whole prompts
        dict(name="append_prompts", op="append", n=16384, H_q=32, H_kv=8, D=128, rot=128, pairs=False, fused=True, far=4096, scaling="none", gather=False, len_seed=4),
        # the accepted ones among the drafted tokens of 64 requests, already rotated
        dict(name="append_commit", op="append", n=300, H_q=0, H_kv=8, D=128, rot=0, pairs=False, fused=False, far=4096, scaling="none", gather=True, len_seed=5),
        # one request, a few hundred tokens in, eight drafted tokens: the latency of a single stream
        dict(name="tree_one", op="tree", B=1, t_min=8, t_max=8, len_min=300, len_max=300, H_q=32, H_kv=8, D=128, width=2, fused=True, len_seed=6),
        # a serving batch of uneven lengths with uneven trees
        dict(name="tree_batch", op="tree", B=64, t_min=3, t_max=16, len_min=200, len_max=4000, H_q=32, H_kv=8, D=128, width=3, fused=True, len_seed=7),
        # few requests with very long contexts, broad trees
        dict(name="tree_long", op="tree", B=4, t_min=32, t_max=32, len_min=120000, len_max=131072, H_q=32, H_kv=8, D=128, width=4, fused=False, len_seed=8),
        # the largest trees, small heads, eight query heads a KV head
        dict(name="tree_wide", op="tree", B=16, t_min=40, t_max=64, len_min=1000, len_max=8192, H_q=32, H_kv=4, D=64, width=4, fused=False, len_seed=9),
        # a chain of four drafts of one request, small vocabulary, 16-bit probabilities: latency
        dict(name="verify_one", op="verify", B=1, t_min=5, t_max=5, vocab=32001, bits=16, width=1, drafts="replace", far=1.0, len_seed=10),
        # chains of eight drafts of a batch
        dict(name="verify_batch", op="verify", B=64, t_min=3, t_max=9, vocab=131072, bits=32, width=1, drafts="replace", far=0.7, len_seed=11),
        # trees whose siblings were drawn without repetition, an odd vocabulary
        dict(name="verify_trees", op="verify", B=128, t_min=8, t_max=16, vocab=100003, bits=32, width=3, drafts="distinct", far=1.0, len_seed=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "append", "tree", "tree", "verify", "verify"])
    H_kv = rng.choice([1, 2, 4, 8])
    D = rng.choice([64, 128, 128])
    seed = rng.randrange(1 << 30)
    if op in ("rotary", "append"):
        gather = op == "append" and rng.random() < 0.3
        return dict(op=op, n=_log(rng, 1, 16384), H_q=0 if gather else H_kv * rng.choice([1, 2, 3, 4]), H_kv=H_kv, D=D,
                    rot=0 if gather else rng.choice([16, 32, D // 2, D, D]), pairs=rng.random() < 0.5, fused=not gather and rng.random() < 0.5,
                    far=_log(rng, 1, 1000000), scaling=rng.choice(["none", "linear", "bands", "ramp"]),
                    len_seed=seed, **(dict(gather=gather) if op == "append" else {}))
    if op == "tree":
        t_max = _log(rng, 1, 64)
        H_q = H_kv * rng.choice([1, 2, 3, 4, 7, 8])
        len_max = _log(rng, 1, 131072)
        most = max(1, min(524288 // len_max, (1 << 28) // (H_q * t_max * len_max)))
        return dict(op=op, B=min(_log(rng, 1, 128), most), t_min=_log(rng, 1, t_max), t_max=t_max, len_min=_log(rng, 1, len_max), len_max=len_max, H_q=H_q, H_kv=H_kv,
                    D=D, width=rng.choice([1, 2, 4]), fused=rng.random() < 0.5, len_seed=seed)
    t_max = _log(rng, 1, 16)
    vocab = _log(rng, 1000, 131072)
    return dict(op=op, B=min(_log(rng, 1, 128), max(1, (1 << 27) // (t_max * vocab))), t_min=_log(rng, 1, t_max), t_max=t_max, vocab=vocab, bits=rng.choice([16, 32]),
                width=rng.choice([1, 1, 2, 3]), drafts=rng.choice(["replace", "distinct", "certain"]), far=round(rng.uniform(0.2, 1.5), 2), len_seed=seed)


def _counts(case, lo, hi, more=0):
    r = random.Random(case["len_seed"] + more)
    return [hi] + [_log(r, lo, hi) for _ in range(case["B"] - 1)]


def _parents(case, counts):
    """Parents of all tokens, request after request, counted from the request's first token: -1 for that one, at most `width` children each."""
    r = random.Random(case["len_seed"] + 2)
    out = []
    for t in counts:
        kids, par = [0] * t, [-1]
        for i in range(1, t):
            p = i - 1
            if case["width"] > 1 and r.random() < 0.6:
                p = r.choice([j for j in range(max(0, i - 8), i) if kids[j] < case["width"]])
            kids[p] += 1
            par.append(p)
        out.append(par)
    return out


def _depths(par):
    depth = []
    for p in par:
        depth.append(0 if p < 0 else depth[p] + 1)
    return depth


def _pages(n):
    return (n + PAGE - 1) // PAGE


def work(case):
    op = case["op"]
    if op == "verify":      # the rows where the walks end, of both models; the gathered entries are nothing beside them
        return {"bytes": case["B"] * case["vocab"] * case["bits"] // 8 * (1 if case["drafts"] == "certain" else 2), "flops": 0}
    D = case["D"]
    if op == "rotary":
        return {"bytes": 4 * case["n"] * D * (case["H_q"] + case["H_kv"]) + 4 * case["n"], "flops": 0}
    if op == "append":      # rows in; rotated queries, pages out; the pages in, their rows out
        n = case["n"]
        return {"bytes": n * D * (4 * case["H_q"] + 4 * case["H_kv"]) + 2 * n * case["H_kv"] * 5 * D // 4 + 4 * n * case["H_kv"] * D, "flops": 0}
    t, n = _counts(case, case["t_min"], case["t_max"], 1), _counts(case, case["len_min"], case["len_max"])
    seen = sum(d + 1 for par in _parents(case, t) for d in _depths(par))
    pairs = sum(a * b for a, b in zip(t, n)) + seen
    return {"bytes": sum(n) * case["H_kv"] * 5 * D // 4 + 4 * sum(t) * D * (case["H_q"] + case["H_kv"]), "flops": 4 * D * case["H_q"] * pairs}


# ---- states -----------------------------------------------------------------------------------------------------------
def _frequencies(case):
    """Radians a position for every pair, in 64 bits, and the factor on cos and sin."""
    rot, kind = case["rot"], case["scaling"]
    f = 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=F64) / max(rot, 1))
    if kind == "linear":
        return f / 4.0, 1.0
    if kind == "bands":     # long waves stretched 8 times, short ones kept, those between blended by their turns over 8192 positions
        mix = ((8192.0 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f * mix + f / 8.0 * (1 - mix), 1.0
    if kind == "ramp":      # the same, blended by the pair's place between those that turn 32 times and once over 4096 positions
        place = lambda turns: rot * math.log(4096.0 / (2 * math.pi * turns)) / (2 * math.log(10000.0))  # noqa: E731
        lo, hi = max(0.0, math.floor(place(32.0))), min(rot - 1.0, math.ceil(place(1.0)))
        mix = 1 - ((torch.arange(rot // 2, dtype=F64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * mix + f / 16.0 * (1 - mix), 0.1 * math.log(16.0) + 1.0
    return f, 1.0


def _random_pages(gen, n_pages, H_kv, D):
    """Pages as a cache holds them: random codes, scales around 0.25, bases around the middle of the range."""
    pages = torch.randint(0, 256, (n_pages, H_kv, 80 * D), dtype=torch.uint8, device="cuda", generator=gen)
    sb = pages[:, :, 64 * D:].view(BF16)                                   # [n_pages][H_kv][2 x 64 x D / 32 pairs]
    scale = 0.25 * torch.exp(0.3 * torch.randn(n_pages, H_kv, 4 * D, device="cuda", generator=gen))
    base = scale * (-7.5 + torch.randn(n_pages, H_kv, 4 * D, device="cuda", generator=gen))
    sb[..., 0::2] = scale.to(BF16)
    sb[..., 1::2] = base.to(BF16)
    return pages


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _offsets(counts):
    return _ints([0] + torch.tensor(counts).cumsum(0).tolist())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    op = case["op"]
    st = dict(op=op, case=case)

    def rows(n, heads, stretch=1.0):
        return (stretch * torch.randn(n, heads, case["D"], device="cuda", generator=gen)).to(BF16)

    if op in ("rotary", "append"):
        n, H_q, H_kv = case["n"], case["H_q"], case["H_kv"]
        total = 2 * n if case.get("gather") else n                         # drafted tokens, about half of them accepted
        if case["fused"]:
            qkv = rows(total, H_q + 2 * H_kv, 1.2)
            st.update(Q=qkv[:, :H_q], K=qkv[:, H_q:H_q + H_kv], V=qkv[:, H_q + H_kv:])
        else:
            st.update(Q=rows(total, H_q, 1.2), K=rows(total, H_kv, 1.2), V=rows(total, H_kv))
        freq, st["magnitude"] = _frequencies(case)
        st.update(freq=freq.cuda(), pos=torch.randint(0, case["far"], (n,), generator=host, dtype=torch.int32).cuda(),
                  Q_out=torch.empty(n, H_q, case["D"], dtype=BF16, device="cuda"), K_out=torch.empty(n, H_kv, case["D"], dtype=BF16, device="cuda"))
        if op == "append":
            n_pages = _pages(n) + 3
            st.update(pages=torch.zeros(n_pages, H_kv, 80 * case["D"], dtype=torch.uint8, device="cuda"),
                      slot=torch.randperm(n_pages * PAGE, generator=host)[:n].sort().values.int().cuda(), V_out=torch.empty_like(st["K_out"]),
                      rows=torch.randperm(total, generator=host)[:n].sort().values.int().cuda() if case["gather"] else None)
    elif op == "tree":
        H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
        t, n = _counts(case, case["t_min"], case["t_max"], 1), _counts(case, case["len_min"], case["len_max"])
        total, n_pages = sum(t), sum(_pages(x) for x in n) + 3
        if case["fused"]:
            qkv = rows(total, H_q + 2 * H_kv, 1.2)
            st.update(Q=qkv[:, :H_q], K=qkv[:, H_q:H_q + H_kv], V=qkv[:, H_q + H_kv:])
        else:
            st.update(Q=rows(total, H_q, 1.2), K=rows(total, H_kv, 1.2), V=rows(total, H_kv))
        order = torch.randperm(n_pages, generator=host).int()
        page_of, at = torch.full((case["B"], max(_pages(x) for x in n)), -1, dtype=torch.int32), 0
        for i, x in enumerate(n):
            page_of[i, :_pages(x)] = order[at:at + _pages(x)]
            at += _pages(x)
        refs = torch.zeros(n_pages, dtype=torch.int32)
        refs[order[:at].long()] = 1
        st.update(pages=_random_pages(gen, n_pages, H_kv, D), page_of=page_of.cuda(), len=_ints(n), refs=refs.cuda(), off=_offsets(t), total=total, t_max=max(t),
                  parent=_ints([p for par in _parents(case, t) for p in par]), O=torch.empty(total, H_q, D, dtype=BF16, device="cuda"))
    else:
        t, V = _counts(case, case["t_min"], case["t_max"], 1), case["vocab"]
        parents = _parents(case, t)
        total = sum(t)
        kind = BF16 if case["bits"] == 16 else F32
        logits = 2.5 * torch.randn(total, V, device="cuda", generator=gen)
        p = torch.softmax(logits, 1).to(kind)
        logits += case["far"] * torch.randn(total, V, device="cuda", generator=gen)     # the drafting model is this far off
        q = torch.softmax(logits, 1).to(kind)
        # children of a token are drawn from its q: the largest of log q + Gumbel noise, without repetition; with repetition each from noise of its own
        first = [a for a, c in zip(torch.tensor([0] + t[:-1]).cumsum(0).tolist(), t) for _ in range(c)]
        flat = [f + p_ if p_ >= 0 else -1 for f, p_ in zip(first, [p_ for par in parents for p_ in par])]
        rank, seen = [], {}
        for f in flat:
            rank.append(seen.get(f, 0))
            seen[f] = rank[-1] + 1
        noise = -torch.log(-torch.log(torch.rand(total, V, device="cuda", generator=gen).clamp_(1e-7, 1 - 1e-6)))
        noise += logits
        best = noise.topk(max(1, max(rank) + 1), 1).indices
        par, rk = _ints(flat).long(), _ints(rank).long()
        token = best[par.clamp(min=0), rk]
        if case["drafts"] == "replace" and max(rank) > 0:
            again = torch.multinomial(torch.softmax(logits, 1)[par.clamp(min=0)], 1, generator=gen)[:, 0]
            token = torch.where(rk == 0, token, again)
        del logits, noise
        st.update(P=p, Q=None if case["drafts"] == "certain" else q, token=token.int(), parent=_ints([x for q_ in parents for x in q_]), off=_offsets(t), total=total,
                  t_max=max(t), u=torch.rand(total, device="cuda", generator=gen), u_next=torch.rand(case["B"], device="cuda", generator=gen),
                  accepted=torch.empty(total, dtype=torch.int32, device="cuda"), next=torch.empty(case["B"], dtype=torch.int32, device="cuda"),
                  new_off=torch.empty(case["B"] + 1, dtype=torch.int32, device="cuda"), rows=torch.empty(total, dtype=torch.int32, device="cuda"))
    if own and op != "verify":
        from paper_2609_24270_b200 import binding as ag
        if op in ("rotary", "append"):
            st["rotary"] = ag.Rotary(st["freq"].data_ptr(), case["rot"], ag.AG_ROTARY_PAIRS if case["pairs"] else ag.AG_ROTARY_HALVES, st["magnitude"])
        if op != "rotary":
            st["pool"] = ag.KV4Pool(st["pages"].data_ptr(), st["pages"].shape[0], case["H_kv"], case["D"])
        if op == "tree":
            size = ag.attention_tree_kv4_workspace(case["B"], st["t_max"], case["H_q"], case["H_kv"], case["D"], st["page_of"].shape[1])
            st["workspace"] = torch.empty(max(1, size), dtype=torch.uint8, device="cuda")
            st["table"] = ag.KV4Table(st["page_of"].data_ptr(), st["len"].data_ptr(), st["refs"].data_ptr(), *st["page_of"].shape)
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(st):
    return (_own if own else _plain)[st["op"]](st)


def _own_rotary(st):
    from paper_2609_24270_b200 import binding as ag
    c = st["case"]
    ag.rotary_apply(st["rotary"], st["pos"].data_ptr(), c["n"], c["D"], q_ptr=st["Q"].data_ptr(), q_out_ptr=st["Q_out"].data_ptr(), H_q=c["H_q"],
                    k_ptr=st["K"].data_ptr(), k_out_ptr=st["K_out"].data_ptr(), H_kv=c["H_kv"], q_stride=st["Q"].stride(0), k_stride=st["K"].stride(0),
                    stream=torch.cuda.current_stream().cuda_stream)
    return dict(Q=st["Q_out"], K=st["K_out"])


def _own_append(st):
    from paper_2609_24270_b200 import binding as ag
    c, stream = st["case"], torch.cuda.current_stream().cuda_stream
    ask_q = dict(q_ptr=st["Q"].data_ptr(), q_out_ptr=st["Q_out"].data_ptr(), H_q=c["H_q"], q_stride=st["Q"].stride(0)) if c["H_q"] else {}
    by_row = dict(from_ptr=st["rows"].data_ptr(), n_rows=st["K"].shape[0]) if c["gather"] else {}
    ag.kv4_append_rotary(st["pool"], st["rotary"] if c["rot"] else None, st["pos"].data_ptr(), st["slot"].data_ptr(), c["n"], st["K"].data_ptr(), st["V"].data_ptr(),
                         k_stride=st["K"].stride(0), v_stride=st["V"].stride(0), stream=stream, **ask_q, **by_row)
    ag.kv4_load(st["pool"], st["slot"].data_ptr(), c["n"], st["K_out"].data_ptr(), st["V_out"].data_ptr(), stream=stream)
    return dict(K=st["K_out"], V=st["V_out"], **(dict(Q=st["Q_out"]) if c["H_q"] else {}))


def _own_tree(st):
    from paper_2609_24270_b200 import binding as ag
    c = st["case"]
    ag.attention_tree_kv4(st["Q"].data_ptr(), st["K"].data_ptr(), st["V"].data_ptr(), st["O"].data_ptr(), st["pool"], st["table"], None, st["off"].data_ptr(),
                          st["parent"].data_ptr(), c["B"], st["total"], st["t_max"], c["H_q"], st["workspace"].data_ptr(), st["workspace"].numel(),
                          q_stride=st["Q"].stride(0), k_stride=st["K"].stride(0), v_stride=st["V"].stride(0), stream=torch.cuda.current_stream().cuda_stream)
    return st["O"]


def _own_verify(st):
    from paper_2609_24270_b200 import binding as ag
    c = st["case"]
    ag.verify_drafts(st["P"].data_ptr(), None if st["Q"] is None else st["Q"].data_ptr(), c["vocab"], st["token"].data_ptr(), st["parent"].data_ptr(),
                     st["off"].data_ptr(), c["B"], st["total"], st["u"].data_ptr(), st["u_next"].data_ptr(), st["accepted"].data_ptr(), st["next"].data_ptr(),
                     st["new_off"].data_ptr(), st["rows"].data_ptr(), bf16=c["bits"] == 16, distinct=c["drafts"] == "distinct",
                     stream=torch.cuda.current_stream().cuda_stream)
    return dict(accepted=st["accepted"], next=st["next"], new_off=st["new_off"], rows=st["rows"])


_own = dict(rotary=_own_rotary, append=_own_append, tree=_own_tree, verify=_own_verify)


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _rotated(st, x):
    """bf16 rows [n][H][D] at the state's positions: angles in 64 bits, the rotation in 32."""
    rot = st["case"]["rot"]
    angle = st["pos"].double()[:, None, None] * st["freq"]                 # [n][1][rot / 2]
    c, s = (angle.cos() * st["magnitude"]).float(), (angle.sin() * st["magnitude"]).float()
    head = x[..., :rot].float()
    a, b = (head[..., 0::2], head[..., 1::2]) if st["case"]["pairs"] else (head[..., :rot // 2], head[..., rot // 2:])
    u, v = a * c - b * s, b * c + a * s
    turned = torch.stack((u, v), -1).flatten(-2) if st["case"]["pairs"] else torch.cat((u, v), -1)
    return torch.cat((turned.to(BF16), x[..., rot:]), -1)


def _plain_rotary(st):
    return dict(Q=_rotated(st, st["Q"]), K=_rotated(st, st["K"]))


def _quantised(x):
    """The values that bf16 rows [n][H_kv][D] have after four bits: groups of 32, scale rounded to bf16."""
    g = x.float().reshape(*x.shape[:-1], -1, 32)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    scale = ((hi - lo) / 15).to(BF16).float()
    code = torch.where(scale > 0, (g - lo) / scale, torch.zeros_like(g)).round().clamp(0, 15)
    return (code * scale + lo).view(x.shape).to(BF16)


def _plain_append(st):
    at = slice(None) if st["rows"] is None else st["rows"].long()
    k = st["K"][at]
    out = dict(K=_quantised(_rotated(st, k) if st["case"]["rot"] else k), V=_quantised(st["V"][at]))
    return dict(out, Q=_rotated(st, st["Q"])) if st["case"]["H_q"] else out


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
    codes = torch.stack((k, v), z).float()                                          # [..., 2, 64, D / 32, 32]
    x = (codes * sb[..., 0:1] + sb[..., 1:2]).flatten(-2).movedim(z - 1, z + 1)     # [..., 2, 64, H_kv, D]
    return x.unbind(z - 1)


def _plain_tree(st):
    c = st["case"]
    B, max_pages = st["page_of"].shape
    T, H_q, H_kv, D = st["t_max"], c["H_q"], c["H_kv"], c["D"]
    G, m = H_q // H_kv, max_pages * PAGE
    i = torch.arange(T, device="cuda")
    off = st["off"].long()
    there = i[None] < (off[1:] - off[:-1])[:, None]                                 # [B][T]
    at = (off[:-1, None] + i).clamp(max=st["total"] - 1)
    # parents -> ancestors and self: paths of up to 64 steps by six squarings
    up = (st["parent"].long()[at][:, :, None] == i) & there[:, :, None]
    seen = (up | torch.eye(T, dtype=torch.bool, device="cuda")).float()
    for _ in range(6):
        seen = ((seen @ seen) > 0).float()
    q = st["Q"].float()[at].view(B, T, H_kv, G, D).permute(0, 2, 3, 1, 4).reshape(B, H_kv, G * T, D)
    k, v = _values(st["pages"][st["page_of"].long().clamp(min=0)], D)               # [B][max_pages][64][H_kv][D]
    k, v = (torch.cat((x.reshape(B, m, H_kv, D), new.float()[at]), 1).transpose(1, 2) for x, new in ((k, st["K"]), (v, st["V"])))
    cached = (torch.arange(m, device="cuda")[None] < st["len"][:, None])[:, None].expand(B, T, m)
    visible = torch.cat((cached, (seen > 0) & there[:, None]), 2)                   # [B][T][m + T]
    s = (q @ k.transpose(2, 3)).view(B, H_kv, G, T, m + T).mul_(1 / math.sqrt(D))
    s.masked_fill_(~visible[:, None, None], -math.inf)
    p = s.sub_(s.amax(-1, keepdim=True)).exp_().view(B, H_kv, G * T, m + T)
    o = (p @ v) / p.sum(-1, keepdim=True)
    return o.view(B, H_kv, G, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, H_q, D)[there].to(BF16)


def _plain_verify(st):
    """The walk of all requests side by side, token after token; whole rows are touched only where a draft has been rejected."""
    c, off = st["case"], st["off"].long()
    B, last = c["B"], st["total"] - 1
    first, count = off[:-1], off[1:] - off[:-1]
    parent, token = st["parent"].long(), st["token"].long()
    q = st["Q"]
    hand = first.clone()                                                            # the token that each walk has in hand
    left = torch.ones(B, dtype=F64, device="cuda")                                  # of q, without the siblings that have been tried
    accepted = torch.zeros(st["total"], dtype=torch.bool, device="cuda")
    accepted[first] = True
    r = st["P"][hand].double()                                                      # [B][vocab]
    tried = torch.zeros(B, c["vocab"], dtype=torch.bool, device="cuda")
    each = torch.arange(B, device="cuda")
    for i in range(1, st["t_max"]):                                                 # a walk: the row a token is judged by hangs on the ones before it
        at = (first + i).clamp(max=last)
        x = token[at]
        asked = (i < count) & (parent[at] == hand - first)
        qx = torch.ones(B, dtype=F64, device="cuda") if q is None else q[hand, x].double() * ~tried[each, x] / left
        ok = asked & (st["u"][at].double() * qx < r[each, x])
        accepted[at[ok]] = True
        hand = torch.where(ok, at, hand)
        r[ok] = st["P"][hand[ok]].double()
        tried[ok] = False
        left[ok] = 1.0
        no = (asked & ~ok).nonzero()[:, 0]
        if q is None:
            rest = r[no]
            rest[torch.arange(no.numel(), device="cuda"), x[no]] = 0
        else:
            rest = (r[no] - q[hand[no]].double() * ~tried[no] / left[no, None]).clamp(min=0)
        total = rest.sum(1, keepdim=True)
        r[no] = torch.where(total > 0, rest / total, r[no])
        if c["drafts"] == "distinct":
            left[no] -= q[hand[no], x[no]].double() * ~tried[no, x[no]]
            tried[no, x[no]] = True
    up = r.cumsum(1)
    nxt = (up <= st["u_next"].double()[:, None] * up[:, -1:]).sum(1)
    new = torch.cumsum(torch.nn.functional.pad(accepted.long(), (1, 0)), 0)
    where = torch.argsort((~accepted).int(), stable=True)
    rows = torch.where(torch.arange(st["total"], device="cuda") < new[-1], where, -1)
    return dict(accepted=accepted.int(), next=nxt.int(), new_off=new[off].int(), rows=rows.int())


_plain = dict(rotary=_plain_rotary, append=_plain_append, tree=_plain_tree, verify=_plain_verify)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------
def _turned64(st, x):
    """[n][H][D] in 64 bits: complex products with magnitude * e^(i angle)."""
    rot = st["case"]["rot"]
    z = torch.polar(torch.full_like(st["freq"], st["magnitude"]).expand(st["pos"].numel(), -1).contiguous(), st["pos"].double()[:, None] * st["freq"][None])[:, None]
    y = x.double().clone()
    i = torch.arange(rot // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if st["case"]["pairs"] else (i, i + rot // 2)
    w = torch.complex(y[..., a], y[..., b]) * z
    y[..., a], y[..., b] = w.real, w.imag
    return y


def _four_bits64(x):
    g = x.unflatten(-1, (-1, 32))
    lo, hi = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
    s = ((hi - lo) / 15).to(BF16).double()
    return (lo + s * torch.round((g - lo) / torch.where(s > 0, s, 1.0)).clamp(max=15)).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "verify":             # whole numbers only
        return None
    D = case["D"]
    if case["op"] == "rotary":
        return dict(Q=_turned64(st, st["Q"]), K=_turned64(st, st["K"]))
    if case["op"] == "append":             # the cache's input is bf16: K is rounded to it once
        at = torch.arange(case["n"], device="cuda") if st["rows"] is None else st["rows"].long()
        k = _turned64(st, st["K"][at]).to(BF16).double() if case["rot"] else st["K"][at].double()
        out = dict(K=_four_bits64(k), V=_four_bits64(st["V"][at].double()))
        return dict(out, Q=_turned64(st, st["Q"])) if case["H_q"] else out
    G, raw, off, par = case["H_q"] // case["H_kv"], st["pages"], st["off"].tolist(), st["parent"].tolist()
    out = torch.empty(st["O"].shape, dtype=F64, device="cuda")
    # where element d of token r of a page lies, written out from the layout's formulas
    r, d = torch.arange(PAGE, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    run_, h, g = r // 16, (r % 16) // 8, r % 8
    k_byte = run_ * 8 * D + h * 4 * D + (4 * g + d % 32 // 8) * (D // 8) + 4 * (d // 32) + d % 8 // 2
    k_high = (d % 2).expand(PAGE, D)
    t, e = r % 8 // 2, r % 2
    v_byte = 32 * D + run_ * 8 * D + h * 4 * D + (4 * (d % 8) + t) * (D // 8) + e * (D // 16) + (d % 16 // 8) * (D // 32) + d // 32
    v_high = (d // 16 % 2).expand(PAGE, D)
    for b, n in enumerate(st["len"].tolist()):
        lo, hi = off[b], off[b + 1]
        T = hi - lo
        sees = torch.zeros(T, T, dtype=torch.bool)
        for i in range(T):
            if par[lo + i] >= 0:
                sees[i] = sees[par[lo + i]]
            sees[i, i] = True
        mask = torch.cat((torch.ones(T, n, dtype=torch.bool), sees), 1).cuda()
        ids = st["page_of"][b, :_pages(n)].long()
        for hk in range(case["H_kv"]):
            block = raw[ids, hk]
            vals = []
            for byte, high, at, new in ((k_byte, k_high, 64 * D, st["K"]), (v_byte, v_high, 72 * D, st["V"])):
                codes = (block[:, byte.reshape(-1)].view(-1, PAGE, D) >> (4 * high)) & 15
                sb = block[:, at:at + 8 * D].contiguous().view(BF16).double().view(-1, PAGE, D // 32, 2)
                held = (codes.double() * sb[..., 0].repeat_interleave(32, -1) + sb[..., 1].repeat_interleave(32, -1)).view(-1, D)[:n]
                vals.append(torch.cat((held, new[lo:hi, hk].double())))
            for hq in range(hk * G, (hk + 1) * G):
                s = st["Q"][lo:hi, hq].double() @ vals[0].T / math.sqrt(D)
                out[lo:hi, hq] = torch.softmax(torch.where(mask, s, -math.inf), 1) @ vals[1]
    return out
