"""The measured work of the key/value-cache operators: what a program that
serves a language model from a paged cache on one GPU has them do -- attention
of new tokens over the pages, attention over the ids an index search returned,
the write of new tokens into the pages, and the eviction of the pages that
drew the least attention.

Operators (key "op" of a case):
  attend      a chunk of new tokens per sequence over its pages, optionally
              with the running sums of attention weight per cached token
  attend_ids  one new token per sequence over a list of cache slots per query
              head, joined with the result of the recent window
  append      the keys and values of the new tokens go into their pages
  evict       pages beyond a budget leave the page table, the ones with the
              smallest accumulated weight first
"""
import math
import random

import numpy as np
import torch

own = False

INVALID = -1  # GRAND_INVALID's bits in an int32 tensor


def _attend(name, **kw):
    c = dict(op="attend", dtype="bf16", n_seq=1, q_heads=32, kv_heads=8, dim=128, page=16, layout="token", max_q=1,
             max_k=1024, spread=False, window=0, weights=False, lens_seed=1)
    c.update(kw)
    return dict(c, name=name)


def _ids(name, **kw):
    c = dict(op="attend_ids", dtype="bf16", n_seq=8, q_heads=32, kv_heads=8, dim=128, page=1, layout="token",
             pool=262_144, k=100, prior=True)
    c.update(kw)
    return dict(c, name=name)


def _append(name, **kw):
    c = dict(op="append", dtype="bf16", n_seq=64, q_heads=32, kv_heads=8, dim=128, page=16, layout="token", max_q=1,
             max_k=1024, spread=False, lens_seed=3)
    c.update(kw)
    return dict(c, name=name)


def _evict(name, **kw):
    c = dict(op="evict", n_seq=64, heads=8, page=16, max_k=8192, spread=True, keep=0.75, sinks=1, recent=8, lens_seed=4)
    c.update(kw)
    return dict(c, name=name)


def listed():
    return [
        # one user, one new token, a short history: the latency of a step
        _attend("attend_one", max_k=1000),
        # a serving batch's step: 64 sequences of any length up to 8,192 tokens
        _attend("attend_step_64", n_seq=64, max_k=8192, spread=True),
        # two very long histories, whose weights are summed for eviction; pages of 64, heads outermost in a page
        _attend("attend_long_weights", n_seq=2, dtype="f16", max_k=131_072, page=64, layout="head", weights=True),
        # prompts read in chunks of 512 beside each other, up to 8,192 tokens of history
        _attend("attend_chunk_512", n_seq=4, max_q=512, max_k=8192, spread=True),
        # the last chunk of a long prompt, whose weights are summed for eviction
        _attend("attend_chunk_2k_weights", max_q=2048, max_k=32_768, weights=True),
        # ragged chunks of a narrow model over a pool of single slots with a sliding window
        _attend("attend_window_d64", n_seq=7, dtype="f16", q_heads=12, kv_heads=12, dim=64, page=1, max_q=300,
                max_k=5001, spread=True, window=1000),
        # a step of 8 sequences over the 100 slots that each head's index search returned (the paper's top-100 lists)
        _ids("ids_8x100"),
        # a full serving batch at the widest result list
        _ids("ids_256x256", n_seq=256, pool=1_000_000, k=256),
        # the step's new tokens
        _append("append_step_64", max_k=8192, spread=True),
        # whole prompts
        _append("append_prompts", n_seq=4, max_q=2048, max_k=2048),
        # 64 histories cut to three quarters, page by page
        _evict("evict_pages_64"),
        # one history of a million single slots cut to the paper's half-pool window
        _evict("evict_slots_1m", n_seq=1, heads=2, page=1, max_k=1_000_000, spread=False, keep=0.5, sinks=4, recent=1000),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 8e14)


def draw(rng):
    """One more case of the ranges above, odd sizes among them, that costs no
    more than the largest listed one."""
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most and _pool_bytes(c) <= 6e9:
            return c


def _draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "attend_ids", "append", "evict"])
    if op == "evict":
        page = rng.choice([1, 1, 16, 16, 64])
        n_seq = _log(rng, 1, 64)
        c = _evict("", n_seq=n_seq, heads=rng.choice([1, 2, 4, 8]), page=page,
                   max_k=_log(rng, max(200, 12 * page), min(1_000_000, 6_000_000 // n_seq)), spread=rng.random() < 0.5,
                   keep=rng.choice([0.1, 0.25, 0.5, 0.75, 0.95]), sinks=rng.choice([0, 1, 4]),
                   recent=rng.choice([0, 1, 5, 8]), lens_seed=rng.randrange(1 << 20))
        del c["name"]
        return c
    kv = rng.choice([1, 2, 4, 8, 8, 12])
    group = rng.choice([1, 2, 4, 4, 5, 7, 8])
    common = dict(dtype=rng.choice(["bf16", "f16"]), kv_heads=kv, q_heads=kv * group,
                  dim=rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256]), page=rng.choice([1, 8, 16, 16, 32, 64, 128]),
                  layout=rng.choice(["token", "head"]))
    if op == "attend":
        n_seq = _log(rng, 1, 64)
        max_q = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
        c = _attend("", n_seq=n_seq, max_q=max_q, max_k=_log(rng, max(16, max_q), 131_072), spread=rng.random() < 0.6,
                    window=0 if rng.random() < 0.7 else _log(rng, 64, 4096), weights=rng.random() < 0.4,
                    lens_seed=rng.randrange(1 << 20), **common)
    elif op == "attend_ids":
        c = _ids("", n_seq=_log(rng, 1, 256), pool=_log(rng, 4_096, 1_000_000), k=_log(rng, 1, 256),
                 prior=rng.random() < 0.6, **common)
        c["pool"] = -(-c["pool"] // c["page"]) * c["page"]
    else:
        max_q = 1 if rng.random() < 0.4 else _log(rng, 2, 4096)
        c = _append("", n_seq=_log(rng, 1, 64), max_q=max_q, max_k=_log(rng, max(16, max_q), 8192),
                    spread=rng.random() < 0.6, lens_seed=rng.randrange(1 << 20), **common)
    del c["name"]
    return c


# ------------------------------------------------------------------- sizes
def _lengths(case):
    """(chunk lengths, cached lengths including the chunk): fixed by the case,
    so that the work is.  The first sequence has the largest of both."""
    r = random.Random(case["lens_seed"])
    qs, ks = [], []
    for b in range(case["n_seq"]):
        q, k = case.get("max_q", 1), case["max_k"]
        if case["spread"] and b:
            q = 1 if q == 1 else r.randint(1, q)
            k = r.randint(min(q, k), k)
        qs.append(q)
        ks.append(k)
    return qs, ks


def _visible(q, k, window):
    """Key positions that the rows of a chunk see, summed over its rows."""
    if not window:
        return q * k - q * (q - 1) // 2
    return sum(min(k - q + i + 1, window) for i in range(q))


def _pages(case):
    return [-(-k // case["page"]) for k in _lengths(case)[1]]


def _pool_bytes(case):
    if case["op"] == "evict":
        return 0
    slots = case["pool"] if case["op"] == "attend_ids" else sum(_pages(case)) * case["page"]
    return slots * case["kv_heads"] * case["dim"] * 4


def work(case):
    op = case["op"]
    if op == "evict":
        qs, ks = _lengths(case)
        n = _pages(case)
        return {"bytes": 2 * 4 * (case["heads"] * sum(ks) + sum(n)) + 12 * case["n_seq"], "flops": case["heads"] * sum(ks)}
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    if op == "attend_ids":
        b, k = case["n_seq"], case["k"]
        rows = b * hq
        io = rows * (2 * d * 2 + 4) + (rows * (2 * d + 4) if case["prior"] else 0)
        # slots read twice only because two lists hold them need not be fetched twice
        pairs = min(rows * k, case["pool"] * hk)
        return {"bytes": io + rows * k * 4 + pairs * d * 4, "flops": rows * k * d * 4}
    qs, ks = _lengths(case)
    tok = sum(qs)
    if op == "append":
        return {"bytes": 2 * 2 * tok * hk * d * 2 + 4 * tok, "flops": 0}
    w = case["window"]
    seen = sum(min(k, q + w - 1) if w else k for q, k in zip(qs, ks))
    pairs = sum(_visible(q, k, w) for q, k in zip(qs, ks))
    b = seen * hk * d * 4 + tok * hq * (2 * d * 2 + 4) + 4 * sum(-(-min(k, q + w - 1 if w else k) // case["page"])
                                                                for q, k in zip(qs, ks))
    if case["weights"]:
        b += 2 * 4 * hk * sum(ks)
    return {"bytes": b, "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------- inputs
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _pool(case, n_pages, gen):
    """Key and value pages as (page, slot, head, element) views: heads inside
    a slot in memory, or slots inside a head."""
    ps, hk, d = case["page"], case["kv_heads"], case["dim"]
    shape = (n_pages, ps, hk, d) if case["layout"] == "token" else (n_pages, hk, ps, d)
    pools = []
    for _ in range(2):
        x = torch.empty(shape, dtype=_TYPES[case["dtype"]], device="cuda")
        x.normal_(generator=gen)
        pools.append(x if case["layout"] == "token" else x.transpose(1, 2))
    return pools


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 17)
    op, b = case["op"], case["n_seq"]
    st = {"case": case}

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def normal(*s):
        return torch.empty(s, dtype=_TYPES[case["dtype"]], device="cuda").normal_(generator=gen)

    if op == "attend_ids":
        st["k_pages"], st["v_pages"] = _pool(case, case["pool"] // case["page"], gen)
        # a list of distinct slots per head, as a search returns them; every eighth list is short
        start = torch.randint(0, case["pool"], (b, case["q_heads"], 1), generator=gen, device="cuda")
        step = next(p for p in (99_991, 99_989, 99_971) if math.gcd(p, case["pool"]) == 1)
        ids = (start + step * torch.arange(case["k"], device="cuda")) % case["pool"]
        short = torch.randint(0, 8, (b, case["q_heads"], 1), generator=gen, device="cuda") == 0
        count = torch.randint(0, case["k"] + 1, (b, case["q_heads"], 1), generator=gen, device="cuda")
        ids[short & (torch.arange(case["k"], device="cuda") >= count)] = INVALID
        st["ids"] = ids.to(torch.int32)
        st["q"] = normal(b, case["q_heads"], case["dim"]) * 2
        if case["prior"]:
            st["prior"] = (normal(b, case["q_heads"], case["dim"]) * 0.2,
                           torch.randn(b, case["q_heads"], generator=gen, device="cuda") + math.log(case["k"] + 1))
        _plan(st)
        return st
    qs, ks = _lengths(case)
    n = _pages(case)
    st["qs"], st["ks"] = qs, ks
    st["lens"] = ints(ks)
    order = torch.randperm(sum(n), generator=gen, device="cuda").to(torch.int32)
    table = torch.full((b, max(n)), INVALID, dtype=torch.int32, device="cuda")
    at = 0
    for i, m in enumerate(n):
        table[i, :m] = order[at:at + m]
        at += m
    st["table"] = table
    if op == "evict":
        # sums of softmax weights: heavy-tailed, a tenth of the tokens never attended
        w = torch.rand(b, case["heads"], case["max_k"], generator=gen, device="cuda")
        st["weights"] = torch.where(w < 0.1, torch.zeros_like(w), w.pow(8))
        for i, k in enumerate(ks):
            st["weights"][i, :, k:] = 0
        st["budget"] = ints([max(case["sinks"] + case["recent"] + 1, int(m * case["keep"])) for m in n])
        _plan(st)
        return st
    st["k_pages"], st["v_pages"] = _pool(case, sum(n), gen)
    starts = np.concatenate([[0], np.cumsum(qs)])
    st["q_start"] = ints(starts.tolist())
    st["starts"] = starts.tolist()
    if op == "append":
        st["k"] = normal(sum(qs), case["kv_heads"], case["dim"])
        st["v"] = normal(sum(qs), case["kv_heads"], case["dim"])
    else:
        st["q"] = normal(sum(qs), case["q_heads"], case["dim"]) * 2
        if case["weights"]:
            st["weights"] = torch.rand(b, case["kv_heads"], case["max_k"], generator=gen, device="cuda").pow(4)
            st["weights_out"] = torch.zeros_like(st["weights"])
    _plan(st)
    return st


def _plan(st):
    """The handle and the description of the sequences that a program keeps."""
    if not own:
        return
    from paper_2608_21163_amd import Cache

    c = st["case"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "evict":
        st["cache"] = Cache("bf16", q_heads=c["heads"], kv_heads=c["heads"], head_dim=64, page_size=c["page"], stream=stream)
    else:
        st["cache"] = Cache(c["dtype"], q_heads=c["q_heads"], kv_heads=c["kv_heads"], head_dim=c["dim"],
                            page_size=c["page"], stream=stream)
    if c["op"] != "attend_ids":
        q_start = st.get("q_start")
        st["seqs"] = st["cache"].sequences(st["table"], st["lens"], q_start=q_start, max_q=c.get("max_q", 1),
                                           max_k=c["max_k"])


# ------------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return _RUN_OWN[op](state)
    return _RUN_PLAIN[op](state)


def _own_attend(st):
    c = st["case"]
    return st["cache"].attend(st["seqs"], st["q"], st["k_pages"], st["v_pages"], scale=c["dim"] ** -0.5,
                              window=c["window"], weights=st.get("weights"), weights_out=st.get("weights_out"))


def _own_ids(st):
    return st["cache"].attend_ids(st["q"], st["k_pages"], st["v_pages"], st["ids"], scale=st["case"]["dim"] ** -0.5,
                                  prior=st.get("prior"))


def _own_append(st):
    st["cache"].append(st["seqs"], st["k"], st["v"], st["k_pages"], st["v_pages"])
    return st["k_pages"], st["v_pages"]


def _own_evict(st):
    c = st["case"]
    return st["cache"].evict(st["seqs"], st["weights"], st["budget"], sinks=c["sinks"], recent=c["recent"])


def _slots(st, b):
    """(page, slot) of every cached token of sequence b."""
    ps, k = st["case"]["page"], st["ks"][b]
    pos = torch.arange(k, device="cuda")
    return st["table"][b].long()[pos // ps], pos % ps


def _plain_attend(st):
    c = st["case"]
    hk, g, d, w = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"], c["window"]
    out = torch.empty_like(st["q"])
    lse = torch.empty(out.shape[:2], dtype=torch.float32, device="cuda")
    for b, (ql, kl) in enumerate(zip(st["qs"], st["ks"])):
        r0 = st["starts"][b]
        page, slot = _slots(st, b)
        first = max(0, kl - ql - w + 1) if w else 0
        page, slot = page[first:], slot[first:]
        k = st["k_pages"][page, slot].float()                      # keys x heads x elements
        v = st["v_pages"][page, slot].float()
        q = st["q"][r0:r0 + ql].float().view(ql, hk, g, d)
        at = torch.arange(kl - ql, kl, device="cuda")[:, None]
        key = torch.arange(first, kl, device="cuda")[None, :]
        see = key <= at
        if w:
            see &= key > at - w
        see = see[:, None, :].expand(ql, g, kl - first).reshape(ql * g, kl - first)
        for h in range(hk):
            qh = q[:, h].reshape(ql * g, d)
            s = (qh @ k[:, h].t().contiguous()) * d ** -0.5
            s = torch.where(see, s, torch.full_like(s, -math.inf))
            m = s.max(1, keepdim=True).values
            p = torch.exp(s - m)
            l = p.sum(1, keepdim=True)
            o = (p @ v[:, h].contiguous()) / l
            out[r0:r0 + ql, h * g:(h + 1) * g] = o.view(ql, g, d).to(out.dtype)
            lse[r0:r0 + ql, h * g:(h + 1) * g] = (m + torch.log(l)).view(ql, g)
            if c["weights"]:
                new = st["weights"][b, h, :kl].clone()
                new[first:] += (p / l).sum(0)
                st["weights_out"][b, h, :kl] = new
    if c["weights"]:
        return out, lse, st["weights_out"]
    return out, lse


def _plain_ids(st):
    c = st["case"]
    hq, d, ps = c["q_heads"], c["dim"], c["page"]
    g = hq // c["kv_heads"]
    q, ids = st["q"], st["ids"].long()
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    head = (torch.arange(hq, device="cuda") // g)[None, :, None]
    step = max(1, 400_000_000 // (hq * c["k"] * d * 4))           # sequences at a time: the gathered rows fit
    for b in range(0, q.shape[0], step):
        i = ids[b:b + step]
        ok = i >= 0
        at = i.clamp(min=0)
        k = st["k_pages"][at // ps, at % ps, head].float()
        v = st["v_pages"][at // ps, at % ps, head].float()
        s = (k * q[b:b + step].float()[:, :, None, :]).sum(-1) * d ** -0.5
        s = torch.where(ok, s, torch.full_like(s, -math.inf))
        m = s.max(-1, keepdim=True).values
        p = torch.where(ok, torch.exp(s - m), torch.zeros_like(s))
        l = p.sum(-1, keepdim=True)
        o = (p[..., None] * v).sum(2) / torch.where(l > 0, l, torch.ones_like(l))
        z = (m + torch.log(l)).squeeze(-1)
        z = torch.where(ok.any(-1), z, torch.full_like(z, -math.inf))
        if c["prior"]:
            o0, z0 = st["prior"][0][b:b + step].float(), st["prior"][1][b:b + step]
            top = torch.maximum(z0, z)
            both = top + torch.log(torch.exp(z0 - top) + torch.exp(z - top))
            o = torch.exp(z0 - both)[..., None] * o0 + torch.exp(z - both)[..., None] * o
            z = both
        out[b:b + step] = o.to(out.dtype)
        lse[b:b + step] = z
    return out, lse


def _plain_append(st):
    for b, (ql, kl) in enumerate(zip(st["qs"], st["ks"])):
        r0 = st["starts"][b]
        page, slot = _slots(st, b)
        st["k_pages"][page[kl - ql:], slot[kl - ql:]] = st["k"][r0:r0 + ql]
        st["v_pages"][page[kl - ql:], slot[kl - ql:]] = st["v"][r0:r0 + ql]
    return st["k_pages"], st["v_pages"]


def _plain_evict(st):
    c = st["case"]
    ps, heads = c["page"], c["heads"]
    table, lens, w = st["table"], st["lens"].long()[:, None], st["weights"]
    b, n_max = table.shape
    cap = w.shape[2]
    pages = -(-lens // ps)
    x = torch.zeros(b, heads, n_max * ps, device="cuda")
    x[:, :, :min(cap, n_max * ps)] = w[:, :, :n_max * ps]
    x = torch.where(torch.arange(n_max * ps, device="cuda") < lens[:, None], x, torch.zeros_like(x)).view(b, heads, n_max, ps)
    score = torch.zeros(b, n_max, device="cuda")
    for h in range(heads):                                         # in this order, in 32 bits
        for t in range(ps):
            score = score + x[:, h, :, t]
    at = torch.arange(n_max, device="cuda")[None, :]
    live = at < pages
    recent = torch.clamp((lens % ps != 0).long(), min=c["recent"])
    fixed = live & ((at < c["sinks"]) | (at >= pages - recent))
    budget = st["budget"].long()[:, None]
    need = torch.where(pages <= budget, pages, budget) - fixed.sum(1, keepdim=True)
    score = torch.where(torch.isnan(score), torch.full_like(score, -math.inf), score)
    score = torch.where(live & ~fixed, score, torch.full_like(score, -math.inf))
    rest = live & ~fixed
    # rank among the pages that may go: those first, by (score descending, page ascending)
    order = torch.sort(score, dim=1, descending=True, stable=True).indices
    first = torch.sort(rest.gather(1, order).to(torch.int8), dim=1, descending=True, stable=True).indices
    order = order.gather(1, first)
    rank = torch.empty_like(order).scatter_(1, order, at.expand(b, n_max).contiguous())
    keep = fixed | (rest & (rank < need))
    gone = live & ~keep

    def pack(mask):
        to = torch.cumsum(mask.long(), 1) - 1
        res = torch.full((b, n_max + 1), INVALID, dtype=torch.int32, device="cuda")
        res.scatter_(1, torch.where(mask, to, torch.full_like(to, n_max)), table)
        src = torch.full((b, n_max + 1), -1, dtype=torch.long, device="cuda")
        src.scatter_(1, torch.where(mask, to, torch.full_like(to, n_max)), at.expand(b, n_max).contiguous())
        return res[:, :n_max].contiguous(), src[:, :n_max]

    new_table, src = pack(keep)
    freed, _ = pack(gone)
    n_freed = gone.sum(1, keepdim=True)
    new_lens = lens - n_freed * ps
    j = torch.arange(cap, device="cuda")[None, :]
    p = src.gather(1, (j // ps).clamp(max=n_max - 1).expand(b, cap))
    tok = (p.clamp(min=0) * ps + j % ps).clamp(max=cap - 1)
    new_w = w.gather(2, tok[:, None, :].expand(b, heads, cap).contiguous())
    new_w = torch.where((j < new_lens)[:, None, :], new_w, torch.zeros_like(new_w))
    return new_table, new_w, new_lens[:, 0].to(torch.int32), freed, n_freed[:, 0].to(torch.int32)


_RUN_OWN = {"attend": _own_attend, "attend_ids": _own_ids, "append": _own_append, "evict": _own_evict}
_RUN_PLAIN = {"attend": _plain_attend, "attend_ids": _plain_ids, "append": _plain_append, "evict": _plain_evict}


# ------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions, one sequence and head (or one list) after another, in
    64 bits; the eviction's order is defined on sums in 32 bits, so those are
    taken in 32 bits here too, by numpy."""
    st = _inputs(case, seed)
    op = case["op"]
    if op == "append":
        k, v = st["k_pages"], st["v_pages"]
        for b in range(case["n_seq"]):
            for i in range(st["qs"][b]):
                pos = st["ks"][b] - st["qs"][b] + i
                page = int(st["table"][b, pos // case["page"]]) if i == 0 or pos % case["page"] == 0 else page
                k[page, pos % case["page"]] = st["k"][st["starts"][b] + i]
                v[page, pos % case["page"]] = st["v"][st["starts"][b] + i]
        return k.double(), v.double()
    if op == "evict":
        return _exact_evict(case, st)
    if op == "attend_ids":
        return _exact_ids(case, st)
    return _exact_attend(case, st)


def _inputs(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _exact_attend(case, st):
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    if 4 * d * hq * sum(_visible(q, k, 0) for q, k in zip(st["qs"], st["ks"])) > 4e12:
        return None
    tok = sum(st["qs"])
    out = torch.zeros(tok, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((tok, hq), -math.inf, dtype=torch.float64, device="cuda")
    mass = st["weights"].double() if case["weights"] else None
    if mass is not None:
        for b, kl in enumerate(st["ks"]):
            mass[b, :, kl:] = 0
    for b, (ql, kl) in enumerate(zip(st["qs"], st["ks"])):
        pos = torch.arange(kl, device="cuda")
        flat = st["table"][b, pos // case["page"]].long(), pos % case["page"]
        lo = st["starts"][b]
        rows = max(1, 120_000_000 // kl)
        for h in range(hk):
            key = st["k_pages"][..., h, :][flat].double()
            val = st["v_pages"][..., h, :][flat].double()
            for head in range(h * (hq // hk), (h + 1) * (hq // hk)):
                for i in range(0, ql, rows):
                    n = min(rows, ql - i)
                    query = st["q"][lo + i:lo + i + n, head].double()
                    score = torch.matmul(query, key.T.contiguous()) / math.sqrt(d)
                    where = torch.arange(kl - ql + i, kl - ql + i + n, device="cuda").unsqueeze(1)
                    hidden = pos.unsqueeze(0) > where
                    if case["window"]:
                        hidden = hidden | (pos.unsqueeze(0) + case["window"] <= where)
                    score = score.masked_fill(hidden, -math.inf)
                    z = torch.logsumexp(score, 1)
                    prob = (score - z.unsqueeze(1)).exp()
                    out[lo + i:lo + i + n, head] = torch.matmul(prob, val)
                    lse[lo + i:lo + i + n, head] = z
                    if mass is not None:
                        mass[b, h, :kl] += prob.sum(0)
    return (out, lse) if mass is None else (out, lse, mass)


def _exact_ids(case, st):
    b, hq, d = case["n_seq"], case["q_heads"], case["dim"]
    out = torch.zeros(b, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, hq), -math.inf, dtype=torch.float64, device="cuda")
    for head in range(hq):
        h = head // (hq // case["kv_heads"])
        keys, vals = st["k_pages"][:, :, h], st["v_pages"][:, :, h]
        for i in range(0, b, 64):
            ids = st["ids"][i:i + 64, head].long()
            gone = ids < 0
            ids = ids.masked_fill(gone, 0)
            page, slot = torch.div(ids, case["page"], rounding_mode="floor"), ids % case["page"]
            query = st["q"][i:i + 64, head].double()
            score = torch.matmul(keys[page, slot].double(), query.unsqueeze(2)).squeeze(2) / math.sqrt(d)
            score = score.masked_fill(gone, -math.inf)
            z = torch.logsumexp(score, 1)
            prob = (score - z.unsqueeze(1)).exp().masked_fill(gone, 0.0)
            part = torch.matmul(prob.unsqueeze(1), vals[page, slot].double()).squeeze(1)
            if case["prior"]:
                z0 = st["prior"][1][i:i + 64, head].double()
                joint = torch.logaddexp(z0, z)
                part = part * (z - joint).exp().unsqueeze(1) + st["prior"][0][i:i + 64, head].double() * (z0 - joint).exp().unsqueeze(1)
                z = joint
            out[i:i + 64, head] = part
            lse[i:i + 64, head] = z
    return out, lse


def _exact_evict(case, st):
    ps, heads = case["page"], case["heads"]
    table, w, budget = st["table"].cpu().numpy(), st["weights"].cpu().numpy(), st["budget"].cpu().numpy()
    new_table, freed = np.full_like(table, INVALID), np.full_like(table, INVALID)
    new_w = np.zeros_like(w)
    lens, counts = [], []
    for b, length in enumerate(st["ks"]):
        n = -(-length // ps)
        padded = np.zeros((heads, n * ps), np.float32)
        padded[:, :length] = w[b, :, :length]
        score = np.zeros(n, np.float32)
        for row in padded.reshape(heads, n, ps):
            for t in range(ps):
                score = np.add(score, row[:, t], dtype=np.float32)
        tail = max(case["recent"], 1 if length % ps else 0)
        held = [p for p in range(n) if p < case["sinks"] or p >= n - tail]
        keep = np.zeros(n, bool)
        keep[held] = True
        free = np.flatnonzero(~keep)
        room = max(0, min(n, int(budget[b])) - len(held))
        best = free[np.lexsort((free, -score[free].astype(np.float64)))][:room]
        keep[best] = True
        kept, gone = np.flatnonzero(keep), np.flatnonzero(~keep)
        new_table[b, :len(kept)] = table[b, kept]
        freed[b, :len(gone)] = table[b, gone]
        size = length - len(gone) * ps
        tokens = (kept[:, None] * ps + np.arange(ps)).reshape(-1)[:size]
        new_w[b, :, :size] = w[b][:, tokens]
        lens.append(size)
        counts.append(len(gone))
    return (torch.from_numpy(new_table), torch.from_numpy(new_w.astype(np.float64)), torch.tensor(lens, dtype=torch.int32),
            torch.from_numpy(freed), torch.tensor(counts, dtype=torch.int32))
