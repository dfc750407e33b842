"""The measured work of the cache operators beside those of operators.py: a
cache held in 4 bits, windows whose first tokens stay visible, and sequences
that share pages.

Operators (key "op" of a case):
  attend         a chunk of new tokens per sequence over 16-bit pages, with a
                 sliding window and some first tokens that every row sees
  attend_packed  a chunk per sequence over pages held in 4 bits, optionally with
                 window, first tokens and running sums of attention weight
  ids_packed     one new token per sequence over a list of 4-bit slots per query
                 head, joined with the result of the recent window
  append_packed  the keys and values of the new tokens go into 4-bit pages, and
                 are read back as they are held (as an index of the keys needs them)
  pages          what: "branch"   sequences go on from copies of others (a step of
                                  a beam or of parallel samples): shared pages,
                                  new pages, copies of the partly filled ones
                       "release"  finished sequences give their pages back
                       "compact"  the pages in use move to the pool's front

Packed rows: blocks of 32 elements, each 16 bytes of codes (the element of even
index in a byte's low half) and one scale byte s.  A code is a sign and a
magnitude of 0, 0.5, 1, 1.5, 2, 3, 4 or 6; the value is that times 2^(s - 127).
"""
import math
import random

import numpy as np
import torch

own = False

INVALID = -1  # GRAND_INVALID's bits in an int32 tensor
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EXPONENTS = {"bf16": (-125, 125), "f16": (-23, 13)}  # of scales, so that all values are ordinary ones of the type


def _case(op, name, **kw):
    c = dict(op=op, dtype="bf16", n_seq=1, q_heads=32, kv_heads=8, dim=128, page=16, layout="head", max_q=1, max_k=1024,
             spread=False, window=0, sinks=0, weights=False, lens_seed=1)
    c.update(kw)
    return dict(c, name=name)


def _ids(name, **kw):
    c = dict(op="ids_packed", dtype="bf16", n_seq=8, q_heads=32, kv_heads=8, dim=128, page=1, layout="token", pool=262_144,
             k=100, prior=True)
    c.update(kw)
    return dict(c, name=name)


def _pages(what, name, **kw):
    c = dict(op="pages", what=what, dtype="bf16", n_seq=64, kv_heads=8, dim=128, page=16, layout="token", width=4, max_k=4096,
             spare=0.25, lens_seed=5)
    c.update(kw)
    return dict(c, name=name)


def listed():
    return [
        # a serving batch's step: 64 streams of any length up to 8,192 tokens, of which the last 1,024 and the first 4 are seen
        _case("attend", "sinks_step_64", n_seq=64, max_k=8192, spread=True, window=1024, sinks=4, layout="token"),
        # ragged chunks of a narrow model over a pool of single slots, whose weights are summed for eviction
        _case("attend", "sinks_chunk_d64", n_seq=7, dtype="f16", q_heads=12, kv_heads=12, dim=64, page=1, max_q=300, max_k=5001,
              spread=True, window=1000, sinks=33, weights=True, layout="token"),
        # a serving batch's step over a packed cache, heads outermost in a page
        _case("attend_packed", "packed_step_64", n_seq=64, max_k=8192, spread=True),
        # two very long histories, whose weights are summed for eviction; heads inside a slot
        _case("attend_packed", "packed_long_weights", n_seq=2, dtype="f16", max_k=131_072, page=64, layout="token", weights=True),
        # the last chunk of a long prompt
        _case("attend_packed", "packed_chunk_2k", max_q=2048, max_k=32_768),
        # a step of 8 sequences over the 100 slots that each head's index search returned (the paper's top-100 lists)
        _ids("packed_ids_8x100"),
        # a full serving batch at the widest result list
        _ids("packed_ids_256x256", n_seq=256, pool=1_000_000, k=256),
        # the step's new tokens
        _case("append_packed", "packed_append_64", n_seq=64, max_k=1000, spread=True, lens_seed=3),
        # whole prompts
        _case("append_packed", "packed_append_prompts", n_seq=4, max_q=2048, max_k=2048, lens_seed=3),
        # 16 prompts with four beams each: every beam goes on from one of its prompt's
        _pages("branch", "branch_64"),
        # a third of a serving batch's sequences have ended
        _pages("release", "release_512", n_seq=512, width=2, max_k=8192),
        # a pool after a busy hour, half of it free, made ready to be handed back
        _pages("compact", "compact_half", n_seq=32, width=1, max_k=4096, spare=1.0),
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
    op = rng.choice(["attend", "attend", "attend_packed", "attend_packed", "attend_packed", "ids_packed", "append_packed", "pages"])
    kv = rng.choice([1, 2, 4, 8, 8, 12])
    common = dict(dtype=rng.choice(["bf16", "f16"]), kv_heads=kv, dim=rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256]),
                  page=rng.choice([1, 8, 16, 16, 32, 64, 128]), layout=rng.choice(["token", "head"]))
    if op == "pages":
        width = rng.choice([1, 2, 4, 8])
        c = _pages(rng.choice(["branch", "release", "compact"]), "", n_seq=width * _log(rng, 1, 512 // width), width=width,
                   max_k=_log(rng, 4 * common["page"], 16_384), spare=rng.choice([0.2, 0.5, 1.0]), lens_seed=rng.randrange(1 << 20), **common)
        del c["name"]
        return c
    common["q_heads"] = kv * rng.choice([1, 2, 4, 4, 5, 7, 8])
    if op == "ids_packed":
        c = _ids("", n_seq=_log(rng, 1, 256), pool=_log(rng, 4_096, 1_000_000), k=_log(rng, 1, 256), prior=rng.random() < 0.6, **common)
        c["pool"] = -(-c["pool"] // c["page"]) * c["page"]
        del c["name"]
        return c
    n_seq = _log(rng, 1, 64)
    max_q = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
    if op == "append_packed":
        # (pools that a pass returns whole: they stay small)
        c = _case(op, "", n_seq=n_seq, max_q=max_q, max_k=_log(rng, max(16, max_q), max(1024, max_q)), spread=rng.random() < 0.6,
                  lens_seed=rng.randrange(1 << 20), **common)
    else:
        windowed = op == "attend" or rng.random() < 0.3
        c = _case(op, "", n_seq=n_seq, max_q=max_q, max_k=_log(rng, max(16, max_q), 131_072), spread=rng.random() < 0.6,
                  window=_log(rng, 64, 4096) if windowed else 0, sinks=rng.choice([1, 4, 4, 16, 33, 64, 100]) if windowed else 0,
                  weights=rng.random() < 0.4, lens_seed=rng.randrange(1 << 20), **common)
    del c["name"]
    return c


# ------------------------------------------------------------------- sizes
def _lengths(case):
    """(chunk lengths, cached lengths including the chunk): fixed by the case,
    so that the work is.  The first sequence has the largest of both."""
    r = random.Random(case["lens_seed"])
    qs, ks = [], []
    for b in range(case["n_seq"]):
        q, k = case["max_q"], case["max_k"]
        if case["spread"] and b:
            q = 1 if q == 1 else r.randint(1, q)
            k = r.randint(min(q, k), k)
        qs.append(q)
        ks.append(k)
    return qs, ks


def _groups(case):
    """The sequences of a pages case: (lens, pages shared by a group's
    sequences, parents, ended): groups of `width` sequences have a common
    front of whole pages; a sequence goes on from one of its group's, and a
    third have ended."""
    r = random.Random(case["lens_seed"])
    ps, lens, common = case["page"], [], []
    for _ in range(case["n_seq"] // case["width"]):
        front = r.randint(0, case["max_k"] // ps - 1)
        common.append(front)
        for _ in range(case["width"]):
            lens.append(front * ps + r.randint(1, case["max_k"] - front * ps))
    n, w = case["n_seq"], case["width"]
    parents = [b // w * w + r.randrange(w) for b in range(n)]
    return lens, common, parents, sorted(r.sample(range(n), -(-n // 3)))


def _counts(case):
    """(pages that tables name, each counted once; names in tables; pages of the pool)."""
    lens, common, _, _ = _groups(case)
    ps, w = case["page"], case["width"]
    names = sum(-(-n // ps) for n in lens)
    used = names - sum(c * (w - 1) for c in common)
    return used, names, used + max(2 * case["n_seq"], int(used * case["spare"]))


def _row(case):
    """Bytes of a packed row: codes and scales."""
    blocks = -(-case["dim"] // 32)
    return case["dim"] // 2 + blocks


def _page_count(case):
    return [-(-k // case["page"]) for k in _lengths(case)[1]]


def _pool_bytes(case):
    if case["op"] == "pages":
        if case["what"] == "release":
            return 0
        return 4 * case["kv_heads"] * case["dim"] * case["page"] * _counts(case)[2]
    slots = case["pool"] if case["op"] == "ids_packed" else sum(_page_count(case)) * case["page"]
    return slots * case["kv_heads"] * (case["dim"] * 4 if case["op"] == "attend" else 2 * _row(case))


def _seen(q, k, window, sinks):
    """(Key positions that the rows of a chunk see, summed over its rows; tokens that some row sees)."""
    if not window:
        return q * k - q * (q - 1) // 2, k
    pairs = 0
    for i in range(q):
        n = k - q + i + 1
        pairs += min(n, window) + max(0, min(sinks, n - window))
    first = max(0, k - q - window + 1)
    return pairs, k - first + min(sinks, first)


def work(case):
    op, hk, d = case["op"], case["kv_heads"], case["dim"]
    if op == "pages":
        return _pages_work(case)
    if op == "ids_packed":
        hq, b, k = case["q_heads"], case["n_seq"], case["k"]
        rows = b * hq
        io = rows * (2 * d * 2 + 4) + (rows * (2 * d + 4) if case["prior"] else 0)
        # slots read twice only because two lists hold them need not be fetched twice
        pairs = min(rows * k, case["pool"] * hk)
        return {"bytes": io + rows * k * 4 + pairs * 2 * _row(case), "flops": rows * k * d * 4}
    qs, ks = _lengths(case)
    tok = sum(qs)
    if op == "append_packed":
        # rows in, codes and scales out and in, rows out
        return {"bytes": 2 * tok * hk * (2 * 2 * d + 2 * _row(case)) + 8 * tok, "flops": 2 * tok * hk * d * 2}
    hq = case["q_heads"]
    seen = [_seen(q, k, case["window"], case["sinks"]) for q, k in zip(qs, ks)]
    kept = sum(s for _, s in seen)
    b = kept * hk * (d * 4 if op == "attend" else 2 * _row(case)) + tok * hq * (2 * d * 2 + 4) + 4 * (kept // case["page"])
    if case["weights"]:
        b += 2 * 4 * hk * sum(ks)
    return {"bytes": b, "flops": 4 * d * hq * sum(p for p, _ in seen)}


def _pages_work(case):
    lens, common, parents, ended = _groups(case)
    ps, w = case["page"], case["width"]
    n = [-(-x // ps) for x in lens]
    used, names, pool = _counts(case)
    page = 2 * 2 * case["kv_heads"] * case["dim"] * ps
    refs = 2 * 4 * pool
    if case["what"] == "release":
        gone = set(ended)
        return {"bytes": refs + 4 * sum(n[b] for b in ended) + 4 * pool, "flops": len(gone)}
    if case["what"] == "compact":
        moved = used * (pool - used) // pool
        return {"bytes": refs + 2 * 4 * names + 2 * moved * (page + 4), "flops": names}
    copies = 0
    for b in range(case["n_seq"]):
        if lens[parents[b]] % ps and parents.count(parents[b]) > 1:
            copies += 1
    return {"bytes": refs + 2 * 4 * (names + sum(n[p] for p in parents)) + 2 * copies * page, "flops": names}


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


def _channels(case, gen):
    """What the elements of keys are multiplied by: some channels of a head are larger than the rest."""
    x = torch.rand(case["kv_heads"], case["dim"], generator=gen, device="cuda")
    return torch.where(x < 0.05, torch.full_like(x, 3.0), torch.ones_like(x))


def _packed_pool(case, n_pages, gen):
    """[(codes, scales) of keys, of values], views as above, of normal rows."""
    ps, hk, d = case["page"], case["kv_heads"], case["dim"]
    blocks = -(-d // 32)
    tall = _channels(case, gen)
    res = []
    for which in range(2):
        codes = torch.empty((n_pages, hk, ps, 16 * blocks), dtype=torch.uint8, device="cuda")
        scales = torch.empty((n_pages, hk, ps, blocks), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 25) // (hk * ps * d))
        for p in range(0, n_pages, step):
            x = torch.empty((min(step, n_pages - p), hk, ps, d), device="cuda").normal_(generator=gen)
            if which == 0:
                x = x * tall[:, None, :]
            codes[p:p + step], scales[p:p + step] = _pack(x, case["dtype"])
        if case["layout"] == "token":
            codes, scales = codes.transpose(1, 2).contiguous(), scales.transpose(1, 2).contiguous()
            res.append((codes, scales))
        else:
            res.append((codes.transpose(1, 2), scales.transpose(1, 2)))
    return res


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 17)
    op, b = case["op"], case["n_seq"]
    st = {"case": case}

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def normal(*s):
        return torch.empty(s, dtype=_TYPES[case["dtype"]], device="cuda").normal_(generator=gen)

    if op == "pages":
        _prepare_pages(st, gen)
    elif op == "ids_packed":
        st["k_packed"], st["v_packed"] = _packed_pool(case, case["pool"] // case["page"], gen)
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
    else:
        qs, ks = _lengths(case)
        n = _page_count(case)
        st["qs"], st["ks"], st["lens"] = qs, ks, ints(ks)
        order = torch.randperm(sum(n), generator=gen, device="cuda").to(torch.int32)
        st["table"] = torch.full((b, max(n)), INVALID, dtype=torch.int32, device="cuda")
        at = 0
        for i, m in enumerate(n):
            st["table"][i, :m] = order[at:at + m]
            at += m
        if op == "attend":
            st["k_pages"], st["v_pages"] = _pool(case, sum(n), gen)
        else:
            st["k_packed"], st["v_packed"] = _packed_pool(case, sum(n), gen)
        starts = np.concatenate([[0], np.cumsum(qs)])
        st["q_start"], st["starts"] = ints(starts.tolist()), starts.tolist()
        if op == "append_packed":
            st["k"] = normal(sum(qs), case["kv_heads"], case["dim"]) * _channels(case, gen).to(_TYPES[case["dtype"]])
            st["v"] = normal(sum(qs), case["kv_heads"], case["dim"])
            slots = [st["table"][i, pos // case["page"]] * case["page"] + pos % case["page"]
                     for i, pos in enumerate(torch.arange(k - q, k, device="cuda") for q, k in zip(qs, ks))]
            st["slots"] = torch.cat(slots).to(torch.int32)
        else:
            st["q"] = normal(sum(qs), case["q_heads"], case["dim"]) * 2
            if case["weights"]:
                st["weights"] = torch.rand(b, case["kv_heads"], case["max_k"], generator=gen, device="cuda").pow(4)
                st["weights_out"] = torch.zeros_like(st["weights"])
    _plan(st)
    return st


def _prepare_pages(st, gen):
    case = st["case"]
    lens, common, parents, ended = _groups(case)
    ps, w, n_seq = case["page"], case["width"], case["n_seq"]
    _, _, pool = _counts(case)
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32).cpu().numpy()
    table = np.full((n_seq, -(-case["max_k"] // ps) + 1), INVALID, np.int32)
    refs = np.zeros(pool, np.int32)
    at = 0
    for g, front in enumerate(common):
        shared, at = order[at:at + front], at + front
        refs[shared] += w
        for b in range(g * w, (g + 1) * w):
            rest = -(-lens[b] // ps) - front
            table[b, :front], table[b, front:front + rest] = shared, order[at:at + rest]
            refs[order[at:at + rest]] += 1
            at += rest
    st["table"], st["refs"] = torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda()
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if case["what"] == "release":
        # the rows of the sequences that have ended
        st["gone"] = torch.full_like(st["table"], INVALID)[:len(ended)]
        for i, b in enumerate(ended):
            n = -(-lens[b] // ps)
            st["gone"][i, :n] = st["table"][b, :n]
        return
    st["parents"] = torch.tensor(parents, dtype=torch.int32, device="cuda")
    st["new"] = torch.ones(n_seq, dtype=torch.int32, device="cuda")
    st["refs_out"] = torch.empty_like(st["refs"])
    st["k_pages"], st["v_pages"] = _pool(case, pool, gen)


def _plan(st):
    """The handle and the description of the sequences that a program keeps."""
    if not own:
        return
    from paper_2608_21163_amd import Cache, Packed

    c = st["case"]
    st["cache"] = Cache(c["dtype"], q_heads=c.get("q_heads", c["kv_heads"]), kv_heads=c["kv_heads"], head_dim=c["dim"],
                        page_size=c["page"], stream=torch.cuda.current_stream().cuda_stream)
    if "k_packed" in st:
        st["k_pages"], st["v_pages"] = Packed(*st["k_packed"]), Packed(*st["v_packed"])
    if c["op"] == "pages":
        st["seqs"] = st["cache"].sequences(st["table"], st["lens"], max_k=c["max_k"])
    elif c["op"] != "ids_packed":
        st["seqs"] = st["cache"].sequences(st["table"], st["lens"], q_start=st["q_start"], max_q=c["max_q"], max_k=c["max_k"])


# ------------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return _RUN_OWN[op](state)
    return _RUN_PLAIN[op](state)


def _own_attend(st):
    c = st["case"]
    return st["cache"].attend(st["seqs"], st["q"], st["k_pages"], st["v_pages"], scale=c["dim"] ** -0.5, window=c["window"],
                              sinks=c["sinks"], weights=st.get("weights"), weights_out=st.get("weights_out"))


def _own_ids(st):
    return st["cache"].attend_ids(st["q"], st["k_pages"], st["v_pages"], st["ids"], scale=st["case"]["dim"] ** -0.5,
                                  prior=st.get("prior"))


def _own_append(st):
    st["cache"].append(st["seqs"], st["k"], st["v"], st["k_pages"], st["v_pages"])
    k, v = st["cache"].read(st["slots"], st["k_pages"], st["v_pages"])
    return k, v, *st["k_packed"], *st["v_packed"]


def _own_pages(st):
    cache, what = st["cache"], st["case"]["what"]
    if what == "release":
        return cache.release(st["gone"], st["refs"], refs_out=torch.empty_like(st["refs"]))
    if what == "compact":
        table, refs, src, dst, moves = cache.compact(st["seqs"], st["refs"], refs_out=st["refs_out"])
        cache.copy_pages(st["k_pages"], st["v_pages"], src, dst)
        return table, refs, src, dst, moves, st["k_pages"], st["v_pages"]
    table, lens, refs = cache.fork(st["seqs"], st["parents"], st["refs"], drop=True, refs_out=st["refs_out"])
    seqs = cache.sequences(table, lens, max_k=st["case"]["max_k"])
    table, lens, src, dst = cache.grow(seqs, st["new"], refs)
    cache.copy_pages(st["k_pages"], st["v_pages"], src, dst)
    return table, lens, refs, src, dst, st["k_pages"], st["v_pages"]


def _pack(x, dtype):
    """Codes and scales of rows (last axis) of 32-bit values."""
    lo, hi = EXPONENTS[dtype]
    d = x.shape[-1]
    blocks = -(-d // 32)
    if d % 32:
        x = torch.cat([x, torch.zeros(*x.shape[:-1], blocks * 32 - d, device=x.device)], -1)
    x = x.reshape(*x.shape[:-1], blocks, 32)
    # the smallest exponent at which no element is 7 or more
    top = x.abs().amax(-1, keepdim=True) / 7
    fraction, e = torch.frexp(top)
    e = e.clamp(lo, hi)
    e = torch.where(top == 0, torch.full_like(e, lo), e)
    y = x * _power_table(torch.float32)[127 - e]
    m = y.abs()
    # borders between neighbours; a value on one goes to the even code
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75).to(torch.uint8) + (m > 1.25).to(torch.uint8) + (m >= 1.75).to(torch.uint8)
            + (m > 2.5).to(torch.uint8) + (m >= 3.5).to(torch.uint8) + (m > 5).to(torch.uint8))
    code = code + 8 * torch.signbit(y).to(torch.uint8)
    code = code.reshape(*code.shape[:-2], blocks * 32)
    return code[..., 0::2] + 16 * code[..., 1::2], (e[..., 0] + 127).to(torch.uint8)


_VALUES = {}


def _power_table(dtype):
    """2^(i - 127), without a function's rounding."""
    if dtype not in _VALUES:
        _VALUES[dtype] = torch.tensor([2.0 ** min(i - 127, 127) for i in range(256)], dtype=dtype, device="cuda")
    return _VALUES[dtype]


def _unpack(codes, scales, dim):
    """32-bit values of packed rows."""
    if "of_byte" not in _VALUES:
        both = [[(-1.0 if (b >> s) & 8 else 1.0) * LEVELS[(b >> s) & 7] for s in (0, 4)] for b in range(256)]
        _VALUES["of_byte"] = torch.tensor(both, dtype=torch.float32, device=codes.device)
    x = _VALUES["of_byte"][codes.int()].flatten(-2)
    x = x.reshape(*x.shape[:-1], scales.shape[-1], 32)
    x = x * _power_table(torch.float32)[scales.int()][..., None]
    return x.flatten(-2)[..., :dim]


def _slots(st, b):
    """(page, slot) of every cached token of sequence b."""
    ps, k = st["case"]["page"], st["ks"][b]
    pos = torch.arange(k, device="cuda")
    return st["table"][b].long()[pos // ps], pos % ps


def _rows_of(st, which, page, slot):
    """Keys x heads x elements in 32 bits."""
    if which + "_packed" in st:
        codes, scales = st[which + "_packed"]
        return _unpack(codes[page, slot], scales[page, slot], st["case"]["dim"])
    return st[which + "_pages"][page, slot].float()


def _plain_attend(st):
    c = st["case"]
    hk, g, d, w, sinks = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"], c["window"], c["sinks"]
    out = torch.empty_like(st["q"])
    lse = torch.empty(out.shape[:2], dtype=torch.float32, device="cuda")
    for b, (ql, kl) in enumerate(zip(st["qs"], st["ks"])):
        r0 = st["starts"][b]
        key = torch.arange(kl, device="cuda")
        if w:
            # tokens that some row sees
            key = key[(key > kl - ql - w) | (key < sinks)]
        page, slot = _slots(st, b)
        k, v = _rows_of(st, "k", page[key], slot[key]), _rows_of(st, "v", page[key], slot[key])
        q = st["q"][r0:r0 + ql].float().view(ql, hk, g, d)
        at = torch.arange(kl - ql, kl, device="cuda")[:, None]
        see = key <= at
        if w:
            see &= (key > at - w) | (key < sinks)
        see = see[:, None, :].expand(ql, g, len(key)).reshape(ql * g, len(key))
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
                new[key] += (p / l).sum(0)
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
        k, v = (_unpack(codes[at // ps, at % ps, head], scales[at // ps, at % ps, head], d)
                for codes, scales in (st["k_packed"], st["v_packed"]))
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
    c = st["case"]
    slots = st["slots"].long()
    page, slot = slots // c["page"], slots % c["page"]
    res = []
    for which in "kv":
        codes, scales = st[which + "_packed"]
        codes[page, slot], scales[page, slot] = _pack(st[which].float(), c["dtype"])
        res.append(_unpack(codes[page, slot], scales[page, slot], c["dim"]).to(st[which].dtype))
    return *res, *st["k_packed"], *st["v_packed"]


def _plain_pages(st):
    c, table, refs = st["case"], st["table"], st["refs"]
    ps, n_pages = c["page"], len(refs)
    what = c["what"]

    def names(t, keep):
        return torch.bincount(t[keep].long(), minlength=n_pages).to(torch.int32)

    def pad(x, n):
        return torch.cat([x.to(torch.int32), torch.full((n - len(x),), INVALID, dtype=torch.int32, device="cuda")])

    if what == "release":
        left = refs - names(st["gone"], st["gone"] != INVALID)
        freed = torch.nonzero((refs > 0) & (left == 0))[:, 0]
        return left, pad(freed, min(n_pages, st["gone"].numel())), torch.full((1,), len(freed), dtype=torch.int32, device="cuda")
    at = torch.arange(table.shape[1], device="cuda")
    lens = st["lens"].long()
    mine = at < (-(-lens // ps))[:, None]
    if what == "compact":
        live = refs > 0
        n_live = int(live.sum())
        at_page = torch.arange(n_pages, device="cuda")
        src, dst = at_page[live & (at_page >= n_live)], at_page[~live & (at_page < n_live)]
        to = at_page.clone()
        to[src] = dst
        new_table = torch.where(mine, to[table.long().clamp(min=0)].to(torch.int32), torch.full_like(table, INVALID))
        new_refs = refs.clone()
        new_refs[dst], new_refs[src] = refs[src], 0
        for x in (st["k_pages"], st["v_pages"]):
            x[dst] = x[src]
        count = torch.full((1,), len(src), dtype=torch.int32, device="cuda")
        return new_table, new_refs, pad(src, n_pages), pad(dst, n_pages), count, st["k_pages"], st["v_pages"]
    # every sequence goes on from its parent's
    parents = st["parents"].long()
    keep = mine[parents]
    new = torch.where(keep, table[parents], torch.full_like(table, INVALID))
    refs = refs + names(new, keep) - names(table, mine)
    lens = lens[parents]
    # pages for one more token each: of the partly filled last one a copy, if others name it
    n0, n1 = -(-lens // ps), -(-(lens + st["new"]) // ps)
    last = new.gather(1, (n0 - 1).clamp(min=0)[:, None])[:, 0]
    copy = (lens % ps != 0) & (refs[last.long().clamp(min=0)] > 1)
    need = n1 - n0 + copy
    free = torch.nonzero(refs == 0)[:, 0].to(torch.int32)
    row = torch.repeat_interleave(torch.arange(len(need), device="cuda"), need)
    nth = torch.arange(len(row), device="cuda") - (torch.cumsum(need, 0) - need)[row]
    src = torch.where(copy, last, torch.full_like(last, INVALID))
    given = free[:len(row)]
    new[row, n0[row] - copy[row].long() + nth] = given
    refs[given.long()] = 1
    refs = refs - names(src, copy)
    dst = torch.where(copy, new.gather(1, (n0 - 1).clamp(min=0)[:, None])[:, 0], torch.full_like(last, INVALID))
    for x in (st["k_pages"], st["v_pages"]):
        x[dst[copy].long()] = x[src[copy].long()]
    return new, (lens + st["new"]).to(torch.int32), refs, src, dst, st["k_pages"], st["v_pages"]


_RUN_OWN = {"attend": _own_attend, "attend_packed": _own_attend, "ids_packed": _own_ids, "append_packed": _own_append,
            "pages": _own_pages}
_RUN_PLAIN = {"attend": _plain_attend, "attend_packed": _plain_attend, "ids_packed": _plain_ids, "append_packed": _plain_append,
              "pages": _plain_pages}


# ------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions, one sequence and head (or one list, block or page)
    after another, in 64 bits."""
    st = _inputs(case, seed)
    op = case["op"]
    if op == "pages":
        return _exact_pages(case, st)
    if op == "append_packed":
        return _exact_append(case, st)
    if op == "ids_packed":
        return _exact_ids(case, st)
    return _exact_attend(case, st)


def _inputs(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _decode(codes, scales, dim):
    """64-bit values of packed rows, by arithmetic on the codes' bits."""
    nibbles = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()
    sign = torch.where(nibbles >= 8, -1.0, 1.0)
    nibbles = nibbles - 8 * (nibbles >= 8)
    power, half = torch.div(nibbles, 2, rounding_mode="floor"), nibbles % 2
    size = torch.where(power == 0, half / 2, (1 + half / 2) * 2.0 ** (power - 1))
    factor = _power_table(torch.float64)[scales.int()].repeat_interleave(32, -1)
    return (sign * size * factor)[..., :dim]


def _exact_attend(case, st):
    hq, hk, d, w = case["q_heads"], case["kv_heads"], case["dim"], case["window"]
    if 4 * d * hq * sum(_seen(q, k, 0, 0)[0] for q, k in zip(st["qs"], st["ks"])) > 4e12:
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
            if case["op"] == "attend":
                key, val = (st[n][..., h, :][flat].double() for n in ("k_pages", "v_pages"))
            else:
                key, val = (_decode(c[..., h, :][flat], s[..., h, :][flat], d) for c, s in (st["k_packed"], st["v_packed"]))
            for head in range(h * (hq // hk), (h + 1) * (hq // hk)):
                for i in range(0, ql, rows):
                    n = min(rows, ql - i)
                    query = st["q"][lo + i:lo + i + n, head].double()
                    score = torch.matmul(query, key.T.contiguous()) / math.sqrt(d)
                    where = torch.arange(kl - ql + i, kl - ql + i + n, device="cuda").unsqueeze(1)
                    hidden = pos.unsqueeze(0) > where
                    if w:
                        hidden = hidden | ((pos.unsqueeze(0) + w <= where) & (pos.unsqueeze(0) >= case["sinks"]))
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
        for i in range(0, b, 64):
            ids = st["ids"][i:i + 64, head].long()
            gone = ids < 0
            ids = ids.masked_fill(gone, 0)
            page, slot = torch.div(ids, case["page"], rounding_mode="floor"), ids % case["page"]
            keys, vals = (_decode(c[page, slot, h], s[page, slot, h], d) for c, s in (st["k_packed"], st["v_packed"]))
            query = st["q"][i:i + 64, head].double()
            score = torch.matmul(keys, query.unsqueeze(2)).squeeze(2) / math.sqrt(d)
            score = score.masked_fill(gone, -math.inf)
            z = torch.logsumexp(score, 1)
            prob = (score - z.unsqueeze(1)).exp().masked_fill(gone, 0.0)
            part = torch.matmul(prob.unsqueeze(1), vals).squeeze(1)
            if case["prior"]:
                z0 = st["prior"][1][i:i + 64, head].double()
                joint = torch.logaddexp(z0, z)
                part = part * (z - joint).exp().unsqueeze(1) + st["prior"][0][i:i + 64, head].double() * (z0 - joint).exp().unsqueeze(1)
                z = joint
            out[i:i + 64, head] = part
            lse[i:i + 64, head] = z
    return out, lse


def _exact_append(case, st):
    """The nearest of all values of a block's scale, the even code on a tie."""
    d, (lo, hi) = case["dim"], EXPONENTS[case["dtype"]]
    blocks = -(-d // 32)
    level = np.array(LEVELS)
    values, pools = [], []
    for which in "kv":
        x = st[which].double().cpu().numpy()
        x = np.concatenate([x, np.zeros(x.shape[:-1] + (blocks * 32 - d,))], -1).reshape(*x.shape[:-1], blocks, 32)
        top = np.abs(x).max(-1)
        e = np.full(top.shape, lo)
        for power in range(max(lo, -40), min(hi, 20)):    # all that the inputs need
            e[top >= 7 * 2.0 ** power] = power + 1
        y = np.abs(x) / 2.0 ** e[..., None]
        code = np.zeros(y.shape, np.int64)
        for i in range(1, 8):
            border = (level[i - 1] + level[i]) / 2
            code[(y > border) | ((y == border) & (i % 2 == 0))] = i
        value = np.where(np.signbit(x), -1.0, 1.0) * level[code] * 2.0 ** e[..., None]
        values.append(torch.from_numpy(value.reshape(*value.shape[:-2], -1)[..., :d].copy()))
        code = (code + 8 * np.signbit(x)).reshape(*code.shape[:-2], -1)
        codes, scales = (t.cpu().numpy().copy() for t in st[which + "_packed"])
        for i, slot in enumerate(st["slots"].cpu().numpy()):
            codes[slot // case["page"], slot % case["page"]] = code[i, :, 0::2] | code[i, :, 1::2] << 4
            scales[slot // case["page"], slot % case["page"]] = e[i] + 127
        pools += [torch.from_numpy(codes), torch.from_numpy(scales)]
    return *values, *pools


def _exact_pages(case, st):
    ps, what = case["page"], case["what"]
    table, refs = st["table"].cpu().numpy(), st["refs"].cpu().numpy().copy()
    lens = st["lens"].cpu().numpy()
    n_pages = len(refs)
    t = torch.from_numpy
    if what == "release":
        freed = []
        for page in st["gone"].cpu().numpy().ravel():
            if page != INVALID:
                refs[page] -= 1
                if refs[page] == 0:
                    freed.append(page)
        res = np.full(min(n_pages, st["gone"].numel()), INVALID, np.int32)
        res[:len(freed)] = sorted(freed)
        return t(refs), t(res), torch.tensor([len(freed)], dtype=torch.int32)
    k, v = st["k_pages"], st["v_pages"]
    if what == "compact":
        n_live = int((refs > 0).sum())
        holes = iter([p for p in range(n_live) if refs[p] == 0])
        to, src, dst = list(range(n_pages)), np.full(n_pages, INVALID, np.int32), np.full(n_pages, INVALID, np.int32)
        moves = 0
        for page in range(n_live, n_pages):
            if refs[page]:
                to[page] = next(holes)
                src[moves], dst[moves] = page, to[page]
                refs[to[page]], refs[page] = refs[page], 0
                moves += 1
        new = np.full_like(table, INVALID)
        for b in range(case["n_seq"]):
            for i in range(-(-int(lens[b]) // ps)):
                new[b, i] = to[table[b, i]]
        if moves:
            index_s, index_d = (torch.from_numpy(x[:moves]).long().cuda() for x in (src, dst))
            k[index_d], v[index_d] = k[index_s], v[index_s]
        return t(new), t(refs), t(src), t(dst), torch.tensor([moves], dtype=torch.int32), k.double(), v.double()
    n_seq = case["n_seq"]
    parents = st["parents"].cpu().numpy()
    new = np.full_like(table, INVALID)
    for b in range(n_seq):
        for i in range(-(-int(lens[b]) // ps)):
            refs[table[b, i]] -= 1
    for b, p in enumerate(parents):
        for i in range(-(-int(lens[p]) // ps)):
            new[b, i] = table[p, i]
            refs[table[p, i]] += 1
    free = iter([p for p in range(n_pages) if refs[p] == 0])
    new_lens = np.array([lens[p] + 1 for p in parents], np.int32)
    src, dst, shared = np.full(n_seq, INVALID, np.int32), np.full(n_seq, INVALID, np.int32), refs.copy()
    for b in range(n_seq):
        old = int(new_lens[b]) - 1
        if old % ps == 0:
            new[b, old // ps] = next(free)
            refs[new[b, old // ps]] = 1
        elif shared[new[b, old // ps]] > 1:
            src[b], dst[b] = new[b, old // ps], next(free)
            new[b, old // ps] = dst[b]
            refs[src[b]] -= 1
            refs[dst[b]] = 1
            k[int(dst[b])], v[int(dst[b])] = k[int(src[b])], v[int(src[b])]
    return t(new), t(new_lens), t(refs), t(src), t(dst), k.double(), v.double()
