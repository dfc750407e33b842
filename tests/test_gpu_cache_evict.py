"""grand_cache_evict and grand_cache_attend_ids against their definitions:
ties, zeros of both signs, NaN, budgets below what is fixed, lengths of
nothing and partly filled pages; lists of every kind, priors, refusals."""
import math

import numpy as np
import pytest

from cache_ref import INVALID, evict_ref, ids_ref
from parity import say

pytestmark = pytest.mark.gpu


def evict(page, heads, lens, budget, sinks, recent, weights, table, cap=None):
    import torch

    from paper_2608_21163_amd import Cache

    cache = Cache("bf16", heads, heads, 64, page, stream=torch.cuda.current_stream().cuda_stream)
    s = cache.sequences(torch.from_numpy(table.view(np.int32)).cuda(), torch.from_numpy(lens.view(np.int32)).cuda(), max_k=int(lens.max(initial=0)))
    got = cache.evict(s, weights, torch.from_numpy(budget.view(np.int32)).cuda(), sinks, recent)
    cache.check()
    cache.close()
    return [x.cpu().numpy() for x in got]


def check(page, heads, lens, budget, sinks, recent, weights, extra_pages=2):
    import torch

    lens, budget = np.array(lens, np.uint32), np.array(budget, np.uint32)
    n = -(-int(lens.max(initial=0)) // page) + extra_pages
    table = np.random.default_rng(1).permutation(len(lens) * n).astype(np.uint32).reshape(len(lens), n)
    want = evict_ref(table, lens, weights, budget, page, sinks, recent)
    got = evict(page, heads, lens, budget, sinks, recent, torch.from_numpy(weights).cuda(), table)
    for name, w, g in zip(("table", "weights", "lens", "freed", "n_freed"), want, got):
        same = np.array_equal(w.view(np.uint32), g.view(np.uint32))
        assert same, name


def random_weights(seed, n, heads, cap, ties=False):
    r = np.random.default_rng(seed)
    w = r.random((n, heads, cap)).astype(np.float32) ** 6
    if ties:
        w = np.round(w * 3) / 3
    w[r.random(w.shape) < 0.1] = 0
    return w.astype(np.float32)


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("page,heads,lens,budget", [
    (1, 1, [50], [20]), (16, 2, [100, 33, 16, 0, 1], [3, 1, 1, 4, 0]), (8, 3, [8 * 40, 8 * 40 - 1], [11, 39]),
    (1, 2, [5000, 1, 2049], [1234, 1, 2048]), (64, 8, [64 * 9, 700], [4, 400]), (1, 1, [40_000], [17]), (1, 1, [40_000], [39_999]),
    (4, 1, [4 * 1500, 4 * 1024, 4 * 1025], [700, 1, 1024])])
@pytest.mark.parametrize("sinks,recent", [(0, 0), (1, 4), (3, 100000)])
def test_evict(ties, page, heads, lens, budget, sinks, recent):
    say(f"[evict] pages of {page}, {heads} heads, {lens} -> {budget}, {sinks} {recent} ties {ties}")
    check(page, heads, lens, budget, sinks, recent, random_weights(page + heads, len(lens), heads, max(lens) + 3, ties))


@pytest.mark.parametrize("n", [2000, 70_000])
def test_odd_scores(n):
    """NaN counts as -inf, both zeros are one, infinities order as numbers
    do, and equal scores stay lowest index first."""
    w = np.random.default_rng(0).choice(np.array([0.0, -0.0, 1.0, -1.0, math.inf, -math.inf, math.nan, 1e-42, -1e-42, 3.4e38], np.float32),
                                        (1, 1, n)).astype(np.float32)
    for budget in (1, n // 10, n // 2, n - n // 20, n - 1):
        say(f"[evict odd] {n} -> {budget}")
        check(1, 1, [n], [budget], 0, 0, w)


@pytest.mark.parametrize("value", [0.0, 2.5])
def test_all_scores_equal(value):
    w = np.full((2, 1, 3000), value, np.float32)
    check(1, 1, [3000, 2999], [1000, 1], 0, 0, w)


def test_long_histories():
    w = random_weights(3, 2, 2, 300_001)
    check(1, 2, [300_001, 123_457], [150_000, 100_000], 4, 1000, w)


def test_strided_weights_and_length_zero():
    import torch

    w = random_weights(4, 2, 3, 64)
    lens, budget = np.array([60, 0], np.uint32), np.array([2, 0], np.uint32)
    table = np.arange(8, dtype=np.uint32).reshape(2, 4)
    want = evict_ref(table, lens, w, budget, 16, 0, 0)
    wide = torch.full((2, 7, 100), math.nan, device="cuda")
    wide[:, 1:4, :64] = torch.from_numpy(w).cuda()
    got = evict(16, 3, lens, budget, 0, 0, wide[:, 1:4, :64], table)
    assert all(np.array_equal(a.view(np.uint32), b.view(np.uint32)) for a, b in zip(want, got))


def test_evict_refusals_and_reports():
    import torch

    from paper_2608_21163_amd import Cache, GrandError
    from paper_2608_21163_amd.grand import E_ARG

    cache = Cache("bf16", 2, 2, 64, 16)
    table = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    lens = torch.tensor([64, 30], dtype=torch.int32, device="cuda")
    budget = torch.tensor([1, 1], dtype=torch.int32, device="cuda")
    w = torch.zeros(2, 2, 64, device="cuda")
    s = cache.sequences(table, lens, max_k=64)
    for bad in (lambda: cache.evict(s, w[:, :, :60], budget), lambda: cache.evict(s, w.double(), budget), lambda: cache.evict(s, w, budget[:1]),
                lambda: cache.evict(s, w, budget.float())):
        with pytest.raises(ValueError):
            bad()
    s = cache.sequences(table, lens, max_k=50)
    cache.evict(s, w, budget)
    with pytest.raises(GrandError) as e:
        cache.check()
    assert e.value.code == E_ARG and "sequence 0" in str(e.value)
    cache.check()


# ------------------------------------------------------------------ lists
def make_ids(dtype, hq, hk, dim, page, slots, b, k, seed=0, layout="token"):
    import torch

    g = torch.Generator().manual_seed(seed)
    td = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    kp = torch.randn(slots // page, page, hk, dim, generator=g).to(td)
    vp = torch.randn(slots // page, page, hk, dim, generator=g).to(td)
    q = (torch.randn(b, hq, dim, generator=g) * 2).to(td)
    ids = torch.randint(0, slots, (b, hq, k), generator=g).to(torch.int32)
    ids[torch.rand(b, hq, k, generator=g) < 0.2] = -1
    if b * hq > 1:
        ids.view(b * hq, k)[1] = -1                                  # a list of nothing
    up = (lambda x: x.cuda().transpose(1, 2).contiguous().transpose(1, 2)) if layout == "head" else (lambda x: x.cuda())
    return dict(dtype=dtype, hq=hq, hk=hk, dim=dim, page=page, k=kp, v=vp, kp=up(kp), vp=up(vp), q=q, ids=ids)


def run_ids(c, ids=None, prior=None, **kw):
    import torch

    from paper_2608_21163_amd import Cache

    cache = Cache(c["dtype"], c["hq"], c["hk"], c["dim"], c["page"], stream=torch.cuda.current_stream().cuda_stream)
    out, lse = cache.attend_ids(c["q"].cuda(), c["kp"], c["vp"], c["ids"].cuda() if ids is None else ids, prior=prior, **kw)
    cache.check()
    cache.close()
    return out, lse


def compare_ids(c, out, lse, ids=None, prior=None, scale=None):
    ids = (c["ids"] if ids is None else ids).cpu().numpy().view(np.uint32)
    flat = [x.double().numpy().reshape(-1, c["hk"], c["dim"]) for x in (c["k"], c["v"])]
    p = None if prior is None else (prior[0].double().cpu().numpy(), prior[1].double().cpu().numpy())
    o, z, bound, z_err = ids_ref(c["q"].double().numpy(), *flat, ids, c["dim"] ** -0.5 if scale is None else scale, p)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = np.isneginf(z)
    assert np.array_equal(np.isneginf(lse), empty) and not out[empty].any()
    err = np.abs(out - o)
    assert (err <= bound(c["dtype"])).all(), f"out off by {err.max()}"
    zerr = np.abs(np.where(empty, 0, lse) - np.where(empty, 0, z))
    assert (zerr <= z_err + 1e-30).all(), f"lse off by {zerr.max()}"


@pytest.mark.parametrize("dtype,layout", [("bf16", "token"), ("f16", "head")])
@pytest.mark.parametrize("hq,hk,dim,page,b,k", [(4, 2, 64, 1, 3, 10), (8, 8, 128, 16, 2, 100), (14, 2, 80, 8, 1, 33), (5, 1, 256, 64, 2, 7),
                                                (3, 3, 8, 2, 2, 300), (6, 2, 192, 1, 2, 256), (2, 1, 96, 4, 70, 1), (1, 1, 64, 1, 1, 1),
                                                (4, 1, 128, 1, 2, 1000)])
@pytest.mark.parametrize("with_prior", [False, True])
def test_lists(dtype, layout, hq, hk, dim, page, b, k, with_prior):
    import torch

    say(f"[ids] {dtype} {layout} {hq}/{hk} x {dim}, pages of {page}, {b} x {k}, prior {with_prior}")
    c = make_ids(dtype, hq, hk, dim, page, 512, b, k, seed=k, layout=layout)
    prior = None
    if with_prior:
        g = torch.Generator().manual_seed(7)
        prior = ((torch.randn(b, hq, dim, generator=g)).to(c["q"].dtype).cuda(), torch.randn(b, hq, generator=g).cuda() * 3)
        prior[1].view(-1)[0] = -math.inf
        prior[1].view(-1)[-1] = -math.inf
    compare_ids(c, *run_ids(c, prior=prior), prior=prior)


def test_nothing_to_attend_to():
    import torch

    c = make_ids("bf16", 4, 2, 64, 1, 64, 2, 5)
    ids = torch.full((2, 4, 5), -1, dtype=torch.int32, device="cuda")
    out, lse = run_ids(c, ids)
    assert not out.any() and torch.isneginf(lse).all()
    out, lse = run_ids(c, ids[:, :, :0])
    assert not out.any() and torch.isneginf(lse).all()
    nan = torch.full((2, 4, 64), math.nan, dtype=torch.bfloat16, device="cuda")     # an empty window's out is never read
    out, lse = run_ids(c, ids, prior=(nan, torch.full((2, 4), -math.inf, device="cuda")))
    assert not out.any() and torch.isneginf(lse).all()
    prior = (torch.randn(2, 4, 64, device="cuda").bfloat16(), torch.randn(2, 4, device="cuda"))
    out, lse = run_ids(c, ids, prior=prior)
    assert torch.equal(out, prior[0]) and torch.allclose(lse, prior[1], rtol=1e-6, atol=1e-6)


def test_slots_outside_the_lists_hold_anything():
    import torch

    c = make_ids("f16", 4, 2, 64, 4, 256, 2, 30, seed=3)
    c["ids"] = torch.where(c["ids"] < 0, c["ids"], c["ids"] % 100 + 50)
    clean = run_ids(c)
    kp, vp = c["kp"].clone(), c["vp"].clone()
    for x in (kp, vp):
        x.view(256, 2, 64)[:50] = math.nan
        x.view(256, 2, 64)[150:] = math.inf
    got = run_ids(dict(c, kp=kp, vp=vp))
    assert torch.equal(clean[0], got[0]) and torch.equal(clean[1], got[1])


def test_shared_lists():
    """A list for every sequence or key/value head, by strides of 0."""
    import torch

    c = make_ids("bf16", 6, 2, 64, 1, 128, 3, 20)
    for ids in (c["ids"][:, :1].cuda().expand(3, 6, 20), c["ids"][:1, :1].cuda().expand(3, 6, 20)):
        compare_ids(c, *run_ids(c, ids), ids=ids)


def test_joined_with_the_window():
    """Lists and window of one cache: together they are attention over all
    of it."""
    import torch

    from paper_2608_21163_amd import Cache

    g = torch.Generator().manual_seed(0)
    b, n, hq, hk, dim, w = 2, 200, 4, 2, 64, 31
    kp = torch.randn(b * n, 1, hk, dim, generator=g).bfloat16().cuda()
    vp = torch.randn(b * n, 1, hk, dim, generator=g).bfloat16().cuda()
    q = torch.randn(b, hq, dim, generator=g).bfloat16().cuda()
    table = torch.randperm(b * n, generator=g).to(torch.int32).view(b, n).cuda()
    cache = Cache("bf16", hq, hk, dim, 1, stream=torch.cuda.current_stream().cuda_stream)
    s = cache.sequences(table, torch.tensor([n, n], dtype=torch.int32).cuda(), max_k=n)
    whole, z = cache.attend(s, q, kp, vp)
    near = cache.attend(s, q, kp, vp, window=w)
    out, lse = cache.attend_ids(q, kp, vp, table[:, None, :n - w].expand(b, hq, n - w), prior=near)
    cache.check()
    # the window's part was rounded to bf16 once more, probabilities once on one side only
    assert torch.allclose(lse, z, rtol=0, atol=2e-5)
    assert ((out.float() - whole.float()).abs() <= 2.0 ** -7 * (1 + whole.float().abs())).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_results_in_place_of_the_earlier_ones(dim):
    import torch

    from paper_2608_21163_amd import Cache

    g = torch.Generator().manual_seed(dim)
    b, hq, hk, n, k = 64, 8, 2, 300, 40
    kp, vp = (torch.randn(n, 1, hk, dim, generator=g).bfloat16().cuda() for _ in range(2))
    q, o = (torch.randn(b, hq, dim, generator=g).bfloat16().cuda() for _ in range(2))
    z = torch.randn(b, hq, generator=g).cuda()
    ids = torch.randint(0, n, (b, hq, k), generator=g).to(torch.int32).cuda()
    cache = Cache("bf16", hq, hk, dim, 1, stream=torch.cuda.current_stream().cuda_stream)
    want, zw = cache.attend_ids(q, kp, vp, ids, prior=(o, z))
    out, lse = o.clone(), z.clone()
    cache.attend_ids(q, kp, vp, ids, prior=(out, lse), out=out, lse=lse)
    cache.check()
    assert torch.equal(out, want) and torch.equal(lse, zw)


def test_ids_refusals_and_reports():
    import torch

    from paper_2608_21163_amd import Cache, GrandError
    from paper_2608_21163_amd.grand import E_ARG, E_ID

    c = make_ids("bf16", 4, 2, 64, 4, 64, 2, 5)
    cache = Cache("bf16", 4, 2, 64, 4, stream=torch.cuda.current_stream().cuda_stream)
    q, ids = c["q"].cuda(), c["ids"].cuda()
    good = cache.attend_ids(q, c["kp"], c["vp"], ids)
    bad = ids.clone()
    bad[1, 2, 3] = 64
    out, lse = cache.attend_ids(q, c["kp"], c["vp"], bad)
    with pytest.raises(GrandError) as e:
        cache.check()
    assert e.value.code == E_ID and "sequence 1" in str(e.value)
    assert torch.equal(out[0], good[0][0])
    with pytest.raises(GrandError) as e:
        cache.attend_ids(q, c["kp"], c["vp"], ids, scale=-1.0)
    assert e.value.code == E_ARG
    for f in (lambda: cache.attend_ids(q, c["kp"], c["vp"], ids[0]), lambda: cache.attend_ids(q, c["kp"], c["vp"], ids.long()),
              lambda: cache.attend_ids(q[:1], c["kp"], c["vp"], ids), lambda: cache.attend_ids(q, c["kp"], c["vp"], ids, prior=(q, good[1][:1])),
              lambda: cache.attend_ids(q.half(), c["kp"], c["vp"], ids)):
        with pytest.raises(ValueError):
            f()
    cache.check()
