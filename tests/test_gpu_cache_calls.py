"""How programs use one cache handle: many splits, shared pages, calls of all
kinds after each other and in one captured graph, long tables."""
import math

import numpy as np
import pytest

from cache_ref import attend_ref, evict_ref, ids_ref
from parity import say
from test_gpu_cache_attend import cache_for, compare, make, run, seqs_for
from test_gpu_cache_evict import check, random_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ks", [140_000, 530_001])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_more_splits_than_threads(ks, dtype):
    """One head over a long cache: over 256 and over 1,024 splits of 512 keys."""
    import torch

    say(f"[cache splits] {ks} {dtype}")
    c = make(dtype, 2, 1, 16, 64, qs=(1,), ks=(ks,), seed=3)
    before = torch.rand(1, 1, ks, device="cuda")
    after = before.clone()
    out, lse, w = run(c, weights=after)
    compare(c, out, lse, weights=after, before=before)


@pytest.mark.parametrize("ks,window", [(1024, 0), (2048, 0), (2048, 512), (4096, 1000)])
@pytest.mark.parametrize("qs", [(1, 1, 1), (1, 30, 200)])
def test_bounds_that_splits_divide(ks, window, qs):
    """Caches and bounds of whole splits, with and without a window."""
    say(f"[cache splits] {qs} over {ks}, window {window}")
    c = make("bf16", 4, 1, 64, 16, qs=qs, ks=(ks, ks - 1, ks // 2), seed=ks)
    compare(c, *run(c, window=window), window=window)


@pytest.mark.parametrize("qs", [(1, 1, 1, 1), (40, 3, 65, 1)])
def test_sequences_that_share_pages(qs):
    """Four sequences name the same pages of a prefix, and their own behind it."""
    import torch

    say(f"[cache shared pages] {qs}")
    ks = (700, 650, 790, 641)
    c = make("f16", 8, 2, 64, 16, qs=qs, ks=ks, seed=11)
    for b in range(1, 4):
        c["table"][b, :32] = c["table"][0, :32]
        for name in ("keys", "vals"):
            c[name][b][:512] = c[name][0][:512]
    before = torch.rand(4, 2, max(ks), device="cuda")
    after = before.clone()
    out, lse, w = run(c, weights=after)
    compare(c, out, lse, weights=after, before=before)


@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("sinks,recent", [(0, 0), (2, 7)])
def test_long_tables_of_pages(page, sinks, recent):
    """Over 8,192 pages of several slots, an empty sequence and one that keeps
    nothing beside them."""
    n = 9001
    lens = [n * page - 1, 0, n * page, 5 * page]
    say(f"[evict long] pages of {page}, {lens}, {sinks} {recent}")
    check(page, 2, lens, [4000, 3, 0, 2], sinks, recent, random_weights(page, 4, 2, n * page + 2))


def test_evictions_after_larger_calls():
    """One handle: a long attention, a long eviction, then short ones on the
    workspace that those left."""
    import torch

    c = make("bf16", 2, 2, 64, 1, qs=(1, 1), ks=(20_000, 9_000), seed=2)
    cache = cache_for(c)
    w = torch.rand(2, 2, 20_000, device="cuda")
    s = seqs_for(cache, c)
    cache.attend(s, c["q"].cuda(), c["k_pages"], c["v_pages"], weights=w)
    for ks, budget in (((20_000, 9_000), (300, 8_999)), ((700, 300), (600, 1)), ((9_500, 31), (100, 30)), ((64, 3), (9, 9))):
        say(f"[evict after] {ks} -> {budget}")
        lens, n = torch.tensor(ks, dtype=torch.int32, device="cuda"), max(ks)
        table = c["table"][:, :n].contiguous()
        part = w[:, :, :n].contiguous()
        got = cache.evict(cache.sequences(table, lens, max_k=n), part, torch.tensor(budget, dtype=torch.int32, device="cuda"), sinks=1, recent=2)
        cache.check()
        want = evict_ref(table.cpu().numpy().view(np.uint32), np.array(ks), part.cpu().numpy(), np.array(budget), 1, 1, 2)
        assert all(np.array_equal(a.view(np.uint32), b.cpu().numpy().view(np.uint32)) for a, b in zip(want, got))


def test_a_captured_step_of_every_call():
    """Append, attention over the pages and over listed ids, and eviction,
    captured together on one handle, replayed with other inputs."""
    import torch

    from paper_2608_21163_amd import Cache

    n, hq, hk, dim, kl = 3, 4, 2, 64, 600
    stream = torch.cuda.Stream()
    cache = Cache("f16", hq, hk, dim, 1, stream=stream.cuda_stream)
    g = torch.Generator().manual_seed(4)
    kp, vp = (torch.randn(n * kl, 1, hk, dim, generator=g).half().cuda() for _ in range(2))
    table = torch.randperm(n * kl, generator=g).to(torch.int32).view(n, kl).cuda()
    lens = torch.tensor([kl, 431, 77], dtype=torch.int32, device="cuda")
    budget = torch.tensor([500, 10, 80], dtype=torch.int32, device="cuda")
    q, out, out2 = (torch.zeros(n, hq, dim, dtype=torch.float16, device="cuda") for _ in range(3))
    k, v = (torch.zeros(n, hk, dim, dtype=torch.float16, device="cuda") for _ in range(2))
    ids = torch.full((n, hq, 20), -1, dtype=torch.int32, device="cuda")
    lse, lse2 = torch.zeros(n, hq, device="cuda"), torch.zeros(n, hq, device="cuda")
    w, wo = torch.zeros(n, hk, kl, device="cuda"), torch.zeros(n, hk, kl, device="cuda")
    s = cache.sequences(table, lens, max_k=kl)

    def step():
        cache.append(s, k, v, kp, vp)
        cache.attend(s, q, kp, vp, weights=w, weights_out=wo, out=out, lse=lse)
        cache.attend_ids(q, kp, vp, ids, prior=(out, lse), out=out2, lse=lse2)
        return cache.evict(s, wo, budget, sinks=2, recent=3)

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        evicted = step()
    for i in range(3):
        say(f"[cache graph] replay {i}")
        g = torch.Generator().manual_seed(10 + i)
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g))
        w.copy_(torch.rand(w.shape, generator=g))
        ids.copy_(torch.randint(0, n * kl, ids.shape, generator=g))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, wo, out2, lse2, *evicted)]
        for x in (out, lse, wo, out2, lse2, *evicted):
            x.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            again = step()
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, wo, out2, lse2, *again)))
        # and the definitions
        tab, kf, vf = table.cpu().numpy(), kp.double().cpu().numpy(), vp.double().cpu().numpy()
        for b, length in enumerate(lens.tolist()):
            at = tab[b, :length]
            ro, rz, rw, bound, z_err, w_err = attend_ref(q[b:b + 1].double().cpu().numpy(), kf[at, 0], vf[at, 0], length - 1, dim ** -0.5)
            assert (np.abs(got[0][b:b + 1].double().cpu().numpy() - ro) <= bound("f16")).all()
            new, old = got[2][b].double().cpu().numpy()[:, :length], w[b].double().cpu().numpy()[:, :length]
            assert (np.abs(new - old - rw) <= w_err + 2.0 ** -23 * (old + rw)).all()
        o, z, bound, z_err = ids_ref(q.double().cpu().numpy(), kf[:, 0], vf[:, 0], ids.cpu().numpy().view(np.uint32), dim ** -0.5,
                                     (got[0].double().cpu().numpy(), got[1].double().cpu().numpy()))
        assert (np.abs(got[3].double().cpu().numpy() - o) <= bound("f16")).all()
        want = evict_ref(tab.view(np.uint32), lens.cpu().numpy(), got[2].cpu().numpy(), budget.cpu().numpy(), 1, 2, 3)
        assert all(np.array_equal(a.view(np.uint32), x.cpu().numpy().view(np.uint32)) for a, x in zip(want, got[5:]))
    cache.check()
    del graph
    cache.close()


def test_lists_longer_than_a_round():
    """Ids that name one slot many times."""
    import torch

    from paper_2608_21163_amd import Cache

    g = torch.Generator().manual_seed(0)
    kp, vp = (torch.randn(50, 1, 1, 64, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(1, 1, 64, generator=g).bfloat16().cuda()
    cache = Cache("bf16", 1, 1, 64, 1)
    ids = torch.full((1, 1, 5000), 7, dtype=torch.int32, device="cuda")
    out, lse = cache.attend_ids(q, kp, vp, ids)
    one, z = cache.attend_ids(q, kp, vp, ids[:, :, :1].contiguous())
    cache.check()
    assert torch.equal(out, one) and abs(float(lse - z) - math.log(5000)) < 1e-5


def test_waiting_calls_inside_a_capture():
    """The check and a change of streams are refused while the stream is
    captured; the capture and the handle go on."""
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_STATE

    c = make(qs=(1, 1), ks=(300, 40))
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    cache = cache_for(c)
    cache.set_stream(stream.cuda_stream)
    s, q = seqs_for(cache, c), c["q"].cuda()
    out, lse = torch.zeros_like(q), torch.zeros(2, 4, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cache.attend(s, q, c["k_pages"], c["v_pages"], out=out, lse=lse)
        for call in (cache.check, lambda: cache.set_stream(other.cuda_stream)):
            with pytest.raises(GrandError) as e:
                call()
            assert e.value.code == E_STATE and "capture" in str(e.value)
    for _ in range(3):
        out.zero_(), lse.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        compare(c, out, lse)
    cache.check()
    cache.set_stream(other.cuda_stream)
    cache.check()
    del graph
    cache.close()


def test_weights_of_no_cached_tokens():
    """Nothing cached and weights without entries: empty rows as without them."""
    import torch

    c = make(qs=(2, 1), ks=(0, 0))
    w = torch.zeros(2, 2, 0, device="cuda")
    out, lse, got = run(c, weights=w)
    assert got is w and not out.any() and torch.isneginf(lse).all()


def test_axes_of_one_in_any_layout():
    """One head, one sequence, one token: views whose strides there are not
    what a packed tensor has."""
    import torch

    c = make("f16", 1, 1, 64, 16, qs=(1,), ks=(130,), seed=6)
    want = run(c)
    k = c["k_pages"].as_strided(c["k_pages"].shape, (1024, 64, 1000, 1))     # the same memory, another stride of the head
    table = c["table"].as_strided(c["table"].shape, (1, 1))
    q = c["q"].cuda().as_strided((1, 1, 64), (3, 5, 1))
    assert k.stride() != c["v_pages"].stride()
    cache = cache_for(c)
    s = cache.sequences(table, c["lens"], max_k=130)
    out, lse = cache.attend(s, q, k, c["v_pages"])
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    cache.append(s, q, q, k, c["v_pages"])
    cache.check()
    assert torch.equal(k[int(table[0, 129 // 16]), 129 % 16, 0], q[0, 0])


def test_described_sequences_are_not_written_to():
    """n_tokens is what the rows must have, where it is given; where not, it is
    the rows' of each call, and the description stays as it is for others."""
    import torch

    c = make(qs=(2, 1), ks=(30, 40))
    want = run(c)
    cache = cache_for(c)
    q = c["q"].cuda()
    more = torch.cat([q, q])                      # rows of no sequence behind
    loose = seqs_for(cache, c)
    before = bytes(loose.c)
    for rows in (q, more, q):
        out, lse = cache.attend(loose, rows, c["k_pages"], c["v_pages"])
        assert torch.equal(out[:3], want[0]) and torch.equal(lse[:3], want[1])
    assert bytes(loose.c) == before
    fixed = cache.sequences(c["table"], c["lens"], c["q_start"], n_tokens=3, max_q=2, max_k=40)
    assert torch.equal(cache.attend(fixed, q, c["k_pages"], c["v_pages"])[0], want[0])
    kv = torch.zeros(6, 2, 64, dtype=torch.bfloat16, device="cuda")
    one = cache.sequences(c["table"], c["lens"], n_tokens=2, max_k=40)
    for bad in (lambda: cache.attend(fixed, more, c["k_pages"], c["v_pages"]), lambda: cache.append(fixed, kv, kv, c["k_pages"], c["v_pages"]),
                lambda: cache.attend(one, q, c["k_pages"], c["v_pages"]),
                lambda: cache.sequences(c["table"], c["lens"], n_tokens=3, max_k=40),
                lambda: cache.sequences(c["table"], c["lens"], c["q_start"], n_tokens=-1)):
        with pytest.raises(ValueError):
            bad()
    cache.check()
