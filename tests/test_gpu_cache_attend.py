"""grand_cache_attend and grand_cache_append against the definitions in 64
bits: types, head layouts, page sizes and orders, chunk and cache lengths
from nothing to several splits, windows, hidden tokens that hold anything,
weights, streams, graphs and offsets above 32 bits."""
import math

import numpy as np
import pytest

from cache_ref import attend_ref
from parity import say

pytestmark = pytest.mark.gpu


def make(dtype="bf16", hq=4, hk=2, dim=64, page=16, layout="token", qs=(3,), ks=(40,), seed=0, spare_pages=3, max_pages=None,
         scale_q=2.0, poison=True):
    """A cache with random pages; slots that hold no token hold NaN."""
    import torch

    g = torch.Generator().manual_seed(seed)
    td = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    n = [-(-k // page) for k in ks]
    pages = sum(n) + spare_pages
    order = torch.randperm(pages, generator=g)[:sum(n)].to(torch.int32)
    width = max(n + [1]) if max_pages is None else max_pages
    table = torch.full((len(ks), width), -1, dtype=torch.int32)
    at = 0
    k_pages = torch.full((pages, page, hk, dim), math.nan if poison else 0.0, dtype=td)
    v_pages = k_pages.clone()
    keys, vals = [], []
    for b, m in enumerate(n):
        table[b, :m] = order[at:at + m]
        at += m
        k = torch.randn(ks[b], hk, dim, generator=g).to(td)
        v = torch.randn(ks[b], hk, dim, generator=g).to(td)
        pos = torch.arange(ks[b])
        k_pages[table[b, pos // page].long(), pos % page] = k
        v_pages[table[b, pos // page].long(), pos % page] = v
        keys.append(k)
        vals.append(v)
    q = (torch.randn(sum(qs), hq, dim, generator=g) * scale_q).to(td)

    def up(x):
        if layout == "head":
            return x.cuda().transpose(1, 2).contiguous().transpose(1, 2)
        return x.cuda()

    starts = np.concatenate([[0], np.cumsum(qs)]).astype(np.int32)
    return dict(dtype=dtype, hq=hq, hk=hk, dim=dim, page=page, qs=qs, ks=ks, keys=keys, vals=vals, q=q, starts=starts,
                table=table.cuda(), k_pages=up(k_pages), v_pages=up(v_pages), q_start=torch.from_numpy(starts).cuda(),
                lens=torch.tensor(ks, dtype=torch.int32).cuda())


def cache_for(c, **kw):
    import torch

    from paper_2608_21163_amd import Cache
    return Cache(c["dtype"], c["hq"], c["hk"], c["dim"], c["page"], stream=torch.cuda.current_stream().cuda_stream, **kw)


def seqs_for(cache, c, max_q=None, max_k=None):
    return cache.sequences(c["table"], c["lens"], c["q_start"], max_q=max(c["qs"]) if max_q is None else max_q,
                           max_k=max(c["ks"]) if max_k is None else max_k)


def compare(c, out, lse, causal=True, window=0, scale=None, weights=None, before=None):
    scale = c["dim"] ** -0.5 if scale is None else scale
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, (ql, kl) in enumerate(zip(c["qs"], c["ks"])):
        r0 = int(c["starts"][b])
        ro, rz, rw, bound, z_err, w_err = attend_ref(c["q"][r0:r0 + ql].double().numpy(), c["keys"][b].double().numpy(),
                                                     c["vals"][b].double().numpy(), kl - ql, scale, causal, window)
        o, z = out[r0:r0 + ql], lse[r0:r0 + ql]
        empty = np.isneginf(rz)
        assert np.array_equal(np.isneginf(z), empty), f"sequence {b}: rows that see nothing"
        assert not o[empty].any()
        err, lim = np.abs(o - ro), bound(c["dtype"])
        assert (err <= lim).all(), f"sequence {b}: out off by {err.max()} (bound there {lim.flat[err.argmax()]})"
        zerr = np.abs(np.where(empty, 0, z) - np.where(empty, 0, rz))
        assert (zerr <= z_err + 1e-30).all(), f"sequence {b}: lse off by {zerr.max()} (bound {z_err.flat[zerr.argmax()]})"
        if weights is not None:
            old, new = before[b].double().cpu().numpy(), weights[b].double().cpu().numpy()
            werr = np.abs(new[:, :kl] - old[:, :kl] - rw)
            lim = w_err + 2.0 ** -23 * (np.abs(old[:, :kl]) + rw) + 1e-7 * 0
            assert (werr <= lim + 1e-30).all(), f"sequence {b}: weights off by {werr.max()}"
            assert np.array_equal(new[:, kl:], old[:, kl:]), "entries past the length changed"


def run(c, max_q=None, max_k=None, **kw):
    cache = cache_for(c)
    out = cache.attend(seqs_for(cache, c, max_q, max_k), c["q"].cuda(), c["k_pages"], c["v_pages"], **kw)
    cache.check()
    cache.close()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("hq,hk,dim,page", [(4, 2, 64, 16), (8, 8, 128, 1), (14, 2, 80, 8), (5, 1, 256, 64), (3, 3, 8, 2),
                                            (6, 2, 192, 32), (4, 4, 104, 128), (40, 1, 64, 16), (2, 1, 96, 1024)])
def test_heads_and_layouts(dtype, layout, hq, hk, dim, page):
    say(f"[cache heads] {dtype} {layout} {hq}/{hk} x {dim}, pages of {page}")
    c = make(dtype, hq, hk, dim, page, layout, qs=(3, 1, 9), ks=(70, 33, 9), seed=hq * dim)
    compare(c, *run(c))


LENGTHS = {
    "one_token": ((1,), (1,)),
    "single_tokens": ((1, 1, 1, 1, 1), (1, 31, 32, 33, 129)),
    "nothing_cached": ((2, 1, 3), (0, 0, 5)),
    "no_new_tokens": ((0, 4, 0, 1), (7, 4, 0, 200)),
    "chunk_longer_than_cache": ((5, 40, 3), (2, 20, 3)),
    "whole_prompts": ((64, 65, 127, 1), (64, 65, 127, 1)),
    "tile_edges": ((63, 64, 65, 128), (64, 128, 129, 191)),
    "long_ragged": ((1, 7, 2, 8), (2900, 700, 3, 1500)),
    "long_chunks": ((130, 40, 1), (1300, 900, 640)),
}


@pytest.mark.parametrize("name", LENGTHS)
@pytest.mark.parametrize("dtype,hq,hk,dim", [("bf16", 4, 2, 64), ("f16", 6, 1, 128)])
def test_lengths(name, dtype, hq, hk, dim):
    say(f"[cache lengths] {name} {dtype} {hq}/{hk} x {dim}")
    qs, ks = LENGTHS[name]
    c = make(dtype, hq, hk, dim, 16, qs=qs, ks=ks, seed=len(name))
    compare(c, *run(c))


@pytest.mark.parametrize("dim", [72, 96, 136, 192])
def test_chunks_of_rows_that_are_no_power_of_two(dim):
    import torch

    say(f"[cache chunks] {dim}")
    c = make("bf16", 6, 2, dim, 4, qs=(50, 7, 1), ks=(333, 130, 64), seed=dim)
    before = torch.rand(3, 2, 340, device="cuda")
    after = before.clone()
    out, lse, w = run(c, weights=after)
    compare(c, out, lse, weights=after, before=before)
    compare(c, *run(c, window=40), window=40)


def test_bounds_may_be_loose():
    """max_q and max_k are upper bounds: far larger ones change nothing but
    the order of sums."""
    c = make(qs=(1, 2), ks=(100, 17), max_pages=400)
    compare(c, *run(c, max_q=3, max_k=6400))
    compare(c, *run(c, max_q=500, max_k=6400))


@pytest.mark.parametrize("window", [1, 7, 32, 33, 100, 100000])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("qs,ks", [((1, 1), (300, 40)), ((50, 33), (300, 33)), ((3, 5), (2, 700))])
def test_windows(window, causal, qs, ks):
    say(f"[cache windows] {window} causal {causal} {qs} {ks}")
    c = make(qs=qs, ks=ks, seed=window)
    compare(c, *run(c, window=window, causal=causal), causal=causal, window=window)


@pytest.mark.parametrize("page", [1, 8, 16])
@pytest.mark.parametrize("qs,ks", [((1, 1), (301, 90)), ((3,), (777,)), ((50, 33), (300, 95))])
def test_pages_behind_the_window_may_be_gone(page, qs, ks):
    """Every page that the window has left is freed: no results change and
    nothing is reported; one page further is."""
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ID

    window = 37
    c = make(qs=qs, ks=ks, page=page)
    want = run(c, window=window)
    w = torch.zeros(len(ks), c["hk"], max(ks), device="cuda")
    cache = cache_for(c)
    for b, (ql, kl) in enumerate(zip(qs, ks)):
        c["table"][b, :max(0, kl - ql - window + 1) // page] = -1
    s = seqs_for(cache, c)
    q = c["q"].cuda()
    got = cache.attend(s, q, c["k_pages"], c["v_pages"], window=window)
    with_weights = cache.attend(s, q, c["k_pages"], c["v_pages"], window=window, weights=w)
    cache.check()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(with_weights, want))
    c["table"][0, max(0, ks[0] - qs[0] - window + 1) // page] = -1
    cache.attend(s, q, c["k_pages"], c["v_pages"], window=window)
    with pytest.raises(GrandError) as e:
        cache.check()
    assert e.value.code == E_ID


def test_not_causal():
    c = make("f16", qs=(5, 60), ks=(5, 200))
    compare(c, *run(c, causal=False), causal=False)


@pytest.mark.parametrize("scale", [1e-3, 1.0, 37.5])
def test_scales(scale):
    c = make("f16", qs=(4, 40), ks=(50, 90), scale_q=0.5)
    compare(c, *run(c, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("qs,ks,window", [((4,), (40,), 0), ((70,), (150,), 0), ((3,), (90,), 8), ((60,), (120,), 16)])
def test_hidden_tokens_hold_anything(dtype, qs, ks, window):
    """Keys and values of hidden tokens are infinite or NaN: rows that do
    not see them are as without them, rows that do are not finite."""
    import torch

    say(f"[cache hidden] {dtype} {qs} {ks} window {window}")
    c = make(dtype, qs=qs, ks=ks, seed=5)
    clean = run(c, window=window)
    bad = [(ks[0] - 1, math.nan), (ks[0] - 2, math.inf)] + ([(ks[0] - qs[0] - window, -math.inf)] if window else [])
    vals = c["v_pages"].clone()
    keys = c["k_pages"].clone()
    for pos, x in bad:
        page = int(c["table"][0, pos // c["page"]])
        vals[page, pos % c["page"]] = x
    out, lse = run(dict(c, v_pages=vals), window=window)
    rows = torch.arange(qs[0]) + ks[0] - qs[0]
    sees = torch.zeros(qs[0], dtype=torch.bool)
    for pos, _ in bad:
        sees |= (rows >= pos) & ((rows - pos < window) if window else (rows >= 0))
    assert torch.equal(lse, clean[1])
    assert torch.equal(out[~sees.cuda()], clean[0][~sees.cuda()])
    assert not torch.isfinite(out[sees.cuda()]).any()
    for pos, x in bad:
        page = int(c["table"][0, pos // c["page"]])
        keys[page, pos % c["page"]] = x
    out, lse = run(dict(c, k_pages=keys), window=window)
    assert torch.equal(out[~sees.cuda()], clean[0][~sees.cuda()]) and torch.equal(lse[~sees.cuda()], clean[1][~sees.cuda()])


def test_infinite_values_seen():
    """An infinite value of a seen token gives an infinite result, of both
    signs NaN."""
    import torch

    c = make(qs=(2,), ks=(37,), seed=2)
    t = c["table"][0]
    for pos, d, x in ((36, 0, math.inf), (35, 1, -math.inf), (35, 2, math.inf), (36, 2, -math.inf), (3, 3, math.inf)):
        c["v_pages"][int(t[pos // 16]), pos % 16, :, d] = x
    out, _ = run(c)
    o = out[:, :, :4].float().cpu()
    assert torch.isfinite(o[0, :, 0]).all() and (o[1, :, 0] == math.inf).all()
    assert (o[:, :, 1] == -math.inf).all()
    assert (o[0, :, 2] == math.inf).all() and torch.isnan(o[1, :, 2]).all()
    assert (o[:, :, 3] == math.inf).all()


def test_strided_rows_and_tables():
    """q and out are parts of wider rows, the table is part of a wider one."""
    import torch

    c = make("f16", 4, 2, 64, qs=(3, 20), ks=(30, 80), seed=9)
    wide = torch.full((23, 12, 64), 7.0, dtype=torch.float16, device="cuda")
    wide[:, 2:6] = c["q"].cuda()
    table = torch.full((2, 11), -1, dtype=torch.int32, device="cuda")
    table[:, :c["table"].shape[1]] = c["table"]
    target = torch.full((23, 9, 64), 5.0, dtype=torch.float16, device="cuda")
    cache = cache_for(c)
    s = cache.sequences(table[:, :c["table"].shape[1]], c["lens"], c["q_start"], max_q=20, max_k=80)
    out, lse = cache.attend(s, wide[:, 2:6], c["k_pages"], c["v_pages"], out=target[:, 4:8])
    cache.check()
    compare(c, out, lse)
    assert (target[:, :4] == 5).all() and (target[:, 8:] == 5).all()


@pytest.mark.parametrize("qs,ks,window", [((1, 1, 1), (1, 90, 1400), 0), ((3, 1), (200, 65), 0), ((40, 0, 70), (300, 9, 70), 0),
                                          ((2, 50), (100, 50), 20), ((1, 1), (500, 60), 33), ((4, 9), (2, 3), 0)])
@pytest.mark.parametrize("dtype,hq,hk,dim", [("bf16", 4, 2, 64), ("f16", 8, 8, 128), ("bf16", 5, 1, 256)])
def test_weights(qs, ks, window, dtype, hq, hk, dim):
    import torch

    say(f"[cache weights] {qs} {ks} window {window} {dtype} {hq}/{hk} x {dim}")
    c = make(dtype, hq, hk, dim, qs=qs, ks=ks, seed=sum(ks))
    before = torch.rand(len(ks), hk, max(ks) + 5, device="cuda")
    after = before.clone()
    out, lse, w = run(c, window=window, weights=after)
    assert w is after
    compare(c, out, lse, window=window, weights=after, before=before)
    other = before.clone()
    out2, lse2, w2 = run(c, window=window, weights=before, weights_out=other)
    assert w2 is other and torch.equal(other, after) and torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("qs,ks", [((5, 0, 2), (40, 0, 700)), ((60, 3), (300, 0)), ((300,), (900,))])
def test_weights_without_causality(window, qs, ks):
    import torch

    say(f"[cache weights] not causal, window {window} {qs} {ks}")
    c = make("f16", 8, 1, 64, qs=qs, ks=ks, seed=window)
    before = torch.rand(len(ks), 1, max(ks), device="cuda")
    after = before.clone()
    out, lse, w = run(c, window=window, causal=False, weights=after)
    compare(c, out, lse, causal=False, window=window, weights=after, before=before)


@pytest.mark.parametrize("qs,ks,window", [((4,), (90,), 0), ((70,), (300,), 0), ((3,), (90,), 8), ((60,), (200,), 16)])
def test_weights_of_hidden_tokens_that_hold_anything(qs, ks, window):
    """Keys of tokens that some rows do not see are infinite or NaN: the
    weights that those rows give are as without them."""
    import torch

    say(f"[cache weights] hidden {qs} {ks} window {window}")
    c = make("bf16", 4, 2, 64, qs=qs, ks=ks, seed=8)
    zero = torch.zeros(1, 2, ks[0], device="cuda")
    only = dict(c, lens=c["lens"] - 1, ks=(ks[0] - 1,), qs=(qs[0] - 1,), q=c["q"][:qs[0] - 1],
                q_start=torch.tensor([0, qs[0] - 1], dtype=torch.int32, device="cuda"))
    want = run(only, window=window, weights=zero.clone())[2]       # the chunk without its last token
    keys = c["k_pages"].clone()
    for pos, x in [(ks[0] - 1, math.nan)] + ([(ks[0] - qs[0] - window, math.inf)] if window else []):
        keys[int(c["table"][0, pos // 16]), pos % 16] = x
    got = run(dict(only, k_pages=keys), window=window, weights=zero.clone())[2]
    assert torch.equal(got, want)
    # the last token's own row is the only one that sees its key
    whole = run(dict(c, k_pages=keys), window=window, weights=zero.clone())[2]
    first = max(0, ks[0] - window) if window else 0
    assert torch.isnan(whole[0, :, first:]).all()
    assert torch.allclose(whole[0, :, :first], want[0, :, :first], rtol=1e-6, atol=0)


def test_weights_sum_to_rows():
    """Every row that sees anything hands out a weight of one."""
    import torch

    c = make(qs=(30, 2), ks=(250, 77))
    w = torch.zeros(2, 2, 250, device="cuda")
    run(c, weights=w)
    total = w.double().sum(2).cpu()
    assert torch.allclose(total, torch.tensor([[60.0, 60.0], [4.0, 4.0]], dtype=torch.float64), rtol=1e-5, atol=0)


@pytest.mark.parametrize("qs,ks", [((1, 1), (300, 40)), ((3, 9), (2500, 31)), ((100, 33), (150, 33)), ((200,), (3000,))])
def test_results_in_place_of_the_queries(qs, ks):
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ARG

    c = make(qs=qs, ks=ks)
    want = run(c)
    cache = cache_for(c)
    s, q = seqs_for(cache, c), c["q"].cuda()
    got = cache.attend(s, q, c["k_pages"], c["v_pages"], out=q)
    assert torch.equal(q, want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(GrandError) as e:
        cache.attend(s, q, c["k_pages"], c["v_pages"], out=q, weights=torch.zeros(len(ks), 2, max(ks), device="cuda"))
    assert e.value.code == E_ARG and "out is q" in str(e.value)


def test_repeated_calls_agree_bit_by_bit():
    import torch

    for qs, ks in (((1, 1), (3000, 900)), ((100,), (1500,))):
        c = make(qs=qs, ks=ks)
        w = torch.zeros(len(ks), 2, max(ks), device="cuda")
        first = [x.clone() for x in run(c, weights=w, weights_out=torch.zeros_like(w))]
        for _ in range(3):
            again = run(c, weights=w, weights_out=torch.zeros_like(w))
            assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_another_stream():
    import torch

    c = make(qs=(1, 1), ks=(2500, 300))
    want = run(c)
    side = torch.cuda.Stream()
    cache = cache_for(c)
    s = seqs_for(cache, c)
    q = c["q"].cuda()
    torch.cuda.synchronize()
    cache.set_stream(side.cuda_stream)
    with torch.cuda.stream(side):
        out, lse = cache.attend(s, q, c["k_pages"], c["v_pages"])
    side.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_results_belong_to_the_caches_stream():
    """Memory that the current stream's program has given back is not used
    for results on another stream, where nothing orders the two."""
    import torch

    c = make(qs=(1, 1), ks=(2500, 300))
    want = run(c)
    side = torch.cuda.Stream()
    cache = cache_for(c)
    s, q = seqs_for(cache, c), c["q"].cuda()
    torch.cuda.synchronize()
    cache.set_stream(side.cuda_stream)
    back = [torch.empty_like(want[0]), torch.empty_like(want[1])]
    gone = [x.data_ptr() for x in back]
    del back
    out, lse = cache.attend(s, q, c["k_pages"], c["v_pages"])
    side.synchronize()
    assert out.data_ptr() not in gone and lse.data_ptr() not in gone
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_graph_replays():
    """A captured step gives the eager results on every replay, with other
    work between them and other contents of its inputs."""
    import torch

    c = make(qs=(1, 1, 1), ks=(1800, 40, 333))
    stream = torch.cuda.Stream()
    cache = cache_for(c)
    cache.set_stream(stream.cuda_stream)
    s = seqs_for(cache, c)
    q = c["q"].cuda()
    w = torch.zeros(3, 2, 1800, device="cuda")
    wo = torch.zeros_like(w)
    out, lse = torch.zeros_like(q), torch.zeros(3, 4, device="cuda")
    torch.cuda.synchronize()

    def step():
        cache.attend(s, q, c["k_pages"], c["v_pages"], weights=w, weights_out=wo, out=out, lse=lse)

    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for i in range(4):
        q.copy_((torch.randn(q.shape, generator=torch.Generator().manual_seed(i)) * 2).to(q.dtype))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, wo)]
        out.zero_(), lse.zero_(), wo.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            step()
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, wo)))
    del graph
    cache.close()


def test_capture_cannot_grow_the_workspace():
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_CAPACITY

    c = make(qs=(1,), ks=(3000,))
    stream = torch.cuda.Stream()
    cache = cache_for(c)
    cache.set_stream(stream.cuda_stream)
    s = seqs_for(cache, c)
    q = c["q"].cuda()
    out, lse = torch.zeros_like(q), torch.zeros(1, 4, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        with pytest.raises(GrandError) as e:
            cache.attend(s, q, c["k_pages"], c["v_pages"], out=out, lse=lse)
        out.zero_()
    assert e.value.code == E_CAPACITY
    del graph
    with torch.cuda.stream(stream):
        cache.attend(s, q, c["k_pages"], c["v_pages"], out=out, lse=lse)
    stream.synchronize()
    compare(c, out, lse)
    cache.close()


def test_graphs_outlive_a_larger_workspace():
    """A graph's workspace is not given back when a later call needs more."""
    import torch

    c, big = make(qs=(1,), ks=(1800,)), make(qs=(1, 1, 1, 1), ks=(9000,) * 4, seed=1)
    stream = torch.cuda.Stream()
    cache = cache_for(c)
    cache.set_stream(stream.cuda_stream)
    s, q = seqs_for(cache, c), c["q"].cuda()
    w = torch.zeros(1, 2, 1800, device="cuda")
    wo = torch.zeros_like(w)
    out, lse = torch.zeros_like(q), torch.zeros(1, 4, device="cuda")
    torch.cuda.synchronize()

    def step():
        cache.attend(s, q, c["k_pages"], c["v_pages"], weights=w, weights_out=wo, out=out, lse=lse)

    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    want = [x.clone() for x in (out, lse, wo)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    sb, qb, wb = seqs_for(cache, big), big["q"].cuda(), torch.zeros(4, 2, 9000, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(stream):
            got = cache.attend(sb, qb, big["k_pages"], big["v_pages"], weights=wb, weights_out=torch.zeros_like(wb))
        stream.synchronize()
        compare(big, got[0], got[1], weights=got[2], before=wb)
        out.zero_(), lse.zero_(), wo.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, lse, wo), want))
    del graph
    cache.close()


def test_offsets_above_32_bits():
    """Pages far beyond 2^32 bytes of a pool."""
    import torch

    from paper_2608_21163_amd import Cache

    page, hk, dim, n = 16, 2, 64, 1_200_000   # 4.9 GB each of keys and values
    k_pages = torch.empty(n, page, hk, dim, dtype=torch.bfloat16, device="cuda")
    v_pages = torch.empty_like(k_pages)
    c = make(qs=(2, 33), ks=(40, 50), seed=4)
    table = torch.full_like(c["table"], -1)
    for b, kl in enumerate(c["ks"]):
        for p in range(-(-kl // page)):
            to = n - 1 - 7 * p - b
            table[b, p] = to
            k_pages[to] = c["k_pages"][int(c["table"][b, p])]
            v_pages[to] = c["v_pages"][int(c["table"][b, p])]
    cache = Cache("bf16", 4, 2, dim, page, stream=torch.cuda.current_stream().cuda_stream)
    s = cache.sequences(table, c["lens"], c["q_start"], max_q=33, max_k=50)
    w = torch.zeros(2, 2, 50, device="cuda")
    out, lse, w = cache.attend(s, c["q"].cuda(), k_pages, v_pages, weights=w)
    cache.check()
    compare(c, out, lse, weights=w, before=torch.zeros(2, 2, 50))
    new = torch.randn(35, hk, dim, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    cache.append(s, new, new * 2, k_pages, v_pages)
    cache.check()
    assert torch.equal(k_pages[n - 1 - 14, 8 - 2:8], new[:2]) and torch.equal(v_pages[n - 1 - 14, 6:8], new[:2] * 2)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("page,dim,hk,qs,ks", [(16, 64, 2, (1, 1), (1, 40)), (1, 104, 3, (5, 0, 2), (9, 4, 2)), (64, 256, 1, (70,), (100,)),
                                               (8, 128, 8, (33, 17), (33, 100))])
def test_append(dtype, layout, page, dim, hk, qs, ks):
    import torch

    say(f"[cache append] {dtype} {layout} {page} {dim} {hk} {qs} {ks}")
    c = make(dtype, hk, hk, dim, page, layout, qs=qs, ks=ks, poison=False)
    want_k, want_v = c["k_pages"].clone(), c["v_pages"].clone()
    wide = torch.randn(sum(qs), 3 * hk, dim, device="cuda").to(c["q"].dtype)   # new keys and values inside wider rows
    k, v = wide[:, hk:2 * hk], wide[:, 2 * hk:]
    for b, (ql, kl) in enumerate(zip(qs, ks)):
        for i in range(ql):
            pos = kl - ql + i
            at = int(c["table"][b, pos // page]), pos % page
            want_k[at], want_v[at] = k[int(c["starts"][b]) + i], v[int(c["starts"][b]) + i]
    cache = cache_for(c)
    cache.append(seqs_for(cache, c), k, v, c["k_pages"], c["v_pages"])
    cache.check()
    assert torch.equal(c["k_pages"], want_k) and torch.equal(c["v_pages"], want_v)


def test_without_starts_every_sequence_has_one_new_token():
    import torch

    c = make(qs=(1, 1, 1), ks=(5, 90, 33))
    cache = cache_for(c)
    s = cache.sequences(c["table"], c["lens"], max_k=90)
    out, lse = cache.attend(s, c["q"].cuda(), c["k_pages"], c["v_pages"])
    compare(c, out, lse)
    s = cache.sequences(c["table"], c["lens"])           # max_k from the table's width
    out, lse = cache.attend(s, c["q"].cuda(), c["k_pages"], c["v_pages"])
    compare(c, out, lse)
    k = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(s, k, k, c["k_pages"], c["v_pages"])
    cache.check()
    assert (c["k_pages"][int(c["table"][1, 89 // 16]), 89 % 16] == 1).all()


def test_tables_of_no_pages():
    """Nothing cached at all: a table without columns."""
    import torch

    from paper_2608_21163_amd import Cache

    cache = Cache("bf16", 4, 2, 64, 16, stream=torch.cuda.current_stream().cuda_stream)
    pages = torch.zeros(1, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
    for n in (1, 20):
        s = cache.sequences(torch.zeros(2, 0, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"),
                            torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"), max_q=n)
        q = torch.ones(2 * n, 4, 64, dtype=torch.bfloat16, device="cuda")
        out, lse = cache.attend(s, q, pages, pages)
        cache.check()
        assert not out.any() and torch.isneginf(lse).all()
    table, w, lens, freed, n_freed = cache.evict(s, torch.ones(2, 2, 3, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert table.shape == (2, 0) and not w.any() and not lens.any() and not n_freed.any()
    cache.check()


def test_what_kernels_report():
    """Values in device memory that are out of range: nothing outside the
    buffers is touched, other sequences keep their results, check() says
    what was wrong, once."""
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ARG, E_ID

    c = make(qs=(1, 1), ks=(40, 50))
    want = run(c)
    cache = cache_for(c)
    q = c["q"].cuda()

    def attempt(code, **kw):
        d = dict(c, **kw)
        out, lse = cache.attend(cache.sequences(d["table"], d["lens"], d["q_start"], max_q=1, max_k=50), q, c["k_pages"], c["v_pages"])
        with pytest.raises(GrandError) as e:
            cache.check()
        assert e.value.code == code and "sequence 1" in str(e.value)
        assert torch.equal(out[0], want[0][0]) and torch.equal(lse[0], want[1][0])
        cache.check()

    table = c["table"].clone()
    table[1, 2] = c["k_pages"].shape[0]
    attempt(E_ID, table=table)
    attempt(E_ID, table=torch.where(torch.arange(2, device="cuda")[:, None] == 1, torch.full_like(table, -1), c["table"]))
    attempt(E_ARG, lens=torch.tensor([40, 51], dtype=torch.int32, device="cuda"))
    attempt(E_ARG, q_start=torch.tensor([0, 1, 9], dtype=torch.int32, device="cuda"))
    k = torch.ones(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    before = c["k_pages"].clone()
    d = cache.sequences(table, torch.tensor([40, 48], dtype=torch.int32, device="cuda"), c["q_start"], max_q=1, max_k=50)
    cache.append(d, k, k, c["k_pages"], c["v_pages"])
    with pytest.raises(GrandError):
        cache.check()
    at = int(c["table"][0, 2]), 7
    before[at] = 1
    assert torch.equal(torch.nan_to_num(c["k_pages"]), torch.nan_to_num(before))


def test_refusals():
    import torch

    from paper_2608_21163_amd import Cache, GrandError
    from paper_2608_21163_amd.grand import E_ARG

    c = make(qs=(1, 2), ks=(20, 30))
    cache = cache_for(c)
    q, kp, vp = c["q"].cuda(), c["k_pages"], c["v_pages"]
    s = seqs_for(cache, c)
    good = cache.attend(s, q, kp, vp)

    def refused(text, *a, **kw):
        with pytest.raises(GrandError) as e:
            cache.attend(*a, **kw)
        assert e.value.code == E_ARG and text in str(e.value)

    refused("scale", s, q, kp, vp, scale=0.0)
    refused("scale", s, q, kp, vp, scale=float("nan"))
    refused("scale", s, q, kp, vp, scale=float("inf"))
    refused("max_k", cache.sequences(c["table"], c["lens"], c["q_start"], max_q=2, max_k=33), q, kp, vp)
    flat = torch.zeros(3 * 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")
    refused("aligned", s, flat[4:].view(3, 4, 64), kp, vp)
    refused("strides", s, torch.zeros(3, 4, 68, dtype=torch.bfloat16, device="cuda")[:, :, :64], kp, vp)
    refused("overlap", s, q, kp, vp, out=torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda").expand(3, 4, 64))
    refused("overlap", s, q, kp, vp, weights=torch.zeros(1, 2, 32, device="cuda").expand(2, 2, 32))
    short = seqs_for(cache, c)
    short.c.n_seq = 1 << 15            # lens, table and starts are far shorter (beyond any allocator's rounding)
    short.c.table_stride = 1 << 16
    refused("shorter", short, q, kp, vp)
    host = seqs_for(cache, c)
    lens = np.array([20, 30], np.uint32)
    host.c.lens = lens.ctypes.data
    refused("not memory of GPU", host, q, kp, vp)
    for bad in (lambda: cache.attend(s, q.float(), kp, vp), lambda: cache.attend(s, q[:, :2], kp, vp),
                lambda: cache.attend(s, q, kp, vp[:, :8]), lambda: cache.attend(s, q, kp, vp.transpose(1, 2).contiguous().transpose(1, 2)),
                lambda: cache.attend(s, c["q"], kp, vp), lambda: cache.attend(s, q, kp, vp, weights_out=torch.zeros(2, 2, 32, device="cuda")),
                lambda: cache.attend(s, q, kp, vp, weights=torch.zeros(2, 2, 29, device="cuda")),
                lambda: cache.sequences(c["table"].long(), c["lens"]), lambda: cache.sequences(c["table"][:1], c["lens"]),
                lambda: cache.append(s, q, q, kp, vp), lambda: Cache("f32")):
        with pytest.raises(ValueError):
            bad()
    for kw in (dict(q_heads=5, kv_heads=2), dict(head_dim=12), dict(head_dim=264), dict(page_size=3), dict(page_size=2048), dict(kv_heads=0)):
        with pytest.raises(GrandError) as e:
            Cache(**kw)
        assert e.value.code == E_ARG
    again = cache.attend(s, q, kp, vp)   # the handle is as it was
    assert torch.equal(good[0], again[0])
    cache.check()
