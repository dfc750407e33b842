"""The operators of caches held in 4 bits, and attention with first tokens
that stay visible, against the definitions in 64 bits: types, head layouts,
page sizes and orders, lengths from nothing to several splits, windows, blocks
of NaN, what unused slots hold, offsets above 32 bits, weights, lists."""
import math

import numpy as np
import pytest

from cache_ref import INVALID, ids_ref
from packed_ref import EXPONENTS, attend_ref, pack, unpack, visible
from parity import say
from test_gpu_cache_attend import LENGTHS, cache_for, make, seqs_for

pytestmark = pytest.mark.gpu


def packed(c, layout="head", seed=0):
    """The cache of make() in 4 bits: its pools, and the values that they
    stand for in place of the keys and values.  Unused slots hold any codes
    and scales."""
    import torch

    from paper_2608_21163_amd import Packed

    r = np.random.default_rng(seed)
    pages, blocks = c["k_pages"].shape[0], -(-c["dim"] // 32)
    res = dict(c)
    for pool, rows in (("k_pages", "keys"), ("v_pages", "vals")):
        codes = r.integers(0, 256, (pages, c["page"], c["hk"], 16 * blocks), dtype=np.uint8)
        scales = r.integers(0, 256, (pages, c["page"], c["hk"], blocks), dtype=np.uint8)
        values = []
        for b, x in enumerate(c[rows]):
            pc, ps = pack(x.double().numpy(), c["dtype"])
            pos = np.arange(len(x))
            table = c["table"][b].cpu().numpy()
            codes[table[pos // c["page"]], pos % c["page"]], scales[table[pos // c["page"]], pos % c["page"]] = pc, ps
            values.append(torch.from_numpy(unpack(pc, ps, c["dim"], c["dtype"])))
        res[rows], res[pool] = values, as_packed(codes, scales, layout)
        res[pool + "_np"] = codes, scales
    return res


def as_packed(codes, scales, layout):
    """token: slots of all heads; head: heads outermost in a page; rows: a row's
    scales behind its codes, in one buffer."""
    import torch

    from paper_2608_21163_amd import Packed

    codes, scales = torch.from_numpy(codes), torch.from_numpy(scales)
    if layout == "rows":
        n, blocks = codes.shape[-1], scales.shape[-1]
        both = torch.zeros(*codes.shape[:3], n + (blocks + 15) // 16 * 16, dtype=torch.uint8)
        both[..., :n], both[..., n:n + blocks] = codes, scales
        both = both.cuda()
        return Packed(both[..., :n], both[..., n:n + blocks])
    if layout == "head":
        return Packed(*(x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (codes, scales)))
    return Packed(codes.cuda(), scales.cuda())


def compare(c, out, lse, causal=True, window=0, sinks=0, scale=None, weights=None, before=None):
    scale = c["dim"] ** -0.5 if scale is None else scale
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, (ql, kl) in enumerate(zip(c["qs"], c["ks"])):
        r0 = int(c["starts"][b])
        ro, rz, rw, bound, z_err, w_err = attend_ref(c["q"][r0:r0 + ql].double().numpy(), c["keys"][b].double().numpy(),
                                                     c["vals"][b].double().numpy(), kl - ql, scale, causal, window, sinks)
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
            lim = w_err + 2.0 ** -23 * (np.abs(old[:, :kl]) + rw)
            assert (werr <= lim + 1e-30).all(), f"sequence {b}: weights off by {werr.max()}"
            assert np.array_equal(new[:, kl:], old[:, kl:]), "entries past the length changed"


def run(c, max_q=None, max_k=None, **kw):
    cache = cache_for(c)
    out = cache.attend(seqs_for(cache, c, max_q, max_k), c["q"].cuda(), c["k_pages"], c["v_pages"], **kw)
    cache.check()
    cache.close()
    return out


def weighted(c, **kw):
    import torch

    before = torch.rand(len(c["ks"]), c["hk"], max(max(c["ks"]), 1) + 3, device="cuda")
    after = before.clone()
    out, lse, _ = run(c, weights=after, **kw)
    compare(c, out, lse, weights=after, before=before, **kw)


# ------------------------------------------------------------ packed pages
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["token", "head", "rows"])
@pytest.mark.parametrize("hq,hk,dim,page", [(4, 2, 64, 16), (8, 8, 128, 1), (14, 2, 80, 8), (5, 1, 256, 64), (3, 3, 8, 2),
                                            (6, 2, 192, 32), (4, 4, 104, 128), (40, 1, 64, 16), (2, 1, 96, 1024), (2, 2, 40, 4)])
def test_heads_and_layouts(dtype, layout, hq, hk, dim, page):
    say(f"[packed heads] {dtype} {layout} {hq}/{hk} x {dim}, pages of {page}")
    c = packed(make(dtype, hq, hk, dim, page, qs=(3, 1, 9), ks=(70, 33, 9), seed=hq * dim), layout)
    compare(c, *run(c))


@pytest.mark.parametrize("name", LENGTHS)
@pytest.mark.parametrize("dtype,hq,hk,dim", [("bf16", 4, 2, 64), ("f16", 6, 1, 128)])
def test_lengths(name, dtype, hq, hk, dim):
    say(f"[packed lengths] {name} {dtype} {hq}/{hk} x {dim}")
    qs, ks = LENGTHS[name]
    c = packed(make(dtype, hq, hk, dim, 16, qs=qs, ks=ks, seed=len(name)))
    compare(c, *run(c))


@pytest.mark.parametrize("dim", [72, 96, 136, 192, 256])
def test_chunks_of_other_rows(dim):
    say(f"[packed chunks] {dim}")
    c = packed(make("bf16", 6, 2, dim, 4, qs=(50, 7, 1), ks=(333, 130, 64), seed=dim))
    weighted(c)
    weighted(c, window=40, sinks=3)


@pytest.mark.parametrize("qs,ks,window,sinks", [((1, 1, 1), (1, 90, 1400), 0, 0), ((3, 1), (200, 65), 0, 0), ((40, 0, 70), (300, 9, 70), 0, 0),
                                                ((2, 50), (100, 50), 20, 2), ((1, 1), (500, 60), 33, 40), ((4, 9), (2, 3), 0, 0)])
@pytest.mark.parametrize("dtype,hq,hk,dim", [("bf16", 4, 2, 64), ("f16", 8, 8, 128), ("bf16", 5, 1, 256)])
def test_weights(qs, ks, window, sinks, dtype, hq, hk, dim):
    say(f"[packed weights] {qs} {ks} window {window} {sinks} {dtype} {hq}/{hk} x {dim}")
    c = packed(make(dtype, hq, hk, dim, qs=qs, ks=ks, seed=sum(ks)))
    weighted(c, window=window, sinks=sinks)


def nan_block(c, which, pos, block, head=slice(None)):
    """A block of a token becomes NaN, in one of the ways that count as it."""
    page = int(c["table"][0, pos // c["page"]])
    scales = c[which].scales
    scales[page, pos % c["page"], head, block] = 255 if pos % 2 else EXPONENTS[c["dtype"]][1] + 128


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("qs,ks,window,sinks", [((4,), (40,), 0, 0), ((70,), (150,), 0, 0), ((3,), (90,), 8, 4), ((60,), (190,), 16, 5)])
def test_blocks_of_nan(dtype, dim, qs, ks, window, sinks):
    """Rows that do not see such a token are as without it; of those that do, the
    elements of a value's block, or the whole row of a key's, are NaN."""
    import torch

    say(f"[packed nan] {dtype} {dim} {qs} {ks} window {window} {sinks}")
    c = packed(make(dtype, qs=qs, ks=ks, dim=dim, seed=5))
    clean = run(c, window=window, sinks=sinks)
    bad = [ks[0] - 1, ks[0] - 2] + ([ks[0] - qs[0] - window] if window else [])
    rows = np.arange(qs[0]) + ks[0] - qs[0]
    for pos in bad:
        nan_block(c, "v_pages", pos, 1)
    sees = np.array([visible(p, ks[0], True, window, sinks)[bad].any() for p in rows])
    assert sees.any() and not sees.all()
    sees = torch.from_numpy(sees).cuda()
    out, lse = run(c, window=window, sinks=sinks)
    assert torch.equal(lse, clean[1]) and torch.equal(out[~sees], clean[0][~sees])
    assert torch.isnan(out[sees][..., 32:64]).all() and torch.equal(out[..., :32], clean[0][..., :32]) and torch.equal(out[..., 64:], clean[0][..., 64:])
    for pos in bad:
        nan_block(c, "k_pages", pos, 0)
    out, lse = run(c, window=window, sinks=sinks)
    assert torch.equal(out[~sees], clean[0][~sees]) and torch.equal(lse[~sees], clean[1][~sees]) and torch.isnan(out[sees]).all()
    w = torch.zeros(1, c["hk"], ks[0], device="cuda")
    run(c, window=window, sinks=sinks, weights=w)
    only = np.any([visible(p, ks[0], True, window, sinks) for p in rows[sees.cpu().numpy()]], 0)
    assert torch.isnan(w[0, :, torch.from_numpy(only).cuda()]).all() and torch.isfinite(w[0, :, torch.from_numpy(~only).cuda()]).all()


def test_not_causal_and_scales():
    c = packed(make("f16", qs=(5, 60), ks=(5, 200)))
    compare(c, *run(c, causal=False), causal=False)
    compare(c, *run(c, scale=3.5), scale=3.5)


def test_pages_outside_the_pool_are_reported():
    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ID

    for qs, ks in (((1, 1), (301, 90)), ((70, 3), (301, 90))):
        c = packed(make(qs=qs, ks=ks))
        c["table"][1, 2] = c["k_pages"].codes.shape[0]
        with pytest.raises(GrandError) as e:
            run(c)
        assert e.value.code == E_ID


def test_offsets_above_32_bits():
    """Pages more than 4 GiB apart: tokens lie in the first and the last."""
    import torch

    from paper_2608_21163_amd import Cache, Packed

    pages, hk, dim = 700_000, 8, 128
    codes = torch.zeros(pages, hk, 16, 64, dtype=torch.uint8, device="cuda").transpose(1, 2)
    scales = torch.full((pages, hk, 16, 4), 127, dtype=torch.uint8, device="cuda").transpose(1, 2)
    assert codes.numel() > 5 << 30
    cache = Cache("bf16", 8, hk, dim, 16, stream=torch.cuda.current_stream().cuda_stream)
    g = torch.Generator().manual_seed(1)
    k, v, q = (torch.randn(40, hk, dim, generator=g).bfloat16() for _ in range(3))
    table = torch.tensor([[0, pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([40], dtype=torch.int32, device="cuda")
    s = cache.sequences(table, lens, torch.tensor([0, 40], dtype=torch.int32, device="cuda"), max_q=40, max_k=40)
    both = Packed(codes, scales)
    rows = k.cuda()
    cache.append(s, rows, rows, both, both)
    held = torch.from_numpy(unpack(*pack(k.double().numpy(), "bf16"), dim, "bf16"))
    out, lse = cache.attend(s, q.cuda(), both, both)
    slots = torch.tensor([(pages - 2) * 16 + 7, 3], dtype=torch.int32, device="cuda")
    rk, _ = cache.read(slots, both, both)
    cache.check()
    cache.close()
    assert torch.equal(rk.cpu().double(), held[[39, 3]])
    compare(dict(dtype="bf16", dim=dim, q=q, keys=[held], vals=[held], qs=(40,), ks=(40,), starts=[0]), out, lse)


# ------------------------------------------------------------ append and read
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["token", "head", "rows"])
@pytest.mark.parametrize("hk,dim,page", [(2, 64, 16), (8, 128, 1), (2, 80, 8), (1, 256, 64), (3, 8, 2), (5, 104, 4)])
def test_append_and_read(dtype, layout, hk, dim, page):
    """Codes and scales are the definition's; nothing else in the pools
    changes; reading gives their values."""
    import torch

    say(f"[packed append] {dtype} {layout} {hk} x {dim}, pages of {page}")
    qs, ks = (3, 0, 20, 1), (40, 9, 20, 65)
    c = packed(make(dtype, hk, hk, dim, page, qs=qs, ks=ks, seed=dim), layout, seed=3)
    r = np.random.default_rng(dim)
    rows = []
    for _ in range(2):
        x = r.standard_normal((sum(qs), hk, dim)) * 2.0 ** r.integers(-6, 6, (sum(qs), hk, 1))
        x[0, 0] = 0
        x[1, 0, :4] = [-0.0, 0.25, -0.75, 1.25]
        if dim > 32:
            x[2, -1, 32:] = 0
        rows.append(torch.from_numpy(x).to(c["q"].dtype))
    cache = cache_for(c)
    cache.append(seqs_for(cache, c), rows[0].cuda(), rows[1].cuda(), c["k_pages"], c["v_pages"])
    slots = []
    for b, (ql, kl) in enumerate(zip(qs, ks)):
        for pos in range(kl - ql, kl):
            slots.append(int(c["table"][b, pos // page]) * page + pos % page)
    read = cache.read(torch.tensor(slots + [-1], dtype=torch.int32, device="cuda"), c["k_pages"], c["v_pages"])
    cache.check()
    cache.close()
    for name, x, got in (("k_pages", rows[0], read[0]), ("v_pages", rows[1], read[1])):
        codes, scales = (y.copy() for y in c[name + "_np"])
        pc, ps = pack(x.double().numpy(), dtype)
        for i, s in enumerate(slots):
            codes[s // page, s % page], scales[s // page, s % page] = pc[i], ps[i]
        assert np.array_equal(c[name].codes.cpu().numpy(), codes) and np.array_equal(c[name].scales.cpu().numpy(), scales)
        assert np.array_equal(got[:-1].double().cpu().numpy(), unpack(pc, ps, dim, dtype)) and not got[-1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_number_packs(dtype):
    """Every finite 16-bit number as the largest of a block and beside a
    larger one, and blocks with infinities and NaN."""
    import torch

    from paper_2608_21163_amd import Cache

    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view({"bf16": torch.bfloat16, "f16": torch.float16}[dtype])
    x = torch.cat([x.repeat(2), x.flip(0)])[:3 * 65536]
    step = torch.arange(len(x)) % 31 + 1
    rows = torch.zeros(len(x), 32, dtype=x.dtype)
    rows[:, 0] = x
    rows[65536:, 1] = (x[65536:].float() * (1 + step[65536:] / 8)).to(x.dtype)
    rows = rows.view(-1, 1, 32)
    n = len(rows)
    cache = Cache(dtype, 1, 1, 32, 1024, stream=torch.cuda.current_stream().cuda_stream)
    k, v = cache.packed_pages(n // 1024)
    table = torch.arange(n // 1024, dtype=torch.int32, device="cuda")[None]
    s = cache.sequences(table, torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                        max_q=n, max_k=n)
    cache.append(s, rows.cuda(), rows.cuda(), k, v)
    cache.check()
    codes, scales = pack(rows.double().numpy(), dtype)
    assert np.array_equal(k.scales.reshape(n, 1, 1).cpu().numpy(), scales)
    assert np.array_equal(k.codes.reshape(n, 1, 16).cpu().numpy(), codes) and torch.equal(v.codes, k.codes)
    got, _ = cache.read(torch.arange(n, dtype=torch.int32, device="cuda"), k, v)
    want = unpack(codes, scales, 32, dtype)
    assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    fine = np.isfinite(want).all(-1)[:, 0]
    err = np.abs(want - rows.double().numpy())[fine, 0]
    top = np.abs(rows.double().numpy())[fine, 0].max(-1, keepdims=True)
    # half a step where steps are largest, 2^e with 3.5 * 2^e at most the largest element; fp16 ends at 6 * 2^13
    ordinary = top[:, 0] < 7 * 2.0 ** EXPONENTS[dtype][1]
    assert (err[ordinary] <= np.maximum(top[ordinary] / 3.5, 2.0 ** (EXPONENTS[dtype][0] - 2))).all()
    cache.close()


# ------------------------------------------------------------ listed slots
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["token", "head", "rows"])
@pytest.mark.parametrize("hq,hk,dim,page,n", [(4, 2, 64, 1, 37), (8, 8, 128, 16, 300), (6, 2, 80, 8, 1), (5, 1, 256, 4, 700), (3, 3, 8, 2, 5),
                                              (8, 4, 192, 1, 64)])
@pytest.mark.parametrize("prior", [False, True])
def test_listed_slots(dtype, layout, hq, hk, dim, page, n, prior):
    import torch

    say(f"[packed ids] {dtype} {layout} {hq}/{hk} x {dim} pages of {page}, lists of {n}, prior {prior}")
    c = packed(make(dtype, hq, hk, dim, page, qs=(1,), ks=(600,), seed=n), layout)
    r = np.random.default_rng(n)
    slots = np.array([int(c["table"][0, p // page]) * page + p % page for p in range(600)])
    b = 3
    q = torch.from_numpy(r.standard_normal((b, hq, dim)) * 2).to(c["q"].dtype)
    pick = r.integers(0, 600, (b, hq, n))
    ids = slots[pick].astype(np.uint32)
    ids[r.random(ids.shape) < 0.1] = INVALID
    ids[1, 0] = INVALID
    po = torch.from_numpy(r.standard_normal((b, hq, dim))).to(q.dtype)
    pz = torch.from_numpy(r.standard_normal((b, hq))).float()
    pz[1, 1], pz[1, 0] = -math.inf, -math.inf
    cache = cache_for(c)
    got = cache.attend_ids(q.cuda(), c["k_pages"], c["v_pages"], torch.from_numpy(ids.astype(np.int32)).cuda(),
                           prior=(po.cuda(), pz.cuda()) if prior else None)
    cache.check()
    cache.close()
    total = c["k_pages"].codes.shape[0] * page
    flat = [np.zeros((total, hk, dim)) for _ in range(2)]
    for x, rows in zip(flat, (c["keys"], c["vals"])):
        x[slots] = rows[0].numpy()
    want, z, bound, z_err = ids_ref(q.double().numpy(), *flat, ids, dim ** -0.5, (po.double().numpy(), pz.double().numpy()) if prior else None)
    o, l = got[0].double().cpu().numpy(), got[1].double().cpu().numpy()
    assert (np.abs(o - want) <= bound(dtype)).all()
    empty = np.isneginf(z)
    assert np.array_equal(np.isneginf(l), empty) and empty.any()
    assert (np.abs(np.where(empty, 0, l) - np.where(empty, 0, z)) <= z_err + 1e-30).all()


def ragged(n, most_q, longest, seed, empty=0.2):
    """n sequences, some of no new tokens, some of no tokens at all."""
    r = np.random.default_rng(seed)
    qs = np.where(r.random(n) < empty, 0, r.integers(1, most_q + 1, n))
    ks = np.where(r.random(n) < empty, qs, qs + r.integers(0, longest, n))
    qs[n // 3], qs[-1] = 1, 1
    ks[n // 3], ks[-1] = 1, longest
    return tuple(qs.tolist()), tuple(ks.tolist())


MANY = [(70, 1, 900), (129, 4, 700), (1024, 1, 520), (1025, 1, 520), (3, 2, 20_000), (40, 8, 7000)]


@pytest.mark.parametrize("n,most_q,longest", MANY)
@pytest.mark.parametrize("dtype,hq,hk,dim,window,sinks", [("bf16", 4, 2, 128, 0, 0), ("f16", 4, 1, 64, 0, 0), ("bf16", 2, 2, 64, 300, 40)])
def test_many_sequences(n, most_q, longest, dtype, hq, hk, dim, window, sinks):
    """Few rows of many sequences share the card by their keys: empty and short ones among long ones, and one long one last."""
    say(f"[packed many] {n} of up to {most_q} tokens and {longest} keys, {dtype} {hq}/{hk} x {dim}, window {window} {sinks}")
    qs, ks = ragged(n, most_q, longest, n + most_q)
    c = packed(make(dtype, hq, hk, dim, 16, qs=qs, ks=ks, seed=n))
    weighted(c, window=window, sinks=sinks)
    compare(c, *run(c, max_q=most_q + 1, max_k=c["table"].shape[1] * 16, window=window, sinks=sinks), window=window, sinks=sinks)


def test_one_long_sequence_among_short_ones():
    """... and alone, in one page order after the other."""
    for qs, ks in (((1,) * 64, (3,) * 40 + (12_000,) + (2,) * 23), ((1,), (30_001,)), ((0,) * 63 + (1,), (0,) * 63 + (9000,)),
                   ((0,) * 5, (700,) * 5)):
        c = packed(make("bf16", 8, 2, 128, 16, qs=qs, ks=ks, seed=len(qs)))
        if sum(qs):
            weighted(c)
        else:
            run(c)


@pytest.mark.parametrize("n,longest", [(9, 3000), (70, 900)])
def test_captured_steps_of_changing_lengths(n, longest):
    """Shares follow the lengths of a replay, not those of the capture; two graphs take turns in one workspace."""
    import torch

    from paper_2608_21163_amd import Cache

    stream = torch.cuda.Stream()
    r = np.random.default_rng(n)
    c = packed(make("bf16", 4, 2, 128, 16, qs=(1,) * n, ks=(longest,) * n, seed=n))
    cache = Cache(c["dtype"], c["hq"], c["hk"], c["dim"], c["page"], stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        q, lens = c["q"].cuda(), c["lens"].clone()
        s = cache.sequences(c["table"], lens, max_k=longest)
        weights = torch.zeros(n, 2, longest, device="cuda")
        calls = [lambda: cache.attend(s, q, c["k_pages"], c["v_pages"]),
                 lambda: cache.attend(s, q, c["k_pages"], c["v_pages"], window=700, sinks=20, weights=weights, weights_out=torch.empty_like(weights))]
        for call in calls:
            call()
        stream.synchronize()
        graphs = []
        for call in calls:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                res = call()
            graphs.append((g, res))
        for i in range(8):
            kl = r.integers(0, longest + 1, n)
            kl[r.integers(0, n)] = longest
            lens.copy_(torch.from_numpy(kl.astype(np.int32)))
            weights.copy_(torch.rand(weights.shape))
            for (g, got), call in zip(graphs, calls):
                g.replay()
                got = [x.clone() for x in got]
                want = call()
                seen = torch.arange(longest, device="cuda") < torch.from_numpy(kl).cuda()[:, None, None]
                assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
                assert len(got) < 3 or torch.equal(*(torch.where(seen, x[2], 0.0) for x in (got, want))), i
    cache.check()
    cache.close()


def test_refusals_of_the_binding():
    c = packed(make(qs=(1,), ks=(40,)))
    whole = make(qs=(1,), ks=(40,))
    for kw in (dict(sinks=-1), dict(sinks=1 << 32)):
        with pytest.raises(ValueError):
            run(c, window=4, **kw)
    for k, v in ((c["k_pages"], whole["v_pages"]), (whole["k_pages"], c["v_pages"])):
        with pytest.raises(ValueError):
            run(dict(c, k_pages=k, v_pages=v))


# ------------------------------------------------------------ first tokens
@pytest.mark.parametrize("kind", ["whole", "packed"])
@pytest.mark.parametrize("window,sinks", [(1, 1), (7, 4), (32, 32), (33, 64), (100, 5), (40, 65), (100000, 3), (40, 100000)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("qs,ks", [((1, 1, 1), (700, 40, 3)), ((50, 33, 2), (500, 33, 260)), ((3, 5, 0), (2, 900, 7)), ((300,), (1111,))])
def test_first_tokens(kind, window, sinks, causal, qs, ks):
    say(f"[sinks] {kind} window {window} {sinks} causal {causal} {qs} {ks}")
    c = make(qs=qs, ks=ks, seed=window + sinks)
    c = packed(c) if kind == "packed" else c
    weighted(c, window=window, sinks=sinks, causal=causal)


@pytest.mark.parametrize("dtype,hq,hk,dim,page", [("f16", 12, 12, 64, 1), ("bf16", 4, 1, 192, 8), ("f16", 5, 1, 256, 16), ("bf16", 8, 8, 96, 64),
                                                  ("bf16", 32, 1, 80, 16)])
@pytest.mark.parametrize("kind", ["whole", "packed"])
def test_first_tokens_of_other_heads(kind, dtype, hq, hk, dim, page):
    say(f"[sinks heads] {kind} {dtype} {hq}/{hk} x {dim} pages of {page}")
    for qs, ks in (((1, 1), (1500, 77)), ((80, 2), (600, 400))):
        c = make(dtype, hq, hk, dim, page, qs=qs, ks=ks, seed=dim)
        c = packed(c) if kind == "packed" else c
        weighted(c, window=70, sinks=9)


@pytest.mark.parametrize("kind", ["whole", "packed"])
def test_no_first_tokens_is_the_window(kind):
    """sinks 0, and sinks without a window, change nothing, bit by bit."""
    import torch

    for qs, ks in (((1, 1), (1500, 77)), ((80, 2), (600, 400))):
        c = make(qs=qs, ks=ks)
        c = packed(c) if kind == "packed" else c
        assert all(torch.equal(a, b) for a, b in zip(run(c, sinks=8), run(c)))
        near = run(c, window=64)
        assert all(torch.equal(a, b) for a, b in zip(run(c, window=64, sinks=0), near))
        assert not torch.equal(run(c, window=64, sinks=1)[0], near[0])


@pytest.mark.parametrize("kind", ["whole", "packed"])
@pytest.mark.parametrize("page", [1, 8, 16])
@pytest.mark.parametrize("qs,ks", [((1, 1), (301, 90)), ((3,), (777,)), ((50, 33), (300, 95))])
def test_pages_between_may_be_gone(kind, page, qs, ks):
    """Pages between the first tokens and the window are freed: no results
    change and nothing is reported; a page of the first tokens is."""
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ID

    window, sinks = 37, 5
    c = make(qs=qs, ks=ks, page=page)
    c = packed(c) if kind == "packed" else c
    want = run(c, window=window, sinks=sinks)
    for b, (ql, kl) in enumerate(zip(qs, ks)):
        c["table"][b, -(-sinks // page):max(0, kl - ql - window + 1) // page] = -1
    got = run(c, window=window, sinks=sinks)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    w = torch.zeros(len(ks), c["hk"], max(ks), device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(run(c, window=window, sinks=sinks, weights=w), want))
    c["table"][0, (sinks - 1) // page] = -1
    with pytest.raises(GrandError) as e:
        run(c, window=window, sinks=sinks)
    assert e.value.code == E_ID


@pytest.mark.parametrize("qs,ks", [((3,), (90,)), ((60,), (190,))])
def test_first_tokens_hidden_ones_hold_anything(qs, ks):
    """Between the first tokens and a row's window lie NaN and infinities."""
    import torch

    c = make(qs=qs, ks=ks, seed=5)
    window, sinks = 16, 5
    clean = run(c, window=window, sinks=sinks)
    for pos, x in ((sinks, math.nan), (sinks + 1, math.inf), (ks[0] - qs[0] - window - 1, -math.inf)):
        for pool in ("k_pages", "v_pages"):
            c[pool][int(c["table"][0, pos // 16]), pos % 16] = x
    out, lse = run(c, window=window, sinks=sinks)
    assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
    c["v_pages"][int(c["table"][0, 0]), 4] = math.inf            # a first token: every row sees it
    out, lse = run(c, window=window, sinks=sinks)
    assert (out == math.inf).all() and torch.equal(lse, clean[1])


def test_long_histories_of_first_tokens():
    """Several splits of the first tokens and of the window."""
    for qs, ks in (((1, 1), (9000, 5000)), ((20, 70), (5000, 3001))):
        c = make("f16", 4, 1, 64, 16, qs=qs, ks=ks, seed=1)
        weighted(c, window=2100, sinks=1500)
        weighted(packed(c), window=2100, sinks=1500)


@pytest.mark.parametrize("kind", ["whole", "packed"])
@pytest.mark.parametrize("qs,ks,window,sinks", [((70, 1, 33), (4000, 700, 33), 200, 10), ((40,), (5000,), 64, 300), ((64, 64), (2500, 1000), 1, 257),
                                                ((300,), (3500,), 500, 0), ((40, 40), (1800, 1800), 1700, 3)])
def test_weights_far_from_the_window(kind, qs, ks, window, sinks):
    """Keys that no row of a chunk sees lie between the first tokens and the windows: their weights stay."""
    say(f"[weights] {kind} {qs} {ks} window {window} {sinks}")
    for dtype, hq, hk, dim in (("bf16", 4, 2, 64), ("f16", 5, 1, 128)):
        c = make(dtype, hq, hk, dim, qs=qs, ks=ks, seed=window)
        weighted(packed(c) if kind == "packed" else c, window=window, sinks=sinks)
        weighted(packed(c) if kind == "packed" else c, window=window, sinks=sinks, causal=False)


@pytest.mark.parametrize("n,most_q", [(127, 1), (128, 1), (130, 3)])
def test_first_tokens_of_many_sequences(n, most_q):
    """A workgroup a sequence and head where there are enough of them."""
    qs, ks = ragged(n, most_q, 1500, n)
    for dtype, hq, hk, dim in (("bf16", 4, 2, 64), ("f16", 2, 2, 128)):
        c = make(dtype, hq, hk, dim, qs=qs, ks=ks, seed=n)
        weighted(c, window=600, sinks=30)


@pytest.mark.parametrize("dim,n", [(64, 70), (128, 255), (128, 256), (128, 300), (256, 60)])
def test_many_lists(dim, n):
    """Enough lists for a wave each, in place over an earlier result, some lists empty."""
    import torch

    say(f"[packed ids] 300 x 8 lists of {n}, {dim}")
    c = packed(make("bf16", 8, 2, dim, 16, qs=(1,), ks=(600,), seed=n))
    r = np.random.default_rng(n)
    slots = np.array([int(c["table"][0, p // 16]) * 16 + p % 16 for p in range(600)])
    b = 300
    q = torch.from_numpy(r.standard_normal((b, 8, dim)) * 2).to(c["q"].dtype)
    ids = slots[r.integers(0, 600, (b, 8, n))].astype(np.uint32)
    ids[7], ids[9, 3, 5:], ids[r.random(ids.shape) < 0.05] = INVALID, INVALID, INVALID
    po, pz = torch.from_numpy(r.standard_normal((b, 8, dim))).to(q.dtype), torch.from_numpy(r.standard_normal((b, 8))).float()
    pz[7, 2] = -math.inf
    out, lse = po.cuda(), pz.cuda()
    cache = cache_for(c)
    cache.attend_ids(q.cuda(), c["k_pages"], c["v_pages"], torch.from_numpy(ids.astype(np.int32)).cuda(), prior=(out, lse), out=out, lse=lse)
    cache.check()
    cache.close()
    total = c["k_pages"].codes.shape[0] * 16
    flat = [np.zeros((total, 2, dim)) for _ in range(2)]
    for x, rows in zip(flat, (c["keys"], c["vals"])):
        x[slots] = rows[0].numpy()
    some = [0, 7, 9, 133, 299]
    want, z, bound, z_err = ids_ref(q[some].double().numpy(), *flat, ids[some], dim ** -0.5, (po[some].double().numpy(), pz[some].double().numpy()))
    o, l = out.double().cpu().numpy()[some], lse.double().cpu().numpy()[some]
    assert (np.abs(o - want) <= bound("bf16")).all()
    empty = np.isneginf(z)
    assert np.array_equal(np.isneginf(l), empty) and empty.any()
    assert (np.abs(np.where(empty, 0, l) - np.where(empty, 0, z)) <= z_err + 1e-30).all()
    with_ids = ids.astype(np.int32)
    with_ids[11, 2, 1] = total          # a slot outside the pool: passed over, and reported
    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ID
    cache = cache_for(c)
    cache.attend_ids(q.cuda(), c["k_pages"], c["v_pages"], torch.from_numpy(with_ids).cuda())
    with pytest.raises(GrandError) as e:
        cache.check()
    assert e.value.code == E_ID
    cache.close()


@pytest.mark.parametrize("kind", ["whole", "packed"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (10, 4)])
def test_weights_of_chunks_without_cached_tokens(kind, window, sinks):
    """max_k 0, and chunks of more rows than a tile's: every row sees nothing."""
    import torch

    say(f"[no cached tokens] {kind} window {window} {sinks}")
    c = make("bf16", 8, 2, 64, 16, qs=(40, 70), ks=(0, 0))
    c = packed(c) if kind == "packed" else c
    none = torch.empty(2, 2, 0, device="cuda")
    out, lse, _ = run(c, weights=none, window=window, sinks=sinks)
    assert not out.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("kind", ["whole", "packed"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,sinks", [(300, 0), (300, 270), (40, 600), (1000, 3), (1, 0)])
def test_weights_of_windows_in_long_caches(kind, causal, window, sinks):
    """Tiles of keys that no row sees lie before, between and behind those that have sums,
    with one split of the rows and with several; a sequence is shorter than its window, one than its chunk."""
    say(f"[windowed weights] {kind} causal {causal} window {window} {sinks}")
    for most in (40, 300):                               # rows: one split; three, but for the shorter chunks
        c = make("f16", 4, 2, 64, 8, qs=(most, 20, 7, 35, 0), ks=(2900, 1500, 200, 30, 700), seed=window + most)
        c = packed(c) if kind == "packed" else c
        weighted(c, causal=causal, window=window, sinks=sinks)


def rounded(x, dtype):
    """Values as the 16-bit type holds them, its numbers below the normal range among them."""
    import torch

    if dtype == "f16":
        return x.astype(np.float16).astype(np.float64)
    return torch.from_numpy(x).float().bfloat16().double().numpy()       # (32 bits hold all of them)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_scale_and_code(dtype):
    """All 256 scales with all 16 codes, those among them that no append writes: rows read back, and
    what a single cached token gives, by each kernel, are the values rounded to the type."""
    import torch

    from paper_2608_21163_amd import Cache

    say(f"[every scale] {dtype}")
    codes = np.tile(np.array([2 * i | (2 * i + 1) << 4 for i in range(8)] * 2, np.uint8), (16, 16, 1, 1))
    scales = np.arange(256, dtype=np.uint8).reshape(16, 16, 1, 1)
    want = rounded(unpack(codes, scales, 32, dtype).reshape(256, 32), dtype)
    cache = Cache(dtype, 1, 1, 32, 16, stream=torch.cuda.current_stream().cuda_stream)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    for layout in ("rows", "token"):
        k, v = (as_packed(codes, scales, layout) for _ in range(2))
        for x in cache.read(ints(range(256)), k, v):
            assert np.array_equal(x[:, 0].double().cpu().numpy(), want, equal_nan=True)
    one = as_packed(codes, np.full_like(scales, 127), "token")
    q = torch.zeros(256, 1, 32, dtype=cache.torch_dtype, device="cuda")
    got = [cache.attend_ids(q, one, v, ints(range(256)).view(256, 1, 1))[0]]
    # sequences of one cached token each: slot 0 of pages of one slot
    flat = Cache(dtype, 1, 1, 32, 1, stream=torch.cuda.current_stream().cuda_stream)
    each = [type(x)(*(y.reshape(256, 1, 1, -1) for y in x)) for x in (as_packed(codes, np.full_like(scales, 127), "token"), as_packed(codes, scales, "token"))]
    got.append(flat.attend(flat.sequences(ints(range(256)).view(256, 1), ints([1] * 256)), q, *each)[0])
    # (chunks of 40 rows: the last of each sees the token)
    starts, many = ints(range(0, 257 * 40, 40)), torch.zeros(256 * 40, 1, 32, dtype=cache.torch_dtype, device="cuda")
    got.append(flat.attend(flat.sequences(ints(range(256)).view(256, 1), ints([1] * 256), starts, max_q=40), many, *each)[0][39::40])
    cache.check()
    flat.check()
    for name, x in zip(("list", "token", "chunk"), got):
        assert np.array_equal(x[:, 0].double().cpu().numpy(), want, equal_nan=True), name
    cache.close()
    flat.close()


@pytest.mark.parametrize("dtype,low,power", [("bf16", 0, 124), ("f16", 98, 12)])
@pytest.mark.parametrize("most_q", [1, 50])
def test_scales_that_no_append_writes(dtype, low, power, most_q):
    """Small scales beside each other in the keys (large queries) and in the values: keys, and
    the values of chunks, are rounded to the type, the values of lists are not."""
    import torch

    say(f"[small scales] {dtype} up to {most_q} tokens")
    c = packed(make(dtype, 4, 2, 64, 16, qs=(most_q, 1), ks=(70, 33), seed=most_q))
    r = np.random.default_rng(most_q)
    c["q"] = (c["q"].double() / 2 * 2.0 ** power).to(c["q"].dtype)
    # (bf16 ends at 2^128, fp16 at 2^16: no draw may pass that, as an infinite query gives no value with a key of 0)
    assert torch.isfinite(c["q"]).all()
    exact, total = {}, c["k_pages"].codes.shape[0] * 16
    for pool, name, span in (("k_pages", "keys", 4 if dtype == "bf16" else 10), ("v_pages", "vals", 12)):
        codes, scales = c[pool + "_np"]
        scales = r.integers(low, low + span, scales.shape).astype(np.uint8)
        c[pool] = as_packed(codes, scales, "head")
        exact[name] = unpack(codes, scales, 64, dtype).reshape(total, 2, 64)
        table = c["table"].cpu().numpy()
        slots = [table[b, np.arange(k) // 16] * 16 + np.arange(k) % 16 for b, k in enumerate(c["ks"])]
        c[name] = [torch.from_numpy(rounded(exact[name][x], dtype)) for x in slots]
    weighted(c, scale=1.0)
    ids = r.integers(0, total, (len(c["q"]), 4, 60)).astype(np.uint32)
    cache = cache_for(c)
    out, lse = cache.attend_ids(c["q"].cuda(), c["k_pages"], c["v_pages"], torch.from_numpy(ids.astype(np.int32)).cuda(), scale=1.0)
    cache.check()
    cache.close()
    want, z, bound, z_err = ids_ref(c["q"].double().numpy(), rounded(exact["keys"], dtype), exact["vals"], ids, 1.0)
    assert (np.abs(out.double().cpu().numpy() - want) <= bound(dtype)).all()
    assert (np.abs(lse.double().cpu().numpy() - z) <= z_err + 1e-30).all()


def one_buffer(n, page, hk, blocks, by):
    """A pool's codes and scales in one buffer: behind each other in every page, head of a
    page, or slot."""
    import torch

    from paper_2608_21163_amd import Packed

    row = 16 * blocks
    inner = {"page": page * hk, "head": page, "slot": hk}[by]
    outer = page * hk // inner
    size = -(-inner * (row + blocks) // 16) * 16
    x = torch.zeros(n, outer, size, dtype=torch.uint8, device="cuda")
    parts = x[:, :, :inner * row].unflatten(2, (inner, row))
    scales = x[:, :, inner * row:inner * (row + blocks)].unflatten(2, (inner, blocks))
    if by == "page":
        return Packed(parts[:, 0].unflatten(1, (page, hk)), scales[:, 0].unflatten(1, (page, hk)))
    if by == "head":
        return Packed(parts.transpose(1, 2), scales.transpose(1, 2))
    return Packed(parts, scales)


@pytest.mark.parametrize("by", ["page", "head", "slot"])
@pytest.mark.parametrize("hk,dim,page", [(2, 64, 16), (3, 40, 8), (1, 128, 64), (4, 256, 2)])
def test_codes_and_scales_in_one_buffer(by, hk, dim, page):
    """Appends, copies, attention and rows read back give what pools of four buffers give, bit by bit."""
    import torch

    from paper_2608_21163_amd import Packed

    say(f"[one buffer] by {by}, {hk} x {dim}, pages of {page}")
    c = make("bf16", 2 * hk, hk, dim, page, qs=(90, 20), ks=(90, 33), seed=dim)
    n, blocks = c["k_pages"].shape[0], -(-dim // 32)
    cache = cache_for(c)
    s = seqs_for(cache, c)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(110, hk, dim, device="cuda", generator=g).bfloat16() for _ in range(2))
    src, dst = c["table"][0, :1].clone(), torch.tensor([n - 1], dtype=torch.int32, device="cuda")
    used = set(c["table"][c["table"] >= 0].tolist())
    dst[0] = next(p for p in range(n) if p not in used)
    both = []
    for pools in (tuple(one_buffer(n, page, hk, blocks, by) for _ in range(2)),
                  tuple(Packed(torch.zeros(n, page, hk, 16 * blocks, dtype=torch.uint8, device="cuda"),
                               torch.zeros(n, page, hk, blocks, dtype=torch.uint8, device="cuda")) for _ in range(2))):
        cache.append(s, k, v, *pools)
        cache.copy_pages(*pools, src, dst)
        out = cache.attend(s, c["q"].cuda(), *pools)
        rows = cache.read(torch.arange(n * page, dtype=torch.int32, device="cuda"), *pools)
        cache.check()
        both.append([x.contiguous() for x in (*out, *rows, *pools[0], *pools[1])])
    assert all(torch.equal(a, b) for a, b in zip(*both))
    cache.close()
