"""Pages that sequences share (fork, grow, release, compact, copies) against
their definitions, in pools from one page to several workgroups' and where
lists, tables and pools run out; and all cache operators together."""
import math

import numpy as np
import pytest

from cache_ref import INVALID
from packed_ref import compact_ref, fork_ref, grow_ref, names, release_ref
from parity import say
from test_gpu_cache_attend import cache_for, make, seqs_for
from test_gpu_packed import as_packed, compare, packed

pytestmark = pytest.mark.gpu


def shared_sequences(n_seq, page, n_pages, width, seed, longest=None):
    """(table, lens, refs): rows of `width` pages, some of which begin with
    another row's pages; entries behind a row's pages are anything."""
    r = np.random.default_rng(seed)
    order = list(r.permutation(n_pages))
    table = r.integers(0, 2 ** 32, (n_seq, width), dtype=np.uint64).astype(np.uint32)
    lens = np.zeros(n_seq, np.uint32)
    for b in range(n_seq):
        want = int(r.integers(0, (longest or width * page) + 1))
        n, have = -(-want // page), 0
        if b and r.random() < 0.6:
            other = int(r.integers(0, b))
            have = min(n, -(-int(lens[other]) // page))
            if r.random() < 0.5 and have:      # the other's whole row, its partly filled page too
                want, n = int(lens[other]), -(-int(lens[other]) // page)
                have = n
            elif have and lens[other] % page and have == -(-int(lens[other]) // page):
                have -= 1
            table[b, :have] = table[other, :have]
        if n - have > len(order):
            n = have
            want = min(want, n * page)
        for i in range(have, n):
            table[b, i] = order.pop()
        lens[b] = want
    return table, lens, names(table, lens, page, n_pages)


def cache_of(page=16, hk=2, dim=64, dtype="bf16", hq=None):
    import torch

    from paper_2608_21163_amd import Cache
    return Cache(dtype, hq or hk, hk, dim, page, stream=torch.cuda.current_stream().cuda_stream)


def ints(x):
    import torch

    return torch.from_numpy(np.ascontiguousarray(np.asarray(x).astype(np.uint32).view(np.int32))).cuda()


def back(x):
    return x.cpu().numpy().view(np.uint32)


def equal(got, want):
    got, want = back(got), np.asarray(want).astype(np.uint32)
    assert got.shape == want.shape and np.array_equal(got, want), (got[got != want][:8], want[got != want][:8])


SIZES = [(1, 16, 1, 1), (3, 1, 40, 12), (5, 16, 64, 9), (40, 4, 2048, 70), (64, 16, 2049, 40), (7, 64, 70_000, 3000), (300, 8, 9000, 33)]


@pytest.mark.parametrize("n_seq,page,n_pages,width", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("drop", [False, True])
def test_fork(n_seq, page, n_pages, width, in_place, drop):
    import torch

    say(f"[fork] {n_seq} rows of {width} pages of {page}, pool {n_pages}, in place {in_place}, drop {drop}")
    table, lens, refs = shared_sequences(n_seq, page, n_pages, width, n_seq)
    r = np.random.default_rng(width)
    parents = r.integers(0, n_seq, n_seq + 3).astype(np.uint32)
    parents[r.random(len(parents)) < 0.1] = INVALID
    want = fork_ref(table, lens, page, parents, refs, drop)
    cache = cache_of(page)
    t, l, c = ints(table), ints(lens), ints(refs)
    out = c if in_place else torch.full_like(c, -7)
    got = cache.fork(cache.sequences(t, l), ints(parents), c, drop=drop, refs_out=None if in_place else out)
    cache.check()
    assert got[2] is out
    for g, w in zip(got, want):
        equal(g, w)
    equal(t, table)
    if not in_place:
        equal(c, refs)
    cache.close()


@pytest.mark.parametrize("n_seq,page,n_pages,width", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("most", [1, 40])
def test_grow(n_seq, page, n_pages, width, in_place, most):
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ARG, E_CAPACITY

    say(f"[grow] {n_seq} rows of {width} pages of {page}, pool {n_pages}, in place {in_place}, up to {most}")
    table, lens, refs = shared_sequences(n_seq, page, n_pages, width, n_seq + most, longest=max(1, width * page * 3 // 4))
    new = np.random.default_rng(most).integers(0, most + 1, n_seq).astype(np.uint32)
    want = grow_ref(table, lens, page, new, refs)
    cache = cache_of(page)
    wide = ints(np.concatenate([table, np.full((n_seq, 3), 9, np.uint32)], 1))   # a table with a stride of its own
    t, l, c = wide[:, :width], ints(lens), ints(refs)
    out = c if in_place else torch.full_like(c, -7)
    got = cache.grow(cache.sequences(t, l), ints(new), c, refs_out=None if in_place else out)
    assert got[0] is t and got[1] is l
    for g, w in zip((t, l, out, got[2], got[3]), want):
        equal(g.contiguous(), w)
    assert (wide[:, width:] == 9).all()
    if want[5]:
        with pytest.raises(GrandError) as e:
            cache.check()
        assert e.value.code in (E_ARG, E_CAPACITY)
    cache.check()
    equal(out, names(want[0], want[1], page, n_pages)) if want[5] == [] else None
    cache.close()


@pytest.mark.parametrize("n_seq", [255, 256, 257, 2047, 2048, 2049, 5000])
@pytest.mark.parametrize("short", [0, 1, 700])
def test_grow_of_many_sequences(n_seq, short):
    """Some wait for pages where the pool is `short` of them."""
    from paper_2608_21163_amd import GrandError

    r = np.random.default_rng(n_seq + short)
    page = 4
    lens = r.integers(0, 17, n_seq)
    held = -(-lens // page)
    new = r.integers(0, 9, n_seq)
    want_pages = int((-(-(lens + new) // page) - held).sum())
    n_pages = int(held.sum()) + max(0, want_pages - short)
    order = r.permutation(n_pages)
    table, at = np.full((n_seq, 7), INVALID, np.uint32), 0
    for b in range(n_seq):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    lens, new = lens.astype(np.uint32), new.astype(np.uint32)
    refs = names(table, lens, page, n_pages)
    want = grow_ref(table, lens, page, new, refs)
    assert bool(want[5]) == bool(short)
    cache = cache_of(page)
    t, l, c = ints(table), ints(lens), ints(refs)
    got = cache.grow(cache.sequences(t, l), ints(new), c)
    for g, w in zip((t, l, c, got[2], got[3]), want):
        equal(g, w)
    if short:
        with pytest.raises(GrandError):
            cache.check()
    cache.check()
    cache.close()


def test_grow_when_pages_run_out():
    """In order: what does not fit stays as it was, and so does what comes after it and needs a page."""
    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_CAPACITY

    page = 4
    table = np.full((6, 8), INVALID, np.uint32)
    for b in range(6):
        table[b, 0] = b
    lens = np.array([4, 3, 4, 2, 4, 0], np.uint32)
    refs = np.array([1] * 5 + [0] * 5, np.int64)          # five free pages
    new = np.array([9, 1, 9, 2, 1, 1], np.uint32)         # 3, 0, 3 (does not fit), 0, 1, 1
    want = grow_ref(table, lens, page, new, refs)
    assert want[5] == [2, 4, 5] and list(want[1]) == [13, 4, 4, 4, 4, 0]
    cache = cache_of(page)
    t, l, c = ints(table), ints(lens), ints(refs)
    _, _, src, dst = cache.grow(cache.sequences(t, l), ints(new), c)
    for g, w in zip((t, l, c, src, dst), want):
        equal(g, w)
    with pytest.raises(GrandError) as e:
        cache.check()
    assert e.value.code == E_CAPACITY
    cache.close()


@pytest.mark.parametrize("n_seq,page,n_pages,width", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("counts", ["none", "pages", "tokens"])
def test_release(n_seq, page, n_pages, width, in_place, counts):
    import torch

    say(f"[release] {n_seq} rows of {width} pages of {page}, pool {n_pages}, in place {in_place}, {counts}")
    table, lens, refs = shared_sequences(n_seq, page, n_pages, width, n_seq)
    gone = np.random.default_rng(n_pages).permutation(n_seq)[:(n_seq + 1) // 2]
    ids, n = table[gone], -(-lens[gone].astype(np.int64) // page)
    if counts == "none":
        ids = np.where(np.arange(width) < n[:, None], ids, INVALID).astype(np.uint32)
    want = release_ref(ids, None if counts == "none" else n, refs)
    cache = cache_of(page)
    t, c = ints(ids), ints(refs)
    out = c if in_place else torch.full_like(c, -7)
    got = cache.release(t, c, counts=None if counts == "none" else ints(n if counts == "pages" else lens[gone]), tokens=counts == "tokens",
                        refs_out=None if in_place else out)
    cache.check()
    equal(got[0], want[0])
    equal(got[1], want[1])
    assert int(got[2]) == want[2]
    cache.close()


def test_release_of_more_names_than_counted():
    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ARG

    refs, ids = np.array([2, 0, 1], np.int64), np.array([[0, 1, 2, 2, 0]], np.uint32)
    cache = cache_of()
    c = ints(refs)
    got = cache.release(ints(ids), c)
    for g, w in zip(got[:2], release_ref(ids, None, refs)):
        equal(g, w)
    assert int(got[2]) == 2
    with pytest.raises(GrandError) as e:
        cache.check()
    assert e.value.code == E_ARG
    cache.close()


@pytest.mark.parametrize("n_pages", [524_288, 524_289, 1_000_001])
@pytest.mark.parametrize("in_place", [False, True])
def test_release_in_large_pools(n_pages, in_place):
    import torch

    from paper_2608_21163_amd import GrandError

    r = np.random.default_rng(n_pages)
    refs = r.integers(0, 4, n_pages)
    refs[-1] = refs[0] = 1
    ids = r.integers(0, n_pages, (64, 5000)).astype(np.uint32)
    ids[3, 17], ids[60, 4999] = n_pages - 1, 0
    cache = cache_of()
    c, t = ints(refs), ints(ids)
    out = c if in_place else torch.full_like(c, -7)
    got = cache.release(t, c, refs_out=None if in_place else out)
    want = release_ref(ids, None, refs)
    equal(got[0], want[0])
    equal(got[1], want[1])
    assert int(got[2]) == want[2] > 10_000
    with pytest.raises(GrandError):         # a quarter of the pages are named though free
        cache.check()
    cache.close()


@pytest.mark.parametrize("n_seq,page,n_pages,width", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(n_seq, page, n_pages, width, in_place):
    import ctypes

    import torch

    say(f"[compact] {n_seq} rows of {width} pages of {page}, pool {n_pages}, in place {in_place}")
    table, lens, refs = shared_sequences(n_seq, page, n_pages, width, n_seq)
    want = compact_ref(table, lens, page, refs)
    cache = cache_of(page)
    t, l, c = ints(table), ints(lens), ints(refs)
    s = cache.sequences(t, l)
    if in_place:
        src, dst, moves = torch.empty_like(c), torch.empty_like(c), torch.empty(1, dtype=torch.int32, device="cuda")
        cache._check(cache.lib.grand_pages_compact(cache.h, s.ref, n_pages, c.data_ptr(), c.data_ptr(), t.data_ptr(), src.data_ptr(),
                                                   dst.data_ptr(), moves.data_ptr()))
        got = t, c, src, dst, moves
        mine = np.arange(width) < (-(-lens.astype(np.int64) // page))[:, None]
        want = (np.where(mine, want[0], table),) + want[1:]          # behind a row's pages nothing changes
    else:
        got = cache.compact(s, c, refs_out=torch.full_like(c, -7))
        equal(t, table)
        equal(c, refs)
    cache.check()
    for g, w in zip(got[:4], want):
        equal(g, w)
    assert int(got[4]) == want[4]
    cache.close()


@pytest.mark.parametrize("n_pages", [1, 63, 64, 2047, 2048, 4097])
@pytest.mark.parametrize("fill", ["none", "all", "front", "back", "odd"])
def test_compact_extremes(n_pages, fill):
    """Pools that are empty, full, compact, the other way round or full of holes, without sequences."""
    import torch

    refs = {"none": np.zeros(n_pages), "all": np.ones(n_pages), "front": np.arange(n_pages) < n_pages // 3,
            "back": np.arange(n_pages) >= n_pages // 3, "odd": np.arange(n_pages) % 2}[fill].astype(np.int64)
    want = compact_ref(np.zeros((0, 4), np.uint32), np.zeros(0), 16, refs)
    cache = cache_of()
    got = cache.compact(cache.sequences(torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")),
                        ints(refs))
    cache.check()
    for g, w in zip(got[:4], want):
        equal(g, w)
    assert int(got[4]) == want[4]
    cache.close()


@pytest.mark.parametrize("kind", ["token", "head", "gaps", "packed-token", "packed-head", "packed-rows"])
@pytest.mark.parametrize("hk,dim,page", [(2, 64, 16), (8, 128, 16), (1, 8, 1), (3, 40, 2), (8, 128, 64), (1, 256, 1), (1, 64, 16)])
def test_copies(kind, hk, dim, page):
    """Pages go where the lists say, entries without a page or with one from
    outside the pool are passed over, everything else stays."""
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ID

    say(f"[copy pages] {kind} {hk} x {dim}, pages of {page}")
    r, n, blocks = np.random.default_rng(dim), 50, -(-dim // 32)
    cache = cache_of(page, hk, dim)
    order = r.permutation(n).astype(np.uint32)
    src, dst = order[:20].copy(), order[20:40].copy()
    src[3], dst[5], src[7] = INVALID, INVALID, src[8]
    pools = []
    for _ in range(2):
        if kind.startswith("packed"):
            codes = r.integers(0, 256, (n, page, hk, 16 * blocks), dtype=np.uint8)
            scales = r.integers(0, 256, (n, page, hk, blocks), dtype=np.uint8)
            pools.append(as_packed(codes, scales, kind[7:]))
        else:
            x = torch.from_numpy(r.standard_normal((n, page, hk, dim))).bfloat16().cuda()
            if kind == "head":
                x = x.transpose(1, 2).contiguous().transpose(1, 2)
            elif kind == "gaps":
                big = torch.zeros(n, page, hk + 1, dim + 8, dtype=torch.bfloat16, device="cuda")
                big[:, :, :hk, :dim] = x
                x = big[:, :, :hk, :dim]
            pools.append(x)
    parts = [x for p in pools for x in (p if kind.startswith("packed") else (p,))]
    want = [x.clone() for x in parts]
    for s, d in zip(src, dst):
        if INVALID not in (s, d):
            for w in want:
                w[int(d)] = w[int(s)]
    cache.copy_pages(*pools, ints(src), ints(dst))
    cache.check()
    assert all(torch.equal(a, b) for a, b in zip(parts, want))
    for bad in ((np.array([n, 1]), np.array([0, 1])), (np.array([0, 1]), np.array([n + 5, 1]))):
        cache.copy_pages(*pools, ints(bad[0]), ints(bad[1]))
        assert all(torch.equal(a, b) for a, b in zip(parts, want))
        with pytest.raises(GrandError) as e:
            cache.check()
        assert e.value.code == E_ID
    cache.copy_pages(*pools, ints(src[:0]), ints(dst[:0]))
    cache.close()


def test_ids_out_of_range_are_reported():
    """Page ids, parents and lengths outside their range: reported, and nothing outside the buffers is touched."""
    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ARG, E_ID

    page, n_pages = 4, 10
    table, lens, refs = np.array([[0, 1, 77], [2, 3, 4]], np.uint32), np.array([10, 9], np.uint32), np.array([1] * 5 + [0] * 5, np.int64)
    cache = cache_of(page)

    def reported(code, call):
        call()
        with pytest.raises(GrandError) as e:
            cache.check()
        assert e.value.code == code
        cache.check()

    s = cache.sequences(ints(table), ints(lens))
    reported(E_ID, lambda: cache.fork(s, ints([0]), ints(refs)))
    reported(E_ARG, lambda: cache.fork(s, ints([1, 2]), ints(refs)))
    reported(E_ID, lambda: cache.grow(cache.sequences(ints(table), ints(lens)), ints([1, 1]), ints(refs)))
    reported(E_ID, lambda: cache.release(ints(table), ints(refs)))
    reported(E_ARG, lambda: cache.release(ints(table), ints(refs), counts=ints([2, 4])))
    reported(E_ID, lambda: cache.compact(s, ints(refs)))
    unnamed = cache.sequences(ints([[0, 1, 8]]), ints([12]))
    reported(E_ARG, lambda: cache.compact(unnamed, ints(refs)))      # page 8 is named, and its count is 0
    short = cache.sequences(ints(table), ints([10, 500]), max_k=12)
    reported(E_ARG, lambda: cache.fork(short, ints([1]), ints(refs)))
    reported(E_ARG, lambda: cache.grow(cache.sequences(ints([[0, 1, 2]]), ints([12])), ints([1]), ints(refs)))   # the row is full
    cache.close()


def beam_state(kind, seed=0):
    """Four beams over one prompt, their own tokens behind it."""
    c = make("f16", 8, 2, 64, 16, qs=(1, 1, 1, 1), ks=(70, 70, 70, 70), seed=seed, spare_pages=24, max_pages=8)
    for b in range(1, 4):
        c["table"][b, :4] = c["table"][0, :4]
        for name in ("keys", "vals"):
            c[name][b][:64] = c[name][0][:64]
    return packed(c, kind) if kind != "whole" else c


@pytest.mark.parametrize("kind", ["whole", "token", "rows"])
def test_steps_of_a_beam(kind):
    """Beams go on from one another's, get pages, write their tokens and
    attend, for 40 steps; at the end one is given back and the pool is made compact.
    Results are those of caches that share nothing."""
    import torch

    from packed_ref import pack, unpack
    say(f"[beam] {kind}")
    c = beam_state(kind)
    cache = cache_for(c)
    refs = ints(names(c["table"].cpu().numpy().view(np.uint32), [70] * 4, 16, c["k_pages"][0].shape[0] if kind != "whole" else c["k_pages"].shape[0]))
    table, lens = c["table"], c["lens"]
    one = ints([1, 1, 1, 1])
    g = torch.Generator().manual_seed(4)
    keys, vals = c["keys"], c["vals"]
    for step in range(40):
        parents = torch.randint(0, 4, (4,), generator=g)
        table, lens, refs = cache.fork(cache.sequences(table, lens), ints(parents.numpy()), refs, drop=True)
        s = cache.sequences(table, lens, max_k=128)
        _, _, src, dst = cache.grow(s, one, refs)
        cache.copy_pages(c["k_pages"], c["v_pages"], src, dst)
        k, v, q = (torch.randn(4, n, 64, generator=g).half() for n in (2, 2, 8))
        cache.append(s, k.cuda(), v.cuda(), c["k_pages"], c["v_pages"])
        out, lse = cache.attend(s, q.cuda(), c["k_pages"], c["v_pages"])

        def held(x):
            return x if kind == "whole" else torch.from_numpy(unpack(*pack(x.double().numpy(), "f16"), 64, "f16"))
        keys = [torch.cat([keys[p], held(k[b:b + 1])]) for b, p in enumerate(parents)]
        vals = [torch.cat([vals[p], held(v[b:b + 1])]) for b, p in enumerate(parents)]
        if step % 8 == 7 or step < 2:
            compare(dict(dtype="f16", dim=64, q=q, keys=keys, vals=vals, qs=(1,) * 4, ks=(71 + step,) * 4, starts=range(5)), out, lse)
    cache.check()
    n_pages = len(refs)
    equal(refs, names(back(table), [110] * 4, 16, n_pages))
    _, freed, n_freed = cache.release(table[:1], refs, counts=lens[:1], tokens=True)
    table, lens = table[1:].contiguous(), lens[1:].contiguous()
    equal(refs, names(back(table), [110] * 3, 16, n_pages))
    table, refs, src, dst, moves = cache.compact(cache.sequences(table, lens), refs)
    cache.copy_pages(c["k_pages"], c["v_pages"], src, dst)
    used = int((refs > 0).sum())
    assert used < n_pages and (refs[:used] > 0).all() and int(table[:, :7].max()) == used - 1
    s = cache.sequences(table, lens, max_k=110)
    front = [type(p)(*(x[:used] for x in p)) if kind != "whole" else p[:used] for p in (c["k_pages"], c["v_pages"])]
    out, lse = cache.attend(s, q[1:].cuda(), *front)
    cache.check()
    compare(dict(dtype="f16", dim=64, q=q[1:], keys=keys[1:], vals=vals[1:], qs=(1,) * 3, ks=(110,) * 3, starts=range(4)), out, lse)
    cache.close()


def test_evicted_pages_that_others_share():
    """What an eviction frees goes back by release: pages that another
    sequence names stay, and their data with them."""
    import torch

    c = make(qs=(1, 1), ks=(100, 100), page=16, spare_pages=4)
    c["table"][1, :4] = c["table"][0, :4]
    n_pages = c["k_pages"].shape[0]
    refs = ints(names(back(c["table"]), [100, 100], 16, n_pages))
    cache = cache_for(c)
    w = torch.arange(100, device="cuda").float().repeat(2, 2, 1)
    table, _, lens, freed, n_freed = cache.evict(seqs_for(cache, c), w, ints([3, 7]), recent=1)
    old = back(c["table"])
    assert back(n_freed).tolist() == [4, 0]                   # of the first sequence, its first four pages
    refs, gone, n_gone = cache.release(freed, refs, counts=n_freed)
    cache.check()
    assert int(n_gone) == 0 and (refs[torch.from_numpy(old[0, :4].astype(np.int64)).cuda()] == 1).all()
    equal(refs, names(back(table), back(lens), 16, n_pages))
    cache.close()


@pytest.mark.parametrize("kind", ["whole", "token"])
def test_a_captured_step(kind):
    """A step of a beam in one captured graph, replayed with other parents, other
    rows and eager work between: every replay gives what eager calls give."""
    import torch

    say(f"[captured beam] {kind}")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c, e = beam_state(kind, 1), beam_state(kind, 1)
        n_pages = (c["k_pages"] if kind == "whole" else c["k_pages"].codes).shape[0]
        refs0 = names(back(c["table"]), [70] * 4, 16, n_pages)
        sides = []
        for x in (c, e):
            cache = cache_for(x)
            st = dict(cache=cache, table=x["table"].clone(), lens=x["lens"].clone(), refs=ints(refs0), parents=ints([0, 1, 2, 3]), one=ints([1] * 4),
                      k=torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda"), v=torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda"),
                      q=torch.zeros(4, 8, 64, dtype=torch.float16, device="cuda"), pages=(x["k_pages"], x["v_pages"]))
            sides.append(st)

        def step(st):
            cache = st["cache"]
            table, lens, _ = cache.fork(cache.sequences(st["table"], st["lens"]), st["parents"], st["refs"], drop=True)
            st["table"].copy_(table)
            st["lens"].copy_(lens)
            s = cache.sequences(st["table"], st["lens"], max_k=128)
            _, _, src, dst = cache.grow(s, st["one"], st["refs"])
            cache.copy_pages(*st["pages"], src, dst)
            cache.append(s, st["k"], st["v"], *st["pages"])
            return cache.attend(s, st["q"], *st["pages"], window=40, sinks=4)

        saved = [x.clone() for x in (sides[0]["table"], sides[0]["lens"], sides[0]["refs"])]
        pools = [y for p in sides[0]["pages"] for y in (p if kind != "whole" else (p,))]
        pools_saved = [y.clone() for y in pools]
        step(sides[0])                                        # workspaces grow outside the capture
        for x, y in zip((sides[0]["table"], sides[0]["lens"], sides[0]["refs"]), saved):
            x.copy_(y)
        for x, y in zip(pools, pools_saved):
            x.copy_(y)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            captured = step(sides[0])
        g = torch.Generator().manual_seed(2)
        for i in range(30):
            fresh = [torch.randint(0, 4, (4,), generator=g).int()] + [torch.randn(4, n, 64, generator=g).half() for n in (2, 2, 8)]
            for st in sides:
                for name, x in zip(("parents", "k", "v", "q"), fresh):
                    st[name].copy_(x)
            graph.replay()
            want = step(sides[1])
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(captured, want)), i
            assert all(torch.equal(sides[0][n], sides[1][n]) for n in ("table", "lens", "refs")), i
        for st in sides:
            st["cache"].check()
            st["cache"].close()


def test_calls_on_another_stream():
    """A handle on its own stream, beside work on the current one: calls are ordered by the handle's."""
    import torch

    stream = torch.cuda.Stream()
    c = packed(make(qs=(1, 3), ks=(90, 400)))
    from paper_2608_21163_amd import Cache

    cache = Cache(c["dtype"], c["hq"], c["hk"], c["dim"], c["page"], stream=stream.cuda_stream)
    q = c["q"].cuda()
    torch.cuda.synchronize()
    s = cache.sequences(c["table"], c["lens"], c["q_start"], max_q=3, max_k=400)
    outs = [cache.attend(s, q, c["k_pages"], c["v_pages"], window=50, sinks=2) for _ in range(3)]
    rows = cache.read(ints([int(c["table"][0, 0]) * 16]), c["k_pages"], c["v_pages"])
    stream.synchronize()
    for out, lse in outs:
        compare(c, out, lse, window=50, sinks=2)
    assert np.array_equal(rows[0][0].double().cpu().numpy(), c["keys"][0][0].numpy())
    cache.check()
    cache.close()


def test_calls_that_the_binding_does_not_make():
    """Keys or values read alone, and attention without its log-sum-exps."""
    import torch

    k = packed(make(qs=(1, 1), ks=(90, 700)))
    cache = cache_for(k)
    slots = ints([int(k["table"][1, p // 16]) * 16 + p % 16 for p in (0, 77, 699)])
    both = cache.read(slots, k["k_pages"], k["v_pages"])
    pages = cache._packed(k["k_pages"], k["v_pages"])
    for i, name in enumerate(("k", "v")):
        x = torch.empty_like(both[0])
        r = cache._rows(name, x, k["hk"], 3)
        cache._check(cache.lib.grand_packed_read(cache.h, 3, slots.data_ptr(), pages, r if i == 0 else None, r if i == 1 else None))
        cache.check()
        assert torch.equal(x, both[i])
    q, s = k["q"].cuda(), seqs_for(cache, k)
    out, lse = cache.attend(s, q, k["k_pages"], k["v_pages"])
    alone = torch.full_like(out, 7)
    n, ref = cache._tokens(s, q)
    cache._check(cache.lib.grand_cache_attend_packed(cache.h, ref, cache._rows("q", q, k["hq"], n), pages, k["dim"] ** -0.5, 1, 0, 0,
                                                     cache._rows("out", alone, k["hq"], n), None, None, None))
    cache.check()
    assert torch.equal(alone, out)
    cache.close()


@pytest.mark.parametrize("in_place", [False, True])
def test_growth_past_max_k(in_place):
    """A call may bring a length above max_k. A sequence that has one before the
    call stays as it was, whatever its row holds there, and is reported; the others grow."""
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ARG

    page = 4
    table = np.array([[0, 1, 77, 5], [2, INVALID, INVALID, INVALID], [3, 1, INVALID, INVALID]], np.uint32)
    lens, refs = np.array([8, 4, 7], np.uint32), np.array([1, 2, 1, 1, 0, 0, 0, 0], np.int64)
    cache = cache_of(page)
    t, l, c = ints(table), ints(lens), ints(refs)
    s = cache.sequences(t, l, max_k=7)

    def grow(new, c):
        out = c if in_place else torch.full_like(c, -7)
        return cache.grow(s, ints(new), c, refs_out=out)[2:] + (out,)
    # lengths 8 (above max_k), 4 and 7: pages 4 for the second, 5 for the third's copy
    src, dst, c = grow([9, 4, 1], c)
    for g, w in ((t, [table[0], [2, 4, INVALID, INVALID], [3, 5, INVALID, INVALID]]), (l, [8, 8, 8]), (c, [1, 1, 1, 1, 1, 1, 0, 0]),
                 (src, [INVALID, INVALID, 1]), (dst, [INVALID, INVALID, 5])):
        equal(g, w)
    with pytest.raises(GrandError) as e:
        cache.check()
    assert e.value.code == E_ARG
    # all three are above it now
    before = [x.clone() for x in (t, l, c)]
    src, dst, c = grow([1, 1, 1], c)
    assert all(torch.equal(a, b) for a, b in zip((t, l, c), before)) and (src == -1).all() and (dst == -1).all()
    with pytest.raises(GrandError) as e:
        cache.check()
    assert e.value.code == E_ARG
    cache.check()
    cache.close()


@pytest.mark.parametrize("in_place", [False, True])
def test_fork_that_drops_more_names_than_counted(in_place):
    """Names are dropped before new ones are counted: a count that they would take
    below 0 is reported and starts from there, in whatever order names come."""
    import torch

    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ARG

    say(f"[fork, dropped too often] in place {in_place}")
    page, n_seq, width = 4, 200, 90
    r = np.random.default_rng(3)
    table = r.integers(0, 70, (n_seq, width)).astype(np.uint32)
    lens = r.integers(0, width * page + 1, n_seq).astype(np.uint32)
    held = names(table, lens, page, 100)
    refs = np.where(np.arange(100) % 7 == 0, held // 2, held + np.arange(100) % 3)   # every seventh has too low a count
    parents = r.integers(0, n_seq, 50).astype(np.uint32)
    new, new_lens, added = fork_ref(table, lens, page, parents, np.zeros(100, np.int64), False)
    cache = cache_of(page)
    t, l = ints(table), ints(lens)
    for n_out in (50, 0):
        c = ints(refs)
        out = c if in_place else torch.full_like(c, -7)
        got = cache.fork(cache.sequences(t, l), ints(parents[:n_out]), c, drop=True, refs_out=out)
        equal(got[0], new[:n_out])
        equal(got[1], new_lens[:n_out])
        equal(out, np.maximum(refs - held, 0) + (added if n_out else 0))
        with pytest.raises(GrandError) as e:
            cache.check()
        assert e.value.code == E_ARG and "names" in str(e.value)
    # one page, one name, never counted; the rest of the pool is found as before
    c = ints([1, 0, 0])
    cache.fork(cache.sequences(ints([[0, 1]]), ints([8])), ints([]), c, drop=True)
    equal(c, [0, 0, 0])
    with pytest.raises(GrandError):
        cache.check()
    cache.check()
    cache.close()


@pytest.mark.parametrize("n_seq,counted", [(3, 2), (300, 2), (300, 299), (300, 300)])
def test_growth_of_more_sequences_than_a_page_counts(n_seq, counted):
    """Every sequence gets its copy of the partly filled page that they share; names
    beyond its count are reported, and the count ends at 0."""
    from paper_2608_21163_amd import GrandError
    from paper_2608_21163_amd.grand import E_ARG

    table, lens = np.zeros((n_seq, 2), np.uint32), np.full(n_seq, 3, np.uint32)
    refs = np.zeros(n_seq + 5, np.int64)
    refs[0], refs[1] = counted, 7
    cache = cache_of(4)
    t, l, c = ints(table), ints(lens), ints(refs)
    _, _, src, dst = cache.grow(cache.sequences(t, l), ints(np.ones(n_seq)), c)
    new = np.arange(2, n_seq + 2)
    equal(c, np.concatenate([[0, 7], np.ones(n_seq), np.zeros(3)]))
    equal(t, np.stack([new, 0 * new], 1))
    equal(l, lens + 1)
    equal(src, 0 * new)
    equal(dst, new)
    if counted < n_seq:
        with pytest.raises(GrandError) as e:
            cache.check()
        assert e.value.code == E_ARG and "names" in str(e.value)
    cache.check()
    cache.close()
