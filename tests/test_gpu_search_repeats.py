"""Lists that name an id more than once, as a reader sees one that is being
rewritten: searches find what they find in the graph without the repeats, and
read no ids from memory that nothing wrote."""
import numpy as np
import pytest

from parity import say

pytestmark = pytest.mark.gpu

INVALID = 0xFFFFFFFF


@pytest.mark.parametrize("kind,dtype", [("u8_128", "u8"), ("f32_96", "f32")])
@pytest.mark.parametrize("beam", [40, 64, 128, 256])
@pytest.mark.parametrize("reader", [False, True])
@pytest.mark.parametrize("degree", [6, 30, 60])
def test_repeated_ids(kind, dtype, beam, reader, degree):
    from paper_2608_21163_amd import GrandIndex, Reader
    from workloads import IndexConfig

    say(f"[repeats] {kind} beam {beam} reader {reader} degree {degree}")
    dim, n, R = int(kind.split("_")[1]), 5000, 64
    r = np.random.default_rng(degree)
    vecs = r.integers(0, 256, (n, dim)).astype(np.uint8) if dtype == "u8" else r.standard_normal((n, dim)).astype(np.float32)
    adj = np.full((n, R), INVALID, np.uint32)
    for u in range(n):
        adj[u, :degree] = r.choice(np.delete(np.arange(n), u), degree, replace=False)
    twice = adj.copy()
    for u in range(n):                                  # behind the list: some of its ids again, in any order
        m = min(R - degree, degree)
        twice[u, degree:degree + m] = r.permutation(adj[u, :degree])[:m]
        if u % 2:
            r.shuffle(twice[u, :degree + m])
            first = np.unique(twice[u, :degree + m], return_index=True)[1]
            adj[u, :degree] = twice[u, np.sort(first)]  # the same list in the order of first occurrence
    q = r.integers(0, 256, (300, dim)).astype(np.uint8) if dtype == "u8" else r.standard_normal((300, dim)).astype(np.float32)
    got = []
    for lists in (adj, twice):
        g = GrandIndex.from_config(IndexConfig("vamana", dtype, "l2", dim, n, R, 64), max_batch=1000)
        g.import_graph(vecs, lists, (lists != INVALID).sum(1).astype(np.uint32), np.ones(n, np.uint8), 17)
        x = Reader(g) if reader else g
        got.append([x.search(q, 10, beam) for _ in range(3)])
        if reader:
            x.close()
        g.close()
    for a, b in zip(*got):
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
