"""The retrieval example runs the cache operators and the index together:
its bookkeeping holds, and its answers differ from attention over the whole
cache by no more than what the retrieved slots leave out."""
import os
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def test_retrieval_cache():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import retrieval_cache

    report, used = retrieval_cache.main(prompt=3000, chunk=700, answers=12)
    assert used["length"] == used["slots"] == 2048 and used["free"] == 4096 - 2048 and used["indexed"]
    for r in report:
        # what is left out has a weight of 1 - caught: a part of the whole
        # that values of that size can move it by twice, and two roundings
        left = 1 - r["caught"]
        assert (left > -1e-3).all()
        assert (r["error"] <= 2 * r["largest"] * (left + 2e-3) + 4 * 2.0 ** -8 * r["largest"]).all()
    assert sum(r["caught"].mean() for r in report) / len(report) > 0.9


def test_every_token_can_be_reached():
    """When an answer's searches run, each cached token is in the window, in
    its key/value head's index, or a listed sink: also right after a token has left
    the window, and while the sinks are leaving it."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import numpy as np
    import retrieval_cache

    window, sinks = 64, 4
    layer = retrieval_cache.RetrievalLayer(slots=1024, budget=512, window=window, sinks=sinks, k=32, beam=64)
    q, k, v = retrieval_cache.conversation(700, layer.hq, layer.hk, layer.dim)
    attend_ids, seen = layer.cache.attend_ids, []

    def watched(rows, k_pages, v_pages, ids, **kw):
        table = layer.table[0, :layer.length].tolist()
        for h, index in enumerate(layer.index):
            held = set(np.flatnonzero(index.export()["active"]).tolist())
            listed = set(ids[0, h * layer.hq // layer.hk, layer.k:].tolist()) - {-1}
            near = set(table[-window:])
            assert held | listed | near == set(table) and not (held | listed) & near and not held & listed
        seen.append(len(table))
        return attend_ids(rows, k_pages, v_pages, ids, **kw)

    layer.cache.attend_ids = watched
    for i in range(window + 8):
        layer.answer(q[i:i + 1], k[i:i + 1], v[i:i + 1])
    layer.read(q[80:680], k[80:680], v[80:680])
    for i in range(690, 694):
        layer.answer(q[i:i + 1], k[i:i + 1], v[i:i + 1])
    assert seen == list(range(1, window + 9)) + [513] * 4
    layer.cache.attend_ids = attend_ids
    layer.close()
