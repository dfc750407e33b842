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
