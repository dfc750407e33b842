"""Numbers at the edges of the cache operators' types: infinite keys whose
weight is zero."""
import math

import numpy as np
import pytest

from cache_ref import attend_ref
from parity import say
from test_gpu_cache_attend import make, run

pytestmark = pytest.mark.gpu


def put(c, pages, b, pos, x):
    """Token pos of sequence b holds x (kv_heads x dim)."""
    pages[int(c["table"][b, pos // c["page"]]), pos % c["page"]] = x.to(pages.dtype).to(pages.device)


@pytest.mark.parametrize("qs,hq,hk", [(3, 4, 2), (32, 4, 2), (33, 4, 2), (77, 3, 1), (300, 8, 1)])
@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f16", 128), ("bf16", 256)])
@pytest.mark.parametrize("causal", [True, False])
def test_a_seen_key_of_weight_zero(qs, hq, hk, dtype, dim, causal):
    """An infinite element of a key that every row sees makes its score -inf:
    results and weights are those without that token, its own weight is 0,
    whether the rows fill the kernels' tiles or not."""
    import torch

    say(f"[cache zero weight] {qs} rows {hq}/{hk} x {dim} {dtype} causal {causal}")
    kl, at = qs + 67, 5
    c = make(dtype, hq, hk, dim, 16, qs=(qs,), ks=(kl,), seed=qs + dim)
    c["q"][..., 0] = -(c["q"][..., 0].abs() + 0.125)
    c["keys"][0][at, :, 0] = math.inf
    put(c, c["k_pages"], 0, at, c["keys"][0][at])
    before = torch.rand(1, hk, kl, device="cuda")
    out, lse, w = run(c, causal=causal, weights=before, weights_out=before.clone())
    left = [j for j in range(kl) if j != at]
    k, v = (c[n][0][left].double().numpy() for n in ("keys", "vals"))
    ro, rz, rw, bound, z_err, w_err = attend_ref(c["q"].double().numpy(), k, v, kl - qs - 1, dim ** -0.5, causal)
    assert (np.abs(out.double().cpu().numpy() - ro) <= bound(dtype)).all()
    assert (np.abs(lse.double().cpu().numpy() - rz) <= z_err).all()
    old, new = (x[0].double().cpu().numpy() for x in (before, w))
    assert np.array_equal(new[:, at], old[:, at])
    assert (np.abs(new[:, left] - old[:, left] - rw) <= w_err + 2.0 ** -23 * (old[:, left] + rw)).all()
