"""Numbers at the edges of the cache operators' types: infinite keys whose
weight is zero, and many small probabilities beside a large one."""
import math

import numpy as np
import pytest

from cache_ref import attend_ref
from parity import say
from test_gpu_cache_attend import cache_for, make, run

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


@pytest.mark.parametrize("qs,ks,copies", [(1, 4000, 1), (1, 40_000, 512), (3, 9000, 200), (40, 4000, 1), (40, 4000, 512), (130, 2500, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_small_probabilities_beside_a_large_one(qs, ks, copies, dtype, dim):
    """A first token that draws nearly all of the weight, 18.5 to 19.5 above the
    others in natural units (2^-27): together they are what is left of the result,
    as its own values are zero.  f16 holds multiples of 2^-24 below its normal
    range; the products take probabilities of up to 2^14 (single tokens) and 2^7 times
    the running maximum's (chunks), so half of such a step is 2^-39 and 2^-32
    of the largest.  With many sequences (here the same one) the cache is in
    one or two splits."""
    import torch

    say(f"[cache small probabilities] {copies} x {qs} over {ks} x {dim} {dtype}")
    c = make(dtype, 2, 1, dim, 16, qs=(qs,), ks=(ks,), seed=ks)
    g = torch.Generator().manual_seed(1)
    td = c["q"].dtype
    c["q"].zero_()
    c["q"][..., 0] = 1
    k = torch.zeros(ks, 1, dim)
    k[:, 0, 0] = torch.rand(ks, generator=g) - 0.5
    k[0, 0, 0] = 19
    v = torch.rand(ks, 1, dim, generator=g) + 0.5
    v[0] = 0
    c["keys"][0], c["vals"][0] = k.to(td), v.to(td)
    pos = torch.arange(ks)
    page = c["table"][0].cpu()[pos // 16].long()
    for name, x in (("k_pages", c["keys"][0]), ("v_pages", c["vals"][0])):
        c[name][page.cuda(), (pos % 16).cuda()] = x.cuda()
    cache = cache_for(c)
    s = cache.sequences(c["table"].repeat(copies, 1), c["lens"].repeat(copies), torch.arange(copies + 1, dtype=torch.int32).cuda() * qs,
                        max_q=qs, max_k=ks)
    out, lse = cache.attend(s, c["q"].cuda().repeat(copies, 1, 1), c["k_pages"], c["v_pages"], scale=1.0)
    cache.check()
    out, lse = (x.view(copies, *x[:qs].shape) for x in (out, lse))
    assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
    ro, rz, _, _, z_err, _ = attend_ref(c["q"].double().numpy(), c["keys"][0].double().numpy(), c["vals"][0].double().numpy(), ks - qs, 1.0)
    # roundings of probabilities and result, the sums' 32 bits, and steps below f16's normal range (values are at most 1.5)
    lim = 2.1 * {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype] * np.abs(ro) + 2 * z_err[..., None] * np.abs(ro)
    if dtype == "f16":
        lim += 2.0 ** -25 + 1.5 * ks * 2.0 ** (-39 if qs * 2 <= 32 else -32)
    err = np.abs(out[0].double().cpu().numpy() - ro)
    assert (err <= lim).all(), f"off by {err.max()} of {np.abs(ro).max()}, allowed {lim.min()}"
    assert (np.abs(lse[0].double().cpu().numpy() - rz) <= z_err).all()
