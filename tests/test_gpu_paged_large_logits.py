"""Logits of 2^37 and more, of either sign, where half a unit in the last place is thousands: the row of a paged step
with the largest one still has all of the weight, be it a row of the window, the partner or the new row."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import E4M3, f64, quantise
from tests.paged_ref import Cache

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,quantised", [(BF, False), (BF, True), (F, True), (F, False)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S,rows,kw,pi", [(5, 200, 150, 170), (2, 3000, 2500, 2600)])   # whole windows; split ones
@pytest.mark.parametrize("top", ["window", "partner", "new"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("clamp", [0.0, 1e38])
def test_dominating_row(device, dtype, quantised, D, S, rows, kw, pi, top, sign, clamp):
    Hk, G, page = 2, 3, 16
    cache = Cache(S, Hk, D, page, -(-rows // page), dtype, quantised, 1)
    assert (pa.pi_attn_paged_workspace(dtype, S, Hk * G, Hk, D, page, cache.max_pages, kw) > 0) == (rows > 1000)
    g = torch.Generator().manual_seed(7)
    lens = [rows - 1 - 7 * s for s in range(S)]
    way = torch.where(torch.rand(Hk, D, generator=g) < 0.5, -1.0, 1.0)
    q = (way[:, None] * (1 + torch.rand(S, Hk, G, 1, generator=g)) * 2.0 ** 16).to(dtype)
    # keys along the queries: one of 2^18, the others below 2^17; or all against them, one of 2^18, the others from 2^19 on
    large = sign * 2.0 ** 18

    def keys(*shape):
        x = torch.rand(*shape, generator=g)
        return (sign * x * 2.0 ** 17 if sign > 0 else -(1 + x) * 2.0 ** 19)[..., None]

    stored = keys(cache.k.shape[0], Hk, page) * way[:, None]
    k_new = keys(S, Hk) * way
    v_new = torch.randn(S, Hk, D, generator=g).to(dtype)
    table = cache.table.cpu()
    for s, t in enumerate(lens):
        j = {"window": t - kw // 2 - s, "partner": t - pi, "new": t}[top]
        if j == t:
            k_new[s] = large * way
        else:
            stored[table[s, j // page], :, j % page] = large * way
    if quantised:
        c, e = quantise(stored)
        cache.k.copy_(torch.from_numpy(c).float().to(E4M3))
        cache.k_exp.copy_(torch.from_numpy(e))
    else:
        cache.k.copy_(stored)
    lse = torch.empty(S, Hk * G, device="cuda")
    out = pa.pi_attn_decode_step_paged(torch.tensor(lens, dtype=torch.int32, device="cuda"), q.view(S, Hk * G, D).cuda(),
                                       k_new.to(dtype).cuda(), v_new.cuda(), cache.k, cache.v, cache.table,
                                       torch.zeros(Hk * G, device="cuda"), kw, pi, **cache.args(), logit_clamp=clamp, lse=lse)
    _, vals = cache.values()
    out = f64(out).reshape(S, Hk, G, D)
    # the weights: two bf16 terms (2^-15), or three and fp32; the division (2^-22); the output's rounding
    rel = 2.0 ** -8 + 2.0 ** -15 + 2.0 ** -22 if dtype == BF else 2.0 ** -22
    for s, t in enumerate(lens):
        j = {"window": t - kw // 2 - s, "partner": t - pi, "new": t}[top]
        want = vals[cache.entry(s, j), :, j % page][:, None]
        assert np.all(np.abs(out[s] - want) <= rel * np.abs(want)), (s, j)
    # products of D terms (the queries exact), and a few roundings
    want = np.abs(f64(q)).sum(-1).reshape(S, Hk * G) * large / np.sqrt(D)
    assert np.all(np.abs(f64(lse) - want) <= (D + 16) * 2.0 ** -24 * np.abs(want))
