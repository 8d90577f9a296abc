"""Infinities in a paged step: in a query, where a clamp makes its logits finite; in a cached row, whose key head alone they
reach."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import f64
from tests.paged_ref import HALF, Cache, frequencies

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
INF = float("inf")
TYPES = [(BF, False), (BF, True), (F, True), (F, False)]
GATE_EPS = 1e-4


def problem(dtype, quantised, D, n, seed=3):
    S, Hk, G = 2, 2, 3
    cache = Cache(S, Hk, D, 16, -(-n // 16), dtype, quantised, seed)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn(S, Hk * G, D, generator=g).to(dtype).cuda()
    k, v = (torch.randn(S, Hk, D, generator=g).to(dtype).cuda() for _ in range(2))
    gate = (torch.rand(Hk * G, generator=g) * 2 - 1).cuda()
    return cache, q, k, v, gate, torch.tensor([n - 1, n - 20], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,quantised", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,kw,pi", [(150, 100, 130), (3000, 2500, 2600)])
@pytest.mark.parametrize("value", [INF, -INF, 3.4e38])
@pytest.mark.parametrize("turns", [False, True])
def test_query_under_a_clamp(device, dtype, quantised, D, n, kw, pi, value, turns):
    """An element of a query that is infinite, or past bfloat16's largest: every logit is the clamp, with the sign of the
    key's element.  (The element is of a pair that is not turned.)"""
    cache, q, k, v, gate, lens = problem(dtype, quantised, D, n)
    if value == 3.4e38 and dtype == BF:
        value = torch.finfo(BF).max
    at, clamp = D // 2 - 3, 3.0
    # no zeros there, for which an infinity has no product
    k[..., at] = torch.where(k[..., at].abs() < 0.5, 0.5, k[..., at])
    y = cache.k.float()[..., at]
    raw = torch.uint8 if quantised else dtype
    cache.k.view(raw)[..., at] = torch.where(y.abs() < 0.25, 0.25, y).to(cache.k.dtype).view(raw)
    q[:, 1::2, at] = value
    lse = torch.empty(q.shape[:2], device="cuda")
    out = pa.pi_attn_decode_step_paged(lens, q, k, v, cache.k, cache.v, cache.table, gate, kw, pi, **cache.args(), logit_clamp=clamp,
                                       freq=frequencies(D // 4).cuda() if turns else None, lse=lse)
    keys, vals = cache.values()
    for s, t in enumerate(lens.tolist()):
        rows = list(range(max(0, t - kw), t + 1)) + ([t - pi] if t >= pi else [])
        kk, vv = (np.stack([x[cache.entry(s, j), :, j % 16] for j in rows], 1) for x in (keys, vals))
        assert (kk[..., at] != 0).all()
        for h in range(1, q.shape[1], 2):
            d = np.sign(kk[h // 3][:, at]) * np.sign(value) * clamp
            p = np.exp(d - d.max())
            want = p @ vv[h // 3] / p.sum()
            # exponents of up to 2 * 3 * log2 e (two roundings), the exponential, sums of n; weights as two bf16 terms
            delta = 2.0 ** -24 * (16 * (clamp + 8) + len(rows)) + (2.0 ** -16 if dtype == BF else 0.0)
            tol = 2 * delta * (p @ np.abs(vv[h // 3])) / p.sum()
            tol = tol + HALF[dtype] * (np.abs(want) + tol)
            worst = (np.abs(f64(out[s, h]) - want) - tol).max()
            assert worst <= 0, (s, h, worst)
            top = d.max() + np.log(p.sum())
            assert abs(float(lse[s, h]) - top) <= delta + 8 * 2.0 ** -24 * abs(top)


@pytest.mark.parametrize("dtype,quantised", [(BF, False), (F, False)])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("n,kw", [(150, 100), (3000, 2500)])
def test_cached_row(device, dtype, quantised, which, n, kw):
    """A row with an infinity: its key head's queries are not finite (in the element concerned, for a value); the others' are as
    without it."""
    cache, q, k, v, gate, lens = problem(dtype, quantised, 64, n)
    q[:, 3:, 5] = q[:, 3:, 5].abs() + 0.25   # a logit of +inf, or a weight above 0
    args = lambda: (lens, q, k, v, cache.k, cache.v, cache.table, gate, kw, 0)   # noqa: E731
    want = pa.pi_attn_decode_step_paged(*args())
    for s, t in enumerate(lens.tolist()):
        getattr(cache, which)[cache.entry(s, t - 9), 1, (t - 9) % 16, 5] = INF
    out = pa.pi_attn_decode_step_paged(*args())
    assert torch.equal(out[:, :3], want[:, :3])
    assert not torch.isfinite(out[:, 3:, 5]).any()
    if which == "v":
        rest = [i for i in range(64) if i != 5]
        assert torch.equal(out[:, 3:, rest], want[:, 3:, rest])
