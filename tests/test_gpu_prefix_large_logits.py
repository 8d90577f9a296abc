"""Logits of 2^37 and more, of either sign, where half a unit in the last place is
thousands: the row with the largest one still has all of the weight, however the
prefix is read."""
import numpy as np
import pytest
import torch

from tests.cached_ref import f64, value_of
from tests.test_gpu_decode_cached import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("S,D", [(5, 64), (5, 128), (40, 64), (40, 128), (70, 128), (140, 64)])
@pytest.mark.parametrize("plen", [200, 3000])   # read by each sequence, in chunks
@pytest.mark.parametrize("sign", [1, -1])
def test_dominating_row(device, dtype, quant, S, D, plen, sign):
    H, cap, row = 2, 30, plen - 77
    p = Problem(dtype, quant, S, H, D, plen, cap, plen + cap, 0, [(7 * s) % cap for s in range(S)])
    g = torch.Generator(device="cuda").manual_seed(7)
    way = torch.where(torch.rand(H, D, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    size = 1 + torch.rand(S, H, 1, generator=g, device="cuda")
    p.q.copy_(way * size * 2.0 ** 16)
    # keys along the queries: one of 2^18, the others below 2^17; or all against them, one of 2^18, the others from 2^19 on
    top = sign * 2.0 ** 18

    def keys(*shape):
        x = torch.rand(shape, generator=g, device="cuda")
        return (sign * x * 2.0 ** 17 if sign > 0 else -(1 + x) * 2.0 ** 19)[..., None] * way[:, None]

    shared, own = keys(H, plen), keys(S, H, cap)
    shared[:, row] = top * way
    p.kn.copy_(keys(S, H, 1)[:, :, 0])
    for table, byte, x in ((p.shared[0], p.shared_exp[0], shared), (p.own[0], p.own_exp[0], own)):
        x = x.to(dtype)
        if quant:
            c, e = Problem.cached(x)
            table.view(torch.uint8).copy_(c.view(torch.uint8))
            byte.copy_(e)
        else:
            table.copy_(x)
    value = value_of(p.shared[1][:, row], p.shared_exp[1][:, row]) if quant else f64(p.shared[1][:, row])
    out = f64(p.run())
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    # the weights: two bf16 terms (2^-15); the division (2^-22)
    assert np.all(np.abs(out - value) <= (half + 2.0 ** -15 + 2.0 ** -22 if dtype == torch.bfloat16 else 2.0 ** -22) * np.abs(value))
    # products of D terms, and a few roundings
    lse = f64(p.q).__abs__().sum(-1) * top / np.sqrt(D)
    assert np.all(np.abs(f64(p.lse) - lse) <= (D + 16) * 2.0 ** -24 * np.abs(lse))
