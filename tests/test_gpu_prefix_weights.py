"""bf16 steps behind a prefix that is taken in chunks: the weights of its rows enter
the value product as two bf16 terms, so that the output is as near the definition
as where every sequence reads the rows for itself.

Bound: that of cached_ref.Step with no weight rounded, and the rest that two terms
leave.  The first is the weight without its low 16 bits or rounded, which leaves
less than 2^-7 of it; the second is that rest within half a step, 2^-8 of it: 2^-15
of sum(p |v|).  So that one term alone does not pass, rows cancel: each dim has the
values 1 and -1 in one row each, and the queries are small (the bound of the scores
grows with them).
"""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import Step, f64, value_of
from tests.test_gpu_decode_cached import Problem

pytestmark = pytest.mark.gpu


def rows_of(p):
    """Every sequence's rows as stored, and the new one: float64 [H, rows, D]."""
    p.expected()   # p.new
    shared = [value_of(c, e) if p.quant else f64(c) for c, e in zip(p.shared, p.shared_exp)]
    own = [value_of(c, e) if p.quant else f64(c) for c, e in zip(p.own, p.own_exp)]
    return [[np.concatenate([a, b[s][:, :n], c[s][:, None]], 1) for a, b, c in zip(shared, own, p.new)]
            for s, n in enumerate(p.lens_np)]


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [5, 40, 100])   # each shape of work-group: rings of their own, one for two groups, for four
def test_weights(device, quant, D, S):
    plen, k, cap = 2700 if D == 64 else 1400, 2600 if D == 64 else 1300, 40
    p = Problem(torch.bfloat16, quant, S, 2, D, plen, cap, k, 0, [(7 * s) % cap for s in range(S)])
    assert 2 * k * D * (1 if quant else 2) > 300 << 10   # too long to be read by each sequence
    p.q.mul_(0.125)
    for x in (p.shared[1], p.own[1], p.vn):
        x.copy_(torch.zeros_like(x, dtype=torch.float32).to(x.dtype))
    v = torch.zeros(2, plen, D, device="cuda")
    at = torch.arange(D, device="cuda")
    v[:, plen - k + 100 + 3 * at, at], v[:, plen - 1 - 5 * at, at] = 1.0, -1.0
    if quant:
        p.shared_exp[1].fill_(127), p.own_exp[1].fill_(127)
    p.shared[1].copy_(v.to(p.shared[1].dtype))
    rows = rows_of(p)
    want = Step(p.q, p.gate, k, 0, 0.0, rows, torch.bfloat16, 0)
    # sum(p |v|), at most: the definition's own output for the magnitudes
    size = Step(p.q, p.gate, k, 0, 0.0, [[a, np.abs(b)] for a, b in rows], torch.bfloat16, 0).out
    want.out_tol += 2.0 ** -15 * size
    want.check(p.run(), p.lse)


@pytest.mark.parametrize("S", [5, 40, 100])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_infinite_values_stay_infinite(device, S, sign):
    """An infinite value in a row of every window, whatever the row's weight (1, which leaves no rest, among them): an
    infinity of its sign, and nothing else changes."""
    D, plen, cap = 128, 1400, 40
    p = Problem(torch.bfloat16, False, S, 2, D, plen, cap, plen + cap, 0, [(7 * s) % cap for s in range(S)])
    p.q[0] = 0.0   # weights of 1 before they are normalised
    want = p.expected()
    p.shared[1][:, 700, 77] = sign * float("inf")
    out = f64(p.run())
    assert np.all(out[:, :, 77] == sign * np.inf)
    keep = np.arange(D) != 77
    assert np.all(np.abs(out - want.out)[:, :, keep] <= want.out_tol[:, :, keep])
    assert np.all(np.abs(f64(p.lse) - want.lse) <= want.lse_tol)
