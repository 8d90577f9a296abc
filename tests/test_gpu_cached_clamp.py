"""Logit clamp and keys that are not numbers: the logit stays NaN, and with it the
outputs of the sequences that attend the row, wherever the row lies."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import E4M3
from tests.test_gpu_decode_cached import Problem

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def spoil(rows, at, quant):
    """One element of row `at` of every head of rows [H, n, D] is not a number."""
    if quant:
        rows.view(torch.uint8)[:, at, 11] = 0xff
    else:
        rows[:, at, 11] = float("nan")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("S,D,plen,k,pi", [
    (9, 64, 0, 60, 80), (9, 128, 0, 60, 80),               # own rows alone
    (9, 64, 300, 200, 260), (9, 128, 300, 200, 260),       # a prefix that every sequence reads
    (9, 128, 1700, 1500, 1650), (40, 128, 1700, 1500, 1650), (70, 64, 2900, 2700, 2800)])   # one in chunks
def test_nan_keys(device, dtype, quant, S, D, plen, k, pi):
    cap = 150
    lens = [(i * 29) % cap for i in range(S)]
    p = Problem(dtype, quant, S, 2, D, plen, cap, k, pi, lens, clamp=4.0)
    if plen:   # in the windows of the shorter sequences; the partner of one
        spoil(p.shared[0], plen - k + 40, quant)
        spoil(p.shared[0], plen + lens[3] - pi, quant)
    spoil(p.own[0][1], lens[1] - 1, quant)                 # the last row of a window
    spoil(p.own[0][2], max(lens[2] - k, 0), quant)         # the first
    if plen == 0:
        spoil(p.own[0][4], lens[4] - pi, quant)            # a partner
    p.kn[5, 0, 3] = float("nan")                           # a new row of one head
    want = p.expected()
    hit = np.isnan(want.lse)
    assert hit[1:3].all() and hit[5, 0] and (plen > 0 or hit[4].all()) and not hit.all()
    want.check(p.run(), p.lse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
def test_new_rows_that_are_not_finite(device, dtype, what):
    """Stored as NaN in a quantised cache, and attended so."""
    p = Problem(dtype, True, 3, 2, 64, 0, 50, 20, 0, [5, 40, 0], clamp=4.0)
    p.kn[1, 1, 7] = what
    want = p.expected()
    out = p.run()
    want.check(out, p.lse)
    assert bool(torch.isnan(out[1, 1]).all()) and not bool(torch.isnan(out[0]).any())
    assert p.own[0].view(torch.uint8).view(E4M3)[1, 1, 40].float().isnan().sum() == 1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("k", [3, 60, 300])
def test_plain_step(device, dtype, D, k):
    """pi_attn_decode_step, which the others extend: the same."""
    cap, pi = k + 90, k + 20
    lens = [0, k, k + 30, k + 60, 2, k + 89]
    p = Problem(dtype, False, 6, 2, D, 0, cap, k, pi, lens, clamp=4.0)
    spoil(p.own[0][1], k - 1, False)
    spoil(p.own[0][2], 30, False)
    spoil(p.own[0][3], 60 - 20, False)   # a partner
    p.kn[4, 1, 5] = float("nan")
    want = p.expected()
    assert np.array_equal(np.isnan(want.lse).any(1), [False, True, True, True, True, False])
    lse = torch.empty(6, 2, device="cuda")
    want.check(pa.pi_attn_decode_step(p.lens, p.q, p.kn, p.vn, *p.own, p.gate, k, pi, logit_clamp=4.0, lse=lse), lse)
