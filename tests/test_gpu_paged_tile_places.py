"""The new row and the partner at every place of a tile of the paged step, and rows that are not there at every place but
theirs: what the pages hold at those places is NaN, and none of it reaches the result."""
import pytest
import torch

from tests.paged_ref import Cache
from tests.test_gpu_decode_paged import new_rows, run_with_nan

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def spoil(cache, e, rows):
    for x in (cache.k, cache.v):
        if cache.k_exp is None:
            x[e, :, rows] = float("nan")
        else:
            x.view(torch.uint8)[e, :, rows] = 0x7f
    for x in (cache.k_exp, cache.v_exp):
        if x is not None:
            x[e, :, rows] = 255


@pytest.mark.parametrize("dtype,quantised", [(BF, False), (BF, True), (F, True), (F, False)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gone", [False, True])
@pytest.mark.parametrize("partner", [False, True])
def test_every_place(device, dtype, quantised, D, gone, partner):
    """Windows of 0 to 70 rows, pages of one row: the row behind the window's last is the new one, the next the partner."""
    for n in range(71):
        t, kw = (n + 7, n) if partner else (n, 70)
        cache = Cache(1, 1, D, 1, t + 1, dtype, quantised, 1)
        q, k, v, gate = new_rows(1, 3, 1, D, dtype, 2)
        if gone:
            for j in range(t - n, t):
                if j % 3 != 0:
                    cache.table[0, j] = -1
        # the pool's row 0, which rows that are not there read, is no row of the sequence's window
        cache.table[cache.table == 0] = -1
        if cache.entry(0, t) < 0:
            cache.table[0, t] = next(e for e in range(1, t + 3) if e not in cache.table.tolist()[0])
        named = set(cache.table.tolist()[0]) - {cache.entry(0, t)}
        for e in set(range(cache.k.shape[0])) - named:         # what the new row's place held among them
            spoil(cache, e, slice(None))
        out, _ = run_with_nan(cache, [t], q, k, v, gate, kw, kw + 1 if partner else 0, 0.0)
        assert torch.isfinite(out).all(), n
