"""Rows into and out of quantised caches in large calls: runs of one head's rows,
heads first, accesses past the caches.  Codes, bytes and values of sampled heads
against the definition bit by bit, what lies beside them on the device."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import value_of
from tests.test_gpu_cache_rows import cache, check_rows, rows

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]

# S, H, n, D
RUNS = [(3, 16, 1501, 64), (3, 16, 1501, 128),       # 2^16 rows and more: runs, the last one not whole
        (9, 120, 64, 64), (5, 103, 129, 128),        # runs of short sequences
        (1, 64, 4100, 64), (2, 40, 6600, 128),       # 2^18 rows a sequence: heads first as [S][n][H][D]
        (1, 32, 4200, 128),                          # more than 96 MB in all: stored past the caches
        (64, 32, 50, 128), (300, 8, 30, 64)]         # rows of each sequence too few for a run


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["shnd", "snhd"])
@pytest.mark.parametrize("S,H,n,D", RUNS)
@pytest.mark.parametrize("ragged", [False, True])
def test_store_and_load(device, dtype, layout, S, H, n, D, ragged):
    cap = n + 9
    k, v = rows(S, H, n, D, dtype, S + n, layout)
    kc, vc, ke, ve = cache(S, H, cap, D)
    g = np.random.default_rng(n)
    # rows before and behind the cache among the ragged ones
    start = g.integers(-20, 30, S).astype(np.int32) if ragged else np.zeros(S, np.int32)
    count = g.integers(0, n + 1, S).astype(np.int32) if ragged else np.full(S, n, np.int32)
    if ragged:
        count[0] = n
    at = dict(start=torch.tensor(start, device="cuda"), count=torch.tensor(count, device="cuda")) if ragged else {}
    pa.pi_attn_cache_store(k, v, kc, vc, ke, ve, **at)
    heads = sorted({0, H - 1, *g.integers(0, H, 2).tolist()})
    seqs = sorted({0, S - 1, *g.integers(0, S, 3).tolist()})
    there = torch.zeros(S, cap, dtype=torch.bool, device="cuda")
    for s in range(S):
        there[s, max(int(start[s]), 0):max(int(start[s] + count[s]), 0)] = True
    for codes, byte in ((kc, ke), (vc, ve)):   # everything else as it was
        assert bool((codes.view(torch.uint8) == 0x5a).all(-1).logical_or(there[:, None]).all())
        assert bool((byte == 0x5a).logical_or(there[:, None]).all())
    for s in seqs:
        lo, hi = max(0, -int(start[s])), min(int(count[s]), cap - int(start[s]))   # rows that are stored
        if hi > lo:
            a = int(start[s])
            for codes, byte, x in ((kc, ke, k), (vc, ve, v)):
                check_rows(codes[s, heads, a + lo:a + hi], byte[s, heads, a + lo:a + hi], x[s, heads, lo:hi])
    # read back in the same layout, beside rows that stay
    shape = (S, n + 2, H, D) if layout == "snhd" else (S, H, n + 2, D)
    buf = [torch.full(shape, 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    views = [(b.transpose(1, 2) if layout == "snhd" else b) for b in buf]
    lk, lv = (x[:, :, 1:1 + n] for x in views)
    pa.pi_attn_cache_load(kc, vc, ke, ve, n, k=lk, v=lv, **at)
    for x in views:
        assert bool((x[:, :, 0] == 7).all()) and bool((x[:, :, n + 1] == 7).all())
    i = torch.arange(n, device="cuda")[None]
    place = i + torch.tensor(start, device="cuda")[:, None]
    absent = (place < 0) | (place >= cap) | (i >= torch.tensor(count, device="cuda")[:, None])
    for got, codes, byte in ((lk, kc, ke), (lv, vc, ve)):
        assert not got.masked_fill(~absent[:, None, :, None], 0).any()
        for s in seqs:
            lo, hi = max(0, -int(start[s])), min(int(count[s]), cap - int(start[s]))
            if hi > lo:
                a = int(start[s])
                want = torch.tensor(value_of(codes[s, heads, a + lo:a + hi], byte[s, heads, a + lo:a + hi])).to(dtype)
                assert torch.equal(got[s, heads, lo:hi].cpu(), want)
