"""The launches that large batches and large transfers take: the paged step with more than 256 work-groups and no split, with more
query heads of a key head than a work-group has, with rows that are not kept in the caches; rotations, stores and loads that
leave the caches alone."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.paged_ref import Cache, frequencies, turned, rounded_tol
from tests.cached_ref import f64
from tests.test_gpu_decode_paged import new_rows, run

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
TYPES = [(BF, False), (BF, True), (F, True), (F, False)]
NAMES = ["bf16", "e4m3-bf16", "e4m3-f32", "f32"]


@pytest.mark.parametrize("dtype,quantised", TYPES, ids=NAMES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S,kw,pi,clamp", [(33, 40, 100, 0.0), (33, 500, 600, 20.0), (32, 500, 600, 0.0)])
def test_full_batch(device, dtype, quantised, D, S, kw, pi, clamp):
    """Windows that are not split: more than 256 (s, key head), kept in the caches or (12 MB and more) not; 256 of them."""
    Hk, page, reach = 8, 16, 640
    cache = Cache(S, Hk, D, page, reach // page, dtype, quantised, 1)
    lens = [(s * reach + reach - 1) // S for s in range(S)]
    lens[5] = reach   # past the table
    cache.table[3, ::2] = -1
    assert pa.pi_attn_paged_workspace(dtype, S, 2 * Hk, Hk, D, page, reach // page, kw) == 0
    run(cache, lens, *new_rows(S, 2 * Hk, Hk, D, dtype, 2), kw, pi, clamp, freq=frequencies(D // 2).cuda())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [9, 17])
@pytest.mark.parametrize("n,kw", [(100, 60), (1500, 1400)])
def test_float32_with_many_queries(device, D, G, n, kw):
    """More than eight query heads of a key head, whole and split windows."""
    cache = Cache(2, 2, D, 16, -(-n // 16), F, False, 1)
    assert (pa.pi_attn_paged_workspace(F, 2, 2 * G, 2, D, 16, cache.max_pages, kw) > 0) == (n > 1000)
    run(cache, [n - 1, n // 2], *new_rows(2, 2 * G, 2, D, F, 2), kw, kw + 7, freq=frequencies(D // 2).cuda())


@pytest.mark.parametrize("dtype,quantised", TYPES, ids=NAMES)
@pytest.mark.parametrize("D", [64, 128])
def test_long_windows_not_kept(device, dtype, quantised, D):
    """Split windows of 12 MB and more."""
    S, Hk, page = 4, 8, 64
    n = 12 * 1024 * 1024 // (2 * S * Hk * D * (1 if quantised else 4 if dtype == F else 2)) + 200
    n = max(n, 1300)
    cache = Cache(S, Hk, D, page, -(-n // page), dtype, quantised, 1)
    assert pa.pi_attn_paged_workspace(dtype, S, 2 * Hk, Hk, D, page, cache.max_pages, n) > 0
    run(cache, [n - 1, n - 700, 5, n // 2], *new_rows(S, 2 * Hk, Hk, D, dtype, 2), n, 0, freq=frequencies(D // 2).cuda())


def heads(B, H, N, D, dtype, layout, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(B, N, H, D, generator=g, device="cuda").to(dtype)
    return x.transpose(1, 2) if layout == "bnhd" else x.transpose(1, 2).contiguous()


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("dtype,to,D", [(F, F, 64), (F, BF, 128), (BF, BF, 128), (BF, F, 128)])
def test_large_rotations(device, dtype, to, D, layout, back):
    """192 MB and more, read and written: as calls of a few positions, bit by bit; the same in place."""
    B, H, Hk, step = 2, 7, 2, 1777
    size = D * sum(4 if x == F else 2 for x in (dtype, to))
    N = (192 << 20) // (size * B * (H + Hk)) + 500
    q, k = heads(B, H, N, D, dtype, layout, 1), heads(B, Hk, N, D, dtype, layout, 2)
    sections, freq = (D // 8, D // 8, D // 8), frequencies(3 * D // 8).cuda()
    pos = torch.randint(-9, 5000, (3, B, N), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    fn = pa.pi_attn_rotate_backward if back else pa.pi_attn_rotate
    got = fn(q, k, pos, freq, sections, dtype=to)
    for lo in range(0, N, step):
        part = slice(lo, lo + step)
        want = fn(q[:, :, part], k[:, :, part], pos[:, :, part], freq, sections, dtype=to)
        for a, b in zip(got, want):
            assert torch.equal(a[:, :, part], b), lo
    if dtype == to:
        fn(q, k, pos, freq, sections, None, q, k)
        assert torch.equal(q, got[0]) and torch.equal(k, got[1])


ROTATE = [
    # B, H, Hk, N, D, in, out, sections: q and k as views of a projection's [B][N][H][D] output
    (2, 5, 2, 33, 64, F, F, (32,)),
    (1, 4, 1, 70, 128, F, BF, (64,)),
    (2, 7, 7, 29, 128, BF, BF, (16, 24, 24)),
    (3, 1, 3, 17, 64, BF, F, (5, 4, 3)),
]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("case", ROTATE, ids=[f"{c[1]}+{c[2]}x{c[3]}x{c[4]}" for c in ROTATE])
def test_rotations_of_views(device, case, back):
    B, H, Hk, N, D, dtype, to, sections = case
    q, k = heads(B, H, N, D, dtype, "bnhd", 1), heads(B, Hk, N, D, dtype, "bnhd", 2)
    freq = frequencies(sum(sections)).cuda()
    pos = torch.randint(-9, 5000, (len(sections), B, N), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    fn = pa.pi_attn_rotate_backward if back else pa.pi_attn_rotate
    for x, got in zip((q, k), fn(q, k, pos, freq, sections, dtype=to)):
        y, tol = turned(f64(x), np.asarray(pos.cpu())[:, :, None], freq, sections, back)
        worst = (np.abs(f64(got) - y) - rounded_tol(y, tol, to)).max()
        assert worst <= 0, worst


@pytest.mark.parametrize("layout", ["shnd", "snhd"])
@pytest.mark.parametrize("dtype,quantised,D", [(BF, False, 128), (BF, True, 64), (BF, True, 128), (F, False, 64), (F, False, 128),
                                               (F, True, 128)])
def test_large_stores_and_loads(device, dtype, quantised, D, layout):
    """128 MB and more, read and written: as calls of a few rows, bit by bit."""
    S, Hk, page, step = 2, 5, 48, 999
    row = 2 * D * ((4 if dtype == F else 2) + (1 if quantised else 4 if dtype == F else 2))
    n = (128 << 20) // (S * Hk * row) + 300
    k, v = (heads(S, Hk, n, D, dtype, "bnhd" if layout == "snhd" else "bhnd", x) for x in (1, 2))
    freq = frequencies(D // 2).cuda()
    count = torch.tensor([n, n - 123], dtype=torch.int32, device="cuda")
    caches = [Cache(S, Hk, D, page, -(-n // page), dtype, quantised, 1) for _ in range(2)]
    for c in caches:
        c.table[1, 7] = -1
    got, want = caches
    pa.pi_attn_paged_store(k, v, got.k, got.v, got.table, None, count, **got.args(), freq=freq)
    for lo in range(0, n, step):
        part = slice(lo, lo + step)
        start = torch.full((S,), lo, dtype=torch.int32, device="cuda")
        pa.pi_attn_paged_store(k[:, :, part], v[:, :, part], want.k, want.v, want.table, start, count - lo, **want.args(), freq=freq)
    for a, b in zip(got.tensors(), want.tensors()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    out = [x.transpose(1, 2) if layout == "snhd" else x for x in
           (torch.full((S, n, Hk, D) if layout == "snhd" else (S, Hk, n, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))]
    pa.pi_attn_paged_load(got.k, got.v, got.table, n, None, count, **got.args(), k=out[0], v=out[1])
    for lo in range(0, n, step):
        m = min(step, n - lo)
        start = torch.full((S,), lo, dtype=torch.int32, device="cuda")
        few = pa.pi_attn_paged_load(got.k, got.v, got.table, m, start, count - lo, **got.args(), dtype=dtype)
        for a, b in zip(out, few):
            assert torch.equal(a[:, :, lo:lo + m], b), lo
