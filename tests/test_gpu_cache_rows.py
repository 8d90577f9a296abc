"""Rows into and out of quantised caches: codes, bytes and values against the
definition in 64 bits, bit by bit."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import E4M3, quantise, value_of

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def cache(S, H, cap, D, fill=0x5a):
    """Codes and bytes that hold a pattern."""
    kc, vc = (torch.full((S, H, cap, D), fill, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ke, ve = (torch.full((S, H, cap), fill, dtype=torch.uint8, device="cuda") for _ in range(2))
    return kc, vc, ke, ve


def rows(S, H, n, D, dtype, seed, layout="shnd"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    def one():
        shape = (S, n, H, D) if layout == "snhd" else (S, H, n, D)
        x = torch.randn(shape, generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, shape[:3] + (1,),
                                                                                      generator=g, device="cuda"))
        x = x.to(dtype)
        return x.transpose(1, 2) if layout == "snhd" else x
    return one(), one()


def check_rows(codes, byte, x):
    """A cache's rows [..., D] hold x."""
    want, wb = quantise(x)
    got = codes.cpu().view(torch.uint8).view(E4M3).float().double().numpy()
    assert np.array_equal(got, want, equal_nan=True)
    assert np.array_equal(byte.cpu().numpy(), wb)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["shnd", "snhd"])
@pytest.mark.parametrize("S,H,n", [(1, 1, 1), (3, 5, 1), (2, 3, 37), (5, 7, 500)])   # the last: four instructions a lane
def test_store_and_load(device, dtype, D, layout, S, H, n):
    cap = n + 9
    k, v = rows(S, H, n, D, dtype, 3, layout)
    kc, vc, ke, ve = cache(S, H, cap, D)
    g = np.random.default_rng(5)
    start = g.integers(0, 10, S).astype(np.int32)
    count = g.integers(0, n + 1, S).astype(np.int32)
    count[0] = n
    st, ct = torch.tensor(start, device="cuda"), torch.tensor(count, device="cuda")
    assert pa.pi_attn_cache_store(k, v, kc, vc, ke, ve, st, ct) is None
    for s in range(S):
        a, m = int(start[s]), int(count[s])
        for codes, byte, x in ((kc, ke, k), (vc, ve, v)):
            if m:
                check_rows(codes[s, :, a:a + m], byte[s, :, a:a + m], x[s, :, :m])
            rest = torch.ones(cap, dtype=torch.bool)
            rest[a:a + m] = False
            assert bool((codes.view(torch.uint8)[s][:, rest] == 0x5a).all()) and bool((byte[s][:, rest] == 0x5a).all())
    for out_type in TYPES:
        lk, lv = pa.pi_attn_cache_load(kc, vc, ke, ve, n, st, ct, dtype=out_type)
        assert lk.dtype == lv.dtype == out_type
        for got, codes, byte in ((lk, kc, ke), (lv, vc, ve)):
            for s in range(S):
                a, m = int(start[s]), int(count[s])
                want = torch.tensor(value_of(codes[s, :, a:a + m], byte[s, :, a:a + m])).to(out_type)
                assert torch.equal(got[s, :, :m].cpu(), want)
                assert not got[s, :, m:].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_every_code_and_tie(device, dtype):
    """All finite codes as elements, the halves between them (ties to even) and values just beside the halves, at several
    scales, subnormals and both ends of the exponents among them."""
    codes = torch.arange(256, dtype=torch.uint8).view(E4M3).float()
    codes = torch.unique(codes[torch.isfinite(codes)])
    mid = (codes[1:] + codes[:-1]) / 2
    near = torch.cat([mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -7)])
    x = torch.cat([codes, mid, near])
    x = torch.cat([x, torch.zeros(-len(x) % 63)]).view(-1, 63)
    x = torch.cat([torch.full((len(x), 1), 448.0), x], 1)   # every row's largest is 448: its scale is the power it is given
    big = torch.stack([torch.ldexp(x, torch.tensor(e)) for e in (-126, -125, -60, -1, 0, 1, 60, 118, 119)]).to(dtype)
    assert bool(torch.isfinite(big).all())
    big = big.view(1, 1, -1, 64).cuda()
    kc, vc, ke, ve = cache(1, 1, big.shape[2], 64)
    pa.pi_attn_cache_store(big, -big, kc, vc, ke, ve)
    check_rows(kc, ke, big)
    check_rows(vc, ve, -big)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_scales(device, dtype, D):
    """Rows of one magnitude: each side of 448 * 2^e, zeros, the smallest and the largest numbers."""
    f = torch.finfo(dtype)
    one = torch.tensor([0.0, 448.0, 448 * (1 + f.eps), 1.75, 1.75 * (1 + f.eps), 447.0, 1.0, 2.0 ** -118 * 1.75, 2.0 ** -118,
                        2.0 ** -119, f.tiny, f.tiny * f.eps, f.max, f.max / 2, f.max * 1.75 / 2], dtype=torch.float64)
    x = torch.zeros(1, 1, len(one), D, dtype=dtype)
    x[0, 0, :, D - 3] = one.to(dtype)
    x[0, 0, :, 5] = -one.to(dtype) / 3
    x = x.cuda()
    kc, vc, ke, ve = cache(1, 1, len(one), D)
    pa.pi_attn_cache_store(x, -x, kc, vc, ke, ve)
    check_rows(kc, ke, x)
    check_rows(vc, ve, -x)


@pytest.mark.parametrize("dtype", TYPES)
def test_not_finite(device, dtype):
    """Infinities and NaN become NaN and leave the scale to the other elements; they come back as NaN."""
    k, v = rows(1, 2, 6, 64, dtype, 9)
    k[0, 0, 1, 3], k[0, 0, 2, 63], k[0, 1, 3, 0] = float("inf"), float("-inf"), float("nan")
    k[0, 1, 4] = float("inf")   # none left: the smallest scale
    kc, vc, ke, ve = cache(1, 2, 6, 64)
    pa.pi_attn_cache_store(k, v, kc, vc, ke, ve)
    check_rows(kc, ke, k)
    check_rows(vc, ve, v)
    lk, lv = pa.pi_attn_cache_load(kc, vc, ke, ve, 6)
    assert torch.equal(torch.isnan(lk), ~torch.isfinite(k)) and bool(torch.isfinite(lv).all())


def test_rows_outside_the_cache(device):
    """Places before and behind the cache: dropped on the way in, zeros on the way out; starts near the ends of int32 too."""
    n, cap, D = 8, 10, 64
    start = torch.tensor([-3, 6, -9, 10, 2 ** 31 - 4, -2 ** 31, 1], dtype=torch.int32, device="cuda")
    count = torch.tensor([8, 100, 8, 8, 8, 8, -5], dtype=torch.int32, device="cuda")
    S = len(start)
    k, v = rows(S, 2, n, D, torch.bfloat16, 11)
    kc, vc, ke, ve = cache(S, 2, cap, D)
    pa.pi_attn_cache_store(k, v, kc, vc, ke, ve, start, count)
    raw = kc.view(torch.uint8)
    check_rows(kc[0, :, :5], ke[0, :, :5], k[0, :, 3:])
    check_rows(kc[1, :, 6:], ke[1, :, 6:], k[1, :, :4])
    assert bool((raw[0, :, 5:] == 0x5a).all()) and bool((raw[1, :, :6] == 0x5a).all()) and bool((raw[2:] == 0x5a).all())
    assert bool((ke[2:] == 0x5a).all()) and bool((ve[2:] == 0x5a).all())
    lk, _ = pa.pi_attn_cache_load(kc, vc, ke, ve, n, start, count, dtype=torch.float32)
    assert not lk[0, :, :3].any() and torch.equal(lk[0, :, 3:].cpu().double(), torch.tensor(value_of(kc[0, :, :5], ke[0, :, :5])))
    assert not lk[1, :, 4:].any() and not lk[2:].any()


def test_outputs_given_and_empty(device):
    """Outputs in the projection's layout, their neighbours left alone; calls with nothing to do."""
    S, H, n, D = 2, 3, 20, 64
    k, v = rows(S, H, n, D, torch.float32, 13)
    kc, vc, ke, ve = cache(S, H, n, D)
    pa.pi_attn_cache_store(k, v, kc, vc, ke, ve)
    buf = [torch.full((S, n + 4, H, D), 7.0, device="cuda") for _ in range(2)]
    ok, ov = (b[:, 2:2 + n].transpose(1, 2) for b in buf)
    r = pa.pi_attn_cache_load(kc, vc, ke, ve, n, k=ok, v=ov)
    assert r[0] is ok and r[1] is ov
    want = pa.pi_attn_cache_load(kc, vc, ke, ve, n, dtype=torch.float32)
    assert torch.equal(ok, want[0]) and torch.equal(ov, want[1])
    for b in buf:
        assert bool((b[:, :2] == 7).all()) and bool((b[:, 2 + n:] == 7).all())
    a, b = pa.pi_attn_cache_load(kc, vc, ke, ve, 0)
    assert a.shape == b.shape == (S, H, 0, D)
    before = kc.view(torch.uint8).clone()
    pa.pi_attn_cache_store(k[:, :, :0], v[:, :, :0], kc, vc, ke, ve)
    assert torch.equal(kc.view(torch.uint8), before)


def test_captured(device):
    """Store and load in a graph, replayed on new rows and places."""
    S, H, n, D = 2, 4, 300, 128
    k, v = rows(S, H, n, D, torch.bfloat16, 17)
    kc, vc, ke, ve = cache(S, H, 2 * n, D)
    start = torch.zeros(S, dtype=torch.int32, device="cuda")
    ok, ov = torch.empty_like(k), torch.empty_like(v)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pa.pi_attn_cache_store(k, v, kc, vc, ke, ve, start)
        pa.pi_attn_cache_load(kc, vc, ke, ve, n, start, k=ok, v=ov)
    for i in range(3):
        nk, nv = rows(S, H, n, D, torch.bfloat16, 20 + i)
        k.copy_(nk), v.copy_(nv), start.fill_(i * 100)
        graph.replay()
        torch.cuda.synchronize()
        kc2, vc2, ke2, ve2 = cache(S, H, n, D)
        pa.pi_attn_cache_store(nk, nv, kc2, vc2, ke2, ve2)
        wk, wv = pa.pi_attn_cache_load(kc2, vc2, ke2, ve2, n)
        assert torch.equal(ok, wk) and torch.equal(ov, wv)


def test_past_32_bits(device):
    """A cache of more than 2^32 bytes: the last sequence's rows."""
    S, H, cap, D = 9, 32, 131072, 128
    kc, vc = (torch.zeros((S, H, cap, D), dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ke, ve = (torch.zeros((S, H, cap), dtype=torch.uint8, device="cuda") for _ in range(2))
    k, v = rows(S, H, 3, D, torch.bfloat16, 23)
    start = torch.full((S,), cap - 3, dtype=torch.int32, device="cuda")
    pa.pi_attn_cache_store(k, v, kc, vc, ke, ve, start)
    check_rows(kc[S - 1, :, cap - 3:], ke[S - 1, :, cap - 3:], k[S - 1])
    check_rows(vc[S - 1, :, cap - 3:], ve[S - 1, :, cap - 3:], v[S - 1])
    lk, lv = pa.pi_attn_cache_load(kc, vc, ke, ve, 3, start, dtype=torch.float32)
    assert torch.equal(lv[S - 1].cpu().double(), torch.tensor(value_of(vc[S - 1, :, cap - 3:], ve[S - 1, :, cap - 3:])))
