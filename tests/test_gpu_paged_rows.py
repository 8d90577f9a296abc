"""Rows into and out of paged caches: bit by bit where nothing is computed, within derived bounds where keys
are turned."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import E4M3, f64, quantise
from tests.paged_ref import Cache, frequencies, rounded_tol, turned

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def rows(S, Hk, n, D, dtype, layout, seed):
    g = torch.Generator().manual_seed(seed)
    out = []
    for _ in range(2):
        x = (torch.randn(S, n, Hk, D, generator=g) * (0.01 + 3 * torch.rand(S, n, Hk, 1, generator=g))).to(dtype).cuda()
        out.append(x.transpose(1, 2) if layout == "snhd" else x.transpose(1, 2).contiguous())
    return out


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def places(cache, start, count, n):
    """(s, i, page, row) of every row that has a place."""
    for s in range(cache.S):
        for i in range(min(n, count[s])):
            e = cache.entry(s, start[s] + i)
            if e >= 0:
                yield s, i, e, (start[s] + i) % cache.page


CASES = [
    # S, Hk, D, page, max_pages, n, dtype, quantised, layout, start, count
    (1, 1, 64, 1, 3, 1, F, False, "shnd", [0], [1]),
    (3, 4, 64, 5, 9, 33, F, False, "shnd", [0, 3, 40], [33, 20, 33]),
    (3, 2, 128, 16, 4, 50, BF, False, "snhd", [-7, 14, 60], [50, 0, -3]),
    (2, 3, 128, 64, 2, 128, BF, False, "shnd", [0, 1], [128, 128]),
    (5, 1, 64, 7, 6, 11, BF, True, "snhd", [0, 5, 30, 41, 42], [11, 11, 11, 11, 1]),
    (2, 5, 128, 32, 3, 70, F, True, "shnd", [2, 26], [70, 69]),
    (40, 8, 128, 16, 2, 1, BF, False, "shnd", list(range(40)), [1] * 40),
    (2, 8, 64, 16, 40, 600, BF, True, "snhd", [17, 0], [600, 599]),
    (1, 17, 64, 3, 500, 1400, F, False, "snhd", [99], [1400]),
]


def spoil_table(cache):
    """Entries that name no page, in the last sequence."""
    if cache.max_pages > 2:
        cache.table[-1, 1] = -1
        cache.table[-1, 2] = cache.k.shape[0]
    if cache.max_pages > 5:
        cache.table[-1, 5] = -2 ** 31
        cache.table[-1, 4] = 2 ** 31 - 1


@pytest.mark.parametrize("spoiled", [False, True])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}x{c[5]}x{c[2]}-{c[3]}-{'e4m3' if c[7] else 'plain'}" for c in CASES])
def test_store_and_load(device, case, spoiled):
    S, Hk, D, page, max_pages, n, dt, quantised, layout, start, count = case
    cache = Cache(S, Hk, D, page, max_pages, dt, quantised, 1)
    if spoiled:
        spoil_table(cache)
    k, v = rows(S, Hk, n, D, dt, layout, 2)
    want = [t.clone() for t in cache.tensors()]
    for s, i, e, r in places(cache, start, count, n):
        if quantised:
            for x, codes, byte in ((k, 0, 2), (v, 1, 3)):
                c, b = quantise(x[s, :, i])
                want[codes].view(torch.uint8)[e, :, r] = torch.from_numpy(c).float().to(E4M3).view(torch.uint8).cuda()
                want[byte][e, :, r] = torch.from_numpy(b).cuda()
        else:
            want[0][e, :, r], want[1][e, :, r] = k[s, :, i], v[s, :, i]
    pa.pi_attn_paged_store(k, v, cache.k, cache.v, cache.table, i32(*start), i32(*count), **cache.args())
    for got, w in zip(cache.tensors(), want):
        assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))
    # back in sequence, zeros where there is none
    out = [torch.full((S, n, Hk, D), 7.0, dtype=dt, device="cuda").transpose(1, 2) for _ in range(2)]
    ko, vo = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, n, i32(*start), i32(*count), **cache.args(), k=out[0], v=out[1])
    keys, vals = cache.values()
    wk, wv = np.zeros((S, Hk, n, D)), np.zeros((S, Hk, n, D))
    for s, i, e, r in places(cache, start, count, n):
        wk[s, :, i], wv[s, :, i] = keys[e, :, r], vals[e, :, r]
    assert np.array_equal(f64(ko), wk) and np.array_equal(f64(vo), wv)
    assert ko.data_ptr() == out[0].data_ptr()
    k2, v2 = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, n, i32(*start), i32(*count), **cache.args(), dtype=dt)
    assert k2.is_contiguous() and torch.equal(k2, ko) and torch.equal(v2, vo)


TURNED = [
    # S, Hk, D, page, n, dtype, quantised, sections, with positions of its own
    (2, 3, 64, 5, 33, F, False, (32,), False),
    (3, 8, 128, 16, 50, BF, False, (16, 24, 24), True),
    (2, 2, 128, 64, 100, BF, False, (20,), True),
    (2, 4, 64, 16, 40, BF, True, (32,), False),
    (2, 5, 128, 7, 40, F, True, (10, 11, 12), True),
]


@pytest.mark.parametrize("case", TURNED, ids=[f"{c[1]}x{c[2]}-{len(c[7])}-{'e4m3' if c[6] else 'plain'}" for c in TURNED])
def test_store_turns_the_keys(device, case):
    S, Hk, D, page, n, dt, quantised, sections, own = case
    max_pages = n // page + 4
    cache = Cache(S, Hk, D, page, max_pages, dt, quantised, 1)
    k, v = rows(S, Hk, n, D, dt, "snhd", 2)
    start, count, freq = [3 * s + 1 for s in range(S)], [n] * S, frequencies(sum(sections)).cuda()
    if own:
        pos = torch.randint(-5, 4000, (len(sections), S, n), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
        at = np.asarray(pos.cpu())
    else:
        pos = None
        at = np.array([[[start[s] + i for i in range(n)] for s in range(S)]] * len(sections))
    untouched = [t.clone() for t in cache.tensors()]
    pa.pi_attn_paged_store(k, v, cache.k, cache.v, cache.table, i32(*start), None, **cache.args(), freq=freq, pos=pos,
                           sections=sections)
    y, tol = turned(f64(k), at[:, :, None], freq, sections)
    keys, vals = cache.values()
    mine = set()
    for s, i, e, r in places(cache, start, count, n):
        mine.add((e, r))
        if quantised:
            # half a step of e4m3: 2^-4 of the value, or 2^-10 of the row's scale
            scale = np.ldexp(1.0, cache.k_exp[e, :, r].cpu().numpy().astype(int) - 127)[:, None]
            bound = tol[s, :, i] + np.maximum(2.0 ** -4 * np.abs(y[s, :, i]) + tol[s, :, i], 2.0 ** -10 * scale)
            # the least scale that holds the row, but for the rounding
            top, off = np.abs(y[s, :, i]).max(-1), tol[s, :, i].max(-1)
            assert (top - off <= 448 * scale[:, 0]).all() and (top + off > 224 * scale[:, 0]).all()
            c, b = quantise(v[s, :, i])
            assert np.array_equal(c * np.ldexp(1.0, b.astype(int) - 127)[:, None], vals[e, :, r])
        else:
            bound = rounded_tol(y[s, :, i], tol[s, :, i], dt)
            assert np.array_equal(f64(v[s, :, i]), vals[e, :, r])
        worst = (np.abs(keys[e, :, r] - y[s, :, i]) - bound).max()
        assert worst <= 0, worst
    for t, before in zip(cache.tensors(), untouched):
        for e in range(t.shape[0]):
            for r in range(page):
                if (e, r) not in mine:
                    assert torch.equal(t[e, :, r].view(torch.uint8), before[e, :, r].view(torch.uint8))


def test_store_turns_as_rotate_does(device):
    """bf16 pages hold what pi_attn_rotate gives, bit by bit."""
    S, Hk, n, D = 3, 4, 100, 128
    cache = Cache(S, Hk, D, 16, 8, BF, False, 1)
    k, v = rows(S, Hk, n, D, BF, "snhd", 2)
    freq, sections = frequencies(60).cuda(), (20, 20, 20)
    pos = torch.randint(0, 4000, (3, S, n), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    pa.pi_attn_paged_store(k, v, cache.k, cache.v, cache.table, freq=freq, pos=pos, sections=sections)
    kt, _ = pa.pi_attn_rotate(k, None, pos, freq, sections)
    ko, vo = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, n)
    assert torch.equal(ko, kt) and torch.equal(vo, v)


def test_special_values(device):
    """Infinities and NaN in plain pages pass bit by bit; in quantised ones they are NaN and leave the scale to the others."""
    k, v = rows(1, 2, 6, 64, BF, "shnd", 2)
    k[0, 0, 1, 3], k[0, 1, 2, 4], v[0, 0, 3, 5] = float("inf"), float("nan"), float("-inf")
    k[0, 0, 4] = 0.0
    cache = Cache(1, 2, 64, 4, 2, BF, False, 1)
    pa.pi_attn_paged_store(k, v, cache.k, cache.v, cache.table)
    ko, vo = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, 6)
    assert torch.equal(ko.view(torch.int16), k.view(torch.int16)) and torch.equal(vo.view(torch.int16), v.view(torch.int16))
    cache = Cache(1, 2, 64, 4, 2, BF, True, 1)
    pa.pi_attn_paged_store(k, v, cache.k, cache.v, cache.table, **cache.args())
    c, b = quantise(k[0])
    keys, _ = cache.values()
    for i in range(6):
        e, r = cache.entry(0, i), i % 4
        want = c[:, i] * np.ldexp(1.0, b[:, i].astype(int) - 127)[:, None]
        assert np.array_equal(keys[e, :, r], want, equal_nan=True)


def test_pages_shared_and_appended_in_two_calls(device):
    """Two sequences read one page; a second call goes on behind the first, over a page's end."""
    cache = Cache(2, 2, 64, 8, 3, BF, False, 1)
    cache.table[1, 0] = cache.table[0, 0]
    k, v = rows(1, 2, 8, 64, BF, "shnd", 2)
    pa.pi_attn_paged_store(k, v, cache.k, cache.v, cache.table[:1])
    k2, v2 = rows(2, 2, 5, 64, BF, "shnd", 3)
    pa.pi_attn_paged_store(k2, v2, cache.k, cache.v, cache.table, start=i32(8, 8))
    k3, v3 = rows(2, 2, 5, 64, BF, "shnd", 4)
    pa.pi_attn_paged_store(k3, v3, cache.k, cache.v, cache.table, start=i32(13, 13))
    ko, vo = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, 18)
    assert torch.equal(ko, torch.cat([k.expand(2, -1, -1, -1), k2, k3], 2))
    assert torch.equal(vo, torch.cat([v.expand(2, -1, -1, -1), v2, v3], 2))


@pytest.mark.parametrize("quantised", [False, True])
def test_large_pools(device, quantised):
    """Pages past 2^31 elements of the pool."""
    D, page, Hk = 128, 64, 8
    n_pages = (1 << 31) // (page * Hk * D) + 9
    dt = E4M3 if quantised else BF
    pages = [torch.zeros(n_pages, Hk, page, D, dtype=torch.uint8 if quantised else BF, device="cuda") for _ in range(2)]
    kp, vp = (p.view(E4M3) if quantised else p for p in pages)
    ke, ve = (torch.full((n_pages, Hk, page), 127, dtype=torch.uint8, device="cuda") if quantised else None for _ in range(2))
    table = i32(n_pages - 1, 0, n_pages - 2)[None].contiguous()
    k, v = rows(1, Hk, 3 * page, D, BF, "shnd", 2)
    pa.pi_attn_paged_store(k, v, kp, vp, table, k_exp=ke, v_exp=ve)
    ko, vo = pa.pi_attn_paged_load(kp, vp, table, 3 * page, k_exp=ke, v_exp=ve, dtype=BF)
    if quantised:
        for x, y in ((k, ko), (v, vo)):
            c, b = quantise(x)
            assert np.array_equal(f64(y), c * np.ldexp(1.0, b.astype(int) - 127)[..., None])
    else:
        assert torch.equal(ko, k) and torch.equal(vo, v)


def test_rows_past_32_bits(device):
    """Rows more than 2^31 elements into k and v: as a call of those rows alone."""
    n, D, page = (1 << 31) // 64 + 500, 64, 256
    k = torch.zeros(1, 1, n, D, dtype=BF, device="cuda")
    v = torch.zeros(1, 1, n, D, dtype=BF, device="cuda")
    k[:, :, -90:], v[:, :, -90:] = rows(1, 1, 90, D, BF, "shnd", 2)
    count = n // page + 1
    pages = [torch.full((count, 1, page, D), 3.0, dtype=BF, device="cuda") for _ in range(2)]
    table = torch.arange(count, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    freq = frequencies(32).cuda()
    pa.pi_attn_paged_store(k, v, *pages, table, freq=freq)
    kt, _ = pa.pi_attn_rotate(k[:, :, -90:].contiguous(), None, torch.arange(n - 90, n, dtype=torch.int32, device="cuda"), freq)
    del k
    ko, vo = pa.pi_attn_paged_load(*pages, table, n)
    assert torch.equal(ko[:, :, -90:], kt) and torch.equal(vo, v) and not ko[:, :, :-90].any()
    assert (pages[0].view(-1, D)[n % page:page] == 3.0).all()   # behind the last row, in the last page


def test_on_a_given_stream_and_python_path(device, monkeypatch):
    S, Hk, n, D = 2, 3, 40, 64
    k, v = rows(S, Hk, n, D, BF, "snhd", 2)
    freq = frequencies(32).cuda()
    got = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(pa, "_native", pa._PythonOnly)
        for given in (False, True):
            cache = Cache(S, Hk, D, 16, 4, BF, True, 1)
            st = torch.cuda.Stream() if given else None
            if st:
                st.wait_stream(torch.cuda.current_stream())
            pa.pi_attn_paged_store(k, v, cache.k, cache.v, cache.table, i32(1, 2), i32(40, 7), **cache.args(), freq=freq, stream=st)
            out = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, 50, i32(0, 1), **cache.args(), dtype=F, stream=st)
            torch.cuda.synchronize()
            got.append([t.view(torch.uint8).cpu() for t in (*cache.tensors(), *out)])
    for g in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], g))


def test_refusals(device):
    cache = Cache(2, 3, 64, 16, 4, BF, False, 1)
    q = Cache(2, 3, 64, 16, 4, BF, True, 1)
    k, v = rows(2, 3, 10, 64, BF, "shnd", 2)
    store, load = pa.pi_attn_paged_store, pa.pi_attn_paged_load
    args = (cache.k, cache.v, cache.table)
    for bad in (lambda: store(k[:, :2], v[:, :2], *args), lambda: store(k[:1], v[:1], *args), lambda: store(k, v[:, :, :9], *args),
                lambda: store(k, v.transpose(1, 2).contiguous().transpose(1, 2), *args), lambda: store(k, v, cache.k[::2], cache.v[::2], cache.table),
                lambda: store(k, v, cache.k, cache.v, cache.table.long()), lambda: store(k, v, cache.k, cache.v, cache.table[0]),
                lambda: store(k, v, cache.k, cache.v, cache.table.t().contiguous().t()),
                lambda: store(k, v, *args, start=i32(1)), lambda: store(k, v, *args, count=i32(1, 2).long()),
                lambda: store(k, v, *args, k_exp=q.k_exp, v_exp=q.v_exp), lambda: store(k, v, q.k, q.v, q.table),
                lambda: store(k, v, q.k, q.v, q.table, k_exp=q.k_exp, v_exp=q.v_exp[:1]),
                lambda: store(k, v, *args, pos=i32(1)), lambda: store(k, v, *args, freq=frequencies(40).cuda()),
                lambda: load(*args, -1), lambda: load(*args, 1 << 31),
                lambda: load(*args, 9, k=k), lambda: load(*args, 9, k=k, v=v), lambda: load(*args, 10, start=i32(1))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: store(k.float(), v.float(), *args), lambda: load(*args, 10, dtype=F), lambda: load(*args, 10, k=k.float(), v=v.float())):
        with pytest.raises((TypeError, ValueError)):
            bad()
    assert load(*args, 0)[0].shape == (2, 3, 0, 64)
