"""Refusals of the quantised-cache and shared-prefix calls, and their workspace's
size: on the host, nothing is enqueued."""
import ctypes

import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import E4M3, quantise

EINVAL, EUNSUP = -1, -2


@pytest.fixture(scope="module")
def lib():
    return pa.library()


def vp(x):
    return None if x is None else ctypes.c_void_p(x)


def store(lib, **kw):
    a = dict(dtype=1, S=2, H=3, D=64, n=10, cap=20, k=16, v=16, sb=3 * 640, sh=640, sn=64, start=None, count=None, kc=16,
             vc=16, ke=1, ve=1, stream=None)
    a.update(kw)
    return lib.pi_attn_cache_store(a["dtype"], a["S"], a["H"], a["D"], a["n"], a["cap"], vp(a["k"]), vp(a["v"]), a["sb"],
                                   a["sh"], a["sn"], vp(a["start"]), vp(a["count"]), vp(a["kc"]), vp(a["vc"]),
                                   vp(a["ke"]), vp(a["ve"]), vp(a["stream"]))


def load(lib, **kw):
    a = dict(dtype=1, S=2, H=3, D=64, n=10, cap=20, k=16, v=16, sb=3 * 640, sh=640, sn=64, start=None, count=None, kc=16,
             vc=16, ke=1, ve=1, stream=None)
    a.update(kw)
    return lib.pi_attn_cache_load(a["dtype"], a["S"], a["H"], a["D"], a["n"], a["cap"], vp(a["kc"]), vp(a["vc"]),
                                  vp(a["ke"]), vp(a["ve"]), vp(a["start"]), vp(a["count"]), vp(a["k"]), vp(a["v"]),
                                  a["sb"], a["sh"], a["sn"], vp(a["stream"]))


ROWS = [(dict(dtype=2), EUNSUP), (dict(D=96), EUNSUP), (dict(S=-1), EINVAL), (dict(H=-1), EINVAL), (dict(n=-1), EINVAL),
        (dict(cap=0), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(kc=None), EINVAL),
        (dict(vc=None), EINVAL), (dict(ke=None), EINVAL), (dict(ve=None), EINVAL), (dict(k=8), EINVAL),
        (dict(v=24), EINVAL), (dict(kc=8), EINVAL), (dict(vc=20), EINVAL), (dict(sn=68), EINVAL), (dict(sh=-640), EINVAL),
        (dict(sb=4), EINVAL), (dict(dtype=0, sn=66), EINVAL), (dict(start=2), EINVAL), (dict(count=6), EINVAL),
        (dict(S=1 << 12, H=1 << 10, n=1 << 9), EINVAL), (dict(S=1 << 16, H=1 << 15, n=0), EINVAL)]


@pytest.mark.parametrize("call", [store, load])
@pytest.mark.parametrize("kw,code", ROWS)
def test_rows_reject(lib, call, kw, code):
    assert call(lib, **kw) == code


@pytest.mark.parametrize("kw", [dict(sn=56), dict(sn=0), dict(sh=0), dict(sb=8)])
def test_load_rejects_rows_that_meet(lib, kw):
    assert load(lib, **kw) == EINVAL


@pytest.mark.parametrize("call", [store, load])
@pytest.mark.parametrize("kw", [dict(S=0), dict(H=0), dict(n=0), dict(n=0, k=None, kc=None, ke=None)])
def test_rows_empty_is_noop(lib, call, kw):
    assert call(lib, **kw) == 0


# A prefix and windows that need a workspace.
BASE = dict(dtype=1, S=2, H=3, D=64, plen=20000, pcap=20000, cap=20, k=30000, pi=0, li=16, lo=None, q=16, kn=16, vn=16, kp=16,
            vp=16, kpe=1, vpe=1, kc=16, vc=16, ke=1, ve=1, gate=16, gss=0, gsh=1, scale=0.125, clamp=0.0, out=16, lse=None,
            work=16, stream=None)


def step(lib, a):
    return (vp(a["li"]), vp(a["lo"]), vp(a["q"]), vp(a["kn"]), vp(a["vn"]))


def e4m3(lib, **kw):
    a = dict(BASE, k=9000, cap=9001, **{x: y for x, y in kw.items() if x not in ("k", "cap")})
    a.update(kw)
    return lib.pi_attn_decode_step_e4m3(a["dtype"], a["S"], a["H"], a["D"], a["cap"], a["k"], a["pi"], *step(lib, a),
                                        vp(a["kc"]), vp(a["vc"]), vp(a["ke"]), vp(a["ve"]), vp(a["gate"]), a["gss"],
                                        a["gsh"], a["scale"], a["clamp"], vp(a["out"]), vp(a["lse"]), vp(a["work"]),
                                        vp(a["stream"]))


def prefix(lib, **kw):
    a = dict(BASE, **kw)
    return lib.pi_attn_decode_step_prefix(a["dtype"], a["S"], a["H"], a["D"], a["plen"], a["pcap"], a["cap"], a["k"],
                                          a["pi"], *step(lib, a), vp(a["kp"]), vp(a["vp"]), vp(a["kpe"]), vp(a["vpe"]),
                                          vp(a["kc"]), vp(a["vc"]), vp(a["ke"]), vp(a["ve"]), vp(a["gate"]), a["gss"],
                                          a["gsh"], a["scale"], a["clamp"], vp(a["out"]), vp(a["lse"]), vp(a["work"]),
                                          vp(a["stream"]))


BOTH = [(dict(dtype=2), EUNSUP), (dict(D=32), EUNSUP), (dict(S=-1), EINVAL), (dict(H=-2), EINVAL), (dict(cap=0), EINVAL),
        (dict(k=-1), EINVAL), (dict(pi=-1), EINVAL), (dict(li=None), EINVAL), (dict(q=None), EINVAL), (dict(kn=None), EINVAL),
        (dict(vn=None), EINVAL), (dict(kc=None), EINVAL), (dict(vc=None), EINVAL), (dict(gate=None), EINVAL),
        (dict(out=None), EINVAL), (dict(li=18), EINVAL), (dict(lo=16), EINVAL), (dict(lo=20), EINVAL), (dict(q=8), EINVAL),
        (dict(kc=8), EINVAL), (dict(out=8), EINVAL), (dict(gate=18), EINVAL), (dict(gsh=-1), EINVAL), (dict(lse=18), EINVAL),
        (dict(scale=0.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(clamp=float("nan")), EINVAL),
        (dict(ve=None), EINVAL), (dict(work=None), EINVAL), (dict(work=24), EINVAL),
        (dict(S=1 << 12, H=1 << 12), EUNSUP), (dict(cap=(1 << 31) - 1), EUNSUP)]


@pytest.mark.parametrize("call", [e4m3, prefix])
@pytest.mark.parametrize("kw,code", BOTH)
def test_steps_reject(lib, call, kw, code):
    assert call(lib, **kw) == code


@pytest.mark.parametrize("call", [e4m3, prefix])
@pytest.mark.parametrize("kw", [dict(S=0), dict(H=0), dict(S=0, li=None, q=None, kc=None, ke=None, ve=None, work=None)])
def test_steps_empty_is_noop(lib, call, kw):
    assert call(lib, **kw) == 0


def test_e4m3_needs_bytes(lib):
    assert e4m3(lib, ke=None, ve=None) == EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(plen=-1), EINVAL), (dict(pcap=19999), EINVAL), (dict(kp=None), EINVAL), (dict(vp=None), EINVAL),
    (dict(kp=24), EINVAL), (dict(kpe=None), EINVAL), (dict(vpe=None), EINVAL), (dict(ke=None, ve=None), EINVAL),
    (dict(ke=None, ve=None, kpe=None), EINVAL), (dict(plen=(1 << 31) - 100, pcap=(1 << 31) - 100), EUNSUP),
])
def test_prefix_rejects(lib, kw, code):
    assert prefix(lib, **kw) == code


def test_workspace_size(lib):
    need = pa.pi_attn_decode_workspace
    bf = torch.bfloat16
    assert need(bf, 2, 3, 64, 0, 100, 50) == 0 and need(bf, 0, 3, 64, 100000, 100, 50000) == 0
    assert need(bf, 2, 3, 64, 100000, 100, 0) == 0   # no window rows in the prefix
    assert need(bf, 2, 3, 64, 200, 100, 300) == 0    # few of them: no parts
    for dtype in (bf, torch.float32):
        for D in (64, 128):
            for S, H, plen, cap, k in ((4, 8, 5000, 10, 6000), (200, 32, 70000, 10, 80000), (1, 2, 0, 9000, 9000), (1, 1, 3000, 5, 4000),
                                       (1, 1, 2 ** 30, 2 ** 30 - 5000, 2 ** 31 - 1), (4000, 4000, 64, 9, 64)):
                n = need(dtype, S, H, D, plen, cap, k)
                assert n > 0 and n % (S * H * (D + 2)) == 0
                # a part is at least a tile of rows, or 64 KB of own ones, and they are few
                assert n // (S * H * (D + 2)) <= (min(k, plen) + 63) // 64 + 8 * min(k, cap) * D // 65536
                assert n // (S * H * (D + 2)) <= 1024
    for bad in ((2, 3, 96, 0, 10, 5), (-1, 3, 64, 0, 10, 5), (2, 3, 64, -1, 10, 5), (2, 3, 64, 0, 0, 5), (2, 3, 64, 0, 9, -1),
                (1 << 12, 1 << 12, 64, 0, 9, 9), (1, 1, 64, 1 << 30, 1 << 30, 4)):
        with pytest.raises(pa.PiAttnError):
            need(bf, *bad)
    with pytest.raises(TypeError):
        need(torch.float16, 1, 1, 64, 0, 10, 5)


@pytest.mark.parametrize("at", range(6))
def test_workspace_size_beyond_32_bits(lib, at):
    """Sizes that the C call would take modulo 2^32 (2^32 + 4 for a window of 4)."""
    sizes = [2, 3, 64, 100, 10, 5]
    sizes[at] += 1 << 32
    with pytest.raises(ValueError, match="32 bits"):
        pa.pi_attn_decode_workspace(torch.bfloat16, *sizes)


def test_binding_refuses_cpu_tensors(lib):
    kc = torch.zeros(1, 1, 8, 64).to(E4M3)
    e = torch.zeros(1, 1, 8, dtype=torch.uint8)
    x, y, g = torch.zeros(1, 1, 8, 64), torch.zeros(1, 1, 64), torch.zeros(1)
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(RuntimeError, match="GPU"):
        pa.pi_attn_cache_store(x, x, kc, kc, e, e)
    with pytest.raises(RuntimeError, match="GPU"):
        pa.pi_attn_cache_load(kc, kc, e, e, 3)
    with pytest.raises(RuntimeError, match="GPU"):
        pa.pi_attn_decode_step_e4m3(n, y, y, y, kc, kc, e, e, g, 4, 0)
    with pytest.raises(RuntimeError, match="GPU"):
        pa.pi_attn_decode_step_prefix(n, y, y, y, x[0], x[0], x, x, g, 4, 0)


def test_the_definition_itself():
    """The tests' own quantisation: every code is a value of the type, none is nearer, and no smaller scale holds the row."""
    x = torch.randn(50, 64, generator=torch.Generator().manual_seed(1), dtype=torch.float64) * 3
    codes, byte = quantise(x)
    grid = torch.arange(256, dtype=torch.uint8).view(E4M3).double()
    grid = torch.unique(grid[torch.isfinite(grid)])
    y = torch.ldexp(x, 127 - torch.tensor(byte.astype("int32"))[:, None])
    assert float(y.abs().max()) <= 448 and bool((y.abs().amax(1) > 224).all())
    d = (y[..., None] - grid).abs()
    assert torch.equal((torch.tensor(codes)[..., None] - y[..., None]).abs()[..., 0], d.amin(-1))
