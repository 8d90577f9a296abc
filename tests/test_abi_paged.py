"""Refusals of the rotary positions and of the paged caches' calls, and their workspace's size: on the
host, nothing is enqueued."""
import ctypes

import pytest
import torch

import paper_2511_10696_amd as pa

EINVAL, EUNSUP = -1, -2


@pytest.fixture(scope="module")
def lib():
    return pa.library()


def vp(x):
    return None if x is None else ctypes.c_void_p(x)


def rotate(lib, **kw):
    a = dict(dtype=1, to=1, B=2, H=3, Hk=1, N=10, D=64, back=0, q=16, qs=(1920, 640, 64), k=32, ks=(640, 640, 64), pos=4,
             ps=(0, 10, 1), freq=4, n=(32, 0, 0), qo=48, oqs=(1920, 640, 64), ko=64, oks=(640, 640, 64))
    a.update(kw)
    return lib.pi_attn_rotate(a["dtype"], a["to"], a["B"], a["H"], a["Hk"], a["N"], a["D"], a["back"], vp(a["q"]), *a["qs"],
                              vp(a["k"]), *a["ks"], vp(a["pos"]), *a["ps"], vp(a["freq"]), *a["n"], vp(a["qo"]), *a["oqs"],
                              vp(a["ko"]), *a["oks"], None)


ROTATE = [(dict(dtype=2), EUNSUP), (dict(to=-1), EUNSUP), (dict(D=96), EUNSUP), (dict(B=-1), EINVAL), (dict(H=-1), EINVAL),
          (dict(Hk=-1), EINVAL), (dict(N=-1), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(qo=None), EINVAL),
          (dict(ko=None), EINVAL), (dict(q=8), EINVAL), (dict(k=40), EINVAL), (dict(qo=24), EINVAL), (dict(ko=8), EINVAL),
          (dict(qs=(1920, 640, 65)), EINVAL), (dict(ks=(-640, 640, 64)), EINVAL), (dict(oqs=(1920, 640, 56)), EINVAL),
          (dict(oqs=(1920, 0, 64)), EINVAL), (dict(oks=(0, 640, 64)), EINVAL), (dict(pos=2), EINVAL), (dict(ps=(0, -1, 1)), EINVAL),
          (dict(freq=2), EINVAL), (dict(n=(20, 10, 3)), EINVAL), (dict(n=(20, -1, 3)), EINVAL), (dict(n=(33, 0, 0)), EINVAL),
          (dict(n=(2 ** 31 - 1, 2 ** 31 - 1, 2)), EINVAL),
          (dict(qo=16, oqs=(1920, 64, 192)), EINVAL), (dict(qo=16, to=0), EINVAL), (dict(ko=32, to=0), EINVAL),
          (dict(B=1 << 12, N=1 << 18, H=1, Hk=1), EINVAL), (dict(B=1 << 16, N=1 << 16), EINVAL)]


@pytest.mark.parametrize("kw,code", ROTATE)
def test_rotate_rejects(lib, kw, code):
    assert rotate(lib, **kw) == code


@pytest.mark.parametrize("kw", [dict(B=0), dict(N=0), dict(H=0, Hk=0), dict(B=0, q=None, k=None, qo=None, ko=None)])
def test_rotate_of_nothing(lib, kw):
    assert rotate(lib, **kw) == 0


def rows(lib, store, **kw):
    a = dict(dtype=1, S=2, Hk=3, D=64, n=10, pages=9, page=4, max=5, k=16, v=16, st=(1920, 640, 64), start=None, count=None,
             table=4, kp=16, vp=16, ke=None, ve=None, freq=4, nn=(32, 0, 0), pos=None, ps=(0, 0, 0))
    a.update(kw)
    head = (a["dtype"], a["S"], a["Hk"], a["D"], a["n"], a["pages"], a["page"], a["max"])
    if store:
        return lib.pi_attn_paged_store(*head, vp(a["k"]), vp(a["v"]), *a["st"], vp(a["start"]), vp(a["count"]), vp(a["table"]),
                                       vp(a["kp"]), vp(a["vp"]), vp(a["ke"]), vp(a["ve"]), vp(a["freq"]), *a["nn"], vp(a["pos"]),
                                       *a["ps"], None)
    return lib.pi_attn_paged_load(*head, vp(a["kp"]), vp(a["vp"]), vp(a["ke"]), vp(a["ve"]), vp(a["start"]), vp(a["count"]),
                                  vp(a["table"]), vp(a["k"]), vp(a["v"]), *a["st"], None)


ROWS = [(dict(dtype=2), EUNSUP), (dict(D=32), EUNSUP), (dict(S=-1), EINVAL), (dict(Hk=-1), EINVAL), (dict(n=-1), EINVAL),
        (dict(pages=0), EINVAL), (dict(page=0), EINVAL), (dict(max=0), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
        (dict(table=None), EINVAL), (dict(table=2), EINVAL), (dict(kp=None), EINVAL), (dict(vp=None), EINVAL), (dict(kp=8), EINVAL),
        (dict(vp=4), EINVAL), (dict(k=8), EINVAL), (dict(v=24), EINVAL), (dict(ke=1), EINVAL), (dict(ve=1), EINVAL),
        (dict(st=(1920, 640, 68)), EINVAL), (dict(st=(1920, -640, 64)), EINVAL), (dict(start=2), EINVAL), (dict(count=6), EINVAL),
        (dict(page=1 << 16, max=1 << 15), EUNSUP), (dict(page=2 ** 31 - 4096, max=1), EUNSUP),
        (dict(S=1 << 12, Hk=1 << 10, n=1 << 9), EINVAL), (dict(S=1 << 16, Hk=1 << 15, n=0), EINVAL)]


@pytest.mark.parametrize("store", [True, False])
@pytest.mark.parametrize("kw,code", ROWS)
def test_rows_reject(lib, store, kw, code):
    assert rows(lib, store, **kw) == code


@pytest.mark.parametrize("kw", [dict(nn=(20, 13, 0)), dict(nn=(-1, 2, 2)), dict(freq=6), dict(pos=2), dict(pos=4, ps=(0, -1, 1))])
def test_store_rejects_rotations(lib, kw):
    assert rows(lib, True, **kw) == EINVAL


@pytest.mark.parametrize("st", [(1920, 640, 56), (1920, 640, 0), (1920, 0, 64), (0, 640, 64)])
def test_load_rejects_rows_that_meet(lib, st):
    assert rows(lib, False, st=st) == EINVAL


@pytest.mark.parametrize("store", [True, False])
@pytest.mark.parametrize("kw", [dict(S=0), dict(Hk=0), dict(n=0), dict(n=0, k=None, table=None, kp=None)])
def test_rows_of_nothing(lib, store, kw):
    assert rows(lib, store, **kw) == 0


def step(lib, **kw):
    a = dict(dtype=1, S=2, H=6, Hk=3, D=64, pages=9, page=4, max=5, k=3, pi=7, len_in=4, len_out=64, q=16, kn=16, vn=16, table=4,
             kp=16, vp=16, ke=None, ve=None, freq=4, n=(32, 0, 0), pos=None, ps=(0, 0), gate=4, gs=(0, 1), scale=0.125, clamp=0.0,
             out=16, lse=None, work=None)
    a.update(kw)
    return lib.pi_attn_decode_step_paged(
        a["dtype"], a["S"], a["H"], a["Hk"], a["D"], a["pages"], a["page"], a["max"], a["k"], a["pi"], vp(a["len_in"]),
        vp(a["len_out"]), vp(a["q"]), vp(a["kn"]), vp(a["vn"]), vp(a["table"]), vp(a["kp"]), vp(a["vp"]), vp(a["ke"]), vp(a["ve"]),
        vp(a["freq"]), *a["n"], vp(a["pos"]), *a["ps"], vp(a["gate"]), *a["gs"], a["scale"], a["clamp"], vp(a["out"]), vp(a["lse"]),
        vp(a["work"]), None)


STEP = [(dict(dtype=3), EUNSUP), (dict(D=80), EUNSUP), (dict(S=-1), EINVAL), (dict(H=-3), EINVAL), (dict(Hk=-1), EINVAL),
        (dict(Hk=4), EINVAL), (dict(Hk=0), EINVAL), (dict(H=0), EINVAL), (dict(k=-1), EINVAL), (dict(pi=-1), EINVAL),
        (dict(pages=0), EINVAL), (dict(page=0), EINVAL), (dict(max=0), EINVAL), (dict(scale=0.0), EINVAL),
        (dict(scale=float("inf")), EINVAL), (dict(clamp=float("nan")), EINVAL), (dict(len_in=None), EINVAL), (dict(len_in=2), EINVAL),
        (dict(len_out=8), EINVAL), (dict(len_out=66), EINVAL), (dict(q=None), EINVAL), (dict(kn=None), EINVAL), (dict(vn=None), EINVAL),
        (dict(table=None), EINVAL), (dict(kp=None), EINVAL), (dict(vp=None), EINVAL), (dict(gate=None), EINVAL), (dict(out=None), EINVAL),
        (dict(q=8), EINVAL), (dict(kn=8), EINVAL), (dict(vn=8), EINVAL), (dict(out=8), EINVAL), (dict(kp=8), EINVAL),
        (dict(gate=2), EINVAL), (dict(gs=(-1, 1)), EINVAL), (dict(lse=2), EINVAL), (dict(ke=1), EINVAL), (dict(ve=1), EINVAL),
        (dict(n=(30, 3, 0)), EINVAL), (dict(pos=2), EINVAL), (dict(ps=(-1, 0), pos=4), EINVAL),
        (dict(page=1 << 16, max=1 << 15), EUNSUP), (dict(S=1 << 14, H=1 << 10, Hk=1), EUNSUP),
        (dict(pages=1 << 20, page=1 << 11), EUNSUP), (dict(pages=1 << 20, page=1 << 10, Hk=6), EUNSUP),
        (dict(page=1024, max=64, k=1 << 20), EINVAL), (dict(page=1024, max=64, k=1 << 20, work=8), EINVAL)]


@pytest.mark.parametrize("kw,code", STEP)
def test_step_rejects(lib, kw, code):
    assert step(lib, **kw) == code


@pytest.mark.parametrize("kw", [dict(S=0), dict(H=0, Hk=0), dict(S=0, len_in=None, table=None, q=None)])
def test_step_of_nothing(lib, kw):
    assert step(lib, **kw) == 0


def test_workspace():
    ws = pa.pi_attn_paged_workspace
    bf = torch.bfloat16
    assert ws(bf, 64, 32, 32, 128, 16, 64, 100) == 0                   # short windows are not split
    assert ws(bf, 1, 8, 8, 128, 16, 10000, 1 << 20) % (8 * 130) == 0 < ws(bf, 1, 8, 8, 128, 16, 10000, 1 << 20)
    assert ws(bf, 0, 8, 8, 128, 16, 10000, 1 << 20) == 0
    # the cache's reach bounds the window
    assert ws(bf, 1, 8, 8, 128, 16, 10000, 1 << 30) == ws(bf, 1, 8, 8, 128, 16, 10000, 160000)
    # fewer than 2^32 threads of 256 a part
    assert ws(bf, 1, 1 << 20, 1, 64, 16, 10000, 1 << 20) <= (1 << 23) * 66
    for bad in ((bf, -1, 8, 8, 128, 16, 10, 5), (bf, 1, 8, 3, 128, 16, 10, 5), (bf, 1, 8, 8, 96, 16, 10, 5),
                (bf, 1, 8, 8, 128, 0, 10, 5), (bf, 1, 8, 8, 128, 16, 0, 5), (bf, 1, 8, 8, 128, 16, 10, -1)):
        with pytest.raises(pa.PiAttnError):
            ws(*bad)
    with pytest.raises(ValueError):
        ws(bf, 1, 8, 8, 128, 16, 10, 1 << 31)


def test_cpu_tensors_are_refused():
    q = torch.zeros(1, 1, 4, 64)
    with pytest.raises(RuntimeError):
        pa.pi_attn_rotate(q, q, None, torch.ones(32))
    pages, table = torch.zeros(2, 1, 4, 64), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(RuntimeError):
        pa.pi_attn_paged_store(q, q, pages, pages, table)
    with pytest.raises(RuntimeError):
        pa.pi_attn_paged_load(pages, pages, table, 3)
    with pytest.raises(RuntimeError):
        pa.pi_attn_decode_step_paged(torch.zeros(1, dtype=torch.int32), q[0], q[0], q[0], pages, pages, table, torch.zeros(1), 3, 0)
