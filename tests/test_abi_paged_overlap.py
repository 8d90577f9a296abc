"""Outputs whose rows meet, or that lie on another tensor of the call, are refused on the host by the rotation and the paged
load."""
import pytest

import paper_2511_10696_amd as pa
from tests.test_abi_paged import EINVAL, rotate, rows


@pytest.fixture(scope="module")
def lib():
    return pa.library()


# B = 2, H = 3, Hk = 1, N = 10, D = 64
MEET = [dict(oqs=(1920, 64, 64)),             # heads and positions both a row apart
        dict(oqs=(1920, 320, 64)),            # heads closer than their positions reach
        dict(oqs=(640, 640, 64)),             # sequences on the second head
        dict(oqs=(1280, 640, 64)),            # sequences on the third
        dict(oqs=(128, 1280, 64)),            # sequences two positions apart
        dict(oqs=(1920, 640, 56)), dict(oks=(64, 0, 64)), dict(oks=(320, 0, 64)), dict(oks=(128, 0, 64)),
        dict(H=0, oks=(576, 0, 64)), dict(oqs=(1856, 640, 64))]


@pytest.mark.parametrize("kw", MEET)
def test_rotate_rejects_rows_that_meet(lib, kw):
    assert rotate(lib, **kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(qo=48, ko=48), dict(qo=32), dict(ko=16)])
def test_rotate_rejects_an_output_on_another_tensor(lib, kw):
    """k's result on q's, q's result on k, k's result on q."""
    assert rotate(lib, **kw) == EINVAL


@pytest.mark.parametrize("st", [(1920, 64, 64), (1920, 320, 64), (640, 640, 64), (1280, 640, 64), (128, 1280, 64)])
def test_load_rejects_rows_that_meet(lib, st):
    assert rows(lib, False, st=st, k=1 << 20, v=2 << 20) == EINVAL


def test_load_rejects_keys_on_values(lib):
    assert rows(lib, False, k=1 << 20, v=1 << 20) == EINVAL
