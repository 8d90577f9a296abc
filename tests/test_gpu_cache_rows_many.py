"""Rows into and out of quantised caches by the 2^27: more threads than a launch takes."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import E4M3, quantise, value_of

pytestmark = pytest.mark.gpu


def sample(H):
    """Heads of every part of the range, the ends and the border of 2^23 work-groups of eight rows among them."""
    g = np.random.default_rng(1)
    return torch.tensor(np.unique(np.concatenate([[0, 1, H - 2, H - 1], g.integers(0, H, 500),
                                                  (1 << 26) // 63 + np.arange(-9, 9)])), device="cuda")


def test_store(device):
    """Rows of a prompt that begins before the cache's only row: most are dropped.  Heads lie 16 bytes apart in memory."""
    H, n, D = (1 << 27) // 63 + 99, 63, 128
    base = torch.randn(4 * H + n * D + D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    k = base.as_strided((1, H, n, D), (0, 4, D, 1))
    v = base.as_strided((1, H, n, D), (0, 4, D, 1), 4)
    kc, vc = (torch.full((1, H, 1, D), 0x5a, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ke, ve = (torch.full((1, H, 1), 0x5a, dtype=torch.uint8, device="cuda") for _ in range(2))
    pa.pi_attn_cache_store(k, v, kc, vc, ke, ve, torch.tensor([-62], dtype=torch.int32, device="cuda"))
    at = sample(H)
    for codes, byte, x in ((kc, ke, k), (vc, ve, v)):
        want, wb = quantise(x[0, at, 62])
        got = codes.view(torch.uint8)[0, at, 0].cpu().view(E4M3).double().numpy()
        assert np.array_equal(got, want) and np.array_equal(byte[0, at, 0].cpu().numpy(), wb)


def test_load(device):
    H, n, D = (1 << 27) // 63 + 99, 63, 128
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("two tensors of 69 GB")
    g = torch.Generator(device="cuda").manual_seed(2)
    kc, vc = (torch.randint(0, 0x78, (1, H, 1, D), generator=g, dtype=torch.uint8, device="cuda").view(E4M3)
              for _ in range(2))
    ke, ve = (torch.randint(100, 150, (1, H, 1), generator=g, dtype=torch.uint8, device="cuda") for _ in range(2))
    lk, lv = pa.pi_attn_cache_load(kc, vc, ke, ve, n, torch.tensor([-62], dtype=torch.int32, device="cuda"),
                                   dtype=torch.float32)
    at = sample(H)
    for got, codes, byte in ((lk, kc, ke), (lv, vc, ve)):
        want = value_of(codes.view(torch.uint8)[0, at, 0].view(E4M3), byte[0, at, 0])
        assert np.array_equal(got[0, at, 62].double().cpu().numpy(), want)
        assert not got[0, at, :62].any()
    del lk, lv, got
    torch.cuda.empty_cache()
