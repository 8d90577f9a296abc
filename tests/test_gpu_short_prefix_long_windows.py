"""A short prefix before long windows of own rows, few (s, h): the windows are split
over work-groups as without a prefix."""
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.test_gpu_decode_cached import Problem

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("plen", [1, 20, 200])
@pytest.mark.parametrize("k,pi,clamp", [(8000, 0, 0.0), (4200, 4300, 3.0)])   # over all rows; from the own rows or the prefix
def test_against_the_definition(device, dtype, quant, D, plen, k, pi, clamp):
    cap = 7000
    lens = [0, 1, 4100, 4200 - plen, 6999, cap, -1, 4000]
    Problem(dtype, quant, 8, 1, D, plen, cap, k, pi, lens, clamp).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_same_bits_as_one_cache(device, dtype, quant, D):
    """The same ranges of the same rows, whichever table they lie in."""
    S, H, plen, cap = 8, 8, 150, 9000
    p = Problem(dtype, quant, S, H, D, plen, cap, plen + cap, 0, [0, 700, 8999, 5000, 4321, 64, 2, 8000])
    one = [torch.cat([a.view(torch.uint8)[None].expand(S, *a.view(torch.uint8).shape), b.view(torch.uint8)], 2).view(b.dtype)
           for a, b in zip(p.shared, p.own)]
    exp = [torch.cat([a[None].expand(S, H, plen), b], 2) for a, b in zip(p.shared_exp, p.own_exp)] if quant else None
    out = p.run()
    lse = torch.empty_like(p.lse)
    if quant:
        want = pa.pi_attn_decode_step_e4m3(p.lens + plen, p.q, p.kn, p.vn, *one, *exp, p.gate, p.k, 0, lse=lse)
    else:
        none = torch.empty((H, 0, D), dtype=dtype, device="cuda")
        want = pa.pi_attn_decode_step_prefix(p.lens + plen, p.q, p.kn, p.vn, none, none, *one, p.gate, p.k, 0, lse=lse)
    assert torch.equal(out, want) and torch.equal(p.lse, lse)
