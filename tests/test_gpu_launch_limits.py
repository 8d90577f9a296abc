"""Calls that would take 2^32 threads or more are refused, not served in part."""
import pytest
import torch

import paper_2511_10696_amd as pa

pytestmark = pytest.mark.gpu


def test_forward_of_many_heads(device):
    """2^24 heads of one row, a work-group of 256 threads each."""
    H, D = (1 << 24) + 8, 64
    x = torch.ones(1, 1, 1, D, dtype=torch.bfloat16, device="cuda").expand(1, H, 1, D)
    gate = torch.zeros(1, device="cuda").expand(H)
    out = torch.zeros(1, H, 1, D, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pa.PiAttnError, match="launch"):
        pa.pi_attn_forward(x, x, x, gate, 40, 0, out=out)
    assert not out.any()
    n = (1 << 24) - 8   # the largest
    out = pa.pi_attn_forward(x[:, :n], x[:, :n], x[:, :n], gate[:n], 40, 0)
    assert bool((out == 1).all())
