"""The largest launches of the cached steps: on the host, nothing is enqueued."""
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.test_abi_cached import EUNSUP, prefix

LIMIT = (1 << 24) - 8   # (s, h): work-groups of 256 threads in a multiple of 8, fewer than 2^32 threads


@pytest.mark.parametrize("H", [LIMIT + 1, LIMIT + 7])
def test_prefix_past_the_largest_launch(H):
    assert prefix(pa.library(), S=1, H=H, plen=1, pcap=1, cap=1, k=1) == EUNSUP
    with pytest.raises(pa.PiAttnError):
        pa.pi_attn_decode_workspace(torch.bfloat16, 1, H, 64, 1, 1, 1)


def test_up_to_it():
    assert pa.pi_attn_decode_workspace(torch.bfloat16, 1, LIMIT, 64, 1, 1, 1) == LIMIT * 66
    assert pa.pi_attn_decode_workspace(torch.bfloat16, 1, LIMIT + 7, 64, 0, 1, 1) == 0   # no prefix
