"""Results of a rotation and of a paged load in every order of sequences, heads and positions, as slices of larger tensors."""
import itertools

import pytest
import torch

import paper_2511_10696_amd as pa
from tests.paged_ref import Cache, frequencies

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def laid_out(shape, order, dtype, extra):
    """[., ., ., D] with its first three dimensions in `order` in memory, cut from a tensor with `extra` more of each."""
    x = torch.full([shape[i] + extra for i in order] + [shape[3]], 9.0, dtype=dtype, device="cuda")
    x = x.permute(*(order.index(i) for i in range(3)), 3)
    return x, x[extra:, extra:, extra:]


@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
@pytest.mark.parametrize("shape", [(2, 3, 10, 64), (1, 3, 10, 128), (2, 1, 5, 64), (3, 4, 1, 128)])
def test_rotate(device, shape, order, extra):
    q, k = (torch.randn(shape, generator=torch.Generator().manual_seed(i)).cuda() for i in (1, 2))
    freq = frequencies(shape[3] // 2).cuda()
    want = pa.pi_attn_rotate(q, k, None, freq, dtype=BF)
    (qa, qo), (ka, ko) = (laid_out(shape, order, BF, extra) for _ in range(2))
    pa.pi_attn_rotate(q, k, None, freq, dtype=BF, q_out=qo, k_out=ko)
    for whole, part, w in ((qa, qo, want[0]), (ka, ko, want[1])):
        assert torch.equal(part, w)
        assert int((whole != 9.0).sum()) == int((w != 9.0).sum())   # nothing around it


@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
def test_load(device, order, extra):
    cache = Cache(2, 3, 64, 4, 3, F, False, 1)
    want = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, 10)
    (ka, k), (va, v) = (laid_out((2, 3, 10, 64), order, F, extra) for _ in range(2))
    pa.pi_attn_paged_load(cache.k, cache.v, cache.table, 10, k=k, v=v)
    for whole, part, w in ((ka, k, want[0]), (va, v, want[1])):
        assert torch.equal(part, w)
        assert int((whole != 9.0).sum()) == int((w != 9.0).sum())
