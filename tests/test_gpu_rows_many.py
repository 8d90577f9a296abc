"""Rotations and paged stores of more threads than a launch takes (2^32), against small calls."""
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.paged_ref import Cache, frequencies

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def test_rotate(device):
    """2^28 positions of one head, float32 to bf16: rows that overlap in memory, so that the result alone is large."""
    N, D = (1 << 28) + 99, 128
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("a tensor of 69 GB")
    base = torch.randn(4 * N + D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    q = base.as_strided((1, 1, N, D), (0, 0, 4, 1))
    freq = frequencies(D // 2).cuda()
    got, _ = pa.pi_attn_rotate(q, None, None, freq, dtype=BF)
    border = 1 << 27   # of a launch: 2^23 work-groups of 16 rows
    for lo in (0, border - 50, 12345678, 2 * border - 50, N - 100):
        pos = torch.arange(lo, lo + 100, dtype=torch.int32, device="cuda")
        want, _ = pa.pi_attn_rotate(q[:, :, lo:lo + 100].contiguous(), None, pos, freq, dtype=BF)
        assert torch.equal(got[:, :, lo:lo + 100], want), lo
    # nothing is left out: no row of the result is all zeros
    for part in got[0, 0].split(1 << 24):
        assert part.view(torch.int32).ne(0).any(-1).all()
    del got, part
    torch.cuda.empty_cache()


def test_rotate_heads(device):
    """2^28 heads of one position."""
    H, D = (1 << 28) + 5, 64
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("a tensor of 34 GB")
    base = torch.randn(8 * H + D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=BF)
    q = base.as_strided((1, H, 1, D), (0, 8, 0, 1))
    freq, pos = frequencies(D // 2).cuda(), torch.tensor([1234], dtype=torch.int32, device="cuda")
    got, _ = pa.pi_attn_rotate(q, None, pos, freq)
    border = 1 << 27   # 2^23 work-groups of 16 heads
    for lo in (0, border - 50, 2 * border - 100, H - 100):
        want, _ = pa.pi_attn_rotate(q[:, lo:lo + 100].contiguous(), None, pos, freq)
        assert torch.equal(got[:, lo:lo + 100], want), lo
    for part in got[0, :, 0].split(1 << 24):
        assert part.view(torch.int32).ne(0).any(-1).all()
    del got, part
    torch.cuda.empty_cache()


@pytest.mark.parametrize("quantised", [False, True])
def test_store(device, quantised):
    """2^28 rows given, the last ones in the table's reach."""
    n, D, page, held = (1 << 28) + 99, 128, 16, 200
    base = torch.randn(4 * n + D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    k, v = (base.as_strided((1, 1, n, D), (0, 0, 4, 1), at) for at in (0, 4))
    freq = frequencies(D // 2).cuda()
    for first in (0, (1 << 27) - 90, (1 << 28) - 90, n - held):   # row of k and v that becomes position 0
        cache, want = (Cache(1, 1, D, page, -(-held // page), F, quantised, 2) for _ in range(2))
        pa.pi_attn_paged_store(k, v, cache.k, cache.v, cache.table, torch.tensor([-first], dtype=torch.int32, device="cuda"),
                               torch.tensor([min(n, first + held)], dtype=torch.int32, device="cuda"), **cache.args(), freq=freq)
        few = [x[:, :, first:first + held].contiguous() for x in (k, v)]
        pa.pi_attn_paged_store(*few, want.k, want.v, want.table, **want.args(), freq=freq)
        for a, b in zip(cache.tensors(), want.tensors()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), first
