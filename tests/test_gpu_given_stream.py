"""Calls on a given stream: what they allocate comes from that stream's pool, since
memory that the current stream let go may still be in use there."""
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.test_gpu_decode_cached import Problem

pytestmark = pytest.mark.gpu


def pool_of(t):
    """The stream whose pool a tensor's memory belongs to."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]


def given_stream():
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert side.cuda_stream != torch.cuda.current_stream().cuda_stream
    return side


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("plen", [0, 50, 3000])
def test_cached_steps(device, quant, plen):
    mk = lambda: Problem(torch.bfloat16, quant, 3, 2, 64, plen, 40, plen + 30, 0, [1, 2, 33])
    a, b = mk(), mk()
    want = a.run()
    side = given_stream()
    got = b.run(stream=side)
    side.synchronize()
    assert pool_of(got) == side.cuda_stream
    assert torch.equal(got, want) and torch.equal(a.lse, b.lse) and torch.equal(a.len_out, b.len_out)


@pytest.mark.parametrize("given", ["nothing", "k", "v"])
def test_load(device, given):
    p = Problem(torch.bfloat16, True, 3, 2, 64, 0, 40, 30, 0, [1, 2, 33])
    want = pa.pi_attn_cache_load(*p.own, *p.own_exp, 25)
    side = given_stream()
    mine = {} if given == "nothing" else {given: torch.empty_like(want[0])}
    got = pa.pi_attn_cache_load(*p.own, *p.own_exp, 25, stream=side, **mine)
    side.synchronize()
    for x, y, name in zip(got, want, "kv"):
        assert x is mine[name] if name in mine else pool_of(x) == side.cuda_stream
        assert torch.equal(x.nan_to_num(9), y.nan_to_num(9))
